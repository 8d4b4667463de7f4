"""Timed cases of attention over sequences of different lengths: packed prompts, their gradient, the paged cache.

  append   new keys and values rotated by their position ids into the slots of a paged cache, the queries rotated beside
  decode   one new token a sequence against its paged cache
  prompt   causal attention of whole prompts, packed end to end (forward)
  train    the same, forward and backward

Inputs are seeded Gaussians rounded once to the storage type.  Head counts and dimensions are those of the models and tests
of this repository (16 or 32 heads of 128, 32 of 100, 64 in the tests; 8 key/value heads for 32).
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BASE = 10000.0


def _packed(name, kind, n, longest, H, H_kv, d, dtype="bf16", even=False):
    # n sequences, lengths spread over 1 .. longest (the first one has it); even: all of that length
    return dict(name=name, kind=kind, n=n, longest=longest, H=H, H_kv=H_kv, d=d, dtype=dtype, even=even)


def _cached(name, kind, n, longest, H, H_kv, d, page, dtype="bf16", even=False, order="shd"):
    # n sequences with caches of up to `longest` tokens in pages of `page`; order of a page's axes: slot, head, column or head first
    return dict(_packed(name, kind, n, longest, H, H_kv, d, dtype, even), page=page, order=order)


def listed():
    return [
        # a decode step's new rows: one for each of 32 running sequences
        _cached("append_step", "append", 32, 1, 32, 8, 128, 64),
        # a prefill's rows: packed prompts of up to 4096 tokens
        _cached("append_prompts", "append", 4, 4096, 32, 8, 128, 64, even=True),
        # fp32, odd lengths, head dimension 100, pages with the heads apart
        _cached("append_fp32_d100", "append", 7, 701, 32, 32, 100, 16, "fp32", order="hsd"),
        # latency: one user, a short conversation
        _cached("decode_one", "decode", 1, 1500, 32, 8, 128, 64),
        # serving: 64 users, caches of 1 to 8192 tokens
        _cached("decode_64", "decode", 64, 8192, 32, 8, 128, 64),
        # the long context this library is for: 256k tokens each, 16 heads of which none are shared
        _cached("decode_256k", "decode", 2, 262144, 16, 16, 128, 256, even=True, order="hsd"),
        # fp32, head dimension 100, small pages, four query heads to a key/value head
        _cached("decode_fp32_d100", "decode", 13, 3001, 32, 8, 100, 16, "fp32"),
        # short prompts of a few tokens, where every microsecond is a launch
        _packed("prompt_short", "prompt", 5, 200, 16, 16, 64),
        # prompts of one batch, up to 4096 tokens
        _packed("prompt_4k", "prompt", 8, 4096, 32, 8, 128),
        # long prompts
        _packed("prompt_16k", "prompt", 2, 16384, 8, 8, 128, even=True),
        # training documents of the 3B model's head dimension
        _packed("train_4k_d100", "train", 6, 4096, 32, 32, 100),
        # fp32 numerics, odd lengths, two query heads to a key/value head
        _packed("train_fp32", "train", 5, 777, 16, 8, 64, "fp32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "decode", "decode", "prompt", "train"])
    fp32 = rng.random() < 0.25
    H_kv = rng.choice([1, 2, 4, 8, 16])
    H = H_kv * rng.choice([1, 1, 2, 4, 8]) if H_kv < 8 else H_kv * rng.choice([1, 2, 4])
    d = rng.choice([32, 64, 64, 96, 100, 128, 128, 128, 256])
    dtype = "fp32" if fp32 else "bf16"
    if kind in ("append", "decode"):
        longest = 1 if kind == "append" and rng.random() < 0.4 else _log_uniform(rng, 1, 4096 if kind == "append" else 65536)
        case = _cached(None, kind, _log_uniform(rng, 1, 128), longest, H, H_kv, d, rng.choice([16, 32, 64, 128, 256]), dtype,
                       rng.random() < 0.3, rng.choice(["shd", "hsd"]))
        most = dict(append=(1 << 29) if fp32 else 1 << 28, decode=1 << 32)[kind]
    else:
        case = _packed(None, kind, _log_uniform(rng, 1, 16), _log_uniform(rng, 1, 2048 if fp32 else 8192), H, H_kv, d, dtype, rng.random() < 0.3)
        most = 1 << 33            # bytes of one fp32 array of padded scores
    del case["name"]
    while True:
        if kind in ("append", "decode"):
            size = case["n"] * case["longest"] * (2 * H_kv + (H if kind == "append" else 0)) * d * (4 if fp32 else 2)
        else:
            size = case["n"] * H * case["longest"] ** 2 * 4
        if size <= most:
            return case
        case["n" if case["n"] > 4 else "longest"] = max(1, case["n" if case["n"] > 4 else "longest"] * 2 // 3)


def _lengths(case):
    # of the case alone, not of the seed: what is measured is the same for all inputs of a case
    n, longest = case["n"], case["longest"]
    if case["even"]:
        return [longest] * n
    rng = random.Random(n * 1000003 + longest)
    return [longest] + [rng.randint(1, longest) for _ in range(n - 1)]


def _rows(case):
    return sum(_lengths(case))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, H, H_kv, d, n = DTYPES[case["dtype"]], case["H"], case["H_kv"], case["d"], case["n"]

    def normal(*shape):
        x = torch.empty(shape, dtype=dt, device="cuda")
        flat, part = x.view(-1), 1 << 28
        for i in range(0, flat.numel(), part):
            flat[i:i + part] = torch.randn(min(part, flat.numel() - i), generator=gen, device="cuda")
        return x

    lens = _lengths(case)
    state = dict(case, longest_=max(lens))
    if case["kind"] in ("prompt", "train"):
        T = sum(lens)
        state["offsets"] = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
        state["q"], state["k"], state["v"] = normal(T, H, d), normal(T, H_kv, d), normal(T, H_kv, d)
        if case["kind"] == "train":
            state["dout"] = normal(T, H, d)
        return state
    # the pages of a pool that has been in use: any page may belong to any sequence
    page = case["page"]
    before = [0] * n
    if case["kind"] == "append":    # tokens that the caches hold already
        rng = random.Random(n * 7919 + case["longest"])
        before = [rng.randint(0, 4 * page) if case["longest"] > 1 else rng.randint(0, 32 * page) for _ in range(n)]
    pages = [-(-(b + x) // page) for b, x in zip(before, lens)]
    pool = sum(pages) + 3
    order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    width = max(pages)
    table = torch.zeros(n, width, dtype=torch.int32)
    at = 0
    host = order.cpu()
    for s, p in enumerate(pages):
        table[s, :p] = host[at:at + p]
        at += p
    shape = (pool, page, H_kv, d) if case["order"] == "shd" else (pool, H_kv, page, d)
    view = (lambda x: x) if case["order"] == "shd" else (lambda x: x.permute(0, 2, 1, 3))
    if case["kind"] == "decode":
        state["k_cache"], state["v_cache"] = view(normal(*shape)), view(normal(*shape))
        state["table"] = table.cuda()
        state["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        state["q"] = normal(n, H, d)
        return state
    state["k_cache"], state["v_cache"] = (view(torch.zeros(shape, dtype=dt, device="cuda")) for _ in range(2))
    T = sum(lens)
    pos = torch.cat([torch.arange(b, b + x) for b, x in zip(before, lens)])
    seq = torch.repeat_interleave(torch.arange(n), torch.tensor(lens))
    state["pos"] = pos.to(torch.int32).cuda()
    state["slot"] = (table[seq, pos // page].long() * page + pos % page).to(torch.int32).cuda()
    state["q"], state["k"], state["v"] = normal(T, H, d), normal(T, H_kv, d), normal(T, H_kv, d)
    return state


# ---------------------------------------------------------------- the framework's calls


def _own(s):
    from paper_2311_09431_amd import binding as sa
    if s["kind"] == "append":
        q, k = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        sa.sa_cache_append(s["k"], s["v"], s["slot"], s["k_cache"], s["v_cache"], pos=s["pos"], k_out=k, q=s["q"], q_out=q, base=BASE)
        return {"q": q, "k": k, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    q = s["q"]
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[1], q.shape[0], dtype=torch.float32, device=q.device)
    if s["kind"] == "decode":
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        work = torch.empty(sa.sa_attn_decode_workspace(q, s["k_cache"]), dtype=torch.uint8, device=q.device)
        sa.sa_attn_decode(q, s["k_cache"], s["v_cache"], s["table"], s["lens"], out, lse, work)
        return {"out": out, "lse": lse}
    sa.sa_attn_packed_fwd(q, s["k"], s["v"], s["offsets"], out, lse, s["longest_"])
    if s["kind"] == "prompt":
        return {"out": out, "lse": lse}
    delta, dq, dk, dv = torch.empty_like(lse), torch.empty_like(q), torch.empty_like(s["k"]), torch.empty_like(s["v"])
    sa.sa_attn_packed_bwd(q, s["k"], s["v"], out, s["dout"], lse, s["offsets"], delta, dq, dk, dv, s["longest_"])
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


# ---------------------------------------------------------------- the plain forms


def _rotate(x, pos):
    half = x.shape[-1] // 2
    freq = BASE ** (-torch.arange(half, dtype=torch.float64, device=x.device) * 2 / x.shape[-1])
    angle = pos.double()[:, None, None] * freq
    c, sn = angle.cos().float(), angle.sin().float()
    lo, hi = x.float().split(half, -1)
    return torch.cat([lo * c - hi * sn, hi * c + lo * sn], -1).to(x.dtype)


def _plain_append(s):
    q, k = _rotate(s["q"], s["pos"]), _rotate(s["k"], s["pos"])
    slot = s["slot"].long()
    page, at = slot // s["page"], slot % s["page"]
    s["k_cache"][page, at] = k
    s["v_cache"][page, at] = s["v"]
    return {"q": q, "k": k, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_decode(s):
    q, table, lens = s["q"], s["table"].long(), s["lens"]
    B, H, d = q.shape
    H_kv = s["H_kv"]
    L = table.shape[1] * s["page"]
    k = s["k_cache"][table].float().reshape(B, L, H_kv, d).permute(0, 2, 3, 1)
    x = torch.matmul(q.float().view(B, H_kv, H // H_kv, d), k) / math.sqrt(d)
    del k
    x = x.masked_fill(torch.arange(L, device=q.device) >= lens[:, None, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = (x - top).exp()
    total = p.sum(-1, keepdim=True)
    v = s["v_cache"][table].float().reshape(B, L, H_kv, d).permute(0, 2, 1, 3)
    out = torch.matmul(p, v) / total
    return {"out": out.reshape(B, H, d).to(q.dtype), "lse": (top + total.log()).reshape(B, H)}


def _padded(s):
    """Where the packed rows lie in [sequence, row of it], and which of the padded rows are none."""
    off = s["offsets"].long()
    T, L = s["q"].shape[0], s["longest_"]
    rows = torch.arange(T, device=off.device)
    seq = torch.searchsorted(off, rows, right=True) - 1
    at = torch.arange(L, device=off.device)
    index = (off[:-1, None] + at).clamp(max=T - 1)
    return index, at < (off[1:] - off[:-1])[:, None], seq, rows - off[seq]


def _plain_packed(s):
    q, H_kv, d, L = s["q"], s["H_kv"], s["d"], s["longest_"]
    T, H, n = q.shape[0], s["H"], s["n"]
    G = H // H_kv
    index, there, seq, row = _padded(s)

    def pad(x, heads):       # [n, H_kv, heads of the group x rows, d], zeros where no row is
        x = (x[index].float() * there[:, :, None, None]).view(n, L, H_kv, heads // H_kv, d)
        return x.permute(0, 2, 3, 1, 4).reshape(n, H_kv, heads // H_kv * L, d)

    def packed(x, heads):    # back to the packed rows
        return x.reshape(n, H_kv, heads // H_kv, L, d)[seq, :, :, row].reshape(T, heads, d).to(q.dtype)

    qp, kp, vp = pad(q, H), pad(s["k"], H_kv), pad(s["v"], H_kv)
    at = torch.arange(L, device=q.device)
    hidden = at[None, :] > at[:, None]
    x = torch.matmul(qp, kp.transpose(2, 3)).view(n, H_kv, G, L, L).div_(math.sqrt(d)).masked_fill_(hidden, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(total).view(n, H_kv, G * L, L)
    o = torch.matmul(p, vp)
    lse = (top + total.log()).view(n, H, L)[seq, :, row].t().contiguous()
    out = {"out": packed(o, H), "lse": lse}
    if s["kind"] == "prompt":
        return out
    gp = pad(s["dout"], H)
    dv = torch.matmul(p.transpose(2, 3), gp)
    ds = torch.matmul(gp, vp.transpose(2, 3)).sub_((gp * o).sum(-1, keepdim=True)).mul_(p)
    del p, x
    dq = torch.matmul(ds, kp) / math.sqrt(d)
    dk = torch.matmul(ds.transpose(2, 3), qp) / math.sqrt(d)
    return {**out, "dq": packed(dq, H), "dk": packed(dk, H_kv), "dv": packed(dv, H_kv)}


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "decode": _plain_decode, "prompt": _plain_packed, "train": _plain_packed}[state["kind"]](state)


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    es, H, H_kv, d, lens = 4 if case["dtype"] == "fp32" else 2, case["H"], case["H_kv"], case["d"], _lengths(case)
    T = sum(lens)
    if case["kind"] == "append":    # q, k, v read; q, k and the two slots written; ids
        return {"bytes": T * (2 * H + 5 * H_kv) * d * es + 8 * T, "flops": 3 * T * (H + H_kv) * d}
    if case["kind"] == "decode":
        return {"bytes": 2 * T * H_kv * d * es + len(lens) * H * (2 * d * es + 4), "flops": 4 * T * H * d}
    pairs = sum(x * (x + 1) // 2 for x in lens)
    forward = {"bytes": T * (2 * H + 2 * H_kv) * d * es + 4 * T * H, "flops": 4 * pairs * H * d}
    if case["kind"] == "prompt":
        return forward
    return {"bytes": forward["bytes"] + T * (4 * H + 4 * H_kv) * d * es + 4 * T * H, "flops": 14 * pairs * H * d}


# ---------------------------------------------------------------- the definition in 64 bits


def _attention(q, k, v, causal):
    """O [rows, d] and LSE [rows] of one head in 64 bits, and the weights."""
    x = q @ k.t() / math.sqrt(q.shape[1])
    if causal:
        x = x + torch.triu(torch.full_like(x, -math.inf), 1)
    lse = torch.logsumexp(x, 1)
    w = torch.exp(x - lse[:, None])
    return w @ v, lse, w


def exact(case, seed):
    s = prepare(case, seed)
    H, G, d = case["H"], case["H"] // case["H_kv"], case["d"]
    if case["kind"] == "append":
        half = d // 2
        turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), s["pos"].double()[:, None]
                           * torch.exp(torch.arange(half, device="cuda", dtype=torch.float64) * (-2 * math.log(BASE) / d)))
        got = {}
        for name in ("q", "k"):
            x = s[name].double()
            z = torch.complex(x[..., :half], x[..., half:]) * turn[:, None, :]
            got[name] = torch.cat([z.real, z.imag], -1)
        # the caches hold zeros but for the new rows
        for name, rows in (("k_cache", got["k"]), ("v_cache", s["v"].double())):
            cache = torch.zeros(s[name].shape, dtype=torch.float64, device="cuda")
            cache.view(-1, *cache.shape[2:]).index_copy_(0, s["slot"].long(), rows)
            got[name] = cache
        return got
    lens = _lengths(case)
    if case["kind"] == "decode":
        out = torch.empty(case["n"], H, d, dtype=torch.float64, device="cuda")
        lse = torch.empty(case["n"], H, dtype=torch.float64, device="cuda")
        for b, x in enumerate(lens):
            ids = s["table"][b, :-(-x // case["page"])].long()
            for h in range(case["H_kv"]):
                k, v = (s[c][ids, :, h].reshape(-1, d)[:x].double() for c in ("k_cache", "v_cache"))
                mine = slice(h * G, (h + 1) * G)
                out[b, mine], lse[b, mine], _ = _attention(s["q"][b, mine].double(), k, v, False)
        return {"out": out, "lse": lse}
    q, k, v = (s[c].double() for c in "qkv")
    got = {"out": torch.empty_like(q), "lse": torch.empty(H, q.shape[0], dtype=torch.float64, device="cuda")}
    train = case["kind"] == "train"
    if train:
        g = s["dout"].double()
        got.update(dq=torch.empty_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v))
    first = 0
    for x in lens:
        r = slice(first, first + x)
        first += x
        for h in range(H):
            o, l, w = _attention(q[r, h], k[r, h // G], v[r, h // G], True)
            got["out"][r, h], got["lse"][h, r] = o, l
            if train:
                dp = g[r, h] @ v[r, h // G].t()
                ds = w * (dp - (w * dp).sum(1, keepdim=True)) / math.sqrt(d)
                got["dq"][r, h] = ds @ k[r, h // G]
                got["dk"][r, h // G] += ds.t() @ q[r, h]
                got["dv"][r, h // G] += w.t() @ g[r, h]
    return got
