"""Timed cases of attention with a sliding window, of drafted tokens over the paged cache, and of moving what the cache holds.

  prompt   causal attention of packed prompts, each token over a window of the last ones and a few first ones (forward)
  train    the same, forward and backward
  decode   one new token a sequence over the window and the first tokens of its paged cache
  tree     the drafted tokens of each sequence, each over the cached tokens and those of the draft that it descends from
  copy     pages of the cache copied to others
  accept   the accepted tokens of each draft moved up behind the tokens in front of it

Inputs are seeded Gaussians rounded once to the storage type.  Head counts and dimensions are those of the models and tests
of this repository (16 or 32 heads of 128, 32 of 100, 64 in the tests; 8 key/value heads for 32).
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
PACKED = ("prompt", "train")


def _packed(name, kind, n, longest, H, H_kv, d, window, sinks, dtype="bf16", even=False):
    # n sequences, lengths spread over 1 .. longest (the first one has it); even: all of that length
    return dict(name=name, kind=kind, n=n, longest=longest, H=H, H_kv=H_kv, d=d, window=window, sinks=sinks, dtype=dtype, even=even)


def _cached(name, kind, n, longest, H, H_kv, d, page, dtype="bf16", even=False, order="shd", **more):
    # n sequences with caches of up to `longest` tokens in pages of `page`; order of a page's axes: slot, head, column or head first
    return dict(name=name, kind=kind, n=n, longest=longest, H=H, H_kv=H_kv, d=d, page=page, dtype=dtype, even=even, order=order, **more)


def listed():
    return [
        # short prompts of a few tokens under a small window, where every microsecond is a launch
        _packed("prompt_short", "prompt", 5, 200, 16, 16, 64, 64, 4),
        # the long prompt that a window is for
        _packed("prompt_32k", "prompt", 1, 32768, 16, 8, 128, 4096, 4, even=True),
        # training on long documents
        _packed("train_16k", "train", 2, 16384, 16, 8, 128, 2048, 4),
        # fp32 numerics, odd lengths, head dimension 100, two query heads to a key/value head
        _packed("train_fp32_d100", "train", 5, 777, 16, 8, 100, 100, 5, "fp32"),
        # serving: 64 users, caches of 1 to 8192 tokens
        _cached("decode_64", "decode", 64, 8192, 32, 8, 128, 64, window=1024, sinks=4),
        # the long context this library is for, 256k tokens, under a long window; 16 heads of which none are shared
        _cached("decode_256k", "decode", 2, 262144, 16, 16, 128, 256, even=True, order="hsd", window=32768, sinks=64),
        # latency: one user, a short conversation, eight drafted tokens
        _cached("tree_one", "tree", 1, 1500, 32, 8, 128, 64, draft=8),
        # serving: 32 users, caches of 1 to 8192 tokens, trees of up to 32
        _cached("tree_32", "tree", 32, 8192, 32, 8, 128, 64, draft=32),
        # 64 sequences forked: the last page of each, as far as it is filled
        _cached("copy_fork", "copy", 64, 1, 32, 8, 128, 64, part=True),
        # a pool pushed together: whole pages, 0.5 GB of them
        _cached("copy_pool", "copy", 2048, 1, 32, 8, 128, 64, part=False),
        # the accepted ones of 64 users' drafts
        _cached("accept_64", "accept", 64, 8192, 32, 8, 128, 64, draft=32),
        # fp32, head dimension 100, small pages, heads apart
        _cached("accept_fp32_d100", "accept", 13, 3001, 32, 8, 100, 16, "fp32", order="hsd", draft=13),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "train", "decode", "tree", "tree", "copy", "accept"])
    H_kv = rng.choice([1, 2, 4, 8, 16])
    H = H_kv * rng.choice([1, 1, 2, 4, 8]) if H_kv < 8 else H_kv * rng.choice([1, 2, 4])
    d = rng.choice([32, 64, 64, 96, 100, 128, 128, 128, 256])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    es = 4 if dtype == "fp32" else 2
    if kind in PACKED:
        longest = _log_uniform(rng, 1, 4096 if dtype == "fp32" else 16384)
        case = _packed(None, kind, _log_uniform(rng, 1, 16), longest, H, H_kv, d, _log_uniform(rng, 1, 4096), rng.choice([0, 1, 4, 4, 33, 130]), dtype,
                       rng.random() < 0.3)
        size = lambda c: c["n"] * H * c["longest"] * (2 * min(c["longest"], c["window"]) + c["sinks"]) * 4       # noqa: E731  (bytes of its fp32 scores)
        most = 1 << 32
    else:
        case = _cached(None, kind, _log_uniform(rng, 1, 64 if kind == "tree" else 128), _log_uniform(rng, 1, 65536), H, H_kv, d, rng.choice([16, 32, 64, 128, 256]),
                       dtype, rng.random() < 0.3, rng.choice(["shd", "hsd"]))
        size = lambda c: c["n"] * c["longest"] * 2 * H_kv * d * es      # noqa: E731  (bytes cached)
        most = 1 << 31
        if kind == "decode":
            case.update(window=_log_uniform(rng, 1, 32768), sinks=rng.choice([0, 1, 4, 64, 130]))
        elif kind == "tree":
            case.update(draft=rng.randint(1, 64))
            scores = H * case["draft"] * 8
            size = lambda c: c["n"] * c["longest"] * (scores + 2 * H_kv * d * es)      # noqa: E731
        elif kind == "accept":
            case.update(draft=rng.randint(1, 64))
        else:
            case.update(longest=1, n=_log_uniform(rng, 1, 4096), part=rng.random() < 0.5)
            size = lambda c: c["n"] * c["page"] * 2 * H_kv * d * es     # noqa: E731
            most = 1 << 29
    del case["name"]
    while size(case) > most:
        key = "n" if case["n"] > 4 else "longest"
        case[key] = max(1, case[key] * 2 // 3)
    return case


def _spread(case, most, salt):
    # 1 .. most for each of n, the first one the most: of the case alone, not of the seed, so what is measured is the same for all inputs
    rng = random.Random(case["n"] * 1000003 + most + salt)
    return [most] + [most if case["even"] else rng.randint(1, most) for _ in range(case["n"] - 1)]


def _lengths(case):
    return _spread(case, case["longest"], 0)


def _drafts(case):
    return _spread(case, case["draft"], 7)


def _accepted(case):
    # of a draft about a third of its depth, at least its first token
    rng = random.Random(case["n"] * 7919 + case["draft"])
    return [rng.randint(1, max(1, x // 3)) for x in _drafts(case)]


def _tokens(case):
    # of each page that is copied: all of them, or 1 .. page
    return _spread(case, case["page"], 3) if case["part"] else [case["page"]] * case["n"]


def prepare(case, seed):
    gen, host = torch.Generator(device="cuda"), torch.Generator()
    gen.manual_seed(seed)
    host.manual_seed(seed)
    dt, H, H_kv, d, n = DTYPES[case["dtype"]], case["H"], case["H_kv"], case["d"], case["n"]

    def normal(*shape):
        x = torch.empty(shape, dtype=dt, device="cuda")
        flat, part = x.view(-1), 1 << 28
        for i in range(0, flat.numel(), part):
            flat[i:i + part] = torch.randn(min(part, flat.numel() - i), generator=gen, device="cuda")
        return x

    def ints(x):
        return torch.as_tensor(x).to(torch.int32).cuda()

    state = dict(case)
    lens = _lengths(case)
    if case["kind"] in PACKED:
        T = sum(lens)
        state["longest_"] = max(lens)
        state["offsets"] = ints([0] + lens).cumsum(0).to(torch.int32)
        state["q"], state["k"], state["v"] = normal(T, H, d), normal(T, H_kv, d), normal(T, H_kv, d)
        if case["kind"] == "train":
            state["dout"] = normal(T, H, d)
        return state
    page = case["page"]

    def caches(pool):
        shape = (pool, page, H_kv, d) if case["order"] == "shd" else (pool, H_kv, page, d)
        view = (lambda x: x) if case["order"] == "shd" else (lambda x: x.permute(0, 2, 1, 3))
        state["k_cache"], state["v_cache"] = view(normal(*shape)), view(normal(*shape))

    if case["kind"] == "copy":
        caches(2 * n + 3)
        order = torch.randperm(2 * n + 3, generator=host)
        state["from"], state["to"], state["tokens"] = ints(order[:n]), ints(order[n:2 * n]), ints(_tokens(case))
        return state
    # the pages of a pool that has been in use: any page may belong to any sequence
    drafts = _drafts(case) if "draft" in case else [0] * n
    pages = [-(-(x + y) // page) for x, y in zip(lens, drafts)]
    caches(sum(pages) + 3)
    order = torch.randperm(sum(pages) + 3, generator=host).to(torch.int32)
    table = torch.zeros(n, max(pages), dtype=torch.int32)
    at = 0
    for s, p in enumerate(pages):
        table[s, :p] = order[at:at + p]
        at += p
    state["table"], state["lens"] = table.cuda(), ints(lens)
    if case["kind"] == "decode":
        state["q"] = normal(n, H, d)
        return state
    T = case["draft"]
    state["drafts"] = ints(drafts)
    if case["kind"] == "accept":
        # tokens of a draft in its order, of each draft as many as were accepted
        state["accepted"] = ints(_accepted(case))
        chosen = torch.zeros(n, T, dtype=torch.int32)
        for s, (x, y) in enumerate(zip(_accepted(case), drafts)):
            chosen[s, :x] = torch.randperm(y, generator=host)[:x].sort().values
        state["chosen"] = chosen.cuda()
        state["lens_after"] = torch.empty_like(state["lens"])
        return state
    # a tree: each token hangs on an earlier one or on the last cached token, and sees whom it descends from and itself
    seen = torch.zeros(n, T + 1, dtype=torch.int64)        # [.., 0]: the cached token
    rows = torch.arange(n)
    for i in range(T):
        seen[:, i + 1] = seen[rows, torch.randint(0, i + 1, (n,), generator=host)] | (1 << i if i < 63 else -(1 << 63))
    state["seen"] = seen[:, 1:].contiguous().cuda()
    state["q"] = normal(n, T, H, d)
    # rows of a shorter draft stay as they are
    state["out"] = torch.zeros(n, T, H, d, dtype=dt, device="cuda")
    state["lse"] = torch.zeros(n, T, H, dtype=torch.float32, device="cuda")
    return state


# ---------------------------------------------------------------- the framework's calls


def _own(s):
    from paper_2311_09431_amd import binding as sa
    kind = s["kind"]
    if kind == "copy":
        sa.sa_cache_copy(s["k_cache"], s["v_cache"], s["from"], s["to"], s["tokens"] if s["part"] else None)
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if kind == "accept":
        sa.sa_cache_accept(s["k_cache"], s["v_cache"], s["table"], s["lens"], s["chosen"], s["accepted"], s["lens_after"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "lens": s["lens_after"]}
    q = s["q"]
    if kind == "tree":
        work = torch.empty(sa.sa_attn_tree_workspace(q, s["k_cache"]), dtype=torch.uint8, device=q.device)
        sa.sa_attn_tree(q, s["k_cache"], s["v_cache"], s["table"], s["lens"], s["seen"], s["out"], s["lse"], work, drafts=s["drafts"])
        return {"out": s["out"], "lse": s["lse"]}
    out = torch.empty_like(q)
    if kind == "decode":
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        work = torch.empty(sa.sa_attn_decode_workspace(q, s["k_cache"]), dtype=torch.uint8, device=q.device)
        sa.sa_attn_window_decode(q, s["k_cache"], s["v_cache"], s["table"], s["lens"], out, lse, work, s["window"], s["sinks"])
        return {"out": out, "lse": lse}
    lse = torch.empty(q.shape[1], q.shape[0], dtype=torch.float32, device=q.device)
    sa.sa_attn_window_fwd(q, s["k"], s["v"], s["offsets"], out, lse, s["longest_"], s["window"], s["sinks"])
    if kind == "prompt":
        return {"out": out, "lse": lse}
    delta, dq, dk, dv = torch.empty_like(lse), torch.empty_like(q), torch.empty_like(s["k"]), torch.empty_like(s["v"])
    work = torch.empty(sa.sa_attn_window_bwd_workspace(q, s["k"], s["offsets"], s["longest_"], s["window"], s["sinks"]), dtype=torch.uint8, device=q.device)
    sa.sa_attn_window_bwd(q, s["k"], s["v"], out, s["dout"], lse, s["offsets"], delta, dq, dk, dv, work, s["longest_"], s["window"], s["sinks"])
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


# ---------------------------------------------------------------- the plain forms


def _plain_copy(s):
    at = torch.arange(s["page"], device=s["from"].device)
    copied = (at < s["tokens"][:, None])[:, :, None, None]
    for cache in (s["k_cache"], s["v_cache"]):
        cache[s["to"].long()] = torch.where(copied, cache[s["from"].long()], cache[s["to"].long()])
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _slots(s, token):
    # page and place in it of token numbers [sequence, any]
    return s["table"].long().gather(1, token // s["page"]), token % s["page"]


def _plain_accept(s):
    lens, chosen = s["lens"].long()[:, None], s["chosen"].long()
    i = torch.arange(chosen.shape[1], device=lens.device)[None, :]
    taken = i < s["accepted"][:, None]
    # (in the place of what is not accepted the last token in front of the draft, onto itself)
    page, at = _slots(s, torch.where(taken, lens + chosen, lens - 1))
    new_page, new_at = _slots(s, torch.where(taken, lens + i, lens - 1))
    for cache in (s["k_cache"], s["v_cache"]):
        cache[new_page, new_at] = cache[page, at]
    s["lens_after"].copy_(s["lens"] + s["accepted"])
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "lens": s["lens_after"]}


def _softmax(x):
    """exp(x - max) of the last axis, its sum, and the log-sum-exp."""
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return p, total, top + total.log()


def _cached_rows(s, name):
    # [sequence, key/value head, token, d]
    table = s["table"].long()
    B, L = table.shape[0], table.shape[1] * s["page"]
    return s[name][table].float().reshape(B, L, s["H_kv"], s["d"]).permute(0, 2, 1, 3)


def _plain_decode(s):
    q, lens = s["q"], s["lens"][:, None, None, None]
    B, H, d = q.shape
    k = _cached_rows(s, "k_cache")
    x = torch.matmul(q.float().view(B, s["H_kv"], H // s["H_kv"], d), k.transpose(2, 3)) / math.sqrt(d)
    del k
    at = torch.arange(x.shape[-1], device=q.device)
    x = x.masked_fill(~((at < lens) & ((at >= lens - s["window"]) | (at < s["sinks"]))), -math.inf)
    p, total, lse = _softmax(x)
    out = torch.matmul(p, _cached_rows(s, "v_cache")) / total
    return {"out": out.reshape(B, H, d).to(q.dtype), "lse": lse.reshape(B, H)}


def _plain_tree(s):
    q, H_kv, lens = s["q"], s["H_kv"], s["lens"].long()
    B, T, H, d = q.shape
    G = H // H_kv
    k = _cached_rows(s, "k_cache")
    x = torch.matmul(q.float().view(B, T, H_kv, G, d).permute(0, 2, 1, 3, 4).reshape(B, H_kv, T * G, d), k.transpose(2, 3)) / math.sqrt(d)
    del k
    nth = torch.arange(x.shape[-1], device=q.device) - lens[:, None]        # of the draft; negative: cached before
    bit = (s["seen"][:, :, None] >> nth.clamp(0, 63)[:, None, :]) & 1
    sees = (nth[:, None, :] < 0) | ((nth[:, None, :] < s["drafts"][:, None, None]) & (bit != 0))        # [B, T, L]
    x = x.view(B, H_kv, T, G, -1).masked_fill_(~sees[:, None, :, None, :], -math.inf).view(B, H_kv, T * G, -1)
    p, total, lse = _softmax(x)
    out = torch.matmul(p, _cached_rows(s, "v_cache")) / total
    rows = (torch.arange(T, device=q.device) < s["drafts"][:, None])[:, :, None]
    out = out.view(B, H_kv, T, G, d).permute(0, 2, 1, 3, 4).reshape(B, T, H, d).to(q.dtype)
    lse = lse.view(B, H_kv, T, G).permute(0, 2, 1, 3).reshape(B, T, H)
    s["out"].copy_(torch.where(rows[..., None], out, s["out"]))
    s["lse"].copy_(torch.where(rows, lse, s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


def _plain_packed(s):
    """Blocks of C rows, each over its own keys and those of the block before it, and beside them the first tokens."""
    q, H, H_kv, d, n, S = s["q"], s["H"], s["H_kv"], s["d"], s["n"], min(s["sinks"], s["longest_"])
    T, G, dev = q.shape[0], s["H"] // s["H_kv"], q.device
    C = min(s["window"], s["longest_"])
    blocks = -(-s["longest_"] // C)
    before = 1 if s["window"] > 1 and blocks > 1 else 0
    L, span = blocks * C, (1 + before) * C
    off = s["offsets"].long()
    rows = torch.arange(T, device=dev)
    seq = torch.searchsorted(off, rows, right=True) - 1
    row = rows - off[seq]
    at = torch.arange(L, device=dev)
    index, there = (off[:-1, None] + at).clamp(max=T - 1), at < (off[1:] - off[:-1])[:, None]

    def pad(x, heads):       # [n, H_kv, block, heads of the group x rows, d], zeros where no row is
        x = (x[index].float() * there[:, :, None, None]).view(n, blocks, C, H_kv, heads // H_kv, d)
        return x.permute(0, 3, 1, 4, 2, 5).reshape(n, H_kv, blocks, heads // H_kv * C, d)

    def packed(x, heads):    # back to the packed rows
        x = x.reshape(n, H_kv, blocks, heads // H_kv, C, -1)
        return x[seq, :, row // C, :, row % C].reshape(T, heads, -1)

    def spans(x):            # rows of the block before in front of each block's own
        return torch.cat([torch.cat([torch.zeros_like(x[:, :, :1]), x[:, :, :-1]], 2), x], 3) if before else x

    def unspanned(x):        # the sum of what the two blocks that have a row say of it
        if not before:
            return x
        y = x[:, :, :, C:].clone()
        y[:, :, :-1] += x[:, :, 1:, :C]
        return y

    def firsts(x):           # of each sequence, for all its blocks
        return x.reshape(n, H_kv, 1, L, d)[:, :, :, :S]

    qp, k, v = pad(q, H), pad(s["k"], H_kv), pad(s["v"], H_kv)
    kp, vp, k0, v0 = spans(k), spans(v), firsts(k), firsts(v)
    # rows of a block against its span, and against the first tokens; a first token within the window counts there
    a, b = torch.arange(C, device=dev)[:, None] + before * C, torch.arange(span, device=dev)[None, :]
    near = (b <= a) & (a - b < s["window"])
    if before:
        near = near.expand(blocks, C, span) & ((torch.arange(blocks, device=dev)[:, None, None] > 0) | (b >= C))
    else:
        near = near.expand(blocks, C, span)
    far = torch.arange(S, device=dev) <= torch.arange(L, device=dev).view(blocks, C, 1) - s["window"]
    sees = torch.cat([near, far], -1)[:, None].expand(blocks, G, C, span + S).reshape(blocks, G * C, span + S)
    x = torch.cat([torch.matmul(qp, kp.transpose(3, 4)), torch.matmul(qp, k0.transpose(3, 4))], -1).div_(math.sqrt(d)).masked_fill_(~sees, -math.inf)
    p, total, lse = _softmax(x)
    p = p.div_(total)
    o = torch.matmul(p[..., :span], vp) + torch.matmul(p[..., span:], v0)
    out = {"out": packed(o, H).to(q.dtype), "lse": packed(lse, H)[..., 0].t().contiguous()}
    if s["kind"] == "prompt":
        return out
    gp = pad(s["dout"], H)
    ds = torch.cat([torch.matmul(gp, vp.transpose(3, 4)), torch.matmul(gp, v0.transpose(3, 4))], -1).sub_((gp * o).sum(-1, keepdim=True)).mul_(p)
    ds = ds.div_(math.sqrt(d))
    dq = torch.matmul(ds[..., :span], kp) + torch.matmul(ds[..., span:], k0)

    def of_keys(w, x):       # sum over the rows that see a key of w times x
        y = unspanned(torch.matmul(w[..., :span].transpose(3, 4), x)).reshape(n, H_kv, L, d)
        y[:, :, :S] += torch.matmul(w[..., span:].transpose(3, 4), x).sum(2)
        return packed(y.view(n, H_kv, blocks, C, d), H_kv).to(q.dtype)

    return {**out, "dq": packed(dq, H).to(q.dtype), "dk": of_keys(ds, qp), "dv": of_keys(p, gp)}


def run(state):
    if own:
        return _own(state)
    return {"prompt": _plain_packed, "train": _plain_packed, "decode": _plain_decode, "tree": _plain_tree, "copy": _plain_copy,
            "accept": _plain_accept}[state["kind"]](state)


# ---------------------------------------------------------------- what a pass cannot do without


def _pairs(n, window, sinks):
    """(row, key) pairs of a sequence of n rows: the nearest `window` keys, and of those further back the first `sinks`."""
    def ramp(m, most):       # 1 + 2 + .. up to m terms, none above `most`
        return m * (m + 1) // 2 if m <= most else most * (most + 1) // 2 + (m - most) * most
    return ramp(n, window) + ramp(max(0, n - window), sinks)


def work(case):
    es, H, H_kv, d, lens = 4 if case["dtype"] == "fp32" else 2, case["H"], case["H_kv"], case["d"], _lengths(case)
    token = 2 * H_kv * d * es           # a key and a value
    if case["kind"] == "copy":
        return {"bytes": 2 * token * sum(_tokens(case)) + 8 * case["n"], "flops": 0}
    if case["kind"] == "accept":
        return {"bytes": 2 * token * sum(_accepted(case)) + 4 * sum(_accepted(case)), "flops": 0}
    if case["kind"] == "decode":
        seen = sum(min(x, case["window"] + min(case["sinks"], max(0, x - case["window"]))) for x in lens)
        return {"bytes": token * seen + case["n"] * H * (2 * d * es + 4), "flops": 4 * seen * H * d}
    if case["kind"] == "tree":
        drafts = _drafts(case)
        return {"bytes": token * (sum(lens) + sum(drafts)) + sum(drafts) * H * (2 * d * es + 4), "flops": 4 * sum(x * y for x, y in zip(lens, drafts)) * H * d}
    T = sum(lens)
    pairs = sum(_pairs(x, case["window"], case["sinks"]) for x in lens)
    forward = {"bytes": T * (2 * H + 2 * H_kv) * d * es + 4 * T * H, "flops": 4 * pairs * H * d}
    if case["kind"] == "prompt":
        return forward
    return {"bytes": forward["bytes"] + T * (4 * H + 4 * H_kv) * d * es + 4 * T * H, "flops": 14 * pairs * H * d}


# ---------------------------------------------------------------- the definition in 64 bits


def _rows_of(q, k, v, sees):
    """O, LSE and weights of rows q over keys k, v, of those that sees [row, key] names."""
    x = (q @ k.t() / math.sqrt(q.shape[1])).masked_fill(~sees, -math.inf)
    lse = torch.logsumexp(x, 1)
    w = torch.exp(x - lse[:, None])
    return w @ v, lse, w


def _exact_packed(case, s):
    H, G, d, window, sinks = case["H"], case["H"] // case["H_kv"], case["d"], case["window"], case["sinks"]
    q, k, v = (s[c].double() for c in "qkv")
    got = {"out": torch.empty_like(q), "lse": torch.empty(H, q.shape[0], dtype=torch.float64, device="cuda")}
    train = case["kind"] == "train"
    if train:
        g = s["dout"].double()
        got.update(dq=torch.empty_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v))
    first = 0
    for n in _lengths(case):
        for r0 in range(0, n, 2048):
            r1 = min(n, r0 + 2048)
            lo = max(0, r0 - window + 1)
            ids = torch.cat([torch.arange(min(sinks, lo), device="cuda"), torch.arange(lo, r1, device="cuda")])
            a = torch.arange(r0, r1, device="cuda")[:, None]
            sees = (ids <= a) & ((a - ids < window) | (ids < sinks))
            r, ids = slice(first + r0, first + r1), ids + first
            for h in range(H):
                keys, values = k[ids, h // G], v[ids, h // G]
                o, l, w = _rows_of(q[r, h], keys, values, sees)
                got["out"][r, h], got["lse"][h, r] = o, l
                if train:
                    dp = g[r, h] @ values.t()
                    ds = w * (dp - (w * dp).sum(1, keepdim=True)) / math.sqrt(d)
                    got["dq"][r, h] = ds @ keys
                    got["dk"][:, h // G].index_add_(0, ids, ds.t() @ q[r, h])
                    got["dv"][:, h // G].index_add_(0, ids, w.t() @ g[r, h])
        first += n
    return got


def exact(case, seed):
    s = prepare(case, seed)
    H, G, d, kind, lens = case["H"], case["H"] // case["H_kv"], case["d"], case["kind"], _lengths(case)
    if kind in PACKED:
        return _exact_packed(case, s)
    if kind == "copy":
        for name in ("k_cache", "v_cache"):
            s[name] = s[name].double()
            for src, dst, x in zip(s["from"].tolist(), s["to"].tolist(), _tokens(case)):
                s[name][dst, :x] = s[name][src, :x]
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    table, page = s["table"].tolist(), case["page"]
    if kind == "accept":
        got = {"k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double(), "lens": None}
        chosen = s["chosen"].tolist()
        for b, (n, x) in enumerate(zip(lens, _accepted(case))):
            for i in range(x):      # (ascending: no token is written before it is read)
                src, dst = n + chosen[b][i], n + i
                for name in ("k_cache", "v_cache"):
                    got[name][table[b][dst // page], dst % page] = got[name][table[b][src // page], src % page]
        return got
    T = case["draft"] if kind == "tree" else 1
    drafts = _drafts(case) if kind == "tree" else [0] * case["n"]
    out = torch.zeros(case["n"], T, H, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(case["n"], T, H, dtype=torch.float64, device="cuda")
    bits = 1 << torch.arange(64, device="cuda")
    for b, n in enumerate(lens):
        m, rows = n + drafts[b], drafts[b] if kind == "tree" else 1
        pages = s["table"][b, :-(-m // page)].long()
        at = torch.arange(m, device="cuda")[None, :]
        if kind == "tree":
            sees = (at < n).expand(rows, m).clone()
            sees[:, n:] = (s["seen"][b, :rows, None] & bits[:rows]) != 0
        else:
            sees = (at >= n - case["window"]) | (at < case["sinks"])
        used = sees.any(0).nonzero()[:, 0]
        sees = sees[:, used].repeat_interleave(G, 0)
        for h in range(case["H_kv"]):
            k, v = (s[c][pages[used // page], used % page, h].double() for c in ("k_cache", "v_cache"))
            mine = slice(h * G, (h + 1) * G)
            q = (s["q"][b, :rows, mine] if kind == "tree" else s["q"][b:b + 1, mine]).double().reshape(rows * G, d)
            o, l, _ = _rows_of(q, k, v, sees)
            out[b, :rows, mine], lse[b, :rows, mine] = o.view(rows, G, d), l.view(rows, G)
    return {"out": out, "lse": lse} if kind == "tree" else {"out": out[:, 0], "lse": lse[:, 0]}
