"""Timed cases of the operators around a prefix cache held in 4 bits: rows made from a layer's projections (norm and
rotation), rows appended to the cache, accepted rows committed, and tree attention that reads it.

`run` computes an operator in its plain form from elementary torch operations, or, with `own`, through the library."""
import math

import numpy as np
import torch

own = False

PAGE = 32          # cache rows of a page

# trees of the repository's workloads: (roots; children per level)
TREES = {
    "token": (1, ()),
    "binary": (1, (2, 2, 2)),
    "static": (1, (4, 2, 2, 1)),
    "deep": (1, (4, 2, 2, 1, 1, 1, 1, 1)),
    "forest": (8, (1, 2, 2, 1, 1, 1)),
    "two_roots": (2, (4, 3, 1, 1)),
    "fork": (16, (1, 1, 1, 1)),
}


def listed():
    return [
        # one new token of one sequence: the call whose latency a user waits for
        dict(name="attend_token_b1", op="attend", dtype="bf16", B=1, Hq=32, Hkv=8, D=128, tree="token", L=1001, ragged=False, sliced=False),
        # single tokens of a batch of long conversations, grouped queries
        dict(name="attend_token_b8_long", op="attend", dtype="bf16", B=8, Hq=32, Hkv=8, D=128, tree="token", L=32001, ragged=True, sliced=False),
        # the repository's long-context workload: a 45-node tree per sequence
        dict(name="attend_tree_b16_4096", op="attend", dtype="bf16", B=16, Hq=32, Hkv=32, D=128, tree="static", L=4096, ragged=False, sliced=False),
        # target-initialised forest, ragged prefixes, per-sequence slices
        dict(name="attend_forest_b32", op="attend", dtype="bf16", B=32, Hq=32, Hkv=32, D=128, tree="forest", L=4096, ragged=True, sliced=True),
        # fp32 tensors and 64-wide heads, the small checking workload
        dict(name="attend_fp32_d64", op="attend", dtype="f32", B=2, Hq=4, Hkv=4, D=64, tree="binary", L=131, ragged=True, sliced=False),
        # one new token's projections
        dict(name="rope_token_b1", op="rope", dtype="bf16", B=1, Hq=32, Hkv=8, D=128, tree="token", T=0, pos=1001, norm=True, rot=128, interleaved=False),
        # a verify step's tree rows, Llama-style (rotation only)
        dict(name="rope_tree_b16", op="rope", dtype="bf16", B=16, Hq=32, Hkv=32, D=128, tree="static", T=0, pos=4096, norm=False, rot=128, interleaved=False),
        # a prompt, far positions, part of the head rotated
        dict(name="rope_prompt_8191", op="rope", dtype="bf16", B=1, Hq=32, Hkv=8, D=128, tree="", T=8191, pos=120000, norm=True, rot=64, interleaved=True),
        # a prompt's rows into the cache
        dict(name="append_prompt_8191", op="append", dtype="bf16", B=1, H=32, D=128, T=8191, start=0),
        # a chunk that starts and ends inside a page, fp32
        dict(name="append_chunk_fp32", op="append", dtype="f32", B=4, H=4, D=64, T=45, start=77),
        # accepted rows of a small model's step
        dict(name="commit_l2_b4", op="commit", dtype="bf16", layers=2, B=4, H=8, D=128, tree="static", L=512),
        # accepted rows of all layers of the long-context workload's model
        dict(name="commit_l32_b16", op="commit", dtype="bf16", layers=32, B=16, H=32, D=128, tree="static", L=512),
    ]


def _span(rng, lo, hi):
    """A whole number whose logarithm is spread evenly over the range."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "rope", "append", "commit"])
    D = rng.choice([128, 128, 128, 64])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "attend":
        Hkv, G = rng.choice([(4, 1), (8, 1), (32, 1), (8, 4), (4, 8), (2, 3), (8, 2)])
        small = dtype == "f32" or D == 64
        tree = rng.choice(sorted(TREES))
        while True:
            B, L = _span(rng, 1, 8 if small else 32), _span(rng, 1, 3000 if small else 32768)
            if B * Hkv * G * _nodes(tree) * L <= 32 * 32 * 45 * 4096 and B * Hkv * L <= 32 * 32 * 4096:
                break
        return dict(op=op, dtype=dtype, B=B, Hq=Hkv * G, Hkv=Hkv, D=D, tree=tree, L=L, ragged=rng.random() < 0.5, sliced=rng.random() < 0.5)
    if op == "rope":
        Hkv, G = rng.choice([(4, 1), (8, 4), (32, 1), (2, 3)])
        c = dict(op=op, dtype=dtype, Hq=Hkv * G, Hkv=Hkv, D=D, pos=_span(rng, 1, 200000), norm=rng.random() < 0.5, rot=rng.choice([D, D, D // 2]), interleaved=rng.random() < 0.5)
        if rng.random() < 0.5:
            return dict(c, tree=rng.choice(sorted(TREES)), T=0, B=_span(rng, 1, 16))
        return dict(c, tree="", T=_span(rng, 1, 4096), B=rng.choice([1, 1, 2]))
    if op == "append":
        return dict(op=op, dtype=dtype, B=rng.choice([1, 2, 4]), H=rng.choice([2, 8, 32]), D=D, T=_span(rng, 1, 2000), start=_span(rng, 1, 1000) - 1)
    return dict(op=op, dtype=dtype, layers=_span(rng, 1, 16), B=_span(rng, 1, 16), H=rng.choice([2, 8, 32]), D=D, tree=rng.choice(sorted(t for t in TREES if TREES[t][1])), L=_span(rng, 1, 512))


def _parents(tree):
    roots, branching = TREES[tree]
    parent, first, count = [-1] * roots, 0, roots
    for k in branching:
        parent += [first + i // k for i in range(count * k)]
        first, count = first + count, count * k
    return parent


def _nodes(tree):
    return len(_parents(tree))


def _levels(tree):
    """First node of every level, and the number of nodes."""
    roots, branching = TREES[tree]
    ls, count = [0, roots], roots
    for k in branching:
        count *= k
        ls.append(ls[-1] + count)
    return ls


def _lens(case, order):
    B, L = case["B"], case["L"]
    lens = [L if not case["ragged"] else max(0, L - (15 * L * b) // (16 * B)) for b in range(B)]
    ls = _levels(case["tree"])
    act = [ls[1 + b % (len(ls) - 1)] if case["sliced"] else ls[-1] for b in range(B)]
    return [lens[i] for i in order], [act[i] for i in order]


def _accepted(case):
    depth = len(TREES[case["tree"]][1])
    return [b % (depth + 1) for b in range(case["B"])]


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ------------------------------------------------------------------ the 4-bit form of rows

def _quantise(x):
    """Codes 0..15, scale and offset of rows (last axis): value = scale * (16 + code) + offset, both bf16."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    s = ((hi - lo) / 15).to(torch.bfloat16)
    o = (lo - 16 * s.to(x.dtype)).to(torch.bfloat16)
    sx = s.to(x.dtype)
    code = ((x - o.to(x.dtype)) / torch.where(sx > 0, sx, torch.ones_like(sx))).round().clamp(16, 31) - 16
    return torch.where(sx > 0, code, torch.zeros_like(code)).to(torch.uint8), s, o


def _bytes_of(c):
    """Codes [..., 4 words, 2, 2, 2] (value 8w + 2i + h at [w, i // 2, i % 2, h]) to bytes [..., 16]."""
    c = c.movedim(-1, -3)                                  # [..., w, h, i // 2, i % 2]
    return (c[..., 0] | (c[..., 1] << 4)).flatten(-3)


def _codes_of(b):
    """The inverse: bytes [..., 16] to codes [..., 32]."""
    b = b.unflatten(-1, (4, 2, 2))                         # [..., w, h, i // 2]
    c = torch.stack([b & 15, b >> 4], dim=-1)              # [..., w, h, i // 2, i % 2]
    return c.movedim(-3, -1).flatten(-4)


def _pack(k, v):
    """Cache pages [B, H, P, 32 D + 256] of rows [B, H, 32 P, D]."""
    B, H, R, D = k.shape
    P = R // PAGE
    (ck, sk, ok), (cv, sv, ov) = _quantise(k), _quantise(v)
    kb = _bytes_of(ck.view(B, H, P, PAGE, D // 32, 4, 2, 2, 2)).transpose(3, 4)      # [B, H, P, D / 32, 32, 16]
    vb = _bytes_of(cv.view(B, H, P, PAGE, D).transpose(3, 4).unflatten(-1, (4, 2, 2, 2)))   # [B, H, P, D, 16]
    sc = torch.stack([t.view(B, H, P, PAGE) for t in (sk, ok, sv, ov)], dim=3)
    return torch.cat([kb.flatten(3), vb.flatten(3), sc.flatten(3).contiguous().view(torch.uint8)], dim=3).contiguous()


def _unpack(cache, D):
    """Rows [B, H, 32 P, D] in fp32 of cache pages."""
    B, H, P, _ = cache.shape
    kb, vb, sc = cache.split([16 * D, 16 * D, 256], dim=3)
    sc = sc.contiguous().view(torch.bfloat16).view(B, H, P, 4, PAGE, 1).float()
    ck = _codes_of(kb.reshape(B, H, P, D // 32, PAGE, 16).transpose(3, 4)).flatten(-2)
    cv = _codes_of(vb.reshape(B, H, P, D, 16)).transpose(-1, -2)
    k = sc[:, :, :, 0] * (ck.float() + 16) + sc[:, :, :, 1]
    v = sc[:, :, :, 2] * (cv.float() + 16) + sc[:, :, :, 3]
    return k.reshape(B, H, P * PAGE, D), v.reshape(B, H, P * PAGE, D)


# ------------------------------------------------------------------ inputs

def _tree_tensors(tree):
    parent = _parents(tree)
    N = len(parent)
    see = np.zeros((N, N), dtype=bool)
    depth = np.zeros(N, dtype=np.int32)
    for n, p in enumerate(parent):
        if p >= 0:
            see[n] = see[p]
            depth[n] = depth[p] + 1
        see[n, n] = True
    words = (N + 63) // 64
    bits = np.zeros((N, words), dtype=np.uint64)
    for j in range(N):
        bits[:, j // 64] |= see[:, j].astype(np.uint64) << np.uint64(j % 64)
    ls = np.asarray(_levels(tree), dtype=np.int32)
    start = np.zeros(N + 1, dtype=np.int32)
    start[: len(ls)] = ls
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    return dict(anc=dev(bits.view(np.int64)), see=dev(see), depth=dev(depth), level_start=dev(start), level_start_host=ls,
                parent=dev(np.asarray(parent, dtype=np.int32)), N=N, levels=len(ls) - 1, roots=parent.count(-1), words=words)


def _rows(g, shape):
    """Key rows: a channel's own offset plus unit noise."""
    B, H, _, D = shape
    return torch.randn(shape, generator=g, device="cuda").add_(torch.randn((1, H, 1, D), generator=g, device="cuda"))


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    dt = _dtype(case)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    st = dict(case)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    if case["op"] == "attend":
        order = np.random.RandomState(seed).permutation(case["B"]).tolist()
        lens, act = _lens(case, order)
        t = _tree_tensors(case["tree"])
        B, Hq, Hkv, D, N = case["B"], case["Hq"], case["Hkv"], case["D"], t["N"]
        P = -(-case["L"] // PAGE)
        st.update(t, cache=_pack(_rows(g, (B, Hkv, P * PAGE, D)), rnd(B, Hkv, P * PAGE, D)),
                  q=rnd(B, Hq, N, D).to(dt), k_tree=_rows(g, (B, Hkv, N, D)).to(dt), v_tree=rnd(B, Hkv, N, D).to(dt),
                  out=torch.zeros((B, Hq, N, D), dtype=dt, device="cuda"), lens=i32(lens), act=i32(act) if case["sliced"] else None,
                  workspace=torch.zeros(96 << 20, dtype=torch.uint8, device="cuda"))
    elif case["op"] == "rope":
        t = _tree_tensors(case["tree"]) if case["tree"] else dict(N=case["T"], depth=None)
        B, Hq, Hkv, D, N = case["B"], case["Hq"], case["Hkv"], case["D"], t["N"]
        half = case["rot"] // 2
        x = rnd(B, N, Hq + 2 * Hkv, D).to(dt)              # a layer's fused projection
        st.update(t, x=x, parts=x.split([Hq, Hkv, Hkv], dim=2), lens=i32([max(0, case["pos"] - 3 * b) for b in range(B)]),
                  freqs=10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half),
                  wq=(1 + 0.1 * rnd(D)).to(dt) if case["norm"] else None, wk=(1 + 0.1 * rnd(D)).to(dt) if case["norm"] else None,
                  out=tuple(torch.zeros((B, h, N, D), dtype=dt, device="cuda") for h in (Hq, Hkv, Hkv)))
    elif case["op"] == "append":
        B, H, D, T = case["B"], case["H"], case["D"], case["T"]
        start = [case["start"] + 5 * b for b in range(B)]
        P = -(-(max(start) + T) // PAGE)
        st.update(k=_rows(g, (B, H, T, D)).to(dt), v=rnd(B, H, T, D).to(dt), start=i32(start),
                  cache=torch.zeros((B, H, P, 32 * D + 256), dtype=torch.uint8, device="cuda"))
        st["cache_ptrs"] = torch.tensor([st["cache"].data_ptr()], dtype=torch.int64, device="cuda")
        st["back"] = tuple(torch.zeros((1, B, H, T, D), dtype=dt, device="cuda") for _ in range(2))
    else:
        t = _tree_tensors(case["tree"])
        n, B, H, D, N = case["layers"], case["B"], case["H"], case["D"], t["N"]
        P = -(-(case["L"] + t["levels"] + 4) // PAGE)
        rs = np.random.RandomState(seed)
        accepted, nodes, ls = _accepted(case), np.full((B, t["levels"]), -1, dtype=np.int32), t["level_start_host"]
        for b, a in enumerate(accepted):
            for d in range(a):
                nodes[b, d] = rs.randint(ls[d + 1], ls[d + 2])
        st.update(t, k=rnd(n, B, H, N, D).to(dt), v=rnd(n, B, H, N, D).to(dt),
                  cache=torch.zeros((n, B, H, P, 32 * D + 256), dtype=torch.uint8, device="cuda"),
                  lens0=i32([max(0, case["L"] - 2 * b) for b in range(B)]), lens=i32([0] * B), count=i32([1 + a for a in accepted]),
                  verified=dict(accept_len=i32(accepted), out_nodes=i32(nodes.tolist()), best_root=i32([rs.randint(t["roots"]) for _ in range(B)])))
        for name in ("k", "v", "cache"):
            st[name + "_ptrs"] = torch.tensor([x.data_ptr() for x in st[name]], dtype=torch.int64, device="cuda")
        st["back"] = tuple(torch.zeros((n, B, H, t["levels"], D), dtype=dt, device="cuda") for _ in range(2))
    return st


# ------------------------------------------------------------------ one pass

def _mask(mcsd, st):
    return mcsd.TreeMask(st["anc"], st["depth"], st["level_start"], st["level_start_host"], st["parent"], st["N"], st["levels"], st["roots"], st["words"])


def run(st):
    if own:
        return _run_own(st)
    return {"attend": _attend, "rope": _rope, "append": _append, "commit": _commit}[st["op"]](st)


def _run_own(st):
    import paper_2409_10644_b200 as mcsd
    dt = torch.bfloat16 if st["dtype"] == "bf16" else torch.float32
    if st["op"] == "attend":
        return mcsd.mcsd_tree_attention_kv4(st["q"], st["cache"], st["k_tree"], st["v_tree"], st["lens"], st["act"], _mask(mcsd, st),
                                            out=st["out"], workspace=st["workspace"])
    if st["op"] == "rope":
        q, k, v = st["parts"]
        return mcsd.mcsd_qk_norm_rope(q, k, v, st["lens"], st["freqs"], depth=st["depth"], q_weight=st["wq"], k_weight=st["wk"],
                                      eps=1e-6, interleaved=st["interleaved"], out=st["out"])
    B, H, D, L_max = st["B"], st["H"], st["D"], st["cache"].shape[-2] * PAGE
    if st["op"] == "append":
        mcsd.mcsd_append_kv4(st["k"], st["v"], st["cache"], st["start"])
        return mcsd.mcsd_read_kv4(st["cache_ptrs"], st["start"], st["T"], None, B, H, D, L_max, dt, out=st["back"])
    st["lens"].copy_(st["lens0"])                          # every pass commits the same step
    mcsd.mcsd_commit_kv4(st["cache_ptrs"], st["k_ptrs"], st["v_ptrs"], st["lens"], st["verified"], _mask(mcsd, st), B, H, D, L_max, dt)
    back = mcsd.mcsd_read_kv4(st["cache_ptrs"], st["lens0"], st["levels"], st["count"], B, H, D, L_max, dt, out=st["back"])
    return back + (st["lens"],)


def _attend(st):
    B, Hq, Hkv, D, N = st["B"], st["Hq"], st["Hkv"], st["D"], st["N"]
    G = Hq // Hkv
    k, v = _unpack(st["cache"], D)
    k, v = torch.cat([k, st["k_tree"].float()], 2), torch.cat([v, st["v_tree"].float()], 2)
    rows = st["cache"].shape[2] * PAGE
    before = torch.arange(rows, device="cuda") < st["lens"].view(B, 1)
    see = torch.cat([before.view(B, 1, rows).expand(B, N, rows), st["see"].expand(B, N, N)], 2)
    s = torch.matmul(st["q"].float().reshape(B, Hkv, G * N, D), k.transpose(-1, -2)) / math.sqrt(D)
    s = s.view(B, Hkv, G, N, rows + N).masked_fill_(~see.view(B, 1, 1, N, rows + N), -math.inf)
    s = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.matmul(s.view(B, Hkv, G * N, rows + N), v).view(B, Hkv, G, N, D) / s.sum(-1, keepdim=True)
    o = o.view(B, Hq, N, D)
    if st["act"] is not None:                              # rows behind the active nodes stay as they were
        o = o * (torch.arange(N, device="cuda").view(1, 1, N, 1) < st["act"].view(B, 1, 1, 1))
    return o.to(st["q"].dtype)


def _rope(st):
    q, k, v = (x.float().transpose(1, 2) for x in st["parts"])
    step = torch.arange(st["N"], device="cuda") if st["depth"] is None else st["depth"]
    angle = (st["lens"].view(-1, 1, 1, 1) + step.view(1, 1, -1, 1)).double() * st["freqs"]
    cos, sin = angle.cos().float(), angle.sin().float()
    out = []
    for x, w in ((q, st["wq"]), (k, st["wk"])):
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        rot, rest = x[..., : st["rot"]], x[..., st["rot"]:]
        if st["interleaved"]:
            a, b = rot[..., 0::2], rot[..., 1::2]
            rot = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
        else:
            a, b = rot.chunk(2, dim=-1)
            rot = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
        out.append(torch.cat([rot, rest], dim=-1).to(st["x"].dtype))
    return (*out, v.to(st["x"].dtype))


def _stored(x):
    """What the cache gives back for rows x: the decision between two codes is taken in 64 bits."""
    c, s, o = _quantise(x.double())
    return (s.float() * (c.float() + 16) + o.float()).to(x.dtype)


def _append(st):
    return _stored(st["k"]).unsqueeze(0), _stored(st["v"]).unsqueeze(0)


def _commit(st):
    n, B, H, D, levels = st["layers"], st["B"], st["H"], st["D"], st["levels"]
    ver = st["verified"]
    node = torch.cat([ver["best_root"].view(B, 1), ver["out_nodes"]], 1)[:, :levels].clamp(min=0).long()
    there = torch.arange(levels, device="cuda").view(1, levels) < st["count"].view(B, 1)
    at = node.view(1, B, 1, levels, 1).expand(n, B, H, levels, D)
    k, v = (_stored(x.gather(3, at)) * there.view(1, B, 1, levels, 1) for x in (st["k"], st["v"]))
    return k, v, st["lens0"] + st["count"]


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    D = case["D"]
    row4 = D + 8                                           # a key and a value row in 4 bits, with their scales
    if case["op"] == "attend":
        lens, act = _lens(case, range(case["B"]))
        N = _nodes(case["tree"])
        pairs = sum(a * (n + a) for n, a in zip(lens, act))
        byt = sum(case["Hkv"] * (n * row4 + 2 * a * D * e) + 2 * case["Hq"] * a * D * e for n, a in zip(lens, act)) + N * ((N + 63) // 64) * 8
        return {"bytes": byt, "flops": 4 * D * case["Hq"] * pairs}
    if case["op"] == "rope":
        rows = case["B"] * (_nodes(case["tree"]) if case["tree"] else case["T"])
        return {"bytes": 2 * rows * (case["Hq"] + 2 * case["Hkv"]) * D * e, "flops": rows * (case["Hq"] + case["Hkv"]) * D * 7}
    if case["op"] == "append":
        rows = case["B"] * case["H"] * case["T"]
    else:
        rows = case["layers"] * case["B"] * case["H"] * (1 + sum(_accepted(case)) / case["B"])
    return {"bytes": rows * (2 * (2 * D * e) + 2 * row4), "flops": rows * 2 * D * 6}


# ------------------------------------------------------------------ the same from the definition, in 64 bits

def _exact_rows(words, scales, D):
    """Values [R, D] of one head's K or V codes: `words` int64 [R, D], the code of each value; scales bf16 (s, o) [R]."""
    s, o = scales
    return s.double().unsqueeze(-1) * (16 + words.double()) + o.double().unsqueeze(-1)


def _exact_cache(cache, D):
    """Keys and values of pages [H, P, bytes] in 64 bits, by the position of every code in its page."""
    H, P, _ = cache.shape
    r, d = torch.meshgrid(torch.arange(PAGE, device="cuda"), torch.arange(D, device="cuda"), indexing="ij")

    def code(byte0, e):                                    # value e (0..31) of the chunk at byte0
        w, i, h = e // 8, (e % 8) // 2, e % 2
        bit = 4 * i + 16 * h
        b = cache[:, :, (byte0 + 4 * w + bit // 8).flatten()].long()
        return ((b >> (bit % 8).flatten()) & 15).view(H, P, PAGE, D)

    ck, cv = code((d // 32) * (PAGE * 16) + r * 16, d % 32), code(16 * D + d * 16, r)
    sc = cache[:, :, 32 * D:].contiguous().view(torch.bfloat16)
    sk, ok, sv, ov = (sc[..., i * PAGE:(i + 1) * PAGE] for i in range(4))
    return _exact_rows(ck, (sk, ok), D).reshape(H, P * PAGE, D), _exact_rows(cv, (sv, ov), D).reshape(H, P * PAGE, D)


def _exact_store(x):
    x = x.double()
    lo, hi = x.min(-1).values, x.max(-1).values
    s = ((hi - lo) / 15).to(torch.bfloat16).double()
    o = (lo - 16 * s).to(torch.bfloat16).double()
    level = torch.arange(16, device="cuda", dtype=torch.float64)
    t = (x - o.unsqueeze(-1)) / s.unsqueeze(-1) - 16       # nearest of the sixteen levels; between two, the even one
    c = torch.where(s.unsqueeze(-1) > 0, torch.minimum(torch.maximum(torch.round(t), level[0]), level[15]), level[0])
    return s.unsqueeze(-1) * (16 + c) + o.unsqueeze(-1)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attend":
        G, D, N = case["Hq"] // case["Hkv"], case["D"], st["N"]
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        for b in range(case["B"]):
            L, a = int(st["lens"][b]), N if st["act"] is None else int(st["act"][b])
            ck, cv = _exact_cache(st["cache"][b], D)
            for h in range(case["Hkv"]):
                keys = torch.cat([ck[h, :L], st["k_tree"][b, h, :a].double()])
                vals = torch.cat([cv[h, :L], st["v_tree"][b, h, :a].double()])
                for j in range(h * G, h * G + G):
                    z = st["q"][b, j, :a].double() @ keys.T * (D ** -0.5)
                    z[:, L:][~st["see"][:a, :a]] = -math.inf
                    out[b, j, :a] = torch.softmax(z, -1) @ vals
        return out
    if case["op"] == "rope":
        depth = np.arange(st["N"]) if st["depth"] is None else st["depth"].cpu().numpy()
        pos = torch.from_numpy(st["lens"].cpu().numpy()[:, None].astype(np.float64) + depth).cuda()
        turn = torch.polar(torch.ones_like(pos).unsqueeze(-1), pos.unsqueeze(-1) * st["freqs"]).unsqueeze(1)
        out = []
        for x, w in zip(st["parts"], (st["wq"], st["wk"], None)):
            x = x.double().permute(0, 2, 1, 3).contiguous()
            if len(out) < 2:
                if w is not None:
                    x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["D"] + 1e-6) * w.double()
                half = case["rot"] // 2
                i = torch.arange(half, device="cuda")
                ia, ib = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
                z = torch.complex(x[..., ia], x[..., ib]) * turn
                x[..., ia], x[..., ib] = z.real, z.imag
            out.append(x)
        return tuple(out)
    if case["op"] == "append":
        return _exact_store(st["k"])[None], _exact_store(st["v"])[None]
    back = [torch.zeros(b.shape, dtype=torch.float64, device="cuda") for b in st["back"]]
    root, nodes = st["verified"]["best_root"].tolist(), st["verified"]["out_nodes"].tolist()
    for b, count in enumerate(st["count"].tolist()):
        for t in range(count):
            if t < st["levels"]:
                n = root[b] if t == 0 else nodes[b][t - 1]
                back[0][:, b, :, t], back[1][:, b, :, t] = _exact_store(st["k"][:, b, :, n]), _exact_store(st["v"][:, b, :, n])
    return back[0], back[1], None
