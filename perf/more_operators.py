"""Timed cases of the operators of a verification step whose target keeps one shared latent row a token: rows made from a
layer's projections, tree attention over a latent cache, accepted rows committed, and candidates drawn from filtered logits.

`run` computes an operator in its plain form from elementary torch operations, or, with `own`, through the library."""
import math

import numpy as np
import torch

own = False

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
        # one new token of one sequence, few heads: the call whose latency a user waits for
        dict(name="attend_token_b1", op="attend", dtype="bf16", B=1, H=16, R=512, P=64, tree="token", L=1001, ragged=False, sliced=False),
        # single tokens of a batch of long conversations, many heads
        dict(name="attend_token_b8_long", op="attend", dtype="bf16", B=8, H=128, R=512, P=64, tree="token", L=32001, ragged=True, sliced=False),
        # the repository's long-context workload: a 45-node tree per sequence
        dict(name="attend_tree_b16_4096", op="attend", dtype="bf16", B=16, H=32, R=512, P=64, tree="static", L=4096, ragged=False, sliced=False),
        # target-initialised forest, ragged prefixes, per-sequence slices
        dict(name="attend_forest_b32", op="attend", dtype="bf16", B=32, H=16, R=512, P=64, tree="forest", L=4096, ragged=True, sliced=True),
        # fp32 tensors and a narrow latent, a small checking workload
        dict(name="attend_fp32_r128", op="attend", dtype="f32", B=2, H=4, R=128, P=32, tree="binary", L=131, ragged=True, sliced=False),
        # one new token's projections
        dict(name="rows_token_b1", op="rows", dtype="bf16", B=1, H=16, R=512, P=64, tree="token", T=0, pos=1001, norm=True, interleaved=True),
        # a prompt's rows straight into the cache, far positions
        dict(name="rows_prompt_8191", op="rows", dtype="bf16", B=1, H=32, R=512, P=64, tree="", T=8191, pos=120000, norm=True, interleaved=False),
        # accepted rows of a small model's step
        dict(name="commit_l2_b4", op="commit", dtype="bf16", layers=2, B=4, R=512, P=64, tree="static", L=64),
        # accepted rows of all layers of a large batch
        dict(name="commit_l32_b32", op="commit", dtype="bf16", layers=32, B=32, R=512, P=64, tree="deep", L=64),
        # the four children of one node from a draft's logits: top-k and nucleus
        dict(name="sample_node_v32000", op="sample", dtype="bf16", rows=1, V=32000, K=4, temp=0.7, top_k=50, top_p=0.9, min_p=0.0, probs=True, greedy=False),
        # every node's row of the long-context workload, as verification takes them: probabilities under a wide nucleus
        dict(name="sample_rows720_v32000", op="sample", dtype="f32", rows=720, V=32000, K=4, temp=0.7, top_k=0, top_p=0.95, min_p=0.0, probs=True, greedy=False),
        # next tokens of a decoding batch over a large vocabulary of odd size, all filters, tokens only
        dict(name="sample_b16_v131071", op="sample", dtype="f32", rows=16, V=131071, K=1, temp=1.0, top_k=2000, top_p=0.95, min_p=0.02, probs=False, greedy=True),
    ]


def _span(rng, lo, hi):
    """A whole number whose logarithm is spread evenly over the range."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "sample", "sample", "rows", "commit"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "attend":
        small = dtype == "f32"
        R, P = rng.choice([(512, 64), (256, 64), (128, 32)]) if small else (512, 64)
        tree = rng.choice(sorted(TREES))
        while True:
            B, L = _span(rng, 1, 4 if small else 32), _span(rng, 1, 400 if small else 32768)
            H = rng.choice([2, 4, 5, 8]) if small else rng.choice([4, 8, 16, 20, 32, 64, 128])
            pairs = B * H * _nodes(tree) * (L + _nodes(tree))
            if pairs <= (2 * 4 * 15 * 400 * 16 if small else 16 * 32 * 45 * 4141) and B * L <= 8 * 32001:
                break
        return dict(op=op, dtype=dtype, B=B, H=H, R=R, P=P, tree=tree, L=L, ragged=rng.random() < 0.5, sliced=rng.random() < 0.5)
    R, P = rng.choice([(512, 64), (512, 64), (256, 64), (128, 32)])
    if op == "rows":
        c = dict(op=op, dtype=dtype, H=rng.choice([4, 16, 20, 32, 128]), R=R, P=P, pos=_span(rng, 1, 200000), norm=rng.random() < 0.7, interleaved=rng.random() < 0.5)
        if rng.random() < 0.5:
            return dict(c, tree=rng.choice(sorted(TREES)), T=0, B=_span(rng, 1, 16))
        return dict(c, tree="", T=_span(rng, 1, 2000), B=1)
    if op == "commit":
        return dict(op=op, dtype=dtype, layers=_span(rng, 1, 32), B=_span(rng, 1, 32), R=R, P=P, tree=rng.choice(sorted(t for t in TREES if TREES[t][1])), L=_span(rng, 1, 64))
    while True:
        rows, V = _span(rng, 1, 1024), _span(rng, 1000, 131072)
        if rows * V <= 720 * 32000:
            break
    return dict(op=op, dtype=dtype, rows=rows, V=V, K=rng.choice([0, 1, 2, 4, 8, 16]), temp=rng.choice([0.5, 0.7, 1.0, 1.3]),
                top_k=rng.choice([0, 0, 1, 20, 50, 400, 2000]), top_p=rng.choice([1.0, 0.5, 0.9, 0.95]), min_p=rng.choice([0.0, 0.0, 0.02, 0.1]),
                probs=True, greedy=rng.random() < 0.3)


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


def _clear_of_borders(case, g, logits):
    """Filter thresholds and uniforms per row that stay clear of the borders between two tokens: a nucleus' mass, the
    smallest relative weight and every uniform lie between the values at which an output would change."""
    rows, V, K = case["rows"], case["V"], case["K"]
    uni = lambda *s: torch.rand(s, generator=g, device="cuda", dtype=torch.float64)  # noqa: E731
    temp = torch.full((rows,), case["temp"], device="cuda") * (0.9 + 0.2 * uni(rows)).float()
    if case["greedy"]:
        temp[::3] = 0.0
    order = torch.sort(logits.double(), dim=-1, descending=True, stable=True)
    rel = (order.values - order.values[:, :1]) / torch.where(temp > 0, temp, torch.ones_like(temp)).double().unsqueeze(-1)
    w = rel.exp()
    kept = torch.full((rows, 1), V, device="cuda")
    top_k = top_p = min_p = None
    if case["top_k"] > 0:
        top_k = torch.randint(max(1, case["top_k"] // 2), case["top_k"] + 1, (rows,), generator=g, device="cuda", dtype=torch.int32)
        kept = torch.minimum(kept, top_k.long().unsqueeze(-1))
    c = (w * (torch.arange(V, device="cuda") < kept)).cumsum(-1)
    if case["top_p"] < 1.0:
        m = (c < case["top_p"] * (0.9 + 0.1 * uni(rows, 1)) * c[:, -1:]).sum(-1, keepdim=True)
        hi = c.gather(1, m)
        top_p = ((hi - 0.5 * w.gather(1, m)) / c[:, -1:]).float().squeeze(-1)
        kept = torch.minimum(kept, m + 1)
    if case["min_p"] > 0:
        want = math.log(case["min_p"]) + 0.5 * uni(rows, 1)
        first = (rel >= want).sum(-1, keepdim=True).clamp(min=1, max=V - 32)            # the widest gap near the wanted border
        at = first + torch.arange(32, device="cuda")
        gap = rel.gather(1, at - 1) - rel.gather(1, at)
        j = first + gap.argmax(-1, keepdim=True)
        min_p = torch.exp(0.5 * (rel.gather(1, j - 1) + rel.gather(1, j))).float().squeeze(-1)
        kept = torch.minimum(kept, j)
    kept = torch.where(temp.unsqueeze(-1) > 0, kept, torch.ones_like(kept))
    w = w * (torch.arange(V, device="cuda") < kept)
    c = torch.zeros_like(w).scatter_(1, order.indices, w).cumsum(-1)                    # by token id
    c = c / c[:, -1:]
    u = uni(rows, max(K, 1)).float()
    for last in [False] * 40 + [True]:
        hit = torch.searchsorted(c, u.double(), right=True).clamp(max=V - 1)
        lo = torch.where(hit > 0, c.gather(1, (hit - 1).clamp(min=0)), torch.zeros_like(u, dtype=torch.float64))
        hi = c.gather(1, hit)
        near = torch.minimum(torch.where(lo > 0, u.double() - lo, torch.ones_like(lo)), torch.where(hi < 1, hi - u.double(), torch.ones_like(lo))) < 4e-6
        best = order.indices[:, :1]
        middle = c.gather(1, best) - 0.5 * w[:, :1] / w.sum(-1, keepdim=True)
        u = torch.where(near, middle.float().expand_as(u) if last else uni(rows, max(K, 1)).float(), u)
    return dict(temp=temp, top_k=top_k, top_p=top_p, min_p=min_p, u=u[:, :K].contiguous() if K else None)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    st = dict(case)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    if case["op"] == "sample":
        rows, V = case["rows"], case["V"]
        logits = (3 * rnd(rows, V)).to(_dtype(case))
        st.update(_clear_of_borders(case, g, logits.float()), logits=logits)
        st["prob_out"] = torch.zeros((rows, V), device="cuda") if case["probs"] else None
        st["token_out"] = torch.zeros((rows, case["K"]), dtype=torch.int32, device="cuda") if case["K"] else None
        return st
    dt, R, P, B = _dtype(case), case["R"], case["P"], case["B"]
    W = R + P
    t = _tree_tensors(case["tree"]) if case["tree"] else dict(N=case["T"], depth=None)
    N = t["N"]
    if case["op"] == "attend":
        order = np.random.RandomState(seed).permutation(B).tolist()
        lens, act = _lens(case, order)
        st.update(t, cache=torch.empty((B, case["L"], W), dtype=dt, device="cuda"), tree_rows=rnd(B, N, W).to(dt),
                  q=rnd(B, case["H"], N, W).to(dt), out=torch.zeros((B, case["H"], N, R), dtype=dt, device="cuda"), lens=i32(lens),
                  act=i32(act) if case["sliced"] else None, scale=(128 + P) ** -0.5,     # heads of 128 values in front of the rotated part
                  workspace=torch.zeros(96 << 20, dtype=torch.uint8, device="cuda"))
        for b in range(B):
            st["cache"][b] = rnd(case["L"], W)
    elif case["op"] == "rows":
        H, pos = case["H"], [max(0, case["pos"] - 3 * b) for b in range(B)]
        start = [0] * B if case["tree"] else [(17 + 5 * b) for b in range(B)]            # a prompt goes behind what the cache holds
        half = P // 2
        st.update(t, latent=rnd(B, N, W).to(dt), q_in=rnd(B, N, H, 128 + P).to(dt),     # heads of 128 values and the part that is rotated
                  q=rnd(B, H, N, W).to(dt), rows=torch.zeros((B, N if case["tree"] else N + 64, W), dtype=dt, device="cuda"),
                  lens=i32(pos), start=None if case["tree"] else i32(start), start_host=start, weight=(1 + 0.1 * rnd(R)).to(dt) if case["norm"] else None,
                  freqs=10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half))
    else:
        n, L_max = case["layers"], case["L"] + t["levels"] + 4
        rs = np.random.RandomState(seed)
        accepted, nodes, ls = _accepted(case), np.full((B, t["levels"]), -1, dtype=np.int32), t["level_start_host"]
        for b, a in enumerate(accepted):
            for d in range(a):
                nodes[b, d] = rs.randint(ls[d + 1], ls[d + 2])
        st.update(t, tree_rows=rnd(n, B, N, W).to(dt), cache=rnd(n, B, L_max, W).to(dt), lens0=i32([max(0, case["L"] - 2 * b) for b in range(B)]),
                  lens=i32([0] * B), verified=dict(accept_len=i32(accepted), out_nodes=i32(nodes.tolist()), best_root=i32([rs.randint(t["roots"]) for _ in range(B)])))
        for name in ("tree_rows", "cache"):
            st[name + "_ptrs"] = torch.tensor([x.data_ptr() for x in st[name]], dtype=torch.int64, device="cuda")
    return st


# ------------------------------------------------------------------ one pass

def _mask(mcsd, st):
    return mcsd.TreeMask(st["anc"], st["depth"], st["level_start"], st["level_start_host"], st["parent"], st["N"], st["levels"], st["roots"], st["words"])


def run(st):
    if own:
        return _run_own(st)
    return {"attend": _attend, "rows": _rows, "commit": _commit, "sample": _sample}[st["op"]](st)


def _run_own(st):
    import paper_2409_10644_b200 as mcsd
    if st["op"] == "attend":
        return mcsd.mcsd_tree_attention_latent(st["q"], st["cache"], st["tree_rows"], st["lens"], st["act"], _mask(mcsd, st), softmax_scale=st["scale"],
                                               out=st["out"], workspace=st["workspace"])
    if st["op"] == "rows":
        mcsd.mcsd_latent_rows(st["latent"], st["q_in"][..., 128:], st["lens"], st["freqs"], rows=st["rows"], q=st["q"], row_start=st["start"],
                              depth=st["depth"], weight=st["weight"], eps=1e-6, interleaved=st["interleaved"])
        return st["rows"], st["q"]
    if st["op"] == "commit":
        st["lens"].copy_(st["lens0"])                      # every pass commits the same step
        mcsd.mcsd_commit_latent(st["cache_ptrs"], st["tree_rows_ptrs"], st["lens"], st["verified"], _mask(mcsd, st), st["B"], st["R"] + st["P"],
                                st["cache"].shape[2], st["cache"].dtype)
        return st["cache"], st["lens"]
    return mcsd.mcsd_sample_candidates(st["logits"], st["u"], temperature=st["temp"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"],
                                       probs=st["prob_out"], tokens=st["token_out"])


def _attend(st):
    B, H, N, R, rows = st["B"], st["H"], st["N"], st["R"], st["L"]
    k = torch.cat([st["cache"], st["tree_rows"]], 1).float()
    before = torch.arange(rows, device="cuda") < st["lens"].view(B, 1)
    see = torch.cat([before.view(B, 1, rows).expand(B, N, rows), st["see"].expand(B, N, N)], 2)
    s = torch.matmul(st["q"].float().reshape(B, H * N, -1), k.transpose(-1, -2)) * st["scale"]
    s = s.view(B, H, N, rows + N).masked_fill_(~see.view(B, 1, N, rows + N), -math.inf)
    s = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.matmul(s.view(B, H * N, rows + N), k[..., :R]).view(B, H, N, R) / s.sum(-1, keepdim=True)
    if st["act"] is not None:                              # rows behind the active nodes stay as they were
        o = o * (torch.arange(N, device="cuda").view(1, 1, N, 1) < st["act"].view(B, 1, 1, 1))
    return o.to(st["q"].dtype)


def _turn(x, cos, sin, interleaved):
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _rows(st):
    R, N = st["R"], st["N"]
    step = torch.arange(N, device="cuda") if st["depth"] is None else st["depth"]
    angle = (st["lens"].view(-1, 1, 1) + step.view(1, -1, 1)).double() * st["freqs"]
    cos, sin = angle.cos().float(), angle.sin().float()
    c, r = st["latent"].float().split([R, st["P"]], dim=-1)
    if st["weight"] is not None:
        c = c * torch.rsqrt((c * c).mean(-1, keepdim=True) + 1e-6) * st["weight"].float()
    new = torch.cat([c, _turn(r, cos, sin, st["interleaved"])], dim=-1).to(st["rows"].dtype)
    for b, s in enumerate(st["start_host"]):
        st["rows"][b, s:s + N] = new[b]
    st["q"][..., R:] = _turn(st["q_in"][..., 128:].float().transpose(1, 2), cos.unsqueeze(1), sin.unsqueeze(1), st["interleaved"]).to(st["q"].dtype)
    return st["rows"], st["q"]


def _commit(st):
    B, levels, ver = st["B"], st["levels"], st["verified"]
    L_max = st["cache"].shape[2]
    node = torch.cat([ver["best_root"].view(B, 1), ver["out_nodes"]], 1)[:, :levels].clamp(min=0).long()
    step = torch.arange(levels, device="cuda").view(1, levels)
    row = (st["lens0"].view(B, 1) + step).clamp(max=L_max - 1)
    there = ((step <= ver["accept_len"].view(B, 1)) & (st["lens0"].view(B, 1) + step < L_max)).view(1, B, levels, 1)
    at = torch.arange(B, device="cuda").view(B, 1)
    st["cache"][:, at, row] = torch.where(there, st["tree_rows"][:, at, node], st["cache"][:, at, row])
    st["lens"].copy_((st["lens0"] + 1 + ver["accept_len"]).clamp(max=L_max))
    return st["cache"], st["lens"]


def _sample(st):
    rows, V, K = st["rows"], st["V"], st["K"]
    temp = st["temp"].double().unsqueeze(-1)
    order = torch.sort(st["logits"].double(), dim=-1, descending=True, stable=True)
    w = torch.exp((order.values - order.values[:, :1]) / torch.where(temp > 0, temp, torch.ones_like(temp)))
    rank = torch.arange(V, device="cuda")
    keep = (temp > 0) | (rank < 1)
    if st["top_k"] is not None:
        keep = keep & (rank < st["top_k"].unsqueeze(-1))
    if st["top_p"] is not None:
        c = (w * keep).cumsum(-1)
        keep = keep & (c - w * keep < st["top_p"].double().unsqueeze(-1) * c[:, -1:])
    if st["min_p"] is not None:
        keep = keep & (w >= st["min_p"].double().unsqueeze(-1))
    p = torch.zeros_like(w).scatter_(1, order.indices, w * keep)
    out = []
    if K:
        c = p.cumsum(-1)
        out.append(torch.searchsorted(c, st["u"].double() * c[:, -1:], right=True).clamp(max=V - 1).int())
    if st["probs"]:
        out.append((p / p.sum(-1, keepdim=True)).float())
    return tuple(out)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["op"] == "sample":
        e = 2 if case["dtype"] == "bf16" else 4
        n = case["rows"] * case["V"]
        return {"bytes": n * (e + (4 if case["probs"] else 0)) + 8 * case["rows"] * (case["K"] + 2), "flops": 4 * n}
    e, R, P = 2 if case["dtype"] == "bf16" else 4, case["R"], case["P"]
    W = R + P
    if case["op"] == "attend":
        lens, act = _lens(case, range(case["B"]))
        pairs = sum(a * (n + a) for n, a in zip(lens, act))
        return {"bytes": e * sum((n + a) * W + case["H"] * a * (W + R) for n, a in zip(lens, act)), "flops": 2 * (W + R) * case["H"] * pairs}
    if case["op"] == "rows":
        rows = case["B"] * (_nodes(case["tree"]) if case["tree"] else case["T"])
        return {"bytes": 2 * e * rows * (W + case["H"] * P), "flops": rows * (4 * R + 3 * P * (1 + case["H"]))}
    rows = case["layers"] * sum(1 + a for a in _accepted(case))
    return {"bytes": 2 * e * rows * W, "flops": 0}


# ------------------------------------------------------------------ the same from the definition, in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attend":
        N, R, H = st["N"], case["R"], case["H"]
        out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
        for b in range(case["B"]):
            L, a = int(st["lens"][b]), N if st["act"] is None else int(st["act"][b])
            keys = torch.cat([st["cache"][b, :L], st["tree_rows"][b, :a]]).double()
            for h in range(H):
                z = st["q"][b, h, :a].double() @ keys.T * st["scale"]
                z[:, L:][~st["see"][:a, :a]] = -math.inf
                out[b, h, :a] = torch.softmax(z, -1) @ keys[:, :R]
        return out
    if case["op"] == "rows":
        depth = np.arange(st["N"]) if st["depth"] is None else st["depth"].cpu().numpy()
        pos = torch.from_numpy(st["lens"].cpu().numpy()[:, None].astype(np.float64) + depth).cuda()
        turn = torch.polar(torch.ones_like(pos).unsqueeze(-1), pos.unsqueeze(-1) * st["freqs"])
        i = torch.arange(case["P"] // 2, device="cuda")
        ia, ib = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + case["P"] // 2)

        def rotated(x, by):
            z = torch.complex(x[..., ia], x[..., ib]) * by
            x[..., ia], x[..., ib] = z.real, z.imag
            return x

        new = st["latent"].double()
        if st["weight"] is not None:
            c = new[..., : case["R"]]
            new[..., : case["R"]] = c / torch.sqrt(c.square().sum(-1, keepdim=True) / case["R"] + 1e-6) * st["weight"].double()
        new[..., case["R"]:] = rotated(new[..., case["R"]:].clone(), turn)
        rows, q = st["rows"].double(), st["q"].double()
        for b, s in enumerate(st["start_host"]):
            rows[b, s:s + st["N"]] = new[b]
        q[..., case["R"]:] = rotated(st["q_in"][..., 128:].double().permute(0, 2, 1, 3).contiguous(), turn.unsqueeze(1))
        return rows, q
    if case["op"] == "commit":
        cache, lens = st["cache"].double(), st["lens0"].tolist()
        root, nodes = st["verified"]["best_root"].tolist(), st["verified"]["out_nodes"].tolist()
        for b, a in enumerate(_accepted(case)):
            for t in range(1 + a):
                cache[:, b, lens[b] + t] = st["tree_rows"][:, b, root[b] if t == 0 else nodes[b][t - 1]].double()
        return cache, torch.tensor([n + 1 + a for n, a in zip(lens, _accepted(case))], dtype=torch.int32, device="cuda")
    tokens, probs = [], []
    for r in range(case["rows"]):
        x = st["logits"][r].double()
        T = float(st["temp"][r])
        if T > 0:
            p = torch.softmax(x / T, -1)
            if st["top_k"] is not None:                    # a value's place: how many are larger, or equal with a lower id
                by = torch.argsort(x, descending=True, stable=True)
                p[by[int(st["top_k"][r]):]] = 0
                p = p / p.sum()
            full = p.clone()
            if st["top_p"] is not None:
                by = torch.argsort(x, descending=True, stable=True)
                need = int((torch.cumsum(full[by], 0) < float(st["top_p"][r])).sum()) + 1
                p[by[need:]] = 0
            if st["min_p"] is not None:
                p[full < float(st["min_p"][r]) * full.max()] = 0
            p = p / p.sum()
        else:
            p = torch.zeros_like(x)
            p[int((x == x.max()).nonzero()[0])] = 1
        probs.append(p)
        if case["K"]:
            c = torch.cumsum(p, 0)
            tokens.append(((c.unsqueeze(0) <= st["u"][r].double().unsqueeze(1) * c[-1]).sum(-1)).clamp(max=case["V"] - 1).int())
    return (() if not case["K"] else (torch.stack(tokens),)) + ((torch.stack(probs),) if case["probs"] else ())
