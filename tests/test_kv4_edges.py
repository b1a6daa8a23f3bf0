"""Attention over the 4-bit cache where one call, row or key could disturb another: a workspace that several kernels use in
turn, a key that outweighs the others by far, queries of very different size side by side."""
import numpy as np
import pytest
import torch

from mcsd_inputs import parent_array
from oracle import kv4_oracle as kv4
from oracle import mcsd_oracle as orc
from tests.helpers import to_np
from tests.test_kv4 import TREES, _attend, _check_attention, _off_by_one, _problem, m  # noqa: F401  (m: the fixture)


def _i32(a):
    return None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------------------------- one workspace, several kernels

def _dense(m, q, k_cache, v_cache, kt, vt, lens, tm, ws):
    out = torch.full_like(q, float("nan"))
    m.mcsd_tree_attention(q, k_cache, v_cache, kt, vt, lens, None, tm, out=out, workspace=ws)
    assert m.mcsd_workspace_status(ws) == 0
    return out


@pytest.mark.gpu
def test_one_workspace_for_both_types_both_kernels_and_both_caches(m):  # noqa: F811
    """What one call leaves in a workspace is nothing to the next: every call as with a workspace of its own, to the bit."""
    rng = np.random.default_rng(31)
    parent = parent_array(*TREES["static"])
    tm, lens = m.mcsd_build_mask(parent), [4096]
    L = _i32(lens)
    q, cache, cache_h, kt, vt = _problem(m, rng, torch.float32, 1, 32, 32, 128, parent, lens, None)
    h = [x.to(torch.bfloat16) for x in (q, kt, vt)]
    dense = m.mcsd_read_kv4(m.layer_pointer_table([cache]), _i32([0]), 4096, None, 1, 32, 128, cache.shape[2] * 32, torch.bfloat16)
    dense = [x[0] for x in dense]
    assert m.mcsd_tree_attention_path(1, 32, 32, len(parent), 128, cache.shape[2] * 32, m.MCSD_BF16) == 1
    calls = {
        "fp32": lambda ws: _attend(m, q, cache, kt, vt, L, None, tm, ws),
        "bf16": lambda ws: _attend(m, h[0], cache, h[1], h[2], L, None, tm, ws),
        "bf16 off a 16-byte boundary": lambda ws: _attend(m, _off_by_one(h[0]), cache, h[1], h[2], L, None, tm, ws),
        "dense": lambda ws: _dense(m, h[0], *dense, h[1], h[2], L, tm, ws),
        "dense off a 16-byte boundary": lambda ws: _dense(m, _off_by_one(h[0]), *dense, h[1], h[2], L, tm, ws),
    }
    size = 64 << 20
    want = {name: call(torch.zeros(size, dtype=torch.uint8, device="cuda")) for name, call in calls.items()}
    _check_attention(want["bf16"], h[0], cache_h, h[1], h[2], lens, None, parent, heads=[0, 13, 31])
    _check_attention(want["fp32"], q, cache_h, kt, vt, lens, None, parent, heads=[0, 31])
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    order = ["fp32", "bf16", "bf16", "bf16 off a 16-byte boundary", "bf16", "dense", "bf16", "dense off a 16-byte boundary", "bf16",
             "dense", "fp32", "dense"]
    for i, name in enumerate(order):
        assert torch.equal(calls[name](ws), want[name]), (i, name)


@pytest.mark.gpu
@pytest.mark.parametrize("tree", ["token", "static", "forest"])
def test_a_workspace_full_of_another_calls_scratch(m, tree):  # noqa: F811
    """All of the scratch, from its start to the end of the largest layout, holds floats of a call on the CUDA cores."""
    rng = np.random.default_rng(32)
    wide, parent = parent_array(*TREES["chain"])[:24], parent_array(*TREES[tree])
    tw, tm, lens = m.mcsd_build_mask(wide), m.mcsd_build_mask(parent), [900, 5000]
    q = torch.randn(36, 32, 24, 128, device="cuda")
    cache = m.new_kv4_cache(36, 32, 128, 128, "cuda")
    size = m.mcsd_tree_attention_kv4_workspace_bytes(36, 32, 32, 24, 128, cache.shape[2] * 32, m.MCSD_F32)
    for f, heads in ((m.mcsd_tree_attention_workspace_bytes, (8,)), (m.mcsd_tree_attention_kv4_workspace_bytes, (8, 2))):
        assert size > f(2, *heads, len(parent), 128, 5024, m.MCSD_BF16)
    h, cache2, _, kt2, vt2 = _problem(m, rng, torch.bfloat16, 2, 8, 2, 128, parent, lens, None)
    rows = m.mcsd_read_kv4(m.layer_pointer_table([cache2]), _i32([0, 0]), 5000, None, 2, 2, 128, cache2.shape[2] * 32, torch.bfloat16)
    ws, fresh = (torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2))
    four = lambda ws: _attend(m, h, cache2, kt2, vt2, _i32(lens), None, tm, ws)  # noqa: E731
    dense = lambda ws: _dense(m, h, rows[0][0], rows[1][0], kt2, vt2, _i32(lens), tm, ws)  # noqa: E731
    for call in (four, dense):
        want = call(fresh)
        for _ in range(2):
            _attend(m, q, cache, q, q, _i32([128] * 36), None, tw, ws)
            got = call(ws)
            assert torch.equal(got.nan_to_num(7), want.nan_to_num(7)) and not torch.isnan(got[0]).any()


# ---------------------------------------------------------------------------------------------- one key outweighs the others

def _stored_cache(m, k, v):
    """A 4-bit cache of rows k, v [B][H][T][D] and its bytes."""
    B, H, T, D = k.shape
    cache = m.new_kv4_cache(B, H, T, D, "cuda")
    m.mcsd_append_kv4(k, v, cache, _i32([0] * B))
    return cache, cache.cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("tree", ["token", "static", "forest"])
@pytest.mark.parametrize("sink", [0, 70, 700])
@pytest.mark.parametrize("nats", [10.0, 14.0, 16.0, 22.0, 40.0, 60.0])
def test_keys_far_below_a_dominant_one(m, tree, sink, nats):  # noqa: F811
    """One key (the first of all, or one that no first guess of the row's maximum looks at) outweighs all others by up to e^60, and its
    value is zero, so the result is what the others give: their weights have to keep their relative precision.

    Tolerance per element, u = 2^-8 half a step of bf16 (no product is made of coarser numbers): the result's rounding,
    u |ref|; values, u A with A = sum w |v|; weights, in the products and in the row's sum, 2 u A, since the dominant weight
    is a power of two times its fp32 value in both; the fp32 parts as in _check_attention, whose bounds on scores hold here too."""
    rng = np.random.default_rng(int(nats) + sink)
    parent = parent_array(*TREES[tree])
    N, B, H, D, T = len(parent), 2, 20, 128, 992
    tm, lens = m.mcsd_build_mask(parent), [960, 933]
    way = rng.choice([-1.0, 1.0], size=D)
    q = way + 0.05 * rng.normal(size=(B, H, N, D))
    k = 0.3 * rng.normal(size=(B, H, T, D))
    v = 1.0 + 0.3 * rng.normal(size=(B, H, T, D))
    k[:, :, sink] = way * nats / D ** 0.5                    # score: nats, give or take
    v[:, :, sink] = 0
    kt, vt = 0.3 * rng.normal(size=(B, H, N, D)), 1.0 + 0.3 * rng.normal(size=(B, H, N, D))
    cuda = lambda x, t: torch.from_numpy(x).to("cuda", t)  # noqa: E731
    cache, cache_h = _stored_cache(m, cuda(k, torch.float32), cuda(v, torch.float32))
    q, kt, vt = (cuda(x, torch.bfloat16) for x in (q, kt, vt))
    out = to_np(_attend(m, q, cache, kt, vt, _i32(lens), None, tm)).astype(np.float64)

    kc, vc = kv4.read_rows(cache_h, D)
    assert (vc[:, :, sink] == 0).all()
    qh, kh, vh = (to_np(x).astype(np.float64) for x in (q, kt, vt))
    see, u = orc.dense_mask(parent), 2.0 ** -8
    for b in range(B):
        for g in range(H):
            keys, vals = np.concatenate([kc[b, g, :lens[b]], kh[b, g]]), np.concatenate([vc[b, g, :lens[b]], vh[b, g]])
            z = qh[b, g] @ keys.T * D ** -0.5
            z[:, lens[b]:][~see] = -np.inf
            w = np.exp(z - z.max(-1, keepdims=True))
            assert (z.argmax(-1) == sink).all()
            w /= w.sum(-1, keepdims=True)
            ref, A = w @ vals, w @ np.abs(vals)
            S = (np.abs(qh[b, g]) @ (2 * np.abs(keys).max(-1)[:, None] * np.ones((1, D))).T * D ** -0.5).max(-1, keepdims=True)
            weight = 2 * (2 * (D + 4) * 2.0 ** -23 * S + 2.0 ** -21) + (lens[b] + N + 8) * 2.0 ** -23
            tol = u * np.abs(ref) + 3 * u * A + weight * A
            err = np.abs(out[b, g] - ref)
            assert (err <= tol).all(), (b, g, (err / tol).max(), (err / np.abs(ref)).max())


# ---------------------------------------------------------------------------------------------- queries of different size

def _row_errors(out, q, cache_h, kt, vt, lens, parent, rows):
    """Largest error over its bound for the named query rows (head, node), each against the definition for that row alone.

    u = 2^-8.  Result, values and weights are rounded to at most u each (weights in the products and in their sum: 2 u A).  A
    score is off by the fp32 sums, 2 (D + 4) 2^-23 S as in _check_attention, and by the split of the row's queries: at
    most 2^-14 of the row's own largest element, against codes of at most 15 steps."""
    B, H, N, D = q.shape
    G, u, scale = H // kt.shape[1], 2.0 ** -8, D ** -0.5
    kc, vc = kv4.read_rows(cache_h, D)
    sc = (np.ascontiguousarray(cache_h[..., 32 * D:]).view(np.uint16).astype(np.uint32) << 16).view(np.float32)
    sc = np.abs(sc.astype(np.float64)).reshape(B, H // G, -1, 4, 32)
    qh, kh, vh, o = (to_np(x).astype(np.float64) for x in (q, kt, vt, out))
    worst = 0.0
    for b in range(B):
        n = lens[b]
        for h, r in rows:
            g = h // G
            see = orc.dense_mask(parent)[r]
            keys, vals = np.concatenate([kc[b, g, :n], kh[b, g][see]]), np.concatenate([vc[b, g, :n], vh[b, g][see]])
            steps, offs = sc[b, g, :, 0].reshape(-1)[:n], sc[b, g, :, 1].reshape(-1)[:n]
            x = qh[b, h, r]
            z = keys @ x * scale
            w = np.exp(z - z.max())
            w /= w.sum()
            ref, A = w @ vals, w @ np.abs(vals)
            S = scale * max((np.abs(x).sum() * (31 * steps + offs)).max(), (np.abs(kh[b, g][see]) @ np.abs(x)).max())
            split = 2.0 ** -14 * np.abs(x).max() * scale * 15 * D * steps.max()
            weight = 2 * (2 * (D + 4) * 2.0 ** -23 * S + split + 2.0 ** -21) + (n + N + 8) * 2.0 ** -23
            tol = u * np.abs(ref) + 3 * u * A + weight * A
            assert np.isfinite(o[b, h, r]).all(), (b, h, r)
            err = np.abs(o[b, h, r] - ref)
            worst = max(worst, np.divide(err, tol, out=np.where(err > 0, np.inf, 0.0), where=tol > 0).max())
    return worst


def _scaled_keys(m, cache, kt, T, factor):
    """The cache's first T rows with their keys times factor, its bytes, and the tree's keys likewise."""
    B, H, N, D = kt.shape
    k, v = m.mcsd_read_kv4(m.layer_pointer_table([cache]), _i32([0] * B), T, None, B, H, D, cache.shape[2] * 32, torch.float32)
    cache, cache_h = _stored_cache(m, k[0] * factor, v[0])
    return cache, cache_h, kt * factor


@pytest.mark.gpu
@pytest.mark.parametrize("tree,Hq,Hkv", [("token", 8, 1), ("static", 2, 2), ("binary", 8, 2), ("forest", 1, 1)])
@pytest.mark.parametrize("power", [-16, -12, -8, -4, -2, 10, 16])
def test_rows_of_very_different_size_in_one_work_item(m, tree, Hq, Hkv, power):  # noqa: F811
    """Every other query row (node and head) is 2^power times the others: each row's error is bounded by its own size."""
    rng = np.random.default_rng(40 + power)
    parent = parent_array(*TREES[tree])
    lens = [500, 300]
    q, cache, cache_h, kt, vt = _problem(m, rng, torch.bfloat16, 2, Hq, Hkv, 128, parent, lens, None)
    rows = [(h, r) for h in range(Hq) for r in range(len(parent))]
    for h, r in rows:
        if (h + r) % 2:
            q[:, h, r] *= 2.0 ** power
    if power < 0:                                            # scores of the small rows are of order one all the same
        cache, cache_h, kt = _scaled_keys(m, cache, kt, 512, 2.0 ** -power)
    out = _attend(m, q, cache, kt, vt, _i32(lens), None, m.mcsd_build_mask(parent))
    assert _row_errors(out, q, cache_h, kt, vt, lens, parent, rows) <= 1


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("tree,Hq,Hkv", [("token", 8, 1), ("static", 2, 2), ("binary", 8, 2)])
@pytest.mark.parametrize("size", [2.0 ** -6, 2.0 ** 11])
def test_a_row_that_is_not_finite_leaves_the_others_alone(m, tree, Hq, Hkv, bad, size):  # noqa: F811
    rng = np.random.default_rng(50)
    parent = parent_array(*TREES[tree])
    lens = [700, 129]
    q, cache, cache_h, kt, vt = _problem(m, rng, torch.bfloat16, 2, Hq, Hkv, 128, parent, lens, None)
    cache, cache_h, kt = _scaled_keys(m, cache, kt, 704, 1 / size)
    q *= size
    q[:, 0, 0, 5] = bad
    rows = [(h, r) for h in range(Hq) for r in range(len(parent)) if (h, r) != (0, 0)]
    out = _attend(m, q, cache, kt, vt, _i32(lens), None, m.mcsd_build_mask(parent))
    assert _row_errors(out, q, cache_h, kt, vt, lens, parent, rows) <= 1
