"""Operators around the 4-bit cache in forms that the other tests leave out: several layers read at once, tree rows off 16-byte
boundaries committed, many random launches whose work is cut in many ways, how exact the prefix's products are."""
import numpy as np
import pytest
import torch

from mcsd_inputs import parent_array
from oracle import kv4_oracle as kv4
from oracle import mcsd_oracle as orc
from tests.helpers import to_np
from tests.test_kv4 import TREES, _attend, _noise_cache, _off_by_one, _problem, _rows, m  # noqa: F401  (m: the fixture)


def _i32(a):
    return None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")


def _largest_rows(D, dtype):
    """Rows that reach the largest magnitude the cache takes, on both sides, on one side, and once."""
    rng = np.random.default_rng(D)
    top = 2.0 ** 125 * (1 - 2.0 ** -8)                       # a bf16 number
    x = rng.uniform(-1, 1, size=(4, D)) * top
    x[1] = np.abs(x[1])
    x[2] = -top + 2.0 ** 110 * rng.uniform(size=D)
    x[3] *= 2.0 ** -60
    x[:, 5], x[0, 9] = top, -top
    return torch.from_numpy(x).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_the_oracle_holds_rows_up_to_the_stated_size(dtype, D):
    """Half a step of (hi - lo) / 15 plus the rounding of scale and offset, 2^-8 of 31 scale + |lo|."""
    for x in to_np(_largest_rows(D, dtype)).astype(np.float64):
        _, s, o, _, _ = kv4.quantise_row(x)
        assert np.isfinite([s, o]).all()
        assert np.abs(kv4.stored_row(x) - x).max() <= 0.5 * (x.max() - x.min()) / 15 + 2.0 ** -8 * (31 * s + np.abs(x.min()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_up_to_the_stated_size(m, dtype, D):  # noqa: F811
    x = _largest_rows(D, dtype).view(1, 1, 4, D).cuda()
    cache = m.new_kv4_cache(1, 1, 32, D, "cuda")
    m.mcsd_append_kv4(x, x, cache, _i32([0]))
    want = np.zeros((1, 1, 1, 32 * D + 256), dtype=np.uint8)
    for t, row in enumerate(to_np(x)[0, 0]):
        kv4.write_row(want, 0, 0, t, row, row)
    assert np.array_equal(cache.cpu().numpy(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_read_of_several_layers(m, dtype, D):  # noqa: F811
    rng = np.random.default_rng(D)
    layers, B, H, pages, T = 5, 3, 2, 3, 40
    caches_h = [_noise_cache(rng, B, H, pages, D) for _ in range(layers)]
    caches = [torch.from_numpy(c).cuda() for c in caches_h]
    first, n_rows = [0, 29, 90], [40, 7, 40]                 # the last runs over the end of the cache
    k, v = m.mcsd_read_kv4(m.layer_pointer_table(caches), _i32(first), T, _i32(n_rows), B, H, D, pages * 32, dtype)
    for i in range(layers):
        for got, rows in zip((k[i], v[i]), kv4.read_rows(caches_h[i], D)):
            for b in range(B):
                n = min(n_rows[b], pages * 32 - first[b])
                want = torch.from_numpy(rows[b, :, first[b]:first[b] + n].astype(np.float32)).to(dtype)
                assert torch.equal(got[b, :, :n].cpu(), want) and (got[b, :, n:] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_commit_of_rows_off_16_byte_boundaries(m, dtype, D):  # noqa: F811
    rng = np.random.default_rng(D + 1)
    parent = parent_array(1, (4, 2, 2, 1))
    tm = m.mcsd_build_mask(parent)
    layers, B, H, N, pages = 2, 3, 3, tm.n_nodes, 2
    start, accept = [5, 30, 62], [4, 3, 0]
    nodes = np.full((B, tm.n_levels), -1, dtype=np.int32)
    for b in range(B):
        for d in range(accept[b]):
            nodes[b, d] = rng.integers(tm.level_start_host[d + 1], tm.level_start_host[d + 2])
    ver = dict(accept_len=_i32(accept), out_nodes=_i32(nodes.tolist()), best_root=_i32([0] * B))
    kt, vt = ([_off_by_one(_rows(rng, (B, H, N, D), dtype)) for _ in range(layers)] for _ in range(2))
    caches_h = [_noise_cache(rng, B, H, pages, D) for _ in range(layers)]
    caches = [torch.from_numpy(c.copy()).cuda() for c in caches_h]
    lens = _i32(start)
    m.mcsd_commit_kv4(m.layer_pointer_table(caches), m.layer_pointer_table(kt), m.layer_pointer_table(vt), lens, ver, tm, B, H, D,
                      pages * 32, dtype)
    for c, ch, k, v in zip(caches, caches_h, kt, vt):
        new = kv4.commit(ch, to_np(k), to_np(v), start, accept, nodes, np.zeros(B, dtype=np.int32))
        assert np.array_equal(c.cpu().numpy(), ch)
    assert np.array_equal(lens.cpu().numpy(), new)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(24))
def test_random_launches_on_both_kernels(m, seed):  # noqa: F811
    """The tensor-core kernel cuts work items by cost at places that depend on every length; the CUDA-core kernel, which takes q
    off a 16-byte boundary, does not.  All rows of both have to be there and agree.

    The values lie around 1, so that A = sum w |v| is |result| up to a few per cent.  The tensor-core kernel rounds values, weights
    (in the products and in their sum) and result to u = 2^-8 each at most, 4 u; the other one its result, u; and scores of a
    few units in 32 bits add 2^-12 at most."""
    rng = np.random.default_rng(700 + seed)
    tree = sorted(TREES)[seed % len(TREES)]
    parent = parent_array(*TREES[tree])
    N = len(parent)
    B, (Hkv, G) = int(2 ** rng.uniform(0, 8)), [(1, 1), (8, 1), (2, 4), (1, 16), (3, 3), (32, 1)][seed % 6]
    most = int(min(20000, 2 ** rng.uniform(5, 15), 4e6 / (B * Hkv)))
    lens = [0 if rng.random() < 0.1 else int(rng.integers(0, most + 1)) for _ in range(B)]
    act = None if seed % 2 else [int(rng.integers(0, N + 1)) for _ in range(B)]
    g = torch.Generator("cuda").manual_seed(seed)
    rows = -(-max(lens + [1]) // 32) * 32
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    cache = m.new_kv4_cache(B, Hkv, rows, 128, "cuda")
    m.mcsd_append_kv4(rnd(B, Hkv, rows, 128), 1 + 0.2 * rnd(B, Hkv, rows, 128), cache, _i32([0] * B))
    q, kt, vt = (x.to(torch.bfloat16) for x in (rnd(B, Hkv * G, N, 128), rnd(B, Hkv, N, 128), 1 + 0.2 * rnd(B, Hkv, N, 128)))
    assert m.mcsd_tree_attention_path(B, Hkv * G, Hkv, N, 128, rows, m.MCSD_BF16) == 1
    tm = m.mcsd_build_mask(parent)
    got = _attend(m, q, cache, kt, vt, _i32(lens), _i32(act), tm)
    want = _attend(m, _off_by_one(q), cache, kt, vt, _i32(lens), _i32(act), tm)
    there = torch.ones(B, N, dtype=torch.bool, device="cuda")
    if act is not None:
        there = torch.arange(N, device="cuda") < _i32(act).view(B, 1)
    there = there.view(B, 1, N, 1).expand_as(q)
    assert torch.isnan(got[~there]).all() and torch.isfinite(got[there]).all()
    a, b = got[there].double(), want[there].double()
    assert ((a - b).abs() <= (5 * 2.0 ** -8 * 1.1 + 2.0 ** -12) * b.abs()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("tree,Hq,Hkv,L", [("token", 8, 2, 3000), ("static", 2, 1, 1500), ("forest", 2, 2, 1000)])
def test_prefix_products_keep_eleven_bits(m, tree, Hq, Hkv, L):  # noqa: F811
    """With values of ordinary size and scores of a few units, products over the prefix are made in fp16 (u' = 2^-11 for a value, a
    weight in the product and a weight in the sum), those over the tree in bf16 (u = 2^-8), and the result is rounded once.
    Scores: 2 (D + 4) 2^-23 S as for the other tests, and 2^-14 of the row's largest query against codes of at most 15 steps."""
    rng = np.random.default_rng(L)
    parent = parent_array(*TREES[tree])
    q, cache, cache_h, kt, vt = _problem(m, rng, torch.bfloat16, 1, Hq, Hkv, 128, parent, [L], None)
    out = to_np(_attend(m, q, cache, kt, vt, _i32([L]), None, m.mcsd_build_mask(parent))).astype(np.float64)
    kc, vc = kv4.read_rows(cache_h, 128)
    sc = (np.ascontiguousarray(cache_h[..., 32 * 128:]).view(np.uint16).astype(np.uint32) << 16).view(np.float32)
    sc = np.abs(sc.astype(np.float64)).reshape(1, Hkv, -1, 4, 32)
    qh, kh, vh = (to_np(x).astype(np.float64) for x in (q, kt, vt))
    see, scale, N = orc.dense_mask(parent), 128 ** -0.5, len(parent)
    for h in range(Hq):
        g = h // (Hq // Hkv)
        keys, vals = np.concatenate([kc[0, g, :L], kh[0, g]]), np.concatenate([vc[0, g, :L], vh[0, g]])
        z = qh[0, h] @ keys.T * scale
        z[:, L:][~see] = -np.inf
        w = np.exp(z - z.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        ref, pre, own = w @ vals, w[:, :L] @ np.abs(vals[:L]), w[:, L:] @ np.abs(vals[L:])
        steps, offs = sc[0, g, :, 0].reshape(-1)[:L], sc[0, g, :, 1].reshape(-1)[:L]
        size = np.abs(qh[0, h]).sum(-1, keepdims=True) * max((31 * steps + offs).max(), np.abs(kh[0, g]).max()) * scale
        split = 2.0 ** -14 * np.abs(qh[0, h]).max(-1, keepdims=True) * scale * 15 * 128 * steps.max()
        weight = 2 * (2 * 132 * 2.0 ** -23 * size + split + 2.0 ** -21) + (L + N + 8) * 2.0 ** -23
        # a weight's rounding counts with its value and, through the sum, with the result
        tree_share = w[:, L:].sum(-1, keepdims=True)
        tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -11 * (2 * pre + np.abs(ref)) + 2.0 ** -8 * (2 * own + tree_share * np.abs(ref)) + weight * (pre + own)
        err = np.abs(out[0, h] - ref)
        assert (err <= tol).all(), (h, (err / tol).max())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["usual", "peaked", "a dominant key", "rows of different size"])
@pytest.mark.parametrize("tree,B,Hq,Hkv,L", [("token", 2, 8, 2, 9000), ("static", 4, 8, 8, 1500), ("forest", 6, 4, 4, 700)])
def test_repeated_calls_are_equal_to_the_bit(m, kind, tree, B, Hq, Hkv, L):  # noqa: F811
    """Whichever form a tile takes (fp16 or bf16 weights, split or bf16 queries), timing has no part in it."""
    g = torch.Generator("cuda").manual_seed(L)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    parent = parent_array(*TREES[tree])
    N = len(parent)
    k, q = rnd(B, Hkv, L, 128), rnd(B, Hq, N, 128)
    if kind == "peaked":
        q *= 6
    elif kind == "a dominant key":
        q = q * 0.3 + 1
        k[:, :, L // 3] = 20 / 128 ** 0.5
    elif kind == "rows of different size":
        q[:, ::2, ::3] *= 2.0 ** -9
    cache = m.new_kv4_cache(B, Hkv, L, 128, "cuda")
    m.mcsd_append_kv4(k, rnd(B, Hkv, L, 128), cache, _i32([0] * B))
    q, kt, vt = (x.to(torch.bfloat16) for x in (q, rnd(B, Hkv, N, 128), rnd(B, Hkv, N, 128)))
    tm, lens = m.mcsd_build_mask(parent), _i32([L - 37 * b for b in range(B)])
    want = _attend(m, q, cache, kt, vt, lens, None, tm)
    ws = m.new_workspace(m.mcsd_tree_attention_kv4_workspace_bytes(B, Hq, Hkv, N, 128, cache.shape[2] * 32, m.MCSD_BF16), "cuda")
    outs = [torch.empty_like(q) for _ in range(30)]
    for out in outs:                                         # back to back
        m.mcsd_tree_attention_kv4(q, cache, kt, vt, lens, None, tm, out=out, workspace=ws)
    assert all(torch.equal(out, want) for out in outs) and torch.isfinite(want).all()


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.1, 0.01, 0.5])
@pytest.mark.parametrize("zeros", ["none", "some rows", "all rows"])
def test_scales_and_rows_of_zeros_on_both_kernels(m, scale, zeros):  # noqa: F811
    """Any softmax scale, queries of zeros alone and beside others; bounds as for the random launches, the scores' part for
    scores of up to a hundred (2 (D + 4) 2^-23 S twice, with S below 400: 2^-5 in a weight; none for scales up to a tenth)."""
    g = torch.Generator("cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    parent = parent_array(*TREES["static"])
    N, B, Hq, Hkv, L = len(parent), 2, 4, 2, 600
    q = rnd(B, Hq, N, 128)
    if zeros != "none":
        q[:, :, ::2 if zeros == "some rows" else 1] = 0
    cache = m.new_kv4_cache(B, Hkv, L, 128, "cuda")
    m.mcsd_append_kv4(rnd(B, Hkv, L, 128), 1 + 0.2 * rnd(B, Hkv, L, 128), cache, _i32([0] * B))
    q, kt, vt = (x.to(torch.bfloat16) for x in (q, rnd(B, Hkv, N, 128), 1 + 0.2 * rnd(B, Hkv, N, 128)))
    tm, lens = m.mcsd_build_mask(parent), _i32([L, 129])
    got, want = (m.mcsd_tree_attention_kv4(x, cache, kt, vt, lens, None, tm, softmax_scale=scale).double() for x in (q, _off_by_one(q)))
    bound = 5 * 2.0 ** -8 * 1.1 + 2.0 ** -12 + (2.0 ** -5 if scale > 0.1 else 0)
    assert torch.isfinite(got).all() and ((got - want).abs() <= bound * want.abs()).all()
