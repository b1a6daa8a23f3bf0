"""The 4-bit prefix cache: rows appended, committed and read back (bytes equal to the oracle's), tree attention over it
(against the definition in 64 bits on what the codes stand for), a generation loop of all of it, and refusals."""
import ctypes

import numpy as np
import pytest
import torch

from mcsd_inputs import parent_array
from oracle import kv4_oracle as kv4
from oracle import mcsd_oracle as orc
from tests.helpers import to_np

FAKE = ctypes.c_void_p(0x1000)      # never dereferenced: every call that uses it fails its checks first


@pytest.fixture(scope="module")
def m():
    from paper_2409_10644_b200 import build
    build.build()
    import paper_2409_10644_b200 as pkg
    return pkg


# ---------------------------------------------------------------------------------------------- refusals (host only)

def test_cache_sizes(m):
    assert m.mcsd_kv4_cache_bytes(2, 4, 128, 96) == 2 * 4 * 3 * (32 * 128 + 256)
    assert m.mcsd_kv4_cache_bytes(1, 1, 64, 32) == 32 * 64 + 256
    for bad in ((0, 4, 128, 32), (2, 0, 128, 32), (2, 4, 96, 32), (2, 4, 128, 33), (2, 4, 128, 0), (256, 256, 128, 32)):
        assert m.mcsd_kv4_cache_bytes(*bad) == 0
    with pytest.raises(ValueError):
        m.new_kv4_cache(1, 1, 64, 96, "cpu")


def test_append_and_read_refusals(m):
    def append(k=FAKE, cache=FAKE, start=FAKE, B=2, H=2, T=5, D=128, Lm=64, dtype=0):
        return m.lib.mcsd_append_kv4(k, FAKE, cache, start, None, B, H, T, D, Lm, dtype, None)
    assert append(k=None) == -1
    assert append(cache=None) == -1
    assert append(start=None) == -1
    assert append(dtype=3) == -4
    assert append(T=0) == -2
    assert append(D=80) == -2
    assert append(Lm=40) == -2
    assert append(Lm=0) == -2
    assert append(B=400, H=400) == -2
    assert append(cache=ctypes.c_void_p(0x1008)) == -2

    def read(c=FAKE, nl=1, first=FAKE, T=5, D=128, Lm=64, dtype=0, k=FAKE):
        return m.lib.mcsd_read_kv4(c, nl, first, None, 2, 2, T, D, Lm, dtype, k, FAKE, None)
    assert read(c=None) == -1
    assert read(first=None) == -1
    assert read(k=None) == -1
    assert read(nl=0) == -2
    assert read(nl=70000) == -2
    assert read(T=0) == -2
    assert read(Lm=31) == -2
    assert read(dtype=9) == -4


def test_commit_refusals(m):
    def call(c=FAKE, nl=2, lens=FAKE, levels=4, B=2, H=2, N=15, D=64, Lm=64, dtype=1):
        return m.lib.mcsd_commit_kv4(c, FAKE, FAKE, nl, lens, FAKE, FAKE, FAKE, levels, B, H, N, D, Lm, dtype, None)
    assert call(c=None) == -1
    assert call(lens=None) == -1
    assert call(nl=0) == -2
    assert call(levels=0) == -2
    assert call(levels=16) == -2
    assert call(N=193) == -2
    assert call(D=96) == -2
    assert call(Lm=65) == -2
    assert call(dtype=5) == -4


def test_attention_refusals(m):
    ws = m.mcsd_tree_attention_kv4_workspace_bytes
    assert ws(1, 8, 2, 15, 128, 128, m.MCSD_BF16) >= 256
    assert ws(1, 8, 3, 15, 128, 128, m.MCSD_BF16) == 0
    assert ws(1, 8, 2, 15, 128, 100, m.MCSD_BF16) == 0
    assert ws(1, 8, 2, 193, 128, 128, m.MCSD_BF16) == 0

    def call(q=FAKE, cache=FAKE, anc=FAKE, words=1, B=1, Hq=8, Hkv=2, N=15, D=128, Lm=128, dtype=0, w=FAKE, wsb=1 << 30):
        return m.lib.mcsd_tree_attention_kv4(q, cache, FAKE, FAKE, FAKE, FAKE, None, anc, words, B, Hq, Hkv, N, D, Lm,
                                             ctypes.c_float(0.1), dtype, w, wsb, None)
    assert call(q=None) == -1
    assert call(cache=None) == -1
    assert call(anc=None) == -1
    assert call(w=None) == -1
    assert call(Hkv=3) == -2
    assert call(Hkv=0) == -2
    assert call(Hq=2, Hkv=4) == -2
    assert call(Lm=0) == -2
    assert call(Lm=100) == -2
    assert call(words=0) == -2
    assert call(words=4) == -2
    assert call(N=65) == -2                                  # needs two mask words
    assert call(N=193, words=3) == -2
    assert call(D=256) == -2
    assert call(dtype=2) == -4
    assert call(wsb=128) == -5
    assert call(w=ctypes.c_void_p(0x1010)) == -2
    assert call(cache=ctypes.c_void_p(0x1008)) == -2


def test_binding_refuses_tensors_it_cannot_pass_on(m):
    k = torch.zeros(1, 2, 5, 128, dtype=torch.bfloat16)
    cache = torch.zeros(1, 2, 2, 32 * 128 + 256, dtype=torch.uint8)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        m.mcsd_append_kv4(k, k, cache, i)                    # not on a GPU
    with pytest.raises(ValueError):
        m.mcsd_append_kv4(k.half(), k.half(), cache, i)
    tm = m.TreeMask(torch.zeros(5, 1, dtype=torch.int64), i, i, np.zeros(2, dtype=np.int32), i, 5, 1, 1, 1)
    with pytest.raises(ValueError):
        m.mcsd_tree_attention_kv4(k, cache, k, k, i, None, tm)
    with pytest.raises(ValueError):
        m.mcsd_tree_attention_kv4(k[:, :, :4], cache, k, k, i, None, tm)


def test_oracle_rows_come_back_within_half_a_step():
    """The oracle itself: codes lie in 0..15, a stored row is within half a step plus the rounding of scale and offset."""
    rng = np.random.default_rng(0)
    for scale, shift in ((1.0, 0.0), (1e-3, 5.0), (1e4, -3e4), (1.0, 100.0)):
        for D in (64, 128):
            x = rng.normal(size=D) * scale + shift
            codes, s, o, _, _ = kv4.quantise_row(x)
            assert codes.min() >= 0 and codes.max() <= 15
            bound = 0.5 * s + 2.0 ** -8 * (31 * s + np.abs(x).max())
            assert np.abs(kv4.stored_row(x) - x).max() <= bound
    assert (kv4.stored_row(np.full(64, 3.0)) == 3.0).all()
    cache = rng.integers(0, 256, size=(1, 1, 2, 32 * 64 + 256)).astype(np.uint8)
    cache[..., 32 * 64:] = 0
    before = cache.copy()
    x, y = rng.normal(size=64), rng.normal(size=64)
    kv4.write_row(cache, 0, 0, 37, x, y)
    k, v = kv4.read_rows(cache, 64)
    assert np.array_equal(k[0, 0, 37], kv4.stored_row(x)) and np.array_equal(v[0, 0, 37], kv4.stored_row(y))
    kb, vb = kv4.read_rows(before, 64)
    others = [r for r in range(64) if r != 37]
    assert np.array_equal(k[:, :, others], kb[:, :, others]) and np.array_equal(v[:, :, others], vb[:, :, others])


# ---------------------------------------------------------------------------------------------- rows in and out

def _rows(rng, shape, dtype):
    x = rng.normal(size=shape) + rng.normal(size=shape[:-2] + (1, shape[-1]))
    return torch.from_numpy(x).to("cuda", dtype)


def _noise_cache(rng, B, H, pages, D):
    """A cache full of other rows: any codes, finite scales."""
    c = rng.integers(0, 256, size=(B, H, pages, 32 * D + 256)).astype(np.uint8)
    sc, _ = kv4.to_bf16(rng.uniform(0.01, 0.5, size=(B, H, pages, 128)))
    bits = sc.astype(np.float32).view(np.uint32) >> 16
    c[..., 32 * D:] = bits.astype(np.uint16).view(np.uint8).reshape(B, H, pages, 256)
    return c


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 5, 31, 32, 33, 100])
def test_append_writes_the_oracles_bytes_and_no_others(m, dtype, D, T):
    rng = np.random.default_rng(T + D)
    B, H, pages = 4, 2, 4
    start = [0, 17, 32, 95]                                  # the last runs over the end of the cache for T > 33
    n_new = [T, max(T - 1, 0), T, T]
    cache_h = _noise_cache(rng, B, H, pages, D)
    cache = torch.from_numpy(cache_h.copy()).cuda()
    k, v = _rows(rng, (B, H, T, D), dtype), _rows(rng, (B, H, T, D), dtype)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    m.mcsd_append_kv4(k, v, cache, i32(start), i32(n_new))
    kh, vh = to_np(k), to_np(v)
    for b in range(B):
        for h in range(H):
            for t in range(n_new[b]):
                kv4.write_row(cache_h, b, h, start[b] + t, kh[b, h, t], vh[b, h, t])
    got = cache.cpu().numpy()
    assert np.array_equal(got, cache_h)

    # the same rows as dense tensors: what the codes stand for, rounded once
    ptrs = m.layer_pointer_table([cache])
    dk, dv = m.mcsd_read_kv4(ptrs, i32(start), T + 3, i32([n + 1 for n in n_new]), B, H, D, pages * 32, dtype)
    rk, rv = kv4.read_rows(cache_h, D)
    for b in range(B):
        for t in range(T + 3):
            inside = t < n_new[b] + 1 and start[b] + t < pages * 32
            for x, r in ((dk, rk), (dv, rv)):
                want = torch.from_numpy(r[b, :, start[b] + t].astype(np.float32)).to(dtype) if inside else torch.zeros(H, D, dtype=dtype)
                assert torch.equal(x[0, b, :, t].cpu(), want), (b, t)


@pytest.mark.gpu
def test_append_leaves_sequences_with_nothing_to_store_alone(m):
    rng = np.random.default_rng(1)
    before = torch.from_numpy(_noise_cache(rng, 4, 1, 2, 64)).cuda()
    cache = before.clone()
    k = _rows(rng, (4, 1, 7, 64), torch.bfloat16)
    start = torch.tensor([-1, 64, 3, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    n_new = torch.tensor([7, 7, 0, 7], dtype=torch.int32, device="cuda")
    m.mcsd_append_kv4(k, k, cache, start, n_new)
    assert torch.equal(cache, before)
    out = m.mcsd_read_kv4(m.layer_pointer_table([cache]), start, 5, None, 4, 1, 64, 64, torch.float32)
    assert (out[0][0, 3] == 0).all() and (out[0][0, 1] == 0).all() and (out[0][0, 0, :, 0] == 0).all()
    assert not (out[0][0, 0, :, 1:] == 0).all()              # rows 0.. of the cache


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_with_extreme_values(m, dtype, D):
    rng = np.random.default_rng(3)
    x = rng.normal(size=(1, 1, 8, D))
    x[0, 0, 0] = 0
    x[0, 0, 1] = 3.25                                        # constant
    x[0, 0, 2, 5] = 1e30                                     # one value far out
    x[0, 0, 3] *= 1e-30
    x[0, 0, 4] += 1000                                       # large against its range
    x[0, 0, 5] = np.where(np.arange(D) % 2 == 0, 1.0, -1.0)
    x[0, 0, 6] *= 1e-42                                      # below the normal range
    k = torch.from_numpy(x).to("cuda", dtype)
    cache = m.new_kv4_cache(1, 1, 32, D, "cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    m.mcsd_append_kv4(k, k, cache, zero)
    want = np.zeros((1, 1, 1, 32 * D + 256), dtype=np.uint8)
    kh = to_np(k)
    for t in range(8):
        kv4.write_row(want, 0, 0, t, kh[0, 0, t], kh[0, 0, t])
    assert np.array_equal(cache.cpu().numpy(), want)
    # rows that are not finite: no fault, and the other rows keep theirs
    k[0, 0, 0, 3] = float("inf")
    k[0, 0, 1, 3] = float("nan")
    m.mcsd_append_kv4(k, k, cache, zero)
    back, _ = m.mcsd_read_kv4(m.layer_pointer_table([cache]), zero, 8, None, 1, 1, D, 32, torch.float32)
    rk, _ = kv4.read_rows(want, D)
    assert np.array_equal(back[0, 0, 0, 2:].cpu().numpy(), rk[0, 0, 2:8].astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_commit_writes_the_oracles_bytes_and_no_others(m, dtype, D):
    rng = np.random.default_rng(9)
    parent = parent_array(2, (4, 3, 1, 1))
    tm = m.mcsd_build_mask(parent)
    layers, B, H, N, pages = 3, 6, 2, tm.n_nodes, 3
    lens = [0, 27, 31, 32, 93, 96]                           # inside a page, over its end, over the end of the cache, full
    accept = [0, 4, 4, 2, 4, 3]
    nodes = np.full((B, tm.n_levels), -1, dtype=np.int32)
    for b in range(B):
        for d in range(accept[b]):
            nodes[b, d] = rng.integers(tm.level_start_host[d + 1], tm.level_start_host[d + 2])
    roots = rng.integers(0, 2, size=B).astype(np.int32)
    caches_h = [_noise_cache(rng, B, H, pages, D) for _ in range(layers)]
    caches = [torch.from_numpy(c.copy()).cuda() for c in caches_h]
    kt = [_rows(rng, (B, H, N, D), dtype) for _ in range(layers)]
    vt = [_rows(rng, (B, H, N, D), dtype) for _ in range(layers)]
    dev = lambda a: torch.as_tensor(np.asarray(a, dtype=np.int32)).cuda()  # noqa: E731
    ver = dict(accept_len=dev(accept), out_nodes=dev(nodes), best_root=dev(roots))
    lens_d = dev(lens)
    m.mcsd_commit_kv4(m.layer_pointer_table(caches), m.layer_pointer_table(kt), m.layer_pointer_table(vt), lens_d, ver, tm, B, H, D,
                      pages * 32, dtype)
    for c, ch, k, v in zip(caches, caches_h, kt, vt):
        new = kv4.commit(ch, to_np(k), to_np(v), lens, accept, nodes, roots)
        assert np.array_equal(c.cpu().numpy(), ch)
    assert np.array_equal(lens_d.cpu().numpy(), new)


# ---------------------------------------------------------------------------------------------- attention

def _attend(m, q, cache, kt, vt, lens, act, tm, ws=None):
    B, H, N, D = q.shape
    out = torch.full_like(q, float("nan"))
    if ws is None:
        code = m.MCSD_F32 if q.dtype == torch.float32 else m.MCSD_BF16
        ws = torch.zeros(m.mcsd_tree_attention_kv4_workspace_bytes(B, H, kt.shape[1], N, D, cache.shape[2] * 32, code),
                         dtype=torch.uint8, device="cuda")
    m.mcsd_tree_attention_kv4(q, cache, kt, vt, lens, act, tm, out=out, workspace=ws)
    assert m.mcsd_workspace_status(ws) == 0
    return out


def _check_attention(out, q, cache_h, kt, vt, lens, act, parent, heads=None):
    """Against the definition in 64 bits, elementwise.

    u = 2^-8 (bf16) or 2^-24 (fp32) is half a step of the tensors' type.  Roundings of the result to that type: u |out|.
    With bf16 tensors the weights and the prefix values are rounded to bf16 before their product, each by u of a term,
    so by at most 2 u of A = sum w |v|, and every score, weight and sum is computed in fp32: a score is a sum of D
    products (in 2^-23 steps of the largest partial sum: tensor cores may cut instead of rounding) plus the offset's
    share, which is as large, off by at most 2 (D + 4) 2^-23 S where S = scale * sum |q| |k| bounds the partial sums
    (codes stand for 16 to 31 steps, so a prefix row counts with scale * (16 + code) + |offset|); a weight is off by that
    much twice (its own score and the row's sum) and by 2^-21 for the exponential; the sums over n keys add n 2^-23 A.
    """
    B, H, N, D = q.shape
    G = H // kt.shape[1]
    u = 2.0 ** -24 if q.dtype == torch.float32 else 2.0 ** -8
    kc, vc = kv4.read_rows(cache_h, D)
    sc = (np.ascontiguousarray(cache_h[..., 32 * D:]).view(np.uint16).astype(np.uint32) << 16).view(np.float32)
    sc = np.abs(sc.astype(np.float64)).reshape(B, H // G, -1, 4, 32)
    qh, kh, vh = to_np(q).astype(np.float64), to_np(kt).astype(np.float64), to_np(vt).astype(np.float64)
    scale = D ** -0.5
    o = to_np(out).astype(np.float64)
    sq_err, sq_ref = 0.0, 0.0
    for b in range(B):
        L, n = int(lens[b]), N if act is None else int(act[b])
        assert np.isnan(o[b, :, n:]).all()                   # rows past the active ones are left as they were
        if n == 0:
            continue
        for h in (range(H) if heads is None else heads):
            g = h // G
            keys, vals = np.concatenate([kc[b, g, :L], kh[b, g, :n]]), np.concatenate([vc[b, g, :L], vh[b, g, :n]])
            size = np.concatenate([(31 * sc[b, g, :, 0] + sc[b, g, :, 1]).reshape(-1)[:L, None] * np.ones((1, D)), np.abs(kh[b, g, :n])])
            z = qh[b, h, :n] @ keys.T * scale
            z[:, L:][~orc.dense_mask(parent)[:n, :n]] = -np.inf
            w = np.exp(z - z.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            ref, A = w @ vals, w @ np.abs(vals)
            S = (np.abs(qh[b, h, :n]) @ size.T * scale).max(-1, keepdims=True)
            weight = 2 * (2 * (D + 4) * 2.0 ** -23 * S + 2.0 ** -21) + (L + n + 8) * 2.0 ** -23
            tol = u * np.abs(ref) + (2 * u if q.dtype == torch.bfloat16 else 0) * A + weight * A + 1e-30
            err = np.abs(o[b, h, :n] - ref)
            assert np.isfinite(o[b, h, :n]).all(), (b, h)
            assert (err <= tol).all(), (b, h, L, n, (err / tol).max())
            sq_err, sq_ref = sq_err + (err ** 2).sum(), sq_ref + (ref ** 2).sum()
    if q.dtype == torch.bfloat16 and sq_ref > 0:
        # three independent roundings (weights, values, result), each at most 2^-8 / sqrt(3) in the mean square
        assert np.sqrt(sq_err / sq_ref) <= 2.0 ** -8 * 1.05


def _problem(m, rng, dtype, B, Hq, Hkv, D, parent, lens, act, poison=True, spread=1.0):
    N = len(parent)
    pages = max(1, -(-max(lens) // 32)) + 1
    cache_h = np.zeros((B, Hkv, pages, 32 * D + 256), dtype=np.uint8)
    cache = torch.from_numpy(cache_h).cuda()
    T = pages * 32
    k, v = spread * _rows(rng, (B, Hkv, T, D), torch.float32), _rows(rng, (B, Hkv, T, D), torch.float32)
    m.mcsd_append_kv4(k, v, cache, torch.zeros(B, dtype=torch.int32, device="cuda"))
    cache_h = cache.cpu().numpy()
    q, kt, vt = (spread * _rows(rng, (B, h, N, D), torch.float32).to(dtype) for h in (Hq, Hkv, Hkv))
    q = q.to(dtype); kt = kt.to(dtype); vt = vt.to(dtype)
    if poison:                                               # rows from the length on, inactive rows: anything, NaN scales included
        sc = cache_h[..., 32 * D:].view(np.uint16).reshape(B, Hkv, pages, 4, 32)
        for b in range(B):
            for row in range(lens[b], T):
                sc[b, :, row // 32, :, row % 32] = 0x7FC1 if row % 2 else 0x7F80
        cache = torch.from_numpy(cache_h).cuda()
        if act is not None:
            for b in range(B):
                q[b, :, act[b]:] = float("nan")
                kt[b, :, act[b]:] = float("nan")
                vt[b, :, act[b]:] = float("nan")
    return q, cache, cache_h, kt, vt


def _case(m, dtype, B, Hq, Hkv, D, parent, lens, act, seed, **kw):
    rng = np.random.default_rng(seed)
    q, cache, cache_h, kt, vt = _problem(m, rng, dtype, B, Hq, Hkv, D, parent, lens, act, **kw)
    tm = m.mcsd_build_mask(parent)
    i32 = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    out = _attend(m, q, cache, kt, vt, i32(lens), i32(act), tm)
    _check_attention(out, q, cache_h, kt.nan_to_num(0), vt.nan_to_num(0), lens, act, parent)


TREES = {"token": (1, ()), "pair": (2, ()), "binary": (1, (2, 2, 2)), "static": (1, (4, 2, 2, 1)), "two_roots": (2, (4, 3, 1, 1)),
         "deep": (1, (4, 2, 2, 1, 1, 1, 1, 1)), "forest": (8, (1, 2, 2, 1, 1, 1)), "full": (1, (7, 8, 1, 1)), "chain": (1, (1,) * 63)}
LENS = [0, 1, 31, 32, 33, 127, 128, 129, 300]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 128), (torch.float32, 64)])
@pytest.mark.parametrize("tree", sorted(TREES))
def test_attention_over_lengths_around_pages_and_tiles(m, dtype, D, tree):
    parent = parent_array(*TREES[tree])
    ls = orc.tree_levels(parent)[1]
    _case(m, dtype, len(LENS), 2, 1, D, parent, LENS, None, 11)
    act = [int(ls[1 + b % (len(ls) - 1)]) for b in range(len(LENS))]
    act[3] = 0                                               # a sequence that sits this step out
    _case(m, dtype, len(LENS), 2, 2, D, parent, LENS[::-1], act, 12)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (4, 2), (16, 2), (7, 1), (12, 3), (32, 1)])
def test_attention_with_grouped_queries(m, dtype, D, Hq, Hkv):
    for tree, lens in (("token", [500, 64]), ("static", [200, 1]), ("forest", [77, 160])):
        parent = parent_array(*TREES[tree])
        _case(m, dtype, 2, Hq, Hkv, D, parent, lens, None, Hq)
    parent = parent_array(*TREES["static"])
    _case(m, dtype, 3, Hq, Hkv, D, parent, [33, 0, 260], [45, 5, 13], Hq + 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_with_large_scores(m, dtype):
    """Scores of tens to hundreds: the running maximum moves, and all weight may sit on one key."""
    parent = parent_array(*TREES["static"])
    for spread in (3.0, 6.0):
        _case(m, dtype, 3, 2, 1, 128, parent, [700, 129, 5], None, 21, spread=spread)


@pytest.mark.gpu
def test_attention_reads_the_mask(m):
    """Tree values are one-hot in their node: the output says which nodes a row saw, for every tree and slice."""
    for tree in sorted(TREES):
        parent = parent_array(*TREES[tree])
        N = len(parent)
        for part in range(0, N, 128):
            tm = m.mcsd_build_mask(parent)
            q = torch.zeros(1, 1, N, 128, dtype=torch.bfloat16, device="cuda")
            vt = torch.zeros_like(q)
            for n in range(part, min(N, part + 128)):
                vt[0, 0, n, n - part] = 1
            cache = m.new_kv4_cache(1, 1, 32, 128, "cuda")
            lens = torch.zeros(1, dtype=torch.int32, device="cuda")
            out = to_np(_attend(m, q, cache, q, vt, lens, None, tm))[0, 0]
            see = orc.dense_mask(parent)
            w = min(N, part + 128) - part
            assert np.array_equal(out[:, :w] > 0, see[:, part:part + w])


@pytest.mark.gpu
def test_one_long_sequence_cut_into_many_pieces(m):
    for tree, Hq, Hkv, L in (("token", 8, 1, 40000), ("static", 1, 1, 20001), ("forest", 2, 2, 9000)):
        _case(m, torch.bfloat16, 1, Hq, Hkv, 128, parent_array(*TREES[tree]), [L], None, 5)


@pytest.mark.gpu
def test_many_sequences(m):
    """More sequences than thread blocks, and more than the tensor-core kernel's tables hold."""
    rng = np.random.default_rng(0)
    for B in (200, 256, 300):
        lens = [int(x) for x in rng.integers(0, 140, size=B)]
        _case(m, torch.bfloat16, B, 2, 1, 128, parent_array(1, (2,)), lens, None, B)


@pytest.mark.gpu
def test_workspace_reuse_streams_and_graph_replay(m):
    """One workspace through calls of different shapes, a call on another stream, and a captured call replayed on new data."""
    rng = np.random.default_rng(2)
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    for tree, lens, Hq in (("static", [1000, 3], 4), ("token", [5000, 2000], 8), ("forest", [600, 31], 2)):
        parent = parent_array(*TREES[tree])
        tm = m.mcsd_build_mask(parent)
        q, cache, cache_h, kt, vt = _problem(m, rng, torch.bfloat16, 2, Hq, 2, 128, parent, lens, None)
        for _ in range(3):
            out = _attend(m, q, cache, kt, vt, i32(lens), None, tm, ws)
        _check_attention(out, q, cache_h, kt, vt, lens, None, parent)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = m.mcsd_tree_attention_kv4(q, cache, kt, vt, i32(lens), None, tm)
        side.synchronize()
        assert torch.equal(out, other)                       # the cut depends on shapes alone: equal to the bit
        lens_d, got = i32(lens), torch.empty_like(q)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.mcsd_tree_attention_kv4(q, cache, kt, vt, lens_d, None, tm, out=got, workspace=ws)
        lens_d.copy_(i32([min(lens), min(lens)]))
        graph.replay()
        torch.cuda.synchronize()
        _check_attention(got, q, cache_h, kt, vt, [min(lens)] * 2, None, parent)


# ---------------------------------------------------------------------------------------------- all of it, as a target runs it

@pytest.mark.gpu
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_generation_steps_over_a_4_bit_cache(m, dtype, D):
    """Prompt rows normalised, rotated and appended; then steps of tree rows, attention, verification and commit, with every
    layer's cache, lengths and attention output checked against the oracle after each."""
    rng = np.random.default_rng(17)
    layers, B, Hq, Hkv, V = 2, 3, 4, 2, 50
    parent = parent_array(1, (4, 2, 2, 1))
    tm = m.mcsd_build_mask(parent)
    N, pages = tm.n_nodes, 4
    f = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device="cuda") / (D // 2))
    w = [[(1 + 0.1 * torch.from_numpy(rng.normal(size=D))).to("cuda", dtype) for _ in range(2)] for _ in range(layers)]
    project = lambda n: torch.from_numpy(rng.normal(size=(B, n, Hq + 2 * Hkv, D))).to("cuda", dtype).split([Hq, Hkv, Hkv], 2)  # noqa: E731
    caches = [m.new_kv4_cache(B, Hkv, pages * 32, D, "cuda") for _ in range(layers)]
    ptrs = m.layer_pointer_table(caches)
    T, lens_h = 61, np.array([61, 40, 7], dtype=np.int32)
    lens = torch.from_numpy(lens_h).cuda()
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    want = [np.zeros(c.shape, dtype=np.uint8) for c in caches]
    for i in range(layers):
        _, k, v = m.mcsd_qk_norm_rope(*project(T), zero, f, q_weight=w[i][0], k_weight=w[i][1], n_active=lens)
        m.mcsd_append_kv4(k, v, caches[i], zero, lens)
        for b in range(B):
            for h in range(Hkv):
                for t in range(lens_h[b]):
                    kv4.write_row(want[i], b, h, t, to_np(k[b, h, t]), to_np(v[b, h, t]))
        assert np.array_equal(caches[i].cpu().numpy(), want[i])
    for step in range(3):
        kts, vts = [], []
        for i in range(layers):
            q, kt, vt = m.mcsd_qk_norm_rope(*project(N), lens, f, depth=tm.depth, q_weight=w[i][0], k_weight=w[i][1])
            out = _attend(m, q, caches[i], kt, vt, lens, None, tm)
            _check_attention(out, q, want[i], kt, vt, lens_h, None, parent)
            kts.append(kt)
            vts.append(vt)
        p = torch.softmax(torch.from_numpy(rng.normal(size=(B, N, V))).float().cuda(), -1)
        pd = torch.softmax(p.log() + 0.5 * torch.from_numpy(rng.normal(size=(B, N, V))).float().cuda(), -1)
        tokens = torch.from_numpy(rng.integers(0, V, size=(B, N)).astype(np.int32)).cuda()
        u = torch.from_numpy(rng.uniform(0.001, 0.4, size=(B, N)).astype(np.float32)).cuda()
        ver = m.mcsd_verify_tree(p, pd, tokens, tm, None, u, u)
        m.mcsd_commit_kv4(ptrs, m.layer_pointer_table(kts), m.layer_pointer_table(vts), lens, ver, tm, B, Hkv, D, pages * 32, dtype)
        acc, nodes, root = (ver[x].cpu().numpy() for x in ("accept_len", "out_nodes", "best_root"))
        for i in range(layers):
            new = kv4.commit(want[i], to_np(kts[i]), to_np(vts[i]), lens_h, acc, nodes, root)
            assert np.array_equal(caches[i].cpu().numpy(), want[i])
        lens_h = new
        assert np.array_equal(lens.cpu().numpy(), lens_h)


def _off_by_one(t):
    """The same contiguous tensor one element further on in memory."""
    x = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)[1:].view(t.shape)
    return x.copy_(t)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_off_16_byte_boundaries(m, dtype, D):
    rng = np.random.default_rng(D)
    B, H, pages, T = 2, 2, 3, 50
    k, v = _rows(rng, (B, H, T, D), dtype), _rows(rng, (B, H, T, D), dtype)
    start = torch.tensor([3, 40], dtype=torch.int32, device="cuda")
    caches = [torch.from_numpy(_noise_cache(np.random.default_rng(5), B, H, pages, D)).cuda() for _ in range(2)]
    m.mcsd_append_kv4(k, v, caches[0], start)
    m.mcsd_append_kv4(_off_by_one(k), _off_by_one(v), caches[1], start)
    assert torch.equal(caches[0], caches[1])
    ptrs = m.layer_pointer_table([caches[0]])
    want = m.mcsd_read_kv4(ptrs, start, T, None, B, H, D, pages * 32, dtype)
    out = tuple(_off_by_one(torch.full_like(x, 7)) for x in want)
    m.mcsd_read_kv4(ptrs, start, T, None, B, H, D, pages * 32, dtype, out=out)
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


@pytest.mark.gpu
def test_attention_with_values_of_the_tree_off_16_byte_boundaries(m):
    rng = np.random.default_rng(11)
    parent = parent_array(*TREES["forest"])
    lens = [200, 33]
    q, cache, _, kt, vt = _problem(m, rng, torch.bfloat16, 2, 2, 2, 128, parent, lens, None)
    tm = m.mcsd_build_mask(parent)
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = _attend(m, q, cache, kt, vt, L, None, tm)
    got = _attend(m, q, cache, kt, _off_by_one(vt), L, None, tm)
    assert torch.equal(got, want)                            # the same kernel, the same order of sums
