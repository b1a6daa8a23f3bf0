"""Operators over a latent cache: rows, tree attention and commit against the definition in 64 bits, one verification step of
them together with filtered sampling, and refusals."""
import ctypes

import numpy as np
import pytest
import torch

from mcsd_inputs import parent_array
from oracle import latent_oracle as lat
from oracle import mcsd_oracle as orc
from tests.helpers import to_np
from tests.test_kv4 import m  # noqa: F401  (the fixture)

FAKE = ctypes.c_void_p(0x1000)      # never dereferenced: every call that uses it fails its checks first
NAN = float("nan")
TREES = {"token": (1, ()), "binary": (1, (2, 2, 2)), "static": (1, (4, 2, 2, 1)), "deep": (1, (4, 2, 2, 1, 1, 1, 1, 1)),
         "forest": (8, (1, 2, 2, 1, 1, 1)), "two_roots": (2, (4, 3, 1, 1)), "chain": (1, (1,) * 191)}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _i32(a):
    return None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------------------------- refusals (host only)

def test_rows_refusals(m):  # noqa: F811
    st = (ctypes.c_int64 * 5)(0, 576, 0, 1024, 64)

    def call(lat_in=FAKE, q_in=FAKE, strides=st, eps=1e-6, freqs=FAKE, lens=FAKE, rows=FAKE, L=8, q=FAKE, B=2, H=4, N=5, rank=512, rot=64, dtype=0):
        return m.lib.mcsd_latent_rows(lat_in, q_in, strides, None, eps, freqs, 0, lens, None, None, None, rows, L, q, B, H, N, rank, rot, dtype, None)
    assert call(lat_in=None) == -1
    assert call(q_in=None) == -1
    assert call(strides=None) == -1
    assert call(freqs=None) == -1
    assert call(lens=None) == -1
    assert call(rows=None, q=None) == -1
    assert call(dtype=7) == -4
    assert call(B=0) == -2
    assert call(B=65536) == -2
    assert call(N=0) == -2
    assert call(B=60000, N=60000) == -2
    assert call(L=0) == -2
    assert call(H=0) == -2
    assert call(rank=0) == -2
    assert call(rank=48) == -2
    assert call(rank=544) == -2
    assert call(rot=8) == -2
    assert call(rot=144) == -2
    assert call(rot=-16) == -2
    assert call(eps=-1.0) == -2
    assert call(eps=NAN) == -2
    assert call(rows=None, rot=0, freqs=None) == 0                   # no rotated part, no rows: nothing to do


def test_attention_refusals(m):  # noqa: F811
    need = m.mcsd_tree_attention_latent_workspace_bytes(2, 4, 15, 512, 64, 100, 0)
    assert need > 0

    def call(q=FAKE, cache=FAKE, tree=FAKE, out=FAKE, lens=FAKE, anc=FAKE, words=1, B=2, H=4, N=15, rank=512, rot=64, L=100, dtype=0, ws=FAKE, n=need):
        return m.lib.mcsd_tree_attention_latent(q, cache, tree, out, lens, None, anc, words, B, H, N, rank, rot, L, 0.1, dtype, ws, n, None)
    for name in ("q", "cache", "tree", "out", "lens", "anc", "ws"):
        assert call(**{name: None}) == -1, name
    assert call(dtype=5) == -4
    for bad in (dict(B=0), dict(H=0), dict(N=0), dict(N=193), dict(L=-1), dict(L=(1 << 30) + 1), dict(B=256, H=256), dict(rank=40), dict(rank=1024),
                dict(rot=24), dict(rot=256), dict(words=0), dict(words=4), dict(N=65)):
        assert call(**bad) == -2, bad
    assert call(n=need - 1) == -5
    assert call(ws=ctypes.c_void_p(0x1008)) == -2
    for bad in ((0, 4, 15, 512, 64, 100, 0), (2, 4, 15, 513, 64, 100, 0), (2, 4, 15, 512, 64, 100, 2)):
        assert m.mcsd_tree_attention_latent_workspace_bytes(*bad) == 0


def test_commit_refusals(m):  # noqa: F811
    def call(c=FAKE, t=FAKE, nl=2, lens=FAKE, levels=4, B=2, N=15, width=576, L=64, dtype=0):
        return m.lib.mcsd_commit_latent(c, t, nl, lens, FAKE, FAKE, FAKE, levels, B, N, width, L, dtype, None)
    assert call(c=None) == -1
    assert call(t=None) == -1
    assert call(lens=None) == -1
    assert call(dtype=2) == -4
    for bad in (dict(nl=0), dict(nl=65536), dict(levels=0), dict(levels=16), dict(B=0), dict(B=65536), dict(N=0), dict(N=193), dict(width=16),
                dict(width=570), dict(width=656), dict(L=0)):
        assert call(**bad) == -2, bad


def test_binding_refusals(m):  # noqa: F811
    x = torch.zeros(1, 4, 3, 576)
    with pytest.raises(ValueError):
        m.mcsd_latent_rows(x[0], None, None, None)
    with pytest.raises(ValueError):
        m.mcsd_latent_rows(x[0], None, torch.zeros(1, dtype=torch.int32), None, rows=x[0])      # not on a GPU


def test_oracle_against_heads_of_their_own():
    """The absorbed form is attention with keys and values expanded per head."""
    rng = np.random.default_rng(0)
    R, P, D, L, n = 32, 16, 8, 9, 3
    uk, uv, qn, qr = rng.normal(size=(D, R)), rng.normal(size=(D, R)), rng.normal(size=(n, D)), rng.normal(size=(n, P))
    rows, see = rng.normal(size=(L + n, R + P)), np.tril(np.ones((n, n), bool))
    o, _, _ = lat.latent_attention(np.concatenate([qn @ uk, qr], 1), rows[:L], rows[L:], see, 0.3, R)
    k, v = np.concatenate([rows[:, :R] @ uk.T, rows[:, R:]], 1), rows[:, :R] @ uv.T
    z = np.concatenate([qn, qr], 1) @ k.T * 0.3
    z[:, L:][~see] = -np.inf
    w = np.exp(z)
    assert np.allclose(o @ uv.T, (w / w.sum(-1, keepdims=True)) @ v)


# ---------------------------------------------------------------------------------------------- rows

def _off(t):
    """The same values in a tensor that starts off a 16-byte boundary."""
    buf = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    buf[1:] = t.flatten()
    return buf[1:].view(t.shape)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rank,rot,H,tree,T,norm,aligned", [
    (512, 64, 16, "static", 0, True, True), (512, 64, 5, "", 1, True, True), (512, 64, 4, "", 4099, False, True), (256, 32, 3, "forest", 0, True, False),
    (32, 16, 1, "", 77, True, True), (160, 128, 2, "binary", 0, False, False), (512, 0, 2, "", 9, True, True)])
def test_rows(m, dtype, rank, rot, H, tree, T, norm, aligned, interleaved):  # noqa: F811
    dt, W, B = DT[dtype], rank + rot, 2 if T < 1000 else 1
    g = torch.Generator("cuda").manual_seed(7)
    tm = m.mcsd_build_mask(parent_array(*TREES[tree])) if tree else None
    N = tm.n_nodes if tree else T
    x = (2 * torch.randn(B, N, W, generator=g, device="cuda")).to(dt)
    heads = torch.randn(B, N, H, 24 + rot, generator=g, device="cuda").to(dt)
    if not aligned:
        x, heads = _off(x), _off(heads)
    weight = (1 + 0.2 * torch.randn(rank, generator=g, device="cuda")).to(dt) if norm else None
    freqs = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device="cuda") / max(1, rot // 2)) if rot else None
    lens = [199999, 0][:B]
    act = None if tree == "" else [N, N // 2]
    start = None if tree else [3, N + 1][:B]
    L_rows = N if tree else N + 3
    rows = torch.full((B, L_rows, W), NAN, dtype=dt, device="cuda")
    q = torch.full((B, H, N, W), NAN, dtype=dt, device="cuda")
    if not aligned:
        rows, q = _off(rows), _off(q)
    m.mcsd_latent_rows(x, heads[..., 24:], _i32(lens), freqs, rows=rows, q=q, row_start=_i32(start), depth=tm.depth if tree else None,
                       n_active=_i32(act), weight=weight, eps=1e-5, interleaved=interleaved)
    torch.cuda.synchronize()
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    hf = freqs.cpu().numpy() if rot else np.zeros(0)
    step = tm.depth.cpu().numpy() if tree else np.arange(N)
    got_r, got_q = to_np(rows), to_np(q)
    for b in range(B):
        a = N if act is None else act[b]
        xb, hb = to_np(x[b, :a]), to_np(heads[b, :a, :, 24:])
        want = lat.latent_rows(xb, None if weight is None else to_np(weight), 1e-5, lens[b] + step[:a], hf, rank, interleaved)
        # norm: 21 additions in a row, a division, a root, two products; angle: 2^-24 of a turn's pi, sine and cosine, two products
        size = np.abs(want)
        if rot:
            size[:, rank:] = np.abs(xb[:, rank:]).max(-1, keepdims=True) * 2
        s = 0 if start is None else start[b]
        there = max(0, min(a, L_rows - s))
        err = np.abs(got_r[b, s:s + there] - want[:there])
        assert (err <= (2.0 ** -19 + half) * size[:there] + half * np.abs(want[:there])).all()
        untouched = np.ones(L_rows, bool)
        untouched[s:s + there] = False
        assert np.isnan(got_r[b, untouched]).all()
        if rot:
            want = np.stack([lat.rotate(hb[:, h], lens[b] + step[:a], hf, interleaved) for h in range(H)])
            size = 2 * np.abs(hb).max(-1).T[..., None]
            assert (np.abs(got_q[b, :, :a, rank:] - want) <= 2.0 ** -19 * size + half * np.abs(want)).all()
        assert np.isnan(got_q[b, :, a:]).all() and np.isnan(got_q[b, :, :, :rank]).all()


@pytest.mark.gpu
def test_one_side_alone(m):  # noqa: F811
    x, h = torch.randn(2, 6, 96, device="cuda"), torch.randn(2, 6, 3, 32, device="cuda")
    lens, freqs = _i32([5, 9]), torch.rand(16, dtype=torch.float64, device="cuda")
    rows, q = torch.zeros(2, 6, 96, device="cuda"), torch.zeros(2, 3, 6, 96, device="cuda")
    m.mcsd_latent_rows(x, h, lens, freqs, rows=rows, q=q)
    r1, _ = m.mcsd_latent_rows(x, None, lens, freqs, rows=torch.zeros_like(rows))
    _, q1 = m.mcsd_latent_rows(None, h, lens, freqs, q=torch.zeros_like(q))
    assert torch.equal(r1, rows) and torch.equal(q1, q)
    with pytest.raises(ValueError):
        m.mcsd_latent_rows(x, h[..., ::2], lens, freqs[:8], rows=rows, q=q)
    with pytest.raises(ValueError):
        m.mcsd_latent_rows(x, h, lens, freqs, rows=rows, q=q[:, :2])
    with pytest.raises(ValueError):
        m.mcsd_latent_rows(x.bfloat16(), h, lens, freqs, rows=rows, q=q)


# ---------------------------------------------------------------------------------------------- attention

def _problem(rng_seed, dtype, B, H, rank, rot, parent, lens, spread=1.0):
    g = torch.Generator("cuda").manual_seed(rng_seed)
    N, W, L_max = len(parent), rank + rot, max(max(lens), 1)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    return (spread * rnd(B, H, N, W)).to(DT[dtype]), rnd(B, L_max, W).to(DT[dtype]), rnd(B, N, W).to(DT[dtype])


def _attend(m, q, cache, tree, lens, act, tm, scale, rank, ws=None):  # noqa: F811
    out = torch.full((*q.shape[:3], rank), NAN, dtype=q.dtype, device="cuda")
    if ws is None:
        code = m.MCSD_BF16 if q.dtype == torch.bfloat16 else m.MCSD_F32
        ws = m.new_workspace(m.mcsd_tree_attention_latent_workspace_bytes(*q.shape[:3], rank, q.shape[3] - rank, cache.shape[1], code), "cuda")
    m.mcsd_tree_attention_latent(q, cache, tree, _i32(lens), _i32(act), tm, scale, out=out, workspace=ws)
    assert m.mcsd_workspace_status(ws) == 0
    return out


def _compare(out, q, cache, tree, lens, act, see, scale, rank, heads=None):
    """Every active row within the bound; rows behind them untouched.

    fp32: a score's W products and sums are off by (W + 4) 2^-24 of their absolute sum at most, which moves a weight by twice
    that (numerator and sum); the sums over n keys, the exponentials and the division add (n + 16) 2^-24.
    bf16: weights are rounded to bf16 (2^-8 relative) for the product with the values, the output once more."""
    bf = q.dtype == torch.bfloat16
    got = to_np(out)
    B, H, N, W = q.shape
    for b in range(B):
        L, a = lens[b], N if act is None else act[b]
        assert np.isnan(got[b, :, a:]).all()
        if a == 0:
            continue
        pre, tr = to_np(cache[b, :L]), to_np(tree[b, :a])
        for h in range(H) if heads is None else heads:
            want, size, products = lat.latent_attention(to_np(q[b, h, :a]), pre, tr, see[:a, :a], scale, rank)
            rel = 2 * (W + 4) * 2.0 ** -24 * products + (L + a + 16) * 2.0 ** -24 + (2.0 ** -8 if bf else 0.0)
            bound = rel * size + (2.0 ** -8 if bf else 2.0 ** -24) * np.abs(want) + 1e-30
            err = np.abs(got[b, h, :a] - want)
            assert (err <= bound).all(), (b, h, (err / bound).max())


ATTENTION = [
    # dtype, B, H, rank, rot, tree, lens, active
    ("f32", 2, 4, 128, 32, "binary", [131, 0], None),
    ("f32", 1, 3, 512, 64, "static", [700], [21]),
    ("f32", 3, 2, 32, 0, "token", [1, 0, 33], None),
    ("f32", 1, 5, 480, 128, "forest", [64], [96]),
    ("bf16", 1, 2, 256, 64, "binary", [300], None),
    ("bf16", 1, 16, 512, 64, "token", [1001], None),
    ("bf16", 1, 1, 512, 64, "token", [0], None),
    ("bf16", 3, 1, 512, 64, "token", [1, 31, 32], None),
    ("bf16", 2, 128, 512, 64, "token", [5000, 257], None),
    ("bf16", 2, 8, 512, 64, "static", [2500, 255], None),
    ("bf16", 3, 3, 512, 64, "forest", [700, 256, 1], [160, 8, 0]),
    ("bf16", 2, 20, 512, 64, "deep", [513, 64], [109, 13]),
    ("bf16", 1, 2, 512, 64, "chain", [100], None),
    ("bf16", 40, 4, 512, 64, "two_roots", [97 * (i % 7) for i in range(40)], [1 + (13 * i) % 82 for i in range(40)]),
    ("bf16", 300, 1, 512, 64, "token", [i % 70 for i in range(300)], None),
    ("bf16", 1, 16, 512, 64, "token", [40000], None),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,B,H,rank,rot,tree,lens,act", ATTENTION)
def test_attention(m, dtype, B, H, rank, rot, tree, lens, act):  # noqa: F811
    parent = parent_array(*TREES[tree])
    q, cache, rows = _problem(B + H, dtype, B, H, rank, rot, parent, lens)
    for b, L in enumerate(lens):                                       # what lies behind a sequence is not looked at
        cache[b, L:] = NAN
        if act is not None:
            rows[b, act[b]:] = NAN
            q[b, :, act[b]:] = NAN
    tm, scale = m.mcsd_build_mask(parent), (128 + rot) ** -0.5
    out = _attend(m, q, cache, rows, lens, act, tm, scale, rank)
    heads = None if H <= 8 else [0, H // 2, H - 1]
    _compare(out, q, cache, rows, lens, act, orc.dense_mask(parent), scale, rank, heads)
    again = _attend(m, q, cache, rows, lens, act, tm, scale, rank)
    assert torch.equal(out.nan_to_num(7.0), again.nan_to_num(7.0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,spread", [(0.0, 1.0), (-0.05, 1.0), (1.0, 3.0), (0.07, 0.0)])
def test_scales(m, dtype, scale, spread):  # noqa: F811
    """No difference between keys, the smallest first, one key that outweighs all others by far, queries of zeros."""
    parent = parent_array(*TREES["static"])
    lens = [777, 130]
    q, cache, rows = _problem(3, dtype, 2, 3, 512, 64, parent, lens, spread)
    out = _attend(m, q, cache, rows, lens, None, m.mcsd_build_mask(parent), scale, 512)
    _compare(out, q, cache, rows, lens, None, orc.dense_mask(parent), scale, 512)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_growing_scores(m, dtype):  # noqa: F811
    """Every tile holds a key that outweighs what came before: the running maximum moves all the time."""
    parent = parent_array(*TREES["binary"])
    q, cache, rows = _problem(5, dtype, 1, 4, 512, 64, parent, [3000])
    ramp = torch.linspace(0, 40, 3000, device="cuda")
    cache[0, :, 512:] = 0
    cache[0, :, 512] = ramp.to(cache.dtype)
    q[..., 512:] = 0
    q[..., 512] = 14.0
    out = _attend(m, q, cache, rows, [3000], None, m.mcsd_build_mask(parent), 0.07, 512)
    _compare(out, q, cache, rows, [3000], None, orc.dense_mask(parent), 0.07, 512)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_mask_bits_and_rows_that_see_nothing(m, dtype):  # noqa: F811
    """Random masks, three words a node, some rows without a bit: zeros where the prefix is empty too."""
    rng = np.random.default_rng(8)
    parent = parent_array(*TREES["chain"])
    tm = m.mcsd_build_mask(parent)
    see = rng.random((192, 192)) < 0.3
    see[5] = see[100] = False
    bits = np.zeros((192, 3), dtype=np.uint64)
    for j in range(192):
        bits[:, j // 64] |= see[:, j].astype(np.uint64) << np.uint64(j % 64)
    tm = tm._replace(anc=torch.from_numpy(bits.view(np.int64)).cuda())
    lens = [0, 70]
    q, cache, rows = _problem(6, dtype, 2, 3, 512, 64, parent, lens)
    out = _attend(m, q, cache, rows, lens, None, tm, 0.07, 512)
    assert not out[0, :, 5].any() and not out[0, :, 100].any()
    _compare(out, q, cache, rows, lens, None, see, 0.07, 512)


@pytest.mark.gpu
def test_without_a_cache_and_off_a_16_byte_boundary(m):  # noqa: F811
    parent = parent_array(*TREES["static"])
    tm, see = m.mcsd_build_mask(parent), orc.dense_mask(parent)
    q, cache, rows = _problem(9, "bf16", 2, 4, 512, 64, parent, [90, 33])
    empty = torch.empty(2, 0, 576, dtype=torch.bfloat16, device="cuda")
    out = _attend(m, q, empty, rows, [0, 0], None, tm, 0.07, 512)
    _compare(out, q, cache, rows, [0, 0], None, see, 0.07, 512)
    for i in range(3):
        x = [q, cache, rows]
        x[i] = _off(x[i])
        out = _attend(m, *x, [90, 33], None, tm, 0.07, 512)
        _compare(out, q, cache, rows, [90, 33], None, see, 0.07, 512)
    with pytest.raises(ValueError):
        m.mcsd_tree_attention_latent(q, cache, rows, _i32([90, 33]), None, tm, 0.07)              # no rank
    with pytest.raises(ValueError):
        m.mcsd_tree_attention_latent(q[:, :, :7].contiguous(), cache, rows, _i32([90, 33]), None, tm, 0.07, rank=512)
    with pytest.raises(ValueError):
        m.mcsd_tree_attention_latent(q, cache.float(), rows, _i32([90, 33]), None, tm, 0.07, rank=512)
    with pytest.raises(m.McsdError):
        m.mcsd_tree_attention_latent(q, cache, rows, _i32([90, 33]), None, tm, 0.07, rank=500)


@pytest.mark.gpu
def test_offsets_beyond_32_bits(m):  # noqa: F811
    """Two caches of 2.1 million rows (1.2 thousand million values each): a few rows that outweigh the rest are found."""
    L_max, W = 2_100_000, 576
    cache = torch.zeros(2, L_max, W, dtype=torch.bfloat16, device="cuda")
    lens, at = [2_099_999, 1_900_001], [2_099_998, 1_900_000]
    tm = m.mcsd_build_mask([-1])
    q = torch.zeros(2, 4, 1, W, dtype=torch.bfloat16, device="cuda")
    q[..., 575] = 16.0
    rows = torch.zeros(2, 1, W, dtype=torch.bfloat16, device="cuda")
    for b in range(2):
        cache[b, at[b], 575] = 16.0
        cache[b, at[b], :512] = torch.arange(512, device="cuda").to(torch.bfloat16) + b
        cache[b, lens[b]:] = NAN
    out = _attend(m, q, cache, rows, lens, None, tm, 1.0, 512)
    for b in range(2):
        assert torch.equal(out[b, :, 0], cache[b, at[b], :512].expand(4, 512))


@pytest.mark.gpu
def test_one_workspace_with_the_other_attention_calls(m):  # noqa: F811
    parent = parent_array(*TREES["static"])
    tm, lens = m.mcsd_build_mask(parent), [900, 3100]
    q, cache, rows = _problem(11, "bf16", 2, 8, 512, 64, parent, lens)
    g = torch.Generator("cuda").manual_seed(2)
    d = [torch.randn(2, 8, n, 128, generator=g, device="cuda").bfloat16() for n in (45, 3100, 3100, 45, 45)]
    dense = lambda ws: m.mcsd_tree_attention(*d, _i32(lens), None, tm, workspace=ws)  # noqa: E731
    calls = [lambda ws: _attend(m, q, cache, rows, lens, None, tm, 0.07, 512, ws), dense,
             lambda ws: _attend(m, q.float(), cache.float(), rows.float(), lens, None, tm, 0.07, 512, ws)]
    want = [c(torch.zeros(128 << 20, dtype=torch.uint8, device="cuda")) for c in calls]
    ws = torch.zeros(128 << 20, dtype=torch.uint8, device="cuda")
    for i in (0, 1, 0, 2, 0, 0, 1, 1, 2, 1, 0):
        assert torch.equal(calls[i](ws), want[i])


@pytest.mark.gpu
def test_captured_with_lengths_that_change(m):  # noqa: F811
    parent = parent_array(*TREES["static"])
    tm, see = m.mcsd_build_mask(parent), orc.dense_mask(parent)
    q, cache, rows = _problem(12, "bf16", 3, 4, 512, 64, parent, [2000] * 3)
    lens, act = _i32([2000, 300, 0]), _i32([45, 21, 5])
    out = torch.full((3, 4, 45, 512), NAN, dtype=torch.bfloat16, device="cuda")
    ws = m.new_workspace(m.mcsd_tree_attention_latent_workspace_bytes(3, 4, 45, 512, 64, 2000, 0), "cuda")
    call = lambda: m.mcsd_tree_attention_latent(q, cache, rows, lens, act, tm, 0.07, out=out, workspace=ws)  # noqa: E731
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
    for L, a in (([2000, 300, 0], [45, 21, 5]), ([17, 1999, 1024], [5, 45, 0]), ([0, 0, 0], [1, 1, 1]), ([0, 0, 0], [0, 0, 0]), ([256, 257, 1], [45, 45, 45])):
        lens.copy_(_i32(L))
        act.copy_(_i32(a))
        out.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        _compare(out, q, cache, rows, L, a, see, 0.07, 512)
    assert m.mcsd_workspace_status(ws) == 0


@pytest.mark.gpu
def test_two_calls_at_once(m):  # noqa: F811
    """Calls of two streams, each with its own workspace: items in few pieces and in many, whichever blocks run first."""
    cases = []
    for seed, (B, H, tree, lens) in enumerate([(2, 32, "static", [6000, 300]), (1, 16, "token", [30000]), (3, 64, "token", [9000, 20, 4000])]):
        parent = parent_array(*TREES[tree])
        q, cache, rows = _problem(30 + seed, "bf16", B, H, 512, 64, parent, lens)
        cases.append((q, cache, rows, _i32(lens), m.mcsd_build_mask(parent)))
    size = max(m.mcsd_tree_attention_latent_workspace_bytes(*c[0].shape[:3], 512, 64, c[1].shape[1], m.MCSD_BF16) for c in cases)
    spaces = [m.new_workspace(size, "cuda") for _ in range(2)]
    call = lambda c, ws, out: m.mcsd_tree_attention_latent(*c[:4], None, c[4], 0.07, out=out, workspace=ws)  # noqa: E731
    want = [call(c, spaces[0], torch.empty(*c[0].shape[:3], 512, dtype=torch.bfloat16, device="cuda")) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream(priority=-1)]
    outs = [[], []]
    for i in range(30):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                out = torch.full_like(want[(i + k) % 3], NAN)
                call(cases[(i + k) % 3], spaces[k], out)
                outs[k].append(out)
    torch.cuda.synchronize()
    assert [m.mcsd_workspace_status(ws) for ws in spaces] == [0, 0]
    for k in range(2):
        for i, out in enumerate(outs[k]):
            assert torch.equal(out, want[(i + k) % 3]), (k, i)


@pytest.mark.gpu
def test_two_graphs_share_a_workspace(m):  # noqa: F811
    """Replayed in turn; counters are zero between launches."""
    parent = parent_array(*TREES["static"])
    tm, ws = m.mcsd_build_mask(parent), torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    graphs, s = [], torch.cuda.Stream()
    for seed, (H, dtype, lens) in enumerate([(16, "bf16", [20000, 10]), (2, "f32", [3000, 3001]), (32, "bf16", [7, 900])]):
        q, cache, rows = _problem(40 + seed, dtype, 2, H, 512, 64, parent, lens)
        ln, out = _i32(lens), torch.zeros(2, H, len(parent), 512, dtype=DT[dtype], device="cuda")
        call = lambda: m.mcsd_tree_attention_latent(q, cache, rows, ln, None, tm, 0.07, out=out, workspace=ws)  # noqa: E731, B023
        call()
        torch.cuda.synchronize()
        want, graph = out.clone(), torch.cuda.CUDAGraph()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=s):
            call()
        graphs.append((graph, out, want, (q, cache, rows, ln)))
    for i in (0, 1, 2, 2, 0, 0, 1, 0, 2, 1):
        graph, out, want, _ = graphs[i]
        out.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert m.mcsd_workspace_status(ws) == 0


@pytest.mark.gpu
def test_lengths_out_of_range_are_clamped(m):  # noqa: F811
    parent = parent_array(*TREES["binary"])
    tm = m.mcsd_build_mask(parent)
    for dtype in ("bf16", "f32"):
        q, cache, rows = _problem(13, dtype, 3, 2, 512, 64, parent, [50] * 3)
        a = _attend(m, q, cache, rows, [-5, 90, 50], [20, -1, 15], tm, 0.07, 512)
        b = _attend(m, q, cache, rows, [0, 50, 50], [15, 0, 15], tm, 0.07, 512)
        assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))


# ---------------------------------------------------------------------------------------------- commit

@pytest.mark.gpu
@pytest.mark.parametrize("dtype,layers,B,width,tree,L_max", [("bf16", 1, 1, 576, "token", 5), ("bf16", 11, 5, 576, "deep", 40), ("f32", 3, 2, 160, "two_roots", 9),
                                                             ("bf16", 40, 3, 32, "static", 30)])
@pytest.mark.parametrize("aligned", [True, False])
def test_commit(m, dtype, layers, B, width, tree, L_max, aligned):  # noqa: F811
    rng = np.random.default_rng(4)
    tm = m.mcsd_build_mask(parent_array(*TREES[tree]))
    N, levels = tm.n_nodes, tm.n_levels
    g = torch.Generator("cuda").manual_seed(1)
    caches = [torch.randn(B, L_max, width, generator=g, device="cuda").to(DT[dtype]) for _ in range(layers)]
    rows = [torch.randn(B, N, width, generator=g, device="cuda").to(DT[dtype]) for _ in range(layers)]
    if not aligned:
        caches, rows = [_off(c) for c in caches], [_off(r) for r in rows]
    lens = [int(x) for x in rng.integers(0, L_max + 1, B)]
    lens[0] = L_max - 1
    acc = [int(x) for x in rng.integers(0, levels, B)]
    nodes = rng.integers(0, N, (B, levels))
    for b in range(B):
        nodes[b, acc[b]:] = -1
    if B > 1 and acc[1] > 0:
        nodes[1, 0] = N + 3                                             # malformed: that row stays as it was
    root = [int(x) for x in rng.integers(0, tm.n_roots, B)]
    want = [c.clone() for c in caches]
    for b in range(B):
        for t in range(1 + acc[b]):
            n = root[b] if t == 0 else nodes[b, t - 1]
            if lens[b] + t < L_max and 0 <= n < N:
                for i in range(layers):
                    want[i][b, lens[b] + t] = rows[i][b, n]
    dl = _i32(lens)
    m.mcsd_commit_latent(m.layer_pointer_table(caches), m.layer_pointer_table(rows), dl,
                         dict(accept_len=_i32(acc), out_nodes=_i32(nodes.tolist()), best_root=_i32(root)), tm, B, width, L_max, DT[dtype])
    assert all(torch.equal(a, b) for a, b in zip(caches, want))
    assert dl.tolist() == [min(L_max, n + 1 + a) for n, a in zip(lens, acc)]


# ---------------------------------------------------------------------------------------------- one step of all of it

@pytest.mark.gpu
def test_a_step(m):  # noqa: F811
    """Prompt rows into the caches of two layers, a tree of candidates drawn from filtered draft logits level by level, its rows
    and attention, verification of the target's filtered probabilities, commit; then attention over the grown cache equals
    attention over a cache that held the accepted rows from the start."""
    g = torch.Generator("cuda").manual_seed(21)
    B, H, R, P, V, L_max, layers = 2, 4, 512, 64, 900, 200, 2
    W, parent = R + P, parent_array(1, (4, 2, 2, 1))
    tm = m.mcsd_build_mask(parent)
    N, kids = tm.n_nodes, (4, 2, 2, 1)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    prompt = [100, 37]
    lens, freqs = _i32(prompt), 10000.0 ** (-torch.arange(P // 2, dtype=torch.float64, device="cuda") / (P // 2))
    caches = [torch.zeros(B, L_max, W, dtype=torch.bfloat16, device="cuda") for _ in range(layers)]
    weight = (1 + 0.1 * rnd(R)).bfloat16()
    for c in caches:
        m.mcsd_latent_rows(rnd(B, 100, W).bfloat16(), None, _i32([0, 0]), freqs, rows=c, n_active=lens, weight=weight)
    filters = lambda rows: dict(temperature=torch.full((rows,), 0.8, device="cuda"), top_k=torch.full((rows,), 60, dtype=torch.int32, device="cuda"),  # noqa: E731
                                top_p=torch.full((rows,), 0.95, device="cuda"))
    target = 2 * rnd(B, N, V)
    draft = target + 0.7 * rnd(B, N, V)
    tokens, q_rows = torch.zeros(B, N, dtype=torch.int32, device="cuda"), torch.zeros(B, N, V, device="cuda")
    ls = tm.level_start_host
    for level, k in enumerate(kids):
        lo, hi = int(ls[level]), int(ls[level + 1])
        rows = (hi - lo) * B
        t, p = m.mcsd_sample_candidates(draft[:, lo:hi].reshape(rows, V), torch.rand(rows, k, generator=g, device="cuda"), probs=True, **filters(rows))
        q_rows[:, lo:hi] = p.view(B, hi - lo, V)
        tokens[:, hi:hi + (hi - lo) * k] = t.view(B, (hi - lo) * k)
    leaf = int(ls[-2])
    q_rows[:, leaf:] = m.mcsd_sample_candidates(draft[:, leaf:].reshape(-1, V), probs=True, **filters(B * (N - leaf)))[0].view(B, N - leaf, V)
    (p_rows,) = m.mcsd_sample_candidates(target.view(-1, V), probs=True, **filters(B * N))
    p_rows = p_rows.view(B, N, V)
    drawn = q_rows[:, torch.as_tensor(np.maximum(parent, 0), device="cuda").long()].gather(2, tokens.long().unsqueeze(-1)).squeeze(-1)
    assert (drawn[:, 1:] > 0).all()                                     # every candidate was one that its parent's row keeps
    trees, outs = [], []
    for c in caches:
        q = rnd(B, H, N, W).bfloat16()
        rows = torch.zeros(B, N, W, dtype=torch.bfloat16, device="cuda")
        m.mcsd_latent_rows(rnd(B, N, W).bfloat16(), rnd(B, N, H, P).bfloat16(), lens, freqs, rows=rows, q=q, depth=tm.depth, weight=weight)
        outs.append(_attend(m, q, c, rows, prompt, None, tm, 0.07, R))
        _compare(outs[-1], q, c, rows, prompt, None, orc.dense_mask(parent), 0.07, R)
        trees.append(rows)
    u = lambda: torch.rand(B, N, generator=g, device="cuda")  # noqa: E731
    ver = m.mcsd_verify_tree(p_rows, q_rows, tokens, tm, None, u(), u())
    acc, nodes = ver["accept_len"].tolist(), ver["out_nodes"].tolist()
    for b in range(B):
        kept = p_rows[b, nodes[b][acc[b] - 1] if acc[b] else 0]
        assert kept[ver["out_tokens"][b, acc[b]]] > 0                   # the new token is one that the target's filters keep
    m.mcsd_commit_latent(m.layer_pointer_table(caches), m.layer_pointer_table(trees), lens, ver, tm, B, W, L_max, torch.bfloat16)
    assert lens.tolist() == [n + 1 + a for n, a in zip(prompt, acc)]
    one = m.mcsd_build_mask([-1])
    for c, t in zip(caches, trees):
        for b in range(B):
            path = [0] + nodes[b][: acc[b]]
            assert torch.equal(c[b, prompt[b]:prompt[b] + len(path)], t[b, path])
        q, rows = rnd(B, H, 1, W).bfloat16(), rnd(B, 1, W).bfloat16()
        out = _attend(m, q, c, rows, lens.tolist(), None, one, 0.07, R)
        _compare(out, q, c, rows, lens.tolist(), None, np.ones((1, 1), bool), 0.07, R)


def test_every_selected_path_is_documented(m):  # noqa: F811
    """Workspaces of every shape hold the larger of what the two kernels need, and grow with neither the cache's length nor the
    batch beyond what is cut among the multiprocessors."""
    w = m.mcsd_tree_attention_latent_workspace_bytes
    assert w(1, 16, 1, 512, 64, 1001, 0) > 0 and w(32, 32, 45, 512, 64, 32768, 0) <= 96 << 20
    assert w(8, 128, 1, 512, 64, 32001, 0) <= 96 << 20


# up to 16 query rows a sequence: every split of the keys, sequences of several waves, masks and inactive nodes
FEW = [(1, 16, "token", [1], None), (1, 16, "token", [63], None), (2, 16, "token", [64, 1023], None), (1, 16, "token", [4000], None),
       (3, 8, "two", [700, 0, 129], [2, 1, 2]), (5, 4, "fork3", [300, 64, 5, 0, 1000], [4, 3, 2, 1, 0]), (1, 1, "chain16", [900], None),
       (6, 16, "token", [9000, 0, 100, 5000, 1, 8999], [1, 1, 0, 1, 1, 1]), (1, 4, "fork3", [21000], [3]),
       (130, 5, "token", [(37 * i) % 500 for i in range(130)], None), (40, 16, "token", [(97 * i) % 900 for i in range(40)], None)]
FEW_TREES = {"token": [-1], "two": [-1, -1], "fork3": [-1, 0, 0, 0], "chain16": list(range(-1, 15))}


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,tree,lens,act", FEW)
def test_few_rows(m, B, H, tree, lens, act):  # noqa: F811
    parent = np.array(FEW_TREES[tree], dtype=np.int32)
    q, cache, rows = _problem(50 + B, "bf16", B, H, 512, 64, parent, lens)
    for b, L in enumerate(lens):
        cache[b, L:] = NAN
        if act is not None:
            rows[b, act[b]:] = NAN
            q[b, :, act[b]:] = NAN
    tm = m.mcsd_build_mask(parent)
    out = _attend(m, q, cache, rows, lens, act, tm, 0.07, 512)
    _compare(out, q, cache, rows, lens, act, orc.dense_mask(parent), 0.07, 512, None if B < 10 else [0, H - 1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = _attend(m, q, cache, rows, lens, act, tm, 0.07, 512)
    s.synchronize()
    assert torch.equal(out.nan_to_num(7.0), again.nan_to_num(7.0))


@pytest.mark.gpu
def test_few_rows_that_see_nothing_and_growing_scores(m):  # noqa: F811
    parent = np.array(FEW_TREES["fork3"], dtype=np.int32)
    tm, see = m.mcsd_build_mask(parent), orc.dense_mask(parent).copy()
    q, cache, rows = _problem(60, "bf16", 2, 4, 512, 64, parent, [0, 1500])
    cache = (cache.float() * torch.linspace(0.01, 3.0, cache.shape[1], device="cuda")[None, :, None]).bfloat16()
    tm.anc[2] = 0
    see[2] = False
    out = _attend(m, q, cache, rows, [0, 1500], None, tm, 0.07, 512)
    assert (out[0, :, 2] == 0).all()
    _compare(out, q, cache, rows, [0, 1500], None, see, 0.07, 512)


@pytest.mark.gpu
def test_few_rows_captured(m):  # noqa: F811
    """The choice of kernel goes by L_max, the split of the keys by the lengths a replay finds."""
    tm = m.mcsd_build_mask(np.array(FEW_TREES["token"], dtype=np.int32))
    q, cache, rows = _problem(70, "bf16", 3, 16, 512, 64, [-1], [1500] * 3)
    lens, act = _i32([1500, 0, 3]), _i32([1, 1, 1])
    out = torch.full((3, 16, 1, 512), NAN, dtype=torch.bfloat16, device="cuda")
    ws = m.new_workspace(m.mcsd_tree_attention_latent_workspace_bytes(3, 16, 1, 512, 64, 1500, 0), "cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        m.mcsd_tree_attention_latent(q, cache, rows, lens, act, tm, 0.07, out=out, workspace=ws)
    for L, a in (([1500, 0, 3], [1, 1, 1]), ([64, 1023, 1025], [1, 0, 1]), ([0, 0, 0], [0, 0, 0]), ([1, 1500, 700], [1, 1, 1])):
        lens.copy_(_i32(L))
        act.copy_(_i32(a))
        out.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        _compare(out, q, cache, rows, L, a, np.ones((1, 1), bool), 0.07, 512)
    assert m.mcsd_workspace_status(ws) == 0
