"""mcsd_qk_norm_rope: norm of query and key heads, rotation by position and the change to head-major rows, against the
definition in 64 bits; and its refusals."""
import ctypes

import numpy as np
import pytest
import torch

from mcsd_inputs import parent_array
from oracle import kv4_oracle as kv4
from tests.helpers import to_np

FAKE = ctypes.c_void_p(0x1000)      # never dereferenced: every call that uses it fails its checks first


@pytest.fixture(scope="module")
def m():
    from paper_2409_10644_b200 import build
    build.build()
    import paper_2409_10644_b200 as pkg
    return pkg


def test_refusals(m):
    strides = (ctypes.c_int64 * 6)(*[1024] * 6)

    def call(q=FAKE, st=strides, freqs=FAKE, rot=64, inter=0, lens=FAKE, B=1, Hq=4, Hkv=2, N=5, D=128, dtype=0, eps=1e-6, out=FAKE):
        return m.lib.mcsd_qk_norm_rope(q, FAKE, FAKE, st, None, None, ctypes.c_float(eps), freqs, rot, inter, lens, None, None, out,
                                       FAKE, FAKE, B, Hq, Hkv, N, D, dtype, None)
    assert call(q=None) == -1
    assert call(st=None) == -1
    assert call(freqs=None) == -1
    assert call(lens=None) == -1
    assert call(out=None) == -1
    assert call(dtype=2) == -4
    assert call(D=96) == -2
    assert call(rot=130) == -2
    assert call(rot=-2) == -2
    assert call(rot=63) == -2
    assert call(rot=24) == -2                # half-split rotations come in multiples of 16
    assert call(rot=25, inter=1) == -2
    assert call(B=0) == -2
    assert call(N=0) == -2
    assert call(Hq=0) == -2
    assert call(Hkv=0) == -2
    assert call(B=1 << 16, N=1 << 15) == -2
    assert call(eps=-1.0) == -2
    assert call(eps=float("nan")) == -2


def test_binding_refuses_tensors_it_cannot_pass_on(m):
    x = torch.zeros(1, 3, 4, 128, dtype=torch.bfloat16)
    lens = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        m.mcsd_qk_norm_rope(x, x, x, lens, None)                                  # not on a GPU
    with pytest.raises(ValueError):
        m.mcsd_qk_norm_rope(x.half(), x.half(), x.half(), lens, None)
    with pytest.raises(ValueError):
        m.mcsd_qk_norm_rope(x, x[:, :2], x, lens, None)


def _case(m, dtype, B, N, Hq, Hkv, D, rot, interleaved, norm, pos, depth, sliced, layout, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    H = Hq + 2 * Hkv
    if layout == "fused":
        x = torch.randn((B, N, H, D), generator=g, device="cuda").to(dtype)
        q_in, k_in, v_in = x.split([Hq, Hkv, Hkv], dim=2)
    elif layout == "odd":                    # rows that start off 16-byte boundaries
        x = torch.randn((B, N, H * D + 3), generator=g, device="cuda").to(dtype)
        parts = x[..., 1:1 + H * D].unflatten(2, (H, D))
        q_in, k_in, v_in = parts.split([Hq, Hkv, Hkv], dim=2)
    else:                                    # token-major over the batch: strides of their own
        q_in, k_in, v_in = (torch.randn((N, B, h, D), generator=g, device="cuda").to(dtype).transpose(0, 1) for h in (Hq, Hkv, Hkv))
    wq, wk = ((1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dtype) if norm & bit else None for bit in (1, 2))
    lens = torch.tensor([pos + 7 * b for b in range(B)], dtype=torch.int32, device="cuda")
    freqs = None if rot == 0 else 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device="cuda") / (rot // 2))
    act = torch.tensor([(N * (b + 1)) // (B + 1) for b in range(B)], dtype=torch.int32, device="cuda") if sliced else None
    out = tuple(torch.full((B, h, N, D), float("nan"), dtype=dtype, device="cuda") for h in (Hq, Hkv, Hkv))
    got = m.mcsd_qk_norm_rope(q_in, k_in, v_in, lens, freqs, depth=depth, n_active=act, q_weight=wq, k_weight=wk, eps=1e-5,
                              interleaved=interleaved, out=out)
    torch.cuda.synchronize()
    d = np.arange(N) if depth is None else depth.cpu().numpy()
    positions = lens.cpu().numpy()[:, None].astype(np.int64) + d[None, :]
    f = np.zeros(0) if freqs is None else freqs.cpu().numpy()
    # One rounding to the output type (half a step: 2^-8 or 2^-24 of the value).  Before it, in fp32: the mean of D squares
    # (at most 16 roundings deep, halved by the root), the root, two products and the weight's, i.e. under 16 * 2^-24;
    # the angle's fraction of a turn is rounded to fp32 (pi * 2^-24) and sine and cosine are good to 2 steps; the
    # rotation rounds three times.  Together under 32 * 2^-24 = 2^-19 of |y_a| + |y_c|.
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for x_in, w, y, rotate in ((q_in, wq, got[0], True), (k_in, wk, got[1], True), (v_in, None, got[2], False)):
        ref, size = kv4.norm_rope(to_np(x_in), None if w is None else to_np(w), 1e-5, f, positions, interleaved, rotate)
        y = to_np(y).astype(np.float64)
        for b in range(B):
            n = N if act is None else int(act[b])
            err = np.abs(y[b, :, :n] - ref[b, :, :n])
            assert (err <= step * np.abs(ref[b, :, :n]) + 2.0 ** -19 * size[b, :, :n] + 1e-40).all(), (b, err.max())
            assert np.isnan(y[b, :, n:]).all()           # rows past the active ones are left as they were


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("layout", ["fused", "odd", "own"])
def test_rows_match_the_definition(m, dtype, D, interleaved, layout):
    for i, (B, N, Hq, Hkv, rot, norm, pos, sliced) in enumerate((
            (1, 1, 1, 1, D, 3, 0, False), (1, 1, 32, 8, D, 3, 1000, False), (3, 5, 6, 2, D // 2, 1, 131071, True),
            (2, 33, 3, 3, 16, 2, 2 ** 31 - 100, False), (2, 9, 5, 1, 0, 3, 7, False), (1, 400, 4, 4, D, 0, 12345, True))):
        _case(m, dtype, B, N, Hq, Hkv, D, rot, interleaved, norm, pos, None, sliced, layout, 100 + i)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tree_rows_take_their_depth(m, dtype):
    tm = m.mcsd_build_mask(parent_array(8, (1, 2, 2, 1, 1, 1)))
    _case(m, dtype, 2, tm.n_nodes, 4, 2, 128, 128, False, 3, 4000, tm.depth, True, "fused", 1)


@pytest.mark.gpu
def test_interleaved_rotation_of_any_even_width(m):
    for rot in (2, 6, 30, 126):
        _case(m, torch.float32, 2, 4, 3, 1, 128, rot, True, 3, 500, None, False, "fused", rot)


@pytest.mark.gpu
def test_rows_of_zeros_and_non_finite_rows_stay_in_their_head(m):
    x = torch.randn(1, 2, 3, 128, device="cuda")
    x[0, 0, 0] = 0
    x[0, 1, 1, 5] = float("nan")
    w = torch.ones(128, device="cuda")
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    q, k, v = m.mcsd_qk_norm_rope(x, x, x, lens, None, q_weight=w, k_weight=None, eps=1e-6)
    assert (q[0, 0, 0] == 0).all() and torch.isnan(q[0, 1, 1]).all()
    assert torch.isfinite(q[0, 0]).all() and torch.isfinite(q[0, 1, 0]).all() and torch.isfinite(q[0, 2]).all()
    assert torch.equal(k.nan_to_num(7), x.transpose(1, 2).nan_to_num(7)) and torch.equal(v.nan_to_num(7), x.transpose(1, 2).nan_to_num(7))


@pytest.mark.gpu
def test_another_stream_and_a_captured_call(m):
    B, N, H, D = 2, 6, 4, 128
    x = torch.randn(B, N, 3 * H, D, device="cuda").bfloat16()
    q_in, k_in, v_in = x.split(H, dim=2)
    lens = torch.tensor([3, 50], dtype=torch.int32, device="cuda")
    freqs = 10000.0 ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
    want = m.mcsd_qk_norm_rope(q_in, k_in, v_in, lens, freqs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = m.mcsd_qk_norm_rope(q_in, k_in, v_in, lens, freqs)
    side.synchronize()
    out = tuple(torch.empty_like(t) for t in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.mcsd_qk_norm_rope(q_in, k_in, v_in, lens, freqs, out=out)
    lens += 1                                # a replay reads what the tensors hold then
    graph.replay()
    moved = m.mcsd_qk_norm_rope(q_in, k_in, v_in, lens, freqs)
    torch.cuda.synchronize()
    for a, b, c, d in zip(want, other, out, moved):
        assert torch.equal(a, b) and torch.equal(c, d)
    assert not torch.equal(want[0], moved[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_many_tokens_over_sequence_boundaries(m, dtype, interleaved):
    for D, rot, sliced in ((64, 64, True), (128, 32, True), (128, 128, False)):
        _case(m, dtype, 3, 401, 3, 2, D, rot, interleaved, 3, 777, None, sliced, "fused", D + rot)
