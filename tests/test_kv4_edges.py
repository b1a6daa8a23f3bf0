"""Attention over the 4-bit cache where one call could disturb another: a workspace that several kernels use in turn."""
import numpy as np
import pytest
import torch

from mcsd_inputs import parent_array
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
