"""Candidates from logits: calls that the contract allows and other tests do not make."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import latent_oracle as orc
from tests.test_kv4 import m  # noqa: F401  (the fixture)

FAKE = ctypes.c_void_p(0x1000)      # never dereferenced: every call that uses it fails its checks first


def _call(m, logits=FAKE, stride=100, rows=2, V=100, K=3, u=FAKE, tokens=FAKE, probs=FAKE, stream=None):  # noqa: F811
    return m.lib.mcsd_sample_candidates(logits, stride, m.MCSD_F32, rows, V, None, None, None, None, u, K, tokens, probs, stream)


def test_the_number_of_draws_is_checked_where_there_are_draws(m):  # noqa: F811
    for K in (-1, 0, 1025, 1 << 30):
        assert _call(m, K=K) == -2, K
    assert _call(m, K=-1, u=None, tokens=None) == -2


@pytest.mark.gpu
@pytest.mark.parametrize("K", [0, 1, 1024, 1025, 1 << 30])
def test_probabilities_alone_take_any_number_of_draws(m, K):  # noqa: F811
    x = torch.randn(2, 100, device="cuda")
    probs = torch.full((2, 100), -1.0, device="cuda")
    st = _call(m, logits=x.data_ptr(), K=K, u=None, tokens=None, probs=probs.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
    assert st == 0
    (want,) = m.mcsd_sample_candidates(x, probs=True)
    assert torch.equal(probs, want)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V", [(1, 9001), (150, 4001)])
@pytest.mark.parametrize("k", [257, 600, 2560, 2561])
@pytest.mark.parametrize("steps", [0.001, 0.25])
def test_top_k_alone_beyond_the_short_list(m, rows, V, k, steps):  # noqa: F811
    """The kept tokens, to the token: distinct logits, and logits of which many are equal at the cut."""
    x = 2 * torch.randn(rows, V, generator=torch.Generator("cuda").manual_seed(k), device="cuda")
    x = torch.round(x / steps) * steps
    (probs,) = m.mcsd_sample_candidates(x, top_k=torch.full((rows,), k, dtype=torch.int32, device="cuda"), probs=True)
    for r in range(0, rows, 29):
        want, _ = orc.filtered(x[r].cpu().numpy(), 1.0, k)
        got = probs[r].cpu().numpy()
        assert ((got > 0) == (want > 0)).all() and (got > 0).sum() == k
        # weights 2^-21, a sum of k of them in steps of 2^-31 of the largest, a scale and a product
        assert (np.abs(got - want) <= (2.0 ** -20 + k * 2.0 ** -32) * want).all()


@pytest.mark.gpu
def test_tokens_lighter_than_half_a_step(m):  # noqa: F811
    """Sums are whole numbers of 2^-31 of the largest weight: exp(-23) is less than half of that and is never drawn, but has its
    probability; exp(-21) is 1.6 of it and is drawn."""
    V = 5000
    x = torch.full((2, V), -23.0, device="cuda")
    x[:, 7] = 0.0
    x[1, 4001:] = -21.0
    u = torch.tensor([[0.0, 0.5, 1 - 2.0 ** -24, 0.25]] * 2, device="cuda")
    tokens, probs = m.mcsd_sample_candidates(x, u, probs=True)
    assert tokens[0].tolist() == [7, 7, 7, 7]
    assert tokens[1, [0, 1, 3]].tolist() == [7, 7, 7] and tokens[1, 2] > 4000
    # 999 tokens of 2 steps each behind 2^31, S steps in all: (1 - 2^-24) S is S - 128.0001, and the first running sum above that is
    # S - 128, with 64 tokens left behind it
    assert tokens[1, 2] == V - 1 - 64
    for r in range(2):
        w = np.exp(x[r].double().cpu().numpy())
        got = probs[r].cpu().numpy()
        # half a step for every token of the sum, in the scale
        assert (got > 0).all() and (np.abs(got - w / w.sum()) <= (2.0 ** -20 + V * 2.0 ** -32) * w / w.sum()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V", [(2, 262144), (150, 20001)])
@pytest.mark.parametrize("top_p", [0.25, 0.9])
def test_a_cut_among_weights_that_are_added_up_approximately(m, rows, V, top_p):  # noqa: F811
    """Most of the mass lies in tokens below 2^-9.5 of the largest.  What is kept is a beginning of the order whose mass
    reaches top_p, to what the weights of filters are off by: 3 roundings of the exponent, 3 * 2^-24 * ln 2 * 32, and 2^-22 of the
    exponential, at most 4.5e-6 of a mass on either side, and half a step of 2^-31 a token."""
    x = torch.randn(rows, V, generator=torch.Generator("cuda").manual_seed(V), device="cuda") - 10.0
    x[:, 11] = 0.0
    (probs,) = m.mcsd_sample_candidates(x, top_p=torch.full((rows,), top_p, device="cuda"), probs=True)
    share = float(np.float32(top_p))
    for r in range(0, rows, 37):
        l = x[r].double().cpu().numpy()
        order = np.lexsort((np.arange(V), -l))
        kept = (probs[r].cpu().numpy() > 0)[order]
        n = int(kept.sum())
        assert kept[:n].all()
        c = np.cumsum(np.exp(l[order] - l.max()))
        tol = 2 * 4.5e-6 + V * 2.0 ** -32 / c[-1]
        assert c[n - 1] >= (share - tol) * c[-1] and (c[n - 2] if n > 1 else 0.0) < (share + tol) * c[-1]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V", [(1, 8), (3, 4093), (18, 32000), (160, 9000), (2, 131071)])
@pytest.mark.parametrize("top_p", [None, -1.0, 0.1, 0.9])
def test_a_negative_top_k_is_off(m, rows, V, top_p):  # noqa: F811
    """With every other filter, as without one."""
    g = torch.Generator("cuda").manual_seed(V)
    x, u = 3 * torch.randn(rows, V, generator=g, device="cuda"), torch.rand(rows, 5, generator=g, device="cuda")
    f32 = lambda v: None if v is None else torch.full((rows,), v, device="cuda")  # noqa: E731
    for kw in (dict(), dict(min_p=f32(0.02)), dict(temperature=f32(1.3)), dict(temperature=f32(0.0))):
        want = m.mcsd_sample_candidates(x, u, top_p=f32(top_p), probs=True, **kw)
        for k in (-1, -3, -(1 << 31), 0):
            got = m.mcsd_sample_candidates(x, u, top_k=torch.full((rows,), k, dtype=torch.int32, device="cuda"), top_p=f32(top_p), probs=True, **kw)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), k
