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
