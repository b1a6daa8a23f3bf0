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
