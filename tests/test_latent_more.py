"""Operators over a latent cache: calls of several host threads, and what the shapes and lengths of other tests leave out."""
import threading

import numpy as np
import pytest
import torch

from mcsd_inputs import parent_array
from oracle import mcsd_oracle as orc
from tests.test_kv4 import m  # noqa: F401  (the fixture)
from tests.test_latent import NAN, TREES, _attend, _compare, _i32, _problem


@pytest.mark.gpu
def test_two_host_threads_with_different_widths(m):  # noqa: F811
    """One kernel serves many widths, whose blocks take different amounts of shared memory: what one thread's call asks for must not
    take from another's that is about to launch."""
    parent = parent_array(*TREES["binary"])
    tm, lens, errors, done = m.mcsd_build_mask(parent), [40], [], []

    def work(rank, rot, seed):
        try:
            q, cache, rows = _problem(seed, "f32", 1, 2, rank, rot, parent, lens)
            ln, out = _i32(lens), torch.full((1, 2, len(parent), rank), NAN, device="cuda")
            ws = m.new_workspace(m.mcsd_tree_attention_latent_workspace_bytes(1, 2, len(parent), rank, rot, 40, m.MCSD_F32), "cuda")
            with torch.cuda.stream(torch.cuda.Stream()):
                torch.cuda.current_stream().wait_stream(torch.cuda.default_stream())
                for _ in range(3000):
                    m.mcsd_tree_attention_latent(q, cache, rows, ln, None, tm, 0.07, out=out, workspace=ws)
                torch.cuda.current_stream().synchronize()
            done.append((out, q, cache, rows, rank))
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=a) for a in ((512, 128, 1), (288, 0, 2), (512, 64, 3), (320, 0, 4))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for out, q, cache, rows, rank in done:
        _compare(out, q, cache, rows, lens, None, orc.dense_mask(parent), 0.07, rank)
