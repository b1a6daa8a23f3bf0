"""Barriers that a whole warp has to reach together (`.aligned`, and `bar.sync`, which is) are written by hand in some kernels.  The
instruction leaves it to the program that the lanes are together, so each of them follows a __syncwarp() or __syncthreads()."""
import os
import re

import numpy as np
import pytest
import torch

from mcsd_inputs import parent_array
from oracle import latent_oracle as lat
from tests.test_kv4 import m  # noqa: F401  (the fixture)

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2409_10644_b200", "csrc")


def _unguarded(text):
    """Lines with a hand-written warp-wide barrier whose last statement before it is not one that brings the lanes together."""
    text = re.sub(r"/\*.*?\*/", lambda c: "\n" * c.group().count("\n"), text, flags=re.S)
    lines, bad, before = [re.sub(r"//.*", "", line).strip() for line in text.split("\n")], [], ""
    for i, line in enumerate(lines):
        if re.search(r'"bar(rier\.cluster\.(arrive|wait)[a-z.]*\.aligned|\.sync )', line):
            here = line[:line.index("asm")].strip()
            if not re.search(r"__sync(warp|threads)\(\);( *\{)?$", here or before) and not before.startswith("cg::this_cluster().sync()"):
                bad.append(i + 1)
        if line:
            before = line
    return bad


def test_the_check_finds_what_it_looks_for():
    assert _unguarded('for (;;) {}\n  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");') == [2]
    assert _unguarded('x();\n__syncwarp();  // y\n\nasm volatile("bar.sync 1, 256;" ::: "memory");') == []


@pytest.mark.parametrize("name", ["latent_rows.cu", "sample.cu", "attention_latent_tc.cu"])
def test_barriers_of_a_warp_follow_a_meeting_of_its_lanes(name):
    assert _unguarded(open(os.path.join(CSRC, name)).read()) == []


@pytest.mark.gpu
@pytest.mark.parametrize("layers,B,width,accept", [(1, 1, 48, 0), (9, 3, 80, 2), (17, 2, 560, 4), (33, 5, 112, 1)])
def test_commit_with_lanes_that_leave_at_different_times(m, layers, B, width, accept):  # noqa: F811
    """A block's vectors are no multiple of a warp, so that its lanes leave the copying loop after different trips."""
    tm, L_max = m.mcsd_build_mask(parent_array(1, (4, 2, 2, 1))), 20
    g = torch.Generator("cuda").manual_seed(layers)
    caches = [torch.randn(B, L_max, width, generator=g, device="cuda").bfloat16() for _ in range(layers)]
    trees = [torch.randn(B, tm.n_nodes, width, generator=g, device="cuda").bfloat16() for _ in range(layers)]
    path = [1, 5, 13, 29][:accept]
    want, lens = [c.clone() for c in caches], torch.arange(B, dtype=torch.int32, device="cuda")
    for w, t in zip(want, trees):
        for b in range(B):
            w[b, b:b + 1 + accept] = t[b, [0] + path]
    nodes = torch.tensor([path + [-1] * (tm.n_levels - accept)] * B, dtype=torch.int32, device="cuda")
    full = lambda x: torch.full((B,), x, dtype=torch.int32, device="cuda")  # noqa: E731
    m.mcsd_commit_latent(m.layer_pointer_table(caches), m.layer_pointer_table(trees), lens, dict(accept_len=full(accept), out_nodes=nodes, best_root=full(0)),
                         tm, B, width, L_max, torch.bfloat16)
    assert all(torch.equal(a, b) for a, b in zip(caches, want)) and lens.tolist() == [b + 1 + accept for b in range(B)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V", [(1, 8197), (3, 16391), (2, 50001)])
@pytest.mark.parametrize("top_k", [0, 7])
def test_probabilities_with_lanes_that_leave_at_different_times(m, rows, V, top_k):  # noqa: F811
    """Few rows are shared by a cluster of blocks, whose parts are no multiple of what its threads write at a time."""
    logits = 2 * torch.randn(rows, V, generator=torch.Generator("cuda").manual_seed(V), device="cuda")
    (probs,) = m.mcsd_sample_candidates(logits, top_k=torch.full((rows,), top_k, dtype=torch.int32, device="cuda"), probs=True)
    for r in range(rows):
        want, _ = lat.filtered(logits[r].cpu().numpy(), 1.0, top_k)
        # weights: 2^-21 (exponential and its argument); their sum: half a step of 2^-31 of the largest a token, which is at most
        # the sum itself; a scale and a product in 32 bits
        err = np.abs(probs[r].cpu().numpy() - want)
        assert (err <= (2.0 ** -20 + V * 2.0 ** -32) * want + 2.0 ** -32).all()
