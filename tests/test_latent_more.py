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


# ---------------------------------------------------------------------------------------------- pieces that are joined by others

COUNTERS = slice(256, 256 + 160 * 4 * 4)                              # of a workspace: zero between launches


def _pieces(H, nodes, lens, pairs):
    """How many pieces the items of a launch on tensor memory are cut into (its rule of cutting, said again)."""
    cost = lambda keys: 6 + -(-4 * keys // 256)  # noqa: E731
    shapes = []
    for L, n in zip(lens, nodes):
        tiles = [10] * (L // 256) + ([cost(L % 256)] if L % 256 else []) + [10] * (n // 256) + ([cost(n % 256)] if n % 256 else [])
        shapes += [tiles] * (-(-H * n // 128))
    total, items = sum(14 + sum(t) for t in shapes), len(shapes)
    pairs = max(min(pairs, total // 10), 1)
    few = min(3 * items, pairs)
    if pairs > few and total // few <= total // pairs + 25:
        pairs = few
    owner = lambda u: ((u + 1) * pairs - 1) // total  # noqa: E731
    unit, out = 0, []
    for t in shapes:
        out.append(owner(unit + 14 + sum(t[:-1])) - owner(unit + 14) + 1)
        unit += 14 + sum(t)
    return out


JOINS = {"many": (1, 128, "token", [30000]), "about_ten": (8, 128, "token", [32001 - 1999 * i for i in range(8)]),
         "two_to_four": (30, 128, "token", [4000 - 57 * i for i in range(30)]), "trees": (5, 24, "static", [6000, 300, 2500, 0, 4096]),
         "all_sorts": (6, 128, "token", [30000, 40, 9000, 1, 5000, 300])}


def test_the_joins_cases_hold_every_number_of_pieces():
    seen = {name: set(_pieces(H, [len(parent_array(*TREES[tree]))] * B, lens, 74)) for name, (B, H, tree, lens) in JOINS.items()}
    assert seen["many"] == {74} and set(range(9, 13)) <= seen["about_ten"] and {2, 3, 4} == seen["two_to_four"]
    assert {1, 2, 3, 4, 5} <= seen["trees"] and {1, 47} <= seen["all_sorts"]


def test_patience_is_bounded(m):  # noqa: F811
    assert m.lib.mcsd_selftest_latent_patience((1 << 21) + 1) == -2
    m.mcsd_selftest_latent_patience(1 << 21)
    m.mcsd_selftest_latent_patience()


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(JOINS))
def test_pieces_that_are_not_waited_for(m, name):  # noqa: F811
    """Pairs that give up at once, soon, or while some pieces are in: what they leave is joined by the pair of the last piece, with
    the same result, and the counters are zero for the next launch."""
    B, H, tree, lens = JOINS[name]
    parent = parent_array(*TREES[tree])
    tm = m.mcsd_build_mask(parent)
    q, cache, rows = _problem(80 + B, "bf16", B, H, 512, 64, parent, lens)
    for b, L in enumerate(lens):
        cache[b, L:] = NAN
    ws = m.new_workspace(m.mcsd_tree_attention_latent_workspace_bytes(B, H, len(parent), 512, 64, cache.shape[1], m.MCSD_BF16), "cuda")
    want = _attend(m, q, cache, rows, lens, None, tm, 0.07, 512, ws)
    _compare(want, q, cache, rows, lens, None, orc.dense_mask(parent), 0.07, 512, [0, H // 2, H - 1])
    assert not ws[COUNTERS].any()
    try:
        for cycles in (0, 300, 1000, 3000, 10000, 30000):
            m.mcsd_selftest_latent_patience(cycles)
            for _ in range(4):
                out = _attend(m, q, cache, rows, lens, None, tm, 0.07, 512, ws)
                assert torch.equal(out, want), cycles
                assert not ws[COUNTERS].any(), cycles
    finally:
        m.mcsd_selftest_latent_patience()
    assert torch.equal(_attend(m, q, cache, rows, lens, None, tm, 0.07, 512, ws), want)


@pytest.mark.gpu
def test_pieces_that_are_not_waited_for_next_to_another_stream(m):  # noqa: F811
    """Short patience while another stream's calls hold multiprocessors: some pairs wait long enough, some do not."""
    cases = []
    for name in ("many", "two_to_four", "trees"):
        B, H, tree, lens = JOINS[name]
        parent = parent_array(*TREES[tree])
        cases.append((*_problem(90 + B, "bf16", B, H, 512, 64, parent, lens), _i32(lens), m.mcsd_build_mask(parent)))
    size = max(m.mcsd_tree_attention_latent_workspace_bytes(*c[0].shape[:3], 512, 64, c[1].shape[1], m.MCSD_BF16) for c in cases)
    spaces = [m.new_workspace(size, "cuda") for _ in range(2)]
    call = lambda c, ws, out: m.mcsd_tree_attention_latent(*c[:4], None, c[4], 0.07, out=out, workspace=ws)  # noqa: E731
    want = [call(c, spaces[0], torch.empty(*c[0].shape[:3], 512, dtype=torch.bfloat16, device="cuda")) for c in cases]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream(), torch.cuda.Stream(priority=-1)], []
    try:
        for i in range(24):
            m.mcsd_selftest_latent_patience((0, 2000, 20000, 200000)[i % 4])
            for k, s in enumerate(streams):
                with torch.cuda.stream(s):
                    j = (i + k) % 3
                    outs.append((j, call(cases[j], spaces[k], torch.full_like(want[j], NAN))))
    finally:
        m.mcsd_selftest_latent_patience()
    torch.cuda.synchronize()
    assert [m.mcsd_workspace_status(ws) for ws in spaces] == [0, 0] and not any(ws[COUNTERS].any() for ws in spaces)
    for j, out in outs:
        assert torch.equal(out, want[j])
