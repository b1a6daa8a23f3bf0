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


# ---------------------------------------------------------------------------------------------- kernels, lengths, workspaces

def test_path_refusals_and_shapes_that_need_no_device(m):  # noqa: F811
    path = m.lib.mcsd_tree_attention_latent_path
    assert path(0, 4, 15, 512, 64, 100, 0, None) == -2
    assert path(1, 4, 193, 512, 64, 100, 0, None) == -2
    assert path(1, 4, 15, 500, 64, 100, 0, None) == -2
    assert path(1, 4, 15, 512, 64, -1, 0, None) == -2
    assert path(1, 4, 15, 512, 64, 100, 2, None) == -4
    assert m.mcsd_tree_attention_latent_path(1, 4, 15, 512, 64, 100, m.MCSD_F32) == (0, 4)       # 115 keys: four tiles of 32
    assert m.mcsd_tree_attention_latent_path(2, 32, 45, 512, 64, 4096, m.MCSD_BF16) == (1, 0)
    assert m.mcsd_tree_attention_latent_path(1, 4, 15, 256, 64, 100, m.MCSD_BF16)[0] == 0
    with pytest.raises(m.McsdError):
        m.mcsd_tree_attention_latent_path(1, 0, 15, 512, 64, 100, m.MCSD_BF16)


# dtype, B, H, rank, rot, tree, rows of the cache, lengths, kernel (0 CUDA cores, 1 tensor cores, 2 few rows), least and most splits
KERNELS = {
    "few_small": ("bf16", 100, 16, 512, 64, "token", 200, [(31 * i) % 201 for i in range(100)], 2, 1, 2),
    "few_cluster": ("bf16", 1, 16, 512, 64, "token", 1000, [1000], 2, 9, 16),
    "few_no_cache": ("bf16", 2, 4, 512, 64, "token", 0, [0, 0], 2, 1, 16),
    "few_memory": ("bf16", 1, 16, 512, 64, "token", 20000, [20000], 2, 17, 160),
    "few_memory_short": ("bf16", 1, 16, 512, 64, "token", 131072, [500], 2, 17, 160),
    "few_memory_empty": ("bf16", 2, 8, 512, 64, "token", 131072, [0, 1], 2, 17, 160),
    "tensor": ("bf16", 2, 32, 512, 64, "static", 1500, [1500, 200], 1, 0, 0),
    "tensor_short": ("bf16", 2, 32, 512, 64, "static", 65536, [300, 0], 1, 0, 0),
    "tensor_two_launches": ("bf16", 300, 20, 512, 64, "token", 270, [(83 * i) % 271 for i in range(300)], 1, 0, 0),
    "cuda_cluster": ("f32", 2, 3, 128, 32, "binary", 131, [131, 30], 0, 2, 8),
    "cuda_memory": ("f32", 1, 2, 512, 64, "token", 3000, [3000], 0, 9, 296),
    "cuda_memory_short": ("f32", 1, 2, 128, 32, "token", 131072, [500], 0, 9, 296),
    "cuda_memory_bf16": ("bf16", 1, 4, 256, 64, "binary", 131072, [33], 0, 9, 296),
    "cuda_memory_empty": ("f32", 2, 2, 32, 16, "binary", 70000, [0, 70000], 0, 9, 296),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(KERNELS))
def test_kernels_by_name_and_workspaces_to_the_byte(m, name):  # noqa: F811
    """Each way that the keys are divided, lengths far below the cache's among them, in a workspace of the size that is asked for,
    whose surroundings stay as they were."""
    dtype, B, H, rank, rot, tree, L_max, lens, kernel, least, most = KERNELS[name]
    parent = parent_array(*TREES[tree])
    code = m.MCSD_BF16 if dtype == "bf16" else m.MCSD_F32
    shape = (B, H, len(parent), rank, rot, L_max, code)
    path, splits = m.mcsd_tree_attention_latent_path(*shape)
    assert path == kernel and least <= splits <= most, (path, splits)
    q, cache, rows = _problem(100 + B + L_max, dtype, B, H, rank, rot, parent, [max(L_max, 1)])
    cache = cache[:, :L_max]
    for b, L in enumerate(lens):
        cache[b, L:] = NAN
    tm, need = m.mcsd_build_mask(parent), m.mcsd_tree_attention_latent_workspace_bytes(*shape)
    space = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    ws = space[:need]
    ws.zero_()
    out = _attend(m, q, cache, rows, lens, None, tm, 0.07, rank, ws)
    _compare(out, q, cache, rows, lens, None, orc.dense_mask(parent), 0.07, rank, None if B * H <= 32 else [0, H - 1])
    assert (space[need:] == 0xA5).all() and not ws[COUNTERS].any()
    space[256 + 160 * 16:need] = 0xFF                                  # scratch may hold anything between launches
    assert torch.equal(_attend(m, q, cache, rows, lens, None, tm, 0.07, rank, ws), out)
    assert (space[need:] == 0xA5).all()


@pytest.mark.gpu
def test_every_number_of_blocks_that_few_rows_are_divided_among(m):  # noqa: F811
    """Batches from one sequence up to more than there are multiprocessors: clusters small and large, with and without keys for all."""
    tm, L_max, seen = m.mcsd_build_mask([-1]), 700, {}
    for B in range(1, 301):
        path, splits = m.mcsd_tree_attention_latent_path(B, 3, 1, 512, 64, L_max, m.MCSD_BF16)
        if path == 2:
            seen.setdefault(splits, B)
    assert {1, 2, 3, 4, 16} <= set(seen) and any(5 <= s <= 8 for s in seen) and any(9 <= s <= 15 for s in seen), seen
    for splits, B in seen.items():
        lens = [(149 * i + 11 * splits) % (L_max + 1) for i in range(B)]
        q, cache, rows = _problem(200 + splits, "bf16", B, 3, 512, 64, [-1], [L_max])
        for b, L in enumerate(lens):
            cache[b, L:] = NAN
        out = _attend(m, q, cache, rows, lens, None, tm, 0.07, 512)
        _compare(out, q, cache, rows, lens, None, np.ones((1, 1), bool), 0.07, 512, [0, 2])


def test_an_output_without_its_input_is_refused(m):  # noqa: F811
    rows, q, lens = torch.zeros(1, 3, 96), torch.zeros(1, 2, 3, 96), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="latent_in"):
        m.mcsd_latent_rows(None, None, lens, None, rows=rows)
    with pytest.raises(ValueError, match="q_in"):
        m.mcsd_latent_rows(None, None, lens, None, q=q)
    with pytest.raises(ValueError, match="q_in"):
        m.mcsd_latent_rows(rows, None, lens, None, rows=rows.clone(), q=q)
    with pytest.raises(ValueError, match="latent_in"):
        m.mcsd_latent_rows(None, q[..., :32], lens, torch.zeros(16, dtype=torch.float64), rows=rows, q=q)


@pytest.mark.gpu
def test_captured_where_pieces_go_through_memory(m):  # noqa: F811
    """Two graphs that share a workspace, of few rows and of the CUDA cores' kernel, replayed in turn with lengths that change: the joining
    kernel is launched early and has to find the pieces of its own replay."""
    tm, ws, graphs, s = m.mcsd_build_mask([-1]), torch.zeros(64 << 20, dtype=torch.uint8, device="cuda"), [], torch.cuda.Stream()
    for dtype, rank, rot, H, L_max in (("bf16", 512, 64, 16, 20000), ("f32", 128, 32, 2, 6000)):
        path, splits = m.mcsd_tree_attention_latent_path(1, H, 1, rank, rot, L_max, m.MCSD_BF16 if dtype == "bf16" else m.MCSD_F32)
        assert path == (2 if dtype == "bf16" else 0) and splits > 16
        q, cache, rows = _problem(300 + H, dtype, 1, H, rank, rot, [-1], [L_max])
        lens, out = _i32([L_max]), torch.zeros(1, H, 1, rank, dtype=q.dtype, device="cuda")
        call = lambda: m.mcsd_tree_attention_latent(q, cache, rows, lens, None, tm, 0.07, out=out, workspace=ws)  # noqa: E731, B023
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=s):
            for _ in range(3):
                call()
        graphs.append((graph, q, cache, rows, lens, out, rank))
    for i, L in ((0, 20000), (1, 6000), (0, 1), (0, 777), (1, 0), (1, 5999), (0, 19999), (1, 64)):
        graph, q, cache, rows, lens, out, rank = graphs[i]
        lens.fill_(L)
        out.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        _compare(out, q, cache, rows, [L], None, np.ones((1, 1), bool), 0.07, rank)
