"""Candidates from logits: filters, probabilities and draws against the definition in 64 bits, and refusals."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import latent_oracle as orc
from tests.test_kv4 import m  # noqa: F401  (the fixture)

FAKE = ctypes.c_void_p(0x1000)      # never dereferenced: every call that uses it fails its checks first
INF = float("inf")
# Weights are fp32 with an error of at most 2^-21 (exponential and its argument, in units of 2^-24: two and two) and are
# rounded to 2^-31 of the largest for sums, which are off by n 2^-32 of the largest weight at most when n tokens take part; both
# sides of a ratio: 2^-20 + n 2^-31.
REL = 2.0 ** -20


def test_refusals(m):  # noqa: F811
    def call(logits=FAKE, stride=100, dtype=1, rows=2, V=100, u=FAKE, K=3, tokens=FAKE, probs=FAKE):
        return m.lib.mcsd_sample_candidates(logits, stride, dtype, rows, V, None, None, None, None, u, K, tokens, probs, None)
    assert call(logits=None) == -1
    assert call(tokens=None, probs=None) == -1
    assert call(u=None) == -1
    assert call(dtype=2) == -4
    assert call(rows=0) == -2
    assert call(rows=(1 << 24) + 1) == -2
    assert call(V=0) == -2
    assert call(V=262145, stride=262145) == -2
    assert call(stride=99) == -2
    assert call(K=0) == -2
    assert call(K=1025) == -2
    assert call(K=-1, tokens=None) == -2
    x = torch.zeros(2, 100)
    with pytest.raises(ValueError):
        m.mcsd_sample_candidates(x, probs=True)                                  # not on a GPU
    with pytest.raises(ValueError):
        m.mcsd_sample_candidates(x.double(), probs=True)


def test_oracle_filters():
    """The filters' definition on rows small enough to check by hand."""
    x = np.log(np.array([0.1, 0.4, 0.2, 0.2, 0.1]))
    assert np.allclose(orc.filtered(x, top_k=2)[0], [0, 2 / 3, 1 / 3, 0, 0])     # equal logits: the lower id
    assert np.allclose(orc.filtered(x, top_p=0.75)[0], [0, 0.5, 0.25, 0.25, 0])
    assert np.allclose(orc.filtered(x, top_k=4, top_p=0.5)[0], [0, 2 / 3, 1 / 3, 0, 0])   # 0.9 in the first four
    assert np.allclose(orc.filtered(x, min_p=0.3)[0], [0, 0.5, 0.25, 0.25, 0])
    assert np.allclose(orc.filtered(x, temperature=0.0)[0], [0, 1, 0, 0, 0])
    assert np.allclose(orc.filtered(x, temperature=0.5, top_k=2)[0], [0, 0.8, 0.2, 0, 0])
    assert orc.draws(np.array([0, 0.5, 0, 0.5]), [0.0, 0.49, 0.5, 0.99, 1.0])[0].tolist() == [1, 1, 3, 3, 3]


def _per_row(v, rows, dtype):
    return None if v is None else torch.as_tensor(np.broadcast_to(np.asarray(v), (rows,)).copy()).to(dtype).cuda()


def _check(m, logits, temperature=None, top_k=None, top_p=None, min_p=None, K=3, seed=0, u=None):  # noqa: F811
    """Probabilities of every row, and draws from uniforms that lie clear of the borders."""
    rows, V = logits.shape
    host = logits.float().cpu().numpy()
    rng = np.random.default_rng(seed)
    args = dict(temperature=_per_row(temperature, rows, torch.float32), top_k=_per_row(top_k, rows, torch.int32),
                top_p=_per_row(top_p, rows, torch.float32), min_p=_per_row(min_p, rows, torch.float32))
    at = lambda name, r, off: off if args[name] is None else args[name][r].item()  # noqa: E731
    want, kept = np.zeros((rows, V)), np.zeros((rows, 1))
    uu = rng.random((rows, K)).astype(np.float32) if u is None else np.asarray(u, dtype=np.float32)
    ids = np.zeros((rows, K), dtype=np.int64)
    for r in range(rows):
        want[r], margin = orc.filtered(host[r], at("temperature", r, 1.0), at("top_k", r, 0), at("top_p", r, 1.0), at("min_p", r, 0.0))
        kept[r] = (want[r] > 0).sum()
        slack = 2 * REL + kept[r, 0] * 2.0 ** -31
        assert margin["top_p"] > 2 * REL + margin["among"] * 2.0 ** -31 and margin["min_p"] > REL, "choose another threshold: the case lies on a border"
        for _ in range(200):
            ids[r], d = orc.draws(want[r], uu[r])
            near = d <= slack
            if not near.any() or u is not None:
                break
            uu[r, near] = rng.random(int(near.sum())).astype(np.float32)
        assert u is not None or not near.any()
    tokens, probs = m.mcsd_sample_candidates(logits, torch.from_numpy(uu).cuda(), probs=True, **args)
    got = probs.cpu().numpy()
    assert (got[want > 1e-36] > 0).all() and not got[want == 0].any()
    assert (np.abs(got - want) <= (REL + kept * 2.0 ** -31) * want + 1e-36).all(), np.abs(got - want).max()
    assert np.array_equal(tokens.cpu().numpy(), ids)
    return tokens, probs


CASES = [
    # rows, V, dtype, temperature, top_k, top_p, min_p
    (1, 32000, "bf16", 0.7, 50, 0.9, None),
    (3, 32000, "f32", 0.7, None, 0.95, None),
    (2, 131071, "f32", 1.0, 2000, 0.95, 0.021),
    (2, 200000, "bf16", 1.3, None, None, None),
    (5, 1000, "f32", [0.0, 0.5, 1.0, 2.0, -1.0], [0, 1, 7, 1000, 3], [0.3, 1.0, 0.5, 0.8, 0.1], None),
    (300, 4099, "f32", 1.0, 40, None, 0.05),
    (160, 777, "bf16", 1.0, None, 0.5, None),
    (1, 1, "f32", 1.0, 1, 0.5, 0.5),
    (4, 2, "f32", 1.0, 1, None, None),
    (2, 129, "f32", 3.0, 100, None, None),
    (1, 262144, "bf16", 1.0, 100000, None, None),
    (1, 32769, "f32", 1.0, 5000, 0.9, None),
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V,dtype,temperature,top_k,top_p,min_p", CASES)
def test_filters_and_draws(m, rows, V, dtype, temperature, top_k, top_p, min_p):  # noqa: F811
    for seed in range(100):
        g = torch.Generator("cuda").manual_seed(seed)
        x = (3 * torch.randn(rows, V, generator=g, device="cuda")).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        try:
            _check(m, x, temperature, top_k, top_p, min_p)
            return
        except AssertionError as e:
            if "border" not in str(e):
                raise
    pytest.fail("every seed lies on a border")


@pytest.mark.gpu
def test_rows_apart_and_off_a_16_byte_boundary(m):  # noqa: F811
    big = 3 * torch.randn(7, 5011, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    for dt in (torch.float32, torch.bfloat16):
        x = big.to(dt)
        for part in (x[:, 1:4000], x[::2, 8:4008], x[2:3, 3:]):
            a = m.mcsd_sample_candidates(part, torch.full((part.shape[0], 2), 0.4, device="cuda"), probs=True)
            b = m.mcsd_sample_candidates(part.contiguous(), torch.full((part.shape[0], 2), 0.4, device="cuda"), probs=True)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
            w = torch.softmax(part.double(), -1)
            assert ((a[1] - w).abs() <= 1e-5 * w).all()


@pytest.mark.gpu
def test_rows_without_a_token_and_infinities(m):  # noqa: F811
    x = torch.full((6, 3000), -INF, device="cuda")
    x[1] = float("nan")
    x[2, 77] = -5.0                                                   # one token left
    x[3, 10], x[3, 20], x[3, 30] = INF, INF, 100.0                    # two infinities share the mass
    x[4] = torch.finfo(torch.float32).min                             # masked by the type's lowest value, one not
    x[4, 2999] = 1.0
    x[5, 5], x[5, 6], x[5, 7] = float("nan"), 2.0, 2.0
    u = torch.tensor([[0.0, 0.3, 0.999]], device="cuda").expand(6, 3).contiguous()
    want = torch.zeros_like(x)
    want[2, 77] = want[4, 2999] = 1.0
    want[3, 10] = want[3, 20] = want[5, 6] = want[5, 7] = 0.5
    ids = [[-1] * 3, [-1] * 3, [77] * 3, [10, 10, 20], [2999] * 3, [6, 6, 7]]
    for kw in (dict(), dict(top_k=_per_row(50, 6, torch.int32)), dict(top_p=_per_row(0.9, 6, torch.float32)),
               dict(top_k=_per_row(50, 6, torch.int32), top_p=_per_row(0.99, 6, torch.float32), min_p=_per_row(0.5, 6, torch.float32))):
        tokens, probs = m.mcsd_sample_candidates(x, u, probs=True, **kw)
        assert tokens.tolist() == ids and torch.equal(probs, want), kw
    one = want.clone()
    one[3, 20] = one[5, 7] = 0.0
    one[3, 10] = one[5, 6] = 1.0
    for kw in (dict(temperature=_per_row(0.0, 6, torch.float32)), dict(temperature=_per_row(float("nan"), 6, torch.float32)),
               dict(top_k=_per_row(1, 6, torch.int32)), dict(top_p=_per_row(0.0, 6, torch.float32)), dict(top_p=_per_row(-1.0, 6, torch.float32))):
        tokens, probs = m.mcsd_sample_candidates(x, u, probs=True, **kw)
        assert torch.equal(probs, one), kw
        assert tokens.tolist() == [[-1] * 3, [-1] * 3, [77] * 3, [10] * 3, [2999] * 3, [6] * 3], kw
    off = dict(temperature=_per_row(1.0, 6, torch.float32), top_k=_per_row(-3, 6, torch.int32), top_p=_per_row(float("nan"), 6, torch.float32),
               min_p=_per_row(float("nan"), 6, torch.float32))
    assert torch.equal(m.mcsd_sample_candidates(x, u, probs=True, **off)[1], want)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [1500, 32000, 150000])
def test_equal_logits_go_by_id(m, V):  # noqa: F811
    """Steps of the order that hold more tokens than can be placed at once: all equal, and two values alternating."""
    x = torch.zeros(3, V, device="cuda")
    x[1, ::2] = 1.0
    x[2] = -60000.0
    x[2, V // 3] = 0.0
    k = max(3, V // 5)
    keep = m.mcsd_sample_candidates(x, probs=True, top_k=_per_row(k, 3, torch.int32))[0].cpu().numpy() > 0
    assert keep[0].nonzero()[0].tolist() == list(range(k))
    assert keep[1].nonzero()[0].tolist() == list(range(0, 2 * k, 2))
    p = m.mcsd_sample_candidates(x, probs=True, top_k=_per_row(k, 3, torch.int32))[0]
    assert ((p[0, :k].double() - 1 / k).abs() <= 2.0 ** -22 / k).all() and p[2, V // 3] == 1.0
    share = (k - 0.5) / V                                             # half a token inside the k-th
    keep = m.mcsd_sample_candidates(x[:1], probs=True, top_p=_per_row(share, 1, torch.float32))[0].cpu().numpy() > 0
    assert keep[0].nonzero()[0].tolist() == list(range(k))
    u = (torch.arange(16, device="cuda") + 0.5) / 16
    ids = m.mcsd_sample_candidates(x[:1], u.view(1, 16))[0]
    assert ids[0].tolist() == [int((i + 0.5) / 16 * V) for i in range(16)]


@pytest.mark.gpu
def test_steep_and_flat_temperatures(m):  # noqa: F811
    g = torch.Generator("cuda").manual_seed(3)
    x = 3 * torch.randn(4, 8000, generator=g, device="cuda")
    t = torch.tensor([1e-30, 1e-3, 1e6, INF], device="cuda")
    p = m.mcsd_sample_candidates(x, probs=True, temperature=t)[0].double().cpu()
    want = torch.stack([torch.softmax(r / v, -1) for r, v in zip(x.double().cpu(), t.double().cpu())])
    assert ((p - want).abs() <= (2 * REL + 8000 * 2.0 ** -31) * want + 1e-36).all()
    kept = m.mcsd_sample_candidates(x, probs=True, temperature=t, top_k=_per_row(3, 4, torch.int32))[0]
    top = torch.topk(x, 3).indices.sort(-1).values
    assert kept[3].nonzero().flatten().tolist() == top[3].tolist() and kept[2].nonzero().flatten().tolist() == top[2].tolist()


@pytest.mark.gpu
def test_uniforms_at_the_ends(m):  # noqa: F811
    x = torch.full((1, 5000), -INF, device="cuda")
    x[0, 100], x[0, 4000] = 0.0, 0.0
    u = torch.tensor([[0.0, -1.0, float("nan"), 0.5, 1.0 - 2.0 ** -24, 1.0, 2.0]], device="cuda")
    assert m.mcsd_sample_candidates(x, u)[0].tolist() == [[100, 100, 100, 4000, 4000, 4000, 4000]]


@pytest.mark.gpu
def test_same_results_however_a_row_is_split(m):  # noqa: F811
    """One row alone goes over several blocks, many rows take one each: equal to the bit, and from call to call."""
    g = torch.Generator("cuda").manual_seed(4)
    x = 3 * torch.randn(200, 30000, generator=g, device="cuda")
    u = torch.rand(200, 8, generator=g, device="cuda")
    kw = lambda n: dict(temperature=_per_row(0.8, n, torch.float32), top_k=_per_row(3000, n, torch.int32), top_p=_per_row(0.9, n, torch.float32))  # noqa: E731
    a = m.mcsd_sample_candidates(x, u, probs=True, **kw(200))
    for _ in range(3):
        b = m.mcsd_sample_candidates(x, u, probs=True, **kw(200))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for r in (0, 57, 199):
        for n in (1, 2, 20):
            lo = min(r, 200 - n)
            b = m.mcsd_sample_candidates(x[lo:lo + n], u[lo:lo + n], probs=True, **kw(n))
            assert torch.equal(a[0][lo:lo + n], b[0]) and torch.equal(a[1][lo:lo + n], b[1])


@pytest.mark.gpu
def test_captured_and_on_another_stream(m):  # noqa: F811
    x = torch.randn(3, 4000, device="cuda")
    u = torch.rand(3, 4, device="cuda")
    want = [t.clone() for t in m.mcsd_sample_candidates(x, u, probs=True)]
    tokens, probs = torch.zeros(3, 4, dtype=torch.int32, device="cuda"), torch.zeros(3, 4000, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        m.mcsd_sample_candidates(x, u, tokens=tokens, probs=probs)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(tokens, want[0]) and torch.equal(probs, want[1])
    x.neg_()
    want = m.mcsd_sample_candidates(x, u, probs=True)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(tokens, want[0]) and torch.equal(probs, want[1])


# more tokens above 2^-14 of the largest than a block lists: a higher bound is found (1.0), or not (1.3); large k by finer maxima
MANY = [(160, 32000, 1.0, None, 0.95), (160, 32000, 1.0, None, 0.6), (150, 20000, 1.3, None, 0.95), (150, 20000, 1.3, None, 0.3),
        (149, 16001, 3.0, None, 0.9), (160, 9000, 1.0, 2000, 0.9), (150, 9000, 1.5, 3500, 0.8), (150, 4001, 1.0, 300, None)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V,temperature,top_k,top_p", MANY)
def test_flat_rows_of_many(m, rows, V, temperature, top_k, top_p):  # noqa: F811
    """Rows that take a block each, a few of them against the definition, and all as when they are split over several blocks.

    A token at the cut of such a row weighs less than the sum's error bound (twice REL for the weights, half a step of 2^-31 for
    each of its tokens, on either side of a comparison), so no seed is clear of it: what is kept has to be a beginning of the
    order whose mass reaches top_p by that bound, and without its last token does not exceed it by more."""
    g = torch.Generator("cuda").manual_seed(0)
    x = 3 * torch.randn(rows, V, generator=g, device="cuda")
    u = torch.rand(rows, 5, generator=g, device="cuda")
    kw = lambda n: dict(temperature=_per_row(temperature, n, torch.float32), top_k=_per_row(top_k, n, torch.int32), top_p=_per_row(top_p, n, torch.float32))  # noqa: E731
    tokens, probs = m.mcsd_sample_candidates(x, u, probs=True, **kw(rows))
    T = float(np.float32(temperature))
    for r in (0, 1, rows // 2, rows - 1):
        host, got = x[r].double().cpu().numpy(), probs[r].double().cpu().numpy()
        order = np.lexsort((np.arange(V), -host))[: top_k or V]
        w = np.exp((host[order] - host[order[0]]) / T)
        mass = np.cumsum(w) / w.sum()
        n = int((got > 0).sum())
        assert (got[order[:n]] > 0).all()
        if top_p is None:
            assert n == len(order)
        else:
            p, slack = float(np.float32(top_p)), 2 * REL + len(order) * 2.0 ** -31
            assert mass[n - 1] >= p - slack and (n == 1 or mass[n - 2] < p + slack), (n, mass[n - 1] - p)
        want = np.zeros(V)
        want[order[:n]] = w[:n] / w[:n].sum()
        assert (np.abs(got - want) <= (REL + n * 2.0 ** -31) * want + 1e-36).all()
        run, slack = np.cumsum(want), 2 * REL + n * 2.0 ** -31
        for t, z in zip(tokens[r].tolist(), u[r].tolist()):
            assert want[t] > 0 and run[t] > z - slack and run[t] - want[t] <= z + slack
    for lo, n in ((0, 1), (rows // 2, 2), (rows - 20, 20), (3, 70)):
        t, p = m.mcsd_sample_candidates(x[lo:lo + n], u[lo:lo + n], probs=True, **kw(n))
        assert torch.equal(tokens[lo:lo + n], t) and torch.equal(probs[lo:lo + n], p)
