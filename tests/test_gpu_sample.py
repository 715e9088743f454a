"""Drawing classes from logits: indices against the definition in 64 bits, row by row."""
import math

import pytest
import torch

import paper_2007_07336_amd as M
from tests.ops_util import KIND, TYPES, normal

pytestmark = pytest.mark.gpu
INF = math.inf


def kept_of(x, t, k, p, least):
    """The kept classes of one row and the logarithms of their weights, or None for a row without an answer (double, CPU)."""
    x = x.double()
    V = x.numel()
    if bool(torch.isnan(x).any()) or float(x.max()) in (INF, -INF) or not (0.0 <= t < INF) or math.isnan(p) or math.isnan(least):
        return None
    order = sorted(range(V), key=lambda v: (-float(x[v]), v)) if V <= 4096 else torch.sort(x, descending=True, stable=True).indices.tolist()
    if t == 0.0 or p <= 0.0:
        return order[:1], x * 0.0
    z = (x - x.max()) / t
    w = torch.exp(z)
    n = V if k <= 0 or k >= V else k
    if p < 1.0:
        run = torch.cumsum(w[torch.tensor(order[:n])], 0)
        n = min(n, int((run < p * run[-1]).sum()) + 1)
    kept = [v for v in order[:n] if float(w[v]) >= min(least, 1.0)] if least > 0.0 else order[:n]
    return sorted(kept), z


def answer(x, u, t, k, p, least):
    got = kept_of(x, t, k, p, least)
    if got is None or not (0.0 <= u < 1.0):
        return -1, math.nan, 0.0
    kept, z = got
    w = torch.exp(z[torch.tensor(kept)])
    run = torch.cumsum(w, 0)
    over = (run > u * run[-1]).nonzero()
    at = int(over[0]) if over.numel() else len(kept) - 1
    # how far u is from the nearest border, relative to all weights
    near = float(((run / run[-1]) - u).abs().min())
    return kept[at], float(z[kept[at]] - torch.log(run[-1])), near


def call(x, u, t=None, k=None, p=None, least=None, want=True, **kw):
    B, V = x.shape
    q = M.make_sample(B=B, V=V, dtype=KIND["b" if x.dtype == torch.bfloat16 else "f"])
    index, logprob = torch.full((B,), -7, dtype=torch.int64, device="cuda"), torch.full((B,), 7.0, device="cuda") if want else None
    M.mgrit_sample(q, x, u, t, k, p, least, index, logprob, None, **kw)
    return index, logprob


def check(x, u, t=None, k=None, p=None, least=None):
    index, logprob = call(x, u, t, k, p, least)
    c = [None if a is None else a.cpu() for a in (x, u, t, k, p, least)]
    for b in range(x.shape[0]):
        want, lp, near = answer(c[0][b], float(c[1][b]), *[d if a is None else a[b].item() for a, d in zip(c[2:], (1.0, 0, 1.0, 0.0))])
        what = (b, int(index[b]), want, near)
        # (the weights are 2e-13 off: u within that of a border may fall on either side)
        assert int(index[b]) == want or 0.0 < near < 1.0e-12, what
        if want < 0:
            assert math.isnan(float(logprob[b])), what
        elif int(index[b]) == want:
            # weights to 3e-13 and sums of V of them: the logarithm to 1e-11, then one rounding to float
            assert abs(float(logprob[b]) - lp) <= 2.0 ** -24 * abs(lp) + 1.0e-11, what + (float(logprob[b]), lp)


def uniform(n, seed, lo=0.0, hi=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.rand((n,), generator=g) * (hi - lo) + lo).cuda()


def whole(n, lo, hi, seed):
    return torch.randint(lo, hi, (n,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype", ["f", "b"])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 255, 257, 1000, 2049, 4100])
@pytest.mark.parametrize("given", ["", "t", "k", "p", "m", "tk", "kp", "tkpm"])
def test_classes(dtype, V, given):
    B = 9
    x = normal((B, V), 2.0, dtype, V)
    x[:, V // 3:V // 2] = -INF
    if V == 1:
        x[:, 0] = 0.5
    check(x, uniform(B, 1), t=uniform(B, 2, 0.3, 2.0) if "t" in given else None, k=whole(B, -1, min(V + 2, 60), 3) if "k" in given else None,
          p=uniform(B, 4, 0.05, 1.1) if "p" in given else None, least=uniform(B, 5, -0.01, 0.3) if "m" in given else None)


@pytest.mark.parametrize("dtype,V", [("f", 8193), ("b", 16500), ("f", 33000), ("b", 50021), ("f", 70001), ("b", 140001)])
def test_many_classes(dtype, V):
    B = 4
    x = normal((B, V), 2.0, dtype, V)
    x[1, ::3] = -INF
    u = uniform(B, 1)
    check(x, u)
    check(x, u, t=uniform(B, 2, 0.3, 2.0), k=torch.tensor([1, 50, V - 1, 5000], dtype=torch.int32, device="cuda"),
          p=torch.tensor([0.9, 0.5, 0.99, 0.9], device="cuda"), least=torch.tensor([0.0, 0.01, 1e-4, 0.2], device="cuda"))
    check(x, u, p=torch.tensor([0.9, 0.5, 0.999999, 1e-6], device="cuda"))


@pytest.mark.parametrize("dtype", ["f", "b"])
def test_equal_logits_go_by_index(dtype):
    V, B = 300, 16
    x = torch.zeros((B, V), dtype=TYPES[dtype], device="cuda")
    x[:, 100:110] = 1.0
    x[:, 200:] = -0.0                                              # (the same value as zero)
    check(x, uniform(B, 1), k=whole(B, 1, V, 2))
    check(x, uniform(B, 1), k=torch.full((B,), 15, dtype=torch.int32, device="cuda"), p=uniform(B, 3, 0.3, 1.0))
    check(x, uniform(B, 1), p=uniform(B, 3, 0.01, 1.0))
    y = torch.full((B, V), -INF, dtype=TYPES[dtype], device="cuda")
    y[:, 17] = -3.0
    index, _ = call(y, uniform(B, 1), k=whole(B, 1, V, 2), p=uniform(B, 3))
    assert bool((index == 17).all())


@pytest.mark.parametrize("dtype", ["f", "b"])
@pytest.mark.parametrize("V", [5, 700, 9000])
def test_temperature_zero_and_the_first_of_the_order(dtype, V):
    x = normal((8, V), 1.0, dtype, 3)
    x[:, V // 2] = 20.0
    x[:4, V - 1] = 20.0
    u, zero = uniform(8, 1), torch.zeros((8,), device="cuda")
    for kw in (dict(t=zero), dict(p=zero), dict(k=torch.ones((8,), dtype=torch.int32, device="cuda")), dict(t=zero, k=whole(8, 1, 9, 1), p=uniform(8, 2), least=uniform(8, 3))):
        index, logprob = call(x, u, **kw)
        assert bool((index == V // 2).all()) and bool((logprob == 0.0).all()), kw
    index, _ = call(x, u, least=torch.full((8,), 5.0, device="cuda"))       # above 1 as 1: the equal largest ones
    assert bool(((index == V // 2) | (index == V - 1)).all())


def test_rows_without_an_answer_and_ends_of_the_interval():
    V = 100
    x = normal((12, V), 1.0, "f", 4)
    x[0, 5], x[1, 5], x[2, :] = math.nan, INF, -INF
    t, u, p, least = torch.ones((12,)), torch.full((12,), 0.5), torch.full((12,), 0.9), torch.zeros((12,))
    t[3], t[4], t[5], u[6], u[7], u[8], p[9], least[10] = -1.0, math.nan, INF, 1.0, -0.1, math.nan, math.nan, math.nan
    index, logprob = call(x, u.cuda(), t.cuda(), None, p.cuda(), least.cuda())
    assert bool((index[:11] == -1).all()) and bool(torch.isnan(logprob[:11]).all()) and int(index[11]) >= 0
    y = normal((2, V), 1.0, "f", 5)
    y[:, :3], y[:, -4:] = -INF, -INF
    index, _ = call(y, torch.tensor([0.0, 1.0 - 2.0 ** -24], device="cuda"))
    assert index.tolist() == [3, V - 5]


def test_large_offsets_small_temperatures_and_no_logprob():
    x = normal((6, 513), 1.0, "f", 6) * 1.0e30
    t = torch.tensor([1.0e-30, 1.0, 1.0e30, 2.0e30, 1.0e38, 0.5], device="cuda")
    check(x, uniform(6, 1), t=t, p=uniform(6, 2))
    index, logprob = call(x, uniform(6, 1), t=t, want=False)
    assert logprob is None and bool((index >= 0).all())


def test_rows_do_not_touch_each_other_and_streams():
    x = normal((257, 1003), 2.0, "b", 7)
    u, k, p = uniform(257, 1), whole(257, 1, 100, 2), uniform(257, 3, 0.5, 1.0)
    want, wl = call(x, u, None, k, p)
    for r in (0, 100, 256):                                       # (a row inside a larger array begins at any multiple of 16 bytes)
        i, l = call(x[r:r + 1].clone(), u[r:r + 1].clone(), None, k[r:r + 1].clone(), p[r:r + 1].clone())
        assert int(i[0]) == int(want[r]) and float(l[0]) == float(wl[r])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        i, _ = call(x, u, None, k, p)
        j, _ = call(x, u, None, k, p, stream=side)
    side.synchronize()
    assert torch.equal(i, want) and torch.equal(j, want)


def test_replays():
    x, u = normal((5, 3000), 2.0, "f", 8), uniform(5, 1)
    k, p = whole(5, 1, 100, 2), uniform(5, 3, 0.5, 1.0)
    q = M.make_sample(B=5, V=3000)
    index, logprob = torch.zeros((5,), dtype=torch.int64, device="cuda"), torch.zeros((5,), device="cuda")
    run = lambda: M.mgrit_sample(q, x, u, None, k, p, None, index, logprob, None)                      # noqa: E731
    run()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        run()
    for replay in range(3):
        x.add_(normal(x.shape, 0.5, "f", 20 + replay))
        u.copy_(uniform(5, 30 + replay))
        run()
        want = index.clone(), logprob.clone()
        index.fill_(-9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(index, want[0]) and torch.equal(logprob, want[1]), replay


@pytest.mark.parametrize("dtype", ["f", "b"])
@pytest.mark.parametrize("V", [600, 5000, 30000, 90000])
def test_rows_that_crowd_into_few_bins(dtype, V):
    """Masks of large negative numbers and of the type's lowest one, values that spread over many magnitudes, many equal ones."""
    x = normal((8, V), 2.0, dtype, V)
    x[0, ::2] = -1.0e4
    x[1, ::2] = torch.finfo(x.dtype).min
    x[2] = (-(torch.arange(V, dtype=torch.float64) % 300) / 3).exp2().to(x.dtype).cuda()
    x[3] = -torch.exp2((torch.arange(V, dtype=torch.float64) % 120)).to(x.dtype).cuda()
    x[4] = 1.5
    x[5, : V - 3] = 0.25
    x[6] = 1.0 + normal((V,), 1.0e-6, dtype, 2)
    x[7, 5] = 60.0
    u = uniform(8, 1)
    for k in (2, 40, V // 2, V - 1):
        check(x, u, k=torch.full((8,), k, dtype=torch.int32, device="cuda"))
    check(x, u, p=uniform(8, 2, 0.1, 1.0))
    check(x, u, t=uniform(8, 3, 0.01, 3.0), p=uniform(8, 2, 0.5, 1.0), k=torch.full((8,), V // 3, dtype=torch.int32, device="cuda"))


def test_logits_that_are_all_but_equal():
    """Differences far below the smallest normal float: the order is theirs, the weights are all the same."""
    V = 700
    x = (torch.arange(V, dtype=torch.float64) * 2.0 ** -149).to(torch.float32).flip(0)[None].repeat(6, 1)
    x[1] = -x[1]
    x[2] = x[2] * 2.0 ** 20
    x[3, ::2] = 0.0
    x = x.cuda()
    u = uniform(6, 1)
    check(x, u, k=whole(6, 2, 30, 2))
    check(x, u, k=whole(6, 2, 30, 2), p=uniform(6, 3, 0.2, 0.9), least=uniform(6, 4, 0.0, 1.0))
    check(x, u, k=torch.full((6,), 500, dtype=torch.int32, device="cuda"), p=uniform(6, 3, 0.2, 0.9))
    check(x, u, p=uniform(6, 3, 0.2, 0.9))
