"""Cross-entropy with its gradient (mgrit_cross_entropy) against 64-bit formulas."""
import math

import pytest
import torch

import paper_2007_07336_amd as M
from tests.ops_util import KIND, TINY, TYPES, near, normal

pytestmark = pytest.mark.gpu
INF = float("inf")


class Loss:
    def __init__(self, B, V, t="f", mean=True, scale=1.0, seed=0, spread=2.0):
        self.B, self.V, self.t, self.mean, self.scale = B, V, t, mean, scale
        self.p = M.make_loss(B=B, V=V, dtype=KIND[t], reduction=M.MGRIT_LOSS_MEAN if mean else M.MGRIT_LOSS_SUM, scale=scale)
        self.x = normal((B, V), spread, t, seed)
        self.labels = torch.randint(0, V, (B,), generator=torch.Generator().manual_seed(seed + 1), dtype=torch.int64).cuda()
        self.ws = torch.full((M.mgrit_cross_entropy_workspace_bytes(self.p),), 0xFF, dtype=torch.uint8, device="cuda")

    def call(self, **kw):
        nan = lambda shape, t="f": torch.full(shape, float("nan"), dtype=TYPES[t], device="cuda")     # noqa: E731
        o = nan((1,)), nan((self.B,)), nan((self.B, self.V), self.t)
        M.mgrit_cross_entropy(self.p, self.x, self.labels, *o, self.ws, **kw)
        return o

    def exact(self):
        """(loss, rows, grad), and bounds of each.  A term exp(x - m) is off by 2^-23 (|x - m| + 2) of itself (rounding of the
        difference, of its product with log2 e, and a step of the instruction); V additions by 2^-24 each."""
        x, y = self.x.double(), self.labels
        counted = y >= 0
        n = max(1, int(counted.sum())) if self.mean else 1
        at = y.clamp(0, self.V - 1)[:, None]
        m = x.max(1, keepdim=True).values
        e = torch.exp(x - m)
        s = e.sum(1, keepdim=True)
        d = (m - x).nan_to_num(0.0, 0.0, 0.0)
        ds = (e * (d + 2.0)).sum(1, keepdim=True) / s * 2.0 ** -23 + self.V * 2.0 ** -24
        l = (torch.log(s) + m - x.gather(1, at))[:, 0]
        lb = (ds[:, 0] + 2.0 ** -22 * (torch.log(s)[:, 0].abs() + m[:, 0].abs() + x.gather(1, at)[:, 0].abs())).nan_to_num(0.0, 0.0, 0.0)
        bad = y >= self.V
        l = torch.where(counted, torch.where(bad, torch.nan, l), 0.0)
        w = self.scale / n
        p = e / s
        hot = torch.zeros_like(p).scatter_(1, at, 1.0)
        g = torch.where(counted[:, None], torch.where(bad[:, None], torch.nan, (p - hot) * w), 0.0)
        gb = (abs(w) * (p * (2.0 ** -23 * (d + 8.0) + ds) + 2.0 ** -22 * hot)).nan_to_num(0.0, 0.0, 0.0)
        total = l.sum() * w
        tb = abs(w) * lb[counted].sum() + 2.0 ** -23 * total.abs().nan_to_num(0.0, 0.0, 0.0)
        return (total.reshape(1), l, g), (tb.reshape(1), torch.where(counted, lb, 0.0), gb)

    def check(self):
        got = self.call()
        want, bound = self.exact()
        for k, name in enumerate(("loss", "rows", "grad")):
            near(got[k], want[k], bound[k] + TINY, (name, self.B, self.V, self.t))
        return got


SHAPES = [(1, 1), (1, 2), (3, 7), (5, 10), (256, 10), (64, 64), (33, 100), (7, 255), (4, 257), (9, 1000), (3, 1023), (3, 1024), (5, 1025), (2, 4099),
          (3, 16384), (2, 16385), (2, 50021), (1, 65536), (2, 65537), (1, 131071), (1, 262147), (2000, 3), (5001, 17)]


@pytest.mark.parametrize("t", ["f", "b"])
@pytest.mark.parametrize("B,V", SHAPES)
def test_loss_and_gradient(B, V, t):
    Loss(B, V, t).check()
    Loss(B, V, t, mean=False, scale=-0.37, seed=5, spread=20.0).check()


@pytest.mark.parametrize("t", ["f", "b"])
@pytest.mark.parametrize("B,V", [(6, 10), (300, 77), (40, 5000), (12, 20001)])
def test_rows_that_do_not_count(B, V, t):
    a = Loss(B, V, t)
    a.labels[::3] = -1
    a.labels[1] = -100
    a.x[0] = float("nan")                                   # whatever an uncounted row holds
    a.x[3] = INF
    got = a.call()
    a.x[0], a.x[3] = 0.0, 0.0
    want, bound = a.exact()
    for k in range(3):
        near(got[k], want[k], bound[k] + TINY, k)
    assert not got[2][::3].any() and not got[1][::3].any()
    a.labels.fill_(-1)
    got = a.call()
    assert all(not t.any() for t in got)                    # nothing counts: zero, and no division by zero


@pytest.mark.parametrize("t", ["f", "b"])
@pytest.mark.parametrize("V", [12, 300, 3000, 20000, 70001])
def test_masked_classes(V, t):
    a = Loss(6, V, t)
    keep = torch.rand(V, generator=torch.Generator().manual_seed(3)) < 0.3
    keep[0] = True
    a.x[:, ~keep.cuda()] = -INF
    a.x[1, :] = -INF                                        # one class left
    a.x[1, V - 1] = 3.0
    a.labels[:] = 0
    a.labels[1] = V - 1
    a.x[2] = torch.finfo(TYPES[t]).min                      # masked by the lowest value: all classes alike
    a.x[3, 1:] = torch.finfo(TYPES[t]).min
    got = a.check()
    assert float(got[1][1]) == 0.0 and not got[2][1].any()


@pytest.mark.parametrize("t", ["f", "b"])
@pytest.mark.parametrize("V", [9, 600, 20000, 70001])
def test_rows_without_a_softmax(V, t):
    a = Loss(8, V, t, mean=False)
    a.x[1, :] = -INF                                        # nothing left
    a.x[2, V // 2] = INF
    a.x[3, V - 1] = float("nan")
    a.x[4, :] = -INF
    a.x[4, 1] = float("nan")
    a.labels[5] = V                                         # no such class
    a.labels[6] = 2 ** 40
    a.x[7, 0], a.labels[7] = -INF, 0                        # a masked class asked for
    loss, rows, grad = a.call()
    ref = Loss(8, V, t, mean=False)
    want, bound = ref.exact()
    near(rows[:1], want[1][:1], bound[1][:1] + TINY, "row 0")
    near(grad[:1], want[2][:1], bound[2][:1] + TINY, "row 0")
    assert torch.isnan(rows[1:7]).all() and torch.isnan(grad[1:7]).all() and torch.isnan(loss).all()
    assert float(rows[7]) == INF and torch.isfinite(grad[7]).all() and float(grad[7, 0]) == -1.0


@pytest.mark.parametrize("t,B,V", [("f", 50, 10), ("b", 9, 1111), ("b", 3, 40001), ("f", 2, 140000)])
def test_gradient_in_the_place_of_the_logits(t, B, V):
    a = Loss(B, V, t)
    loss, rows, grad = a.call()
    l2, r2 = torch.empty_like(loss), torch.empty_like(rows)
    M.mgrit_cross_entropy(a.p, a.x, a.labels, l2, r2, a.x, a.ws)
    assert torch.equal(a.x, grad) and torch.equal(loss, l2) and torch.equal(rows, r2)


def test_outputs_one_at_a_time():
    for B, V, t in ((40, 10, "f"), (11, 2000, "b"), (3, 33333, "b")):
        a = Loss(B, V, t)
        all_ = a.call()
        for k in range(3):
            o = [torch.full_like(x, 5.0) if i == k else None for i, x in enumerate(all_)]
            M.mgrit_cross_entropy(a.p, a.x, a.labels, *o, a.ws)
            assert torch.equal(o[k], all_[k])


def test_no_rows():
    p = M.make_loss(B=0, V=10)
    loss = torch.full((1,), 5.0, device="cuda")
    ws = torch.empty(M.mgrit_cross_entropy_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    M.mgrit_cross_entropy(p, torch.empty((0, 10), device="cuda"), torch.empty((0,), dtype=torch.int64, device="cuda"), loss, None, None, ws)
    assert float(loss) == 0.0


def test_gradient_against_differences():
    a = Loss(20, 13, "f", scale=2.0)
    _, _, grad = a.call()
    v = normal(a.x.shape, 1.0, "f", 9).double()

    def value(t):
        x = a.x.double() + t * v
        return float(2.0 * (torch.logsumexp(x, 1) - x.gather(1, a.labels[:, None])[:, 0]).mean())

    h = 1e-5
    size = float((grad.double() * v).abs().sum())
    assert abs(float((grad.double() * v).sum()) - (value(h) - value(-h)) / (2 * h)) <= 1e-6 * max(size, 1.0)


@pytest.mark.parametrize("t,B,V", [("f", 70, 10), ("b", 5, 20011)])
def test_captured_calls_replay(t, B, V):
    a = Loss(B, V, t)
    o = a.call()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        M.mgrit_cross_entropy(a.p, a.x, a.labels, *o, a.ws)
    for replay in range(3):
        a.x.copy_(normal((B, V), 3.0, t, 20 + replay))
        a.labels[replay::4] = -1
        want = [w.clone() for w in a.call()]
        a.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip(o, want)), replay


def test_nothing_is_written_past_the_outputs():
    for t, B, V in (("f", 5, 10), ("b", 3, 4097), ("b", 2, 33335), ("f", 3, 1023)):
        a = Loss(B, V, t)
        whole = torch.full((B * V + 8192,), 7.0, dtype=TYPES[t], device="cuda")
        rows = torch.full((B + 64,), 7.0, device="cuda")
        M.mgrit_cross_entropy(a.p, a.x, a.labels, None, rows[:B], whole[4096:4096 + B * V].view(B, V), a.ws)
        assert bool((whole[:4096] == 7.0).all()) and bool((whole[4096 + B * V:] == 7.0).all()) and bool((rows[B:] == 7.0).all())


def test_the_largest_number_of_classes():
    """2^31 - 1 classes: a row that does not count is zeroed to its end and no further, the row behind it is right."""
    V = 2 ** 31 - 1
    p = M.make_loss(B=2, V=V, dtype=M.MGRIT_BF16, reduction=M.MGRIT_LOSS_SUM)
    ws = torch.empty(M.mgrit_cross_entropy_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    whole = torch.zeros(2 * V + 4096, dtype=torch.bfloat16, device="cuda")
    whole[:V] = 3.0
    whole[2 * V:] = 7.0
    x, labels, rows = whole[:2 * V].view(2, V), torch.tensor([-1, V - 1], device="cuda"), torch.full((2,), float("nan"), device="cuda")
    M.mgrit_cross_entropy(p, x, labels, None, rows, x, ws)
    assert bool((whole[2 * V:] == 7.0).all()) and float(rows[0]) == 0.0
    # the row behind: log V (2 steps for the logarithm and its product with log 2), 1 / V, and 1 / V - 1 at the label
    assert abs(float(rows[1]) - math.log(V)) <= 2.0 ** -22 * math.log(V)
    third = 1 << 30
    for a in range(0, V, third):
        assert not x[0, a:a + third].any()
        part = x[1, a:min(a + third, V - 1)]
        assert abs(float(part.min()) * V - 1.0) <= 2.0 ** -8 * 1.001 and abs(float(part.max()) * V - 1.0) <= 2.0 ** -8 * 1.001
    assert float(x[1, V - 1]) == -1.0


@pytest.mark.parametrize("t", ["f", "b"])
@pytest.mark.parametrize("V", [1, 10, 300, 3001, 20000, 70001])
@pytest.mark.parametrize("offset", [1e3, -1e4, 2.0 ** 25, 3e38, "lowest"])
def test_losses_do_not_depend_on_a_common_offset(offset, V, t):
    """Logits far from zero: the loss is as exact as that of the differences to the row's maximum, which are exact here or nearly so.
    A row of equal classes has log V, whatever they are."""
    a = Loss(6, V, t, mean=False, scale=0.5)
    c = float(torch.finfo(TYPES[t]).min) if offset == "lowest" else offset
    a.x.copy_(a.x.double() + c if offset != "lowest" else torch.full_like(a.x, c))
    a.x[1] = c
    a.x[2, V // 2:] = -INF
    a.x[2, 0] = c
    a.labels[2] = 0
    x, at = a.x.double(), a.labels[:, None]
    m = x.max(1, keepdim=True).values
    d = m - x
    e = torch.exp(-d)
    s = e.sum(1)
    below = (m - x.gather(1, at))[:, 0]
    want = torch.log(s) + below
    # terms of the sum as in Loss.exact, the logarithm and its product with log 2, the difference to the label and the last addition
    bound = (e * (d.nan_to_num(0.0, 0.0, 0.0) + 2.0)).sum(1) / s * 2.0 ** -23 + V * 2.0 ** -24 + 2.0 ** -22 * (torch.log(s) + below)
    loss, rows, _ = a.call()
    near(rows, want, bound + TINY, "rows")
    near(loss, 0.5 * want.sum().reshape(1), 0.5 * bound.sum() + 2.0 ** -23 * want.sum() + TINY, "loss")
    assert abs(float(rows[1]) - math.log(V)) <= (V * 2.0 ** -24 + 2.0 ** -22 * math.log(V)) + TINY


@pytest.mark.parametrize("t", ["f", "b"])
@pytest.mark.parametrize("V", [1, 1024, 1025, 5000, 70000])
@pytest.mark.parametrize("mean", [True, False])
def test_no_rows_of_many_classes(mean, V, t):
    a = Loss(0, V, t, mean=mean)
    loss = torch.full((1,), 5.0, device="cuda")
    M.mgrit_cross_entropy(a.p, a.x, a.labels, loss, torch.empty((0,), device="cuda"), torch.empty_like(a.x), a.ws)
    assert float(loss) == 0.0
    M.mgrit_cross_entropy(a.p, a.x, a.labels, None, None, torch.empty_like(a.x), a.ws)


def test_more_rows_than_a_launch_has_threads_for():
    """2^24 + 5 rows of 1025 classes are more than 2^32 threads; the rows repeat, so that a small call has all results."""
    B, V, n = (1 << 24) + 5, 1025, 1 << 14
    few = Loss(n, V, "b", mean=False, scale=0.25)
    few.labels[::7] = -1
    _, want_rows, want = few.call()
    p = M.make_loss(B=B, V=V, dtype=M.MGRIT_BF16, reduction=M.MGRIT_LOSS_SUM, scale=0.25)
    x, labels = torch.empty((B, V), dtype=torch.bfloat16, device="cuda"), torch.empty((B,), dtype=torch.int64, device="cuda")
    for a in range(0, B, n):
        k = min(n, B - a)
        x[a:a + k], labels[a:a + k] = few.x[:k], few.labels[:k]
    loss, rows = torch.full((1,), float("nan"), device="cuda"), torch.full((B,), float("nan"), device="cuda")
    ws = torch.empty(M.mgrit_cross_entropy_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    M.mgrit_cross_entropy(p, x, labels, loss, rows, x, ws)
    total, same = 0.0, torch.ones((), dtype=torch.bool, device="cuda")
    for a in range(0, B, n):
        k = min(n, B - a)
        same &= (x[a:a + k] == want[:k]).all() & (rows[a:a + k] == want_rows[:k]).all()
        total += 1 if k == n else 0
    assert bool(same)
    total = 0.25 * (total * float(want_rows.double().sum()) + float(want_rows[:5].double().sum()))
    assert abs(float(loss) - total) <= 2.0 ** -23 * abs(total)
    del x, labels, rows, ws
    torch.cuda.empty_cache()
