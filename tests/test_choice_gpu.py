"""Draws from rows of scores and their loss.

Draws are compared twice. Exactly, with the definition in whole numbers: weights of 31 bits from
float32 exponentials (elementary torch operations on the same device), sorted, summed in int64. And with
plain 64-bit arithmetic from the scores on: a weight's relative error is at most EPS (three roundings of
the exponent, |y| <= 22, 2^-24 each, and the exponential's own 2^-23), so a drawn index's interval
of the running sum must hold u S within EPS S and one unit for each entry, and a row whose nucleus
ends nearer than that to its bound may end on either side."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

EPS = 3 * 22 * 2.0 ** -24 + 2.0 ** -23
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FLT_MAX = float(np.finfo(np.float32).max)
TINY = float(np.finfo(np.float32).tiny)


@pytest.fixture(scope="module")
def emr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_27612_amd import emr as m
    return m


def column(v, rows):
    if torch.is_tensor(v):
        return v.double().cpu().numpy()
    return np.full(rows, float(np.float32(v)))


def whole(x, u, t=1.0, k=0, p=1.0, min_p=0.0):
    """(index, kept weights, y) of the definition in whole numbers."""
    x = x.float()
    rows, n = x.shape
    t, k, p, min_p = (torch.tensor(column(v, rows), device="cuda")[:, None] for v in (t, k, p, min_p))
    x = torch.where(torch.isnan(x), -np.inf, x).clamp(max=FLT_MAX)
    m = x.amax(1, keepdim=True)
    live = x > -np.inf
    order = x.sort(dim=1, descending=True, stable=True)[1]
    y = torch.where(live, (x - m) * (1.0 / t.float().clamp(min=TINY, max=FLT_MAX)), -np.inf)
    q = (torch.exp(y) * 2.0 ** 31).long()
    q = torch.where(t.float() >= TINY, q, torch.zeros_like(q).scatter_(1, order[:, :1], 1 << 31) * live)
    qs = q.gather(1, order)
    rank = torch.arange(n, device="cuda")
    qs = torch.where((k <= 0) | (rank < k), qs, 0)
    total = qs.sum(1, keepdim=True)
    before = qs.cumsum(1) - qs
    qs = torch.where(~(p < 1) | (before == 0) | (before.double() < p * total.double()), qs, 0)
    q = torch.zeros_like(q).scatter_(1, order, qs)
    q = torch.where(q.double() >= min_p.clamp(max=1.0) * 2.0 ** 31, q, 0)
    run = q.cumsum(1)
    total = run[:, -1:]
    at = (u.double().clamp(min=0) * total.double()).long().minimum(total - 1)
    index = torch.searchsorted(run, at, right=True)
    return torch.where(total > 0, index, -1).int(), q, y


def check(emr, x, u, **rule):
    """Draws against both references."""
    names = {"t": "temperature", "k": "top_k", "p": "top_p", "min_p": "min_p"}
    index, logp = emr.emr_sample(x, u, **{names[a]: b for a, b in rule.items()})
    want, q, y = whole(x, u, **rule)
    assert torch.equal(index, want)
    none = want < 0
    total = q.sum(1, keepdim=True).double() / 2.0 ** 31
    lp = y.double().gather(1, want.clamp(min=0).long()) - torch.log(total)
    greedy = ~(torch.tensor(column(rule.get("t", 1.0), len(x)), device="cuda").float() >= TINY)[:, None]
    lp = torch.where(greedy, 0.0, lp)
    assert torch.equal(torch.isinf(logp), none)
    # (one rounding to float32 of a double)
    assert ((logp.double() - lp).abs()[~none] <= 1e-12 + 2.0 ** -23 * lp.abs()[~none]).all()
    near(x, u, index.cpu().numpy(), **rule)
    return index


def near(x, u, index, t=1.0, k=0, p=1.0, min_p=0.0):
    x, u = x.double().cpu().numpy(), u.double().cpu().numpy()
    rows, n = x.shape
    t, k, p, min_p = (column(v, rows) for v in (t, k, p, min_p))
    for r in range(0, rows, max(1, rows // 40)):
        v = np.minimum(np.where(np.isnan(x[r]), -np.inf, x[r]), FLT_MAX)
        if v.max() == -np.inf:
            assert (index[r] == -1).all()
            continue
        if not t[r] >= TINY:
            assert (index[r] == np.argmax(v)).all()
            continue
        w = np.exp((v - v.max()) / min(t[r], FLT_MAX))
        order = np.argsort(-v, kind="stable")
        left = order[:int(k[r])] if k[r] > 0 else order
        slack = EPS * w[left].sum() + len(left) * 2.0 ** -31
        least = most = len(left)
        if p[r] < 1:
            c = np.cumsum(w[left])
            least = 1 + int(np.searchsorted(c, p[r] * c[-1] - 2 * slack))
            most = min(len(left), 1 + int(np.searchsorted(c, p[r] * c[-1] + 2 * slack)))
        sure = w * 0
        sure[left[:least]] = w[left[:least]]
        may = w * 0
        may[left[:most]] = w[left[:most]]
        sure[w < min(min_p[r], 1) * (1 + 2 * EPS)] = 0
        may[w < min(min_p[r], 1) * (1 - 2 * EPS)] = 0
        a, b = np.cumsum(sure), np.cumsum(may)
        wide = 3 * slack + (b[-1] - a[-1])
        for d in range(0, u.shape[1], max(1, u.shape[1] // 40)):
            i = index[r, d]
            assert may[i] > 0 or (w[i] > 0 and b[-1] == 0)
            low = a[i - 1] if i else 0.0
            f = min(max(u[r, d], 0.0), 1.0)
            assert low - wide <= f * b[-1] and f * a[-1] <= b[i] + wide


def scores(seed, rows, n, type="f32", spread=3.0, pad=0, mask=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((rows, n + pad), generator=g, device="cuda") * spread
    if mask and n > 4:
        m = torch.rand((rows, n + pad), generator=g, device="cuda")
        x[m < 0.05] = -np.inf
        x[m > 0.99] = torch.finfo(TYPES[type]).min
        x[5::16] = -np.inf
    return x.to(TYPES[type])[:, :n], torch.rand((rows, 3), generator=g, device="cuda")


SIZES = [1, 2, 3, 8, 63, 64, 65, 100, 255, 256, 257, 1000, 1023, 1024, 1025, 2048, 4097, 10007, 32768, 32771,
         65537, 131073]
RULES = [dict(), dict(t=0.3), dict(k=1), dict(k=7, t=2.0), dict(p=0.9), dict(p=0.02), dict(min_p=0.1),
         dict(k=40, p=0.8, min_p=0.01, t=0.7), dict(k=3000, p=0.97, t=3.0), dict(t=0.0),
         dict(t=30.0, p=0.7)]


@pytest.mark.parametrize("n", SIZES)
def test_sizes_and_rules(emr, n):
    for j, rule in enumerate(RULES):
        rows = 33 if n < 5000 else 6
        x, u = scores(n + j, rows, n, ("f32", "bf16", "f16")[j % 3], pad=(0, 1, 4, 7)[j % 4])
        check(emr, x, u, **rule)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 2, 300, 5000])
def test_rows(emr, rows, type):
    for n in (2, 9, 50, 700, 3000) if rows < 5000 else (2, 9, 50):
        x, u = scores(rows + n, rows, n, type)
        check(emr, x, u, t=0.8, p=0.9)
        check(emr, x, u[:, :1], k=5)


def test_settings_of_rows(emr):
    g = np.random.default_rng(3)
    for n in (20, 777, 5000, 70001):
        x, u = scores(n, 40, n)
        dev = lambda v, d: torch.tensor(v, dtype=d, device="cuda")  # noqa: E731
        t = dev(g.uniform(0.2, 2.0, 40), torch.float32)
        t[3], t[4], t[6] = 0.0, -1.0, float("inf")
        k = dev(g.integers(-1, 60, 40), torch.int32)
        p = dev(g.uniform(0.1, 1.2, 40), torch.float32)
        m = dev(g.uniform(0.0, 0.2, 40), torch.float32)
        check(emr, x, u, t=t, k=k, p=p, min_p=m)


@pytest.mark.parametrize("n", [5, 64, 200, 1024, 5000, 40000, 140000])
def test_equal_scores(emr, n):
    """Whole rows of one score, and rows of few scores: top-k and the nucleus end among equals, which rank
    by index."""
    u = torch.rand((4, 50), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    x = torch.zeros((4, n), device="cuda")
    x[1] = -0.0
    x[1, ::2] = 0.0
    x[2, ::3] = 1.0
    x[3] = torch.arange(n, device="cuda") % 5
    for rule in (dict(), dict(k=3), dict(k=n // 2 + 1), dict(p=0.5), dict(k=n - 1, p=0.3), dict(p=0.999),
                 dict(k=n // 3 + 1, p=0.77, t=0.5), dict(t=0.0)):
        check(emr, x, u, **rule)


@pytest.mark.parametrize("n", [4, 64, 300, 3000, 50000])
def test_special_values(emr, n):
    inf, nan = np.inf, np.nan
    x = torch.randn((9, n), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    x[0] = -inf
    x[1] = nan
    x[2, : n // 2] = nan
    x[3, 1], x[3, n - 1] = inf, inf
    x[4] = torch.finfo(torch.float32).min
    x[5] = -inf
    x[5, n - 1] = -FLT_MAX
    x[6] = FLT_MAX
    x[7, 0], x[7, 1] = FLT_MAX, -FLT_MAX
    x[8] *= 1e-40
    u = torch.tensor([0.0, 0.25, 0.5, 1 - 2.0 ** -24], device="cuda").repeat(9, 1)
    for rule in (dict(), dict(k=2), dict(p=0.4), dict(t=1e-30), dict(t=1e30), dict(min_p=1.0), dict(t=0.0)):
        check(emr, x, u, **rule)
    half = x.to(torch.bfloat16)
    check(emr, half, u, k=2, p=0.9)


@pytest.mark.parametrize("n", [64, 300, 3000, 12000, 50000])
@pytest.mark.parametrize("t", [1.2e-38, 2e-38, 1e-37, 2.7e-37])
def test_least_temperatures(emr, n, t):
    """Temperatures whose reciprocal times the bins of the exponent is past the largest float."""
    for spread in (3.0, 1e-37):
        x, u = scores(n, 12, n, spread=spread)
        for rule in (dict(), dict(k=3), dict(p=0.6), dict(k=200, p=0.9), dict(p=0.95, min_p=0.01)):
            check(emr, x, u, t=t, **rule)


def test_many_draws_of_one_row_follow_their_probabilities(emr):
    """Parents: 200000 draws from 1000 scores; each index as often as its probability says, within five
    standard deviations and one."""
    x, _ = scores(8, 1, 1000, spread=1.0, mask=False)
    u = torch.rand((1, 200000), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    index = check(emr, x, u, k=300)
    _, q, _ = whole(x, u[:, :1], k=300)
    p = (q[0].double() / q.sum()).cpu().numpy()
    seen = np.bincount(index[0].cpu().numpy(), minlength=1000)
    assert (np.abs(seen - 200000 * p) <= 5 * np.sqrt(200000 * p) + 1).all()


@pytest.mark.parametrize("n,draws", [(1, 5), (77, 4097), (1000, 1), (5000, 10000), (300007, 5000)])
def test_many_draws(emr, n, draws):
    x, _ = scores(n, 2, n, spread=1.0)
    u = torch.rand((2, draws), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    check(emr, x, u)
    check(emr, x, u, k=n // 2 + 1, t=0.5, min_p=1e-3)


def test_strides_and_shared_rows(emr):
    x, u = scores(4, 12, 600)
    wide = torch.full((12, 2, 901), 50.0, device="cuda")
    wide[:, 0, 301:] = x
    view = wide[:, 0, 301:]
    a, la = emr.emr_sample(x, u, top_p=0.8)
    b, lb = emr.emr_sample(view, u, top_p=0.8)
    assert torch.equal(a, b) and torch.equal(la, lb)
    c, _ = emr.emr_sample(x.t().contiguous().t(), u, top_p=0.8)
    assert torch.equal(a, c)
    one = x[3:4].expand(12, 600)
    assert one.stride(0) == 0
    check(emr, one, u, p=0.8)
    long, v = scores(5, 1, 6000)
    check(emr, long.expand(9, 6000), v.expand(9, 3).contiguous(), k=30)


@pytest.mark.parametrize("n,rows", [(65, (1 << 24) + 5), (8190, (1 << 22) + 5)])
def test_more_rows_than_a_launch_takes(emr, n, rows):
    """Rows (all the same one) beyond what workgroups of 256 and of 1024 threads in one launch cover: each
    draws as the row alone does."""
    x, _ = scores(n, 1, n)
    u = torch.rand((rows, 1), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    index, logp = emr.emr_sample(x.expand(rows, n), u, top_p=0.9)
    _, q, y = whole(x, u[:1], p=0.9)
    run = q[0].cumsum(0)
    want = torch.searchsorted(run, (u[:, 0].double() * run[-1].double()).long().clamp(max=int(run[-1]) - 1),
                              right=True)
    assert torch.equal(index[:, 0], want.int())
    lp = (y[0].double() - torch.log(run[-1].double() / 2.0 ** 31))[want]
    assert ((logp[:, 0].double() - lp).abs() <= 1e-12 + 2.0 ** -23 * lp.abs()).all()
    k = torch.full((rows,), 1, dtype=torch.int32, device="cuda")  # (settings by row: the last one is its own)
    k[-1] = 0
    index, _ = emr.emr_sample(x.expand(rows, n), u.fill_(1 - 2.0 ** -24), top_k=k)
    _, q, _ = whole(x, u[:1])
    assert (index[:-1] == x[0].argmax()).all()
    assert int(index[-1]) == int(q[0].nonzero().max())


def test_another_stream_and_graph(emr):
    """On a stream of its own, and captured: replays draw from what the scores then hold."""
    s = torch.cuda.Stream()
    for rows, n, draws in ((7, 30, 1), (5, 4000, 2), (2, 70000, 3), (1, 20000, 30000)):
        x, _ = scores(rows, rows, n, mask=False)
        u = torch.rand((rows, draws), device="cuda")
        want = [whole(y, u, k=50, p=0.9)[0] for y in (x, -x, x + 1)]
        torch.cuda.synchronize()
        got, _ = emr.emr_sample(x, u, top_k=50, top_p=0.9, stream=s)
        s.synchronize()
        assert torch.equal(got, want[0])
        g = torch.cuda.CUDAGraph()
        still = x.clone()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            index, _ = emr.emr_sample(still, u, top_k=50, top_p=0.9)
        for k, y in enumerate((x, -x, x + 1)):
            still.copy_(y)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(index, want[k])
            eager, _ = emr.emr_sample(y, u, top_k=50, top_p=0.9)
            assert torch.equal(index, eager)


def test_repeats(emr):
    x, u = scores(17, 64, 20000)
    first = emr.emr_sample(x, u, top_p=0.9)[0].clone()
    for _ in range(5):
        assert torch.equal(emr.emr_sample(x, u, top_p=0.9)[0], first)


# ----------------------------------------------------------------------------- loss

def loss64(x, index, scale, t):
    x = x.double() / float(np.float32(t))
    n = x.shape[1]
    some = (index >= 0) & (index < n) & (x > -np.inf).any(1)
    x = torch.where(some[:, None], x, 0.0)
    logp = x - torch.logsumexp(x, 1, keepdim=True)
    at = index.long().clamp(0, n - 1)[:, None]
    loss = -logp.gather(1, at)[:, 0] * scale.double()
    hot = torch.zeros_like(x).scatter_(1, at, 1.0)
    grad = (torch.exp(logp) - hot) * (scale.double() / t)[:, None]
    return torch.where(some, loss, 0.0), torch.where(some[:, None], grad, 0.0)


def loss_bounds(x, n, scale, t, loss, grad, type):
    """Errors of the loss and the gradient. The exponent y = (x - m) / T has three roundings of its size;
    softmax weights below e^-100 leave the sum as it is, so |y| counts up to 100: their error
    is e1 = 3 100 2^-24 (+ 2^-22 of the exponential); the sum of n positive terms over 64 lanes and
    a chain of n / 64 adds (n / 64 + 8) 2^-24; the loss adds the roundings of y at the index (3 |y| 2^-24) and
    its own; the gradient has one rounding to its type, at the type's least normal at least."""
    y = ((x.double() - x.double().amax(1, keepdim=True)) / t)
    worst = torch.where(y > -np.inf, y.abs(), 0.0).amax(1)
    e1 = 3 * torch.clamp(worst, max=100.0) * 2.0 ** -24 + 2.0 ** -22
    e = e1 + (n / 64 + 8) * 2.0 ** -24
    c = scale.double().abs()
    b_loss = c * (e + 4 * 2.0 ** -24 * worst) + 4 * 2.0 ** -24 * loss.abs() + 1e-30
    unit = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[type]
    least = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}[type]
    b_grad = (c / t * 4)[:, None] * (e[:, None]) * 1.0 + unit * grad.abs() + least
    return b_loss, b_grad


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [1, 2, 10, 63, 64, 65, 255, 1000, 1025, 4096, 9999, 40001])
def test_loss(emr, n, type):
    for rows, t in ((1, 1.0), (37, 0.4), (300 if n < 5000 else 9, 2.5)):
        x, _ = scores(n + rows, rows, n, type)
        g = torch.Generator(device="cuda").manual_seed(n)
        index = torch.randint(0, n, (rows,), generator=g, device="cuda", dtype=torch.int32)
        best = x.float().argmax(1).int()
        index = torch.where(x.float().gather(1, index.long()[:, None])[:, 0] > -1e4, index, best)
        index[2::7] = -1
        index[4::11] = n
        scale = torch.randn((rows,), generator=g, device="cuda")
        loss, grad = emr.emr_answer_loss(x, index, scale, temperature=t)
        want_l, want_g = loss64(x, index, scale, t)
        bl, bg = loss_bounds(x, n, scale, t, want_l, want_g, type)
        assert loss.dtype == torch.float32 and grad.dtype == x.dtype and grad.shape == x.shape
        assert ((loss.double() - want_l).abs() <= bl).all()
        assert ((grad.double() - want_g).abs() <= bg).all()
        assert (grad[x == -np.inf] == 0).all()


def test_loss_gradient_against_differences(emr):
    """Central differences of the loss (in doubles, of the 64-bit formula, h = 1e-4) against the kernel's
    gradient; their error is of the order h^2 / T^3."""
    x, _ = scores(2, 6, 12, mask=False, spread=1.0)
    index = torch.tensor([0, 3, 11, 5, 7, 1], dtype=torch.int32, device="cuda")
    scale = torch.tensor([1.0, -2.0, 0.5, 0.0, 3.0, 1.0], device="cuda")
    _, grad = emr.emr_answer_loss(x, index, scale, temperature=0.7)
    h = 1e-4
    for j in range(12):
        d = torch.zeros_like(x, dtype=torch.float64)
        d[:, j] = h
        up, _ = loss64(x.double() + d, index, scale, 0.7)
        down, _ = loss64(x.double() - d, index, scale, 0.7)
        assert ((up - down) / (2 * h) - grad[:, j].double()).abs().max() < 1e-6


def test_loss_of_masked_answers_scale_and_views(emr):
    x = torch.zeros((4, 6), device="cuda")
    x[:, 2:] = -np.inf
    index = torch.tensor([0, 3, 1, 2], dtype=torch.int32, device="cuda")
    loss, grad = emr.emr_answer_loss(x, index)
    assert torch.isinf(loss[[1, 3]]).all() and (loss[[0, 2]] - np.log(2)).abs().max() < 1e-6
    want = torch.zeros(4, 6, device="cuda")
    want[:, :2] = 0.5
    want[torch.arange(4), index.long()] -= 1
    assert (grad - want).abs().max() < 1e-6
    x, _ = scores(3, 20, 333)
    wide = torch.zeros((20, 400), device="cuda")
    wide[:, 61:394] = x
    index = torch.arange(20, dtype=torch.int32, device="cuda") * 16
    a = emr.emr_answer_loss(x, index)
    b = emr.emr_answer_loss(wide[:, 61:394], index)
    c = emr.emr_answer_loss(x, index, torch.ones(20, device="cuda"))
    for p, q, r in zip(a, b, c):
        assert torch.equal(p, q) and torch.equal(p, r)


def test_loss_nothing_and_in_place(emr):
    import ctypes as C
    x = torch.zeros((0, 5), device="cuda")
    loss, grad = emr.emr_answer_loss(x, torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert loss.numel() == 0 and grad.shape == (0, 5)
    index, logp = emr.emr_sample(x, torch.zeros((0, 2), device="cuda"))
    assert index.shape == (0, 2)
    index, logp = emr.emr_sample(torch.zeros((3, 5), device="cuda"), torch.zeros((3, 0), device="cuda"))
    assert index.shape == (3, 0)
    for n in (9, 700, 20000):  # the gradient over the scores
        x, _ = scores(n, 30, n, mask=False)
        index = torch.arange(30, dtype=torch.int32, device="cuda") % n
        loss, grad = emr.emr_answer_loss(x, index)
        st, y = emr._scores(x.clone())
        out = torch.empty(30, device="cuda")
        emr._check(emr.lib().emr_answer_loss(C.byref(st), C.c_void_p(index.data_ptr()), None, C.c_float(1.0),
                                             C.c_void_p(out.data_ptr()), C.c_void_p(y.data_ptr()), n,
                                             emr._stream_ptr()))
        torch.cuda.synchronize()
        assert torch.equal(y, grad) and torch.equal(out, loss)


@pytest.mark.parametrize("n,rows", [(65, (1 << 26) + 5), (2000, (1 << 24) + 5), (20000, (1 << 23) + 5),
                                    (33000, (1 << 22) + 5)])
def test_loss_of_more_rows_than_a_launch_takes(emr, n, rows):
    """Rows (all the same one) beyond what one launch covers by waves, workgroups of 256, of 512 and of 1024
    threads: each row's loss is the one of a few rows alone, for its own index."""
    import ctypes as C
    x, _ = scores(n, 1, n, "bf16", mask=False)
    g = torch.Generator(device="cuda").manual_seed(n)
    picks = torch.randint(0, n, (7,), generator=g, device="cuda", dtype=torch.int32)
    few, grad = emr.emr_answer_loss(x.expand(7, n), picks, temperature=0.5)
    want, _ = loss64(x.expand(7, n), picks, torch.ones(7, device="cuda"), 0.5)
    bound, _ = loss_bounds(x.expand(7, n), n, torch.ones(7, device="cuda"), 0.5, want, grad.double(), "bf16")
    assert ((few.double() - want).abs() <= bound).all()
    at = torch.arange(rows, device="cuda") % 7
    index = picks[at]
    index[1::1000] = -1
    loss = torch.full((rows,), -1.0, device="cuda")
    st = emr.emr_scores(x.data_ptr(), emr.EMR_BF16, rows, n, 0)
    emr._check(emr.lib().emr_answer_loss(C.byref(st), index.data_ptr(), None, C.c_float(0.5), loss.data_ptr(), None,
                                         0, emr._stream_ptr()))
    assert torch.equal(loss, torch.where(index < 0, 0.0, few[at]))


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [65529, 65530, 65533, 65534, 70001])
def test_loss_of_rows_around_the_registers(emr, n, type):
    """The longest rows that a workgroup's registers hold (fewer by up to a group where unaligned), and those read
    three times."""
    test_loss(emr, n, type)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
def test_long_losses_in_place_and_strided(emr, type):
    import ctypes as C
    n = 70003
    x, _ = scores(n, 5, n, type, pad=6)
    index = x.float().argmax(1).int()
    loss, grad = emr.emr_answer_loss(x, index, temperature=0.7)
    wide = torch.empty((5, n + 6), dtype=x.dtype, device="cuda")
    y = wide[:, 3:n + 3]
    y.copy_(x)
    wide[:, :3], wide[:, n + 3:] = 7.0, 7.0
    st, held = emr._scores(y)
    assert held is y
    out = torch.empty(5, device="cuda")
    emr._check(emr.lib().emr_answer_loss(C.byref(st), index.data_ptr(), None, C.c_float(0.7), out.data_ptr(),
                                         y.data_ptr(), n + 6, emr._stream_ptr()))
    torch.cuda.synchronize()
    assert torch.equal(y, grad) and torch.equal(out, loss)
    assert (wide[:, :3] == 7).all() and (wide[:, n + 3:] == 7).all()


@pytest.mark.parametrize("n", [1048573, 1048574, 1100003, 2200001])
def test_parts_of_more_entries(emr, n):
    """Rows of more than 4096 parts of 256 scores: parts of 512 and more, limits and draws inside them, and equal
    scores across them."""
    for j, rule in enumerate((dict(), dict(k=n // 3, t=3.0), dict(k=100, p=0.9), dict(p=0.97), dict(p=0.5, t=20.0),
                              dict(min_p=0.05, t=2.0))):
        x, u = scores(n + j, 2, n, ("f32", "bf16", "f16")[j % 3], pad=(0, 1, 3)[j % 3])
        check(emr, x, u, **rule)
    x = torch.zeros((2, n), device="cuda")
    x[1] = torch.arange(n, device="cuda") % 5
    u = torch.rand((2, 300), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    for rule in (dict(), dict(k=n // 2 + 1), dict(p=0.5), dict(k=n - 1, p=0.3), dict(k=n // 3 + 1, p=0.77, t=0.5)):
        check(emr, x, u, **rule)


def test_longest_rows(emr):
    """Two rows of 2^31 - 1 scores, the second one unaligned and beyond 2^32 bytes, of which a few are not masked:
    the draws, losses and gradients of those few alone."""
    n, at = (1 << 31) - 1, [0, 5, 1000, 1 << 30, (1 << 31) - 300, (1 << 31) - 2]
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough free device memory")
    few = torch.tensor([[0.5, 1.0, -2.0, 1.0, 0.25, 1.5], [-1.0, 2.0, 0.0, 2.0, 2.0, 0.5]], dtype=torch.bfloat16,
                       device="cuda")
    x = torch.full((2, n), -np.inf, dtype=torch.bfloat16, device="cuda")
    place = torch.tensor(at, device="cuda")
    x[:, place] = few
    u = torch.rand((2, 40), device="cuda", generator=torch.Generator(device="cuda").manual_seed(0))
    for rule in (dict(), dict(top_k=3), dict(top_p=0.6), dict(top_k=5, top_p=0.8, min_p=0.1, temperature=0.6),
                 dict(temperature=0.0)):
        want, lp = emr.emr_sample(few, u, **rule)
        index, logp = emr.emr_sample(x, u, **rule)
        assert torch.equal(index.long(), place[want.long()]) and torch.equal(logp, lp)
    pick = torch.tensor([5, 3], device="cuda")
    loss, grad = emr.emr_answer_loss(x, place[pick].int(), temperature=0.5)
    want, g = emr.emr_answer_loss(few, pick.int(), temperature=0.5)
    # (sums of few and of many lanes: their roundings, and the gradient's to bfloat16)
    assert ((loss - want).abs() <= 2.0 ** -20 * (1 + want.abs())).all()
    assert ((grad[:, place].float() - g.float()).abs() <= 2.0 ** -8 * g.float().abs() + 2.0 ** -20).all()
    assert int((grad[:, ::4099] != 0).sum()) <= 12 and int(torch.count_nonzero(grad[1, 6:1000])) == 0
