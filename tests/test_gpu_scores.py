"""Operators on rows of class scores against plain implementations in 64 bits (scoreutil.py).

Tolerances, in steps of eps = 2^-24 (half a step of float32) unless said otherwise:
* the k best scores are exact, except the logarithm of votes (at most 2 steps, logf);
* a sum of exponentials over n classes: every thread adds at most n / 64 + 1 terms, then trees of
  at most 11 levels; each term is off by at most 4 steps, for the argument's product, its
  exponential and the terms' scaling.  Relative error of the sum: (n / 64 + 16) eps;
* a log-probability is a difference (|z - m| steps of it for the product with 1 / t), a logarithm of
  the sum and two additions: (D + n / 64 + 16) 4 eps with D the largest |z - m|;
* gradients: the same relative to q and to p, and half a step of the output's type.
"""
import warnings

import numpy as np
import pytest

from tests import scoreutil as SU

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS = 2.0 ** -24
INF = float("inf")
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "u8": torch.uint8}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def sc():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1111_1373_amd import scores
    return scores


def _host(x):
    """numpy array of a device tensor (bfloat16 widened)."""
    x = x.detach()
    return (x.float() if x.dtype == torch.bfloat16 else x).cpu().numpy()


def _scores(rng, n, classes, kind, scale=3.0):
    """Device scores with masked classes, NaN, infinities, ties and empty rows among them."""
    if kind == "u8":
        x = (rng.random((n, classes)) ** 4 * 40).astype(np.uint8)
        x[::7] = 0
        return torch.from_numpy(x).cuda()
    x = (rng.standard_normal((n, classes)) * scale).astype(np.float32)
    for r in range(n):
        what = r % 9
        if what == 1:
            x[r, rng.random(classes) < 0.5] = -INF
        elif what == 2:
            x[r] = -INF
        elif what == 3:
            x[r, rng.random(classes) < 0.3] = np.nan
        elif what == 4:
            x[r] = np.float32(rng.integers(-3, 4))                      # one value everywhere
        elif what == 5:
            x[r] = rng.integers(-2, 3, classes)                         # many ties, both zeros
            x[r, x[r] == 0] *= np.where(rng.random((x[r] == 0).sum()) < 0.5, -1, 1)
        elif what == 6:
            x[r] = np.sort(x[r])[:: -1 if r % 2 else 1]
        elif what == 7 and classes > 2:
            x[r, rng.integers(0, classes, 2)] = INF
        elif what == 8:
            lowest = torch.finfo(TYPES[kind]).min
            x[r, rng.random(classes) < 0.5] = lowest                    # a mask by the lowest value
    return torch.from_numpy(x).to(TYPES[kind]).cuda()


def _strided(x, how):
    """The same rows, dense, or inside a wider matrix that starts them off any boundary."""
    if how == "dense":
        return x
    n, classes = x.shape
    wide = torch.zeros(n, classes + 5, dtype=x.dtype, device=x.device)
    wide[:, 3:3 + classes] = x
    return wide[:, 3:3 + classes]


SHAPES = [(1, 1), (700, 2), (300, 7), (65, 8), (300, 9), (129, 31), (257, 32), (70, 64), (40, 65),
          (50, 100), (30, 1000), (27, 1024), (20, 1025), (18, 5000), (10, 8192), (10, 8193),
          (18, 40001)]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "u8"])
@pytest.mark.parametrize("how", ["dense", "strided"])
@pytest.mark.parametrize("n,classes", SHAPES)
def test_top_scores(sc, n, classes, kind, how):
    rng = np.random.default_rng([n, classes, len(kind), len(how)])
    x = _strided(_scores(rng, n, classes, kind), how)
    for k in sorted({1, min(classes, 5), min(classes, 64), min(classes, 256)}):
        print("top", n, classes, kind, how, k, flush=True)
        values, index, lse = sc.top_scores(x, k)
        want_v, want_i, want_l = SU.top_scores(_host(x), k)
        np.testing.assert_array_equal(_host(index), want_i)
        if kind == "u8":
            np.testing.assert_allclose(_host(values), want_v, rtol=4 * EPS)
        else:
            np.testing.assert_array_equal(_host(values), want_v.astype(np.float32))
        got = _host(lse).astype(np.float64)
        ok = np.isfinite(want_l)
        np.testing.assert_array_equal(got[~ok], want_l[~ok])
        err = np.abs(got[ok] - want_l[ok])
        assert (err <= (classes / 64 + 16) * EPS + 2 * EPS * np.abs(want_l[ok])).all(), err.max()


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.7, top_k=5),
            dict(temperature=1.3, top_p=0.8), dict(top_k=40, top_p=0.9, min_p=0.05),
            dict(min_p=0.2), dict(temperature=0.5, top_k=700, top_p=0.5), dict(top_p=0.0),
            dict(top_k=1), dict(min_p=1.0), dict(temperature=0.01, top_p=0.95),
            dict(temperature=20.0, top_p=0.999)]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "u8"])
@pytest.mark.parametrize("how", ["dense", "strided"])
@pytest.mark.parametrize("n,classes", SHAPES)
def test_sample(sc, n, classes, kind, how):
    rng = np.random.default_rng([n, classes, len(kind), len(how), 1])
    x = _strided(_scores(rng, n, classes, kind), how)
    u = rng.random(n).astype(np.float32)
    u[:3] = [0.0, 1 - 2.0 ** -24, 0.5][: min(3, n)]
    ud = torch.from_numpy(u).cuda()
    for s in SETTINGS:
        print("sample", n, classes, kind, how, s, flush=True)
        got = _host(sc.sample(x, ud, **s))
        SU.check_sample(got, _host(x), u, **s, note=str(s))


@pytest.mark.parametrize("kind", ["f32", "u8"])
@pytest.mark.parametrize("classes", [5, 64, 65, 100, 255, 256, 257, 1500])
def test_sample_of_as_many_as_there_are(sc, classes, kind):
    """top_k at, below and above the number of classes, and around what the kernels split by."""
    rng = np.random.default_rng(classes)
    x = _scores(rng, 27, classes, kind)
    u = rng.random(27).astype(np.float32)
    ud = torch.from_numpy(u).cuda()
    for k in (classes - 1, classes, classes + 1, 32, 33, 96, 97, 256, 257):
        for t in (1.0, 0.0):
            print("as many", classes, kind, k, t, flush=True)
            out = torch.full((27,), 123456, dtype=torch.int32, device="cuda")
            sc.sample(x, ud, t, k, 0.95, out=out)
            SU.check_sample(_host(out), _host(x), u, t, k, 0.95)
            per_row = torch.full((27,), k, dtype=torch.int32, device="cuda")
            out.fill_(123456)
            sc.sample(x, ud, t, per_row, 0.95, out=out)
            SU.check_sample(_host(out), _host(x), u, t, k, 0.95)


@pytest.mark.parametrize("kind,classes", [("f32", 40), ("bf16", 300), ("f16", 3001), ("u8", 12),
                                          ("bf16", 20_000)])
def test_sample_settings_of_each_row(sc, kind, classes):
    rng = np.random.default_rng(classes)
    n = 64
    x = _scores(rng, n, classes, kind)
    u = rng.random(n).astype(np.float32)
    t = rng.choice([0.0, 0.5, 1.0, 1.7, -1.0, np.nan], n).astype(np.float32)
    k = rng.choice([-1, 0, 1, 3, 50, 2000, 1 << 30], n).astype(np.int32)
    p = rng.choice([-1.0, 0.0, 0.4, 0.9, 1.0, 2.0, np.nan], n).astype(np.float32)
    m = rng.choice([-1.0, 0.0, 0.1, 1.0, 3.0, np.nan], n).astype(np.float32)
    dev = [torch.from_numpy(v).cuda() for v in (u, t, k, p, m)]
    print("settings", kind, classes, flush=True)
    got = _host(sc.sample(x, *dev))
    SU.check_sample(got, _host(x), u, t, k, np.where(np.isnan(p), 1, np.maximum(p, 0)), m)
    # random numbers outside [0, 1): as the nearest inside, NaN as 0
    odd = torch.tensor([-1.0, float("nan"), 1.0, 7.0] * 16, device="cuda")
    near = np.array([0.0, 0.0, 1.0, 1.0] * 16, dtype=np.float32)
    SU.check_sample(_host(sc.sample(x, odd, 1.0)), _host(x), near)


@pytest.mark.parametrize("kind,classes,values", [("bf16", 100_000, 1), ("f32", 60_000, 1),
                                                 ("bf16", 200_000, 2), ("u8", 150_000, 3),
                                                 ("f16", 5_000, 2)])
def test_long_rows_of_few_values(sc, kind, classes, values):
    """More classes of the deciding score than a workgroup collects: the ties are counted."""
    rng = np.random.default_rng(classes + values)
    x = rng.integers(1, 1 + values, (3, classes))
    x = torch.from_numpy(x.astype(np.uint8)).to(TYPES[kind]).cuda()
    u = rng.random(3).astype(np.float32)
    ud = torch.from_numpy(u).cuda()
    for k in (1, 64, 256):
        print("few values", kind, classes, values, k, flush=True)
        v, i, _ = sc.top_scores(x, k)
        np.testing.assert_array_equal(_host(i), SU.top_scores(_host(x), k)[1])
    for s in (dict(top_k=200), dict(top_k=classes // 3), dict(top_p=0.3), dict(top_p=0.99),
              dict(top_k=classes // 2, top_p=0.7, temperature=0.9)):
        print("few values", kind, classes, values, s, flush=True)
        SU.check_sample(_host(sc.sample(x, ud, **s)), _host(x), u, **s)


def test_neighbouring_best_classes(sc):
    """The best classes side by side, where one wavefront meets most of them, and sorted rows."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((8, 60_000)).astype(np.float32)
    x[0, 4096:4900] += 50
    x[1, :300] += 50
    x[2, -700:] += 50
    x[3] = np.sort(x[3])
    x[4] = np.sort(x[4])[::-1]
    x[5] = -INF
    x[5, 777:900] = rng.standard_normal(123)            # fewer scores than asked for, side by side
    x[6, ::2] = np.nan
    x[7, 30_000:] = -INF
    for rows in (x, np.tile(x, (40, 1))):
        xd = torch.from_numpy(rows).cuda()
        for kind in ("f32", "bf16"):
            xk = xd.to(TYPES[kind])
            for k in (1, 40, 96, 97, 256):
                print("neighbours", len(rows), kind, k, flush=True)
                v, i, _ = sc.top_scores(xk, k)
                np.testing.assert_array_equal(_host(i)[:8], SU.top_scores(_host(xk)[:8], k)[1])
                assert torch.equal(i, i[:8].repeat(len(rows) // 8, 1))


def _teacher(rng, n, classes, k):
    values = (rng.standard_normal((n, k)) * 3).astype(np.float32)
    index = rng.integers(0, classes, (n, k)).astype(np.int32)         # classes occur twice
    index[rng.random((n, k)) < 0.1] = -1
    index[1::11, -1] = classes                                        # no class either
    index[3::11] = -1
    values[5::11, 0] = -INF
    values[6::11] = -INF
    return values, index


def _check_distill(x, values, index, t, g, loss, grad, kind):
    n, classes = x.shape
    want_l, want_g = SU.distill(x, values, index, t, g)
    x64 = x.astype(np.float64)
    z = np.where(x64 == -INF, np.nan, x64)
    with np.errstate(all="ignore"):
        with warnings.catch_warnings():
            warnings.simplefilter("ignore")
            spread = np.nan_to_num(np.nanmax(z, 1) - np.nanmin(z, 1), nan=0.0, posinf=0.0) / t
            vs = np.where(np.isfinite(values), values, np.nan)
            vspread = np.nan_to_num(np.nanmax(vs, 1) - np.nanmin(vs, 1)) / t
            m = np.nanmax(z, 1, keepdims=True)
        d = (spread + vspread + classes / 64 + 16) * 4 * EPS
        ok = np.isfinite(want_l)
        np.testing.assert_array_equal(np.isnan(loss), np.isnan(want_l))
        np.testing.assert_array_equal(loss[~ok], want_l[~ok].astype(np.float32))
        tol = t * t * d * 2 + 2 * EPS * np.abs(want_l)
        bad = np.abs(loss - want_l)[ok] > tol[ok]
        assert not bad.any(), (np.abs(loss - want_l)[ok][bad], tol[ok][bad])
        # |error| <= g t (q + p) d, half a step of the type, and its smallest number
        q = np.nan_to_num(np.exp((np.where(np.isnan(z), -INF, z) - m) / t))
        q = q / np.maximum(q.sum(1, keepdims=True), 1e-300)
        p = np.abs(q * (t * g)[:, None] - want_g)
        tol = (np.abs(t * g)[:, None] * q + p) * d[:, None] * 2 + HALF_STEP[kind] * np.abs(want_g) * 1.01
        tol += {"f32": 2.0 ** -125, "f16": 2.0 ** -25, "bf16": 2.0 ** -125}[kind]
        np.testing.assert_array_equal(np.isnan(grad), np.isnan(want_g))
        err = np.abs(grad - want_g)
        bad = err > tol
        assert not bad.any(), (err[bad][:5], tol[bad][:5], np.argwhere(bad)[:5])


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("how", ["dense", "strided"])
@pytest.mark.parametrize("n,classes,k", [(1, 1, 1), (400, 2, 1), (100, 7, 7), (130, 32, 4),
                                         (40, 64, 64), (12, 40, 200), (45, 65, 9), (30, 1000, 100),
                                         (25, 2048, 256), (14, 2049, 33), (12, 9001, 64),
                                         (700, 2100, 3), (520, 8200, 16), (5, 40_003, 128),
                                         (1, 150_001, 256), (600, 16_400, 8)])
def test_distill(sc, n, classes, k, kind, how):
    rng = np.random.default_rng([n, classes, k, len(kind), len(how)])
    x = (rng.standard_normal((n, classes)) * 3).astype(np.float32)
    x[2::5, ::3] = -INF
    if n > 4:
        x[4] = -INF
    if n > 24:
        x[21, 0] = np.nan
        x[22, classes // 2] = INF
    values, index = _teacher(rng, n, classes, k)
    g = (rng.standard_normal(n) * 2).astype(np.float32)
    x = _strided(torch.from_numpy(x).to(TYPES[kind]).cuda(), how)
    dev = [torch.from_numpy(v).cuda() for v in (values, index)]
    gd = torch.from_numpy(g).cuda()
    for t in (1.0, 2.5):
        print("distill", n, classes, k, kind, how, t, flush=True)
        loss, grad = sc.distill_grad(x, *dev, gd, t)
        _check_distill(_host(x), values, index, t, g, _host(loss), _host(grad), kind)
        print("distill, two calls", flush=True)
        loss2, stats = sc.distill_forward(x, *dev, t)
        out = _strided(torch.full((n, classes), 7.0, dtype=x.dtype, device="cuda"), how)
        grad2 = sc.distill_backward(x, *dev, stats, gd, t, out=out)
        assert grad2 is out
        _check_distill(_host(x), values, index, t, g, _host(loss2), _host(grad2), kind)
        if how == "strided" and n > 1:      # what lies between the rows is left alone
            base = out._base if out._base is not None else out
            assert (base[:, :3] == 0).all() and (base[:, 3 + classes:] == 0).all()


def test_distill_gradient_by_differences(sc):
    """Central differences of the loss, computed in 64 bits from the definition, against autograd."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((6, 90)).astype(np.float32)
    values, index = _teacher(rng, 6, 90, 12)
    g = rng.random(6).astype(np.float32)
    xd = torch.from_numpy(x).cuda().requires_grad_()
    loss = sc.distill_loss(xd, torch.from_numpy(values).cuda(), torch.from_numpy(index).cuda(), 1.5)
    (loss * torch.from_numpy(g).cuda()).sum().backward()
    h = 1e-5
    for r, c in [(0, 0), (1, 50), (2, 89), (4, int(max(index[4, 1], 0))), (5, 17)]:
        lo, hi = x.astype(np.float64), x.astype(np.float64)
        lo[r, c] -= h
        hi[r, c] += h
        want = sum(s * SU.distill(v, values, index, 1.5, g)[0][r] for s, v in ((1, hi), (-1, lo)))
        want *= g[r] / (2 * h)
        # differences: h^2 of a third derivative of order 1, and 2^-53 * 10 / h
        assert abs(float(xd.grad[r, c]) - want) <= 1e-9 + 1e-10 + 64 * EPS, (r, c)


def test_distill_autograd(sc):
    rng = np.random.default_rng(6)
    n, classes, k = 33, 500, 10
    x = torch.from_numpy(rng.standard_normal((n, classes)).astype(np.float32)).cuda()
    values, index = (torch.from_numpy(v).cuda() for v in _teacher(rng, n, classes, k))
    g = torch.full((n,), 1.0 / n, device="cuda")
    _, want = sc.distill_grad(x, values, index, g, 2.0)
    a = x.clone().requires_grad_()
    sc.distill_loss(a, values, index, 2.0).mean().backward()
    # 1 / n reaches the backward pass as a broadcast number
    np.testing.assert_array_equal(_host(a.grad), _host(want))
    b = x.clone().requires_grad_()                                       # through a slice
    sc.distill_loss(b[:, 100:], values, torch.clamp(index, max=399), 2.0).sum().backward()
    assert (b.grad[:, :100] == 0).all() and (b.grad[:, 100:] != 0).any()
    with pytest.raises(RuntimeError):
        loss = sc.distill_loss(a, values, index)
        gr, = torch.autograd.grad(loss.sum(), a, create_graph=True)
        gr.sum().backward()


def test_nothing_to_do(sc):
    for kind in ("f32", "u8"):
        x = torch.empty(0, 9, dtype=TYPES[kind], device="cuda")
        v, i, l = sc.top_scores(x, 3)
        assert v.shape == (0, 3) and i.shape == (0, 3) and l.shape == (0,)
        assert sc.sample(x, torch.empty(0, device="cuda")).shape == (0,)
    x = torch.empty(0, 9, device="cuda", requires_grad=True)
    loss = sc.distill_loss(x, torch.empty(0, 2, device="cuda"),
                           torch.empty(0, 2, dtype=torch.int32, device="cuda"))
    loss.sum().backward()
    assert x.grad.shape == (0, 9)


@pytest.mark.parametrize("classes,kind", [(32, "u8"), (50, "f32"), (700, "bf16"), (40_000, "f16")])
def test_in_a_hip_graph(sc, classes, kind):
    """Two graphs and eager calls in turn, every replay against the eager result."""
    rng = np.random.default_rng(classes)
    n = 40
    xs = [_scores(rng, n, classes, kind) for _ in range(2)]
    u = torch.from_numpy(rng.random(n).astype(np.float32)).cuda()
    student = torch.zeros(n, classes, device="cuda")
    g = torch.ones(n, device="cuda")

    def chain(x):
        v, i, l = sc.top_scores(x, 8)
        label = sc.sample(x, u, 0.8, 0, 0.9)
        v = torch.where(torch.isfinite(v), v, -INF)
        loss, grad = sc.distill_grad(student, v, i, g, 2.0)
        return v, i, l, label, loss, grad

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        chain(xs[0])
    torch.cuda.synchronize()
    ins = [x.clone() for x in xs]
    graphs, outs = [], []
    for x in ins:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(chain(x))
        graphs.append(gr)
    for rep in range(4):
        for which in (0, 1):
            src = xs[(which + rep) % 2]
            ins[which].copy_(src)
            for o in outs[which]:
                o.fill_(77)
            torch.cuda.synchronize()
            graphs[which].replay()
            want = chain(src)
            torch.cuda.synchronize()
            for a, b in zip(outs[which], want):
                np.testing.assert_array_equal(_host(a), _host(b))


def test_training_step_in_a_hip_graph(sc):
    """Loss and backward pass captured while no eager graph of the same leaf lives."""
    rng = np.random.default_rng(8)
    n, classes, k = 24, 9000, 16
    x = torch.from_numpy(rng.standard_normal((n, classes)).astype(np.float32)).cuda().requires_grad_()
    values, index = (torch.from_numpy(v).cuda() for v in _teacher(rng, n, classes, k))

    def step():
        loss = sc.distill_loss(x, values, index, 2.0)
        grad, = torch.autograd.grad(loss, x, torch.ones_like(loss))
        return loss.detach(), grad

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    want = [_host(v) for v in step()]
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        outs = step()
    for _ in range(3):
        for o in outs:
            o.fill_(5)
        torch.cuda.synchronize()
        gr.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            np.testing.assert_array_equal(_host(o), w)


def test_on_other_streams(sc):
    """The same calls on four streams at once."""
    rng = np.random.default_rng(9)
    n, classes = 16, 30_000
    x = _scores(rng, n, classes, "bf16")
    u = torch.from_numpy(rng.random(n).astype(np.float32)).cuda()
    s = torch.zeros(n, classes, device="cuda", dtype=torch.float16)
    v, i, l = sc.top_scores(x, 20)
    v = torch.where(torch.isfinite(v), v, -INF)
    g = torch.ones(n, device="cuda")

    def calls(stream):
        return (*sc.top_scores(x, 20, stream=stream), sc.sample(x, u, 0.9, 0, 0.8, stream=stream),
                *sc.distill_grad(s, v, i, g, 2.0, stream=stream))

    want = [_host(o) for o in calls(None)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    got = [calls(st) for _ in range(3) for st in streams]
    torch.cuda.synchronize()
    for outs in got:
        for a, b in zip(outs, want):
            np.testing.assert_array_equal(_host(a), b)


def test_results_do_not_depend_on_the_run(sc):
    rng = np.random.default_rng(10)
    x = _scores(rng, 18, 70_000, "f32")
    u = torch.from_numpy(rng.random(18).astype(np.float32)).cuda()
    a = sc.sample(x, u, 1.0, 0, 0.95)
    values, index, lse = sc.top_scores(x, 100)
    for _ in range(5):
        assert torch.equal(a, sc.sample(x, u, 1.0, 0, 0.95))
        v, i, l = sc.top_scores(x, 100)
        assert torch.equal(v, values) and torch.equal(i, index) and torch.equal(l, lse)


def test_offsets_past_32_bits(sc):
    """Rows more than 2^32 bytes into a table, of 16 GB."""
    classes, n = 1 << 19, 4100
    x = torch.zeros(n, classes, dtype=torch.float32, device="cuda")[:, : classes - 1]
    assert x.stride(0) * (n - 1) > 1 << 31
    x[n - 1, classes - 2] = 9.0
    x[n - 2, 12345] = 9.0
    v, i, _ = sc.top_scores(x, 2)
    assert i[n - 1].tolist() == [classes - 2, 0] and i[n - 2].tolist() == [12345, 0]
    assert v[n - 1].tolist() == [9.0, 0.0]
    label = sc.sample(x, torch.zeros(n, device="cuda"), 0.1, 0, 0.5)
    assert label[n - 1] == classes - 2 and label[n - 2] == 12345
    value = torch.zeros(n, 1, device="cuda")
    g = torch.ones(n, device="cuda")
    loss, grad = sc.distill_grad(x, value, i[:, :1].contiguous(), g, 1.0)
    assert abs(float(grad[n - 1, classes - 2]) - (8103.0839 / (8103.0839 + classes - 2) - 1)) < 1e-4
    del x, grad
