"""Layer norm of dense and of pulled rows, and its backward pass, against the formulas in 64 bits.

Tolerances: u is the unit rounding of the arithmetic (2^-24, fp64 values 2^-53).  A sum of a row is made of at most 32 values
one after the other per thread and a tree of at most 10 additions, so a mean is off by at most 42 u times the mean of the
magnitudes, a variance by some 90 u of itself (its terms' roundings and the mean's square included) and rstd by 48 u; STEPS = 64
covers the few roundings that follow.  A sum over rows: at most 32 rows per team one after the other, 32 sums of blocks, trees
of 32: COLUMN_STEPS = 160 with the roundings of the terms.  The last rounding to the output's type adds half a step of it.
"""
import threading

import numpy as np
import pytest
import torch

from paper_2104_00501_b200 import binding
from tests.common import dev_keys

pytestmark = pytest.mark.gpu

F32, F64, F16, BF16 = torch.float32, torch.float64, torch.float16, torch.bfloat16
STEPS, COLUMN_STEPS = 64, 160


def unit(t):
    return 2.0 ** -53 if t == F64 else 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    return torch.finfo(t).tiny * torch.finfo(t).eps       # values below the normal range are rounded to multiples of this


@pytest.fixture(scope="module")
def store():
    s = binding.Store(64, 64)
    yield s
    s.close()


def make(n, length, dtype, seed, gap=0, scale=1.5, shift=0.3):
    """A matrix whose rows lie `gap` values apart from one another, on the GPU."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((n, length + gap), generator=g, dtype=F64) * scale + shift).to(dtype)
    return x.cuda()[:, :length]


def params(length, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (1 + 0.2 * torch.randn(length, generator=g)).to(dtype).cuda(), (0.3 * torch.randn(length, generator=g)).to(dtype).cuda()


def reference(x, w, b, eps):
    x = x.double()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1 / torch.sqrt((d * d).mean(1) + eps)
    h = d * rstd[:, None]
    w = torch.ones_like(x[0]) if w is None else w.double()
    b = torch.zeros_like(x[0]) if b is None else b.double()
    return h * w + b, mean, rstd, h, w, b


def check_forward(x, w, b, eps, y, mean, rstd):
    ry, rm, rr, h, wd, bd = reference(x, w, b, eps)
    u = unit(x.dtype)
    size = x.double().abs().mean(1)
    tol = u * STEPS * ((h * wd).abs() + (size * rr)[:, None] * wd.abs() + bd.abs()) + half_step(y.dtype) * ry.abs() + tiny(y.dtype)
    assert ((y.double() - ry).abs() <= tol).all(), ((y.double() - ry).abs() / tol).max()
    assert ((mean.double() - rm).abs() <= u * STEPS * size + tiny(F32)).all()
    # rstd: relative, plus what the mean's error adds to a variance that is itself small against the mean
    assert ((rstd.double() - rr).abs() <= u * STEPS * rr + (u * STEPS * size * rr) ** 2 * rr).all()


SHAPES = [(1, 1), (5, 2), (3, 3), (1, 64), (7, 64), (33, 100), (64, 101), (300, 128), (9, 129), (40, 300), (17, 511), (5, 513), (6, 1000),
          (12, 1024), (3, 1500), (5, 2050), (2, 4096), (4, 4097), (2, 8192), (3, 8200), (1, 16384), (2, 20000), (2500, 32), (700, 500),
          (301, 640), (601, 1024), (299, 2048), (303, 4096), (170, 8200), (151, 16384), (150, 33000)]


@pytest.mark.parametrize("dtype", [F32, F64, F16, BF16])
@pytest.mark.parametrize("n,length", SHAPES)
def test_forward_meets_the_formula(store, n, length, dtype):
    w, b = params(length, dtype, 1)
    x = make(n, length, dtype, n + length)
    y, mean, rstd = store.layer_norm(x, w, b, eps=1e-5)
    assert y.dtype == dtype
    check_forward(x, w, b, 1e-5, y, mean, rstd)


@pytest.mark.parametrize("x_type,y_type,w_type", [(F32, BF16, F32), (F32, F16, F32), (BF16, BF16, F32), (F16, F16, F32), (F32, F32, None)])
@pytest.mark.parametrize("n,length,gap", [(21, 96, 0), (21, 96, 8), (13, 101, 3), (6, 1024, 5), (3, 5000, 1), (2, 17000, 24)])
def test_forward_of_mixed_types_and_of_rows_that_lie_apart(store, n, length, gap, x_type, y_type, w_type):
    w, b = params(length, w_type, 2) if w_type else (None, None)
    x = make(n, length, x_type, 3, gap)
    whole = torch.full((n + 2, length + gap + 1), 7.0, dtype=y_type, device="cuda")
    out = whole[1:n + 1, :length]
    y, mean, rstd = store.layer_norm(x, w, b, eps=1e-3, out=out)
    check_forward(x, w, b, 1e-3, y, mean, rstd)
    whole[1:n + 1, :length] = 7.0
    assert (whole == 7.0).all()                             # nothing beside the rows was written
    assert store.status_check() == 0


def test_forward_without_statistics_in_place_and_with_one_parameter(store):
    x = make(50, 256, F32, 4)
    w, b = params(256, F32, 5)
    y = store.layer_norm(x, w, b)[0]
    assert torch.equal(store.layer_norm(x, w, b, stats=False), y)
    z = x.clone()
    assert store.layer_norm(z, w, b, out=z)[0] is z and torch.equal(z, y)
    only_w, only_b = store.layer_norm(x, w), store.layer_norm(x, None, b)
    check_forward(x, w, None, 1e-5, *only_w)
    check_forward(x, None, b, 1e-5, *only_b)


@pytest.mark.parametrize("length", [96, 128, 500, 1000, 3000, 9000, 18000])
def test_a_large_mean_and_an_outlier_keep_the_variance(store, length):
    # the variance is taken about the mean: values around 4096 that differ by a few sixteenths lose nothing but the mean's rounding
    g = torch.Generator().manual_seed(6)
    x = 4096 + torch.randint(-8, 9, (4, length), generator=g).double() / 16
    x[1] = torch.randn(length, generator=g, dtype=F64)
    x[1, 0] = 10000.0
    x[2] = 3.0                                              # all equal: rstd = 1 / sqrt(eps), y = bias
    x = x.float().cuda()
    w, b = params(length, F32, 7)
    y, mean, rstd = store.layer_norm(x, w, b)
    check_forward(x, w, b, 1e-5, y, mean, rstd)
    assert torch.equal(y[2], b)


def test_nan_and_infinity_stay_in_their_rows(store):
    for length in (100, 300, 2000, 17000):
        x = make(6, length, F32, 8)
        clean = store.layer_norm(x)[0]
        x[1, length // 2], x[4, 0] = float("nan"), float("inf")
        y = store.layer_norm(x)[0]
        assert y[1].isnan().all() and y[4].isnan().any()
        for i in (0, 2, 3, 5):
            assert torch.equal(y[i], clean[i])


# ------------------------------------------------------------------------------------------------
# backward
# ------------------------------------------------------------------------------------------------
def check_grad(x, dy, mean, rstd, w, got):
    dx, dw, db = got
    xd, dyd, m, r = x.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
    wd = torch.ones(x.shape[1], dtype=F64, device=x.device) if w is None else w.double()
    h = (xd - m) * r
    g = dyd * wd
    a, c = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    u = unit(x.dtype)
    eh = u * 3 * h.abs()                                    # of one value of h, from the rounding of its two operations
    if dx is not None:
        ref = r * (g - a - h * c)
        tol = r * u * STEPS * (g.abs() + g.abs().mean(1, keepdim=True) + h.abs() * (g * h).abs().mean(1, keepdim=True)) \
            + r * (h.abs() * (g.abs() * eh).mean(1, keepdim=True) + eh * c.abs()) + half_step(dx.dtype) * ref.abs() + tiny(dx.dtype)
        assert ((dx.double() - ref).abs() <= tol).all(), ((dx.double() - ref).abs() / tol).max()
    if dw is not None:
        ref = (dyd * h).sum(0)
        tol = u * COLUMN_STEPS * (dyd * h).abs().sum(0) + half_step(dw.dtype) * ref.abs() + tiny(dw.dtype)
        assert ((dw.double() - ref).abs() <= tol).all(), ((dw.double() - ref).abs() / tol).max()
        ref = dyd.sum(0)
        tol = u * COLUMN_STEPS * dyd.abs().sum(0) + half_step(db.dtype) * ref.abs() + tiny(db.dtype)
        assert ((db.double() - ref).abs() <= tol).all()


def stats_of(x, eps=1e-5):
    _, m, r, *_ = reference(x, None, None, eps)
    keep = F64 if x.dtype == F64 else F32
    return m.to(keep), r.to(keep)


@pytest.mark.parametrize("x_type,dy_type,w_type", [(F32, F32, F32), (F64, F64, F64), (F16, F16, F16), (BF16, BF16, F32), (F32, BF16, F32),
                                                   (F32, F16, None), (BF16, BF16, BF16)])
@pytest.mark.parametrize("n,length", SHAPES + [(5000, 64), (3000, 257)])
def test_backward_meets_the_formula(store, n, length, x_type, dy_type, w_type):
    x, dy = make(n, length, x_type, n + 2 * length), make(n, length, dy_type, 9, shift=0.1)
    w = params(length, w_type, 1)[0] if w_type else None
    mean, rstd = stats_of(x)
    check_grad(x, dy, mean, rstd, w, store.layer_norm_grad(x, dy, mean, rstd, w))


@pytest.mark.parametrize("n,length,gap", [(30, 96, 8), (50, 101, 2), (8, 1024, 4), (5, 3000, 1), (4, 9000, 8)])
def test_backward_of_rows_that_lie_apart(store, n, length, gap):
    for dtype in (F32, BF16):
        x, dy = make(n, length, dtype, 10, gap), make(n, length, dtype, 11, gap + 3)
        whole = torch.full((n, length + 5), 7.0, dtype=dtype, device="cuda")
        mean, rstd = stats_of(x)
        w = params(length, F32, 1)[0]
        got = store.layer_norm_grad(x, dy, mean, rstd, w, dx=whole[:, :length])
        check_grad(x, dy, mean, rstd, w, got)
        assert (whole[:, length:] == 7.0).all()


def test_backward_gives_only_what_is_asked_for_and_works_in_place(store):
    for length in (64, 100, 400, 2000, 9000):
        x, dy = make(70, length, F32, 12), make(70, length, F32, 13)
        w = params(length, F32, 1)[0]
        mean, rstd = stats_of(x)
        dx, dw, db = store.layer_norm_grad(x, dy, mean, rstd, w)
        only = store.layer_norm_grad(x, dy, mean, rstd, w, need_params=False)
        assert only[1] is None and only[2] is None and torch.equal(only[0], dx)
        only = store.layer_norm_grad(x, dy, mean, rstd, w, need_dx=False)
        assert only[0] is None and torch.equal(only[1], dw) and torch.equal(only[2], db)
        for target in (x.clone(), dy.clone()):
            over_x = store.layer_norm_grad(x if target is not x else target, dy, mean, rstd, w, dx=target)
            assert torch.equal(over_x[0], dx)
        x2, dy2 = x.clone(), dy.clone()
        assert torch.equal(store.layer_norm_grad(x2, dy, mean, rstd, w, dx=x2)[0], dx)
        got = store.layer_norm_grad(x, dy2, mean, rstd, w, dx=dy2)
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw) and torch.equal(got[2], db)
        for _ in range(3):                                  # the order of the additions is fixed
            again = store.layer_norm_grad(x, dy, mean, rstd, w)
            assert all(torch.equal(a, b) for a, b in zip(again, (dx, dw, db)))


def test_no_rows(store):
    x = torch.empty((0, 40), device="cuda")
    y, mean, rstd = store.layer_norm(x)
    assert y.shape == (0, 40) and mean.numel() == rstd.numel() == 0
    dx, dw, db = store.layer_norm_grad(x, x, mean, rstd, torch.ones(40, device="cuda"))
    assert dx.shape == (0, 40) and not dw.any() and not db.any() and dw.numel() == db.numel() == 40


@pytest.mark.parametrize("length", [3, 24, 100, 700])
def test_gradients_against_differences(store, length):
    # central differences of the forward pass in 64 bits with step t: off by t^2 times a third derivative (below 10 per unit of
    # rstd^3 here) and by the roundings of the loss, 2^-53 * |loss| * STEPS / t
    x, dy = make(5, length, F64, 14), make(5, length, F64, 15)
    w, b = (p.double() for p in params(length, F64, 16))
    y, mean, rstd = store.layer_norm(x, w, b, eps=1e-2)
    dx, dw, db = store.layer_norm_grad(x, dy, mean, rstd, w)
    t = 1e-4
    loss = lambda x_, w_, b_: float((store.layer_norm(x_, w_, b_, eps=1e-2, stats=False) * dy).sum())  # noqa: E731
    tol = 100 * t * t * float(rstd.max()) ** 3 * float(dy.abs().sum()) + 2.0 ** -53 * STEPS * float((y * dy).abs().sum()) / t
    rng = np.random.default_rng(0)
    for _ in range(6):
        i, j = int(rng.integers(5)), int(rng.integers(length))
        for what, grad in ((x, dx[i, j]), (w, dw[j]), (b, db[j])):
            at = (i, j) if what is x else (j,)
            up, down = what.clone(), what.clone()
            up[at] += t
            down[at] -= t
            args = [(up if v is what else v, down if v is what else v) for v in (x, w, b)]
            diff = (loss(*(a[0] for a in args)) - loss(*(a[1] for a in args))) / (2 * t)
            assert abs(diff - float(grad)) <= tol, (diff, float(grad), tol)


# ------------------------------------------------------------------------------------------------
# rows of the store
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("value_bytes,length,out", [(4, 64, F32), (4, 4, F32), (4, 100, BF16), (4, 128, F16), (4, 300, F32), (4, 1000, BF16),
                                                    (4, 20000, F32), (8, 100, F64), (8, 2, F64), (8, 1002, F64)])
@pytest.mark.parametrize("hot", [0, 30])
def test_pull_norm_is_the_norm_of_what_pull_gives(value_bytes, length, out, hot):
    nk, n = 500, 333
    rng = np.random.default_rng(17)
    s = binding.Store(nk, length, workers=4, value_bytes=value_bytes, count_accesses=True, deterministic=True)
    s.write_table(0, rng.normal(size=(nk, length)) + 0.2)
    if hot:                                                 # replicas with pending updates: each worker sees its own
        s.set_management(dev_keys(rng.permutation(nk)[:hot]), binding.REPLICATE)
        pk = rng.integers(0, nk, 200)
        s.push(dev_keys(pk), torch.from_numpy(rng.normal(size=(200, length))).to(s.dtype).cuda())
    keys = rng.integers(0, nk, n)
    keys[7] = nk + 5                                        # out of range: a row of zeros
    keys = dev_keys(keys)
    before = s.counts().clone()
    rows = s.pull(keys)
    assert s.status_check() == binding.EKEY
    once = s.counts().clone()
    w, b = params(length, s.dtype, 18)
    y, mean, rstd, pulled = s.pull_norm(keys, w, b, out_dtype=out, rows=True)
    assert s.status_check() == binding.EKEY and s.status_check() == 0
    assert torch.equal(pulled, rows)
    assert torch.equal(s.counts() - once, once - before)    # counted as a pull is
    check_forward(rows, w, b, 1e-5, y, mean, rstd)
    assert torch.equal(s.pull_norm(keys, w, b, out_dtype=out, stats=False), y)
    dy = make(n, length, out, 19)
    check_grad(rows, dy, mean, rstd, w, s.layer_norm_grad(pulled, dy, mean, rstd, w))
    st = s.stats()
    assert (st["hot"] > 0) == bool(hot)


# ------------------------------------------------------------------------------------------------
# streams, graphs, refusals
# ------------------------------------------------------------------------------------------------
def test_another_stream_and_two_captured_graphs(store):
    x, dy = make(500, 200, F32, 20), make(500, 200, F32, 21)
    w, b = params(200, F32, 22)
    want_y, mean, rstd = store.layer_norm(x, w, b)
    want = store.layer_norm_grad(x, dy, mean, rstd, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = store.layer_norm(x, w, b)[0]
        got = store.layer_norm_grad(x, dy, mean, rstd, w)
    side.synchronize()
    assert torch.equal(y, want_y) and all(torch.equal(p, q) for p, q in zip(got, want))
    graphs = []
    for k in range(2):
        xs, dys = x.clone(), dy.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ys, m, r = store.layer_norm(xs, w, b)
            res = store.layer_norm_grad(xs, dys, m, r, w)
        graphs.append((g, xs, dys, ys, res))
    for turn in range(3):
        for k, (g, xs, dys, ys, res) in enumerate(graphs):
            xs.copy_(x + k + turn)
            dys.copy_(dy * (1 + k))
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for (g, *_), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for k, (g, xs, dys, ys, res) in enumerate(graphs):
            yy, m, r = store.layer_norm(xs, w, b)
            assert torch.equal(ys, yy)
            assert all(torch.equal(p, q) for p, q in zip(res, store.layer_norm_grad(xs, dys, m, r, w)))


def refused(code, fn):
    with pytest.raises(binding.NupsError) as e:
        fn()
    assert e.value.code == code


def test_refusals(store):
    x, w = make(4, 64, F32, 23), torch.ones(64, device="cuda")
    mean, rstd = torch.zeros(4, device="cuda"), torch.ones(4, device="cuda")
    EINVAL = binding.EINVAL
    refused(EINVAL, lambda: store.layer_norm(x.int()))
    refused(EINVAL, lambda: store.layer_norm(x[0]))
    refused(EINVAL, lambda: store.layer_norm(x.t()))
    refused(EINVAL, lambda: store.layer_norm(x[:1].expand(4, 64)))
    refused(EINVAL, lambda: store.layer_norm(x, w[:63]))
    refused(EINVAL, lambda: store.layer_norm(x, w.double()))
    refused(EINVAL, lambda: store.layer_norm(x, w, w.half()))
    refused(EINVAL, lambda: store.layer_norm(x.half(), w, out_dtype=F32))
    refused(EINVAL, lambda: store.layer_norm(x, eps=0.0))
    refused(EINVAL, lambda: store.layer_norm(x, eps=float("nan")))
    refused(EINVAL, lambda: store.layer_norm(x.cpu()))
    refused(EINVAL, lambda: store.layer_norm(x[:, :0]))
    refused(EINVAL, lambda: store.layer_norm_grad(x, x[:3], mean, rstd))
    refused(EINVAL, lambda: store.layer_norm_grad(x, x, mean[:3], rstd))
    refused(EINVAL, lambda: store.layer_norm_grad(x, x, mean.double(), rstd))
    refused(EINVAL, lambda: store.layer_norm_grad(x.half(), x, mean, rstd))
    refused(EINVAL, lambda: store.layer_norm_grad(x, x, mean, rstd, dx=x.half()))
    keys = dev_keys(np.arange(4))
    refused(EINVAL, lambda: store.pull_norm(keys, w.half()))
    refused(EINVAL, lambda: store.pull_norm(keys, out_dtype=F64))
    # the C interface itself: too little scratch, no scratch, a stride that makes rows overlap
    L, st, p = store._l, torch.cuda.current_stream().cuda_stream, (lambda t: t.data_ptr())
    dx, dw = torch.full_like(x, 7.0), torch.full_like(w, 7.0)
    scratch = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    for address, size in ((p(scratch), 8), (None, 1 << 16), (p(scratch) + 4, 1 << 15)):
        assert L.nups_layer_norm_grad(store._s, p(x), 0, 64, p(x), 0, 64, 4, 64, p(mean), p(rstd), p(w), 0, p(dx), 64, p(dw), None, address, size, st) == EINVAL
    assert L.nups_layer_norm(store._s, p(x), 0, 63, 4, 64, None, None, 0, 1e-5, p(dx), 0, 64, None, None, st) == EINVAL
    assert L.nups_layer_norm(store._s, p(x), 4, 64, 4, 64, None, None, 0, 1e-5, p(dx), 0, 64, None, None, st) == EINVAL
    assert L.nups_layer_norm(None, p(x), 0, 64, 4, 64, None, None, 0, 1e-5, p(dx), 0, 64, None, None, st) == EINVAL
    torch.cuda.synchronize()
    assert (dx == 7.0).all() and (dw == 7.0).all()          # nothing was enqueued


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("length", [6, 30, 34, 62, 126, 202, 254, 510, 1002, 2046, 4094, 8190, 16382, 20002, 33002])
def test_rows_of_even_length_that_16_byte_loads_cannot_read(store, length, dtype):
    n = 2000 if length < 300 else 170
    x, dy = make(n, length, dtype, length, gap=2), make(n, length, dtype, length + 1, gap=4, shift=0.1)
    w, b = params(length, F32, 3)
    whole = torch.full((n, length + 6), 7.0, dtype=dtype, device="cuda")
    y, mean, rstd = store.layer_norm(x, w, b, eps=1e-5, out=whole[:, 2:length + 2])
    check_forward(x, w, b, 1e-5, y, mean, rstd)
    assert (whole[:, :2] == 7.0).all() and (whole[:, length + 2:] == 7.0).all()
    w1 = torch.cat([w[:1], w])[1:]                    # an address that a pair of weights cannot be read at
    y1, mean1, rstd1 = store.layer_norm(x, w1, b, eps=1e-5)
    assert torch.equal(y1, y) and torch.equal(mean1, mean) and torch.equal(rstd1, rstd)
    grads = store.layer_norm_grad(x, dy, mean, rstd, w, dx=whole[:, 2:length + 2])
    check_grad(x, dy, mean, rstd, w, grads)
    assert (whole[:, :2] == 7.0).all() and (whole[:, length + 2:] == 7.0).all()


@pytest.mark.parametrize("backward", [False, True])
def test_two_threads_with_a_store_each_and_rows_of_two_lengths(backward):
    # both lengths take one kernel, with rings of different sizes.  The C interface itself, so that the threads are in it most of the time
    failures, start = [], threading.Barrier(2)

    def work(length):
        with torch.cuda.stream(torch.cuda.Stream()):
            s = binding.Store(64, 64)
            x, out = make(300, length, BF16, length), torch.empty((300, length), dtype=BF16, device="cuda")
            mean, rstd = stats_of(x)
            L, st, kind = s._l, torch.cuda.current_stream().cuda_stream, binding.TYPES[BF16]
            px, po, pm, pr = (t.data_ptr() for t in (x, out, mean, rstd))
            if backward:
                fn, args = L.nups_layer_norm_grad, (s._s, px, kind, length, px, kind, length, 300, length, pm, pr, None, kind, po, length, None, None, None, 0, st)
            else:
                fn, args = L.nups_layer_norm, (s._s, px, kind, length, 300, length, None, None, kind, 1e-5, po, kind, length, None, None, st)
            start.wait(60)
            refused = sum(fn(*args) != 0 for _ in range(20_000))
            torch.cuda.current_stream().synchronize()
            want = s.layer_norm_grad(x, x, mean, rstd, need_params=False)[0] if backward else s.layer_norm(x, stats=False)
            if refused or not torch.equal(out, want):
                failures.append((length, refused))

    threads = [threading.Thread(target=work, args=(length,)) for length in (4096, 2304)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures


def by_its_statistics(x, w, b, y, mean, rstd):
    """y from the statistics that the call gave: x - mean, rstd, weight and bias are four operations, each off by half a unit of its own
    result, so y is off by 4 units of the difference's part and one of itself.  Rows of equal values whose mean is exact give the bias."""
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    h = h if w is None else h * w.double()
    b = torch.zeros_like(x[0]).double() if b is None else b.double()
    u = unit(x.dtype)
    tol = u * (4 * h.abs() + 2 * (h + b).abs()) + half_step(y.dtype) * (1 + u) * (h + b).abs() + tiny(y.dtype)
    off = (y.double() - (h + b)).abs()
    assert (off <= tol).all(), (off / tol).max()


LEVELS = {F32: (1001.0, -12345.0, 100.0, 0.1, 5000.25), F64: (1001.0, -12345.0, 1e9 + 1, 0.1, 5000.25), F16: (1001.0, -1234.0, 100.0, 0.1, 500.25), BF16: (200.0, -1248.0, 100.0, 0.1, 5.25)}


@pytest.mark.parametrize("dtype", [F32, F64, F16, BF16])
@pytest.mark.parametrize("n,length", [(5, 1), (7, 2), (40, 16), (40, 33), (9, 100), (20, 128), (6, 300), (11, 500), (6, 1000), (5, 2050), (4, 4096), (3, 8200), (2, 20000),
                                      (400, 640), (400, 1024), (320, 2048), (320, 4096), (170, 8192), (160, 16384)])
def test_rows_whose_mean_is_large_against_their_deviation(store, n, length, dtype):
    x = make(n, length, dtype, 31)
    for k, level in enumerate(LEVELS[dtype]):
        x[k::11] = level
        x[k + 5::11] += level
    w, b = params(length, dtype, 32)
    for weight, bias in ((w, b), (None, None)):
        y, mean, rstd = store.layer_norm(x, weight, bias)
        by_its_statistics(x, weight, bias, y, mean, rstd)
        if length <= 1024:                                  # sums of equal values of at most 14 bits are exact
            for k, level in enumerate(LEVELS[dtype][:3]):
                want = torch.zeros_like(y[k::11]) if bias is None else bias.expand_as(y[k::11])
                assert torch.equal(mean[k::11].double(), x[k::11, 0].double()) and torch.equal(y[k::11], want)


@pytest.mark.parametrize("value_bytes,length,out", [(4, 4, F32), (4, 128, BF16), (4, 1000, F32), (8, 100, F64), (4, 20000, F32)])
def test_pulled_rows_whose_mean_is_large_against_their_deviation(value_bytes, length, out):
    s = binding.Store(60, length, value_bytes=value_bytes)
    table = make(60, length, s.dtype, 33)
    table[::3] += 4000.0
    table[1::3] = 1001.0
    s.write_table(0, table.cpu().numpy())
    w, b = params(length, s.dtype, 34)
    y, mean, rstd, rows = s.pull_norm(dev_keys(range(60)), w, b, out_dtype=out, rows=True)
    assert torch.equal(rows, table)
    by_its_statistics(rows, w, b, y, mean, rstd)
    s.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_very_long_rows_of_equal_values(store, dtype):
    # a thread adds 16,384 or 32,768 values of such a row
    x = torch.full((2, 1 << 25), 0.1, dtype=dtype, device="cuda")
    x[1, ::2] = 0.3
    y, mean, rstd = store.layer_norm(x)
    check_forward(x, None, None, 1e-5, y, mean, rstd)
    dy = torch.full_like(x, 0.1)
    dy[1, ::2] = -0.2
    check_grad(x, dy, mean, rstd, None, store.layer_norm_grad(x, dy, mean, rstd, need_params=False))


def test_the_time_of_a_normalised_pull_is_a_pulls():
    s = binding.Store(1000, 64)
    keys = dev_keys(np.arange(500))
    s.kernel_timing(True)
    s.pull(keys)
    y = s.pull_norm(keys)[0]
    s.pull_norm(keys, rows=True)
    s.kernel_timing(False)
    s.pull_norm(keys)
    times = s.kernel_times()
    assert times["pull"][0] > 0 and [n for _, n in times.values()] == [3, 0, 0, 0, 0]
    s.kernel_timing(True)
    assert torch.equal(s.pull_norm(keys)[0], y)
    s.close()
