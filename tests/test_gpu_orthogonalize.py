"""Orthogonalized updates against the iteration in 64 bits.

Tolerance: a step's result is off by at most UNITS = 16 units of 2^-22, in the Frobenius norm and relative to |B| |X| (pairs hold 22
bits of X, A and B; a run of 64 values of K is cut at most twelve times by a unit of 2^-23 of itself, the runs' sum is rounded), with
|B| <= 3.4445 for the default coefficients.  A later step takes an error on with the polynomial's largest slope, its a = 3.4445, while
the result itself grows by |X'| / |X|: the ratios are taken from the reference's own iterates (amplification()).
"""
import numpy as np
import pytest
import torch

from paper_2104_00501_b200 import binding
from tests.common import dev_keys

pytestmark = pytest.mark.gpu
F32, F16, BF16, F64 = torch.float32, torch.float16, torch.bfloat16, torch.float64
DEFAULT = (3.4445, -4.7750, 2.0315)
UNITS = 16


@pytest.fixture(scope="module")
def store():
    s = binding.Store(64, 64)
    yield s
    s.close()


def make(batch, rows, cols, dtype, seed, low=0, gap=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((batch, rows, cols + gap), generator=g, dtype=F64)
    if low:
        x = x * 0.05
        x[..., :cols] += torch.randn((batch, rows, low), generator=g, dtype=F64) @ torch.randn((batch, low, cols), generator=g, dtype=F64)
    return (x * 0.01).to(dtype).cuda()[..., :cols]


def reference(g, steps=5, c=DEFAULT, eps=1e-7):
    """The iterate and the factor by which errors of single steps may show in it, per matrix."""
    c = [float(np.float32(v)) for v in c]
    x = g.double()
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.transpose(-1, -2)
    x = x / (x.square().sum((-1, -2), keepdim=True).sqrt() + eps)
    norms = [x.square().sum((-1, -2)).sqrt()]
    for _ in range(steps):
        a = x @ x.transpose(-1, -2)
        x = c[0] * x + (c[1] * a + c[2] * (a @ a)) @ x
        norms.append(x.square().sum((-1, -2)).sqrt())
    amp, f = torch.zeros_like(norms[0]), torch.ones_like(norms[0])
    for t in reversed(range(steps)):
        f = f * abs(c[0]) * norms[t] / norms[t + 1].clamp(min=1e-300)
        amp = amp + f
    return (x.transpose(-1, -2) if tall else x), amp


def check(store, g, out=None, **kw):
    scale = kw.pop("scale", 1.0)
    got = store.orthogonalize(g, scale=scale, out=out, **kw)
    ref, amp = reference(g, **{"steps": kw.get("steps", 5), "c": kw.get("coefficients", DEFAULT), "eps": kw.get("eps", 1e-7)})
    ref = ref * float(np.float32(scale))
    norm = ref.square().sum((-1, -2)).sqrt()
    tol = (UNITS * 2.0 ** -22 * (1 + amp) + torch.finfo(g.dtype).eps / 2) * norm + torch.finfo(g.dtype).tiny
    off = (got.double() - ref).square().sum((-1, -2)).sqrt()
    assert (off <= tol).all(), (off / tol).max()
    assert store.status_check() == 0
    return got


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (2, 1, 9), (3, 5, 1), (2, 3, 3), (4, 16, 16), (2, 17, 33), (5, 64, 64), (3, 65, 127), (2, 100, 100),
                                             (2, 128, 256), (2, 256, 128), (7, 30, 200), (1, 127, 255)])
def test_small_matrices(store, batch, rows, cols, dtype):
    check(store, make(batch, rows, cols, dtype, rows + cols))
    check(store, make(batch, rows, cols, dtype, rows + cols, low=2), steps=3, scale=-0.02)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("batch,rows,cols", [(1, 129, 129), (2, 64, 257), (1, 257, 64), (1, 1, 300), (3, 200, 300), (2, 300, 1000), (1, 1000, 300), (1, 511, 513),
                                             (2, 256, 256), (1, 768, 768), (1, 640, 2048), (17, 130, 140), (1, 33, 5000), (1, 1300, 1290)])
def test_tiled_matrices(store, batch, rows, cols, dtype):
    check(store, make(batch, rows, cols, dtype, rows + cols, low=8))
    check(store, make(batch, rows, cols, dtype, rows + cols + 1), steps=2, scale=3.0)


def test_many_tiles_and_rounds(store):
    check(store, make(1, 2600, 2700, F32, 1, low=100))      # more tiles than pairs of multiprocessors, 256 columns wide
    check(store, make(40, 520, 520, F32, 2, low=30), steps=2)


@pytest.mark.parametrize("rows,cols,gap", [(40, 50, 6), (50, 40, 3), (130, 200, 5), (300, 150, 8)])
def test_rows_and_matrices_that_lie_apart(store, rows, cols, gap):
    for dtype in (F32, BF16):
        g = make(3, rows, cols, dtype, 3, gap=gap)[::2]     # strides of rows and of matrices
        whole = torch.full((2, rows + 2, cols + 3), 7.0, dtype=dtype, device="cuda")
        check(store, g, out=whole[:, 1:rows + 1, 2:cols + 2])
        whole[:, 1:rows + 1, 2:cols + 2] = 7.0
        assert (whole == 7.0).all()
        one = g[0].clone()
        got = store.orthogonalize(one, out=one)             # in place, and without a batch
        assert got is one and torch.equal(one, store.orthogonalize(g[0]))


def test_zeros_nan_and_infinity_stay_in_their_matrices(store):
    for rows, cols in ((20, 30), (150, 170), (170, 150)):
        g = make(5, rows, cols, F32, 4)
        clean = store.orthogonalize(g)
        g[1] = 0
        g[2, rows // 2, 3] = float("nan")
        g[4, 0, 0] = float("inf")
        got = store.orthogonalize(g)
        assert not got[1].any() and got[2].isnan().all() and got[4].isnan().all()
        assert torch.equal(got[0], clean[0]) and torch.equal(got[3], clean[3])


def test_sizes_of_the_numbers_do_not_matter(store):
    # the norm is summed in 64 bits: powers of two far from 1 change nothing (eps is far below the smaller norm)
    for rows, cols in ((24, 40), (140, 260)):
        g = make(2, rows, cols, F32, 5)
        want = store.orthogonalize(g, eps=1e-37)
        for power in (100, 60, -60):
            assert torch.equal(store.orthogonalize(g * 2.0 ** power, eps=1e-37), want)


def test_singular_values_come_close_to_one(store):
    # the cubic iteration converges to the orthogonal factor: X X^T = I up to the pairs' rounding, and X G^T symmetric
    for rows, cols in ((50, 80), (200, 333), (333, 200)):
        g = make(1, rows, cols, F32, 6)[0]
        x = store.orthogonalize(g, steps=40, coefficients=(1.5, -0.5, 0.0)).double()
        small = x @ x.t() if rows < cols else x.t() @ x
        eye = torch.eye(min(rows, cols), device="cuda", dtype=F64)
        # a step is off by UNITS units relative to |B| |X|, |B| <= 1.5, and forgets earlier errors at s = 1 (slope 0); twice that in X X^T
        assert (small - eye).square().sum().sqrt() <= 2 * 1.5 * UNITS * 2.0 ** -22 * eye.square().sum().sqrt()


def test_results_do_not_change_from_call_to_call_or_with_the_batch(store):
    for rows, cols in ((60, 90), (300, 700)):
        g = make(6, rows, cols, F32, 7)
        a = store.orthogonalize(g)
        for _ in range(3):
            assert torch.equal(store.orthogonalize(g), a)
    assert store.orthogonalize(torch.empty((0, 200, 300), device="cuda")).shape == (0, 200, 300)


def test_streams_and_graphs(store):
    for rows, cols in ((80, 80), (260, 400), (600, 2100)):
        g = make(2, rows, cols, BF16, 8)
        want = store.orthogonalize(g)
        side = [torch.cuda.Stream(), torch.cuda.Stream()]
        outs = []
        for st in side:
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                outs += [store.orthogonalize(g) for _ in range(3)]
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs)
        graphs = []
        for k in range(2):
            x = g.clone()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                y = store.orthogonalize(x)
            graphs.append((graph, x, y))
        for k, (graph, x, y) in enumerate(graphs):
            x.copy_(g * (1 + k))
        torch.cuda.synchronize()
        for _ in range(2):
            for (graph, *_), st in zip(graphs, side):
                with torch.cuda.stream(st):
                    graph.replay()
        torch.cuda.synchronize()
        for graph, x, y in graphs:
            assert torch.equal(y, store.orthogonalize(x))


def refused(code, fn):
    with pytest.raises(binding.NupsError) as e:
        fn()
    assert e.value.code == code


def test_refusals(store):
    E = binding.EINVAL
    g = make(2, 20, 30, F32, 9)
    refused(E, lambda: store.orthogonalize(g.double()))
    refused(E, lambda: store.orthogonalize(g[0, 0]))
    refused(E, lambda: store.orthogonalize(g.transpose(1, 2)))
    refused(E, lambda: store.orthogonalize(g.cpu()))
    refused(E, lambda: store.orthogonalize(g, steps=0))
    refused(E, lambda: store.orthogonalize(g, steps=65))
    refused(E, lambda: store.orthogonalize(g, eps=0.0))
    refused(E, lambda: store.orthogonalize(g, scale=float("inf")))
    refused(E, lambda: store.orthogonalize(g, coefficients=(float("nan"), 0, 0)))
    refused(E, lambda: store.orthogonalize(g, coefficients=(8.0, 0.0, 0.0)))        # a factor above 7.5
    refused(E, lambda: store.orthogonalize(g, coefficients=(1.5, 1.0, 0.0)))        # singular values run away
    refused(E, lambda: store.orthogonalize(g, coefficients=(1.0, 2.0)))
    refused(E, lambda: store.orthogonalize(g, out=g[:1]))
    refused(E, lambda: store.orthogonalize(g, out=g.half()))
    refused(E, lambda: store.orthogonalize(g[:, :0]))
    refused(E, lambda: store.orthogonalize(g[:, :1].expand(2, 20, 30)))
    refused(E, lambda: store.orthogonalize(g[:1].expand(2, 20, 30)))
    L, p = store._l, (lambda t: t.data_ptr())
    import ctypes
    c = (ctypes.c_float * 3)(*DEFAULT)
    big, out = make(1, 200, 300, F32, 10), torch.full((200, 300), 7.0, device="cuda")
    scratch = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    for address, size in ((None, 1 << 22), (p(scratch), 1000), (p(scratch) + 8, 1 << 21)):
        assert L.nups_orthogonalize(store._s, p(big), 0, 300, 0, 1, 200, 300, 5, c, 1e-7, 1.0, p(out), 300, 0, address, size, None) == E
    assert L.nups_orthogonalize(store._s, p(big), 0, 299, 0, 1, 200, 300, 5, c, 1e-7, 1.0, p(out), 300, 0, p(scratch), 1 << 22, None) == E
    assert L.nups_orthogonalize(store._s, p(big), 0, 300, 0, 1, 200, 300, 5, None, 1e-7, 1.0, p(out), 300, 0, p(scratch), 1 << 22, None) == E
    torch.cuda.synchronize()
    assert (out == 7.0).all()


def test_a_step_of_rows_that_hold_matrices():
    # relation matrices of 12 x 16 values in a store's rows: their orthogonalized updates are what push adds
    keys, r, c, rate = 20, 12, 16, 0.1
    s = binding.Store(keys, r * c, workers=2, deterministic=True)
    start = np.random.default_rng(0).normal(size=(keys, r * c)).astype(np.float32)
    s.write_table(0, start)
    at = dev_keys(np.array([3, 17, 8]))
    g = make(3, r, c, F32, 11)
    s.push(at, s.orthogonalize(g, scale=-rate).view(3, r * c))
    ref, _ = reference(g)
    want = torch.from_numpy(start).cuda().double()
    want[at.long()] -= rate * ref.reshape(3, r * c)
    s.sync()
    assert (s.read_table().double() - want).abs().max() <= 1e-4 * rate + 2.0 ** -24 * want.abs().max()


@pytest.mark.parametrize("rows,cols", [(20, 30), (30, 20), (150, 170), (170, 150)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_zeros_and_tiny_matrices_with_a_tiny_eps(store, rows, cols, dtype):
    zeros = torch.zeros((2, rows, cols), dtype=dtype, device="cuda")
    for eps in (1e-30, 1e-35, 1e-38, 1e-44):
        assert not store.orthogonalize(zeros, eps=eps).any()
    for power in (-110, -123, -132):                        # norms of 2^-109 to 2^-131 or so, many of the values below the normal range
        g = (make(2, rows, cols, F64, 61) * 2.0 ** power).to(dtype)
        for eps in (1e-42, 1e-37):
            check(store, g, eps=float(np.float32(eps)))


def test_coefficients_that_send_a_few_singular_values_out_of_range(store):
    # a singular value of 0.9968385 leaves every bound in eight steps; values a thousandth to either side do not
    c, s = (2.77, -5.98, 2.19), 0.9968385
    refused(binding.EINVAL, lambda: store.orthogonalize(torch.diag(torch.tensor([s, (1 - s * s) ** 0.5], device="cuda")), steps=8, coefficients=c))
    # 2.5 and 7.5 themselves, and what lies just beyond
    g = make(1, 10, 20, F32, 62)
    for good, bad in (((2.5, 0.0, 0.0), (2.5001, 0.0, 0.0)), ((7.5, -11.0, 3.0), (7.501, -11.0, 3.0)), ((0.0, 2.5, 0.0), (0.0, -2.501, 0.0))):
        store.orthogonalize(g, steps=1, coefficients=good)
        refused(binding.EINVAL, lambda: store.orthogonalize(g, steps=1, coefficients=bad))
    for steps in (1, 5, 64):
        store.orthogonalize(g, steps=steps)
        store.orthogonalize(g, steps=steps, coefficients=(1.5, -0.5, 0.0))
        store.orthogonalize(g, steps=steps, coefficients=(2.0, -1.5, 0.5))


@pytest.mark.parametrize("rows,cols", [(20, 30), (150, 170), (170, 150)])
def test_tiny_and_huge_scales(store, rows, cols):
    # the iterate is brought to its size by a power of two, then multiplied: one rounding
    g = make(2, rows, cols, F32, 63)
    want = store.orthogonalize(g)
    for scale in (-0.02, 1e-25, -3e-31, 7e-36, 1e30, -3e38):
        assert torch.equal(store.orthogonalize(g, scale=scale), want * torch.tensor(scale, device="cuda"))
