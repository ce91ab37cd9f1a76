"""Layer norm's rings in shared memory (rows of 1 KB and more, more rows than multiprocessors): rows that lie apart, mixed types, in place,
NaN, forward and backward.  Tolerances as in test_gpu_norm.py.
"""
import pytest
import torch

from tests.test_gpu_norm import BF16, F16, F32, F64, check_forward, check_grad, make, params, stats_of, store  # noqa: F401

pytestmark = pytest.mark.gpu

# Several groups of up to four rows per block, the last one not full: up to 148 multiprocessors hold 1 to 9 blocks each.  One length
# with a single group per block as well.
RING = [(12_001, 1024), (401, 1536), (8_003, 1536), (6_005, 2048), (4_003, 4096), (2_001, 8192), (1_003, 16384)]


@pytest.mark.parametrize("x_type,y_type,w_type", [(F32, BF16, F32), (F32, F32, F32), (F32, F16, None), (BF16, BF16, F32), (F16, F16, F16), (F64, F64, F64)])
@pytest.mark.parametrize("n,length", RING)
def test_rings_forward_of_rows_that_lie_apart_of_mixed_types_and_in_place(store, n, length, x_type, y_type, w_type):
    # gaps of whole 16 bytes, so that rows come one copy each
    gap = 32
    w, b = params(length, w_type, 41) if w_type else (None, None)
    x = make(n, length, x_type, 42, gap)
    x[5::7] = x[5::7] + 1000.0
    bad = x[3, 1].clone()
    whole = torch.full((n + 2, length + gap), 7.0, dtype=y_type, device="cuda")
    y, mean, rstd = store.layer_norm(x, w, b, out=whole[1:n + 1, 16:length + 16])
    check_forward(x, w, b, 1e-5, y, mean, rstd)
    dense = store.layer_norm(x.contiguous(), w, b, out_dtype=y_type)
    assert all(torch.equal(p, q) for p, q in zip((y, mean, rstd), dense))
    if x_type == y_type:                                    # in place: the output is written while later groups come in
        for z in (x.clone(), x.contiguous(), make(n, length, x_type, 42, gap)):
            z.copy_(x)
            store.layer_norm(z, w, b, out=z)
            assert torch.equal(z, y)
    x[3, 1], x[n - 1, length - 1] = float("nan"), float("inf")
    spoilt = store.layer_norm(x, w, b, out_dtype=y_type)[0]
    assert spoilt[3].isnan().all() and spoilt[n - 1].isnan().any()
    others = [i for i in range(n) if i not in (3, n - 1)]
    assert torch.equal(spoilt[others], dense[0][others])
    x[3, 1] = bad
    whole[1:n + 1, 16:length + 16] = 7.0
    assert (whole == 7.0).all() and store.status_check() == 0


@pytest.mark.parametrize("x_type,dy_type,w_type", [(F32, F32, F32), (F32, BF16, F32), (F32, F16, None), (BF16, BF16, F32), (F16, F16, F16), (F64, F64, F64)])
@pytest.mark.parametrize("n,length", RING)
def test_rings_backward_of_rows_that_lie_apart_of_mixed_types_and_in_place(store, n, length, x_type, dy_type, w_type):
    x, dy = make(n, length, x_type, 43, 16), make(n, length, dy_type, 44, 48, shift=0.1)
    w = params(length, w_type, 45)[0] if w_type else None
    mean, rstd = stats_of(x)
    whole = torch.full((n + 2, length + 32), 7.0, dtype=x_type, device="cuda")
    got = store.layer_norm_grad(x, dy, mean, rstd, w, dx=whole[1:n + 1, 16:length + 16])
    check_grad(x, dy, mean, rstd, w, got)
    for xs, dys in ((x.contiguous(), dy.contiguous()), (x, dy.contiguous()), (x.contiguous(), dy)):
        assert all(torch.equal(p, q) for p, q in zip(store.layer_norm_grad(xs, dys, mean, rstd, w), got))
    own = x.clone()
    over = store.layer_norm_grad(own, dy, mean, rstd, w, dx=own)
    assert all(torch.equal(p, q) for p, q in zip(over, got))
    if x_type == dy_type:
        own = dy.clone()
        over = store.layer_norm_grad(x, own, mean, rstd, w, dx=own)
        assert all(torch.equal(p, q) for p, q in zip(over, got))
    spoilt = dy.clone()
    spoilt[n // 2, 3] = float("nan")
    dx = store.layer_norm_grad(x, spoilt, mean, rstd, w, need_params=False)[0]
    others = [i for i in range(n) if i != n // 2]
    assert dx[n // 2].isnan().all() and torch.equal(dx[others], got[0][others])
    only = store.layer_norm_grad(x, dy, mean, rstd, w, need_dx=False)
    assert torch.equal(only[1], got[1]) and torch.equal(only[2], got[2])
    whole[1:n + 1, 16:length + 16] = 7.0
    assert (whole == 7.0).all() and store.status_check() == 0


def test_rings_of_two_sizes_in_one_graph(store):
    # both lengths of a pair take one kernel; the graph is put together when the second has been captured
    for lengths in ((4096, 2304), (1600, 1100)):
        parts = [(make(400, length, BF16, length), make(400, length, BF16, length + 1)) for length in lengths]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = []
            for x, dy in parts:
                y, mean, rstd = store.layer_norm(x)
                got += [y, *store.layer_norm_grad(x, dy, mean, rstd)]
        for x, dy in parts:
            x.copy_(x.roll(1, 0))
        for _ in range(2):
            g.replay()
        torch.cuda.synchronize()
        want = []
        for x, dy in parts:
            y, mean, rstd = store.layer_norm(x)
            want += [y, *store.layer_norm_grad(x, dy, mean, rstd)]
        assert all(torch.equal(p, q) for p, q in zip(got, want))
