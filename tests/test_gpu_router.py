"""The router over experts against its formulas in 64 bits.

Tolerances: the device's fast exponential is off by at most 2 + 1.173 |a| units of 2^-23 at an argument a (CUDA's table of
intrinsic functions), so with the largest logit subtracted a term is off by R = 2^-23 (2 + 1.2 spread), spread = the largest
gap between two finite logits of an item.  A probability divides two such numbers; sums of at most 1024 terms in lanes of 32
and a tree add 42 units of 2^-24; sums over items at most 150 (64 items per team here, 40 runs of blocks, trees).
"""
import numpy as np
import pytest
import torch

from paper_2104_00501_b200 import binding

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
U = 2.0 ** -24


@pytest.fixture(scope="module")
def store():
    s = binding.Store(64, 64)
    yield s
    s.close()


def make(n, experts, dtype, seed, gap=0, ties=False):
    g = torch.Generator().manual_seed(seed)
    x = 2 * torch.randn((n, experts + gap), generator=g) + torch.randn(experts + gap, generator=g)
    if ties:
        x = (x * 2).round() / 2
        x[x == 0] = -0.0                                    # zeros of both signs are equal
        x[::3][x[::3] == 0] = 0.0
    return x.to(dtype).cuda()[:, :experts]


def reference(x, top, active, renormalize, balance, z):
    """Everything in 64 bits on the host, item by item where order matters."""
    x = x.double().cpu().numpy()
    n, E = x.shape
    on = np.ones(n, bool) if active is None else active.cpu().numpy().astype(bool)
    on = on & ~np.all(x == -np.inf, axis=1)
    choice = np.full((n, top), -1, np.int64)
    for i in np.nonzero(on)[0]:
        usable = [e for e in range(E) if x[i, e] > -np.inf]
        for j, e in enumerate(sorted(usable, key=lambda e: (-x[i, e], e))[:top]):
            choice[i, j] = e
    safe = np.where(on[:, None], x, 0.0)
    with np.errstate(invalid="ignore"):
        most = safe.max(1, keepdims=True)
        ex = np.exp(safe - most)
        p = ex / ex.sum(1, keepdims=True) * on[:, None]
        lse = np.where(on, (most + np.log(ex.sum(1, keepdims=True)))[:, 0], 0.0)
    counts = np.zeros(E, np.int64)
    np.add.at(counts, choice[choice >= 0], 1)
    T = max(1, on.sum())
    p_c = np.where(choice >= 0, np.take_along_axis(p, np.maximum(choice, 0), 1), 0.0)
    weight = p_c / np.maximum(p_c.sum(1, keepdims=True), 1e-300) if renormalize else p_c
    P = p.sum(0) / T
    B = E / (top * T) * (counts * P).sum()
    Z = (lse ** 2).sum() / T
    return dict(on=on, choice=choice, p=p, lse=lse, counts=counts, T=T, tokens=int(on.sum()), weight=weight, prob=P, B=B, Z=Z, loss=balance * B + z * Z, p_c=p_c)


def spread_of(x):
    v = x.double().cpu().numpy()
    v = np.where(np.isfinite(v), v, np.nan)
    return 0.0 if np.isnan(v).all() else float(np.nanmax(np.nanmax(v, 1) - np.nanmin(v, 1)))


def grad_reference(x, r, top, renormalize, balance, z, dweight, dloss):
    n, E = r["p"].shape
    f = r["counts"] * E / (top * r["T"])
    g = np.broadcast_to(dloss * balance * f / r["T"], (n, E)).copy()
    extra = np.zeros((n, E))
    size = np.zeros((n, E))
    if dweight is not None:
        dw = np.where(r["choice"] >= 0, dweight, 0.0)
        if renormalize:
            mean = (dw * r["weight"]).sum(1, keepdims=True)
            add, mag = r["weight"] * (dw - mean), r["weight"] * (np.abs(dw) + (np.abs(dw) * r["weight"]).sum(1, keepdims=True))
        else:
            add = r["p_c"] * dw
            mag = np.abs(add)
        for i in range(n):
            for j in range(top):
                if r["choice"][i, j] >= 0:
                    extra[i, r["choice"][i, j]] += add[i, j]
                    size[i, r["choice"][i, j]] += mag[i, j]
    lz = dloss * z * 2 * r["lse"][:, None] / r["T"]
    s = (g * r["p"]).sum(1, keepdims=True)
    sa = (np.abs(g) * r["p"]).sum(1, keepdims=True)
    if dweight is not None and not renormalize:
        s = s + extra.sum(1, keepdims=True)
        sa = sa + np.abs(extra).sum(1, keepdims=True)
    d = (r["p"] * (g - s + lz) + extra) * r["on"][:, None]
    return d, r["p"] * (np.abs(g) + sa + np.abs(lz)) + size


def check(store, x, top, active=None, renormalize=False, balance=0.02, z=0.003, out=None, seed=0):
    r = reference(x, top, active, renormalize, balance, z)
    got = store.route(x, top, active=active, renormalize=renormalize, balance=balance, z=z)
    R = 2.0 ** -23 * (2 + 1.2 * spread_of(x)) * 2 + 42 * U
    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    assert np.array_equal(got.choice.cpu().numpy(), r["choice"])
    assert np.array_equal(got.counts.cpu().numpy(), r["counts"]) and got.tokens.item() == r["tokens"]
    tiny = 2.0 ** -125                                      # smaller terms may be flushed to zero
    assert (np.abs(host(got.weight) - r["weight"]) <= 2 * R * r["weight"] + tiny).all()
    assert (np.abs(host(got.lse) - r["lse"]) <= R + 4 * U * np.abs(r["lse"])).all()
    column = R + 150 * U
    assert (np.abs(host(got.prob) - r["prob"]) <= column * r["prob"] + tiny).all()
    B, Z = float(got.loss[1]), float(got.loss[2])
    z_size = float((np.abs(r["lse"]) * (R + 4 * U * np.abs(r["lse"])) * 2).sum() / r["T"]) + 150 * U * r["Z"]
    assert abs(B - r["B"]) <= (column + 50 * U) * r["B"] + tiny
    assert abs(Z - r["Z"]) <= z_size + tiny
    assert abs(float(got.loss[0]) - r["loss"]) <= abs(balance) * (column + 50 * U) * r["B"] + abs(z) * z_size + 4 * U * abs(r["loss"]) + tiny
    g = torch.Generator().manual_seed(seed + 99)
    for dweight, dloss in ((None, None), (torch.randn((x.shape[0], top), generator=g).cuda(), None), (torch.randn((x.shape[0], top), generator=g).cuda() * 1e-3, 0.7)):
        d = store.route_grad(x, got, dweight=dweight, dloss=None if dloss is None else torch.tensor(dloss, device="cuda"), out=out)
        ref, size = grad_reference(x, r, top, renormalize, balance, z, None if dweight is None else host(dweight), 1.0 if dloss is None else float(np.float32(dloss)))
        tol = (4 * R + 60 * U) * size + torch.finfo(x.dtype).eps / 2 * np.abs(ref) + torch.finfo(x.dtype).tiny * torch.finfo(x.dtype).eps
        assert (np.abs(host(d) - ref) <= tol).all(), (np.abs(host(d) - ref) / tol).max()
        assert (host(d)[~r["on"]] == 0).all()
    assert store.status_check() == 0
    return got


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,experts,top", [(1, 1, 1), (3, 2, 2), (24, 64, 2), (70, 5, 5), (33, 12, 1), (500, 16, 16), (40, 17, 3), (9, 100, 8), (300, 128, 32),
                                           (50, 129, 6), (1, 256, 8), (700, 256, 8), (65, 255, 32), (30, 512, 10), (20, 777, 4), (1, 1024, 32), (2500, 8, 2),
                                           (90, 1024, 1)])
def test_routes_meet_the_formula(store, n, experts, top, dtype):
    check(store, make(n, experts, dtype, n + experts), top)
    check(store, make(n, experts, dtype, n + experts + 1, ties=True), top, renormalize=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,experts,top,gap", [(50, 64, 4, 8), (41, 60, 3, 5), (33, 256, 8, 1), (33, 256, 8, 16), (10, 1000, 2, 24)])
def test_items_that_take_no_part_and_rows_that_lie_apart(store, n, experts, top, gap, dtype):
    g = torch.Generator().manual_seed(5)
    active = (torch.rand(n, generator=g) < 0.6).cuda()
    x = make(n, experts, dtype, 6, gap)
    x[~active] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1e30], device="cuda").to(dtype)[torch.arange(int((~active).sum()), device="cuda") % 4][:, None]
    whole = torch.full((n, experts + 7), 3.0, dtype=dtype, device="cuda")
    for renormalize in (False, True):
        check(store, x, top, active=active, renormalize=renormalize, out=whole[:, :experts])
    assert (whole[:, experts:] == 3.0).all()
    got = store.route(x, top, active=active.to(torch.uint8))
    assert (got.choice[~active] == -1).all() and (got.weight[~active] == 0).all()


def test_forbidden_experts_and_items_without_any(store):
    for experts, top in ((12, 3), (64, 4), (200, 8)):
        for dtype in (F32, F16, BF16):
            x = make(60, experts, dtype, 7)
            g = torch.Generator().manual_seed(8)
            x[(torch.rand((60, experts), generator=g) < 0.7).cuda()] = -float("inf")
            x[5] = -float("inf")                            # nothing is left: the item takes no part
            x[6] = -float("inf")
            x[6, experts - 1] = -3.0                        # one expert is left
            check(store, x, top)
            got = check(store, x, top, renormalize=True)
            assert got.tokens.item() <= 59 and got.choice[6].tolist() == [experts - 1] + [-1] * (top - 1) and got.weight[6, 0].item() == 1.0


def test_lowest_finite_logits_are_chosen(store):
    # a mask made of the type's lowest value is a logit like any other: such experts come last, and have no weight
    for dtype in (F32, F16, BF16):
        x = torch.full((9, 20), torch.finfo(dtype).min, dtype=dtype, device="cuda")
        x[1, 3] = 0.0
        got = store.route(x, 4, renormalize=True)
        assert got.choice[0].tolist() == [0, 1, 2, 3] and got.weight[0].tolist() == [0.25] * 4
        assert got.choice[1].tolist() == [3, 0, 1, 2] and got.weight[1].tolist() == [1.0, 0, 0, 0]


def test_nan_and_infinity_show(store):
    x = make(40, 30, F32, 9)
    clean = store.route(x, 3, balance=1.0)
    y = x.clone()
    y[7, 4] = float("nan")
    got = store.route(y, 3, balance=1.0)
    assert 4 not in got.choice[7].tolist() and got.weight[7].isnan().all() and got.loss.isnan().all() and got.prob.isnan().all()
    others = [i for i in range(40) if i != 7]
    assert torch.equal(got.choice[others], clean.choice[others]) and torch.equal(got.weight[others], clean.weight[others])
    y[7, 4] = float("inf")
    got = store.route(y, 3, balance=1.0)
    assert got.choice[7, 0].item() == 4 and got.loss.isnan().all()
    assert torch.equal(got.choice[others], clean.choice[others])


def test_no_items_and_none_that_takes_part(store):
    got = store.route(torch.empty((0, 20), device="cuda"), 2, balance=1.0)
    assert not got.counts.any() and got.tokens.item() == 0 and not got.prob.any() and not got.loss.any()
    assert store.route_grad(torch.empty((0, 20), device="cuda"), got).shape == (0, 20)
    for n in (3, 3000):
        x = make(n, 20, BF16, 10)
        got = store.route(x, 2, active=torch.zeros(n, dtype=torch.bool, device="cuda"), balance=1.0, z=1.0)
        assert not got.counts.any() and got.tokens.item() == 0 and not got.prob.any() and not got.loss.any() and (got.choice == -1).all()
        assert not store.route_grad(x, got, dweight=torch.ones((n, 2), device="cuda")).any()


def test_a_program_that_only_answers(store):
    x = make(100, 60, BF16, 11)
    full, short = store.route(x, 4, renormalize=True, losses=True), store.route(x, 4, renormalize=True)
    assert short.prob is None and short.loss is None and short.lse is None
    for a, b in ((full.choice, short.choice), (full.weight, short.weight), (full.counts, short.counts), (full.tokens, short.tokens)):
        assert torch.equal(a, b)


def test_results_do_not_change_from_call_to_call(store):
    x = make(9000, 256, BF16, 12)
    dw = torch.randn((9000, 8), device="cuda")
    a = store.route(x, 8, balance=1.0, z=1.0)
    da = store.route_grad(x, a, dweight=dw)
    for _ in range(3):
        b = store.route(x, 8, balance=1.0, z=1.0)
        assert all(torch.equal(p, q) for p, q in zip(a[:7], b[:7]))
        assert torch.equal(da, store.route_grad(x, b, dweight=dw))
    y = x.clone()
    assert torch.equal(store.route_grad(y, a, dweight=dw, out=y), da)     # in place


@pytest.mark.parametrize("renormalize", [False, True])
def test_gradients_against_differences(store, renormalize):
    # central differences of loss + sum weight * dweight in float logits, choices kept.  The two sides' roundings bound the
    # quotient's error: each side is off by at most tol_f (the bounds of check()), and t^2 times the third derivative (below 1 here)
    n, E, k, t = 12, 10, 3, 2.0 ** -5
    x = make(n, E, F32, 13)
    dw = torch.randn((n, k), device="cuda") * 0.1
    got = store.route(x, k, renormalize=renormalize, balance=0.5, z=0.1)
    d = store.route_grad(x, got, dweight=dw).double().cpu()

    def value(y):
        r = store.route(y, k, renormalize=renormalize, balance=0.5, z=0.1)
        if not torch.equal(r.choice, got.choice):
            return None
        return float(r.loss[0].double() + (r.weight.double() * dw.double()).sum())

    R = 2.0 ** -23 * (2 + 1.2 * (spread_of(x) + 1)) * 2 + 42 * U
    tol = t * t + 2 * (R + 200 * U) * (float(got.loss[0].abs()) + float(dw.abs().sum())) / t
    seen = 0
    for i in range(n):
        for e in range(0, E, 3):
            up, down = x.clone(), x.clone()
            up[i, e] += t
            down[i, e] -= t
            a, b = value(up), value(down)
            if a is not None and b is not None:
                h = float(up[i, e].double() - down[i, e].double())
                assert abs((a - b) / h - float(d[i, e])) <= tol, ((a - b) / h, float(d[i, e]), tol)
                seen += 1
    assert seen >= 20


def test_graphs_and_streams(store):
    x = make(3000, 64, BF16, 14)
    want = store.route(x, 4, balance=1.0)
    graphs = []
    for k in range(2):
        xs = x.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = store.route(xs, 4, balance=1.0)
            d = store.route_grad(xs, r)
        graphs.append((g, xs, r, d))
    for k, (g, xs, r, d) in enumerate(graphs):
        xs.copy_(x.roll(k, 0))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for (g, *_), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for k, (g, xs, r, d) in enumerate(graphs):
        again = store.route(xs, 4, balance=1.0)
        assert all(torch.equal(p, q) for p, q in zip(r[:7], again[:7])) and torch.equal(d, store.route_grad(xs, again))
    assert torch.equal(graphs[0][2].choice, want.choice)


def refused(code, fn):
    with pytest.raises(binding.NupsError) as e:
        fn()
    assert e.value.code == code


def test_refusals(store):
    E = binding.EINVAL
    x = make(8, 40, F32, 15)
    refused(E, lambda: store.route(x.double(), 2))
    refused(E, lambda: store.route(x, 0))
    refused(E, lambda: store.route(x, 41))
    refused(E, lambda: store.route(make(2, 64, F32, 1), 33))
    refused(E, lambda: store.route(make(2, 1025, F32, 1), 2))
    refused(E, lambda: store.route(x[:, :0], 1))
    refused(E, lambda: store.route(x.t(), 2))
    refused(E, lambda: store.route(x, 2, active=torch.ones(7, dtype=torch.bool, device="cuda")))
    refused(E, lambda: store.route(x, 2, active=torch.ones(8, device="cuda")))
    refused(E, lambda: store.route(x, 2, balance=float("nan")))
    refused(E, lambda: store.route(x.cpu(), 2))
    r = store.route(x, 2, losses=True)
    refused(E, lambda: store.route_grad(x, store.route(x, 2)))
    refused(E, lambda: store.route_grad(x[:7], r))
    refused(E, lambda: store.route_grad(x[:, :39], r))
    refused(E, lambda: store.route_grad(x, r, dweight=torch.ones((8, 3), device="cuda")))
    refused(E, lambda: store.route_grad(x, r, dweight=torch.ones((8, 2), device="cuda", dtype=F16)))
    refused(E, lambda: store.route_grad(x, r, dloss=torch.ones(2, device="cuda")))
    refused(E, lambda: store.route_grad(x, r, out=x.half()))
    L, p = store._l, (lambda t: t.data_ptr())
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    x = make(80, 40, F32, 15)                               # more than one block's items
    r = store.route(x, 2)
    kept = [torch.full_like(t, 7) for t in (r.choice, r.weight, r.counts, r.tokens)]
    for address, size in ((p(small), 8), (None, 1 << 20), (p(small) + 4, 1 << 20)):
        assert L.nups_route(store._s, p(x), 0, 40, 80, 40, 2, None, 0, 0.0, 0.0, p(kept[0]), p(kept[1]), None, p(kept[2]), p(kept[3]), None, None, address, size, None) == E
    assert L.nups_route(store._s, p(x), 0, 39, 80, 40, 2, None, 0, 0.0, 0.0, p(kept[0]), p(kept[1]), None, p(kept[2]), p(kept[3]), None, None, p(small), 1 << 20, None) == E
    torch.cuda.synchronize()
    assert all((t == 7).all() for t in kept)


def test_choices_are_keys_of_a_store():
    # experts are the first keys of a store: the choices are counted, pulled and used for the choice of replicated keys as any keys
    E, L = 16, 8
    s = binding.Store(E, L, workers=2)
    s.write_table(0, np.arange(E * L, dtype=np.float32).reshape(E, L))
    x = make(200, E, F32, 16)
    r = s.route(x, 2, balance=1.0)
    s.count_accesses(r.choice.view(-1))
    assert torch.equal(s.counts(), r.counts)
    hot = s.select_hot(True, 3)
    order = sorted(range(E), key=lambda e: (-r.counts[e].item(), e))[:3]
    assert hot.tolist() == order
    assert torch.equal(s.pull(r.choice.view(-1))[:, 0].long(), r.choice.view(-1).long() * L)


def test_routings_whose_tensors_were_replaced(store):
    E = binding.EINVAL
    x = make(8, 40, F32, 15)
    r = store.route(x, 2, balance=0.01)
    g = store.route_grad(x, r)
    assert torch.equal(store.route_grad(x, r._replace(counts=r.counts.clone(), tokens=r.tokens.reshape(1))), g)
    for other in (dict(counts=r.counts[:1].expand(40)), dict(counts=r.counts.repeat(2)[::2]), dict(counts=r.counts.int()), dict(counts=r.counts.cpu()),
                  dict(tokens=r.tokens.cpu()), dict(tokens=r.counts), dict(choice=r.choice.long()), dict(choice=r.choice[:, :1].expand(8, 2)),
                  dict(choice=r.choice[:, :1]), dict(weight=r.weight[:, :1].expand(8, 2)), dict(weight=r.weight.half()), dict(weight=r.weight.cpu()),
                  dict(lse=r.lse[:1].expand(8)), dict(lse=r.lse.double()), dict(lse=r.lse.cpu())):
        refused(E, lambda: store.route_grad(x, r._replace(**other)))


@pytest.mark.parametrize("shift", [100.0, -6016.0, 60000.0])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n,experts,top", [(40, 12, 2), (33, 64, 4), (50, 100, 8), (60, 256, 8), (21, 333, 3), (12, 1000, 6)])
def test_logits_far_from_zero(store, n, experts, top, dtype, shift):
    # softmax, choices and gradients depend on the logits' differences alone: the bounds hold no part of the logits' own size
    if dtype == F32:
        x = (make(n, experts, F32, 51) * 64).round() / 64 + shift           # exact
    else:
        x = (make(n, experts, F32, 51) + shift).to(dtype)                   # few values, many equal ones
    for renormalize in (False, True):
        got = check(store, x, top, renormalize=renormalize)
    if dtype == F32:                                        # the same differences give the same gradient, whatever the level (z = 0)
        dw = torch.randn((n, top), device="cuda")
        near, far = store.route(x - shift, top, balance=0.5), store.route(x, top, balance=0.5)
        assert torch.equal(near.choice, far.choice) and torch.equal(near.weight, far.weight)
        assert torch.equal(store.route_grad(x - shift, near, dweight=dw), store.route_grad(x, far, dweight=dw))


def test_nan_and_infinity_stay_in_their_items_backward(store):
    x, dw = make(40, 30, F32, 52), torch.randn((40, 3), device="cuda")
    r = store.route(x, 3, balance=1.0, z=0.1)
    clean = store.route_grad(x, r, dweight=dw)
    others = [i for i in range(40) if i not in (7, 9, 11)]
    y = x.clone()
    y[7, 4], y[9, 4] = float("nan"), float("inf")
    y[11] = -float("inf")
    y[11, 2] = float("nan")
    d = store.route_grad(y, r, dweight=dw)
    assert d[[7, 9, 11]].isnan().all() and torch.equal(d[others], clean[others])
