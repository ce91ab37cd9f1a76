"""The operators as a model uses them: embeddings pulled and normalised, routed to experts whose matrices are rows of a second store,
gradients back through both, embeddings updated by push, matrices by an orthogonalized update that push adds.  Against the same
model in 64 bits with torch's differentiation (on the host), and captured into a graph.
"""
import numpy as np
import pytest
import torch

from paper_2104_00501_b200 import binding
from tests.common import dev_keys

pytestmark = pytest.mark.gpu
F64 = torch.float64
KEYS, L, E, K, N = 300, 32, 6, 2, 150
BALANCE, Z, RATE, MUON = 0.02, 0.003, 0.1, 0.05


def setup():
    rng = np.random.default_rng(3)
    emb = rng.normal(size=(KEYS, L)).astype(np.float32)
    mats = (rng.normal(size=(E, L * L)) / np.sqrt(L)).astype(np.float32)
    s = binding.Store(KEYS, L, workers=2, deterministic=True, sync_interval=0)
    s.write_table(0, emb)
    s.set_management(dev_keys(np.arange(0, 40)), binding.REPLICATE)
    m = binding.Store(E, L * L, workers=2, deterministic=True, sync_interval=0)
    m.write_table(0, mats)
    dev = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()  # noqa: E731
    p = dict(keys=dev_keys(rng.integers(0, KEYS, N)), w=dev(1 + 0.1 * rng.normal(size=L)), b=dev(0.1 * rng.normal(size=L)), router=dev(rng.normal(size=(L, E)) * 0.3),
             target=dev(rng.normal(size=(N, L))), active=torch.arange(N, device="cuda") % 10 != 9)
    return s, m, p, emb, mats


def step(s, m, p):
    """One training step; everything that is compared."""
    y, mean, rstd, rows = s.pull_norm(p["keys"], p["w"], p["b"], rows=True)
    logits = y @ p["router"]
    r = s.route(logits, K, active=p["active"], renormalize=True, balance=BALANCE, z=Z)
    mats = m.pull(torch.arange(E, dtype=torch.int32, device="cuda")).view(E, L, L)
    at = r.choice.clamp(min=0).long()
    parts = torch.einsum("nl,nklj->nkj", y, mats[at])                    # what each chosen expert gives
    out = (r.weight[:, :, None] * parts).sum(1)
    err = torch.where(p["active"][:, None], out - p["target"], 0.0)
    dweight = (err[:, None, :] * parts).sum(2).contiguous()
    dlogits = s.route_grad(logits, r, dweight=dweight)
    scaled = r.weight[:, :, None] * err[:, None, :]
    dmats = torch.zeros_like(mats).index_add_(0, at.reshape(-1), torch.einsum("nl,nkj->nklj", y, scaled).reshape(-1, L, L))
    dy = dlogits @ p["router"].t() + torch.einsum("nkj,nklj->nl", scaled, mats[at])
    dx, dw, db = s.layer_norm_grad(rows, dy, mean, rstd, p["w"])
    s.push(p["keys"], (-RATE * dx).contiguous())
    m.push(torch.arange(E, dtype=torch.int32, device="cuda"), m.orthogonalize(dmats, scale=-MUON).view(E, L * L))
    loss = 0.5 * (err * err).sum() + r.loss[0]
    return loss, dw, db, dmats, r.counts, dlogits


def reference(p, emb, mats):
    x = torch.from_numpy(emb).double().requires_grad_()
    M = torch.from_numpy(mats).double().view(E, L, L).requires_grad_()
    w, b, router = (p[k].cpu().double() for k in ("w", "b", "router"))
    w.requires_grad_()
    b.requires_grad_()
    keys, on = p["keys"].cpu().long(), p["active"].cpu()
    rows = x[keys]
    mean = rows.mean(1, keepdim=True)
    y = (rows - mean) / torch.sqrt(((rows - mean) ** 2).mean(1, keepdim=True) + 1e-5) * w + b
    logits = y @ router
    prob = torch.softmax(logits, 1)
    top = torch.topk(logits, K, 1).indices                               # no ties among these
    weight = torch.gather(prob, 1, top)
    weight = weight / weight.sum(1, keepdim=True)
    counts = torch.bincount(top[on].reshape(-1), minlength=E)
    T = int(on.sum())
    balance = E / (K * T) * (counts * (prob[on].sum(0) / T)).sum()
    z = (torch.logsumexp(logits, 1)[on] ** 2).sum() / T
    out = (weight[:, :, None] * torch.einsum("nl,nklj->nkj", y, M[top])).sum(1)
    loss = 0.5 * ((out - p["target"].cpu().double())[on] ** 2).sum() + BALANCE * balance + Z * z
    loss.backward()
    return loss.detach(), w.grad, b.grad, M.grad, counts, x.grad


def iterate(g):
    g = g / (g.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    for _ in range(5):
        a = g @ g.transpose(1, 2)
        g = 3.4445 * g + (-4.7750 * a + 2.0315 * a @ a) @ g
    return g


def close(got, want, part):
    """2-norm of the difference over that of the result.  fp32 throughout: sums of at most N K L = 10,000 terms whose magnitudes exceed
    the result by less than 100 times: 100 * 128 roundings of 2^-24 for the gradients; the orthogonalized update multiplies that
    by at most 3.4445^5 / growth (about 30 here)."""
    off = (got.double().cpu() - want).norm() / want.norm()
    assert off <= part, float(off)


def test_a_training_step():
    s, m, p, emb, mats = setup()
    loss, dw, db, dmats, counts, _ = step(s, m, p)
    rl, rdw, rdb, rdm, rcounts, rdx = reference(p, emb, mats)
    bound = 100 * 128 * 2.0 ** -24
    assert torch.equal(counts.cpu(), rcounts)
    close(loss, rl, bound)
    close(dw, rdw, bound)
    close(db, rdb, bound)
    close(dmats, rdm, bound)
    s.sync()
    m.sync()
    close(s.read_table() - torch.from_numpy(emb).cuda(), -RATE * rdx, bound)
    close(m.read_table().view(E, L, L) - torch.from_numpy(mats).cuda().view(E, L, L), -MUON * iterate(rdm), 30 * bound)
    assert s.status_check() == 0 and m.status_check() == 0


def test_forward_and_backward_captured_and_replayed():
    s, m, p, _, _ = setup()
    y, mean, rstd, rows = s.pull_norm(p["keys"], p["w"], p["b"], rows=True)          # what a capture must not do for the first time
    dy = torch.randn_like(y)

    def run():
        y, mean, rstd, rows = s.pull_norm(p["keys"], p["w"], p["b"], rows=True)
        r = s.route(y @ p["router"], K, active=p["active"], balance=BALANCE, z=Z)
        d = s.route_grad(y @ p["router"], r)
        return (y, r.choice, r.weight, r.counts, r.loss, d, *s.layer_norm_grad(rows, dy, mean, rstd, p["w"]), s.orthogonalize(dy.view(15, 10, L)))

    want = run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    for _ in range(2):
        for t in got:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("n,length", [(1000, 4096), (400, 1000)])
def test_rings_in_a_graph(n, length):
    # the kernels that ask for large shared memory, first used inside a capture
    s = binding.Store(64, 64)
    x, w = torch.randn((n, length), device="cuda"), torch.rand(length, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y, mean, rstd = s.layer_norm(x, w)
        got = s.layer_norm_grad(x, y, mean, rstd, w)
    g.replay()
    torch.cuda.synchronize()
    want = s.layer_norm(x, w)
    assert torch.equal(y, want[0]) and all(torch.equal(a, b) for a, b in zip(got, s.layer_norm_grad(x, y, mean, rstd, w)))
