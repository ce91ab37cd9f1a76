"""The operators where offsets pass 32 bits: the last rows of tensors of more than 2^32 values are what a small call on those rows gives."""
import pytest
import torch

from paper_2104_00501_b200 import binding
from tests.common import dev_keys

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def room(gib):
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of free device memory")


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("length", [4096, 33])
def test_layer_norm_and_its_backward_pass(length):
    room(40)
    n = (1 << 32) // length + 1000
    s = binding.Store(64, 64)
    x = torch.empty((n, length), dtype=BF16, device="cuda").fill_(0.5)
    x[-300:] = torch.randn((300, length), device="cuda").to(BF16)
    w = torch.rand(length, device="cuda")
    tail = x[-300:].clone()
    y, mean, rstd = s.layer_norm(x, w)
    ty, tm, tr = s.layer_norm(tail, w)
    assert torch.equal(y[-300:], ty) and torch.equal(mean[-300:], tm) and torch.equal(rstd[-300:], tr)
    del y
    dx, dw, _ = s.layer_norm_grad(x, x, mean, rstd, w)
    assert torch.equal(dx[-300:], s.layer_norm_grad(tail, tail, tm, tr, w)[0])
    assert s.status_check() == 0


def test_router():
    room(30)
    E = 1000
    n = (1 << 32) // E + 500
    s = binding.Store(64, 64)
    x = torch.zeros((n, E), dtype=BF16, device="cuda")
    x[-100:] = torch.randn((100, E), device="cuda").to(BF16)
    r = s.route(x, 3, balance=1.0)
    t = s.route(x[-100:].clone(), 3, balance=1.0)
    assert torch.equal(r.choice[-100:], t.choice) and torch.equal(r.weight[-100:], t.weight) and torch.equal(r.lse[-100:], t.lse)
    assert r.counts.sum().item() == 3 * n and r.counts[:3].min().item() >= n - 100 and r.tokens.item() == n
    d = s.route_grad(x, r, out=x)                           # in place
    assert torch.isfinite(d[-100:].float()).all() and s.status_check() == 0


def test_normalised_pull():
    room(40)
    keys, length = 36_000_000, 128
    s = binding.Store(keys, length, sync_interval=0)
    s.init_uniform(0, 1, 0.5)
    at = dev_keys([keys - 1, 0, keys - 2, 33_554_432, 33_554_431, keys])
    rows = s.pull(at)
    y, mean, rstd, pulled = s.pull_norm(at, rows=True)
    assert torch.equal(pulled, rows) and s.status_check() == binding.EKEY
    x = rows.double()
    d = x - x.mean(1, keepdim=True)
    ref = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5)
    # 64 roundings of 2^-24, as for layer norm elsewhere; the mean of the magnitudes over the deviation is below 1 here
    assert ((y.double() - ref).abs() <= 64 * 2.0 ** -24 * (ref.abs() + 1)).all()
    s.close()


def test_orthogonalized_update_far_into_a_tensor():
    room(30)
    batch = 60_000
    s = binding.Store(64, 64)
    g = torch.empty((batch, 300, 300), dtype=BF16, device="cuda")         # 5.4e9 values; three matrices of them are taken
    g[-1] = torch.randn((300, 300), device="cuda").to(BF16)
    g[batch // 2] = g[-1]
    g[0] = g[-1]
    part = g[:: batch // 2][:2]
    last = s.orthogonalize(g[-1])
    assert torch.equal(s.orthogonalize(part)[1], last)
    wide = torch.as_strided(g, (2, 300, 300), (4_500_000_000, 300, 1))  # a batch stride beyond 32 bits
    wide[1] = g[-1]
    assert torch.equal(s.orthogonalize(wide)[1], last) and torch.equal(s.orthogonalize(wide)[0], s.orthogonalize(g[0]))


@pytest.mark.parametrize("n,length", [(3_000_000, 300), (4_000_000, 128)])
def test_sums_over_millions_of_rows(n, length):
    # equal values, whose roundings all go one way.  A team adds at most 128 rows one after the other, a block at most 9 such runs, 8 warps
    # and 32 lanes, the last kernel 19 blocks and 32 runs of them: at most 220 roundings with those of the terms
    room(10)
    s = binding.Store(64, 64)
    x = torch.full((n, length), 0.1, device="cuda")
    mean, rstd = torch.full((n,), -0.2, device="cuda"), torch.full((n,), 1.1, device="cuda")
    _, dw, db = s.layer_norm_grad(x, x, mean, rstd, torch.ones(length, device="cuda"), need_dx=False)
    v = x[0, 0].double()
    for got, term in ((db, v), (dw, v * (v - mean[0].double()) * rstd[0].double())):
        assert ((got.double() - n * term).abs() <= 220 * 2.0 ** -24 * n * term).all()


def test_normalised_pull_of_the_longest_rows():
    # rows of 2^28 values and more are refused, as layer_norm refuses them: positions within a row are held in 32 bits
    room(12)
    s = binding.Store(1, 1 << 28)
    with pytest.raises(binding.NupsError) as e:
        s.pull_norm(dev_keys([0]))
    assert e.value.code == binding.EINVAL
    s.close()
    s = binding.Store(1, (1 << 28) - 4)
    s.init_uniform(0, 1, 0.5)
    y, mean, rstd, rows = s.pull_norm(dev_keys([0]), rows=True)
    want = s.layer_norm(rows)
    assert torch.equal(y, want[0]) and torch.equal(mean, want[1]) and torch.equal(rstd, want[2])
    # the sums' own rounding is 2^-53 a step: what is left is the roundings of a difference, its square, the mean and rstd
    x = rows.double()
    m = x.mean()
    v = ((x - m) ** 2).mean()
    assert abs(mean.item() - m) <= 2.0 ** -24 * abs(m) + 1e-9 and abs(rstd.item() * torch.sqrt(v + 1e-5).item() - 1) <= 16 * 2.0 ** -24
    s.close()
