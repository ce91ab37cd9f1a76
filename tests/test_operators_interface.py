"""Argument checks of the operators on model tensors that need no device: a call without a store is refused before anything else."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2104_00501_b200 import binding


def test_calls_without_a_store_are_refused():
    lib = binding.load()
    size = ctypes.c_uint64(77)
    assert lib.nups_layer_norm(None, None, 0, 4, 1, 4, None, None, 0, 1e-5, None, 0, 4, None, None, None) == binding.EINVAL
    assert lib.nups_pull_norm(None, None, 1, None, None, 1e-5, None, 0, None, None, None, None) == binding.EINVAL
    assert lib.nups_layer_norm_grad(None, None, 0, 4, None, 0, 4, 1, 4, None, None, None, 0, None, 4, None, None, None, 0, None) == binding.EINVAL
    assert lib.nups_layer_norm_grad_scratch(None, 1, 4, 0, ctypes.byref(size)) == binding.EINVAL and size.value == 77
    assert lib.nups_route_scratch(None, 1, 4, ctypes.byref(size)) == binding.EINVAL and size.value == 77
    assert lib.nups_route(None, None, 0, 4, 1, 4, 1, None, 0, 0.0, 0.0, None, None, None, None, None, None, None, None, 0, None) == binding.EINVAL
    assert lib.nups_route_grad(None, None, 0, 4, 1, 4, 1, None, 0, 0.0, 0.0, None, None, None, None, None, None, None, None, 4, None) == binding.EINVAL
    assert lib.nups_orthogonalize_scratch(None, 1, 4, 4, ctypes.byref(size)) == binding.EINVAL and size.value == 77
    assert lib.nups_orthogonalize(None, None, 0, 4, 16, 1, 4, 4, 5, None, 1e-7, 1.0, None, 4, 16, None, 0, None) == binding.EINVAL


def test_addresses_that_do_not_suit_their_values_are_refused():
    # before anything is asked of a device.  The store is made up of ones: its device is none, so that a call which is not refused for its
    # address ends with another status; nothing here is ever read at an address
    lib = binding.load()
    fake = ctypes.create_string_buffer(b"\xff" * 65536, 65536)
    store, at, much = ctypes.addressof(fake), 1 << 20, 1 << 50

    def goes_on(call):
        assert call() in (binding.ESTATE, binding.ECUDA)

    def refused(call, *addresses):
        """One address after the other moved by one byte, and by half a value where its values are larger than that."""
        goes_on(lambda: call(**{}))
        for name, size in addresses:
            for off in {1, size // 2, size - 1}:
                assert call(**{name: at + off}) == binding.EINVAL, (name, off)
            goes_on(lambda: call(**{name: at + size}))
            goes_on(lambda: call(**{name: None})) if name in optional else None

    optional = {"w", "b", "mean", "rstd", "rows", "dw", "db", "dloss", "dweight", "lse", "prob", "loss"}
    for x_type, size in ((0, 4), (1, 8), (2, 2), (3, 2)):
        for w_type, w_size in ((x_type, size),) + (((0, 4),) if size == 2 else ()):
            s_size = 8 if x_type == 1 else 4
            refused(lambda x=at, y=at, w=at, b=at, mean=at, rstd=at: lib.nups_layer_norm(store, x, x_type, 9, 5, 9, w, b, w_type, 1e-5, y, x_type, 9, mean, rstd, None),
                    ("x", size), ("y", size), ("w", w_size), ("b", w_size), ("mean", s_size), ("rstd", s_size))
            optional -= {"mean", "rstd"}                    # the backward pass needs them
            refused(lambda x=at, dy=at, w=at, mean=at, rstd=at, dx=at, dw=at, db=at: lib.nups_layer_norm_grad(
                store, x, x_type, 9, dy, x_type, 9, 5, 9, mean, rstd, w, w_type, dx, 9, dw, db, at, much, None),
                    ("x", size), ("dy", size), ("w", w_size), ("mean", s_size), ("rstd", s_size), ("dx", size), ("dw", w_size), ("db", w_size))
            optional |= {"mean", "rstd"}
        if x_type != 1:
            refused(lambda g=at, out=at: lib.nups_orthogonalize(store, g, x_type, 9, 45, 2, 5, 9, 5, (ctypes.c_float * 3)(1.5, -0.5, 0), 1e-7, 1.0, out, 9, 45, None, 0, None),
                    ("g", size), ("out", size))
            refused(lambda x=at, choice=at, weight=at, lse=at, counts=at, tokens=at, prob=at, loss=at: lib.nups_route(
                store, x, x_type, 9, 5, 9, 2, None, 0, 0.0, 0.0, choice, weight, lse, counts, tokens, prob, loss, at, much, None),
                    ("x", size), ("choice", 4), ("weight", 4), ("lse", 4), ("counts", 8), ("tokens", 8), ("prob", 4), ("loss", 4))
            optional -= {"lse"}
            refused(lambda x=at, choice=at, weight=at, lse=at, counts=at, tokens=at, dloss=at, dweight=at, d=at: lib.nups_route_grad(
                store, x, x_type, 9, 5, 9, 2, None, 0, 0.0, 0.0, choice, weight, lse, counts, tokens, dloss, dweight, d, 9, None),
                    ("x", size), ("choice", 4), ("weight", 4), ("lse", 4), ("counts", 8), ("tokens", 8), ("dloss", 4), ("dweight", 4), ("d", size))
            optional |= {"lse"}
    refused(lambda keys=at, w=at, b=at, y=at, rows=at, mean=at, rstd=at: lib.nups_pull_norm(store, keys, 5, w, b, 1e-5, y, 0, rows, mean, rstd, None),
            ("keys", 4), ("w", 4), ("b", 4), ("y", 16), ("rows", 16), ("mean", 4), ("rstd", 4))


# ------------------------------------------------------------------------------------------------
# the binding's own work, on host tensors: a store whose library takes down the calls
# ------------------------------------------------------------------------------------------------
class Calls:
    """Stands for the library: *_scratch calls name 4096 bytes, the others are converted as ctypes would and taken down."""

    def __init__(self):
        self.made, self.types = [], binding.load()

    def __getattr__(self, name):
        types = getattr(self.types, name).argtypes

        def call(*args):
            assert len(args) == len(types)
            if name.endswith("_scratch"):
                args[-1]._obj.value = 4096
            else:
                for kind, value in zip(types, args):
                    kind.from_param(value)
                self.made.append((name, args))
            return 0
        return call


@pytest.fixture
def host(monkeypatch):
    """(store on host tensors, its calls, sizes of the scratch that is held)."""
    held = {}

    def alloc(size, stream):
        at = 1 << 20 | len(held) << 12
        held[at] = size
        return at

    monkeypatch.setattr(binding, "_current_device", lambda: -1)
    monkeypatch.setattr(binding, "_current_stream", lambda index: 0)
    monkeypatch.setattr(binding, "_scratch_alloc", alloc)
    monkeypatch.setattr(binding, "_scratch_free", held.pop)
    s = object.__new__(binding.Store)
    s._l, s._s, s._index, s._scratch_sizes, s.device, s.dtype, s.L = Calls(), None, -1, {}, torch.device("cpu"), torch.float32, 8
    return s, s._l.made, held


def test_scratch_is_given_back_whatever_becomes_of_the_call(host):
    s, made, held = host
    x, mean = torch.ones(200, 300), torch.ones(200)
    s.route(x, 2, losses=True)
    s.layer_norm_grad(x, x, mean, mean)
    s.orthogonalize(x)
    assert [name for name, _ in made] == ["nups_route", "nups_layer_norm_grad", "nups_orthogonalize"] and not held
    for call in (lambda: s.orthogonalize(x, steps=5.0), lambda: s.orthogonalize(x, scale="1"), lambda: s.orthogonalize(x, coefficients=(1, 2, "3")),
                 lambda: s.route(x, 2, z="0"), lambda: s.route(x, 2, renormalize=0.5)):
        with pytest.raises((TypeError, ctypes.ArgumentError)):
            call()
        assert not held


def test_the_module_can_be_imported_on_a_torch_without_cuda():
    # such a torch has none of these names; inputs, oracles and checks of arguments still use the module there
    code = "import torch\nfor name in [n for n in dir(torch._C) if n.startswith('_cuda_')]: delattr(torch._C, name)\nfrom paper_2104_00501_b200 import binding\nassert binding.EXPORTS"
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr


def refused(call):
    with pytest.raises(binding.NupsError) as e:
        call()
    assert e.value.code == binding.EINVAL


def test_an_output_of_another_type_than_the_one_asked_for(host):
    s, made, _ = host
    x, out = torch.ones(4, 8), torch.empty(4, 8, dtype=torch.bfloat16)
    for asked in (torch.float32, torch.float16):
        refused(lambda: s.layer_norm(x, out=out, out_dtype=asked))
    assert not made
    assert s.layer_norm(x, out=out, out_dtype=torch.bfloat16, stats=False) is out and s.layer_norm(x, out=out, stats=False) is out and len(made) == 2


def test_sizes_beyond_32_bits_are_not_cut(host):
    # 2^32 + 4 would arrive as 4.  Tensors without memory: the calls are refused before they ask for an address
    s, made, _ = host
    far = torch.empty((1, 2 ** 32 + 4), dtype=torch.bfloat16, device="meta")
    stat = torch.ones(1)
    refused(lambda: s.layer_norm(far))
    refused(lambda: s.layer_norm_grad(far, far, stat, stat))
    refused(lambda: s.route(far, 2))
    for shape in ((2 ** 32 + 4, 1), (1, 2 ** 32 + 4), (2 ** 32 + 4, 1, 1)):
        refused(lambda: s.orthogonalize(torch.empty(shape, dtype=torch.bfloat16, device="meta")))
    for steps in (2 ** 32 + 5, 5 - 2 ** 32, -1, 0, 65):
        refused(lambda: s.orthogonalize(torch.ones(4, 4), steps=steps))
    assert not made


def test_routings_of_other_shapes(host):
    s, made, _ = host
    x = torch.ones(6, 4)
    r = s.route(x, 2, balance=1.0)
    s.route_grad(x, r)
    calls = len(made)
    for other in (dict(choice=r.choice[:, 0].contiguous()), dict(choice=r.choice.view(6, 2, 1), weight=r.weight.view(6, 2, 1)), dict(lse=torch.ones(6, 2)),
                  dict(lse=torch.ones(())), dict(counts=torch.ones(4, 2, dtype=torch.int64)), dict(counts=torch.ones((), dtype=torch.int64))):
        refused(lambda: s.route_grad(x, r._replace(**other)))
    assert len(made) == calls
