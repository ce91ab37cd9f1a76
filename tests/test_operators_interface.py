"""Argument checks of the operators on model tensors that need no device: a call without a store is refused before anything else."""
import ctypes

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
