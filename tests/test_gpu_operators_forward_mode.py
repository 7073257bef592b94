"""GPU: every operator refuses every floating-point argument that carries a tangent, and writes nothing."""
import pytest
import torch
import torch.autograd.forward_ad as forward

import test_gpu_memory_operators_use
import test_gpu_operators_autograd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("module,k", [(m, k) for m, n in ((test_gpu_operators_autograd, 11), (test_gpu_memory_operators_use, 6))
                                      for k in range(n)])
def test_arguments_with_tangents(module, k):
    call, args, _ = module.calls()[k]
    for name in args:
        a = {n: x.clone() for n, x in args.items()}
        before = {n: x.clone() for n, x in a.items()}
        with forward.dual_level():
            plain = a[name]
            a[name] = forward.make_dual(plain, torch.ones_like(plain))
            with pytest.raises(ValueError, match="tangent"):
                call(a)
            a[name] = plain
            assert all(torch.equal(a[n], before[n]) for n in a)
            call(a)
