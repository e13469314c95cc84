"""The tolerances that attention over caches of 4 bits is held to, against kernels that are right and kernels that are wrong, in 64 bits on the host."""
import numpy as np
import pytest
import torch

import attend4_cases as A
import serve_exact as X


@pytest.mark.parametrize("spec", A.specs(), ids=lambda s: s["name"])
def test_right_and_wrong_kernels(spec):
    call = A.make(spec, "cpu")
    ref, var = call.value()
    to_type = X.to_bf16 if call.c.dtype == torch.bfloat16 else lambda x: x.astype(np.float32).astype(np.float64)
    assert X.wrong(call, to_type(call.value(held=True)[0]), ref, var) == []
    for m in spec["mutants"]:
        assert not X.applies(call, m) or X.wrong(call, to_type(call.value(mutant=m)[0]), ref, var), "nothing says that %r is wrong" % m
