"""Values that nearly cancel in pairs of tokens: what the weights of the second product lose shows in the result, which is small beside what it is
summed from.  Weights of every type are within 2^-20 of themselves (two halves; see decode_reference for the rest of the tolerance)."""
import numpy as np
import pytest

import decode_reference as ref
from test_gpu_cache_attention import HALF, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("fresh", [[1, 3, 2], [20, 1, 9], [50, 7, 33]], ids=["16 rows", "64 rows", "128 rows"])
@pytest.mark.parametrize("bits,dk", [(8, 64), (8, 128), (4, 256)])
def test_values_that_nearly_cancel(dtype, fresh, bits, dk):
    print(f"cancelling values: {dtype}, {bits} bits, dk {dk}, new tokens {fresh}", flush=True)
    p = Problem([12, 40, 64], fresh, kv_heads=1, group=2, dk=dk, bits=bits, dtype=dtype, seed=dk + bits, sharp=0.25)
    for a in (p.kc, p.ks, p.vs):
        a[:, :, 1::2] = a[:, :, 0::2]
    p.vc[:, :, 1::2] = -p.vc[:, :, 0::2]
    p.ks[:, :, 1::2] *= np.float32(1.01)                          # (probabilities that differ by some thousandths)
    want, tol = ref.attention(p.q.double().cpu().numpy(), p.kc, p.vc, p.ks, p.vs, p.table, p.lengths, p.starts, None, None, HALF[dtype], 2.0 ** -20,
                              own_exponents=dtype == "float32")
    tol = tol + (2.0 ** -25 if dtype == "float16" else 0)          # (half a step of fp16's subnormal numbers)
    err = np.abs(p.run().double().cpu().numpy() - want)
    assert (err <= tol).all(), float((err / tol).max())
