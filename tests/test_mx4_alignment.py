"""The pointers that ot_fold_weights_mx4 reads and writes by element (b, bprime):
aligned to their elements, and no further."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as X
from paper_2406_18832_amd import ot
from tests.test_gpu_mx4 import dev, host
from tests.test_mx4_host import CALLS, EINVAL, put, status


@pytest.mark.parametrize("where", ["b", "bprime"])
def test_fold_refuses_pointers_between_elements(where):
    """Before any HIP call: no device is needed."""
    args, at = CALLS["ot_fold_weights_mx4"][0], {"b": 1, "bprime": 8}[where]
    for address in (4097, 4099) + ((4098, 4102) if where == "bprime" else ()):
        assert status("ot_fold_weights_mx4", put(args, at, address)) == EINVAL, address


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [1, 2, 3, 5])
def test_fold_takes_a_bias_and_writes_one_at_any_element(offset):
    N, K = 37, 96
    r = np.random.default_rng(offset)
    W, b = (r.standard_normal(s).astype(np.float16) for s in ((N, K), N + 8))
    z, s = r.uniform(-3, 3, K).astype(np.float32), r.uniform(0.1, 3, K).astype(np.float32)
    c, e, bias = X.fold(W, b[offset:offset + N], z, s)
    Wc, We = ot._mx4_empty(N, K, "cuda")
    out = torch.full((N + 8,), 7.0, device="cuda")
    ot.ot_fold_weights_mx4(dev(W), dev(b)[offset:offset + N], dev(z), dev(s), Wc, We,
                           out[offset:offset + N])
    assert np.array_equal(host(Wc), c) and np.array_equal(host(We), e)
    # a float64 sum of K exact products, then one rounding to fp32
    mags = np.abs(W.astype(np.float64)) @ np.abs(z.astype(np.float64))
    got = host(out)
    assert np.all(np.abs(got[offset:offset + N] - bias) <= 2.0 ** -24 * np.abs(bias) * 1.01 + 2.0 ** -52 * K * mags)
    assert (got[:offset] == 7).all() and (got[offset + N:] == 7).all()
