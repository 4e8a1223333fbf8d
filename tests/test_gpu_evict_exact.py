"""Eviction by attention weight: fp32 weights as exact as fp32, and a selection whose weights do not fit a block's shared memory."""
import numpy as np
import pytest
import torch

from oracle import cache_ops_oracle as co
from paper_2512_10310_b200 import binding as B
from tests.helpers import f64
from tests.test_gpu_evict import DEV, _select, _weights_case

pytestmark = pytest.mark.gpu
# A weight exp(s - lse) in fp32.  s: 128 products are added up in floats, in partial sums under 64 (standard normal keys and queries; half a step of those
# is 2^-19 and a rounding's deviation 0.58 of it); six deviations of 128 of them, 6 * 11.3 * 0.58 * 2^-19, scaled by D^-0.5: 2^-17.2.  The
# exponent itself and lse are under 32 in base 2: three roundings of 2^-20.  Together 2^-16.2 of the weight.  (Products of 11 bits would be 2^-12.)
F32_WEIGHT_ERROR = 2.0 ** -16


@pytest.fixture(scope="module")
def handle():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    h = B.evlnCreate(0)
    yield h
    B.evlnDestroy(h)


@pytest.mark.parametrize("hq,hkv,D,L,n,decay", [
    (2, 1, 64, 256, 64, 0.9), (28, 4, 128, 300, 7, 1.0), (4, 2, 64, 1000, 130, 0.0),      # a thread per key
    (28, 4, 128, 4096, 5, 1.0), (28, 4, 128, 4032, 64, 0.5), (64, 8, 128, 2000, 50, 0.9),  # tiles of keys and rows
])
def test_key_weights_in_fp32(handle, hq, hkv, D, L, n, decay):
    cap = L + n + 3
    q, q_rot, k, keys, lse, weights = _weights_case("f32", hq, hkv, D, L, n, cap, L + n + hq, D ** -0.5)
    ref = co.key_weights(f64(q), keys, f64(lse), L, decay, f64(weights), D ** -0.5)
    out = torch.full_like(weights, -1.0)
    B.evlnKeyWeights(handle, B.step_params("f32", hq, hkv, D, L, n, cap, 1e6), q_rot, k, lse, decay, weights, out)
    worst = float((np.abs(f64(out)[:, :L + n] - ref) / (F32_WEIGHT_ERROR * ref + 1e-30)).max())
    assert worst <= 1.0, f"{worst:.2f} times the bound"


@pytest.mark.parametrize("hkv,num_keys,budget,sinks,recent", [
    (2, 330_001, 100_000, 256, 196), (1, 700_001, 1, 0, 0), (3, 400_000, 399_999, 4, 0), (2, 327_681, 327_681, 0, 0), (2, 350_000, 300, 100, 200),
])
@pytest.mark.parametrize("kind", ["spread", "ties", "zeros"])
def test_select_among_more_keys_than_shared_memory_holds(handle, hkv, num_keys, budget, sinks, recent, kind):
    g = torch.Generator().manual_seed(num_keys + budget)
    w = torch.exp(3.0 * torch.randn(hkv, num_keys + 7, generator=g))
    if kind == "ties":
        w = torch.round(torch.rand(hkv, num_keys + 7, generator=g) * 4) / 4
    elif kind == "zeros":
        w.zero_()
        w[:, ::3] = -0.0
    w[:, num_keys:] = 1e30                                        # not among the keys
    got = _select(handle, w.to(DEV), num_keys, budget, sinks, recent)
    assert np.array_equal(got.cpu().numpy(), co.select_keys(f64(w), num_keys, budget, sinks, recent))
