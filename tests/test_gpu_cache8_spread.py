"""Attention over the 8-bit cache where its pages' value scales are far apart and the weight of a row is on some of them only, against fp64."""
import numpy as np
import pytest
import torch

from oracle import cache_ops_oracle as co
from paper_2512_10310_b200 import binding as B
from tests.helpers import f64
from tests.test_gpu_cache8 import D, DEV, P, P_ERROR, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def handle():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    h = B.evlnCreate(0)
    yield h
    B.evlnDestroy(h)


def _aim(x, bits, size):
    """Rewrites the keys page by page: those of page i of every episode lie along one direction, so that a query along it, of length `size`, scores about
    bits[i] (log2) there.  Returns such queries."""
    u = torch.sign(torch.randn(D, generator=x.g))
    along = size * u * D ** -0.5                         # |q| = size; key c u: score = size * c * sqrt(D) * D^-0.5 = size * c (natural units)
    for b, (L, n) in enumerate(zip(x.lens, x.news)):
        for i in range((L + n + P - 1) // P):
            page, c = x.rows[b][i], bits[i % len(bits)] * float(np.log(2.0)) / size
            k = c * u + 0.3 / size * torch.randn(x.hkv, P, D, generator=x.g)
            s = torch.tensor([co.scale_for(f64(k[g])) for g in range(x.hkv)], dtype=torch.float32)
            x.codes[0][page] = (k / s[:, None, None]).to(torch.float8_e4m3fn).view(torch.uint8).to(DEV)
            x.scales[0][page] = s.to(DEV)
    q = along * (1.0 + 0.02 * torch.randn(x.hkv, x.total * x.G, 1, generator=x.g))
    return q.bfloat16().to(DEV)


def _set_value_scales(x, exponents):
    for b, (L, n) in enumerate(zip(x.lens, x.news)):
        for i in range((L + n + P - 1) // P):
            x.scales[1][x.rows[b][i]] = 2.0 ** exponents[i % len(exponents)]


def _check(x, q_rot, out, lse, some=None):
    """As Batch.check, with room for fp32 scores (2^-24 of their products' sizes, four roundings deep) that reach hundreds."""
    q = f64(q_rot).reshape(x.hkv, -1, x.G, D).transpose(1, 0, 2, 3).reshape(-1, x.hq, D)
    for b, L in enumerate(x.lens):
        if x.news[b] == 0 or (some is not None and b not in some):
            continue
        rows = slice(x.offs[b], x.offs[b + 1])
        k, v = x.episode(0, b), x.episode(1, b)
        ref, ref_lse, size = co.attention(q[rows], k, v, L, D ** -0.5)
        reach = np.abs(q[rows]).sum(-1).max() * np.abs(k).max() * D ** -0.5
        slack = P_ERROR[x.kind] + 2.0 ** -22 * reach
        worst = float((np.abs(f64(out[rows]) - ref) / (2.0 ** -8 * np.abs(ref) + slack * size + 1e-37)).max())
        assert worst <= 1.0, f"episode {b}: {worst:.3g} times the bound"
        assert np.abs(f64(lse[rows]) - ref_lse).max() <= 2.0 ** -14 + 2.0 ** -22 * reach


# (score of each page of 64 keys in bits, exponent of its value scale): the weight on small values and none on large ones; products p v that are alike
# where p and v are 2^33 and more apart; each the other way round
PAGES = {
    "small_values_weigh_10": ([0, -90, 0, -90, 0], [0, 10, -1, 10, 0]),
    "small_values_weigh_20": ([0, -90, 0, -90, 0], [0, 20, -1, 20, 0]),
    "small_values_weigh_30": ([0, -90, 0, -90, 0], [0, 30, -1, 30, 0]),
    "small_values_weigh_60": ([0, -120, 0, -120, 0], [0, 60, -1, 60, 0]),
    "small_values_weigh_110": ([0, -160, 0, -160, 0], [-55, 55, -56, 55, -55]),
    "large_first": ([-90, 0, 0, 0, 0], [40, 0, 1, 0, 0]),
    "large_last": ([0, 0, 0, 0, -90], [0, 1, 0, 0, 40]),
    "products_alike": ([0, -33, 0, -33, -20], [0, 33, -1, 33, 20]),
    "products_alike_far": ([0, -60, -100, -60, -30], [0, 60, 100, 60, 30]),
    "large_values_little_weight": ([0, -33, 0, -33, 0], [0, 40, 0, 40, 0]),
    "rising_scores_falling_values": ([-200, -150, -100, -50, 0], [60, 40, 20, 0, -20]),
    "rising_scores_rising_values": ([-100, -75, -50, -25, 0], [-40, -20, 0, 20, 40]),
    "falling_scores_rising_values": ([0, -25, -50, -75, -100], [-40, -20, 0, 20, 40]),
}


@pytest.mark.parametrize("n", [1, 2, 4, 9, 10])
@pytest.mark.parametrize("kind", list(PAGES))
def test_weight_and_value_scales_apart(handle, kind, n):
    bits, exponents = PAGES[kind]
    x = Batch(handle, [5 * P - 20], [n], 7, 1, seed=n + len(kind))
    x.fill_new()
    q_rot = _aim(x, bits, 16.0)
    _set_value_scales(x, exponents)
    _check(x, q_rot, *x.attend(q_rot))


@pytest.mark.parametrize("n", [1, 2, 4, 9])
@pytest.mark.parametrize("kind", ["small_values_weigh_30", "products_alike", "rising_scores_falling_values", "falling_scores_rising_values"])
def test_weight_and_value_scales_apart_within_a_run(handle, kind, n):
    """Enough episodes and heads that a warp walks over several pages of one of them, and over the border between two."""
    bits, exponents = PAGES[kind]
    x = Batch(handle, [1500 + 13 * b for b in range(20)], [n] * 20, 56, 8, seed=n)
    x.fill_new()
    q_rot = _aim(x, bits, 16.0)
    _set_value_scales(x, exponents)
    _check(x, q_rot, *x.attend(q_rot), some=[0, 7, 19])


@pytest.mark.parametrize("n", [1, 9])
def test_values_near_the_ends_of_the_range(handle, n):
    """Value scales of 2^119 and of 2^-120: sums of many keys stay inside floats."""
    for exponent in (119, -120):
        x = Batch(handle, [2000], [n], 7, 1, seed=n)
        x.fill_new()
        for i in range((2000 + n + P - 1) // P):
            x.scales[1][x.rows[0][i]] = 2.0 ** exponent
        q_rot = x.q_rot(0.1)
        _check(x, q_rot, *x.attend(q_rot))
