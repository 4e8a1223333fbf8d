"""Attention over the 8-bit cache (evlnPaged8StepAttention) at the ends of its range: keys and queries of zero or nearly so, against fp64."""
import numpy as np
import pytest
import torch

from oracle import cache_ops_oracle as co
from paper_2512_10310_b200 import binding as B
from tests.helpers import f64
from tests.test_gpu_cache8 import D, DEV, LSE_ERROR, P, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def handle():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    h = B.evlnCreate(0)
    yield h
    B.evlnDestroy(h)


# new tokens of 7 query heads: 7, 14, 28 and 63 rows on the codes, 70 through the copy
TOKENS = [1, 2, 4, 9, 10]


def _append(x, q, k, v):
    q_rot = torch.empty(x.hkv, x.total * x.G, D, dtype=torch.bfloat16, device=DEV)
    B.evlnPaged8RopeAppend(x.h, x.params(), None, q, k, v, x.lens, x.offs, x.table, q_rot, *x.codes, *x.scales)
    return q_rot


def _zero_keys(x, pages=None):
    """Earlier keys of the first episode (of its pages `pages`) become zeros as an append of zeros leaves them."""
    for i in range((x.lens[0] + P - 1) // P) if pages is None else pages:
        page, used = x.rows[0][i], min(P, x.lens[0] - i * P)
        x.codes[0][page, :, :used] = 0
        x.scales[0][page] = 2.0 ** -120


@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("L", [0, 40, 100, 700])
@pytest.mark.parametrize("q_size,scale", [(0.0, 0.0), (2.0 ** -14, 0.0), (2.0 ** -40, 0.0), (1.0, 2.0 ** -60), (1.0e30, 0.0)])
def test_keys_of_zeros(handle, n, L, q_size, scale):
    """Every key weighs the same, whatever the query: the mean of the values."""
    x = Batch(handle, [L], [n], 14, 2, seed=L + n, scale=scale)
    _zero_keys(x)
    q, k, v = x.tokens()
    _append(x, q, torch.zeros_like(k).contiguous(), v.contiguous())
    q_rot = x.q_rot(q_size)
    out, lse = x.attend(q_rot)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    x.check(q_rot, out, lse)
    count = np.log(np.arange(L + 1, L + n + 1))[:, None]
    assert np.abs(f64(lse) - count).max() <= LSE_ERROR


@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("q_size", [0.0, 2.0 ** -14, 2.0 ** -100])
def test_small_queries_over_pages_of_zeros_and_others(handle, n, q_size):
    x = Batch(handle, [300], [n], 7, 1, seed=n)
    _zero_keys(x, [0, 2])
    x.fill_new()
    q_rot = x.q_rot(q_size)
    out, lse = x.attend(q_rot)
    x.check(q_rot, out, lse)


@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("L", [0, 64, 200])
def test_a_step_of_zeros(handle, n, L):
    """A warm-up on zeroed inputs and a zeroed cache: zeros, and the logarithm of the number of keys."""
    x = Batch(handle, [L], [n], 28, 4, seed=n)
    _zero_keys(x)
    for i in range((L + P - 1) // P):
        x.codes[1][x.rows[0][i]] = 0
        x.scales[1][x.rows[0][i]] = 2.0 ** -120
    q_rot = _append(x, *(torch.zeros(x.total, h, D, dtype=torch.bfloat16, device=DEV) for h in (28, 4, 4)))
    assert bool((q_rot == 0).all())
    out, lse = x.attend(q_rot)
    assert bool((out == 0).all())
    assert np.abs(f64(lse) - np.log(np.arange(L + 1, L + n + 1))[:, None]).max() <= LSE_ERROR


@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("L", [0, 3, 30, 500])
def test_log_sum_exps_of_flat_scores(handle, n, L):
    """Scores of small products, whose log-sum-exps show what exponentials and sums lose: 2^-22 an exponential, a rounding for each of the reference, the
    logarithm and the product (2^-24 of a number the size of the result)."""
    x = Batch(handle, [L], [n], 14, 2, seed=L + n, kv_size=0.1)
    x.fill_new()
    q_rot = x.q_rot(0.05)
    out, lse = x.attend(q_rot)
    x.check(q_rot, out, lse)
    q, k = f64(q_rot).reshape(2, -1, 7, D).transpose(1, 0, 2, 3).reshape(-1, 14, D), x.episode(0, 0)
    ref = co.attention(q, k, np.zeros_like(k), L, D ** -0.5)[1]
    reach = np.abs(q).sum(-1).max() * np.abs(k).max() * D ** -0.5
    assert (np.abs(f64(lse) - ref) <= 2.0 ** -21 + 2.0 ** -22 * (reach + np.abs(ref))).all()


def test_a_frame_beside_single_tokens(handle):
    """One episode of more than 64 rows: the whole batch goes through the copy, single tokens and an idle episode too."""
    x = Batch(handle, [900, 5, 64, 0, 333, 1000], [1, 1, 1, 1, 30, 0], 28, 4, seed=3)
    x.fill_new()
    q_rot = x.q_rot()
    out, lse = x.attend(q_rot)
    x.check(q_rot, out, lse)
