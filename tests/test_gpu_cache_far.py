"""The operators around the cache where elements lie beyond 2^31: the same bits as from a small cache."""
import numpy as np
import pytest
import torch

from oracle import cache_ops_oracle as co
from paper_2512_10310_b200 import binding as B
from tests.helpers import f64
from tests.test_gpu_head_norm import DTYPES, HALF_STEP, _expected

pytestmark = pytest.mark.gpu
DEV, D, CAP = "cuda:0", 128, 9_000_000           # head 2 starts behind 2.3e9 elements
THETA, EPS = 1.0e6, 1e-6


@pytest.fixture(scope="module")
def handle():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    h = B.evlnCreate(0)
    yield h
    B.evlnDestroy(h)


@pytest.mark.parametrize("dtype,hq,L,n", [("bf16", 6, 300, 1), ("bf16", 36, 5000, 3), ("f32", 6, 300, 1), ("f32", 36, 5000, 3)])
def test_key_weights(handle, dtype, hq, L, n):
    """fp32: 2 rows by a thread per key, 36 rows over 118 tiles of keys by tiles."""
    g = torch.Generator().manual_seed(L)
    small = torch.randn(3, L + n, D, generator=g).to(DTYPES[dtype]).to(DEV)
    q = torch.randn(3, n * hq // 3, D, generator=g).to(DTYPES[dtype]).to(DEV)
    lse = (8.0 + torch.rand(n, hq, generator=g)).to(DEV)
    start = torch.rand(3, L + n, generator=g).to(DEV)
    far = torch.empty(3, CAP, D, dtype=DTYPES[dtype], device=DEV)
    far[:, :L + n] = small
    w_far = torch.zeros(3, CAP, device=DEV)
    w_far[:, :L + n] = start
    w_near = start.clone()
    B.evlnKeyWeights(handle, B.step_params(dtype, hq, 3, D, L, n, CAP, THETA), q, far, lse, 0.5, w_far, w_far)
    B.evlnKeyWeights(handle, B.step_params(dtype, hq, 3, D, L, n, L + n, THETA), q, small, lse, 0.5, w_near, w_near)
    assert bool((w_near != 0.5 * start).all())
    assert torch.equal(w_far[:, :L + n], w_near) and not bool(w_far[:, L + n:].any())


@pytest.mark.parametrize("dtype,slack", [("bf16", 2.0 ** -20), ("f32", 2.0 ** -26)])
def test_norm_append_at_the_end_of_a_long_cache(handle, dtype, slack):
    """Angles of 9 million radians: 2^-29 of a turn in double."""
    n, L = 3, CAP - 5
    g = torch.Generator().manual_seed(9)
    x = [torch.randn(n, 3, D, generator=g).to(DTYPES[dtype]).to(DEV) for _ in range(3)]
    k, v = (torch.empty(3, CAP, D, dtype=DTYPES[dtype], device=DEV) for _ in range(2))
    q_rot = torch.empty(3, n, D, dtype=DTYPES[dtype], device=DEV)
    for t in (k, v):
        t[:, L - 2:] = 7.0
    B.evlnNormRopeAppend(handle, B.step_params(dtype, 3, 3, D, L, n, CAP, THETA), B.head_norm(None, None, EPS), *x, q_rot, k, v)
    rq, rk, pq, pk = _expected(x[0], x[1], None, None, EPS, np.arange(L, L + n), THETA)
    for got, ref, pair in ((q_rot.transpose(0, 1), rq, pq), (k[:, L:L + n].transpose(0, 1), rk, pk)):
        assert (np.abs(f64(got) - ref) <= HALF_STEP[dtype] * np.abs(ref) + slack * pair).all()
    assert torch.equal(v[:, L:L + n].transpose(0, 1), x[2])
    for t in (k, v):
        assert bool((t[:, L - 2:L] == 7.0).all()) and bool((t[:, L + n:] == 7.0).all())


def test_gather_in_fp32(handle):
    g = torch.Generator().manual_seed(2)
    slots = [0, 77, CAP - 1]
    rows = torch.randn(2, 3, 3, D, generator=g).to(DEV)
    stores = [torch.empty(3, CAP, D, device=DEV) for _ in range(2)]
    for t, r in zip(stores, rows):
        t[:, slots] = r
    kept = torch.tensor([slots] * 3, dtype=torch.int32, device=DEV)
    near, far = ([torch.zeros(3, 3, D, device=DEV) for _ in range(2)] for _ in range(2))
    B.evlnGatherKeys(handle, B.gather_params("f32", 3, D, CAP, 3, THETA), 3, kept, None, *stores, None, *far)
    small = torch.arange(3, dtype=torch.int32, device=DEV).repeat(3, 1)
    B.evlnGatherKeys(handle, B.gather_params("f32", 3, D, 3, 3, THETA), 3, small, None, *rows, None, *near)
    assert torch.equal(far[0], near[0]) and torch.equal(far[1], near[1])
    ref = np.stack([co.rotate(f64(rows[0, h])[:, None], np.arange(3), THETA)[:, 0] for h in range(3)])
    assert np.abs(f64(far[0]) - ref).max() <= 2.0 ** -21
