"""Norms with the append in fp32: as exact as the rotation without them, whose products and sums are formed in double."""
import numpy as np
import pytest
import torch

from oracle import cache_ops_oracle as co
from paper_2512_10310_b200 import binding as B
from tests.helpers import f64
from tests.test_gpu_head_norm import DEV, _expected, _grouped, _pair, _tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def handle():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    h = B.evlnCreate(0)
    yield h
    B.evlnDestroy(h)


def _near(got, ref, pair):
    # one rounding to float, and what double arithmetic loses before it: angles of 10^5 radians (2^-36 of them in double), a few of 2^-53
    bound = 2.0 ** -24 * np.abs(ref) + 2.0 ** -34 * pair
    worst = float((np.abs(f64(got) - ref) / (bound + 1e-300)).max(initial=0.0))
    assert worst <= 1.0, f"{worst:.2f} times the bound"


@pytest.mark.parametrize("hq,hkv,D,L,n,joined,table,weights", [
    (2, 1, 64, 256, 64, False, False, True), (12, 4, 128, 1, 33, True, True, True), (3, 3, 64, 0, 1, False, False, False),
    (28, 4, 128, 4292, 1, True, False, True), (28, 4, 128, 100000, 196, True, True, True), (64, 8, 128, 9, 700, False, False, False),
    (1, 1, 64, 5, 2000, False, True, True),
])
def test_one_rounding(handle, hq, hkv, D, L, n, joined, table, weights):
    g = torch.Generator().manual_seed(hq + 7 * L + n)
    theta, eps, cap = 1.0e6, 1e-5, L + n
    q, k, v = _tokens(g, "f32", n, hq, hkv, D, joined)
    wq, wk = ((1.0 + 0.3 * torch.randn(D, generator=g)).to(DEV) if weights else None for _ in range(2))
    kc, vc = (torch.zeros(hkv, cap, D, device=DEV) for _ in range(2))
    rope = {}
    if table:
        t = torch.empty(B.evlnRopeTableBytes(D, n), dtype=torch.uint8, device=DEV)
        B.evlnRopeTable(handle, D, theta, L, n, t)
        rope = dict(rope_table=t, rope_table_first_pos=L, rope_table_count=n)
    p = B.step_params("f32", hq, hkv, D, L, n, cap, theta, **rope)
    q_rot = torch.empty(hkv, n * (hq // hkv), D, device=DEV)
    B.evlnNormRopeAppend(handle, p, B.head_norm(wq, wk, eps), q, k, v, q_rot, kc, vc)
    eps = float(np.float32(eps))
    rq, rk, pq, pk = _expected(q, k, None if wq is None else f64(wq), None if wk is None else f64(wk), eps, np.arange(L, L + n), theta)
    _near(q_rot, _grouped(rq, hkv), _grouped(pq, hkv))
    _near(kc[:, L:].transpose(0, 1), rk, pk)
    assert torch.equal(vc[:, L:].transpose(0, 1), v)


@pytest.mark.parametrize("size", [1e-30, 1e-20, 1e20, 1e30])
def test_heads_whose_squares_leave_the_range_of_floats(handle, size):
    g = torch.Generator().manual_seed(4)
    x = [(size * torch.randn(5, h, 128, generator=g)).to(DEV) for h in (6, 2, 2)]
    kc, vc = (torch.zeros(2, 9, 128, device=DEV) for _ in range(2))
    q_rot = torch.empty(2, 15, 128, device=DEV)
    B.evlnNormRopeAppend(handle, B.step_params("f32", 6, 2, 128, 4, 5, 9, 1e4), B.head_norm(None, None, 0.0), *x, q_rot, kc, vc)
    yq, yk = co.rms_norm(f64(x[0]), None, 0.0), co.rms_norm(f64(x[1]), None, 0.0)
    _near(q_rot, _grouped(co.rotate(yq, np.arange(4, 9), 1e4), 2), _grouped(_pair(yq), 2))
    _near(kc[:, 4:].transpose(0, 1), co.rotate(yk, np.arange(4, 9), 1e4), _pair(yk))
