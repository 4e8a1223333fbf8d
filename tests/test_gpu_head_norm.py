"""Norms of queries and keys in the append's pass (evlnNormRopeAppend, evlnPagedNormRopeAppend) against fp64."""
import numpy as np
import pytest
import torch

from oracle import cache_ops_oracle as co
from paper_2512_10310_b200 import binding as B
from tests.helpers import f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# rounding to the storage type: half a step of it, relative to the value
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
# what fp32 arithmetic before it may lose, relative to the larger of the pair that is turned: the sum of squares (fewer than 16
# roundings, halved by the root), root, quotient, two products with weights, cosine and sine, two products and a sum: under 16 of 2^-24
ARITHMETIC = 2.0 ** -20


@pytest.fixture(scope="module")
def handle():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    h = B.evlnCreate(0)
    yield h
    B.evlnDestroy(h)


def _tokens(g, dtype, total, hq, hkv, D, joined):
    """Queries, keys, values: views of rows of one buffer (strides), or tensors of their own; heads of very different sizes."""
    heads = hq + 2 * hkv
    x = torch.randn(total, heads, D, generator=g) * torch.exp(3.0 * torch.randn(1, heads, 1, generator=g))
    x = x.to(DTYPES[dtype])
    if joined:
        row = torch.zeros(total, heads * D + 16, dtype=x.dtype)
        row[:, :heads * D] = x.view(total, -1)
        row = row.to(DEV)
        x = row[:, :heads * D].unflatten(1, (heads, D))
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    x = x.to(DEV)
    return x[:, :hq].contiguous(), x[:, hq:hq + hkv].contiguous(), x[:, hq + hkv:].contiguous()


def _near(got, ref, dtype, pair):
    bound = HALF_STEP[dtype] * np.abs(ref) + ARITHMETIC * pair
    worst = float((np.abs(f64(got) - ref) / (bound + 1e-300)).max(initial=0.0))
    assert worst <= 1.0, f"{worst:.2f} times the bound"


def _pair(y):
    """The larger of the two channels that are turned together, for each channel."""
    half = y.shape[-1] // 2
    m = np.maximum(np.abs(y[..., :half]), np.abs(y[..., half:]))
    return np.concatenate([m, m], axis=-1) * 2.0


def _expected(q, k, wq, wk, eps, positions, theta):
    yq, yk = co.rms_norm(f64(q), wq, eps), co.rms_norm(f64(k), wk, eps)
    return co.rotate(yq, positions, theta), co.rotate(yk, positions, theta), _pair(yq), _pair(yk)


def _grouped(x, hkv):
    t, hq, D = x.shape
    return x.reshape(t, hkv, hq // hkv, D).transpose(1, 0, 2, 3).reshape(hkv, -1, D)


@pytest.mark.parametrize("dtype,hq,hkv,D,L,n,joined,table,weights", [
    ("bf16", 28, 4, 128, 4292, 1, True, True, True),
    ("bf16", 28, 4, 128, 37, 196, False, False, True),
    ("bf16", 64, 8, 128, 100000, 3, True, False, False),
    ("bf16", 2, 1, 64, 0, 5, True, True, True),
    ("bf16", 5, 5, 64, 7, 300, False, True, False),
    ("f32", 2, 1, 64, 256, 64, False, False, True),
    ("f32", 12, 4, 128, 1, 33, True, True, True),
    ("f32", 3, 3, 64, 0, 1, False, False, False),
])
def test_contiguous(handle, dtype, hq, hkv, D, L, n, joined, table, weights):
    g = torch.Generator().manual_seed(hq * 1000 + L + n)
    theta, eps, cap = 1.0e4 if dtype == "f32" else 1.0e6, 1e-5, L + n + 3
    q, k, v = _tokens(g, dtype, n, hq, hkv, D, joined)
    wq, wk = (((1.0 + 0.3 * torch.randn(D, generator=g)).to(DTYPES[dtype]).to(DEV)) if weights else None for _ in range(2))
    kc = torch.full((hkv, cap, D), 7.0, dtype=DTYPES[dtype], device=DEV)
    vc = torch.full((hkv, cap, D), -3.0, dtype=DTYPES[dtype], device=DEV)
    rope = {}
    if table:
        t = torch.empty(B.evlnRopeTableBytes(D, L + n), dtype=torch.uint8, device=DEV)
        B.evlnRopeTable(handle, D, theta, 0, L + n, t)
        rope = dict(rope_table=t, rope_table_first_pos=0, rope_table_count=L + n)
    p = B.step_params(dtype, hq, hkv, D, L, n, cap, theta, **rope)
    q_rot = torch.full((hkv, n * (hq // hkv) + 1, D), 5.0, dtype=DTYPES[dtype], device=DEV)
    flat = q_rot.view(-1)[:hkv * n * (hq // hkv) * D]
    B.evlnNormRopeAppend(handle, p, B.head_norm(wq, wk, eps), q, k, v, flat, kc, vc)
    rq, rk, pq, pk = _expected(q, k, None if wq is None else f64(wq), None if wk is None else f64(wk), eps, np.arange(L, L + n), theta)
    _near(flat.view(hkv, -1, D), _grouped(rq, hkv), dtype, _grouped(pq, hkv))
    _near(kc[:, L:L + n].transpose(0, 1), rk, dtype, pk)
    assert torch.equal(vc[:, L:L + n].transpose(0, 1), v)
    assert bool((kc[:, :L] == 7.0).all()) and bool((kc[:, L + n:] == 7.0).all()) and bool((vc[:, :L] == -3.0).all()) and bool((vc[:, L + n:] == -3.0).all())
    assert bool((q_rot.view(-1)[flat.numel():] == 5.0).all())


@pytest.mark.parametrize("lens,news,hq,hkv,joined,table", [
    ([0, 63, 64, 333, 1000], [70, 1, 129, 0, 37], 28, 4, True, True),
    ([5], [1], 64, 8, False, False),
    ([2000] * 9, [64] * 9, 2, 1, True, False),
])
def test_paged(handle, lens, news, hq, hkv, joined, table):
    g = torch.Generator().manual_seed(len(lens) + hq)
    D, P, eps, theta = 128, 64, 1e-6, 1.0e6
    offs = np.concatenate([[0], np.cumsum(news)]).tolist()
    total = offs[-1]
    need = [(L + n + P - 1) // P for L, n in zip(lens, news)]
    order = torch.randperm(sum(need) + 2, generator=g).tolist()
    width = max(need) + 1
    rows, at = [], 0
    for c in need:
        rows.append(order[at:at + c] + [0] * (width - c))
        at += c
    tab = torch.tensor(rows, dtype=torch.int32, device=DEV)
    pools = [torch.full((len(order), hkv, P, D), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    q, k, v = _tokens(g, "bf16", total, hq, hkv, D, joined)
    wq, wk = ((1.0 + 0.3 * torch.randn(D, generator=g)).bfloat16().to(DEV) for _ in range(2))
    rope = {}
    if table:
        count = max(L + n for L, n in zip(lens, news))
        t = torch.empty(B.evlnRopeTableBytes(D, count), dtype=torch.uint8, device=DEV)
        B.evlnRopeTable(handle, D, theta, 0, count, t)
        rope = dict(rope_table=t, rope_table_first_pos=0, rope_table_count=count)
    p = B.paged_params(hq, hkv, D, len(lens), P, len(order), width, theta, **rope)
    q_rot = torch.empty(hkv, total * (hq // hkv), D, dtype=torch.bfloat16, device=DEV)
    B.evlnPagedNormRopeAppend(handle, p, B.head_norm(wq, wk, eps), q, k, v, lens, offs, tab, q_rot, *pools)
    positions = np.concatenate([np.arange(L, L + n) for L, n in zip(lens, news)])
    rq, rk, pq, pk = _expected(q, k, f64(wq), f64(wk), eps, positions, theta)
    _near(q_rot, _grouped(rq, hkv), "bf16", _grouped(pq, hkv))
    touched = torch.zeros(len(order), P, dtype=torch.bool)
    cleared = torch.zeros(len(order), P, dtype=torch.bool)
    for b, (L, n) in enumerate(zip(lens, news)):
        for i in range(n):
            page, slot = rows[b][(L + i) // P], (L + i) % P
            touched[page, slot] = True
            _near(pools[0][page, :, slot], rk[offs[b] + i], "bf16", pk[offs[b] + i])
            assert torch.equal(pools[1][page, :, slot], v[offs[b] + i])
        if n and (L + n) % P:
            cleared[rows[b][(L + n) // P], (L + n) % P:] = True
    assert bool((pools[0].cpu().transpose(1, 2)[~touched] == 7.0).all())
    assert bool((pools[1].cpu().transpose(1, 2)[cleared] == 0.0).all())
    assert bool((pools[1].cpu().transpose(1, 2)[~touched & ~cleared] == 7.0).all())


def test_in_place_for_one_token_and_heads_of_zeros(handle):
    g = torch.Generator().manual_seed(2)
    hq, hkv, D, L = 28, 4, 128, 11
    q, k, v = _tokens(g, "bf16", 1, hq, hkv, D, False)
    q[0, 3] = 0.0
    k[0, 1] = 0.0
    kc, vc = (torch.zeros(hkv, L + 1, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    p = B.step_params("bf16", hq, hkv, D, L, 1, L + 1, 1.0e6)
    rq, rk, pq, pk = _expected(q, k, None, None, 1e-6, [L], 1.0e6)
    B.evlnNormRopeAppend(handle, p, B.head_norm(None, None, 1e-6), q, k, v, q, kc, vc)       # q_rot over q_new
    _near(q, rq, "bf16", pq)
    _near(kc[:, L:].transpose(0, 1), rk, "bf16", pk)
    assert bool((q[0, 3] == 0).all()) and bool((kc[1, L] == 0).all())


def test_refusals(handle):
    hq, hkv, D = 4, 2, 128
    x = torch.zeros(2, 16, D, dtype=torch.bfloat16, device=DEV)
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:8]
    kc = torch.zeros(hkv, 8, D, dtype=torch.bfloat16, device=DEV)
    q_rot = torch.zeros(hkv, 4, D, dtype=torch.bfloat16, device=DEV)
    p = B.step_params("bf16", hq, hkv, D, 0, 2, 8, 1e6)
    norm = B.head_norm(None, None, 1e-6)

    def refused(status, *args, **kw):
        with pytest.raises(B.EvlnError) as e:
            B.evlnNormRopeAppend(handle, *args, **kw)
        assert e.value.status == status
    refused(B.EVLN_INVALID_VALUE, p, None, q, k, v, q_rot, kc, kc)
    refused(B.EVLN_INVALID_VALUE, p, B.head_norm(None, None, -1.0), q, k, v, q_rot, kc, kc)
    refused(B.EVLN_INVALID_VALUE, p, B.head_norm(None, None, float("nan")), q, k, v, q_rot, kc, kc)
    refused(B.EVLN_INVALID_VALUE, p, B.head_norm(x.data_ptr() + 2, None, 1e-6), q, k, v, q_rot, kc, kc)
    refused(B.EVLN_INVALID_VALUE, p, norm, None, k, v, q_rot, kc, kc, strides=(512, 256, 256))
    refused(B.EVLN_INVALID_VALUE, p, norm, q, k, v, q_rot, kc, kc, strides=(511, 256, 256))
    refused(B.EVLN_INVALID_VALUE, p, norm, q, k, v, q_rot, kc, kc, strides=(516, 256, 256))
    refused(B.EVLN_CACHE_FULL, B.step_params("bf16", hq, hkv, D, 7, 2, 8, 1e6), norm, q, k, v, q_rot, kc, kc)
    refused(B.EVLN_NOT_SUPPORTED, B.step_params("bf16", hq, hkv, 96, 0, 2, 8, 1e6), norm, q, k, v, q_rot, kc, kc)
    B.evlnNormRopeAppend(handle, B.step_params("bf16", hq, hkv, D, 8, 0, 8, 1e6), norm, q, k, v, q_rot, kc, kc)     # no tokens: nothing to do
