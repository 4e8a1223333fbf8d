"""Eviction by attention weight (evlnKeyWeights, evlnSelectKeys, evlnGatherKeys) against fp64."""
import numpy as np
import pytest
import torch

from oracle import cache_ops_oracle as co
from paper_2512_10310_b200 import binding as B
from tests.helpers import f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# A weight exp(s - lse): scores in fp32 from D products, off by at most D 2^-24 of their sizes' sum (under 16 here, D <= 128), and an
# exponential good to 2^-21: all relative to the weight.  Sums of positive terms keep that.
WEIGHT_ERROR = 2.0 ** -13


@pytest.fixture(scope="module")
def handle():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    h = B.evlnCreate(0)
    yield h
    B.evlnDestroy(h)


def _weights_case(dtype, hq, hkv, D, L, n, cap, seed, scale):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(n, hq, D, generator=g).to(DTYPES[dtype])
    k = torch.randn(hkv, cap, D, generator=g).to(DTYPES[dtype])
    k[:, L + n:] = float("nan")                                  # nothing behind the last key is looked at
    G = hq // hkv
    q_rot = q.view(n, hkv, G, D).permute(1, 0, 2, 3).reshape(hkv, n * G, D).contiguous()
    keys = f64(k[:, :L + n]).transpose(1, 0, 2)
    lse = co.attention(f64(q), keys, np.zeros_like(keys), L, scale)[1].astype(np.float32)
    weights = torch.rand(hkv, cap, generator=g)
    weights[:, L:] = float("nan")
    return q, q_rot.to(DEV), k.to(DEV), keys, torch.from_numpy(lse).to(DEV), weights.to(DEV)


@pytest.mark.parametrize("dtype,hq,hkv,D,L,n,decay,scale", [
    ("bf16", 28, 4, 128, 4096, 1, 1.0, 0.0),        # a decoded token: whole tiles in turn
    ("bf16", 28, 4, 128, 500, 196, 0.9, 0.0),       # few tiles: chunks dealt to a cluster
    ("bf16", 28, 4, 128, 3000, 40, 1.0, 0.0),
    ("bf16", 8, 1, 128, 20000, 33, 0.5, 0.0),       # more tiles than SMs, several chunks each
    ("bf16", 64, 8, 128, 2500, 1, 0.0, 0.0),
    ("bf16", 2, 1, 64, 0, 1, 1.0, 0.0),             # one key
    ("bf16", 2, 1, 64, 0, 300, 1.0, 0.3),           # an empty cache: every key has its own rows
    ("bf16", 6, 2, 64, 127, 129, 1.0, 0.0),
    ("bf16", 5, 5, 128, 128, 128, 0.7, 0.05),
    ("bf16", 28, 4, 128, 100, 196, 1.0, 0.0),       # most tiles have keys that only some rows see
    ("bf16", 16, 2, 128, 30000, 17, 1.0, 0.0),      # three chunks of a tile, the last one short
    ("bf16", 16, 1, 64, 20000, 9, 0.5, 0.0),        # two chunks, several tiles a CTA
    ("bf16", 4, 4, 64, 9000, 127, 1.0, 0.0),        # one chunk of 127 rows
    ("bf16", 4, 4, 128, 9000, 128, 1.0, 0.0),       # one whole chunk, tiles in turn
    ("f32", 2, 1, 64, 256, 64, 0.9, 0.0),
    ("f32", 28, 4, 128, 300, 7, 1.0, 0.0),
    ("f32", 3, 3, 128, 0, 1, 1.0, 0.0),
    ("f32", 4, 2, 64, 1000, 130, 0.0, 0.2),
    ("f32", 28, 4, 128, 4096, 5, 1.0, 0.0),         # 35 rows as tiles of keys and rows
    ("f32", 64, 8, 128, 2000, 50, 0.9, 0.0),        # ... several chunks, the last one short, a tile that only some rows see
    ("f32", 12, 1, 128, 15000, 30, 1.0, 0.0),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_key_weights(handle, dtype, hq, hkv, D, L, n, decay, scale, in_place):
    cap = L + n + 5
    q, q_rot, k, keys, lse, weights = _weights_case(dtype, hq, hkv, D, L, n, cap, L + n + hq, scale or D ** -0.5)
    ref = co.key_weights(f64(q), keys, f64(lse), L, decay, f64(weights), scale or D ** -0.5)
    out = weights.clone() if in_place else torch.full_like(weights, -1.0)
    p = B.step_params(dtype, hq, hkv, D, L, n, cap, 1e6, scale)
    B.evlnKeyWeights(handle, p, q_rot, k, lse, decay, out if in_place else weights, out)
    assert B.evlnGetDeviceStatus(handle) == 0
    got = f64(out)
    worst = float((np.abs(got[:, :L + n] - ref) / (WEIGHT_ERROR * ref + 1e-30)).max())
    assert worst <= 1.0, f"{worst:.2f} times the bound"
    assert np.isnan(got[:, L + n:]).all() if in_place else (got[:, L + n:] == -1.0).all()
    again = weights.clone()
    B.evlnKeyWeights(handle, p, q_rot, k, lse, decay, weights, again)
    assert torch.equal(again[:, :L + n], out[:, :L + n])


def test_key_weights_sum_to_the_number_of_queries(handle):
    q, q_rot, k, keys, lse, weights = _weights_case("bf16", 28, 4, 128, 777, 50, 900, 3, 128 ** -0.5)
    out = torch.zeros_like(weights)
    p = B.step_params("bf16", 28, 4, 128, 777, 50, 900, 1e6)
    B.evlnKeyWeights(handle, p, q_rot, k, lse, 0.0, torch.zeros_like(weights), out)
    assert np.abs(f64(out).sum(1) - 7 * 50).max() < 7 * 50 * WEIGHT_ERROR


def _select(handle, w, num_keys, budget, sinks, recent):
    hkv, cap = w.shape
    p = B.gather_params("bf16", hkv, 128, cap, cap, 1e6)
    kept = torch.full((hkv, min(budget, num_keys) + 1), -7, dtype=torch.int32, device=DEV).view(-1)
    B.evlnSelectKeys(handle, p, w, num_keys, budget, sinks, recent, kept)
    count = hkv * min(budget, num_keys)
    assert bool((kept[count:] == -7).all())
    return kept[:count].view(hkv, -1)


@pytest.mark.parametrize("hkv,cap,num_keys,budget,sinks,recent", [
    (4, 20660, 20656, 4096, 256, 196), (1, 1, 1, 1, 0, 0), (2, 9, 7, 3, 1, 1), (2, 9, 7, 3, 2, 1), (3, 2050, 2049, 2048, 0, 0), (3, 2050, 2049, 1, 0, 0),
    (2, 5000, 5000, 777, 0, 100), (2, 100, 60, 80, 3, 3), (2, 100, 60, 60, 30, 30), (8, 65000, 65000, 1000, 4, 32), (1, 50000, 49153, 25000, 0, 0),
])
@pytest.mark.parametrize("kind", ["spread", "ties", "zeros"])
def test_select(handle, hkv, cap, num_keys, budget, sinks, recent, kind):
    g = torch.Generator().manual_seed(num_keys + budget)
    w = torch.exp(3.0 * torch.randn(hkv, cap, generator=g))
    if kind == "ties":
        w = torch.round(torch.rand(hkv, cap, generator=g) * 4) / 4
    elif kind == "zeros":
        w.zero_()
        w[:, ::3] = -0.0
    w[:, num_keys:] = 1e30                                        # not among the keys
    got = _select(handle, w.to(DEV), num_keys, budget, sinks, recent)
    assert np.array_equal(got.cpu().numpy(), co.select_keys(f64(w), num_keys, budget, sinks, recent))


def test_select_of_weights_that_are_not_numbers(handle):
    w = torch.tensor([[float("nan"), 1.0, float("-inf"), float("inf"), -2.0, float("nan"), 0.0, -0.0, 1e-45, 5.0]])
    for budget in range(1, 10):
        got = _select(handle, w.to(DEV), 10, budget, 0, 0)
        assert np.array_equal(got.cpu().numpy(), co.select_keys(f64(w), 10, budget, 0, 0)), budget


@pytest.mark.parametrize("dtype,hkv,D,store,work,kept,rotate,table,with_weights", [
    ("bf16", 4, 128, 3000, 700, 691, True, False, True), ("bf16", 4, 128, 3000, 700, 700, True, True, False), ("bf16", 1, 64, 50, 10, 1, True, False, True),
    ("f32", 2, 64, 333, 77, 77, True, True, True), ("f32", 8, 128, 400, 200, 199, False, False, True), ("bf16", 3, 64, 90, 90, 90, False, False, False),
])
def test_gather(handle, dtype, hkv, D, store, work, kept, rotate, table, with_weights):
    g = torch.Generator().manual_seed(store + kept)
    k, v = (torch.randn(hkv, store, D, generator=g).to(DTYPES[dtype]).to(DEV) for _ in range(2))
    w = torch.rand(hkv, store, generator=g).to(DEV)
    at = torch.stack([torch.randperm(store, generator=g)[:kept] for _ in range(hkv)]).to(torch.int32)
    kw, vw = (torch.full((hkv, work, D), 7.0, dtype=DTYPES[dtype], device=DEV) for _ in range(2))
    ww = torch.full((hkv, work), -1.0, device=DEV)
    rope = {}
    if table:
        t = torch.empty(B.evlnRopeTableBytes(D, kept), dtype=torch.uint8, device=DEV)
        B.evlnRopeTable(handle, D, 1e6, 0, kept, t)
        rope = dict(rope_table=t, rope_table_first_pos=0, rope_table_count=kept)
    p = B.gather_params(dtype, hkv, D, store, work, 1e6, **rope)
    B.evlnGatherKeys(handle, p, kept, at.to(DEV), w if with_weights else None, k, v, ww if with_weights else None, kw, vw, rotate)
    for h in range(hkv):
        rows = at[h].long().to(DEV)
        assert torch.equal(vw[h, :kept], v[h, rows])
        if rotate:
            ref = co.rotate(f64(k[h, rows])[:, None], np.arange(kept), 1e6)[:, 0]
            half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
            size = np.abs(f64(k[h, rows])).max(-1, keepdims=True)
            assert (np.abs(f64(kw[h, :kept]) - ref) <= half * np.abs(ref) + 2.0 ** -23 * size).all()
        else:
            assert torch.equal(kw[h, :kept], k[h, rows])
        if with_weights:
            assert torch.equal(ww[h, :kept], w[h, rows])
    assert bool((kw[:, kept:] == 7.0).all()) and bool((vw[:, kept:] == 7.0).all()) and bool((ww[:, kept if with_weights else 0:] == -1.0).all())


def test_gather_as_the_frame_sampler_lays_out(handle):
    # the same slots for every head: the bits of evlnGatherRope
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(4, 500, 128, generator=g).bfloat16().to(DEV) for _ in range(2))
    p = B.gather_params("bf16", 4, 128, 500, 300, 1e6)
    a = [torch.zeros(4, 300, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    b = [torch.zeros(4, 300, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    B.evlnGatherRope(handle, p, [0, 200], [64, 200], k, v, *a)
    at = torch.cat([torch.arange(64), torch.arange(200, 400)]).to(torch.int32).repeat(4, 1).to(DEV)
    B.evlnGatherKeys(handle, p, 264, at, None, k, v, None, *b)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_slots_outside_the_store_give_zeros(handle):
    k = torch.ones(1, 20, 64, device=DEV)
    p = B.gather_params("f32", 1, 64, 20, 5, 1e4)
    at = torch.tensor([[3, -1, 20, 2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device=DEV)
    kw, vw, ww = torch.full((1, 5, 64), 7.0, device=DEV), torch.full((1, 5, 64), 7.0, device=DEV), torch.full((1, 5), 7.0, device=DEV)
    B.evlnGatherKeys(handle, p, 5, at, torch.ones(1, 20, device=DEV), k, k, ww, kw, vw)
    assert bool((kw[0, 0] != 0).any()) and bool((kw[0, 1:] == 0).all()) and bool((vw[0, 1:] == 0).all()) and ww[0].tolist() == [1.0, 0.0, 0.0, 0.0, 0.0]


def test_a_round_of_eviction_as_it_is_used(handle):
    """A frame attends, its weights are added up, the cache is cut to a budget and the next step runs on what is left: against fp64."""
    hq, hkv, D, L, n, budget, theta = 14, 2, 128, 600, 40, 200, 1e6
    G, cap = hq // hkv, L + n
    g = torch.Generator().manual_seed(6)
    raw_k, raw_v = (torch.randn(hkv, cap, D, generator=g).bfloat16().to(DEV) for _ in range(2))
    # the working cache: all raw keys turned at their places
    every = torch.arange(L, dtype=torch.int32).repeat(hkv, 1).to(DEV)
    kw, vw = (torch.zeros(hkv, cap, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    p_all = B.gather_params("bf16", hkv, D, cap, cap, theta)
    B.evlnGatherKeys(handle, p_all, L, every, None, raw_k, raw_v, None, kw, vw)
    q = torch.randn(n, hq, D, generator=g).bfloat16().to(DEV)
    k_new, v_new = (t[:, L:].transpose(0, 1).contiguous() for t in (raw_k, raw_v))
    p = B.step_params("bf16", hq, hkv, D, L, n, cap, theta)
    q_rot = torch.empty(B.evlnStepQRotSize(handle, p), dtype=torch.uint8, device=DEV)
    ws = torch.empty(B.evlnStepWorkspaceSize(handle, p), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty(n, hq, D, dtype=torch.bfloat16, device=DEV), torch.empty(n, hq, device=DEV)
    B.evlnStep(handle, p, q, k_new, v_new, q_rot, kw, vw, ws, out, lse)
    weights = torch.zeros(hkv, cap, device=DEV)
    B.evlnKeyWeights(handle, p, q_rot, kw, lse, 1.0, weights, weights)
    kept = torch.empty(hkv, budget, dtype=torch.int32, device=DEV)
    B.evlnSelectKeys(handle, p_all, weights, cap, budget, 4, n, kept)
    cut_k, cut_v = (torch.zeros(hkv, budget + 1, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    cut_w = torch.zeros(hkv, budget + 1, device=DEV)
    p_cut = B.gather_params("bf16", hkv, D, cap, budget + 1, theta)
    B.evlnGatherKeys(handle, p_cut, budget, kept, weights, raw_k, raw_v, cut_w, cut_k, cut_v)
    qq = f64(q_rot[:n * hq * D * 2].view(torch.bfloat16)).reshape(hkv, n, G, D).transpose(1, 0, 2, 3).reshape(n, hq, D)
    ref_w = co.key_weights(qq, f64(kw).transpose(1, 0, 2), f64(lse), L, 1.0, np.zeros((hkv, cap)), D ** -0.5)
    assert np.abs(f64(weights) - ref_w).max() <= WEIGHT_ERROR * ref_w.max()
    assert np.array_equal(kept.cpu().numpy(), co.select_keys(f64(weights), cap, budget, 4, n))
    # one more token on the cut cache
    one = [torch.randn(1, h, D, generator=g).bfloat16().to(DEV) for h in (hq, hkv, hkv)]
    p1 = B.step_params("bf16", hq, hkv, D, budget, 1, budget + 1, theta)
    ws1 = torch.empty(max(16, B.evlnStepWorkspaceSize(handle, p1)), dtype=torch.uint8, device=DEV)
    out1 = torch.empty(1, hq, D, dtype=torch.bfloat16, device=DEV)
    q1 = torch.empty(B.evlnStepQRotSize(handle, p1), dtype=torch.uint8, device=DEV)
    B.evlnStep(handle, p1, *one, q1, cut_k, cut_v, ws1, out1)
    keys = np.stack([co.rotate(f64(raw_k[h, kept[h].long()])[:, None], np.arange(budget), theta)[:, 0] for h in range(hkv)], axis=1)
    vals = np.stack([f64(raw_v[h, kept[h].long()]) for h in range(hkv)], axis=1)
    keys = np.concatenate([keys, co.rotate(f64(one[1]), [budget], theta)])
    vals = np.concatenate([vals, f64(one[2])])
    ref, _, size = co.attention(co.rotate(f64(one[0]), [budget], theta), keys, vals, budget, D ** -0.5)
    # keys and queries rounded to bf16 (2^-8 each of scores that reach 4 or so), probabilities and output too
    assert (np.abs(f64(out1) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -5 * size).all()


def test_refusals(handle):
    D = 64
    p = B.step_params("f32", 2, 1, D, 10, 1, 16, 1e4)
    q, k = torch.zeros(2, D, device=DEV), torch.zeros(16, D, device=DEV)
    lse, w = torch.zeros(2, device=DEV), torch.zeros(40, device=DEV)

    def refused(status, call, *args):
        with pytest.raises(B.EvlnError) as e:
            call(handle, *args)
        assert e.value.status == status
    refused(B.EVLN_INVALID_VALUE, B.evlnKeyWeights, p, q, k, lse, -1.0, w, w)
    refused(B.EVLN_INVALID_VALUE, B.evlnKeyWeights, p, q, k, lse, float("nan"), w, w)
    refused(B.EVLN_INVALID_VALUE, B.evlnKeyWeights, p, q, None, lse, 1.0, w, w)
    refused(B.EVLN_INVALID_VALUE, B.evlnKeyWeights, p, q, k, lse, 1.0, w, w[8:])             # neither the same nor apart
    refused(B.EVLN_CACHE_FULL, B.evlnKeyWeights, B.step_params("f32", 2, 1, D, 16, 1, 16, 1e4), q, k, lse, 1.0, w, w)
    gp = B.gather_params("f32", 1, D, 16, 8, 1e4)
    kept = torch.zeros(16, dtype=torch.int32, device=DEV)
    refused(B.EVLN_INVALID_VALUE, B.evlnSelectKeys, gp, w, 17, 4, 0, 0, kept)
    refused(B.EVLN_INVALID_VALUE, B.evlnSelectKeys, gp, w, 16, 4, 3, 2, kept)
    refused(B.EVLN_INVALID_VALUE, B.evlnSelectKeys, gp, w, 16, 4, -1, 2, kept)
    refused(B.EVLN_INVALID_VALUE, B.evlnSelectKeys, gp, None, 16, 4, 0, 0, kept)
    B.evlnSelectKeys(handle, gp, w, 0, 4, 0, 0, kept)
    kw = torch.zeros(8, D, device=DEV)
    refused(B.EVLN_CACHE_FULL, B.evlnGatherKeys, gp, 9, kept, None, k, k, None, kw, kw)
    refused(B.EVLN_INVALID_VALUE, B.evlnGatherKeys, gp, 4, kept, w, k, k, None, kw, kw)
    refused(B.EVLN_INVALID_VALUE, B.evlnGatherKeys, gp, 4, kept, None, k, k, None, k[4:], kw)  # over the store
    refused(B.EVLN_INVALID_VALUE, B.evlnGatherKeys, gp, 4, None, None, k, k, None, kw, kw)
    short = B.gather_params("f32", 1, D, 16, 8, 1e4, rope_table=w, rope_table_first_pos=0, rope_table_count=3)
    refused(B.EVLN_INVALID_VALUE, B.evlnGatherKeys, short, 4, kept, None, k, k, None, kw, kw, True)
    B.evlnGatherKeys(handle, gp, 0, kept, None, k, k, None, kw, kw)
