"""The operators around the cache where offsets pass 32 bits, on several streams at once and as replayed graphs."""
import numpy as np
import pytest
import torch

from oracle import cache_ops_oracle as co
from paper_2512_10310_b200 import binding as B
from tests.helpers import f64
from tests.test_gpu_cache8 import D, DEV, EPS, THETA, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def handle():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    h = B.evlnCreate(0)
    yield h
    B.evlnDestroy(h)


def test_pages_far_into_the_pool(handle):
    """The same episodes on neighbouring pages and on pages spread over pools of 4.9 GB: the same codes, scales and rows."""
    near, far = (Batch(handle, [100, 70, 333], [1, 40, 3], 4, 1, seed=5) for _ in range(2))
    pages, stride = 600_000, 45_000                       # page i of the small pool is page (i + 1) * stride + 7
    codes = [torch.empty(pages, 1, 64, D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.full((pages, 1), float("nan"), device=DEV) for _ in range(2)]
    moved = [(i + 1) * stride + 7 for i in range(far.pages)]
    assert max(moved) < pages and max(moved) * 64 * D > 2 ** 32
    for a, b in zip(codes + scales, far.codes + far.scales):
        a[moved] = b
    far.rows = [[moved[p] for p in row] for row in far.rows]
    far.table = torch.tensor(far.rows, dtype=torch.int32, device=DEV)
    far.codes, far.scales, far.pages = codes, scales, pages
    for x in (near, far):
        x.fill_new()
    for a, b in zip(near.codes + near.scales, far.codes + far.scales):
        a, b = (t.nan_to_num(7.0) if t.is_floating_point() else t for t in (a, b[moved]))
        assert torch.equal(a, b)
    q_rot = near.q_rot()
    for a, b in zip(near.attend(q_rot), far.attend(q_rot)):          # (40 tokens of 4 heads: through the copy, whose softmax references may move differently)
        assert (a.float() - b.float()).abs().max() <= 2.0 ** -6 * a.float().abs().max()


def test_codes_far_into_the_pool(handle):
    near, far = (Batch(handle, [100, 333], [1, 3], 4, 1, seed=6) for _ in range(2))
    pages, stride = 600_000, 55_000
    moved = [(i + 1) * stride + 7 for i in range(far.pages)]
    assert max(moved) < pages and max(moved) * 64 * D > 2 ** 31
    big = [torch.empty(pages, 1, 64, D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.full((pages, 1), float("nan"), device=DEV) for _ in range(2)]
    for a, b in zip(big + scales, far.codes + far.scales):
        a[moved] = b
    far.table = torch.tensor([[moved[p] for p in row] for row in far.rows], dtype=torch.int32, device=DEV)
    far.codes, far.scales, far.pages = big, scales, pages
    for x in (near, far):
        x.fill_new()
    q_rot = near.q_rot()
    for a, b in zip(near.attend(q_rot), far.attend(q_rot)):
        assert torch.equal(a, b)


def test_a_cache_longer_than_32_bits(handle):
    """Two heads of 9 million slots (the second one starts behind 2^31 bytes and ends behind 2^32): append with norms, key weights and gather at the
    far end of the second head."""
    cap, n, L = 9_000_000, 3, 8_999_990
    g = torch.Generator().manual_seed(9)
    k, v = (torch.empty(2, cap, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    x = [torch.randn(n, h, D, generator=g).bfloat16().to(DEV) for h in (2, 2, 2)]
    q_rot = torch.empty(2, n, D, dtype=torch.bfloat16, device=DEV)
    B.evlnNormRopeAppend(handle, B.step_params("bf16", 2, 2, D, L, n, cap, THETA), B.head_norm(None, None, EPS), *x, q_rot, k, v)
    keys = co.rotate(co.rms_norm(f64(x[1]), None, EPS), np.arange(L, L + n), THETA)
    # a rounding to bf16 of numbers up to 16, and angles of 9 million radians in fp64 (2^-53 of them: 1e-9)
    assert np.abs(f64(k[:, L:L + n]).transpose(1, 0, 2) - keys).max() <= 2.0 ** -8 * 16
    assert torch.equal(v[:, L:L + n].transpose(0, 1), x[2])

    kept = torch.tensor([[0, 5], [L, L + n - 1]], dtype=torch.int32, device=DEV)
    k[0, [0, 5]] = 1.5
    v[0, [0, 5]] = -2.5
    kw, vw = (torch.empty(2, 2, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.evlnGatherKeys(handle, B.gather_params("bf16", 2, D, cap, 2, THETA), 2, kept, None, k, v, None, kw, vw, rotate=False)
    assert bool((kw[0] == 1.5).all()) and bool((vw[0] == -2.5).all())
    assert torch.equal(kw[1], k[1, [L, L + n - 1]]) and torch.equal(vw[1], v[1, [L, L + n - 1]])

    # 300 keys of both heads, whose rows lie 2.3 GB apart, against the same keys in a small cache
    small_k = torch.randn(2, 301, D, generator=g).bfloat16().to(DEV)
    k[:, :301] = small_k
    q = torch.randn(2, 1, D, generator=g).bfloat16().to(DEV)
    lse = torch.tensor([[3.0, 4.0]], device=DEV)
    w_far, w_near = torch.zeros(2, cap, device=DEV), torch.zeros(2, 301, device=DEV)
    B.evlnKeyWeights(handle, B.step_params("bf16", 2, 2, D, 300, 1, cap, THETA), q, k, lse, 1.0, w_far, w_far)
    B.evlnKeyWeights(handle, B.step_params("bf16", 2, 2, D, 300, 1, 301, THETA), q, small_k, lse, 1.0, w_near, w_near)
    assert torch.equal(w_far[:, :301], w_near) and not bool(w_far[:, 301:].any())


def test_two_streams_at_once(handle):
    """Two batches, each a chain of append and attention on a stream of its own, many times over: the results of the same alone."""
    a, b = Batch(handle, [4000, 100], [1, 1], 28, 4, seed=1), Batch(handle, [900], [30], 28, 4, seed=2)
    state = []
    for x in (a, b):
        q, k, v = (t.contiguous() for t in x.tokens())
        ws = torch.empty(B.evlnPaged8WorkspaceSize(handle, x.params(), x.lens, x.offs), dtype=torch.uint8, device=DEV)
        q_rot = torch.empty(4, x.total * 7, D, dtype=torch.bfloat16, device=DEV)
        out = torch.full((x.total, 28, D), float("nan"), dtype=torch.bfloat16, device=DEV)
        state.append((x, q, k, v, ws, q_rot, out))

    def step(x, q, k, v, ws, q_rot, out, stream):
        B.evlnPaged8RopeAppend(handle, x.params(), None, q, k, v, x.lens, x.offs, x.table, q_rot, *x.codes, *x.scales, stream=stream)
        B.evlnPaged8StepAttention(handle, x.params(), q_rot, *x.codes, *x.scales, x.lens, x.offs, x.table, ws, out, stream=stream)
    alone = []
    for s in state:
        step(*s, None)
        alone.append(s[-1].clone())
        s[-1].fill_(float("nan"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in state]
    for _ in range(20):
        for s, stream in zip(state, streams):
            step(*s, stream)
    torch.cuda.synchronize()
    assert B.evlnGetDeviceStatus(handle) == 0
    assert torch.equal(state[0][-1], alone[0])
    # (30 tokens go through the copy, whose softmax references may move differently: bf16 outputs a rounding or two apart)
    assert (state[1][-1].float() - alone[1].float()).abs().max() <= 2.0 ** -6 * alone[1].float().abs().max()


def test_norms_and_eviction_as_a_replayed_graph(handle):
    hq, hkv, L, n, budget = 14, 2, 700, 20, 300
    cap, g = 720, torch.Generator().manual_seed(3)
    x = [torch.randn(n, h, D, generator=g).bfloat16().to(DEV) for h in (hq, hkv, hkv)]
    weight = (1.0 + 0.2 * torch.randn(D, generator=g)).bfloat16().to(DEV)
    norm, p = B.head_norm(weight, weight, EPS), B.step_params("bf16", hq, hkv, D, L, n, cap, THETA)
    cache = [torch.randn(hkv, cap, D, generator=g).bfloat16().to(DEV) for _ in range(2)]
    lse = torch.full((n, hq), 8.0, device=DEV)
    start = torch.rand(hkv, cap, generator=g).to(DEV)
    gp = B.gather_params("bf16", hkv, D, cap, budget, THETA)

    def buffers():
        made = dict(q_rot=torch.empty(hkv, n * hq // hkv, D, dtype=torch.bfloat16, device=DEV), k=cache[0].clone(), v=cache[1].clone(), w=start.clone(),
                    kept=torch.empty(hkv, budget, dtype=torch.int32, device=DEV), ww=torch.empty(hkv, budget, device=DEV))
        return made | dict(kw=torch.empty(hkv, budget, D, dtype=torch.bfloat16, device=DEV), vw=torch.empty(hkv, budget, D, dtype=torch.bfloat16, device=DEV))

    def run(b):
        B.evlnNormRopeAppend(handle, p, norm, *x, b["q_rot"], b["k"], b["v"])
        B.evlnKeyWeights(handle, p, b["q_rot"], b["k"], lse, 0.5, start, b["w"])
        B.evlnSelectKeys(handle, gp, b["w"], L + n, budget, 4, n, b["kept"])
        B.evlnGatherKeys(handle, gp, budget, b["kept"], b["w"], b["k"], b["v"], b["ww"], b["kw"], b["vw"], rotate=True)
    eager, played = buffers(), buffers()
    run(eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(played)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run(played)
        for name in ("q_rot", "w", "kept", "ww", "kw", "vw"):
            played[name].fill_(3)
        for _ in range(3):
            graph.replay()
    torch.cuda.synchronize()
    assert B.evlnGetDeviceStatus(handle) == 0
    for name in eager:
        assert torch.equal(eager[name], played[name]), name
