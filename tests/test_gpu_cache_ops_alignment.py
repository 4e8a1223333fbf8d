"""Float and int arrays (log-sum-exps, page tables, scales, weights, slots) that are not aligned to their elements: refused, nothing launched."""
import pytest
import torch

from paper_2512_10310_b200 import binding as B
from tests.test_gpu_cache8 import D, DEV, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def handle():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    h = B.evlnCreate(0)
    yield h
    B.evlnDestroy(h)


def _each_refused(handle, call, args, places, **kw):
    for i in places:
        with pytest.raises(B.EvlnError) as e:
            call(handle, *[a.data_ptr() + 2 if j == i else a for j, a in enumerate(args)], **kw)
        assert e.value.status == B.EVLN_INVALID_VALUE, i


def test_arrays_off_their_alignment_are_refused(handle):
    x = Batch(handle, [70], [1], 4, 2, seed=1)
    q, k, v = (t.contiguous() for t in x.tokens())
    q_rot = torch.empty(2, 2, D, dtype=torch.bfloat16, device=DEV)
    pools = [torch.zeros(x.pages, 2, 64, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    _each_refused(handle, B.evlnPagedNormRopeAppend, [x.params(), B.head_norm(None, None, 1e-6), q, k, v, x.lens, x.offs, x.table, q_rot, *pools], [7])
    append = [x.params(), None, q, k, v, x.lens, x.offs, x.table, q_rot, *x.codes, *x.scales]
    _each_refused(handle, B.evlnPaged8RopeAppend, append, [7, 11, 12])
    B.evlnPaged8RopeAppend(handle, *append)
    ws = torch.empty(B.evlnPaged8WorkspaceSize(handle, x.params(), x.lens, x.offs), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty(1, 4, D, dtype=torch.bfloat16, device=DEV), torch.empty(1, 4, device=DEV)
    _each_refused(handle, B.evlnPaged8StepAttention, [x.params(), q_rot, *x.codes, *x.scales, x.lens, x.offs, x.table, ws, out, lse], [4, 5, 8, 11])

    p = B.step_params("f32", 2, 1, 64, 10, 1, 16, 1e4)
    a, c = torch.zeros(2, 64, device=DEV), torch.zeros(16, 64, device=DEV)
    w, other = torch.zeros(64, device=DEV), torch.zeros(64, device=DEV)
    _each_refused(handle, B.evlnKeyWeights, [p, a, c, lse, 1.0, w, other], [3, 5, 6])
    gp = B.gather_params("f32", 1, 64, 16, 8, 1e4)
    kept = torch.zeros(16, dtype=torch.int32, device=DEV)
    _each_refused(handle, B.evlnSelectKeys, [gp, w, 16, 4, 0, 0, kept], [1, 6])
    work = [torch.zeros(8, 64, device=DEV) for _ in range(2)]
    _each_refused(handle, B.evlnGatherKeys, [gp, 4, kept, w, c, c, other, *work], [2, 3, 6])


def test_arrays_of_the_step_and_paged_calls_off_their_alignment_are_refused(handle):
    x = Batch(handle, [70], [1], 4, 2, seed=1)
    q, k, v = (t.contiguous() for t in x.tokens())
    q_rot, out = torch.empty(2, 2, D, dtype=torch.bfloat16, device=DEV), torch.empty(1, 4, D, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(1, 8, device=DEV)
    pools = [torch.zeros(x.pages, 2, 64, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    _each_refused(handle, B.evlnPagedRopeAppend, [x.params(), q, k, v, x.lens, x.offs, x.table, q_rot, *pools], [6])
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    _each_refused(handle, B.evlnPagedStepAttention, [x.params(), q_rot, *pools, x.lens, x.offs, x.table, ws], [6])
    _each_refused(handle, B.evlnPagedStepCombine, [x.params(), ws, x.lens, x.offs, out, lse], [5])
    p = B.step_params("bf16", 4, 2, D, 70, 1, 71, 1e6)
    cache = [torch.zeros(2, 71, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    _each_refused(handle, B.evlnStepCombine, [p, ws, out, lse], [3])
    _each_refused(handle, B.evlnStep, [p, q, k, v, q_rot, *cache, ws, out, lse], [9])
    with pytest.raises(B.EvlnError):
        B.evlnStepAttentionNoAlloc(p, q_rot, *cache, out, lse.data_ptr() + 2)


def test_a_float_array_may_start_anywhere_else(handle):
    """Weights and log-sum-exps that start 4 bytes behind a 16-byte border: the same results."""
    g = torch.Generator().manual_seed(1)
    p = B.step_params("f32", 2, 1, 64, 10, 1, 16, 1e4)
    q, k = torch.randn(2, 64, generator=g).to(DEV), torch.randn(16, 64, generator=g).to(DEV)
    got = []
    for shift in (0, 1):
        lse, w = torch.ones(2 + shift, device=DEV)[shift:], torch.full((16 + shift,), 0.5, device=DEV)[shift:]
        kept = torch.full((4 + shift,), -1, dtype=torch.int32, device=DEV)[shift:]
        B.evlnKeyWeights(handle, p, q, k, lse, 1.0, w, w)
        B.evlnSelectKeys(handle, B.gather_params("f32", 1, 64, 16, 8, 1e4), w, 11, 4, 1, 1, kept)
        got.append((w, kept))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
