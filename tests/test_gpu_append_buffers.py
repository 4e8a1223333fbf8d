"""Appends with norms and into the 8-bit cache: rotated queries over the new tokens, refused or in place."""
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


def _calls(handle, x, pools):
    """Append of q, k, v with the queries to q_rot, by each of the three calls."""
    norm = B.head_norm(None, None, 1e-6)
    n, hq, hkv = x.total, x.hq, x.hkv
    step = B.step_params("bf16", hq, hkv, D, x.lens[0], n, x.lens[0] + n, 1e6)
    cache = [torch.zeros(hkv, x.lens[0] + n, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    return [lambda q, k, v, to: B.evlnNormRopeAppend(handle, step, norm, q, k, v, to, *cache),
            lambda q, k, v, to: B.evlnPagedNormRopeAppend(handle, x.params(), norm, q, k, v, x.lens, x.offs, x.table, to, *pools),
            lambda q, k, v, to: B.evlnPaged8RopeAppend(handle, x.params(), norm, q, k, v, x.lens, x.offs, x.table, to, *x.codes, *x.scales)]


def _case(handle, n, hq, hkv):
    x = Batch(handle, [100], [n], hq, hkv, seed=n)
    pools = [torch.zeros(x.pages, hkv, 64, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    return x, _calls(handle, x, pools)


@pytest.mark.parametrize("which", range(3))
def test_rotated_queries_over_the_new_tokens_are_refused(handle, which):
    x, calls = _case(handle, 5, 8, 2)
    rows = torch.randn(5, 12, D, generator=x.g).bfloat16().to(DEV)
    before = rows.clone()
    views = rows[:, :8], rows[:, 8:10], rows[:, 10:]
    for to in (rows.view(-1)[:40 * D], rows.view(-1)[D:41 * D], rows.view(-1)[9 * D:49 * D]):
        with pytest.raises(B.EvlnError) as e:
            calls[which](*views, to)
        assert e.value.status == B.EVLN_INVALID_VALUE
    q, k, v = (t.contiguous() for t in views)
    for to in (q, k, v):
        with pytest.raises(B.EvlnError):
            calls[which](q, k, v, to)
    assert torch.equal(rows, before)


@pytest.mark.parametrize("which", range(3))
@pytest.mark.parametrize("n,hq,hkv,joined", [(1, 28, 4, True), (1, 28, 4, False), (300, 7, 1, False)])
def test_in_place_where_the_layouts_are_the_same(handle, which, n, hq, hkv, joined):
    x, calls = _case(handle, n, hq, hkv)
    views = x.tokens()
    q, k, v = views if joined else (t.contiguous() for t in views)
    apart = torch.empty(hkv, n * hq // hkv, D, dtype=torch.bfloat16, device=DEV)
    calls[which](q, k, v, apart)
    calls[which](q, k, v, q)
    assert torch.equal(q.reshape(-1), apart.view(-1))
