"""Attention over the 8-bit cache (evlnPaged8StepAttention): outputs over the queries, and keys cut into splits on the way through the copy."""
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


def _into(x, q_rot, out, lse=None):
    ws = torch.empty(B.evlnPaged8WorkspaceSize(x.h, x.params(), x.lens, x.offs), dtype=torch.uint8, device=DEV)
    B.evlnPaged8StepAttention(x.h, x.params(), q_rot, *x.codes, *x.scales, x.lens, x.offs, x.table, ws, out, lse)


@pytest.mark.parametrize("lens,news,hq,hkv", [([3000], [2], 28, 4), ([100, 700], [1, 1], 28, 4), ([300], [40], 28, 4)])
def test_outputs_over_the_queries_are_refused(handle, lens, news, hq, hkv):
    x = Batch(handle, lens, news, hq, hkv, seed=1)
    x.fill_new()
    size = x.total * hq * D
    room = torch.zeros(2 * size, dtype=torch.bfloat16, device=DEV)
    before = room.clone()
    for at, lse in ((0, None), (8, None), (size - 8, None), (size, room)):
        with pytest.raises(B.EvlnError) as e:
            _into(x, room[:size], room[at:at + size], lse)
        assert e.value.status == B.EVLN_INVALID_VALUE
    assert torch.equal(room, before)
    _into(x, room[:size], room[size:])


@pytest.mark.parametrize("lens,news,hq,hkv", [([9000], [1], 28, 4), ([9000, 20, 333], [1, 2, 3], 7, 1), ([70], [40], 7, 1), ([200], [1], 160, 2)])
def test_in_place_where_the_layouts_are_the_same(handle, lens, news, hq, hkv):
    x = Batch(handle, lens, news, hq, hkv, seed=2)
    x.fill_new()
    q_rot = x.q_rot()
    apart, lse = x.attend(q_rot)
    x.check(q_rot, apart, lse)
    over = q_rot.clone()
    _into(x, over, over)
    if x.kind == "codes":
        assert torch.equal(over.view(-1), apart.view(-1))
    else:
        x.check(q_rot, over.view(apart.shape), lse)


@pytest.mark.parametrize("tiles", [1, 3])
def test_splits_on_the_way_through_the_copy(handle, tiles):
    """kv_chunk_tiles cuts the keys of the copy: joined as the bf16 calls join them; on the codes it is not looked at."""
    for news in ([70, 1, 0, 196], [2, 1, 0, 3]):
        x = Batch(handle, [0, 63, 64, 1000], news, 28, 4, seed=7)
        x.fill_new()
        q_rot, plain = x.q_rot(), x.params
        x.params = lambda **kw: plain(kv_chunk_tiles=tiles, **kw)
        out, lse = x.attend(q_rot)
        x.check(q_rot, out, lse)
