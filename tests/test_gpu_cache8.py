"""The paged cache in 8 bits (evlnPaged8RopeAppend, evlnPaged8StepAttention) against fp64."""
import numpy as np
import pytest
import torch

from oracle import cache_ops_oracle as co
from paper_2512_10310_b200 import binding as B
from tests.helpers import f64

pytestmark = pytest.mark.gpu
DEV, P, D, THETA, EPS = "cuda:0", 64, 128, 1.0e6, 1e-6
# Attention, relative to sum p |v| (p the exact probabilities): on the codes (up to 64 rows per kv head in every episode) p is rounded to halves (2^-11),
# through the bf16 copy to bf16 (2^-8); fp32 scores of a few dozen are off by under 2^-15 of p, and so is the sum of the unrounded p that the
# log-sum-exp comes from.  Then the output's rounding, 2^-8.
P_ERROR = {"codes": 2.0 ** -11 + 2.0 ** -14, "copy": 2.0 ** -8 + 2.0 ** -14}
LSE_ERROR = 2.0 ** -14


@pytest.fixture(scope="module")
def handle():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    h = B.evlnCreate(0)
    yield h
    B.evlnDestroy(h)


class Batch:
    """Episodes on a pool of 8-bit pages that starts out as NaN codes and NaN scales."""

    def __init__(self, handle, lens, news, hq, hkv, seed=0, spare=2, scale=0.0, kv_size=1.0):
        self.h, self.lens, self.news, self.hq, self.hkv, self.G = handle, list(lens), list(news), hq, hkv, hq // hkv
        self.g = torch.Generator().manual_seed(seed)
        self.offs = np.concatenate([[0], np.cumsum(news)]).tolist()
        self.total, self.scale = self.offs[-1], scale
        need = [(L + n + P - 1) // P for L, n in zip(lens, news)]
        order = torch.randperm(sum(need) + spare, generator=self.g).tolist()
        width, at, self.rows = max(need) + 1, 0, []
        for c in need:
            self.rows.append(order[at:at + c] + [0] * (width - c))
            at += c
        self.pages, self.width = len(order), width
        self.table = torch.tensor(self.rows, dtype=torch.int32, device=DEV)
        shape = (self.pages, hkv, P, D)
        self.codes = [torch.full(shape, 0x7F, dtype=torch.uint8, device=DEV) for _ in range(2)]
        self.scales = [torch.full(shape[:2], float("nan"), device=DEV) for _ in range(2)]
        # earlier tokens: pages in 8 bits of sizes that differ by powers of two
        for which in range(2):
            for b, L in enumerate(lens):
                for p in range((L + P - 1) // P):
                    page, used = self.rows[b][p], min(P, L - p * P)
                    x = kv_size * torch.randn(hkv, used, D, generator=self.g) * torch.exp2(torch.randint(-3, 4, (hkv, 1, 1), generator=self.g).float())
                    s = torch.tensor([co.scale_for(f64(x[g])) for g in range(hkv)], dtype=torch.float32)
                    self.codes[which][page, :, :used] = (x / s[:, None, None]).to(torch.float8_e4m3fn).view(torch.uint8).to(DEV)
                    self.scales[which][page] = s.to(DEV)

    def params(self, **kw):
        return B.paged_params(self.hq, self.hkv, D, len(self.lens), P, self.pages, self.width, THETA, self.scale, **kw)

    def values(self, which):
        """The cache as fp64 values, [pages, Hkv, 64, D]."""
        return f64(self.codes[which].view(torch.float8_e4m3fn).float()) * f64(self.scales[which])[:, :, None, None]

    def episode(self, which, b):
        x = self.values(which)[self.rows[b]].transpose(0, 2, 1, 3).reshape(-1, self.hkv, D)
        return x[:self.lens[b] + self.news[b]]

    def tokens(self, sizes=1.0):
        heads = self.hq + 2 * self.hkv
        x = (sizes * torch.randn(self.total, heads, D, generator=self.g)).bfloat16().to(DEV)
        return x[:, :self.hq], x[:, self.hq:self.hq + self.hkv], x[:, self.hq + self.hkv:]

    def q_rot(self, size=1.5):
        return (size * torch.randn(self.hkv, self.total * self.G, D, generator=self.g)).bfloat16().to(DEV)

    def fill_new(self):
        """New tokens as evlnPaged8RopeAppend leaves them."""
        q, k, v = self.tokens()
        out = torch.empty(self.hkv, self.total * self.G, D, dtype=torch.bfloat16, device=DEV)
        B.evlnPaged8RopeAppend(self.h, self.params(), None, q, k, v, self.lens, self.offs, self.table, out, *self.codes, *self.scales)

    def attend(self, q_rot, stream=None):
        ws = torch.full((B.evlnPaged8WorkspaceSize(self.h, self.params(), self.lens, self.offs),), 0xFF, dtype=torch.uint8, device=DEV)
        out = torch.full((self.total, self.hq, D), float("nan"), dtype=torch.bfloat16, device=DEV)
        lse = torch.full((self.total, self.hq), float("nan"), device=DEV)
        B.evlnPaged8StepAttention(self.h, self.params(), q_rot, *self.codes, *self.scales, self.lens, self.offs, self.table, ws, out, lse, stream=stream)
        assert B.evlnGetDeviceStatus(self.h) == 0
        return out, lse

    @property
    def kind(self):
        return "codes" if max(self.news) * self.G <= 64 else "copy"

    def check(self, q_rot, out, lse):
        kind = self.kind
        q = f64(q_rot).reshape(self.hkv, -1, self.G, D).transpose(1, 0, 2, 3).reshape(-1, self.hq, D)
        for b, L in enumerate(self.lens):
            rows = slice(self.offs[b], self.offs[b + 1])
            if self.news[b] == 0:
                continue
            ref, ref_lse, size = co.attention(q[rows], self.episode(0, b), self.episode(1, b), L, self.scale or D ** -0.5)
            bound = 2.0 ** -8 * np.abs(ref) + P_ERROR[kind] * size + 1e-37
            worst = float((np.abs(f64(out[rows]) - ref) / bound).max())
            assert worst <= 1.0, f"episode {b}: {worst:.2f} times the bound"
            assert np.abs(f64(lse[rows]) - ref_lse).max() <= LSE_ERROR


APPENDS = [
    ([0, 63, 64, 333, 100], [70, 1, 129, 0, 37], 28, 4, True),
    ([0, 63, 64, 333, 100], [70, 1, 129, 5, 37], 28, 4, False),
    ([5], [1], 64, 8, True),
    ([1, 62, 127], [1, 1, 1], 2, 1, False),
    ([0], [1], 5, 5, True),
    ([700], [300], 8, 8, False),
]


@pytest.mark.parametrize("lens,news,hq,hkv,norm", APPENDS)
@pytest.mark.parametrize("table", [False, True])
def test_append(handle, lens, news, hq, hkv, norm, table):
    x = Batch(handle, lens, news, hq, hkv, seed=sum(lens) + hq)
    q, k, v = x.tokens(sizes=torch.exp2(torch.randint(-6, 7, (x.total, 1, 1), generator=x.g).float()))
    wq, wk = ((1.0 + 0.3 * torch.randn(D, generator=x.g)).bfloat16().to(DEV) for _ in range(2))
    rope = {}
    if table:
        count = max(L + n for L, n in zip(lens, news))
        t = torch.empty(B.evlnRopeTableBytes(D, count), dtype=torch.uint8, device=DEV)
        B.evlnRopeTable(handle, D, THETA, 0, count, t)
        rope = dict(rope_table=t, rope_table_first_pos=0, rope_table_count=count)
    before = [f64(c.view(torch.float8_e4m3fn).float()) for c in x.codes], [f64(s) for s in x.scales], [c.clone() for c in x.codes]
    q_rot = torch.empty(hkv, x.total * x.G, D, dtype=torch.bfloat16, device=DEV)
    B.evlnPaged8RopeAppend(handle, x.params(**rope), B.head_norm(wq, wk, EPS) if norm else None, q, k, v, lens, x.offs, x.table, q_rot, *x.codes, *x.scales)
    positions = np.concatenate([np.arange(L, L + n) for L, n in zip(lens, news)])
    yq, yk = f64(q), f64(k)
    if norm:
        yq, yk = co.rms_norm(yq, f64(wq), EPS), co.rms_norm(yk, f64(wk), EPS)
    rq, rk = co.rotate(yq, positions, THETA), co.rotate(yk, positions, THETA)
    ref = rq.reshape(-1, hkv, x.G, D).transpose(1, 0, 2, 3).reshape(hkv, -1, D)
    slack = 2.0 ** -19 * np.abs(ref).max(-1, keepdims=True)          # fp32 before the rounding to bf16
    assert (np.abs(f64(q_rot) - ref) <= 2.0 ** -8 * np.abs(ref) + slack).all()
    for which, new, exact in ((0, rk, False), (1, f64(v), True)):
        with np.errstate(invalid="ignore"):
            codes, scales = co.append8(before[0][which], before[1][which], new, lens, x.offs, x.rows, clear=exact)
        got, got_scales = f64(x.codes[which].view(torch.float8_e4m3fn).float()), f64(x.scales[which])
        assert np.array_equal(got_scales, scales, equal_nan=True)
        if exact:
            assert np.array_equal(got, codes, equal_nan=True)
        else:
            # keys are turned in fp32: a value at the border between two codes may fall to either, which is one step (a code's
            # spacing is at most an eighth of it), and few do
            differ = ~((got == codes) | (np.isnan(got) & np.isnan(codes)))
            assert differ.mean() < 1e-4 and (np.abs(got - codes)[differ] <= np.maximum(np.abs(codes)[differ] / 8, 2.0 ** -9)).all()
    if not norm:
        # the queries are those of the append into a bf16 cache, bit for bit
        pools = [torch.zeros(x.pages, hkv, P, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        other = torch.empty_like(q_rot)
        B.evlnPagedRopeAppend(handle, x.params(**rope), q.contiguous(), k.contiguous(), v.contiguous(), lens, x.offs, x.table, other, *pools)
        assert torch.equal(other, q_rot)


def test_append_borders_of_the_scale_and_values_that_are_not_finite(handle):
    x = Batch(handle, [0, 0, 0, 0, 0, 32], [3, 3, 3, 3, 3, 3], 2, 1, seed=3)
    q, k, v = (t.contiguous() for t in x.tokens())
    v.zero_()
    v[0, 0, 0] = 448.0                      # just in reach of scale 1
    v[3, 0, 0] = 450.0                      # just beyond (bf16 has 448 and 450)
    # 6 .. 8 stay zeros: the least scale
    v[9:12, 0] = 2.0 ** -126
    v[12, 0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 3.0])
    v[15, 0, 0], k[15] = 3.0e38, 0.0
    before = x.codes[1].clone()
    old = f64(before.view(torch.float8_e4m3fn).float())
    q_rot = torch.empty(1, x.total * 2, D, dtype=torch.bfloat16, device=DEV)
    B.evlnPaged8RopeAppend(handle, x.params(), None, q, k, v, x.lens, x.offs, x.table, q_rot, *x.codes, *x.scales)
    page = [x.rows[b][0] for b in range(6)]
    got, scale = f64(x.codes[1].view(torch.float8_e4m3fn).float()), f64(x.scales[1])[:, 0]
    assert scale[page[0]] == 1.0 and got[page[0], 0, 0, 0] == 448.0
    assert scale[page[1]] == 2.0 and got[page[1], 0, 0, 0] == 224.0          # 225 ties down to the even code
    assert scale[page[2]] == 2.0 ** -120 and (got[page[2]] == 0).all()
    assert scale[page[3]] == 2.0 ** -120 and (got[page[3], 0, :3] == 2.0 ** -6).all()
    assert scale[page[4]] == 2.0 ** -7 and got[page[4], 0, 0, 0] == 448.0 and got[page[4], 0, 0, 1] == -448.0
    assert np.isnan(got[page[4], 0, 0, 2]) and got[page[4], 0, 0, 3] == 384.0
    # a page that held tokens: the scale grows to 2^120 and the earlier codes, rounded anew, vanish
    assert scale[page[5]] == 2.0 ** 120 and (got[page[5], 0, :32] == 0).all() and np.isfinite(old[page[5], 0, :32]).all()


def test_a_page_filled_token_by_token(handle):
    # 70 appends of one token, sizes growing: what a page holds at the end is what the definition gives, step by step
    x = Batch(handle, [0], [70], 2, 1, seed=8)
    v = (torch.randn(70, 1, D, generator=x.g) * torch.exp2(torch.arange(70).float() / 9)[:, None, None]).bfloat16().to(DEV)
    codes, scales = np.zeros((x.pages, 1, P, D)), np.zeros((x.pages, 1))
    for i in range(70):
        q = torch.zeros(1, 2, D, dtype=torch.bfloat16, device=DEV)
        B.evlnPaged8RopeAppend(handle, x.params(), None, q, v[i:i + 1], v[i:i + 1], [i], [0, 1], x.table, q.clone(), *x.codes, *x.scales)
        codes, scales = co.append8(codes, scales, f64(v[i:i + 1]), [i], [0, 1], x.rows, clear=True)
    for page in x.rows[0][:2]:
        assert np.array_equal(f64(x.codes[1].view(torch.float8_e4m3fn).float())[page], codes[page])
        assert np.array_equal(f64(x.scales[1])[page], scales[page])


ATTENDS = [
    # rows per kv head: up to 8, 16, 32, 64 and more; lengths of one token, ends of pages and stages
    ([0], [1], 2, 1), ([31], [1], 2, 1), ([32], [1], 28, 4), ([63, 64, 65, 0], [1, 1, 1, 1], 28, 4),
    ([1000, 1, 4095, 130], [1, 2, 1, 0], 28, 4), ([777, 64], [4, 3], 28, 4), ([500], [9], 28, 4), ([95, 2000, 7], [8, 20, 30], 28, 4),
    ([8191], [1], 64, 8), ([0, 100], [33, 17], 8, 8), ([1500], [256], 3, 3), ([300], [1], 40, 1), ([5, 6], [11, 1], 12, 1),
]


@pytest.mark.parametrize("lens,news,hq,hkv", ATTENDS)
def test_attention_on_the_codes(handle, lens, news, hq, hkv):
    x = Batch(handle, lens, news, hq, hkv, seed=sum(lens) + sum(news))
    x.fill_new()
    q_rot = x.q_rot()
    out, lse = x.attend(q_rot)
    x.check(q_rot, out, lse)
    if x.kind == "codes":      # (on CTA pairs a row's softmax reference may move, and where to depends on who noticed first)
        again = x.attend(q_rot)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("lens,news,hq,hkv", [([0, 63, 64, 333, 1000], [70, 1, 129, 0, 196], 28, 4), ([50], [300], 1, 1), ([4096], [196], 28, 4)])
def test_attention_through_the_copy(handle, lens, news, hq, hkv):
    x = Batch(handle, lens, news, hq, hkv, seed=sum(lens))
    x.fill_new()
    q_rot = x.q_rot()
    out, lse = x.attend(q_rot)
    x.check(q_rot, out, lse)


def test_attention_many_short_episodes_and_more_units_than_blocks(handle):
    lens = [(37 * b) % 200 for b in range(200)]
    x = Batch(handle, lens, [b % 3 for b in range(200)], 6, 2, seed=5)
    x.fill_new()
    q_rot = x.q_rot()
    out, lse = x.attend(q_rot)
    x.check(q_rot, out, lse)


@pytest.mark.parametrize("q_size,scale", [(40.0, 0.0), (1e-3, 0.0), (1.5, 2.0), (3.0e30, 1e-30)])
def test_attention_sharp_flat_and_scaled_scores(handle, q_size, scale):
    x = Batch(handle, [700, 90], [1, 2], 28, 4, seed=11, scale=scale)
    x.fill_new()
    q_rot = x.q_rot(q_size)
    out, lse = x.attend(q_rot)
    # scores of hundreds are off by 2^-24 of their products' sizes in fp32
    q = f64(q_rot).reshape(4, -1, 7, D).transpose(1, 0, 2, 3).reshape(-1, 28, D)
    for b, L in enumerate(x.lens):
        rows = slice(x.offs[b], x.offs[b + 1])
        k = x.episode(0, b)
        ref, ref_lse, size = co.attention(q[rows], k, x.episode(1, b), L, scale or D ** -0.5)
        reach = max(np.abs(q[rows, h]).sum(-1).max() * np.abs(k[:, h // 7]).max() for h in range(28)) * (scale or D ** -0.5)
        slack = P_ERROR["codes"] + 2.0 ** -22 * reach
        assert (np.abs(f64(out[rows]) - ref) <= 2.0 ** -8 * np.abs(ref) + 2 * slack * size + 1e-37).all()
        assert np.abs(f64(lse[rows]) - ref_lse).max() <= LSE_ERROR + 2.0 ** -22 * reach


def test_value_scales_far_apart(handle):
    # pages whose values differ by 2^60: the large ones decide, whichever comes first, and the sums count every key
    x = Batch(handle, [320], [1], 7, 1, seed=21)
    x.fill_new()
    for order in ([0, 30, -30, 5, 0, 0], [60, 0, 0, 0, 0, -60]):
        for i, e in enumerate(order):
            x.scales[1][x.rows[0][i]] = 2.0 ** e
        q_rot = x.q_rot()
        out, lse = x.attend(q_rot)
        x.check(q_rot, out, lse)


def test_what_is_not_finite_stays_with_its_rows(handle):
    x = Batch(handle, [100, 100], [2, 2], 7, 1, seed=31)
    x.fill_new()
    # NaN behind the end of an episode (key slots: the append leaves them), and in a key that only the second new token sees
    x.codes[0][x.rows[0][1], :, 102 - P:] = 0x7F
    x.codes[0][x.rows[1][1], :, 101 - P] = 0x7F
    q_rot = x.q_rot()
    out, lse = x.attend(q_rot)
    assert bool(torch.isfinite(out[:2]).all()) and bool(torch.isfinite(out[2]).all()) and bool(torch.isnan(out[3]).all()) and bool(torch.isnan(lse[3]).all())
    x.news = [2, 1]
    q = f64(q_rot).reshape(1, -1, 7, D).transpose(1, 0, 2, 3).reshape(-1, 7, D)
    ref, ref_lse, size = co.attention(q[2:3], x.episode(0, 1), x.episode(1, 1), 100, D ** -0.5)
    assert (np.abs(f64(out[2:3]) - ref) <= 2.0 ** -8 * np.abs(ref) + P_ERROR["codes"] * size).all()


def test_a_step_as_it_is_used_captured_and_on_another_stream(handle):
    # append then attention, eagerly and as a replayed graph, on a side stream; three decode steps in a row
    x = Batch(handle, [130, 64, 1], [1, 1, 1], 28, 4, seed=41)
    ref = Batch(handle, [130, 64, 1], [1, 1, 1], 28, 4, seed=41)
    q, k, v = (t.contiguous() for t in x.tokens())
    norm_w = torch.ones(D, dtype=torch.bfloat16, device=DEV)
    norm = B.head_norm(norm_w, norm_w, EPS)
    q_rot = torch.empty(4, 21, D, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(B.evlnPaged8WorkspaceSize(handle, x.params(), x.lens, x.offs), dtype=torch.uint8, device=DEV)
    out = torch.empty(3, 28, D, dtype=torch.bfloat16, device=DEV)

    def step(b, o):
        B.evlnPaged8RopeAppend(handle, b.params(), norm, q, k, v, b.lens, b.offs, b.table, q_rot, *b.codes, *b.scales)
        B.evlnPaged8StepAttention(handle, b.params(), q_rot, *b.codes, *b.scales, b.lens, b.offs, b.table, ws, o)
    eager = torch.empty_like(out)
    step(ref, eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(x, out)
        for _ in range(3):
            out.fill_(float("nan"))
            graph.replay()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, eager)
    # the cache of the graph's steps is that of the eager one
    for a, b in zip(x.codes + x.scales, ref.codes + ref.scales):
        assert torch.equal(a.nan_to_num(7.0) if a.is_floating_point() else a, b.nan_to_num(7.0) if b.is_floating_point() else b)


def test_refusals(handle):
    x = Batch(handle, [10], [1], 4, 2, seed=1)
    x.fill_new()
    q_rot = x.q_rot()
    size = B.evlnPaged8WorkspaceSize(handle, x.params(), x.lens, x.offs)
    ws, out = torch.empty(size, dtype=torch.uint8, device=DEV), torch.empty(1, 4, D, dtype=torch.bfloat16, device=DEV)

    def refused(status, call, *args):
        with pytest.raises(B.EvlnError) as e:
            call(handle, *args)
        assert e.value.status == status
    good = [x.params(), q_rot, *x.codes, *x.scales, x.lens, x.offs, x.table, ws, out]
    for i in (1, 2, 3, 4, 5, 8, 10):
        refused(B.EVLN_INVALID_VALUE, B.evlnPaged8StepAttention, *[None if j == i else a for j, a in enumerate(good)])
    refused(B.EVLN_WORKSPACE_TOO_SMALL, B.evlnPaged8StepAttention, *good[:9], ws[:size - 256], out)
    refused(B.EVLN_INVALID_VALUE, B.evlnPaged8StepAttention, *good[:9], ws[8:], out)
    refused(B.EVLN_CACHE_FULL, B.evlnPaged8StepAttention, good[0], q_rot, *x.codes, *x.scales, [1000], x.offs, x.table, ws, out)
    bad = B.paged_params(4, 2, 64, 1, 64, 4, 4, THETA)
    refused(B.EVLN_NOT_SUPPORTED, B.evlnPaged8StepAttention, bad, *good[1:])
    q, k, v = x.tokens()
    ap = [x.params(), None, q, k, v, x.lens, x.offs, x.table, q_rot, *x.codes, *x.scales]
    for i in (7, 8, 9, 10, 11, 12):
        refused(B.EVLN_INVALID_VALUE, B.evlnPaged8RopeAppend, *[None if j == i else a for j, a in enumerate(ap)])
    refused(B.EVLN_INVALID_VALUE, B.evlnPaged8RopeAppend, ap[0], B.head_norm(None, None, -1.0), *ap[2:])
    # nothing to do: no tokens
    B.evlnPaged8StepAttention(handle, *good[:6], x.lens, [0, 0], x.table, ws, out)
