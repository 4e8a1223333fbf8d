"""Operators around the cache: what is timed of them, their plain forms, and their definitions in 64 bits.

A case is a dict of plain values; its "kind" says which operator it goes through:

  norm_append  per-head norms of queries and keys, rotation and append in one pass (evlnNormRopeAppend on a
               contiguous cache, evlnPagedNormRopeAppend on a page pool)
  append8      the same into a cache held in 8 bits with a scale for each page and kv head (evlnPaged8RopeAppend)
  attend8      step attention over such a cache (evlnPaged8StepAttention)
  key_weights  the attention weight that a step's queries give each cached key (evlnKeyWeights)
  evict        the keys of most accumulated weight chosen and laid out anew (evlnSelectKeys, evlnGatherKeys)

Lengths of a batch come from "lengths", a number that stands for the draw, so that a case fixes its work.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
PAGE = 64
THETA = 1.0e6
EPS = 1.0e-6
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HEADS_7B = {"q_heads": 28, "kv_heads": 4}
HEADS_70B = {"q_heads": 64, "kv_heads": 8}


# ---- cases -----------------------------------------------------------------------------------

def listed():
    one = {"kind": "norm_append", "head_dim": 128, "batch": 0, "lengths": 1}
    many8 = {"batch": 16, "shortest": 1024, "longest": 16384, "lengths": 3}
    weights = {"kind": "key_weights", "dtype": "bf16", "head_dim": 128}
    return [
        # a decoded action token of one layer: a chain of latencies
        {**one, **HEADS_7B, "name": "norm_append_token", "dtype": "bf16", "shortest": 4292, "longest": 4292, "least": 1, "most": 1,
         "joined": True, "table": True},
        # a new frame for each of 16 episodes, queries, keys and values as one projection leaves them
        {**one, **HEADS_7B, **many8, "name": "norm_append_frames", "dtype": "bf16", "least": 196, "most": 196, "joined": True, "table": True},
        # an action token for each of 16 episodes, into pages that are partly filled
        {"kind": "append8", **HEADS_7B, **many8, "name": "append8_tokens", "least": 1, "most": 1, "norm": False, "joined": True, "table": True},
        # a new frame for each, with the norms of queries and keys
        {"kind": "append8", **HEADS_7B, **many8, "name": "append8_frames", "least": 196, "most": 196, "norm": True, "joined": True, "table": True},
        # decoding: one token for each of 16 ragged episodes, whose caches are read once
        {"kind": "attend8", **HEADS_7B, **many8, "name": "attend8_tokens", "least": 1, "most": 1},
        # a chunk of action tokens late in one episode
        {"kind": "attend8", **HEADS_7B, "name": "attend8_chunk", "batch": 1, "shortest": 20656, "longest": 20656, "lengths": 1, "least": 8, "most": 8},
        # a token over a long history on the 70B-class heads
        {"kind": "attend8", **HEADS_70B, "name": "attend8_long_70b", "batch": 1, "shortest": 32768, "longest": 32768, "lengths": 1, "least": 1, "most": 1},
        # a new frame for each of 16 ragged episodes: matrix products bound it
        {"kind": "attend8", **HEADS_7B, **many8, "name": "attend8_frames", "least": 196, "most": 196},
        # what a new frame's queries weigh the cached keys with
        {**weights, **HEADS_7B, "name": "key_weights_frame", "cached": 4096, "new": 196, "decay": 0.9},
        # the same for a decoded token late in an episode: the keys are read once
        {**weights, **HEADS_7B, "name": "key_weights_token", "cached": 20656, "new": 1, "decay": 1.0},
        # a long episode cut to a fifth of its keys, chosen for each kv head, turned to their new places
        {"kind": "evict", "name": "evict_episode", "dtype": "bf16", "kv_heads": 4, "head_dim": 128, "cached": 20656, "budget": 4096, "sinks": 256,
         "recent": 196, "rotate": True},
        # the small single-layer shape in fp32, keys kept at the angles that they have
        {"kind": "evict", "name": "evict_tiny_f32", "dtype": "f32", "kv_heads": 1, "head_dim": 64, "cached": 320, "budget": 128, "sinks": 4,
         "recent": 64, "rotate": False},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    kind = rng.choice(["norm_append", "append8", "attend8", "attend8", "key_weights", "evict"])
    q_heads, kv_heads = rng.choice([(28, 4), (64, 8), (2, 1), (14, 2), (8, 8), (32, 4), (12, 1), (5, 5)])
    case = {"kind": kind, "q_heads": q_heads, "kv_heads": kv_heads}
    if kind in ("norm_append", "append8", "attend8"):
        batch = _log(rng, 1, 24)
        shortest = rng.choice([0, _log(rng, 1, 4096)])
        least = _log(rng, 1, 256)
        case |= {"batch": batch, "lengths": rng.randrange(1 << 20), "shortest": shortest, "longest": shortest + _log(rng, 1, 16384),
                 "least": least, "most": least + rng.choice([0, _log(rng, 1, 64)])}
        if kind != "attend8":
            case |= {"joined": rng.random() < 0.5, "table": rng.random() < 0.5}
        if kind == "append8":
            case["norm"] = rng.random() < 0.5
        if kind == "norm_append":
            case |= {"dtype": "bf16", "head_dim": 128}
            if rng.random() < 0.6:
                case |= {"batch": 0, "dtype": rng.choice(["bf16", "f32"]), "head_dim": rng.choice([64, 128]), "least": case["most"], "shortest": case["longest"]}
    elif kind == "key_weights":
        case |= {"dtype": rng.choice(["bf16", "bf16", "f32"]), "head_dim": rng.choice([64, 128]), "cached": rng.choice([0, _log(rng, 1, 32768)]),
                 "new": _log(rng, 1, 256), "decay": rng.choice([1.0, 0.9, 0.0])}
    else:
        del case["q_heads"]
        cached = _log(rng, 2, 65536)
        budget = _log(rng, 1, cached)
        sinks = rng.randrange(budget // 4 + 1)
        case |= {"dtype": rng.choice(["bf16", "f32"]), "head_dim": rng.choice([64, 128]), "cached": cached, "budget": budget, "sinks": sinks,
                 "recent": rng.randrange((budget - sinks) // 2 + 1), "rotate": rng.random() < 0.5}
    return case


def draw(rng):
    most = [work(c) for c in listed()]
    limit = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    while True:
        case = _draw(rng)
        w = work(case)
        if w["bytes"] <= limit["bytes"] and w["flops"] <= limit["flops"] * (0.1 if case.get("dtype") == "f32" else 1.0):
            return case


def _lengths(case):
    """Cached and new tokens of every episode (one, on a contiguous cache, where "batch" is 0)."""
    r = random.Random(case["lengths"])
    episodes = max(1, case["batch"])
    return [r.randint(case["shortest"], case["longest"]) for _ in range(episodes)], [r.randint(case["least"], case["most"]) for _ in range(episodes)]


def work(case):
    kind = case["kind"]
    if kind == "evict":
        row = case["head_dim"] * (2 if case["dtype"] == "bf16" else 4)
        kept = min(case["budget"], case["cached"])
        moved = case["kv_heads"] * kept * (4 * row + 8 + 4)                    # keys and values, weights, the choice
        turned = case["kv_heads"] * kept * case["head_dim"] * 3 if case["rotate"] else 0
        return {"bytes": moved + 4 * case["kv_heads"] * case["cached"], "flops": turned}
    if kind == "key_weights":
        e, L, n = (2 if case["dtype"] == "bf16" else 4), case["cached"], case["new"]
        pairs = n * L + n * (n + 1) // 2
        moved = (L + n) * case["kv_heads"] * (case["head_dim"] * e + 8) + n * case["q_heads"] * (case["head_dim"] * e + 4)
        return {"bytes": moved, "flops": case["q_heads"] * pairs * 2 * case["head_dim"]}
    lens, news = _lengths(case)
    total, hq, hkv = sum(news), case["q_heads"], case["kv_heads"]
    if kind == "norm_append":
        e, D = (2 if case["dtype"] == "bf16" else 4), case["head_dim"]
        return {"bytes": total * (hq + 2 * hkv) * D * e * 2, "flops": total * (hq + hkv) * D * 7}
    D = 128
    if kind == "append8":
        # new pages are written, the page that a run begins in is read too
        tokens = sum((L + n + PAGE - 1) // PAGE * PAGE - L for L, n in zip(lens, news))
        read = sum(L % PAGE for L, n in zip(lens, news) if n)
        moved = total * (2 * hq + 2 * hkv) * D * 2 + (total + 2 * read) * 2 * hkv * D + (tokens - total) * hkv * D
        return {"bytes": moved, "flops": total * (hq + hkv) * D * (7 if case["norm"] else 3) + 2 * total * hkv * D * 2}
    pairs = sum(n * L + n * (n + 1) // 2 for L, n in zip(lens, news))
    keys = sum(L + n for L, n in zip(lens, news))
    return {"bytes": keys * hkv * 2 * D + total * hq * (D * 4 + 4), "flops": 4 * D * hq * pairs}


# ---- inputs ----------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed & 0x7FFFFFFFFFFF)


def _new_tokens(case, g, total, hq, hkv, D, dtype):
    """Queries, keys and values of the new tokens: views of one projection's rows, or tensors of their own.  Channels differ in size."""
    heads = hq + 2 * hkv
    spread = torch.exp(0.5 * torch.randn(heads, D, generator=g, device=DEV))
    x = (torch.randn(total, heads, D, generator=g, device=DEV) * spread).to(dtype)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    return (q, k, v) if case.get("joined") else (q.contiguous(), k.contiguous(), v.contiguous())


def _norm_weights(g, D, dtype):
    return [(1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dtype) for _ in range(2)]


def _pages(case, seed):
    """Page tables over a shuffled pool, with pages to spare."""
    lens, news = _lengths(case)
    offs = [0]
    for n in news:
        offs.append(offs[-1] + n)
    need = [(L + n + PAGE - 1) // PAGE for L, n in zip(lens, news)]
    order = list(range(sum(need) + 3))
    random.Random(seed).shuffle(order)
    table, at = torch.zeros(len(lens), max(need), dtype=torch.int32), 0
    for b, c in enumerate(need):
        table[b, :c] = torch.tensor(order[at:at + c], dtype=torch.int32)
        at += c
    return lens, news, offs, table, len(order)


def _quantised(x, span):
    """[pages, Hkv, 64, 128] values in 8 bits, a power of two for each page and head; `span` says how the pages' sizes differ."""
    x *= torch.exp2(span)[:, :, None, None]
    most = x.abs().amax(dim=(2, 3))
    scale = torch.exp2(torch.ceil(torch.log2(most / 448.0)).clamp(-120.0, 120.0))
    return (x / scale[:, :, None, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), scale


def _pools8(g, pages, hkv):
    out = []
    for _ in range(2):
        span = 0.5 * torch.randn(pages, hkv, generator=g, device=DEV)
        codes = torch.empty(pages, hkv, PAGE, 128, dtype=torch.float8_e4m3fn, device=DEV)
        scales = torch.empty(pages, hkv, device=DEV)
        for a in range(0, pages, 512):
            b = min(pages, a + 512)
            codes[a:b], scales[a:b] = _quantised(torch.randn(b - a, hkv, PAGE, 128, generator=g, device=DEV), span[a:b])
        out += [codes, scales]
    return out[0], out[2], out[1], out[3]      # k, v, scales of k, of v


def _log_sum_exp(q_rot, k, L, n, G, scale):
    """[n, Hq]: of the scaled products of [Hkv, n G, D] queries and [Hkv, L + n, D] keys, in 64 bits, causal."""
    at = torch.arange(n, device=DEV).repeat_interleave(G)
    hidden = torch.arange(L + n, device=DEV)[None, :] > L + at[:, None]
    rows = [torch.logsumexp((q_rot[h].double() @ k[h].double().T * scale).masked_fill(hidden, -math.inf), dim=1) for h in range(len(q_rot))]
    return torch.stack(rows).view(-1, n, G).permute(1, 0, 2).reshape(n, -1).float().contiguous()


def _inputs(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = {"case": case}
    if kind == "evict":
        dtype, hkv, D, L = DTYPES[case["dtype"]], case["kv_heads"], case["head_dim"], case["cached"]
        s["k"], s["v"] = (torch.randn(hkv, L, D, generator=g, device=DEV).to(dtype) for _ in range(2))
        # accumulated weights: a few keys take most of it; some took none, or the same
        s["weights"] = torch.exp(2.0 * torch.randn(hkv, L, generator=g, device=DEV))
        s["weights"][:, ::7] = 0.0
        kept = min(case["budget"], L)
        s["kept"] = torch.empty(hkv, kept, dtype=torch.int32, device=DEV)
        s["k_work"], s["v_work"] = (torch.zeros(hkv, kept + 5, D, dtype=dtype, device=DEV) for _ in range(2))
        s["weights_work"] = torch.zeros(hkv, kept + 5, device=DEV)
        return s
    hq, hkv = case["q_heads"], case["kv_heads"]
    G = hq // hkv
    if kind == "key_weights":
        dtype, D, L, n = DTYPES[case["dtype"]], case["head_dim"], case["cached"], case["new"]
        s["q_rot"] = (1.5 * torch.randn(hkv, n * G, D, generator=g, device=DEV)).to(dtype)
        s["k"] = torch.randn(hkv, L + n + 9, D, generator=g, device=DEV).to(dtype)
        s["lse"] = _log_sum_exp(s["q_rot"], s["k"][:, :L + n], L, n, G, 1.0 / math.sqrt(D))
        s["weights"] = torch.exp(torch.randn(hkv, L + n + 9, generator=g, device=DEV))
        s["weights_out"] = torch.zeros_like(s["weights"])
        return s
    D = case.get("head_dim", 128)
    dtype = DTYPES[case.get("dtype", "bf16")]
    s["lens"], s["news"], s["offs"], table, s["num_pages"] = _pages(case, seed)
    s["table"], total = table.to(DEV), sum(s["news"])
    paged = case["batch"] > 0
    # where every new token goes, as the plain form wants it
    b = torch.repeat_interleave(torch.arange(len(s["news"])), torch.tensor(s["news"]))
    within = torch.arange(total) - torch.tensor(s["offs"])[b]
    place = torch.tensor(s["lens"])[b] + within
    s["place"] = place.to(DEV)
    s["slot"], s["page"] = (place % PAGE).to(DEV), table[b, place // PAGE].long().to(DEV)
    if kind == "attend8":
        s["q_rot"] = (1.5 * torch.randn(hkv, total * G, D, generator=g, device=DEV)).to(dtype)
        s["k"], s["v"], s["k_scale"], s["v_scale"] = _pools8(g, s["num_pages"], hkv)
        s["episode"], s["within"] = b.to(DEV), within.to(DEV)
        s["out"] = torch.empty(total, hq, D, dtype=dtype, device=DEV)
        s["lse"] = torch.empty(total, hq, device=DEV)
        return s
    s["q_new"], s["k_new"], s["v_new"] = _new_tokens(case, g, total, hq, hkv, D, dtype)
    s["q_rot"] = torch.empty(hkv, total * G, D, dtype=dtype, device=DEV)
    s["norm"] = _norm_weights(g, D, dtype) if case.get("norm", True) else None
    if kind == "append8":
        s["k"], s["v"], s["k_scale"], s["v_scale"] = _pools8(g, s["num_pages"], hkv)
        # the pages that a run touches, and which of their slots hold earlier tokens, new ones and none
        touched = [(e, p) for e, (L, n) in enumerate(zip(s["lens"], s["news"])) for p in range(L // PAGE, (L + n + PAGE - 1) // PAGE)]
        e, p = (torch.tensor(x) for x in zip(*touched))
        at = p[:, None] * PAGE + torch.arange(PAGE)[None, :]
        lens, news, offs = torch.tensor(s["lens"])[e][:, None], torch.tensor(s["news"])[e][:, None], torch.tensor(s["offs"])[:-1][e][:, None]
        s["touched"] = table[e, p].long().to(DEV)
        s["is_new"], s["is_old"] = ((at >= lens) & (at < lens + news)).to(DEV), (at < lens).to(DEV)
        s["token"] = (at - lens + offs).clamp(0, total - 1).to(DEV)
    elif paged:
        shape = (s["num_pages"], hkv, PAGE, D)
        s["k"], s["v"] = (torch.zeros(shape, dtype=dtype, device=DEV) for _ in range(2))
    else:
        shape = (hkv, s["lens"][0] + total + 7, D)
        s["k"], s["v"] = (torch.zeros(shape, dtype=dtype, device=DEV) for _ in range(2))
    return s


_handle = None


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        global _handle
        from paper_2512_10310_b200 import binding as B
        if _handle is None:
            _handle = B.evlnCreate(0)
        s["B"], s["handle"], kind = B, _handle, case["kind"]
        if kind == "evict":
            s["params"] = B.gather_params(case["dtype"], case["kv_heads"], case["head_dim"], s["k"].shape[1], s["k_work"].shape[1], THETA)
            return s
        if kind == "key_weights":
            s["params"] = B.step_params(case["dtype"], case["q_heads"], case["kv_heads"], case["head_dim"], case["cached"], case["new"], s["k"].shape[1], THETA)
            return s
        D, rope = case.get("head_dim", 128), {}
        if case.get("table"):
            count = max(L + n for L, n in zip(s["lens"], s["news"]))
            s["rope"] = torch.empty(B.evlnRopeTableBytes(D, count), dtype=torch.uint8, device=DEV)
            B.evlnRopeTable(_handle, D, THETA, 0, count, s["rope"])
            rope = dict(rope_table=s["rope"], rope_table_first_pos=0, rope_table_count=count)
        if case["batch"] > 0:
            s["params"] = B.paged_params(case["q_heads"], case["kv_heads"], D, case["batch"], PAGE, s["num_pages"], s["table"].shape[1], THETA, **rope)
        else:
            s["params"] = B.step_params(case["dtype"], case["q_heads"], case["kv_heads"], D, s["lens"][0], s["news"][0], s["k"].shape[1], THETA, **rope)
        if kind == "attend8":
            s["workspace"] = torch.empty(max(16, B.evlnPaged8WorkspaceSize(_handle, s["params"], s["lens"], s["offs"])), dtype=torch.uint8, device=DEV)
        else:
            s["head_norm"] = B.head_norm(s["norm"][0], s["norm"][1], EPS) if s["norm"] else None
    return s


# ---- the framework's calls ---------------------------------------------------------------------

def _run_own(s):
    B, h, p, case = s["B"], s["handle"], s["params"], s["case"]
    kind = case["kind"]
    if kind == "norm_append":
        if case["batch"] > 0:
            B.evlnPagedNormRopeAppend(h, p, s["head_norm"], s["q_new"], s["k_new"], s["v_new"], s["lens"], s["offs"], s["table"], s["q_rot"], s["k"], s["v"])
        else:
            B.evlnNormRopeAppend(h, p, s["head_norm"], s["q_new"], s["k_new"], s["v_new"], s["q_rot"], s["k"], s["v"])
        return s["q_rot"], s["k"], s["v"]
    if kind == "append8":
        B.evlnPaged8RopeAppend(h, p, s["head_norm"], s["q_new"], s["k_new"], s["v_new"], s["lens"], s["offs"], s["table"], s["q_rot"], s["k"], s["v"],
                               s["k_scale"], s["v_scale"])
        return s["q_rot"], s["k"], s["v"], s["k_scale"], s["v_scale"]
    if kind == "attend8":
        B.evlnPaged8StepAttention(h, p, s["q_rot"], s["k"], s["v"], s["k_scale"], s["v_scale"], s["lens"], s["offs"], s["table"], s["workspace"], s["out"],
                                  s["lse"])
        return s["out"], s["lse"]
    if kind == "key_weights":
        B.evlnKeyWeights(h, p, s["q_rot"], s["k"], s["lse"], case["decay"], s["weights"], s["weights_out"])
        return s["weights_out"]
    B.evlnSelectKeys(h, p, s["weights"], case["cached"], case["budget"], case["sinks"], case["recent"], s["kept"])
    B.evlnGatherKeys(h, p, s["kept"].shape[1], s["kept"], s["weights"], s["k"], s["v"], s["weights_work"], s["k_work"], s["v_work"], case["rotate"])
    return s["kept"], s["weights_work"], s["k_work"], s["v_work"]


# ---- the plain forms -------------------------------------------------------------------------

def _turn(x, place):
    """x [tokens, heads, D] in 32 bits, turned at the positions; the angles in 64."""
    D = x.shape[-1]
    omega = THETA ** (-2.0 * torch.arange(D // 2, device=DEV, dtype=torch.float64) / D)
    angle = place.double()[:, None] * omega
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _normed(x, w):
    x = x.float()
    return x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * w.float()


def _turned_new(s):
    q, k = (_normed(x, w) for x, w in zip((s["q_new"], s["k_new"]), s["norm"])) if s["norm"] else (s["q_new"].float(), s["k_new"].float())
    return _turn(q, s["place"]), _turn(k, s["place"])


def _grouped(q, hkv):
    """[tokens, Hq, D] -> [Hkv, tokens G, D]"""
    t, hq, D = q.shape
    return q.view(t, hkv, hq // hkv, D).permute(1, 0, 2, 3).reshape(hkv, -1, D)


def _plain_norm_append(s):
    q, k = _turned_new(s)
    hkv, dtype = k.shape[1], s["q_new"].dtype
    s["q_rot"].copy_(_grouped(q, hkv))
    if s["case"]["batch"] > 0:
        s["k"][s["page"], :, s["slot"]] = k.to(dtype)
        s["v"][s["page"], :, s["slot"]] = s["v_new"]
    else:
        s["k"][:, s["place"]] = k.to(dtype).transpose(0, 1)
        s["v"][:, s["place"]] = s["v_new"].transpose(0, 1)
    return s["q_rot"], s["k"], s["v"]


def _plain_page8(s, codes, scales, new, clear):
    """The touched pages with the new tokens in: a scale that covers them, earlier tokens rounded anew where it grew."""
    at, is_new, is_old = s["touched"], s["is_new"][:, None, :, None], s["is_old"][:, None, :, None]
    old_code, old_scale = codes.view(torch.uint8)[at], scales[at][:, :, None, None]
    old = old_code.view(torch.float8_e4m3fn).float()
    x = new[s["token"]].transpose(1, 2)                                             # [pages, Hkv, 64, 128]
    most = torch.where(is_new, x.abs(), 0.0).amax(dim=(2, 3), keepdim=True)
    need = torch.exp2(torch.ceil(torch.log2(most / 448.0)).clamp(-120.0, 120.0))
    need = torch.where(most > need * 448.0, need * 2.0, torch.where((most <= need * 224.0) & (need > 2.0 ** -120), need * 0.5, need))   # log2 is rounded
    held = is_old.any(dim=2, keepdim=True)
    scale = torch.where(held, torch.maximum(need, old_scale), need)
    code = torch.where(is_new, x / scale, old * (old_scale / scale)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    rest = torch.zeros_like(old_code) if clear else old_code
    codes.view(torch.uint8)[at] = torch.where(is_new | is_old, code, rest)
    scales[at] = scale[:, :, 0, 0]


def _plain_append8(s):
    q, k = _turned_new(s)
    s["q_rot"].copy_(_grouped(q, k.shape[1]))
    _plain_page8(s, s["k"], s["k_scale"], k, False)
    _plain_page8(s, s["v"], s["v_scale"], s["v_new"].float(), True)
    return s["q_rot"], s["k"], s["v"], s["k_scale"], s["v_scale"]


def _plain_attend8(s):
    case, table = s["case"], s["table"].long()
    hq, hkv, episodes, most = case["q_heads"], case["kv_heads"], len(s["lens"]), max(s["news"])
    G = hq // hkv
    held = []
    for codes, scales in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])):
        x = codes.view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * scales[table][..., None, None]
        held.append(x.permute(0, 2, 1, 3, 4).reshape(episodes, hkv, -1, 128))
    q = torch.zeros(episodes, most, hkv, G, 128, device=DEV)
    q[s["episode"], s["within"]] = s["q_rot"].view(hkv, -1, G, 128).transpose(0, 1).float()
    scores = q.permute(0, 2, 1, 3, 4).reshape(episodes, hkv, most * G, 128) @ held[0].transpose(2, 3)
    del q
    scores *= 1.0 / math.sqrt(128.0)
    last = torch.tensor(s["lens"], device=DEV)[:, None] + torch.arange(most, device=DEV).repeat_interleave(G)[None, :]
    scores.masked_fill_((torch.arange(scores.shape[3], device=DEV)[None, None, :] > last[:, :, None])[:, None], -math.inf)
    top = scores.amax(dim=3, keepdim=True)
    scores.sub_(top).exp_()
    total = scores.sum(dim=3, keepdim=True)
    out = (scores @ held[1]) / total
    back = lambda x: x.view(episodes, hkv, most, G, -1).permute(0, 2, 1, 3, 4)[s["episode"], s["within"]].reshape(len(s["episode"]), hq, -1)  # noqa: E731
    return back(out).to(s["out"].dtype), back(top + torch.log(total))[..., 0]


def _plain_key_weights(s):
    case = s["case"]
    hkv, G, L, n = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["cached"], case["new"]
    scores = s["q_rot"].float() @ s["k"][:, :L + n].float().transpose(1, 2)
    scores *= 1.0 / math.sqrt(case["head_dim"])
    scores -= s["lse"].view(n, hkv, G).transpose(0, 1).reshape(hkv, n * G, 1)
    last = L + torch.arange(n, device=DEV).repeat_interleave(G)
    scores.masked_fill_(torch.arange(L + n, device=DEV)[None, :] > last[:, None], -math.inf)
    given = scores.exp_().sum(dim=1)
    given[:, :L] += case["decay"] * s["weights"][:, :L]
    s["weights_out"][:, :L + n] = given
    return s["weights_out"]


def _plain_evict(s):
    case = s["case"]
    L, kept, sinks, recent = case["cached"], s["kept"].shape[1], case["sinks"], case["recent"]
    rank = torch.where(torch.isnan(s["weights"]), -math.inf, s["weights"])
    if kept < L:
        rank = rank.clone()
        rank[:, :sinks] = math.inf
        rank[:, L - recent:] = math.inf
    at = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :kept].sort(dim=1).values
    rows = at[:, :, None].expand(-1, -1, case["head_dim"])
    k, v = torch.gather(s["k"], 1, rows), torch.gather(s["v"], 1, rows)
    if case["rotate"]:
        k = _turn(k.float().transpose(0, 1), torch.arange(kept, device=DEV)).transpose(0, 1)
    s["k_work"][:, :kept] = k.to(s["k"].dtype)
    s["v_work"][:, :kept] = v
    s["weights_work"][:, :kept] = torch.gather(s["weights"], 1, at)
    s["kept"].copy_(at)
    return s["kept"], s["weights_work"], s["k_work"], s["v_work"]


_PLAIN = {"norm_append": _plain_norm_append, "append8": _plain_append8, "attend8": _plain_attend8, "key_weights": _plain_key_weights, "evict": _plain_evict}


def run(s):
    if own:
        return _run_own(s)
    return _PLAIN[s["case"]["kind"]](s)


# ---- the definitions, in 64 bits ---------------------------------------------------------------

def _exact_turn(x, pos):
    """x [..., D] in 64 bits turned by the angle of position `pos` (broadcast over all but the last axis): a complex product."""
    D = x.shape[-1]
    z = torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous())
    j = torch.arange(D // 2, device=DEV, dtype=torch.float64)
    w = pos.double()[..., None] * torch.exp(j * (-2.0 * math.log(THETA) / D))
    z = z * torch.polar(torch.ones_like(w), w)
    return torch.cat([z.real, z.imag], dim=-1)


def _exact_norm(x, w):
    x = x.double()
    return x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * w.double()


def _exact_code(x):
    """The nearest number of 4 exponent and 3 fraction bits (ties to even, at most 448) to every one of x."""
    _, e = torch.frexp(x)
    step = torch.exp2(torch.clamp(e - 1, min=-6).double() - 3.0)
    return torch.clamp(torch.round(x / step) * step, -448.0, 448.0)


def _exact_new(s):
    q, k = s["q_new"].double(), s["k_new"].double()
    if s["norm"]:
        q, k = _exact_norm(q, s["norm"][0]), _exact_norm(k, s["norm"][1])
    pos = s["place"][:, None]
    return _exact_turn(q, pos), _exact_turn(k, pos)


def _exact_append(s):
    q, k = _exact_new(s)
    hq, hkv = q.shape[1], k.shape[1]
    G = hq // hkv
    q_rot = torch.stack([q[:, h * G:(h + 1) * G].reshape(-1, q.shape[2]) for h in range(hkv)])
    k_all, v_all = s["k"].double(), s["v"].double()
    for e, (L, n) in enumerate(zip(s["lens"], s["news"])):
        rows = slice(s["offs"][e], s["offs"][e] + n)
        for which, new in ((k_all, k[rows]), (v_all, s["v_new"][rows].double())):
            if s["case"]["batch"] == 0:
                which[:, L:L + n] = new.transpose(0, 1)
                continue
            for p in range(L // PAGE, (L + n + PAGE - 1) // PAGE):
                a, b = max(L, p * PAGE), min(L + n, (p + 1) * PAGE)
                which[int(s["table"][e, p]), :, a - p * PAGE:b - p * PAGE] = new[a - L:b - L].transpose(0, 1)
    return q_rot, k_all, v_all


def _exact_append8(s):
    q, k = _exact_new(s)
    hkv, G = k.shape[1], q.shape[1] // k.shape[1]
    q_rot = torch.stack([q[:, h * G:(h + 1) * G].reshape(-1, q.shape[2]) for h in range(hkv)])
    done = []
    for codes, scales, new, clear in ((s["k"], s["k_scale"], k, False), (s["v"], s["v_scale"], s["v_new"].double(), True)):
        codes, scales = codes.double(), scales.double()
        for e, (L, n) in enumerate(zip(s["lens"], s["news"])):
            for p in range(L // PAGE, (L + n + PAGE - 1) // PAGE):
                page, a, b = int(s["table"][e, p]), max(L, p * PAGE), min(L + n, (p + 1) * PAGE)
                x = new[s["offs"][e] + a - L:s["offs"][e] + b - L].transpose(0, 1)                  # [Hkv, tokens, 128]
                fraction, power = torch.frexp(x.abs().amax(dim=(1, 2)) / 448.0)
                size = torch.exp2((power - (fraction == 0.5).to(power.dtype)).double().clamp(-120, 120))
                size = torch.where(x.abs().amax(dim=(1, 2)) == 0, 2.0 ** -120, size)
                if a > p * PAGE:
                    size = torch.maximum(size, scales[page])
                    codes[page, :, :a - p * PAGE] = _exact_code(codes[page, :, :a - p * PAGE] * (scales[page] / size)[:, None, None])
                codes[page, :, a - p * PAGE:b - p * PAGE] = _exact_code(x / size[:, None, None])
                if clear:
                    codes[page, :, b - p * PAGE:] = 0.0
                scales[page] = size
        done.append((codes, scales))
    return q_rot, done[0][0], done[1][0], done[0][1], done[1][1]


def _exact_attend8(s):
    case = s["case"]
    hkv, G = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    out = torch.empty(sum(s["news"]), hkv, G, 128, dtype=torch.float64, device=DEV)
    lse = torch.empty(sum(s["news"]), hkv, G, dtype=torch.float64, device=DEV)
    for e, (L, n) in enumerate(zip(s["lens"], s["news"])):
        pages = s["table"][e, :(L + n + PAGE - 1) // PAGE].long()
        rows = slice(s["offs"][e], s["offs"][e] + n)
        for h in range(hkv):
            k, v = ((codes.view(torch.uint8)[pages, h].view(torch.float8_e4m3fn).double() * scales[pages, h].double()[:, None, None]).reshape(-1, 128)[:L + n]
                    for codes, scales in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])))
            q = s["q_rot"][h].view(-1, G, 128)[rows].reshape(-1, 128).double()
            t = q @ k.T / math.sqrt(128.0)
            t.masked_fill_(torch.arange(L + n, device=DEV)[None] > L + torch.arange(n, device=DEV).repeat_interleave(G)[:, None], -math.inf)
            lse[rows, h] = torch.logsumexp(t, dim=1).view(n, G)
            out[rows, h] = (torch.softmax(t, dim=1) @ v).view(n, G, 128)
    return out.flatten(1, 2), lse.flatten(1, 2)


def _exact_key_weights(s):
    case = s["case"]
    hkv, G, L, n = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["cached"], case["new"]
    result = s["weights_out"].double()
    for h in range(hkv):
        t = s["q_rot"][h].double() @ s["k"][h, :L + n].double().T / math.sqrt(case["head_dim"])
        p = torch.exp(t - s["lse"][:, h * G:(h + 1) * G].reshape(-1, 1).double())
        p[torch.arange(L + n, device=DEV)[None] > L + torch.arange(n, device=DEV).repeat_interleave(G)[:, None]] = 0.0
        result[h, :L + n] = p.sum(0)
        result[h, :L] += case["decay"] * s["weights"][h, :L].double()
    return result


def _exact_evict(s):
    case = s["case"]
    L, hkv, sinks, recent = case["cached"], case["kv_heads"], case["sinks"], case["recent"]
    kept, w = s["kept"].shape[1], s["weights"].cpu().tolist()
    chosen = []
    for h in range(hkv):
        if kept == L:
            chosen.append(list(range(L)))
            continue
        middle = sorted(range(sinks, L - recent), key=lambda j: (-w[h][j], j))[:kept - sinks - recent]
        chosen.append(list(range(sinks)) + sorted(middle) + list(range(L - recent, L)))
    at = torch.tensor(chosen, device=DEV)
    k_work, v_work, weights = s["k_work"].double(), s["v_work"].double(), s["weights_work"].double()
    for h in range(hkv):
        k = s["k"][h, at[h]].double()
        k_work[h, :kept] = _exact_turn(k, torch.arange(kept, device=DEV)) if case["rotate"] else k
        v_work[h, :kept], weights[h, :kept] = s["v"][h, at[h]].double(), s["weights"][h, at[h]].double()
    return at.to(torch.int32), weights, k_work, v_work


_EXACT = {"norm_append": _exact_append, "append8": _exact_append8, "attend8": _exact_attend8, "key_weights": _exact_key_weights, "evict": _exact_evict}


def exact(case, seed):
    return _EXACT[case["kind"]](_inputs(case, seed))
