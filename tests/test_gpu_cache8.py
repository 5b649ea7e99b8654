"""The paged 8-bit cache on the GPU: appending (codes and scales equal to those of the definition), a decode step over it (within
bounds computed from the operands), both against float64 loops."""
import math

import numpy as np
import pytest
import torch

from paper_2408_01890_amd import lisa
from tests import cache8_ref as cr

pytestmark = pytest.mark.gpu
DEV = "cuda"
I8, E4 = torch.int8, torch.float8_e4m3fn
FMT = {"int8": I8, "e4m3": E4}


def make_pages(lens, P, C, g, absent=()):
    """A state whose pages lie anywhere; `absent`: (sequence, column) entries that name no page."""
    ids = torch.randperm(P, generator=g).tolist()
    table = [[-1] * C for _ in lens]
    for s, n in enumerate(lens):
        for c in range(min(C, -(-n // 64))):
            table[s][c] = ids.pop()
    for k, (s, c) in enumerate(absent):
        table[s][c] = (-1, P, -7, 1 << 30)[k % 4]
    refs = torch.zeros(P, dtype=torch.int32)
    for row in table:
        for p in row:
            if 0 <= p < P:
                refs[p] += 1
    ints = lambda x: torch.as_tensor(x, dtype=torch.int32).to(DEV)  # noqa: E731
    return lisa.Pages(ints(table), ints(lens), ints(refs))


def random_cache(pages, Hkv, w, dk, fmt, g, nan=False):
    """Full of codes, as pages that were used before are; nan: with e4m3 NaN among them."""
    c = lisa.Cache8.empty(pages, Hkv, w, dk, fmt)
    for t in (c.k, c.v):
        if t is not None:
            b = torch.randint(0, 256, t.shape, generator=g, dtype=torch.uint8)
            if fmt == I8:
                b[b == 128] = 0
            else:
                b[(b & 0x7f) == 0x7f] = 0x7f if nan else 0
            t.view(torch.uint8).copy_(b)
    for t in (c.k_scale, c.v_scale):
        if t is not None:
            t.copy_(2.0 ** torch.randint(-7, -4, t.shape, generator=g).float())
    return c


def rand(shape, dtype, g, std=1.0):
    return (torch.randn(shape, generator=g) * std).to(dtype)


def same(cache, ref):
    got = cr.RefCache(cache)
    assert np.array_equal(got.v_scale, ref.v_scale) and np.array_equal(got.v, ref.v, equal_nan=True)
    if cache.width:
        assert np.array_equal(got.k_scale, ref.k_scale) and np.array_equal(got.k, ref.k, equal_nan=True)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hkv,w,dk,lens,counts,L", [
    (2, 22, 128, [1], None, 1),                              # the first token of all
    (8, 22, 128, [300, 64, 65, 128], None, 1),               # a step: inside a page, its last token, its first
    (3, 11, 64, [130, 70, 5, 0], [130, 3, 9, 2], 130),       # prompts, more counted than there are, an empty sequence
    (1, 128, 128, [200, 257], [137, 66], 140),               # a standard layer, from the middle of a page on
    (2, 256, 256, [70], None, 70),
    (2, 7, 24, [66, 1, 129], [2, 0, -3], 5),                 # nothing to do for some
    (2, 0, 128, [100, 64], [40, 64], 64),                    # values alone
    (40, 20, 128, [193], None, 193),
])
def test_append_equals_the_definition(Hkv, w, dk, lens, counts, L, dtype, fmt):
    g = torch.Generator().manual_seed(len(lens) * 1000 + L + w)
    B, C = len(lens), max(1, -(-max(lens) // 64))
    pages = make_pages(lens, B * C + 2, C, g)
    cache = random_cache(pages, Hkv, w, dk, FMT[fmt], g)
    ref = cr.RefCache(cache)
    k = rand((B, Hkv, L, w), dtype, g, 1.28) if w else None
    v = rand((B, Hkv, L, dk), dtype, g, 1.28)
    ref.append(pages.table.tolist(), lens, counts or [L] * B, k, v)
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV)
    kd, vd = k.to(DEV) if w else None, v.to(DEV)
    for _ in range(2):                                       # the call may be repeated
        lisa.lisa_cache8_append(cache, kd, vd, counts=cnt)
        torch.cuda.synchronize()
        assert lisa.last_path() == "cache8_append"
        same(cache, ref)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_passes_over_tokens_without_a_page_and_past_the_table(fmt):
    g = torch.Generator().manual_seed(3)
    lens = [200, 200, 190]
    pages = make_pages(lens, 16, 3, g, absent=[(0, 1), (1, 2), (2, 0), (2, 2)])   # (200 tokens need a fourth column)
    cache = random_cache(pages, 2, 22, 128, FMT[fmt], g)
    ref = cr.RefCache(cache)
    k, v = rand((3, 2, 200, 22), torch.bfloat16, g), rand((3, 2, 200, 128), torch.bfloat16, g)
    ref.append(pages.table.tolist(), lens, [200] * 3, k, v)
    lisa.lisa_cache8_append(cache, k.to(DEV), v.to(DEV))
    same(cache, ref)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_of_extreme_values(dtype, fmt):
    """Zeros, the borders of the scales, the smallest and largest numbers, infinities and NaN: blocks of their own, and in front
    of and behind ordinary tokens."""
    g = torch.Generator().manual_seed(5)
    top = torch.finfo(dtype).max
    kinds = [0.0, 127.0, 127.5, 448.0, 450.0, 1.0, -2.0 ** -126, 2.0 ** -133, top, -top, math.inf, -math.inf, math.nan, 63.5, 224.0, 1e-30]
    v = torch.zeros((len(kinds), 1, 3, 64)).to(dtype)
    k = torch.zeros((len(kinds), 1, 3, 22)).to(dtype)
    for b, x in enumerate(kinds):
        v[b, 0, 0, b] = k[b, 0, 1, b] = x
        v[b, 0, 2, 5:9] = torch.tensor([x, -x / 3, x / 7, 0.3])
        k[b, 0, 2, 3:5] = torch.tensor([x / 5, -0.7])
    for lens in ([3] * len(kinds), [40] * len(kinds), [66] * len(kinds)):   # a fresh page, into one, over its end
        pages = make_pages(lens, 2 * len(kinds), 2, g)
        cache = random_cache(pages, 1, 22, 64, FMT[fmt], g)
        ref = cr.RefCache(cache)
        ref.append(pages.table.tolist(), lens, [3] * len(kinds), k, v)
        lisa.lisa_cache8_append(cache, k.to(DEV), v.to(DEV))
        same(cache, ref)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_scales_that_grow_token_by_token_keep_the_values(fmt):
    """64 tokens, each 12 % larger than the one before, appended one by one: what is stored is within one step of the final
    scale of what was appended (e4m3: one step of its binade, the smallest steps those of the final scale)."""
    g = torch.Generator().manual_seed(9)
    pages = lisa.Pages.empty(2, 1, 1, DEV)
    cache = lisa.Cache8.empty(pages, 1, 22, 128, FMT[fmt])
    xk = (rand((64, 22), torch.float32, g) * 1.12 ** torch.arange(64)[:, None]).bfloat16()
    xv = (rand((64, 128), torch.float32, g) * 1.12 ** torch.arange(64)[:, None]).bfloat16()
    one = torch.ones(1, dtype=torch.int32, device=DEV)
    for t in range(64):
        lisa.lisa_pages_grow(pages, one)
        lisa.lisa_cache8_append(cache, xk[t][None, None, None].to(DEV), xv[t][None, None, None].to(DEV))
    ref = cr.RefCache(cache)
    for name, x in (("k", xk), ("v", xv)):
        s = getattr(ref, name + "_scale")[0, 0]
        got, want = getattr(ref, name)[0, 0][:, :x.shape[1]] * s, cr.values(x)
        step = s if fmt == "int8" else np.maximum(2.0 ** (np.floor(np.log2(np.abs(want) + 1e-300)) - 3), s * 2.0 ** -9)
        assert np.abs(got - want).max() > 0 and np.all(np.abs(got - want) <= step)


MIX = {"add": lisa.MIX_ADD, "concat": lisa.MIX_CONCAT, "plus": lisa.MIX_PLUS, "share": lisa.MIX_SHARE}
ACT = {"relu": lisa.ACT_RELU, "silu": lisa.ACT_SILU, "single": lisa.ACT_SINGLE}


def check_decode(g, fmt, dtype, H, Hkv, dk, w, F, mix, act, lens, Lk=None, absent=(), out_dtype=None, write=True, nan=False, q_std=1.28,
                 prev=None, B=None):
    S, Lk = len(lens), Lk or max(max(lens), 1)
    B = B or S
    C = max(1, -(-max(max(lens), Lk) // 64))
    P = sum(-(-n // 64) for n in lens) + 2
    pages = make_pages(lens, P, C, g, absent)
    cache = random_cache(pages, Hkv, w if mix != "share" else 0, dk, fmt, g, nan)
    if nan:                                                  # NaN only behind the ends
        for s, n in enumerate(lens):
            for c in range(C):
                p = int(pages.table[s, c])
                if 0 <= p < P:
                    m = max(0, min(64, n - 64 * c))
                    for t in (cache.k, cache.v):
                        if t is not None:
                            x = t.view(torch.uint8)[p]
                            part = x[:, :, :m] if t is cache.k else x[:, :, :m]
                            part[(part & 0x7f) == 0x7f] = 0
                            if t is cache.k:
                                x[:, :, m:] = 0x7f
                            else:
                                x[:, :, m:] = 0x7f
    sdt = lisa.score_dtype(dtype)
    q = rand((B, H, w), dtype, g, q_std) if mix != "share" else None
    row = None
    if mix != "std":
        row = prev if prev is not None else rand((B, H, Lk), torch.float32, g).to(sdt)
        for b in range(B):
            row[b, :, max(0, min(lens[b], Lk)):] = math.nan  # not to be read
    Din = 2 * H if mix == "concat" else H
    if act == "single":
        F = H
    w1 = rand((Din, F), dtype, g, 1 / math.sqrt(Din)) if mix in ("add", "concat") else None
    w2 = rand((F, H), dtype, g, 1 / math.sqrt(F)) if mix in ("add", "concat") and act != "single" else None
    ref = cr.RefCache(cache)
    want = cr.decode(ref, pages.table.tolist()[:B], lens[:B], Lk, q, row, w1, w2, mix, act, 1 / math.sqrt(w), dk, H)
    d = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    rows = torch.full((B, H, Lk), 7.0, dtype=sdt, device=DEV)
    if mix == "std":
        got_row, out = lisa.std_attn_decode8(d(q), cache, Lk, want_scores=write, score_row_out=rows if write else None, out_dtype=out_dtype)
    else:
        out, got_row = lisa.lisa_attn_decode8(d(q), cache, d(row), d(w1), d(w2), mix=MIX[mix], act=ACT[act], write_scores=write,
                                              score_row_out=rows if write else None, out_dtype=out_dtype)
    torch.cuda.synchronize()
    assert (got_row is not None) == write
    odt = out_dtype or torch.float32
    worst_r = worst_o = 0.0
    for b, (a, o, there, rb, ob) in enumerate(want):
        n = len(there)
        if write:
            r = cr.values(got_row[b])
            seen = np.zeros(Lk, dtype=bool)
            seen[:n] = there
            assert np.all(r[:, ~seen] == 7.0)                # not written
            lim = 65504.0 if sdt == torch.float16 else np.inf
            err = np.abs(r[:, :n] - np.clip(a, -lim, lim))[:, there]
            tol = (rb + 2.0 ** -25)[:, there]
            assert np.all(err <= tol), (b, float((err / tol).max()))
            worst_r = max(worst_r, float((err / tol).max(initial=0)))
        x = cr.values(out[b])
        tol = ob + np.abs(o) * (torch.finfo(odt).eps / 2) + 1e-30
        err = np.abs(x - o)
        assert np.all(err <= tol), (b, float((err / tol).max()))
        worst_o = max(worst_o, float((err / tol).max()))
        if not there.any():
            assert np.all(x == 0)
    print(f"[decode8] {lisa.last_path()} {mix}/{act} H{H}/{Hkv} dk{dk} w{w} F{F} {fmt} {dtype} lens {lens[:6]}: rows {worst_r:.2f}, out {worst_o:.2f} of the bound",
          flush=True)


SHAPES = [  # H, Hkv, dk, w, F
    (32, 8, 128, 22, 64),
    (32, 32, 128, 22, 64),
    (40, 40, 128, 22, 80),
    (8, 8, 64, 11, 32),
    (6, 2, 40, 9, 20),
    (16, 1, 128, 32, 100),
    (12, 4, 128, 20, 33),
    (64, 8, 128, 40, 128),
]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("mix,act", [("add", "relu"), ("concat", "relu"), ("add", "silu"), ("concat", "silu"), ("add", "single"), ("concat", "single"),
                                     ("plus", "relu"), ("share", "relu")])
def test_lisa_decode8(mix, act, shape, fmt):
    H, Hkv, dk, w, F = shape
    g = torch.Generator().manual_seed(H + dk + w)
    check_decode(g, FMT[fmt], torch.bfloat16, H, Hkv, dk, w, F, mix, act, [1, 130, 0, 64, 65, 191])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", [(32, 8, 128, 128, 0), (32, 32, 128, 128, 0), (40, 40, 128, 128, 0), (8, 8, 64, 64, 0), (6, 2, 40, 40, 0), (16, 1, 128, 128, 0),
                                   (20, 4, 128, 128, 0), (2, 1, 256, 256, 0)])
@pytest.mark.parametrize("write", [True, False])
def test_std_decode8(write, shape, fmt):
    H, Hkv, dk, w, _ = shape
    g = torch.Generator().manual_seed(H + dk)
    check_decode(g, FMT[fmt], torch.bfloat16, H, Hkv, dk, w, 0, "std", "relu", [1, 130, 0, 64, 65, 191], write=write)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("mix", ["add", "concat", "std", "plus", "share"])
def test_float32_decode8(mix, fmt):
    g = torch.Generator().manual_seed(2)
    check_decode(g, FMT[fmt], torch.float32, 8, 4, 64, 64 if mix == "std" else 11, 32, mix, "relu", [1, 0, 63, 200])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("mix", ["add", "std"])
@pytest.mark.parametrize("lens", [[5000], [1, 8200], [4097, 64, 4096, 1], [700] * 9, [90] * 40, [2049, 1000, 3000]])
def test_decode8_of_long_and_many_sequences(lens, mix, fmt):
    g = torch.Generator().manual_seed(len(lens))
    for H, Hkv in ((8, 2), (8, 8)):
        check_decode(g, FMT[fmt], torch.bfloat16, H, Hkv, 128, 128 if mix == "std" else 22, 16, mix, "relu", lens, write=False)


@pytest.mark.parametrize("mix", ["add", "share", "std"])
@pytest.mark.parametrize("H,Hkv,dk,lens,absent", [
    (2, 1, 64, [36000], ()),                                 # more spans than a wave has lanes
    (4, 1, 128, [1500, 40], [(0, c) for c in range(8)]),     # a span without a page, spans behind a sequence's end
    (16, 2, 128, [150, 1], ()),                              # eight heads per kv head, features dealt to two workgroups
    (8, 8, 128, [1100] * 16, ()),                            # features dealt to two workgroups of all pages
    (8, 8, 64, [90] * 70, ()),                               # many short sequences: four waves
    (8, 8, 64, [2100] * 64, ()),                             # many of more than 32 pages: eight
])
def test_decode8_however_the_work_is_dealt(H, Hkv, dk, lens, absent, mix):
    g = torch.Generator().manual_seed(dk + len(lens))
    check_decode(g, I8, torch.bfloat16, H, Hkv, dk, dk if mix == "std" else 22, 16, mix, "relu", lens, absent=absent)


@pytest.mark.parametrize("mix", ["add", "concat", "share", "std"])
@pytest.mark.parametrize("shape", [(32, 8, 128, 22, 64), (6, 2, 40, 9, 20)])
def test_decode8_over_missing_pages_and_with_nan_behind_the_ends(shape, mix):
    H, Hkv, dk, w, F = shape
    g = torch.Generator().manual_seed(8)
    w = dk if mix == "std" else w
    check_decode(g, E4, torch.bfloat16, H, Hkv, dk, w, F, mix, "relu", [150, 130, 33, 320], absent=[(0, 1), (1, 0), (2, 0), (3, 4), (3, 0)], nan=True)


@pytest.mark.parametrize("mix", ["add", "std"])
@pytest.mark.parametrize("shape", [(32, 8, 128, 22, 64), (6, 2, 40, 9, 20)])
def test_rows_wider_and_narrower_than_the_sequences(shape, mix):
    H, Hkv, dk, w, F = shape
    w = dk if mix == "std" else w
    g = torch.Generator().manual_seed(8)
    check_decode(g, I8, torch.bfloat16, H, Hkv, dk, w, F, mix, "relu", [150, 64, 7], Lk=333, out_dtype=torch.bfloat16)
    check_decode(g, I8, torch.bfloat16, H, Hkv, dk, w, F, mix, "relu", [150, 64, 7], Lk=65)     # (the first 65 tokens)
    check_decode(g, I8, torch.bfloat16, H, Hkv, dk, w, F, mix, "relu", [150, 64, 7], B=2)       # (the first two sequences)


@pytest.mark.parametrize("shape", [(32, 8, 128, 22, 64), (6, 2, 40, 9, 20)])
@pytest.mark.parametrize("mix", ["share", "plus"])
def test_scores_masked_with_minus_infinity(mix, shape):
    """A layer without an alignment module hands masks on: masked keys weigh nothing, a row masked throughout gives zeros."""
    H, Hkv, dk, w, F = shape
    g = torch.Generator().manual_seed(4)
    prev = torch.randn((2, H, 130), generator=g).half()
    prev[0, :, 3:90] = -math.inf
    prev[0, 1] = -math.inf
    prev[1, 0, :64] = -math.inf
    lens = [130, 100]
    pages = make_pages(lens, 6, 3, g)
    cache = random_cache(pages, Hkv, w if mix == "plus" else 0, dk, I8, g)
    q = rand((2, H, w), torch.bfloat16, g) if mix == "plus" else None
    out, row = lisa.lisa_attn_decode8(None if q is None else q.to(DEV), cache, prev.to(DEV), None, None, mix=MIX[mix])
    ref = cr.RefCache(cache)
    for b, n in enumerate(lens):
        for h in range(H):
            a = cr.values(prev[b, h, :n])
            if mix == "plus":
                k, _ = ref.tokens("k", pages.table.tolist()[b], n, h // (H // Hkv))
                a = a + k @ cr.values(q[b, h]) / math.sqrt(w)
            v, _ = ref.tokens("v", pages.table.tolist()[b], n, h // (H // Hkv))
            got = cr.values(out[b, h])
            if np.isneginf(a).all():
                assert np.all(got == 0)
                continue
            p = np.exp(a - a.max())
            # scores in float32 from exact products, probabilities to 2^-11
            assert np.all(np.abs(got - p @ v / p.sum()) <= (2.0 ** -10 * (p @ np.abs(v)) + 2.0 ** -15 * np.abs(v).sum(0)) / p.sum())
            r = cr.values(row[b, h, :n])
            fin = np.isfinite(a)
            assert np.all(np.abs(r[fin] - a[fin]) <= 2.0 ** -11 * np.abs(a[fin]) + 2.0 ** -20)
            assert np.all(r[~fin] <= -65504.0)


@pytest.mark.parametrize("q_std", [1e-30, 1e-3, 1e4])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_queries_of_any_size(fmt, q_std):
    g = torch.Generator().manual_seed(6)
    for mix, w in (("std", 128), ("plus", 22)):
        check_decode(g, FMT[fmt], torch.bfloat16, 8, 4, 128, w, 0, mix, "relu", [130, 3], q_std=q_std)
