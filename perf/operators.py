"""Timed cases of the paged 8-bit cache: appending tokens to it, a decode step's attention over it (LiSA layer and
standard layer), and what a server does with its pages (giving, forking, freeing, compacting, copying).

``listed()`` holds the fixed cases, ``draw()`` further ones of the same ranges, ``prepare()`` makes what a program has in
hand before the call, ``run()`` is one pass, ``work()`` the bytes and operations that a pass cannot do without,
``exact()`` the outputs in 64 bits. With ``own`` false ``run()`` computes the operators with elementary operations of
torch, with ``own`` true it calls the library.

The cache. A page holds 64 tokens of one layer. Per page and key/value head:
  k        [ceil(w / 8), 64, 8]  8-bit codes of the key rows (w = r in a LiSA layer, d_k in a standard one), features in
                                 pieces of 8, the last piece filled up with zeros
  v        [d_k, 64]             8-bit codes of the value rows
  k_scale, v_scale               a power of two: a code c stands for c * scale
Codes are whole numbers -127 .. 127 (torch.int8) or e4m3 numbers (torch.float8_e4m3fn); they are returned as such, with
their scales. ``table[s, c]`` is the page of tokens 64 c .. 64 c + 63 of sequence s, ``lens[s]`` the tokens it has,
``refs[p]`` the number of table entries that name page p (0: free).

Shapes are the LLaMA2-7B, LLaMA3-8B and LLaMA2-13B layers of ``synth.py``; the alignment FFN is identity-like plus noise.
"""
import math

import torch

own = False

DEV = "cuda"
PAGE = 64
#        query heads, key/value heads, head dimension, r, F of the alignment FFN
SHAPES = {"7b": (32, 32, 128, 22, 64), "8b": (32, 8, 128, 22, 64), "13b": (40, 40, 128, 22, 80)}
TOP = {"int8": 127.0, "e4m3": 448.0}


def listed():
    return [
        # One user's next token goes into a layer's cache: the smallest call of a serving loop, latency alone.
        {"name": "append_8b_b1_step", "op": "append", "model": "8b", "layer": "lisa", "fmt": "int8", "B": 1, "old": 300, "new": 1},
        # Prompts of several users, of different lengths, behind what their caches hold already.
        {"name": "append_7b_b6_prompts", "op": "append", "model": "7b", "layer": "std", "fmt": "e4m3", "B": 6, "old": 37, "new": 1500},
        # One user's chat, short context: a LiSA layer's attention for one new token.
        {"name": "lisa_8b_b1_ctx300", "op": "lisa", "model": "8b", "module": "add", "fmt": "int8", "B": 1, "ctx": 300},
        # A few users on the paper's default module (concatenation, 2h -> 256 -> h).
        {"name": "lisa_concat_7b_b8_ctx2500", "op": "lisa", "model": "7b", "module": "concat", "fmt": "e4m3", "B": 8, "ctx": 2500},
        # A full batch at a long context: the stream of the caches.
        {"name": "lisa_7b_b64_ctx4097", "op": "lisa", "model": "7b", "module": "add", "fmt": "int8", "B": 64, "ctx": 4097},
        # A standard layer that hands its score row on, an ordinary context.
        {"name": "std_7b_b4_ctx1023", "op": "std", "model": "7b", "fmt": "int8", "B": 4, "ctx": 1023, "row": True},
        # Grouped heads, long contexts, no layer behind that shares the scores.
        {"name": "std_8b_b32_ctx8192", "op": "std", "model": "8b", "fmt": "e4m3", "B": 32, "ctx": 8192, "row": False},
        # Sequences that have ended give their pages back, new prompts take theirs.
        {"name": "turnover_s64_p8192", "op": "turnover", "seqs": 64, "pages": 8192, "ctx": 4000},
        # Four continuations of one prompt: the prompt's last page is copied in every layer, the others are shared.
        {"name": "fork_8b_4_of_1000", "op": "fork", "model": "8b", "layers": 8, "seqs": 8, "pages": 256, "ctx": 1000, "children": 4},
        # Beams of many users at once.
        {"name": "fork_7b_48_of_3000", "op": "fork", "model": "7b", "layers": 12, "seqs": 64, "pages": 1024, "ctx": 3000, "children": 48},
        # A pool that ended sequences have left full of holes is made dense at its front.
        {"name": "compact_8b_p600", "op": "compact", "model": "8b", "layers": 4, "seqs": 24, "pages": 600, "ctx": 1900},
        {"name": "compact_8b_p3001", "op": "compact", "model": "8b", "layers": 12, "seqs": 72, "pages": 3001, "ctx": 4000},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "lisa", "lisa", "lisa", "std", "std", "turnover", "fork", "compact"])
    model = rng.choice(["7b", "8b", "13b"])
    fmt = rng.choice(["int8", "e4m3"])
    if op == "append":
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 4000)
        B = _log_int(rng, 1, max(1, min(64, 9000 // new)))
        return {"op": op, "model": model, "layer": rng.choice(["lisa", "std"]), "fmt": fmt, "B": B, "old": rng.randint(0, 500), "new": new}
    if op in ("lisa", "std"):
        H, Hkv = SHAPES[model][:2]
        ctx = _log_int(rng, 1, 8192)
        B = _log_int(rng, 1, max(1, min(64, 260000 * 32 // (H * ctx) if op == "lisa" else 260000 * 8 // (Hkv * ctx))))
        if op == "lisa":
            return {"op": op, "model": model, "module": rng.choice(["add", "concat"]), "fmt": fmt, "B": B, "ctx": ctx}
        return {"op": op, "model": model, "fmt": fmt, "B": B, "ctx": ctx, "row": rng.random() < 0.5}
    if op == "turnover":
        seqs, ctx = _log_int(rng, 2, 256), _log_int(rng, 20, 6000)
        return {"op": op, "seqs": seqs, "pages": seqs * (ctx // PAGE + 1) + rng.randint(1, 4000), "ctx": ctx}
    if op == "fork":
        seqs, ctx = rng.randint(2, 64), _log_int(rng, 40, 3000)
        children = rng.randint(1, max(1, seqs - 1))
        return {"op": op, "model": "8b", "layers": rng.randint(1, 12), "seqs": seqs, "pages": seqs * (ctx // PAGE + 1) + children + rng.randint(1, 40),
                "ctx": ctx, "children": min(children, seqs - 1)}
    seqs, ctx = rng.randint(4, 60), _log_int(rng, 60, 2500)
    return {"op": op, "model": "8b", "layers": rng.randint(1, 12), "seqs": seqs, "pages": seqs * (ctx // PAGE + 1) + rng.randint(1, 100), "ctx": ctx}


# ---- sizes of a case ----------------------------------------------------------------------------
def _dims(case):
    """H, Hkv, d_k, width of the key rows, F"""
    H, Hkv, dk, r, F = SHAPES[case["model"]]
    if case.get("module") == "concat":                       # the paper's widths
        r, F = 20, 256
    std = case["op"] == "std" or case.get("layer") == "std"
    return H, Hkv, dk, dk if std else r, F


def _lens(n, ctx):
    """Tokens of n sequences: different, the first has ctx, all at least half of that."""
    return [ctx - (37 * s * s + 11 * s) % max(1, (ctx + 1) // 2) for s in range(n)]


def _counts(case):
    """New tokens of each sequence of an append."""
    return [1 if case["new"] == 1 else n for n in _lens(case["B"], case["new"])]


def _pages(n):
    return (n + PAGE - 1) // PAGE


# ---- inputs ---------------------------------------------------------------------------------------
def _codes(shape, fmt, std, g):
    """Codes of normally distributed values, `std` steps wide."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float16) * std
    return x.round_().clamp_(-127, 127).to(torch.int8) if fmt == "int8" else x.clamp_(-448, 448).to(torch.float8_e4m3fn)


def _pool(pages, Hkv, w, dk, fmt, g):
    """A layer's pool of pages full of tokens: rows of unit scale, quantised."""
    kp = (w + 7) // 8
    k = _codes((pages, Hkv, kp, PAGE, 8), fmt, 24.0, g)
    if w % 8:
        k[:, :, -1, :, w % 8:] = 0
    scale = [torch.pow(2.0, torch.randint(-6, -3, (pages, Hkv), generator=g, device=DEV, dtype=torch.float32)) for _ in range(2)]
    return {"k": k, "k_scale": scale[0], "v": _codes((pages, Hkv, dk, PAGE), fmt, 24.0, g), "v_scale": scale[1]}


def _table(lens, columns, pages, g):
    """A page table whose pages lie anywhere in the pool, and how often each page is named."""
    ids = torch.randperm(pages, generator=g, device=DEV, dtype=torch.int32)
    n = torch.tensor([_pages(x) for x in lens], device=DEV)
    at = torch.cumsum(n, 0)[:, None] - n[:, None] + torch.arange(columns, device=DEV)[None]
    there = torch.arange(columns, device=DEV)[None] < n[:, None]
    table = torch.where(there, ids[at.clamp(max=pages - 1)], -1).to(torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    refs.index_add_(0, table[there].long(), torch.ones_like(table[there]))
    return table.contiguous(), refs


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    s = dict(case)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    normal = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    if case["op"] in ("append", "lisa", "std"):
        B, fmt = case["B"], case["fmt"]
        H, Hkv, dk, w, F = _dims(case)
        if case["op"] == "append":
            counts = _counts(case)
            lens = [o + n for o, n in zip([case["old"] * (b + 1) // B for b in range(B)], counts)]
        else:
            lens = _lens(B, case["ctx"])
        columns = _pages(max(lens))
        pages = sum(_pages(n) for n in lens) + 3
        s["table"], s["refs"] = _table(lens, columns, pages, g)
        s["lens"] = ints(lens)
        s.update(_pool(pages, Hkv, w, dk, fmt, g), w=w, Hkv=Hkv, H=H, dk=dk)
        if case["op"] == "append":
            s["counts"] = ints(counts)
            new = max(counts)
            s["k_new"], s["v_new"] = normal(B, Hkv, new, w).bfloat16(), normal(B, Hkv, new, dk).bfloat16()
            s["k_new"] *= 1.28
            s["v_new"] *= 1.28
            return s
        Lk = max(lens)
        s["Lk"] = Lk
        s["q"] = (1.28 * normal(B, H, w)).bfloat16()
        s["row_out"] = torch.zeros((B, H, Lk), dtype=torch.float16, device=DEV)
        if case["op"] == "lisa":
            s["row"] = normal(B, H, Lk).half()
            din = 2 * H if case["module"] == "concat" else H
            w1, w2 = 0.02 * normal(din, F), 0.02 * normal(F, H)
            eye = torch.eye(H, device=DEV)
            w1[:H, :H] += eye
            w1[:H, H:2 * H] -= eye
            w2[:H] += eye
            w2[H:2 * H] -= eye
            if case["module"] == "concat" and F >= 4 * H:    # the correction passes through too
                w1[H:, 2 * H:3 * H] += eye
                w1[H:, 3 * H:4 * H] -= eye
                w2[2 * H:3 * H] += eye
                w2[3 * H:4 * H] -= eye
            s["w1"], s["w2"] = w1.bfloat16(), w2.bfloat16()
        return s
    S, P = case["seqs"], case["pages"]
    lens = _lens(S, case["ctx"])
    columns = _pages(case["ctx"] + 1)
    if case["op"] == "turnover":
        ended = list(range(1, S, 4)) if S > 1 else [0]
        s["ended"] = ints(ended)
        kept = [0 if i in ended else n for i, n in enumerate(lens)]
        s["add"] = ints([n if i in ended else 0 for i, n in enumerate(lens)])
        s["table"], s["refs"] = _table(kept, columns, P, g)
        s["lens"] = ints(kept)
        _grow(s, s["add"])                                   # (the pages that a turn gives them: every pass finds what the one before left)
        return s
    if case["op"] == "fork":
        n = min(case["children"], S - 1)
        live = S - n
        lens = [x if i < live else 0 for i, x in enumerate(lens)]
        s["src"] = ints([i * i % live for i in range(n)])
        s["dst"] = ints([S - 1 - i for i in range(n)])
        s["add"] = ints([0 if i < live else 1 for i in range(S)])
    else:
        lens = [x if i % 3 != 1 else 0 for i, x in enumerate(lens)]     # every third sequence has ended
    s["table"], s["refs"] = _table(lens, columns, P, g)
    s["lens"] = ints(lens)
    _, Hkv, dk, r, _ = SHAPES[case["model"]]
    s.update(Hkv=Hkv, dk=dk, w=r)
    s["pools"] = [_pool(P, Hkv, r, dk, "int8", g) for _ in range(case["layers"])]
    if case["op"] == "compact":
        s["table0"], s["refs0"] = s["table"].clone(), s["refs"].clone()
    return s


# ---- plain forms ------------------------------------------------------------------------------------
def _round_e4m3(x):
    """x (within +-448) to the nearest e4m3 number, ties to even."""
    step = torch.exp2(torch.frexp(x)[1].clamp(min=-5).float() - 4)
    return torch.round(x / step) * step


def _exponent(m, top):
    """The smallest e >= -126 with m <= top * 2^e."""
    e = torch.frexp(m)[1] - math.frexp(top)[1]
    return (e + (torch.ldexp(torch.full_like(m, top), e) < m)).clamp(min=-126)


def _append(s, k_new, v_new, counts):
    """The last counts[b] tokens of every sequence go into its pages; scales grow where they have to."""
    lens, table, fmt = s["lens"].long(), s["table"], s["fmt"]
    B, Hkv, N, w = k_new.shape
    at = (lens - counts)[:, None] + torch.arange(N, device=DEV)[None]                 # position of every row
    there = torch.arange(N, device=DEV)[None] < counts[:, None]
    first = (lens - counts) // PAGE                                                   # page columns that the call touches
    span = (N + PAGE - 2) // PAGE + 1
    col = first[:, None] + torch.arange(span, device=DEV)[None]
    touched = (col * PAGE < lens[:, None]) & (counts[:, None] > 0)
    page = torch.gather(table, 1, col.clamp(max=table.shape[1] - 1)).long()
    rel = torch.where(there, at - first[:, None] * PAGE, span * PAGE)                 # (rows that do not count go behind the end)
    grid = lambda: torch.zeros((B, span * PAGE + 1), device=DEV)  # noqa: E731
    fresh = grid().scatter_(1, rel, 1.0)[:, :-1].view(B, span, 1, PAGE) > 0           # tokens of this call
    pos = col[:, :, None, None] * PAGE + torch.arange(PAGE, device=DEV)
    kept = (pos < (lens - counts)[:, None, None, None]).expand(B, span, 1, PAGE)      # tokens that were there before
    begun = (col * PAGE < (lens - counts)[:, None])[:, :, None]
    for name, new in (("k", k_new), ("v", v_new)):
        code, scale = s[name], s[name + "_scale"]
        x = torch.zeros((B, Hkv, span * PAGE + 1, new.shape[3]), device=DEV)
        x = x.scatter_(2, rel[:, None, :, None].expand(B, Hkv, N, new.shape[3]), new.float())[:, :, :-1]
        x = x.view(B, Hkv, span, PAGE, -1).transpose(1, 2)                            # [B, span, Hkv, PAGE, width]
        m = (x.abs() * fresh[..., None]).amax((3, 4))
        old = scale[page]
        now = torch.ldexp(torch.ones_like(m), _exponent(m, TOP[fmt]))
        now = torch.where(begun, torch.maximum(old, now), now)
        was = code[page].float()
        was = was.transpose(3, 4) if name == "v" else was.transpose(3, 4).reshape(B, span, Hkv, PAGE, -1)[..., :new.shape[3]]
        x = torch.where(kept[..., None], was * old[..., None, None], x)
        y = x / now[..., None, None]
        y = torch.round(y).clamp(-127, 127) if fmt == "int8" else _round_e4m3(y.clamp(-448, 448))
        y = torch.where((kept | fresh)[..., None], y, was)                            # tokens behind the end stay
        if name == "v":
            y = y.transpose(3, 4)
        else:
            y = torch.nn.functional.pad(y, (0, -w % 8)).view(B, span, Hkv, PAGE, -1, 8).transpose(3, 4)
        code.view(torch.int8).index_put_((page[touched],), y.to(code.dtype)[touched].contiguous().view(torch.int8))
        scale.index_put_((page[touched],), now[touched])
    return s["k"], s["k_scale"], s["v"], s["v_scale"]


def _tokens(s, name):
    """Keys [B, Hkv, columns * PAGE, w] or values [B, Hkv, columns * PAGE, d_k] of all sequences."""
    page = s["table"].clamp(min=0).long()
    x = s[name].view(torch.int8)[page].view(s[name].dtype).float() * s[name + "_scale"][page][..., None, None, None] if name == "k" else \
        s[name].view(torch.int8)[page].view(s[name].dtype).float() * s[name + "_scale"][page][..., None, None]
    B, C, Hkv = x.shape[:3]
    if name == "v":
        return x.permute(0, 2, 1, 4, 3).reshape(B, Hkv, C * PAGE, -1)
    return x.permute(0, 2, 1, 4, 3, 5).reshape(B, Hkv, C * PAGE, -1)[..., :s["w"]]


def _attend(s):
    """Scores of a layer, its softmax over a sequence's tokens and P V; the score row in half."""
    B, H, Lk, Hkv = s["B"], s["H"], s["Lk"], s["Hkv"]
    q = s["q"].float().view(B, Hkv, H // Hkv, s["w"])
    a = torch.matmul(_tokens(s, "k")[:, :, :Lk], q.transpose(2, 3).contiguous()).transpose(2, 3).reshape(B, H, Lk) / math.sqrt(s["w"])
    if s["op"] == "lisa":
        x = torch.where(torch.arange(Lk, device=DEV) < s["lens"][:, None, None], s["row"].float(), 0.0)
        if s["module"] == "concat":
            x = torch.cat([x, a], 1)
        hid = torch.relu(torch.matmul(x.transpose(1, 2).contiguous(), s["w1"].float()))
        y = torch.matmul(hid, s["w2"].float()).transpose(1, 2)
        a = y if s["module"] == "concat" else y + a
    there = torch.arange(Lk, device=DEV) < s["lens"][:, None, None]
    p = torch.where(there, a, -math.inf)
    p = torch.exp(p - p.amax(2, keepdim=True))
    o = torch.matmul(p.view(B, Hkv, H // Hkv, Lk), _tokens(s, "v")[:, :, :Lk]).view(B, H, -1) / p.sum(2, keepdim=True)
    return o.bfloat16(), torch.where(there, a, 0.0).clamp(-65504, 65504).half()


def _by_rank(mark):
    """The indices at which `mark` is set, in ascending order, and behind them -1."""
    n = mark.numel()
    rank = torch.where(mark, torch.cumsum(mark, 0) - 1, n)
    return torch.full((n + 1,), -1, device=DEV, dtype=torch.int64).scatter_(0, rank, torch.arange(n, device=DEV))[:n]


def _grow(s, add):
    """Sequence i is given add[i] more tokens and the pages they need, in order of i, the free pages in ascending order."""
    table, lens, refs = s["table"], s["lens"], s["refs"]
    S, C = table.shape
    want = lens + add
    have, need = (lens + PAGE - 1) // PAGE, (want + PAGE - 1) // PAGE
    fits = (add >= 0) & (want <= C * PAGE)
    more = torch.where(fits, need - have, 0)
    upto = torch.cumsum(more, 0)
    free = refs == 0
    done = fits & ((more == 0) | (upto <= free.sum()))
    ids = _by_rank(free)
    c = torch.arange(C, device=DEV)[None]
    new = done[:, None] & (c >= have[:, None]) & (c < need[:, None])
    pick = (upto - more)[:, None] + c - have[:, None]
    table.copy_(torch.where(new, ids[pick.clamp(0, ids.numel() - 1)], table.long()))
    refs.index_add_(0, torch.where(new, table, 0).flatten().long(), new.flatten().to(torch.int32))
    lens.copy_(torch.where(done, want, lens))
    return done.to(torch.int32)


def _first(i, n, good):
    """Which entries of i are the first to name their sequence (of n) among those that `good` marks."""
    k = torch.arange(i.numel(), device=DEV)
    at = torch.full((n,), i.numel(), device=DEV).scatter_reduce_(0, i.clamp(0, n - 1).long(), torch.where(good, k, i.numel()), "amin")
    return good & (at[i.clamp(0, n - 1).long()] == k)


def _free(s, seqs):
    """The sequences give their pages back."""
    table, lens, refs = s["table"], s["lens"], s["refs"]
    S, C = table.shape
    done = _first(seqs, S, (seqs >= 0) & (seqs < S))
    gone = torch.zeros(S, dtype=torch.int32, device=DEV).index_add_(0, seqs.clamp(0, S - 1).long(), done.to(torch.int32)) > 0
    drop = gone[:, None] & (table >= 0) & (torch.arange(C, device=DEV)[None] < (lens[:, None] + PAGE - 1) // PAGE)
    refs.index_add_(0, torch.where(drop, table, 0).flatten().long(), -drop.flatten().to(torch.int32))
    table.copy_(torch.where(gone[:, None], -1, table))
    lens.copy_(torch.where(gone, 0, lens))
    return done.to(torch.int32)


def _fork(s, src, dst):
    """Sequence dst[i] becomes what src[i] is: the same pages but for a last one that is not full, which is copied."""
    table, lens, refs = s["table"], s["lens"], s["refs"]
    S, C = table.shape
    a, b = src.clamp(0, S - 1).long(), dst.clamp(0, S - 1).long()
    good = (src >= 0) & (src < S) & (dst >= 0) & (dst < S) & (src != dst) & (lens[b] == 0)
    good = _first(dst, S, good)
    n = lens[a]
    part = good & (n % PAGE != 0)
    upto = torch.cumsum(part, 0)
    free = refs == 0
    done = good & (~part | (upto <= free.sum()))
    part = part & done
    ids = _by_rank(free)
    new = torch.where(part, ids[(upto - 1).clamp(0, ids.numel() - 1)], -1)
    last = torch.where(part, torch.gather(table[a], 1, (n // PAGE).clamp(max=C - 1)[:, None].long())[:, 0], -1)
    c = torch.arange(C, device=DEV)[None]
    share = done[:, None] & (c < (n // PAGE)[:, None])
    rows = torch.where(share, table[a], -1)
    rows = torch.where(part[:, None] & (c == (n // PAGE)[:, None]), new[:, None].to(torch.int32), rows)
    refs.index_add_(0, rows.clamp(min=0).flatten().long(), (rows >= 0).flatten().to(torch.int32))
    at = torch.where(done, b, S)
    table.copy_(torch.cat([table, table[:1]]).index_copy_(0, at, rows)[:S])
    lens.copy_(torch.cat([lens, lens[:1]]).index_copy_(0, at, n)[:S])
    return done.to(torch.int32), torch.stack([last, new.to(torch.int32)], 1)


def _compact(s):
    """The used pages take the places 0 .. used - 1: those behind go, in order, to the free places in front."""
    table, refs = s["table"], s["refs"]
    P = refs.numel()
    i = torch.arange(P, device=DEV)
    used = refs > 0
    n = used.sum()
    source, target = _by_rank(used & (i >= n)), _by_rank(~used & (i < n))
    moved = source >= 0
    to = torch.cat([i, i[:1]]).scatter_(0, torch.where(moved, source, P), torch.where(moved, target, 0))
    was = refs.clone()
    refs.copy_(torch.where(i < n, was, 0))
    refs.scatter_reduce_(0, torch.where(moved, target, 0), torch.where(moved, was[source.clamp(min=0)], 0), "amax")
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], -1))
    return torch.stack([source, target], 1)[:P // 2].to(torch.int32)


def _copy(pools, copies):
    """Pages copies[i, 0] of every pool to pages copies[i, 1]; -1: nothing."""
    there = copies[:, 0] >= 0
    a, b = copies[there, 0].long(), copies[there, 1].long()
    for p in pools:
        for name in ("k", "k_scale", "v", "v_scale"):
            p[name].index_copy_(0, b, p[name][a])


# ---- one pass ---------------------------------------------------------------------------------------
def _handles(s):
    """What a program keeps of the library: the pages' state and the layers' caches, made of its tensors."""
    from paper_2408_01890_amd import lisa
    if "handles" not in s:
        pages = lisa.Pages(s["table"], s["lens"], s["refs"])
        s["handles"] = lisa, pages, [lisa.Cache8(pages, p["k"], p["k_scale"], p["v"], p["v_scale"], s["w"]) for p in s.get("pools", [s] if "k" in s else [])]
    return s["handles"]


def run(s):
    op = s["op"]
    if own:
        lisa, pages, caches = _handles(s)
    if op == "append":
        if own:
            lisa.lisa_cache8_append(caches[0], s["k_new"], s["v_new"], counts=s["counts"])
        else:
            _append(s, s["k_new"], s["v_new"], s["counts"])
        return s["k"], s["k_scale"], s["v"], s["v_scale"]
    if op == "lisa":
        if own:
            mix = lisa.MIX_CONCAT if s["module"] == "concat" else lisa.MIX_ADD
            return lisa.lisa_attn_decode8(s["q"], caches[0], s["row"], s["w1"], s["w2"], mix=mix, out_dtype=torch.bfloat16, score_row_out=s["row_out"])
        return _attend(s)
    if op == "std":
        if own:
            row, out = lisa.std_attn_decode8(s["q"], caches[0], s["Lk"], want_scores=s["row"], score_row_out=s["row_out"] if s["row"] else None, out_dtype=torch.bfloat16)
        else:
            out, row = _attend(s)
        return (out, row) if s["row"] else out
    state = s["table"], s["lens"], s["refs"]
    if op == "turnover":
        freed = lisa.lisa_pages_free(pages, s["ended"]) if own else _free(s, s["ended"])
        given = lisa.lisa_pages_grow(pages, s["add"]) if own else _grow(s, s["add"])
        return (freed, given, *state)
    if op == "fork":
        # the children live for one token and end: every pass finds what the one before found
        if own:
            done, copies = lisa.lisa_pages_fork(pages, s["src"], s["dst"])
            lisa.lisa_pages_copy(caches, copies)
            given = lisa.lisa_pages_grow(pages, s["add"])
            freed = lisa.lisa_pages_free(pages, s["dst"])
        else:
            done, copies = _fork(s, s["src"], s["dst"])
            _copy(s["pools"], copies)
            given = _grow(s, s["add"])
            freed = _free(s, s["dst"])
        return (done, copies, given, freed, *state, [[p[n] for n in ("k", "k_scale", "v", "v_scale")] for p in s["pools"]])
    # (a dense pool has nothing to move: a pass starts from the table and counts with the holes)
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    copies = lisa.lisa_pages_compact(pages) if own else _compact(s)
    lisa.lisa_pages_copy(caches, copies) if own else _copy(s["pools"], copies)
    return (copies, *state, [[p[n] for n in ("k", "k_scale", "v", "v_scale")] for p in s["pools"]])


# ---- what a pass cannot do without --------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op in ("append", "lisa", "std"):
        H, Hkv, dk, w, F = _dims(case)
        B, wp = case["B"], (w + 7) // 8 * 8
    if op == "append":                                       # bf16 rows in, codes and scales out
        n = sum(_counts(case))
        touched = sum(_pages(case["old"] * (b + 1) // B % PAGE + c) for b, c in enumerate(_counts(case)))
        return {"bytes": n * Hkv * (2 * (w + dk) + wp + dk) + touched * Hkv * 8, "flops": 2 * n * Hkv * (w + dk)}
    if op in ("lisa", "std"):
        lens = _lens(B, case["ctx"])
        n, pages = sum(lens), sum(_pages(x) for x in lens)
        rows = (2 if op == "lisa" else 0) + (2 if op == "lisa" or case["row"] else 0)
        ffn = 2 * ((2 if case.get("module") == "concat" else 1) * H * F + F * H) if op == "lisa" else 0
        return {"bytes": n * (Hkv * (wp + dk) + H * rows) + pages * (8 * Hkv + 4) + B * H * (2 * w + 2 * dk) + (ffn if op == "lisa" else 0),
                "flops": n * (2 * H * (w + dk) + ffn)}
    S, P, C = case["seqs"], case["pages"], _pages(case["ctx"] + 1)
    lens = _lens(S, case["ctx"])
    if op == "turnover":                                     # the ended sequences' table entries twice, the counts of the pages looked through
        n = sum(_pages(lens[i]) for i in (range(1, S, 4) if S > 1 else [0]))
        return {"bytes": 4 * (P + 6 * n + 4 * S), "flops": P + 2 * n}
    _, Hkv, dk, r, _ = SHAPES[case["model"]]
    page = case["layers"] * Hkv * ((r + 7) // 8 * 8 * PAGE + dk * PAGE + 8)
    if op == "fork":
        n = min(case["children"], S - 1)
        src = [i * i % (S - n) for i in range(n)]
        parts = sum(lens[i] % PAGE != 0 for i in src)
        return {"bytes": 2 * parts * page + 4 * (P + 6 * sum(_pages(lens[i]) for i in src) + 4 * S), "flops": P}
    used = sum(_pages(x) for i, x in enumerate(lens) if i % 3 != 1)
    moves = used * (P - used) // P                           # (the pages lie anywhere: as many of them behind the front as the share of holes)
    return {"bytes": 2 * moves * page + 4 * (2 * P + 2 * S * C + 2 * moves), "flops": P}


# ---- in 64 bits -----------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    table, lens = s["table"].tolist(), s["lens"].tolist()
    if op in ("lisa", "std"):
        H, Hkv, Lk, dk, w = s["H"], s["Hkv"], s["Lk"], s["dk"], s["w"]
        outs, rows = torch.zeros((s["B"], H, dk), dtype=torch.float64, device=DEV), torch.zeros((s["B"], H, Lk), dtype=torch.float64, device=DEV)
        for b, n in enumerate(lens):
            j = torch.arange(n, device=DEV)
            page = s["table"][b].long()[j // PAGE]
            for h in range(Hkv):
                heads = slice(h * H // Hkv, (h + 1) * H // Hkv)
                key = s["k"].view(torch.int8)[page, h, :, j % PAGE].contiguous().view(s["k"].dtype).double().reshape(n, -1)[:, :w] * s["k_scale"][page, h].double()[:, None]
                rows[b, heads, :n] = (s["q"][b, heads].double() @ key.T) / math.sqrt(w)
            if op == "lisa":
                x = s["row"][b, :, :n].double()
                if case["module"] == "concat":
                    rows[b, :, :n] = s["w2"].double().T @ (s["w1"].double().T @ torch.cat([x, rows[b, :, :n]])).clamp(min=0)
                else:
                    rows[b, :, :n] += s["w2"].double().T @ (s["w1"].double().T @ x).clamp(min=0)
            p = torch.softmax(rows[b, :, :n], 1)
            for h in range(Hkv):
                heads = slice(h * H // Hkv, (h + 1) * H // Hkv)
                val = s["v"].view(torch.int8)[page, h, :, j % PAGE].contiguous().view(s["v"].dtype).double() * s["v_scale"][page, h].double()[:, None]
                outs[b, heads] = p[heads] @ val
        return outs if op == "std" and not case["row"] else (outs, rows)
    if op == "append":
        top = TOP[case["fmt"]]
        out = {n: s[n].double() for n in ("k", "k_scale", "v", "v_scale")}
        for b, (n, c) in enumerate(zip(lens, s["counts"].tolist())):
            for col in range((n - c) // PAGE, _pages(n)):
                lo, hi, page = max(n - c, col * PAGE) - col * PAGE, min(n, (col + 1) * PAGE) - col * PAGE, table[b][col]
                row = col * PAGE + lo - (n - c)
                for name in ("k", "v"):
                    x = s[name + "_new"][b, :, row:row + hi - lo].double()                  # [Hkv, tokens, width]
                    m = x.abs().amax((1, 2)).clamp(min=2.0 ** -200)
                    scale = torch.exp2(torch.ceil(torch.log2(m / top)).clamp(min=-126))
                    old = out[name + "_scale"][page].clone()
                    if lo:
                        scale = torch.maximum(scale, old)
                    nearest = (lambda v: torch.round(v).clamp(-127, 127)) if case["fmt"] == "int8" else \
                        (lambda v: (lambda u: torch.round(v / u) * u)(torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)))
                    code = out[name][page].transpose(1, 2).reshape(x.shape[0], PAGE, -1) if name == "k" else out[name][page].transpose(1, 2).contiguous()
                    code[:, :lo] = nearest(code[:, :lo] * (old / scale)[:, None, None])
                    code[:, lo:hi, :x.shape[2]] = nearest(x / scale[:, None, None])
                    out[name][page] = code.view(x.shape[0], PAGE, -1, 8).transpose(1, 2) if name == "k" else code.transpose(1, 2)
                    out[name + "_scale"][page] = scale
        whole = case["fmt"] == "int8"
        return tuple(out[n].to(torch.int64) if whole and n in ("k", "v") else out[n] for n in ("k", "k_scale", "v", "v_scale"))
    # the pages: whole numbers and bytes that are moved, with the lists of a program on the host
    refs = s["refs"].tolist()
    S, P = len(lens), len(refs)

    def give(need):
        free = [p for p in range(P) if refs[p] == 0]
        for p in free[:need]:
            refs[p] += 1
        return free[:need]

    def drop(seqs):
        for i in seqs:
            for c in range(_pages(lens[i])):
                refs[table[i][c]] -= 1
            table[i], lens[i] = [-1] * len(table[i]), 0
        return [1] * len(seqs)

    def more(add):
        for i, n in enumerate(add):
            for c in range(_pages(lens[i]), _pages(lens[i] + n)):
                table[i][c] = give(1)[0]
            lens[i] += n
        return [1] * len(add)

    copies = []
    if op == "turnover":
        first = [drop(s["ended"].tolist()), more(s["add"].tolist())]
    elif op == "fork":
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            table[b], lens[b] = list(table[a]), lens[a]
            full = lens[a] // PAGE
            for c in range(full):
                refs[table[a][c]] += 1
            copies.append([-1, -1])
            if lens[a] % PAGE:
                copies[-1] = [table[a][full], give(1)[0]]
                table[b][full] = copies[-1][1]
        first = [[1] * len(copies), copies, more(s["add"].tolist()), drop(s["dst"].tolist())]
    else:
        used = sum(r > 0 for r in refs)
        copies = [[a, b] for a, b in zip([p for p in range(used, P) if refs[p]], [p for p in range(used) if not refs[p]])]
        for a, b in copies:
            refs[a], refs[b] = 0, refs[a]
        to = dict(copies)
        table = [[to.get(p, p) for p in row] for row in table]
        first = [copies + [[-1, -1]] * (P // 2 - len(copies))]
    ints = lambda x: torch.tensor(x, dtype=torch.int64)  # noqa: E731
    first = tuple(ints(x) for x in (*first, table, lens, refs))
    if op == "turnover":
        return first
    pools = []
    for p in s["pools"]:
        for a, b in copies:
            if a >= 0:
                for n in ("k", "k_scale", "v", "v_scale"):
                    p[n][b] = p[n][a]
        pools.append([p["k"].to(torch.int64), p["k_scale"].double(), p["v"].to(torch.int64), p["v_scale"].double()])
    return (*first, pools)
