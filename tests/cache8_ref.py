"""The paged 8-bit cache in 64 bits and plain loops, for its tests: codes and scales, a decode step's attention over them with
bounds on what the kernels may be off, and the page state as lists."""
import math

import numpy as np
import torch

PAGE = 64
TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def block_scale(m, fmt):
    """2^e, the smallest e >= -126 with m <= top * 2^e."""
    e = -126
    if m > 0:
        e = max(e, math.ceil(math.log2(m / TOP[fmt])) - 1)
        while m > TOP[fmt] * 2.0 ** e:
            e += 1
    return 2.0 ** e


def round_codes(x, fmt):
    """float64 values (already over the scale) -> the codes' values, to nearest even, saturating."""
    x = np.asarray(x, dtype=np.float64)
    if fmt == torch.int8:
        return np.where(np.isnan(x), 0.0, np.clip(np.rint(np.nan_to_num(x, nan=0.0)), -127, 127))
    y = np.clip(x, -448, 448)
    with np.errstate(invalid="ignore"):
        step = 2.0 ** (np.maximum(np.frexp(np.nan_to_num(y))[1] - 1, -6) - 3)
        return np.rint(y / step) * step


def values(t):
    """Codes as float64 (e4m3 through its own table of values)."""
    return t.detach().cpu().float().double().numpy()


class RefCache:
    """Codes as [pages, Hkv, 64, features] float64 with their scales."""

    def __init__(self, cache):
        self.fmt, self.w = cache.v.dtype, cache.width
        self.v = values(cache.v).transpose(0, 1, 3, 2).copy()
        self.v_scale = values(cache.v_scale)
        if cache.width:
            k = values(cache.k)
            self.k = k.transpose(0, 1, 3, 2, 4).reshape(*k.shape[:2], PAGE, -1).copy()
            self.k_scale = values(cache.k_scale)

    def append(self, table, lens, counts, k_new, v_new):
        for b in range(v_new.shape[0]):
            n = int(lens[b])
            c = min(max(int(counts[b]), 0), v_new.shape[2], n)
            for name, new in (("k", k_new), ("v", v_new)):
                if new is None:
                    continue
                code, scale = getattr(self, name), getattr(self, name + "_scale")
                new = values(new)
                for col in sorted({j // PAGE for j in range(n - c, n)}):
                    page = int(table[b][col]) if col < len(table[b]) else -1
                    if not 0 <= page < code.shape[0]:
                        continue
                    js = [j for j in range(n - c, n) if j // PAGE == col]
                    lo, rows = js[0] % PAGE, [j - (n - c) for j in js]
                    for h in range(code.shape[1]):
                        x = new[b, h, rows]
                        fin = np.abs(x[np.isfinite(x)])
                        s = block_scale(fin.max() if fin.size else 0.0, self.fmt)
                        if lo:
                            s = max(s, scale[page, h])
                            if s > scale[page, h]:
                                code[page, h, :lo] = round_codes(code[page, h, :lo] * (scale[page, h] / s), self.fmt)
                        code[page, h, lo:lo + len(js), :x.shape[1]] = round_codes(x / s, self.fmt)
                        code[page, h, lo:lo + len(js), x.shape[1]:] = 0
                        scale[page, h] = s

    def tokens(self, name, table_row, n, h):
        """[n, features] float64 and which of the tokens have a page."""
        code, scale = getattr(self, name), getattr(self, name + "_scale")
        pages = [int(table_row[j // PAGE]) for j in range(n)]
        there = np.array([0 <= p < code.shape[0] for p in pages], dtype=bool)
        rows = [code[p, h, j % PAGE] * scale[p, h] if t else np.zeros(code.shape[3]) for j, (p, t) in enumerate(zip(pages, there))]
        x = np.array(rows).reshape(n, code.shape[3])
        return (x[:, :self.w] if name == "k" else x), there


def decode(ref, table, lens, Lk, q, prev, w1, w2, mix, act, scale, dk, H):
    """A decode step in float64.  mix: 'add', 'concat', 'plus', 'share', 'std'.  Returns per sequence (rows [H, n], out [H, dk],
    there [n], row_bound [H, n], out_bound [H, dk]): how far a kernel may be off that keeps to what the library says of
    its precision - A_{n-1} and emitted scores in half (2^-11 of each), hidden units and A_delta as an FFN input as two half numbers (2^-22 of
    each; a second one below 2^-14 is a whole number of 2^-24), sums in float32 (2^-24 a term), probabilities to 2^-11.  float32 calls have no
    half and keep probabilities to 2^-22."""
    f32 = q is not None and q.dtype == torch.float32 or prev is not None and prev.dtype == torch.float32
    half = 2.0 ** -24 if f32 else 2.0 ** -11
    two, least = (2.0 ** -24, 0.0) if f32 else (2.0 ** -22, 2.0 ** -25)
    out = []
    for b in range(len(lens)):
        n = max(0, min(int(lens[b]), Lk))
        Hkv = ref.v.shape[1]
        G = H // Hkv
        a, e = np.zeros((H, n)), np.zeros((H, n))
        there = np.array([0 <= int(table[b][j // PAGE]) < ref.v.shape[0] for j in range(n)], dtype=bool)
        if mix != "share":
            qd = values(q[b])
            for h in range(H):
                k, _ = ref.tokens("k", table[b], n, h // G)
                a[h] = k @ qd[h] * scale
                # float32 sums; the matrix-core kernels cut q to 24 bits of its largest element (e4m3: to 12 bits of
                # each, with the largest of 2^-17 of it)
                e[h] = np.abs(k) @ (np.abs(qd[h]) * 2.0 ** -12 * (0 if f32 or ref.fmt == torch.int8 else 1) + np.abs(qd[h]).max() * 2.0 ** (-22 if f32 or ref.fmt == torch.int8 else -17)) * scale
                e[h] += np.abs(k) @ np.abs(qd[h]) * scale * 2.0 ** -24 * (ref.w + 4)
        if prev is not None:
            x = values(prev[b, :, :n])
            if mix in ("add", "concat"):
                W1 = values(w1)
                xin, ein = (np.concatenate([x, a]), np.concatenate([np.zeros_like(x), e + two * np.abs(a) + least])) if mix == "concat" else (x, np.zeros_like(x))
                u = W1.T @ xin
                eu = np.abs(W1).T @ ein + np.abs(W1).T @ np.abs(xin) * 2.0 ** -24 * (len(W1) + 4)
                if act == "single":
                    y, ey = u, eu + two * np.abs(u) + least
                else:
                    hid = np.maximum(u, 0) if act == "relu" else u / (1 + np.exp(-u))
                    ehid = 1.1 * eu + (two + 2.0 ** -21) * np.abs(hid) + least
                    W2 = values(w2)
                    y = W2.T @ hid
                    ey = np.abs(W2).T @ ehid + np.abs(W2).T @ np.abs(hid) * 2.0 ** -24 * (len(W2) + 4)
                # weights as half: exact from 2^-14 on, below that within 2^-25
                ey += 0 if f32 else 2.0 ** -25 * (np.abs(xin).sum(0) + (np.abs(hid).sum(0) if act != "single" else 0)) * 4
                a, e = (y, ey) if mix == "concat" else (y + a, ey + e)
            else:
                a = x + a
                e = e + 2.0 ** -23 * (np.abs(x) + np.abs(a))
        seen = np.where(there[None], a, -np.inf)
        top = seen.max(1, initial=-np.inf, keepdims=True)
        with np.errstate(invalid="ignore"):
            p = np.where(np.isfinite(top), np.exp(seen - np.where(np.isfinite(top), top, 0)), 0.0)
        l = p.sum(1, keepdims=True)
        o, ob = np.zeros((H, dk)), np.zeros((H, dk))
        pe = 2.0 ** -22 if f32 else 2.0 ** -11
        # probabilities: the exponent's error and the kernel's exp; e4m3 on the matrix cores: 2^-12 of each, none below 2^-17 of the largest
        floor = 0 if f32 else 2.0 ** -16
        for h in range(H):
            if l[h] == 0:
                continue
            v, _ = ref.tokens("v", table[b], n, h // G)
            o[h] = p[h] @ v / l[h]
            ep = p[h] * (np.expm1(2 * e[h].max(initial=0)) + pe + 2.0 ** -20 * (1 + np.abs(seen[h] - top[h]).clip(0, 100))) + floor
            ep = np.where(there, ep, 0)
            ob[h] = (ep @ np.abs(v) + ep.sum() * np.abs(o[h]) + (n + 8) * 2.0 ** -24 * (p[h] @ np.abs(v))) / l[h]
        out.append((a, o, there, e + half * np.abs(a), ob))
    return out


class RefPages:
    """The page state as lists."""

    def __init__(self, P, S, C):
        self.table, self.lens, self.refs = [[-1] * C for _ in range(S)], [0] * S, [0] * P

    @staticmethod
    def pages(n):
        return (n + PAGE - 1) // PAGE

    def free_pages(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def grow(self, add):
        free, upto, done = self.free_pages(), 0, []
        for s, n in enumerate(add):
            want, have = self.pages(self.lens[s] + n) if n >= 0 else 0, self.pages(self.lens[s])
            if n < 0 or self.lens[s] + n > len(self.table[s]) * PAGE:
                done.append(0)
                continue
            more = want - have
            upto += more
            if more and upto > len(free):
                done.append(0)
                continue
            for c, p in zip(range(have, want), free[upto - more:upto]):
                self.table[s][c] = p
                self.refs[p] += 1
            self.lens[s] += n
            done.append(1)
        return done

    def fork(self, src, dst):
        free, given, done, copies, lens, named = self.free_pages(), 0, [], [], list(self.lens), set()
        S = len(lens)
        for a, b in zip(src, dst):
            done.append(0)
            copies.append([-1, -1])
            if not (0 <= a < S and 0 <= b < S) or a == b or lens[b] != 0 or b in named:
                continue
            named.add(b)
            n = lens[a]
            part = n % PAGE != 0
            given += part
            if part and given > len(free):
                continue
            row = list(self.table[a][:n // PAGE])
            for p in row:
                self.refs[p] += 1
            if part:
                copies[-1] = [self.table[a][n // PAGE], free[given - 1]]
                row.append(free[given - 1])
                self.refs[row[-1]] += 1
            self.table[b] = row + [-1] * (len(self.table[b]) - len(row))
            self.lens[b] = n
            done[-1] = 1
        return done, copies

    def free(self, seqs):
        done, named = [], set()
        for s in seqs:
            done.append(int(0 <= s < len(self.lens) and s not in named))
            if done[-1]:
                named.add(s)
                for p in self.table[s][:self.pages(self.lens[s])]:
                    self.refs[p] -= 1
                self.table[s], self.lens[s] = [-1] * len(self.table[s]), 0
        return done

    def compact(self):
        P, used = len(self.refs), sum(r > 0 for r in self.refs)
        moves = list(zip([p for p in range(used, P) if self.refs[p]], [p for p in range(used) if not self.refs[p]]))
        to = dict(moves)
        for a, b in moves:
            self.refs[a], self.refs[b] = 0, self.refs[a]
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return [list(m) for m in moves] + [[-1, -1]] * (P // 2 - len(moves))
