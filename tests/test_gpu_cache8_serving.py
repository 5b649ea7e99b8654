"""A server's run on the paged 8-bit caches, all calls together: prompts, a fork, decode steps through a standard, a LiSA and a
direct-sharing layer, sequences that end, compaction; eager and as a captured graph, on another stream."""
import math

import numpy as np
import pytest
import torch

from paper_2408_01890_amd import lisa
from tests import cache8_ref as cr

pytestmark = pytest.mark.gpu
DEV = "cuda"
H, HKV, DK, R, F = 16, 4, 128, 22, 32


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Model:
    def __init__(self, fmt, seed, S=6, P=40, C=5):
        self.g = torch.Generator().manual_seed(seed)
        self.pages = lisa.Pages.empty(P, S, C, DEV)
        self.S, self.Lk = S, C * 64
        self.std = lisa.Cache8.empty(self.pages, HKV, DK, DK, fmt)
        self.lisa = lisa.Cache8.empty(self.pages, HKV, R, DK, fmt)
        self.share = lisa.Cache8.empty(self.pages, HKV, 0, DK, fmt)
        self.caches = [self.std, self.lisa, self.share]
        self.w1 = (torch.randn((H, F), generator=self.g) / 4).bfloat16().to(DEV)
        self.w2 = (torch.randn((F, H), generator=self.g) / 6).bfloat16().to(DEV)
        self.rows = [torch.zeros((S, H, self.Lk), dtype=torch.float16, device=DEV) for _ in range(3)]

    def rand(self, *shape):
        return (1.28 * torch.randn(shape, generator=self.g)).bfloat16().to(DEV)

    def inputs(self, L):
        return {"q": self.rand(self.S, H, DK), "q_lr": self.rand(self.S, H, R), "k": self.rand(self.S, HKV, L, DK), "k_lr": self.rand(self.S, HKV, L, R),
                "v": [self.rand(self.S, HKV, L, DK) for _ in range(3)]}

    def append(self, x, counts):
        for c, k, v in zip(self.caches, (x["k"], x["k_lr"], None), x["v"]):
            lisa.lisa_cache8_append(c, k, v, counts=counts)

    def step(self, x, add):
        lisa.lisa_pages_grow(self.pages, add)
        self.append(x, add)
        r = self.rows
        _, o0 = lisa.std_attn_decode8(x["q"], self.std, self.Lk, score_row_out=r[0])
        o1, _ = lisa.lisa_attn_decode8(x["q_lr"], self.lisa, r[0], self.w1, self.w2, score_row_out=r[1])
        o2, _ = lisa.lisa_attn_decode8(None, self.share, r[1], None, None, mix=lisa.MIX_SHARE, score_row_out=r[2])
        return o0, o1, o2

    def check(self, x, outs):
        lens, table = self.pages.lens.tolist(), self.pages.table.tolist()
        r = [t.cpu() for t in self.rows]
        for o, cache, q, prev, mix, w in ((outs[0], self.std, x["q"], None, "std", DK), (outs[1], self.lisa, x["q_lr"], r[0], "add", R),
                                          (outs[2], self.share, None, r[1], "share", 1)):
            want = cr.decode(cr.RefCache(cache), table, lens, self.Lk, q, prev, self.w1, self.w2, mix, "relu", 1 / math.sqrt(w), DK, H)
            for b in range(self.S):
                got, tol = cr.values(o[b]), want[b][4] + 2.0 ** -24 * np.abs(want[b][1]) + 1e-30
                assert np.all(np.abs(got - want[b][1]) <= tol), (mix, b, float((np.abs(got - want[b][1]) / tol).max()))

    def state(self):
        parts = [t for c in self.caches for t in (c.k, c.k_scale, c.v, c.v_scale) if t is not None]
        return [t.view(torch.uint8).clone() for t in (*parts, *self.rows, self.pages.table, self.pages.lens, self.pages.refs)]


@pytest.mark.parametrize("fmt", [torch.int8, torch.float8_e4m3fn])
def test_a_servers_run(fmt):
    m = Model(fmt, 1)
    prompts = ints([100, 64, 1, 0, 0, 0])
    assert lisa.lisa_pages_grow(m.pages, prompts).tolist() == [1] * 6
    x = m.inputs(100)
    m.append(x, prompts)
    alive = [1, 1, 1, 0, 0, 0]
    for step in range(9):
        if step == 2:                                        # two continuations of the first prompt
            done, copies = lisa.lisa_pages_fork(m.pages, ints([0, 0]), ints([3, 5]))
            lisa.lisa_pages_copy(m.caches, copies)
            assert done.tolist() == [1, 1] and m.pages.refs[m.pages.table[0, 0]].item() == 3
            for c in m.caches:                               # the same bytes behind both tables
                a, b = m.pages.table[0, 1].item(), m.pages.table[3, 1].item()
                assert a != b and torch.equal(c.v.view(torch.uint8)[a], c.v.view(torch.uint8)[b])
            alive = [1, 1, 1, 1, 0, 1]
        if step == 5:                                        # two end, what is left moves together
            lisa.lisa_pages_free(m.pages, ints([1, 3]))
            alive = [1, 0, 1, 0, 0, 1]
            lisa.lisa_pages_copy(m.caches, lisa.lisa_pages_compact(m.pages))
            used = int((m.pages.refs > 0).sum())
            assert bool((m.pages.refs[:used] > 0).all())
        x = m.inputs(1)
        m.check(x, m.step(x, ints(alive)))
    assert m.pages.lens.tolist() == [109, 0, 10, 0, 0, 109]   # (forked at 102 tokens, 7 steps since)
    ref = [0] * 40
    for s, n in enumerate(m.pages.lens.tolist()):
        for c in range(-(-n // 64)):
            ref[m.pages.table[s, c].item()] += 1
    assert m.pages.refs.tolist() == ref


@pytest.mark.parametrize("fmt", [torch.int8, torch.float8_e4m3fn])
def test_a_captured_step_equals_the_eager_one_at_every_replay(fmt):
    """Also with eager work on other data between the replays, and two graphs of the same calls side by side."""
    models = [Model(fmt, s) for s in (1, 1, 2, 2)]            # (eager, captured) twice
    add = ints([1, 1, 1, 0, 1, 0])
    for m in models:
        lisa.lisa_pages_grow(m.pages, ints([60, 127, 1, 0, 200, 0]))
        m.append(m.inputs(200), ints([60, 127, 1, 0, 200, 0]))
    steps = [[m.inputs(1) for _ in range(6)] for m in models]
    warm = Model(fmt, 7)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        warm.step(warm.inputs(1), add)
    s.synchronize()
    graphs, still, outs = [], [], []
    for i in (1, 3):
        fixed = models[i].inputs(1)
        g = torch.cuda.CUDAGraph()
        before = models[i].state()
        with torch.cuda.graph(g):
            o = models[i].step(fixed, add)
        assert all(torch.equal(a, b) for a, b in zip(before, models[i].state()))   # (captured, not run)
        graphs.append(g), still.append(fixed), outs.append(o)
    for t in range(6):
        for n, i in enumerate((1, 3)):
            want = models[i - 1].step(steps[i - 1][t], add)
            for k, x in still[n].items():
                for a, b in zip(x if k == "v" else [x], steps[i - 1][t][k] if k == "v" else [steps[i - 1][t][k]]):
                    a.copy_(b)
            graphs[n].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, outs[n]))
            assert all(torch.equal(a, b) for a, b in zip(models[i - 1].state(), models[i].state()))
    models[1].check(steps[0][5], outs[0])


def test_calls_on_another_stream_follow_its_work():
    a, b = Model(torch.int8, 3), Model(torch.int8, 3)
    add = ints([70, 1, 0, 64, 5, 9])
    xa, xb = a.inputs(70), b.inputs(70)
    one = ints([1] * 6)
    ya, yb = a.inputs(1), b.inputs(1)
    lisa.lisa_pages_grow(a.pages, add)
    a.append(xa, add)
    want = a.step(ya, one)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        lisa.lisa_pages_grow(b.pages, add)
        b.append(xb, add)
        got = b.step(yb, one)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state()))
