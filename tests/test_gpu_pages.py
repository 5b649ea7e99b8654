"""Page state and page copies on the GPU against lists on the host: equal, call after call."""
import random

import pytest
import torch

from paper_2408_01890_amd import lisa
from tests import cache8_ref as cr

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def equal(pages, ref):
    assert pages.lens.tolist() == ref.lens
    assert pages.table.tolist() == ref.table
    assert pages.refs.tolist() == ref.refs


@pytest.mark.parametrize("P,S,C,seed", [(1, 1, 1, 0), (7, 3, 2, 1), (40, 9, 6, 2), (300, 33, 20, 3), (5000, 70, 100, 4), (9000, 1500, 9, 5), (64, 2000, 3, 6), (3000, 2600, 3, 7)])
def test_random_calls_equal_the_lists(P, S, C, seed):
    r = random.Random(seed)
    pages, ref = lisa.Pages.empty(P, S, C, DEV), cr.RefPages(P, S, C)
    for step in range(40):
        op = r.choice(["grow", "grow", "grow1", "fork", "free", "compact"])
        if op == "grow":
            add = [r.choice([0, 0, 1, 63, 64, 65, r.randint(0, 64 * C), -1, 2 ** 31 - 1]) if r.random() < 0.4 else 0 for _ in range(S)]
        elif op == "grow1":
            add = [int(n > 0) for n in ref.lens]
        if op.startswith("grow"):
            done = lisa.lisa_pages_grow(pages, ints(add))
            assert done.tolist() == ref.grow(add)
        elif op == "fork":
            n = r.randint(1, S)
            src, dst = [r.randint(-1, S) for _ in range(n)], [r.randint(-1, S) for _ in range(n)]
            done, copies = lisa.lisa_pages_fork(pages, ints(src), ints(dst))
            wd, wc = ref.fork(src, dst)
            assert done.tolist() == wd and copies.tolist() == wc
        elif op == "free":
            seqs = [r.choice([r.randint(0, S - 1), r.randint(-2, S + 1)]) for _ in range(r.randint(1, max(1, S // 3)))]
            assert lisa.lisa_pages_free(pages, ints(seqs)).tolist() == ref.free(seqs)
        else:
            copies = lisa.lisa_pages_compact(pages)
            assert copies.reshape(-1, 2).tolist() == ref.compact()
        equal(pages, ref)
    assert lisa.last_path() == "pages"


def test_growth_stops_at_the_first_sequence_that_the_pages_do_not_reach():
    pages, ref = lisa.Pages.empty(10, 6, 8, DEV), cr.RefPages(10, 6, 8)
    for add in ([64 * 4, 64 * 5, 64 * 3, 0, 1, 0], [10, 0, 64, 7, 0, 0], [0, 0, 0, 0, 0, 64 * 9]):
        assert lisa.lisa_pages_grow(pages, ints(add)).tolist() == ref.grow(add)
        equal(pages, ref)
    # 4 + 5 of 10 pages, 3 more do not fit, nor then the 1 behind them; the last page goes to the 10 tokens behind the 256
    assert ref.lens == [266, 320, 0, 0, 0, 0]


def fill(cache, g):
    for t in (cache.k, cache.v):
        if t is not None:
            t.view(torch.uint8).copy_(torch.randint(0, 256, t.shape, generator=g, dtype=torch.uint8))
    for t in (cache.k_scale, cache.v_scale):
        if t is not None:
            t.copy_(torch.randn(t.shape, generator=g))


@pytest.mark.parametrize("n_caches", [1, 3, 70])
def test_copy_moves_pages_of_all_caches(n_caches):
    g = torch.Generator().manual_seed(n_caches)
    P = 23
    pages = lisa.Pages.empty(P, 2, 4, DEV)
    kinds = [(2, 22, 128, torch.int8), (3, 128, 128, torch.float8_e4m3fn), (1, 0, 40, torch.int8), (5, 7, 24, torch.int8)]
    caches = [lisa.Cache8.empty(pages, *kinds[i % 4][:3], kinds[i % 4][3]) for i in range(n_caches)]
    for c in caches:
        fill(c, g)
    parts = lambda c: [t.view(torch.uint8).clone() for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None]  # noqa: E731
    before = [parts(c) for c in caches]
    copies = [[3, 9], [-1, -1], [22, 0], [5, 6], [P, 1], [2, -3], [1 << 30, 4], [3, 10]]
    lisa.lisa_pages_copy(caches, ints(copies))
    for c, was in zip(caches, before):
        for t, w in zip(parts(c), was):
            want = w.clone()
            for a, b in copies:
                if 0 <= a < P and 0 <= b < P:
                    want[b] = w[a]
            assert torch.equal(t, want)


def test_nothing_to_copy_is_no_call():
    pages = lisa.Pages.empty(1, 1, 1, DEV)
    lisa.lisa_pages_copy([lisa.Cache8.empty(pages, 1, 8, 8)], lisa.lisa_pages_compact(pages))
    lisa.lisa_pages_copy([], ints([[0, 0]]))
