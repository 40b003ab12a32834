"""The paged cache's operators against plain python on the same numbers: reserve (with copies of shared pages), write, commit, fork, truncate;
what they refuse, and that nothing else changes."""
import numpy as np
import pytest
import torch

from _serving import gen, make_cache

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
EMPTY, FULL, INVALID, SHARED = 1, 2, 4, 8


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Plain:
    """The same cache in numpy, one token at a time."""

    def __init__(self, c):
        self.ps, self.cap = c.page_size, c.max_pages * c.page_size
        self.take(c)

    def take(self, c):
        self.k, self.v = (x.view(torch.int16).cpu().numpy().copy() for x in (c.k, c.v))
        self.table, self.length, self.refs = (x.cpu().numpy().copy() for x in (c.page_table, c.length, c.refcount))
        self.status = c.status.view(torch.int32).cpu().numpy().copy()
        return self

    def same_as(self, c, tag=""):
        o = Plain.__new__(Plain).take(c)
        for name in ("table", "length", "refs", "status", "k", "v"):
            np.testing.assert_array_equal(getattr(o, name), getattr(self, name), err_msg="%s %s" % (tag, name))

    def write(self, layer, k, v, n_new):
        k, v = (x.contiguous().view(torch.int16).cpu().numpy() for x in (k, v))
        for b in range(len(self.length)):
            for t in range(min(n_new[b], k.shape[1])):
                at = self.length[b] + t
                if at >= self.cap:
                    self.status[b] |= FULL
                    break
                page = self.table[b, at // self.ps]
                if page < 0 or page >= len(self.refs):
                    self.status[b] |= INVALID
                elif self.refs[page] > 1:
                    self.status[b] |= SHARED
                else:
                    self.k[layer, page, :, at % self.ps], self.v[layer, page, :, at % self.ps] = k[b, t], v[b, t]

    def reserve(self, n_new):
        refs0, free = self.refs.copy(), [p for p in range(len(self.refs)) if self.refs[p] == 0]
        used = 0
        full = False
        for b in range(len(self.length)):
            n, l = n_new[b], self.length[b]
            if n <= 0:
                continue
            if l + n > self.cap:
                self.status[b] |= FULL
                continue
            places = range(l // self.ps, -(-(l + n) // self.ps))
            if any(self.table[b, i] != -1 and not 0 <= self.table[b, i] < len(self.refs) for i in places):
                self.status[b] |= INVALID
                continue
            fresh = [i for i in places if self.table[b, i] < 0 or refs0[self.table[b, i]] > 1]
            start, used = used, used + len(fresh)
            if fresh and used > len(free):
                self.status[b] |= EMPTY
                continue
            for i, page in zip(fresh, free[start:]):
                old = self.table[b, i]
                if old >= 0:
                    self.refs[old] -= 1
                    if i == l // self.ps:
                        m = l % self.ps
                        self.k[:, page, :, :m], self.v[:, page, :, :m] = self.k[:, old, :, :m], self.v[:, old, :, :m]
                self.refs[page] += 1
                self.table[b, i] = page

    def commit(self, path, n_path):
        for b in range(len(self.length)):
            n, l = min(max(n_path[b], 0), path.shape[1]), self.length[b]
            p = path[b][:n]
            why = 0
            for i in range(n):
                if p[i] < i or (i and p[i] <= p[i - 1]):
                    why |= INVALID
                    continue
                for at, written in ((l + int(p[i]), False), (l + i, p[i] != i)):
                    page = self.table[b, at // self.ps] if at < self.cap else -1
                    if not 0 <= page < len(self.refs):
                        why |= INVALID
                    elif written and self.refs[page] > 1:
                        why |= SHARED
            if why:
                self.status[b] |= why
                continue
            for i in range(n):
                a, z = l + int(p[i]), l + i
                pa, pz = self.table[b, a // self.ps], self.table[b, z // self.ps]
                for x in (self.k, self.v):
                    x[:, pz, :, z % self.ps] = x[:, pa, :, a % self.ps]
            self.length[b] = l + n

    def let_go(self, b, page):
        if 0 <= page < len(self.refs) and self.refs[page] > 0:
            self.refs[page] -= 1
        elif page != -1:
            self.status[b] |= INVALID

    def truncate(self, new_length, keep):
        for b in range(len(self.length)):
            if new_length is not None:
                self.length[b] = min(self.length[b], max(new_length[b], 0))
            for i in range(min(-(-(self.length[b] + keep) // self.ps), self.table.shape[1]), self.table.shape[1]):
                self.let_go(b, self.table[b, i])
                self.table[b, i] = -1

    def fork(self, src, dst):
        B = len(self.length)
        pairs = [(s, d) for s, d in zip(src, dst) if 0 <= s < B and 0 <= d < B and s != d]
        for i, (s, d) in enumerate(pairs):
            if any(j != i and (d2 == d or s2 == d or d2 == s) for j, (s2, d2) in enumerate(pairs)):
                self.status[d] |= INVALID
                continue
            held = -(-self.length[s] // self.ps)
            old = self.table[d].copy()
            self.table[d] = -1
            for i2 in range(held):
                page = self.table[s, i2]
                if 0 <= page < len(self.refs):
                    self.refs[page] += 1
                    self.table[d, i2] = page
                else:
                    self.status[d] |= INVALID
            for page in old:
                self.let_go(d, page)
            self.length[d] = self.length[s]


@pytest.mark.parametrize("dtype,D,ps,Hkv,layers", [(BF, 64, 16, 2, 3), (HF, 128, 32, 1, 2), (BF, 256, 64, 3, 1), (BF, 128, 256, 8, 2), (HF, 64, 128, 5, 4)])
def test_a_life_of_a_cache(dtype, D, ps, Hkv, layers):
    """Random calls one after the other, each compared with the plain cache: pools that run out, forks of forks, odd paths."""
    from paper_2502_13652_amd import PagedCache
    B, max_pages = 7, 6
    cap = max_pages * ps
    c = PagedCache(B, layers, 20, ps, Hkv, D, max_pages, dtype=dtype)
    c.k.normal_()
    c.v.normal_()
    p = Plain(c)
    rng = np.random.default_rng(D + ps)
    seen = 0
    for step in range(120):
        op = rng.choice(["reserve", "reserve", "write", "commit", "fork", "truncate"])
        n = rng.integers(-1, int(rng.choice([3, ps + 2, 2 * ps])), B).astype(np.int32)
        print("cache", step, op, n.tolist(), p.length.tolist(), flush=True)
        if op == "reserve":
            c.reserve(ints(n.tolist()))
            p.reserve(n)
        elif op == "write":
            T = int(rng.integers(1, ps + 5))
            x = torch.randn((B, T, 3 * Hkv, D), generator=gen(step, "cuda"), device="cuda").to(dtype)
            layer = int(rng.integers(0, layers))
            whole = rng.random() < 0.2
            c.write(layer, x[:, :, :Hkv], x[:, :, Hkv:2 * Hkv], n_new=None if whole else ints(n.tolist()))
            p.write(layer, x[:, :, :Hkv], x[:, :, Hkv:2 * Hkv], [T] * B if whole else n)
        elif op == "commit":
            m = int(rng.integers(1, 20))
            path = np.sort(np.stack([rng.choice(2 * ps, m, replace=False) for _ in range(B)]), 1).astype(np.int32) if rng.random() < 0.7 else \
                np.tile(np.arange(m, dtype=np.int32), (B, 1))
            if rng.random() < 0.3:
                path[int(rng.integers(0, B))] = rng.integers(-2, m + 1, m)
            c.commit(ints(path.tolist()), ints(n.tolist()))
            p.commit(path, n)
        elif op == "fork":
            m = int(rng.integers(1, 6))
            s, d = rng.integers(-1, B + 1, m), rng.integers(-1, B + 1, m)
            c.fork(ints(s.tolist()), ints(d.tolist()))
            p.fork(s.tolist(), d.tolist())
        else:
            keep = int(rng.integers(0, 2 * ps))
            to = None if rng.random() < 0.3 else rng.integers(-1, cap, B)
            c.truncate(None if to is None else ints(to.tolist()), keep=keep)
            p.truncate(to, keep)
        torch.cuda.synchronize()
        p.same_as(c, "step %d %s" % (step, op))
        for b in range(B):
            assert 0 <= p.length[b] <= cap
        seen |= int(np.bitwise_or.reduce(p.status))
        if step % 10 == 9:
            c.status.view(torch.int32).zero_()
            p.status[:] = 0
    held = np.zeros(len(p.refs), int)
    for page in p.table[p.table >= 0]:
        held[page] += 1
    np.testing.assert_array_equal(held, p.refs)               # nothing lost, nothing held twice
    assert seen & INVALID                                     # (which of the other refusals occur is the numbers' affair)


def test_a_large_pool_gives_the_lowest_pages():
    from paper_2502_13652_amd import PagedCache
    B, pages = 300, 20000
    c = PagedCache(B, 1, pages, 16, 1, 64, 200, dtype=BF)
    g = gen(5)
    c.refcount.copy_((torch.rand(pages, generator=g) < 0.6).to(torch.int32))
    want = torch.nonzero(c.refcount.cpu() == 0).flatten().tolist()
    n = torch.randint(0, 400, (B,), generator=g, dtype=torch.int32)
    c.reserve(n.cuda())
    at = 0
    for b in range(B):
        m = -(-int(n[b]) // 16)
        row = c.page_table[b].tolist()
        if at + m <= len(want) and row[:m] == want[at:at + m]:
            assert row[m:] == [-1] * (200 - m) and int(c.status.view(torch.int32)[b]) == 0
        else:                                                 # the pool has run out
            assert at + m > len(want) and row == [-1] * 200 and int(c.status.view(torch.int32)[b]) == EMPTY, b
        at += m
    assert int((c.page_table >= 0).sum()) <= len(want)


def test_the_largest_batch():
    from paper_2502_13652_amd import PagedCache
    B = 4096
    c = PagedCache(B, 1, 3 * B, 16, 1, 64, 3, dtype=BF)
    c.reserve(ints([17] * B))
    torch.cuda.synchronize()
    assert torch.equal(c.page_table[:, :2].flatten().cpu(), torch.arange(2 * B, dtype=torch.int32)) and bool((c.page_table[:, 2] == -1).all())
    c.length.fill_(17)
    c.fork(ints(list(range(0, B, 2))), ints(list(range(1, B, 2))))
    assert bool((c.page_table[1::2] == c.page_table[::2]).all()) and int(c.refcount.sum()) == 2 * B and int((c.refcount == 2).sum()) == B
    c.truncate(ints([0] * B))
    assert bool((c.refcount == 0).all()) and bool((c.page_table == -1).all()) and bool((c.length == 0).all()) and int(c.status.view(torch.int32).abs().sum()) == 0


def test_more_places_asked_for_than_31_bits_count():
    """4096 sequences that ask for half a million pages each of a pool of 64 (a page table of 8.6 GB): nobody gets any, and all are told so, the last one too, which asks for one."""
    from paper_2502_13652_amd import PagedCache
    B, max_pages = 4096, (1 << 19) + 256
    c = PagedCache(B, 1, 64, 16, 1, 64, max_pages, dtype=BF)
    assert (B - 1) * max_pages > 1 << 31
    n = torch.full((B,), max_pages * 16, dtype=torch.int32, device="cuda")
    n[-1] = 1
    print("reserve, %d places" % (B * max_pages), flush=True)
    c.reserve(n)
    torch.cuda.synchronize()
    assert c.status.view(torch.int32).tolist() == [EMPTY] * B
    assert bool((c.refcount == 0).all()) and int(c.page_table.max()) == -1 and int(c.page_table.min()) == -1
    n[:64] = 16                                              # the first 64 get one each, the rest none
    c.status.view(torch.int32).zero_()
    c.reserve(n)
    torch.cuda.synchronize()
    assert c.status.view(torch.int32).tolist() == [0] * 64 + [EMPTY] * (B - 64)
    assert c.page_table[:, 0].tolist() == list(range(64)) + [-1] * (B - 64) and bool((c.refcount == 1).all())


def test_a_long_path_and_the_largest_tree():
    c = make_cache([5, 900], 1025, 64, 2, 64, BF, seed=4, layers=2)
    p = Plain(c)
    path = np.stack([np.arange(1025), np.arange(1025)]).astype(np.int32)
    path[1, :500] = np.sort(np.random.default_rng(1).choice(1025, 500, replace=False))
    c.commit(ints(path.tolist()), ints([1025, 500]))
    p.commit(path, [1025, 500])
    p.same_as(c)


def test_numbers_that_cannot_be_change_nothing():
    c = make_cache([20, 20, 20], 40, 16, 1, 64, BF, seed=1, max_pages=6)
    c.length.copy_(ints([-7, 10 ** 9, 20]))
    c.page_table[2, 1] = 10 ** 9
    k, v, refs = c.k.clone(), c.v.clone(), c.refcount.clone()
    x = torch.ones((3, 2, 1, 64), dtype=BF, device="cuda")
    c.write(0, x, x, n_new=ints([-3, 5, 2]))                 # nothing; no room; no page
    c.commit(ints([[1, 2], [0, 1], [2 ** 31 - 1, 5]]), ints([0, 2, 2]))
    assert torch.equal(c.k, k) and torch.equal(c.v, v) and torch.equal(c.refcount, refs)
    assert c.status.view(torch.int32).tolist() == [0, FULL | INVALID, INVALID]
    c.reserve(ints([2 ** 31 - 1, 1, 1]))
    assert torch.equal(c.refcount, refs) and c.status.view(torch.int32).tolist() == [FULL, FULL | INVALID, INVALID]
    c.refcount.zero_()
    c.truncate(ints([0, 0, 0]))                              # pages that nobody is said to hold
    assert bool((c.refcount == 0).all()) and bool((c.page_table == -1).all())


def test_calls_are_captured_and_replayed():
    """A step in a graph: reserve, write, commit, truncate, replayed on changing inputs, against the same calls made eagerly."""
    caches = [make_cache([10, 33, 0], 0, 16, 2, 64, BF, seed=6, layers=2, spare=30, max_pages=20) for _ in range(2)]
    T = 20
    n_new, path, n_path = ints([T, T, T]), ints([[0] * 5] * 3), ints([0, 0, 0])
    x = torch.randn((3, T, 2, 64), device="cuda").to(BF)

    def step(c):
        c.reserve(n_new)
        for layer in range(2):
            c.write(layer, x, x, n_new=n_new)
        c.commit(path, n_path)
        c.truncate(keep=0)
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step(caches[0])
    for i in range(6):
        x.copy_(torch.randn((3, T, 2, 64), generator=gen(i, "cuda"), device="cuda"))
        path.copy_(ints([sorted(np.random.default_rng(10 * i + b).choice(T, 5, replace=False).tolist()) for b in range(3)]))
        n_path.copy_(ints([i % 6, 5, 1]))
        n_new.copy_(ints([T, T - i % 2, T]))
        g.replay()
        step(caches[1])
        torch.cuda.synchronize()
        a, b = caches
        for name in ("page_table", "length", "refcount"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (i, name)
        for name in ("k", "v"):
            held = a.refcount > 0
            assert torch.equal(getattr(a, name)[:, held].view(torch.int16), getattr(b, name)[:, held].view(torch.int16))
        assert int(a.status.view(torch.int32).abs().sum()) == 0


def test_refusals():
    from paper_2502_13652_amd.binding import C2TError
    c = make_cache([10, 20], 4, 16, 2, 64, BF, seed=1)
    x = torch.zeros((2, 3, 2, 64), dtype=BF, device="cuda")
    for bad in (lambda: c.reserve(torch.zeros(2, device="cuda")), lambda: c.reserve(ints([1])), lambda: c.reserve(torch.zeros(2, dtype=torch.int32)),
                lambda: c.write(0, x, x[:, :2]), lambda: c.write(0, x.float(), x.float()), lambda: c.write(0, x[:, :, :1], x[:, :, :1]),
                lambda: c.write(0, x.transpose(1, 2), x.transpose(1, 2)), lambda: c.write(0, x, x, n_new=ints([1, 2, 3])), lambda: c.write(0, x[:, :0], x[:, :0]),
                lambda: c.commit(ints([[1], [1]]), ints([1])), lambda: c.commit(ints([1, 1]), ints([1, 1])),
                lambda: c.fork(ints([0]), ints([0, 1])), lambda: c.truncate(ints([0]))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: c.write(1, x, x), lambda: c.truncate(keep=-1), lambda: c.fork(ints([]), ints([])), lambda: c.commit(ints([[], []]), ints([0, 0]))):
        with pytest.raises(C2TError) as e:
            bad()
        assert e.value.code == -1
