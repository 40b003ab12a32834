"""PagedCache.append against the rotation's formula in 64 bits and against write: padded trees and packed prompts, both kinds of pairs, parts of a head turned, far
positions, pages that are missing, shared or full, rows of no token."""
import pytest
import torch

from _layer import turned_reference
from _serving import gen, gathered, make_cache

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
FULL, INVALID, SHARED = 2, 4, 8


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def frequencies(dim, base=10000.0):
    return [base ** (-2.0 * j / dim) for j in range(dim // 2)]


def projected(shape, Hq, Hkv, D, dtype, seed):
    fused = torch.randn(shape + (Hq + 2 * Hkv, D), generator=gen(seed, "cuda"), device="cuda").to(dtype)
    return fused[..., :Hq, :], fused[..., Hq:Hq + Hkv, :], fused[..., Hq + Hkv:, :]


def near(got, want, tol):
    assert bool(((got.double() - want).abs() <= tol).all()), float(((got.double() - want).abs() - tol).max())


def same_pool(cache, k, v):
    assert torch.equal(cache.k.view(torch.int16), k.view(torch.int16)) and torch.equal(cache.v.view(torch.int16), v.view(torch.int16))


@pytest.mark.parametrize("D,dim,neighbours", [(64, 64, False), (128, 128, False), (256, 256, False), (64, 64, True), (128, 32, False), (256, 64, True), (64, 16, True), (128, 16, False), (256, 240, False)])
@pytest.mark.parametrize("dtype,Hq,Hkv,ps,T,N", [(BF, 4, 2, 16, 1, 0), (BF, 8, 1, 32, 21, 20), (HF, 6, 6, 64, 33, 28), (BF, 32, 8, 16, 9, 9), (HF, 5, 1, 256, 70, 0)])
def test_tokens_and_trees(D, dim, neighbours, dtype, Hq, Hkv, ps, T, N):
    from paper_2502_13652_amd import Rotation
    lens = [0, 15, 700, 31, 16]
    news = [T, max(T - 3, 0), T, 0, max(T // 2, 1)]
    cache = make_cache(lens, T, ps, Hkv, D, dtype, D + T, layers=2)
    plain = make_cache(lens, T, ps, Hkv, D, dtype, D + T, layers=2)
    q, k, v = projected((5, T), Hq, Hkv, D, dtype, T + dim)
    position = None
    if N:
        position = torch.randint(1, 9, (5, N), generator=gen(N), dtype=torch.int32).cuda()
    rotation = Rotation(dim, neighbours=neighbours)
    q_out = torch.full((5, T, Hq, D), 3.0, dtype=dtype, device="cuda")
    k_out = torch.full((5, T, Hkv, D), 3.0, dtype=dtype, device="cuda")
    got = cache.append(1, q, k, v, rotation, n_new=ints(news), position=position, q_out=q_out, k_out=k_out)
    assert got is q_out
    chain = T - N
    for b, n in enumerate(news):
        where = [lens[b] + t if t < chain else lens[b] + chain - 1 + int(position[b, t - chain]) for t in range(n)]
        if n:
            near(q_out[b, :n], *turned_reference(q[b, :n], where, dim, frequencies(dim), neighbours, 1.0))
            near(k_out[b, :n], *turned_reference(k[b, :n], where, dim, frequencies(dim), neighbours, 1.0))
        assert bool((q_out[b, n:] == 3.0).all()) and bool((k_out[b, n:] == 3.0).all())
    # the cache holds what write makes of the turned keys, and nothing else has changed
    plain.write(1, k_out, v.contiguous(), n_new=ints(news))
    same_pool(cache, plain.k, plain.v)
    assert cache.length.tolist() == lens and bool((cache.status.view(torch.int32) == 0).all())
    # in place, and a new tensor
    fresh = cache.append(1, q, k, v, rotation, n_new=ints(news), position=position)
    q2, k2 = q.clone(), k.clone()
    v2 = v.contiguous()
    cache.append(1, q2, k2, v2, rotation, n_new=ints(news), position=position, q_out=q2, k_out=k2)
    same_pool(cache, plain.k, plain.v)
    for b, n in enumerate(news):
        assert torch.equal(q2[b, :n], q_out[b, :n]) and torch.equal(k2[b, :n], k_out[b, :n]) and torch.equal(fresh[b, :n], q_out[b, :n])
        assert torch.equal(q2[b, n:], q[b, n:]) and torch.equal(k2[b, n:], k[b, n:])


@pytest.mark.parametrize("dtype,D,dim,neighbours", [(BF, 128, 128, False), (HF, 64, 32, True), (BF, 256, 128, False)])
@pytest.mark.parametrize("news", [[1], [0, 3, 0, 0, 50, 1, 16], [129, 1, 64], [3] * 70, [1, 0] * 300])
def test_packed_prompts(dtype, D, dim, neighbours, news):
    from paper_2502_13652_amd import Rotation
    Hq, Hkv, ps = 4, 2, 16
    lens = [(7 * b) % 40 for b in range(len(news))]
    cache = make_cache(lens, max(news), ps, Hkv, D, dtype, len(news))
    k0, v0 = cache.k.clone(), cache.v.clone()
    at = [2]
    for n in news:
        at.append(at[-1] + n)
    rows = at[-1] + 3
    q, k, v = projected((rows,), Hq, Hkv, D, dtype, rows)
    q_out = torch.full((rows, Hq, D), 3.0, dtype=dtype, device="cuda")
    k_out = torch.full((rows, Hkv, D), 3.0, dtype=dtype, device="cuda")
    cache.append(0, q, k, v, Rotation(dim, base=500.0, neighbours=neighbours, magnitude=1.25), starts=ints(at), q_out=q_out, k_out=k_out)
    where = [lens[b] + t for b, n in enumerate(news) for t in range(n)]
    for x, y in ((q, q_out), (k, k_out)):
        near(y[2:at[-1]], *turned_reference(x[2:at[-1]], where, dim, frequencies(dim, 500.0), neighbours, 1.25))
        assert bool((y[:2] == 3.0).all()) and bool((y[at[-1]:] == 3.0).all())
    touched = torch.zeros(cache.k.shape[1:4], dtype=torch.bool, device="cuda")
    for b, n in enumerate(news):
        kc, vc, ok = gathered(cache, b, 0, lens[b] + n)
        assert bool(ok.all()) and torch.equal(kc[:, lens[b]:].transpose(0, 1), k_out[at[b]:at[b + 1]].double()) and \
            torch.equal(vc[:, lens[b]:].transpose(0, 1), v[at[b]:at[b + 1]].double())
        places = torch.arange(lens[b], lens[b] + n, device="cuda")
        touched[cache.page_table[b].long()[places // ps], :, places % ps] = True
    assert torch.equal(cache.k[0][~touched], k0[0][~touched]) and torch.equal(cache.v[0][~touched], v0[0][~touched])


def test_far_positions_are_as_exact_as_near_ones():
    from paper_2502_13652_amd import Rotation
    q, k, v = projected((1, 6), 2, 1, 64, HF, 3)
    cache = make_cache([10], 6, 16, 1, 64, HF, 4)
    offsets = [-2 ** 31, -12345678, 0, 99999999, 2 ** 31 - 1, 2 ** 30 + 7]
    f = [1.0, 0.3, 1e-3, 1e-9, 3.0, 6.25, -1.0, 1000.5] * 4
    out = cache.append(0, q, k, v, Rotation(64, frequencies=f, magnitude=-0.5), position=ints([offsets]))
    near(out[0], *turned_reference(q[0], [10 - 1 + p for p in offsets], 64, f, False, -0.5))


def test_quarter_turns():
    """Angles at and next to the corners of the sine's cases."""
    from paper_2502_13652_amd import Rotation
    import math
    f = [2 * math.pi * (i / 16 + d) for i in range(16) for d in (0.0, 1e-7)]
    q, k, v = projected((1, 3), 2, 1, 64, HF, 5)
    cache = make_cache([0], 3, 16, 1, 64, HF, 6)
    out = cache.append(0, q, k, v, Rotation(64, frequencies=f))
    near(out[0], *turned_reference(q[0], [0, 1, 2], 64, f, False, 1.0))
    assert torch.equal(out[0, 0], q[0, 0])                  # position 0: not turned


def test_what_the_cache_cannot_take():
    from paper_2502_13652_amd import Rotation
    Hq, Hkv, D, ps, T = 2, 1, 64, 16, 20
    cache = make_cache([0, 0, 0, 28, 0], T, ps, Hkv, D, BF, 7, max_pages=3)
    cache.length[3] = 40                                    # room for 8 more
    cache.page_table[1, 1], cache.page_table[2, 0] = 9999, -7
    cache.refcount[cache.page_table[4, 0].long()] = 2
    k0, v0 = cache.k.clone(), cache.v.clone()
    q, k, v = projected((5, T), Hq, Hkv, D, BF, 8)
    rotation = Rotation(64)
    k_out = torch.zeros((5, T, Hkv, D), dtype=BF, device="cuda")
    out = cache.append(0, q, k, v, rotation, k_out=k_out)
    assert cache.status.view(torch.int32).tolist() == [0, INVALID, INVALID, FULL, SHARED]
    lens = [0, 0, 0, 40, 0]
    for b in range(5):                                      # queries and turned keys come out whole
        where = [lens[b] + t for t in range(T)]
        near(out[b], *turned_reference(q[b], where, 64, frequencies(64), False, 1.0))
        near(k_out[b], *turned_reference(k[b], where, 64, frequencies(64), False, 1.0))
    want_k, want_v = k0.clone(), v0.clone()
    for b, ts in ((0, range(T)), (1, range(16)), (2, range(16, T)), (3, range(8)), (4, range(16, T))):
        for t in ts:
            at = lens[b] + t
            page = int(cache.page_table[b, at // ps])
            want_k[0, page, :, at % ps], want_v[0, page, :, at % ps] = k_out[b, t], v[b, t]
    same_pool(cache, want_k, want_v)
    # the same packed
    cache.k.copy_(k0), cache.v.copy_(v0), cache.status.zero_()
    flat = lambda x: x.reshape(5 * T, -1, D)
    packed = cache.append(0, flat(q), flat(k), flat(v), rotation, starts=ints([b * T for b in range(6)]))
    assert torch.equal(packed.view(5, T, Hq, D), out) and cache.status.view(torch.int32).tolist() == [0, INVALID, INVALID, FULL, SHARED]
    same_pool(cache, want_k, want_v)


def test_starts_that_make_no_sense():
    from paper_2502_13652_amd import Rotation
    cache = make_cache([0, 0, 0, 0], 40, 16, 1, 64, BF, 9)
    k0 = cache.k.clone()
    q, k, v = projected((40,), 2, 1, 64, BF, 10)
    for at in ([-5, -1, -1, -1, -1], [100, 200, 300, 400, 500], [2 ** 31 - 1, -2 ** 31, 0, 0, 0], [-3, 50, 50, 50, 50], [0, 0, 41, 41, 41], [0, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1]):
        out = cache.append(0, q, k, v, Rotation(64), starts=ints(at), q_out=torch.full((40, 2, 64), 3.0, dtype=BF, device="cuda"))
        assert bool((out == 3.0).all()) and torch.equal(cache.k, k0)


@pytest.mark.parametrize("n,at", [(3, [50, 20, 90, 10]), (4, [50, 20, 90, 10, 10]), (5, [90, 95, 0, 30, 200, 0]), (2, [10, 0, 100]),
                                  (200, [0, 10] + [200] * 70 + [40, 60] + [30] * 3 + [200] * 122 + [90, 100]), (130, [100] * 65 + [3, 40] + [2 ** 31 - 1, -1] * 32),
                                  (70, [0, 300, 10, 40, 40, -5] + [40] * 60 + [70, 200, 70, 95, 100])])
def test_sequences_between_starts_that_fall(n, at):
    """A sequence whose own start and end make sense is taken whole, others are left out whole."""
    from paper_2502_13652_amd import Rotation
    assert len(at) == n + 1
    lens = [b % 20 for b in range(n)]
    cache = make_cache(lens, 100, 16, 1, 64, BF, n)
    k0, v0 = cache.k.clone(), cache.v.clone()
    q, k, v = projected((100,), 2, 1, 64, BF, 10 + n)
    out, k_out = (torch.full((100, h, 64), 3.0, dtype=BF, device="cuda") for h in (2, 1))
    cache.append(0, q, k, v, Rotation(64), starts=ints(at), q_out=out, k_out=k_out)
    held = torch.zeros(100, dtype=torch.bool)
    for b in range(n):
        a, z = at[b], at[b + 1]
        if not 0 <= a < z <= 100:
            continue
        assert not bool(held[a:z].any())                     # (the lists are made so that no two share a row)
        held[a:z] = True
        where = [lens[b] + t for t in range(z - a)]
        near(out[a:z], *turned_reference(q[a:z], where, 64, frequencies(64), False, 1.0))
        near(k_out[a:z], *turned_reference(k[a:z], where, 64, frequencies(64), False, 1.0))
        for t in range(z - a):
            page = int(cache.page_table[b, where[t] // 16])
            k0[0, page, :, where[t] % 16], v0[0, page, :, where[t] % 16] = k_out[a + t], v[a + t]
    assert bool(held.any()) and bool((out[~held] == 3.0).all()) and bool((k_out[~held] == 3.0).all())
    same_pool(cache, k0, v0)
    assert int(cache.status.view(torch.int32).abs().sum()) == 0


def test_empty_refused_streams_and_graphs():
    from paper_2502_13652_amd import Rotation
    cache = make_cache([5, 6], 12, 16, 2, 64, BF, 11)
    q, k, v = projected((2, 4), 4, 2, 64, BF, 12)
    r = Rotation(64)
    assert cache.append(0, q[:, :0].reshape(0, 4, 64), k[:, :0].reshape(0, 2, 64), v[:, :0].reshape(0, 2, 64), r, starts=ints([0, 0, 0])).shape == (0, 4, 64)
    flat = lambda x: x.reshape(8, -1, 64)
    for args, kw in (((q, k, v[:, :3], r), {}), ((q, k[:, :3], v[:, :3], r), {}), ((q.float(), k, v, r), {}), ((q[:1], k, v, r), {}), ((q, k, v.contiguous(), r), {}),
                     ((q, k, v, r), dict(n_new=ints([1]))), ((q, k, v, r), dict(position=ints([[1], [2], [3]]))), ((q, k, v, r), dict(starts=ints([0, 4, 8]))),
                     ((flat(q), flat(k), flat(v), r), dict(starts=ints([0, 4]))), ((flat(q), flat(k), flat(v), r), dict(starts=ints([0, 4, 8]), n_new=ints([1, 1]))),
                     ((q, k, v, r), dict(q_out=q[:, :2])), ((q, k, v, r), dict(k_out=q)), ((q, k, v, Rotation(64, device="cpu")), {})):
        with pytest.raises(ValueError):
            cache.append(0, *args, **kw)
    with pytest.raises(Exception, match="invalid"):
        cache.append(1, q, k, v, r)
    with pytest.raises(Exception, match="invalid"):
        cache.append(0, q, k, v, Rotation(128))              # wider than a head
    with pytest.raises(Exception, match="invalid"):
        cache.append(0, q[:, :, :3], k, v, r)
    with pytest.raises(Exception, match="invalid"):
        cache.append(0, q, k, v, r, position=torch.zeros((2, 5), dtype=torch.int32, device="cuda"))
    other = torch.zeros((1, 4, 4, 64), dtype=BF, device="cuda").expand(2, 4, 4, 64)
    with pytest.raises(Exception, match="invalid"):
        cache.append(0, q, k, v, r, q_out=other)             # two sequences in one place
    want = cache.append(0, q, k, v, r)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = cache.append(0, q, k, v, r, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    out, n_new = torch.zeros_like(want), ints([4, 4])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.append(0, q, k, v, r, n_new=n_new, q_out=out)
    for lens, news in (([5, 6], [4, 2]), ([0, 9], [1, 4]), ([12, 3], [0, 3])):
        cache.length.copy_(ints(lens)), n_new.copy_(ints(news)), out.fill_(2.0)
        graph.replay()
        torch.cuda.synchronize()
        for b, n in enumerate(news):
            if n:
                near(out[b, :n], *turned_reference(q[b, :n], [lens[b] + t for t in range(n)], 64, frequencies(64), False, 1.0))
            assert bool((out[b, n:] == 2.0).all())


def test_rows_and_pages_whose_offsets_pass_32_bits():
    from paper_2502_13652_amd import PagedCache, Rotation
    pages = 140000                                           # of 32 KiB each: 4.6 GB of keys
    cache = PagedCache(3, 1, pages, 16, 8, 128, 4)
    taken = [7, pages - 1, pages - 2, 131072, 3, 100000]
    cache.page_table.copy_(torch.tensor([taken[0:2] + [-1, -1], taken[2:4] + [-1, -1], taken[4:6] + [-1, -1]], dtype=torch.int32))
    cache.refcount[taken] = 1
    cache.length.copy_(torch.tensor([3, 14, 0], dtype=torch.int32))
    q, k, v = (x.contiguous() for x in projected((3, 17), 8, 8, 128, BF, 23))
    apart = torch.empty(2 * 2 ** 30 + 40 * 17 * 1024, dtype=BF, device="cuda")
    far = [apart.as_strided((3, 17, 8, 128), (2 ** 30, 1024, 128, 1), 17 * 1024 * i) for i in range(5)]
    for to, x in zip(far, (q, k, v)):
        to.copy_(x)
    cache.append(0, *far[:3], Rotation(128), q_out=far[3], k_out=far[4])
    assert int(cache.status.view(torch.int32).abs().sum()) == 0
    for b, n in enumerate((3, 14, 0)):
        where = list(range(n, n + 17))
        for got, x in ((far[3], q), (far[4], k)):
            near(got[b], *turned_reference(x[b], where, 128, frequencies(128), False, 1.0))
        kc, vc, ok = gathered(cache, b, 0, n + 17)
        assert bool(ok.all()) and torch.equal(kc[:, n:].transpose(0, 1), far[4][b].double()) and torch.equal(vc[:, n:].transpose(0, 1), v[b].double())
