"""Attention over the paged cache against the definition in 64 bits: types, head layouts, lengths, masks that leave rows empty, values that
must not matter, pages that are none, strides, streams, graphs."""
import pytest
import torch

from _serving import attention_reference, gen, make_cache, random_tree

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def check(cache, layer, q, n_new, mask=None, scale=None, lse=True, tag="", **kw):
    B, T, H, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    n_list = [T] * B if n_new is None else n_new
    n_dev = None if n_new is None else torch.tensor(n_new, dtype=torch.int32, device="cuda")
    out = torch.full((B, T, H, D), 7.0, dtype=q.dtype, device="cuda")
    ls = torch.full((B, T, H), 7.0, device="cuda") if lse else None
    print("attention", tag, tuple(q.shape), "nodes", 0 if mask is None else mask.shape[-1], "lens", cache.length.tolist()[:8], "n_new", n_list[:8], flush=True)
    got = cache.attention(layer, q, n_new=n_dev, mask=mask, scale=scale, out=out, lse=ls, **kw)
    torch.cuda.synchronize()
    assert got is out
    caps = cache.max_pages * cache.page_size
    lens = [min(max(l, 0), caps) for l in cache.length.tolist()]
    real = [max(0, min(n, T, caps - l)) for n, l in zip(n_list, lens)]
    want, want_lse, tol, tol_lse = attention_reference(cache, layer, q, real, mask, scale, lens)
    for b in range(B):
        n = real[b]
        assert bool((out[b, n:] == 7.0).all()), "rows behind n_new were written"
        if ls is not None:
            assert bool((ls[b, n:] == 7.0).all())
        if n == 0:
            continue
        w, g, t = want[b, :n], out[b, :n].double(), tol[b, :n]
        bad = torch.isnan(w)
        assert bool((torch.isnan(g) == bad).all()), "NaN where it should not be, or none"
        inf = torch.isinf(w)
        assert bool((g[inf] == w[inf]).all())
        err = torch.where(bad | inf, 0.0, (g - w).abs() - torch.where(torch.isfinite(t), t, 0.0))
        assert float(err.max()) <= 0, "%s seq %d: off by %g more than %g" % (tag, b, float(err.max()), float(t.flatten()[err.flatten().argmax()]))
        if ls is not None:
            w, g, t = want_lse[b, :n], ls[b, :n].double(), tol_lse[b, :n]
            same = (w == g) | (torch.isnan(w) & torch.isnan(g))
            assert bool((same | ((g - w).abs() <= t)).all()), "%s seq %d lse" % (tag, b)
    return out


def queries(B, T, H, D, dtype, seed, fused=0):
    """Contiguous, or a slice of a wider projection's output."""
    x = torch.randn((B, T, H + fused, D), generator=gen(seed, "cuda"), device="cuda").to(dtype)
    return x[:, :, :H]


# rows a cached head: 1 .. 16, 17 .. 32, 33 .. 64 and more take different kernels
SHAPES = [(1, 1, 1, 1), (3, 1, 8, 2), (2, 1, 32, 1), (2, 3, 24, 4), (2, 17, 4, 4), (3, 8, 16, 4), (2, 9, 28, 4), (1, 33, 4, 1), (2, 40, 12, 2), (1, 130, 6, 2)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("B,T,H,Hkv", SHAPES)
def test_causal_chunks(B, T, H, Hkv, D, dtype):
    lens = [0, 77, 300][:B] if B > 1 else [45]
    cache = make_cache(lens, T, 16, Hkv, D, dtype, seed=B * 1000 + T * 10 + H)
    check(cache, 0, queries(B, T, H, D, dtype, T, fused=3), None, tag="causal")


@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
def test_page_sizes_and_lengths_round_tiles_and_pages(ps):
    lens = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513]
    for T in (1, 2, 21):
        cache = make_cache(lens, T, ps, 2, 64, BF, seed=ps + T, layers=3)
        check(cache, 2, queries(len(lens), T, 6, 64, BF, ps), None, tag="page %d" % ps)


@pytest.mark.parametrize("D,dtype,H,Hkv", [(128, BF, 8, 2), (64, HF, 4, 4), (256, BF, 4, 1), (128, HF, 32, 4)])
@pytest.mark.parametrize("chain,nodes,width", [(1, 1, 1), (1, 10, 4), (1, 60, 10), (0, 12, 4), (5, 33, 16), (2, 131, 32)])
def test_trees(chain, nodes, width, D, dtype, H, Hkv):
    lens = [0, 3, 90, 257]
    T = chain + nodes
    cache = make_cache(lens, T, 16, Hkv, D, dtype, seed=nodes)
    mask = torch.stack([random_tree(nodes, width, gen(b + nodes))[1] for b in range(4)])
    n_new = [T, chain + nodes // 2, 0, max(1, chain)]
    for b, n in enumerate(n_new):                            # nodes a tree does not have: finalize_tree leaves zeros
        mask[b, max(0, n - chain):] = 0
        mask[b, :, max(0, n - chain):] = 0
    check(cache, 0, queries(4, T, H, D, dtype, chain), n_new, mask.cuda(), tag="tree")


def test_rows_that_see_nothing():
    # no prefix, no chain: a node whose mask row is empty sees nothing; neither does one whose page there is none of
    for H, Hkv in ((4, 4), (16, 2), (32, 1)):
        cache = make_cache([0, 0, 40], 20, 16, Hkv, 128, BF, seed=3)
        mask = torch.stack([random_tree(20, 5, gen(b))[1] for b in range(3)])
        mask[0, 7] = 0
        mask[1] = 0
        mask[2, 19] = 0
        out = check(cache, 0, queries(3, 20, H, 128, BF, 1), [20, 20, 20], mask.cuda(), tag="empty rows")
        assert bool((out[0, 7] == 0).all()) and bool((out[1] == 0).all()) and bool((out[2, 19] != 0).any())
        cache.page_table[0] = -1
        out = check(cache, 0, queries(3, 20, H, 128, BF, 1), [20, 20, 20], mask.cuda(), tag="no pages")
        assert bool((out[0] == 0).all())


@pytest.mark.parametrize("H,T", [(2, 1), (8, 3), (8, 8), (16, 40)])
def test_pages_that_are_none_are_left_out(H, T):
    cache = make_cache([100, 200, 30], T, 16, 2, 64, BF, seed=9)
    cache.page_table[0, 2] = -1
    cache.page_table[1, 0] = cache.pages
    cache.page_table[1, 5] = 2 ** 31 - 1
    cache.page_table[2, 1] = -2 ** 31
    check(cache, 0, queries(3, T, H, 64, BF, 1), None, tag="bad pages")


# of all kernels, of parts that are joined either way, and of more sequences than a wavefront has lanes
@pytest.mark.parametrize("H,Hkv,T,D,B", [(2, 2, 1, 64, 3), (8, 2, 3, 128, 3), (8, 2, 8, 64, 3), (16, 2, 40, 128, 3), (4, 2, 70, 256, 3), (2, 1, 1, 64, 130)])
def test_what_attention_leaves_out_shows_in_the_status(H, Hkv, T, D, B):
    full, invalid = 2, 4
    lens = ([100, 5000, 30] + [20] * B)[:B]
    cache = make_cache(lens, T, 16, Hkv, D, BF, seed=9, max_pages=-(-(5000 + T) // 16))
    q = queries(B, T, H, D, BF, 1)
    status = lambda: cache.status.view(torch.int32).tolist()
    n = [T] * B
    cache.page_table[0, -(-(100 + T) // 16):] = -1           # none behind its keys: nothing is left out
    check(cache, 0, q, None, tag="all there")
    assert status() == [0] * B
    n[2] = 0
    cache.page_table[2] = -1                                 # nothing is asked of it
    cache.page_table[1, 200] = -7
    check(cache, 0, q, n, tag="a page is missing")
    assert status() == [0, invalid] + [0] * (B - 2)
    cache.status.view(torch.int32).zero_()
    cache.length[B - 1] = cache.max_pages * 16 - T + 1       # room for all tokens but one
    cache.page_table[B - 1, :] = 0
    n[B - 1] = T
    check(cache, 0, q, n, tag="no room")
    want = [0, invalid] + [0] * (B - 2)
    want[B - 1] |= full
    assert status() == want
    cache.length[B - 1] = 10 ** 9                            # and none at all, for more than there are slots
    cache.status.view(torch.int32).zero_()
    check(cache, 0, q, [0] * (B - 1) + [T + 5], tag="full")
    assert status() == [0] * (B - 1) + [full]


def test_lengths_and_counts_out_of_range():
    cache = make_cache([40, 40, 40, 40], 8, 16, 2, 64, BF, seed=1)
    cache.length.copy_(torch.tensor([-5, 10 ** 9, 44, 40], dtype=torch.int32))
    check(cache, 0, queries(4, 8, 4, 64, BF, 2), [8, 8, 100, -3], tag="clamped")


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("H,Hkv,T0", [(2, 2, 1), (8, 2, 1), (16, 2, 1), (8, 1, 5)])
def test_what_a_row_does_not_see_cannot_matter(H, Hkv, T0, D):
    """Infinities and NaN behind the last token, in slots behind n_new, and in nodes that a row does not see."""
    nodes, chain = 12, T0
    T = chain + nodes
    lens = [5, 70, 31]
    cache = make_cache(lens, T, 16, Hkv, D, BF, seed=21)
    mask = torch.stack([random_tree(nodes, 4, gen(b))[1] for b in range(3)])
    n_new = [T, T - 4, T]
    mask[1, nodes - 4:] = 0
    mask[1, :, nodes - 4:] = 0
    q = queries(3, T, H, D, BF, 5)
    clean = check(cache, 0, q, n_new, mask.cuda(), tag="clean").clone()
    bad = torch.tensor([float("nan"), float("inf"), float("-inf"), torch.finfo(BF).max], device="cuda").to(BF)

    def poison(b, at, what, x):
        page, row = int(cache.page_table[b, at // 16]), at % 16
        what[0, page, :, row] = x
    held = [-(-(l + T) // 16) * 16 for l in lens]
    for b in range(3):                                       # behind the last token
        for at in range(lens[b] + n_new[b], held[b]):
            poison(b, at, cache.k, bad[at % 4])
            poison(b, at, cache.v, bad[(at + 1) % 4])
    dirty = check(cache, 0, q, n_new, mask.cuda(), tag="behind the last")
    for b in range(3):
        assert torch.equal(dirty[b, :n_new[b]], clean[b, :n_new[b]])
    leaf = nodes - 1                                         # nobody else sees the last node
    assert int(mask[0, :, leaf].sum()) == 1
    for kind in range(3):
        poison(0, lens[0] + chain + leaf, cache.v, bad[kind])
        poison(0, lens[0] + chain + leaf, cache.k, bad[3 - kind if kind else 0])
        got = check(cache, 0, q, n_new, mask.cuda(), tag="a node that others do not see")
        assert torch.equal(got[0, :T - 1], clean[0, :T - 1])
    # one element of a value that two rows see
    page, row = int(cache.page_table[2, (lens[2] + chain) // 16]), (lens[2] + chain) % 16
    cache.v[0, page, :, row, 3] = float("inf")
    got = check(cache, 0, q, n_new, mask.cuda(), tag="an infinite value")
    sees = mask[2, :, 0].bool()
    assert bool(torch.isinf(got[2, chain:, :, 3][sees.cuda()]).all()) and torch.equal(got[2, chain:][~sees.cuda()], clean[2, chain:][~sees.cuda()])


@pytest.mark.parametrize("B,T,H,Hkv,D,lens", [(1, 1, 8, 1, 128, [20011]), (2, 1, 4, 4, 64, [9000, 3]), (1, 4, 32, 4, 128, [7777]), (3, 20, 16, 2, 128, [5000, 1, 12000]),
                                              (1, 2, 16, 1, 256, [6001]), (1, 40, 8, 2, 256, [3003]), (70, 1, 8, 2, 64, None), (130, 2, 4, 1, 64, None)])
def test_long_sequences_are_split_and_joined(B, T, H, Hkv, D, lens):
    lens = lens or [(b * 37) % 900 + (6000 if b == 5 else 0) for b in range(B)]
    cache = make_cache(lens, T, 32, Hkv, D, BF, seed=B)
    check(cache, 0, queries(B, T, H, D, BF, 3), [T - (b % 2) * (T > 1) for b in range(B)], tag="split")


@pytest.mark.parametrize("D,dtype", [(64, HF), (128, BF), (256, BF)])
@pytest.mark.parametrize("B,Hkv,T,H,nodes", [(31, 8, 5, 32, 4), (32, 8, 5, 32, 4), (255, 1, 17, 1, 0), (256, 1, 32, 1, 31), (64, 8, 3, 16, 2), (63, 8, 1, 8, 0)])
def test_many_sequences_of_few_rows(B, Hkv, T, H, nodes, D, dtype):
    """Numbers of sequences at which a call of few rows takes another kernel or other parts."""
    lens = [(b * 37) % 150 + (900 if b == 7 else 0) for b in range(B)]
    cache = make_cache(lens, T, 16, Hkv, D, dtype, seed=B + T)
    mask = torch.stack([random_tree(nodes, 3, gen(b))[1] for b in range(B)]).cuda() if nodes else None
    check(cache, 0, queries(B, T, H, D, dtype, 3), [T - (b % 3 == 1) * (T > 1) for b in range(B)], mask, tag="many")


def test_the_largest_batch():
    lens = [(b * 7919) % 70 for b in range(4096)]
    cache = make_cache(lens, 1, 16, 1, 64, BF, seed=5)
    n = [(b * 31) % 3 != 0 for b in range(4096)]
    q = queries(4096, 1, 2, 64, BF, 1)
    out = cache.attention(0, q, n_new=torch.tensor(n, dtype=torch.int32, device="cuda"), out=torch.full_like(q, 7.0))
    few = list(range(0, 4096, 97))
    for b in few:
        want = attention_reference(_one(cache, b), 0, q[b:b + 1], [int(n[b])], None, 0.125, [lens[b]])
        if n[b]:
            assert bool(((out[b:b + 1].double() - want[0]).abs() <= want[2]).all()), b
        else:
            assert bool((out[b] == 7.0).all())


def _one(cache, b):
    from paper_2502_13652_amd import PagedCache
    return PagedCache.of_tensors(cache.k, cache.v, cache.page_table[b:b + 1].contiguous(), cache.length[b:b + 1].contiguous(), cache.refcount)


def test_the_largest_tree():
    cache = make_cache([77], 1025, 32, 1, 64, BF, seed=9)
    mask = random_tree(1024, 8, gen(3))[1][None].cuda()
    check(cache, 0, queries(1, 1025, 2, 64, BF, 4), None, mask, tag="1024 nodes")


def test_a_long_prompt_in_chunks():
    cache = make_cache([0, 700], 600, 64, 2, 64, HF, seed=4)
    check(cache, 0, queries(2, 600, 6, 64, HF, 3), [600, 333], tag="chunk")


def test_large_scores_and_scales():
    cache = make_cache([64, 5], 3, 16, 2, 128, BF, seed=8)
    q = queries(2, 3, 4, 128, BF, 3)
    check(cache, 0, q, None, scale=0.0, tag="flat")
    cache.k.mul_(30)
    check(cache, 0, q, None, scale=1.0, tag="sharp")
    q[0, 0] = float("nan")
    q[1, 2, 1, 5] = float("inf")
    check(cache, 0, q, None, tag="queries that are no numbers")


def test_offsets_past_32_bits():
    # the last layer's pages begin beyond 2^32 bytes, and beyond 2^31 elements, of each pool
    from paper_2502_13652_amd import PagedCache
    layers, pages, Hkv, ps, D = 9, 1024, 8, 256, 128
    cache = PagedCache(2, layers, pages, ps, Hkv, D, 8, dtype=BF)
    assert cache.k.numel() > 2 ** 31
    small = make_cache([300, 777], 2, ps, Hkv, D, BF, seed=2)
    n = small.pages
    cache.k[layers - 1, pages - n:] = small.k[0]
    cache.v[layers - 1, pages - n:] = small.v[0]
    t = small.page_table
    cache.page_table[:, :t.shape[1]] = torch.where(t >= 0, t + (pages - n), t)
    cache.length.copy_(small.length)
    q = queries(2, 2, 16, D, BF, 1)
    a, b = cache.attention(layers - 1, q), small.attention(0, q)
    assert torch.equal(a, b)


def test_heads_past_31_bits():
    """So many query heads over one cached head that the last ones lie beyond 2^31 bytes of their token's row.  One key: each gets its value, whatever it asks."""
    H, D = (1 << 22) + 200, 256
    cache = make_cache([0], 1, 16, 1, D, BF, seed=3)
    q = torch.zeros((1, 1, H, D), dtype=BF, device="cuda")
    q[0, 0, -300:] = queries(1, 1, 300, D, BF, 5)[0, 0]
    lse = torch.zeros((1, 1, H), device="cuda")
    out = cache.attention(0, q, lse=lse)
    page = int(cache.page_table[0, 0])
    assert bool((out[0, 0] == cache.v[0, page, 0, 0]).all())
    k, last = cache.k[0, page, 0, 0].double(), q[0, 0, -300:].double()
    x, size = last @ k * D ** -0.5, last.abs() @ k.abs() * D ** -0.5
    tol = (D + 4) * 2.0 ** -24 * size + 4 * 2.0 ** -23 * (1 + size) + 66 * 2.0 ** -23 + x.abs() * 2.0 ** -22       # as attention_reference counts them
    assert bool((lse[0, 0, :-300].abs() <= 70 * 2.0 ** -23).all()) and bool(((lse[0, 0, -300:].double() - x).abs() <= tol).all())


def test_strided_outputs_and_single_heads():
    cache = make_cache([33, 64], 5, 16, 1, 64, BF, seed=6)
    q = queries(2, 5, 3, 64, BF, 2, fused=2)
    want = cache.attention(0, q)
    wide = torch.full((2, 5, 7, 64), 3.0, dtype=BF, device="cuda")
    out = wide[:, :, 2:5]
    cache.attention(0, q, out=out)
    assert torch.equal(out, want) and bool((wide[:, :, :2] == 3).all()) and bool((wide[:, :, 5:] == 3).all())
    one = q[:, :, :1]
    assert torch.equal(cache.attention(0, one), want[:, :, :1])


def test_the_same_call_gives_the_same_bits_on_streams_and_in_graphs():
    lens = [5000, 10, 900]
    cache = make_cache(lens, 33, 16, 2, 128, BF, seed=12)
    mask = torch.stack([random_tree(32, 8, gen(b))[1] for b in range(3)]).cuda()
    q = queries(3, 33, 8, 128, BF, 4)
    n_new = torch.tensor([33, 20, 1], dtype=torch.int32, device="cuda")
    want = cache.attention(0, q, n_new=n_new, mask=mask, out=torch.zeros_like(q))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = torch.zeros_like(q)
    cache.attention(0, q, n_new=n_new, mask=mask, out=got, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.attention(0, q, n_new=n_new, mask=mask, out=out)
    for length in ([5000, 10, 900], [1, 3000, 0], [4999, 11, 901]):
        cache.length.copy_(torch.tensor(length, dtype=torch.int32))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        again = cache.attention(0, q, n_new=n_new, mask=mask, out=torch.zeros_like(q))
        torch.cuda.synchronize()
        assert torch.equal(out, again)


def test_graphs_replayed_at_once_have_workspaces_of_their_own():
    """Long splits in two graphs on two streams and an eager call beside them, over and over; a graph captured before any eager call."""
    lens = [30000, 10, 900]
    cache = make_cache(lens, 2, 16, 1, 128, BF, seed=12)
    qs = [queries(3, 2, 8, 128, BF, 4 + i) for i in range(3)]
    outs = [torch.zeros_like(q) for q in qs]
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cache.attention(0, qs[i], out=outs[i])
        graphs.append(g)
    want = [make_cache(lens, 2, 16, 1, 128, BF, seed=12).attention(0, q) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        cache.attention(0, qs[2], out=outs[2])
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


def test_a_stream_clears_the_counters_that_it_uses():
    """The first call on a stream, where memory holds other values and the current stream is busy."""
    cache = make_cache([20000], 1, 16, 1, 128, BF, seed=3)
    q = queries(1, 1, 4, 128, BF, 4)
    want = cache.attention(0, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (torch.cuda.current_stream(), s):
        with torch.cuda.stream(stream):
            held = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (1 << 21, 1 << 23, 1 << 24, 1 << 26)]
            del held
    torch.cuda.synchronize()
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    cache.attention(0, q, out=out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    torch.cuda.synchronize()
    fresh = make_cache([20000], 1, 16, 1, 128, BF, seed=3)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        out = fresh.attention(0, q, stream=torch.cuda.default_stream())
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_captures_leave_no_workspaces_behind():
    cache = make_cache([3000, 7], 1, 16, 1, 64, BF, seed=3)
    q = queries(2, 1, 4, 64, BF, 4)
    want = cache.attention(0, q)
    s = torch.cuda.Stream()
    graphs = []
    for _ in range(3):
        g, out = torch.cuda.CUDAGraph(), torch.zeros_like(q)
        with torch.cuda.graph(g, stream=s):
            cache.attention(0, q, out=out)
            cache.attention(0, q, out=out)
        graphs.append((g, out))
    assert sum(len(w) for _, w in cache._attention_ws.values()) == 2
    for _ in range(3):
        for g, out in graphs:
            out.zero_()
            g.replay()
            other = torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda")
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            del other


# of all kernels, and of parts that are joined by the last of them and by a launch
MEANS = [(2, 1, 8, 2, [3, 170]), (2, 4, 8, 2, [0, 140]), (1, 9, 16, 4, [210]), (2, 40, 8, 2, [5, 150]), (1, 70, 4, 2, [180])]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("B,T,H,Hkv,lens", MEANS + [(1, 1, 4, 1, [3500]), (1, 20, 4, 1, [3000]), (1, 70, 2, 1, [2500])])
def test_a_mean_of_equal_values_is_that_value(B, T, H, Hkv, lens, D, dtype):
    """Sharp rows over values that are the same for all keys: what the weights' rounding to 16 bits adds to the weighted sum it adds to the divisor too.  What is left is the sums'
    roundings in fp32, at most n 2^-23 relative in each for n keys (the terms have one sign), and two of the division: below half a step of a bf16 value,
    2^-9 relative at least, for 8000 keys, and of an fp16 one, 2^-12, for 1000: rounding then gives the value itself."""
    if dtype is HF:
        lens = [min(l, 900) for l in lens]
    cache = make_cache(lens, T, 16, Hkv, D, dtype, seed=D + T)
    c = torch.randn((1, 1, Hkv, 1, D), generator=gen(D, "cuda"), device="cuda").to(dtype)
    c[..., ::4] = c[..., ::4].sign()
    cache.v.copy_(c.expand_as(cache.v))
    q = queries(B, T, H, D, dtype, T)
    print("equal values", (B, T, H, Hkv, D), lens, dtype, flush=True)
    out = cache.attention(0, q, scale=4 * D ** -0.5, lse=torch.empty((B, T, H), device="cuda") if T % 2 else None)
    assert torch.equal(out, c[0, 0, :, 0].repeat_interleave(H // Hkv, 0)[None, None].expand_as(out))


@pytest.mark.parametrize("bits", [24.9, 25.1, 28.0])
@pytest.mark.parametrize("B,T,H,Hkv,D", [(1, 1, 4, 1, 64), (1, 20, 3, 1, 128), (1, 70, 2, 1, 64), (1, 5, 2, 1, 256), (1, 70, 2, 1, 256)])
def test_half_precision_tails_behind_a_sharp_key(B, T, H, Hkv, D, bits):
    """One key has next to all of a row's weight and a value of 0 in half of the dimensions: what comes out there is the sum of 30000 weights of about 2^-25 of its.
    Halves below 2^-14 are multiples of 2^-24: with the row's largest weight at 2^13 or more a weight is off by 2^-38 of it at most, n of them by n 2^-38 (the values are 1), and the output,
    itself such a half, by 2^-25."""
    n = 30000
    for at in (0, 17, n - 1):                                # where the sharp key lies
        cache = make_cache([n], T, 64, Hkv, D, HF, seed=7)
        cache.k.zero_()
        cache.v.fill_(1.0)
        page, row = int(cache.page_table[0, at // 64]), at % 64
        cache.k[0, page, :, row, 0] = bits * 0.6931471805599453
        cache.v[0, page, :, row, ::2] = 0.0
        q = torch.zeros((B, T, H, D), dtype=HF, device="cuda")
        q[..., 0] = 1.0
        print("tail", (T, H, D), bits, at, flush=True)
        lse = torch.zeros((B, T, H), device="cuda")
        got = cache.attention(0, q, scale=1.0, lse=lse)
        want, want_lse, tol, tol_lse = attention_reference(cache, 0, q, [T], None, 1.0)
        assert 1e-6 * 2 ** (28 - bits) < float(want[0, 0, 0, 0]) < 1e-3
        err = (got.double() - want).abs() - tol - n * 2.0 ** -38 - 2.0 ** -25
        assert float(err.max()) <= 0, (float(got[0, 0, 0, 0]), float(want[0, 0, 0, 0]))
        assert bool(((lse.double() - want_lse).abs() <= tol_lse).all())


@pytest.mark.parametrize("T,H,Hkv,D", [(1, 4, 1, 128), (20, 3, 1, 64), (70, 2, 1, 128), (5, 2, 1, 256), (70, 2, 1, 256)])
def test_values_near_the_largest_do_not_overflow(T, H, Hkv, D):
    """Values of 2^125: two keys weigh something, the later one 2^6.9 times as much as the first, in another tile of the same wavefront's.  The sum
    of their weights is below 2 where none is above 1, and the mean is 2^125."""
    cache = make_cache([300], T, 16, Hkv, D, BF, seed=7)
    cache.k.zero_()
    cache.k[..., 0] = -80.0
    for at, x in ((0, 0.0), (128, 4.8)):
        cache.k[0, int(cache.page_table[0, at // 16]), :, at % 16, 0] = x
    cache.v.fill_(2.0 ** 125)
    q = torch.zeros((1, T, H, D), dtype=BF, device="cuda")
    q[..., 0] = 1.0
    assert bool((cache.attention(0, q, scale=1.0) == 2.0 ** 125).all())


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("T,H,Hkv,D,n", [(1, 4, 1, 128, 90), (1, 4, 1, 64, 5000), (20, 3, 1, 64, 300), (70, 2, 1, 128, 400), (5, 2, 1, 256, 90), (70, 2, 1, 256, 3000)])
def test_scores_of_any_size(T, H, Hkv, D, n, sign, dtype):
    """Scores of 2^19 to 2^35 (2^26 for halves), far apart or equal: a row is the value of its largest score's key, or the mean of two whose scores are the same.  The scores are
    exact, two differ by 2^-7 of their size at least, so all other weights are 0."""
    at = [n // 3, n - 2]
    pick = torch.randint(0, 60, (n,), generator=gen(n))
    for power in (10, 13) if dtype is HF else (10, 15, 17):
        size = 2.0 ** power
        for both in (False, True):
            cache = make_cache([n], T, 16, Hkv, D, dtype, seed=7)
            cache.k.zero_()
            pos = torch.arange(n, device="cuda")
            page, row = cache.page_table[0].long()[pos // 16], pos % 16
            level = pick.clone()
            level[at[0]], level[at[1]] = 64, 64 if both else 63       # 63 and fewer: at least a 128th less
            cache.k[0, page, 0, row, 0] = (sign * size * (1 + sign * level.cuda() / 128)).to(dtype)
            last = cache.page_table[0].long()[(n + torch.arange(T, device="cuda")) // 16]
            cache.k[0, last, 0, (n + torch.arange(T, device="cuda")) % 16, 0] = float(sign * size)      # the new tokens: level 0
            q = torch.zeros((1, T, H, D), dtype=dtype, device="cuda")
            q[..., 0] = size
            print("scores", (T, H, D, n), sign, dtype, power, both, flush=True)
            lse = torch.zeros((1, T, H), device="cuda")
            got = cache.attention(0, q, scale=1.0, lse=lse)
            v = [cache.v[0, page[i], 0, row[i]].double() for i in at]
            want = (v[0] + v[1]) / 2 if both else v[0]
            u = torch.finfo(dtype).eps / 2
            assert bool(((got.double() - want).abs() <= u * want.abs() + 2.0 ** -22 * (v[0].abs() + v[1].abs())).all())
            top = float(cache.k[0, page[at[0]], 0, row[at[0]], 0]) * float(q[0, 0, 0, 0])
            assert bool(((lse.double() - top).abs() <= 1 + 2.0 ** -22 * abs(top)).all())


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("H,T,D", [(4, 1, 128), (3, 20, 64), (2, 70, 128), (2, 5, 256)])
def test_the_log_of_a_number_of_equal_weights(H, T, D, dtype):
    """Scores of 0: the sum of n weights is exact, and what is left is the logarithm's step (2^-23 relative), its product's with log 2 and that constant's, 2^-24 each."""
    lens = [0, 1, 2, 4, 6, 10, 30, 99, 700]
    cache = make_cache(lens, T, 16, 1, D, dtype, seed=3)
    lse = torch.zeros((len(lens), T, H), device="cuda")
    cache.attention(0, torch.zeros((len(lens), T, H, D), dtype=dtype, device="cuda"), lse=lse)
    want = torch.log(torch.tensor(lens, device="cuda").double()[:, None] + 1 + torch.arange(T, device="cuda"))[:, :, None]
    assert bool(((lse.double() - want).abs() <= 2.0 ** -22 * want).all()), float(((lse.double() - want).abs() - 2.0 ** -22 * want).max())


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("B,T,H,Hkv,D", [(7, 1, 8, 2, 128), (7, 1, 8, 8, 64), (7, 3, 16, 4, 128), (7, 5, 6, 2, 64)])
def test_few_rows_are_as_exact_as_their_type(B, T, H, Hkv, D, dtype):
    """Rows that share a tile of 16: their weights are taken as two numbers of 16 bits, which a weight differs from by 2^-16 of it at most (each leaves half a step, 2^-8 or less).  Values that are positive, so
    that the sum of weighted sizes is the output itself; but for that difference the tolerance is attention_reference's without its term for weights of one such number."""
    lens = [0, 1, 2, 5, 40, 300, 3000][:B]
    cache = make_cache(lens, T, 16, Hkv, D, dtype, seed=D + T)
    cache.v.copy_((cache.v.float().abs() * 3 + 0.01).to(dtype))
    q = queries(B, T, H, D, dtype, T)
    got = cache.attention(0, q)
    want, _, tol, _ = attention_reference(cache, 0, q, [T] * B, None, D ** -0.5)
    u = torch.finfo(dtype).eps / 2
    tol = tol - want * u * (1 + u) + want * 2.0 ** -16
    assert float(((got.double() - want).abs() - tol).max()) <= 0


def test_refusals():
    from paper_2502_13652_amd import PagedCache
    from paper_2502_13652_amd.binding import C2TError
    cache = make_cache([10, 20], 4, 16, 2, 64, BF, seed=1)
    q = queries(2, 4, 4, 64, BF, 1)
    for bad in (q.float(), q[:1], q[:, :, :, :32], q.transpose(1, 2), q.cpu()):
        with pytest.raises(ValueError):
            cache.attention(0, bad)
    for kw in (dict(n_new=torch.zeros(2, device="cuda")), dict(n_new=torch.zeros(3, dtype=torch.int32, device="cuda")),
               dict(mask=torch.zeros((2, 3, 4), dtype=torch.uint8, device="cuda")), dict(mask=torch.zeros((2, 3, 3), device="cuda")),
               dict(lse=torch.zeros((2, 4, 3), device="cuda")), dict(out=torch.zeros((2, 4, 4, 32), dtype=BF, device="cuda"))):
        with pytest.raises(ValueError):
            cache.attention(0, q, **kw)
    for kw, code in ((dict(layer=1), -1), (dict(layer=-1), -1), (dict(layer=0, mask=torch.zeros((2, 5, 5), dtype=torch.uint8, device="cuda")), -1),
                     (dict(layer=0, scale=float("nan")), -1), (dict(layer=0, scale=-1.0), -1)):
        with pytest.raises(C2TError) as e:
            cache.attention(q=q, **kw)
        assert e.value.code == code
    with pytest.raises(C2TError) as e:
        cache.attention(0, q[:, :, :3])                      # three query heads over two cached ones
    assert e.value.code == -1
    with pytest.raises(C2TError) as e:
        cache.attention(0, q, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -3
    need = cache.attention_workspace_bytes(4, 4)
    for bad in (torch.zeros(need, dtype=torch.uint8), torch.zeros(need, dtype=torch.int32, device="cuda"), torch.zeros(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            cache.attention(0, q, workspace=bad)
    for kw in (dict(page_size=24), dict(page_size=512), dict(head_dim=96), dict(batch=5000)):
        a = dict(batch=2, layers=1, pages=4, page_size=16, kv_heads=1, head_dim=64, max_pages=2)
        a.update(kw)
        with pytest.raises(C2TError) as e:
            PagedCache(**a)
        assert e.value.code == -2
