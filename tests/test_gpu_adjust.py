"""Penalties, biases and masks on logits against the definition in 64 bits: rows of a tree and of a context's frontier."""
import numpy as np
import pytest
import torch

import workloads as W
from _harness import make_gpu, to_np
from _serving import adjust_reference, gen, half_step, random_tree

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make_terms(B, rows, V, seed, ctx=200, biases=40, allowed="row", few=0):
    rng = np.random.default_rng(seed)
    top = min(V, few) if few else V
    t = dict(tokens=rng.integers(-2, top + 2, (B, ctx)), n_tokens=rng.integers(0, ctx + 1, B), n_prompt=None,
             repetition=rng.uniform(0.8, 1.6, B), frequency=rng.uniform(-0.5, 1.0, B), presence=rng.uniform(-0.5, 1.0, B),
             bias_tokens=rng.integers(-1, top + 1, (B, biases)), bias=4 * rng.standard_normal((B, biases)), n_bias=rng.integers(0, biases + 1, B), allowed=None)
    t["n_tokens"][0] = ctx
    t["n_prompt"] = (t["n_tokens"] * rng.uniform(0, 1.2, B)).astype(int)
    words = (V + 31) // 32
    if allowed:
        r = rows if allowed == "row" else 1
        t["allowed"] = rng.integers(0, 1 << 32, (B, r, words), dtype=np.uint32)
        t["allowed"][:, ::2] |= rng.integers(0, 1 << 32, (B, (r + 1) // 2, words), dtype=np.uint32)
        t["allowed"][0, 0] = 0xffffffff
        t["allowed"][-1, -1] = 0                             # a state that allows nothing
    return t


def on_gpu(t):
    from paper_2502_13652_amd import LogitAdjustments
    kw = {}
    for k, v in t.items():
        if v is None:
            continue
        if k == "allowed":
            kw[k] = torch.from_numpy(v.view(np.int32)).cuda()
        else:
            kw[k] = torch.from_numpy(np.asarray(v)).to(F32 if k in ("repetition", "frequency", "presence", "bias") else torch.int32).cuda()
    t32 = {k: (None if v is None else v.astype(np.float32).astype(np.float64) if k in ("repetition", "frequency", "presence", "bias") else v) for k, v in t.items()}
    return LogitAdjustments(**kw), t32


def check_row(x, got, t, b, path, r, dtype, tag):
    """x, got: the row's V logits before and after, as float64; bits must be kept where nothing is done."""
    toks = [] if t.get("tokens") is None else t["tokens"][b][:max(0, t["n_tokens"][b])].tolist()
    n_prompt = 0 if t.get("n_prompt") is None else min(int(t["n_prompt"][b]), len(toks))
    al = None if t.get("allowed") is None else t["allowed"][b][min(r, t["allowed"].shape[1] - 1)]
    want, touched = adjust_reference(x, toks, n_prompt, path, t, b, al)
    # past the type's largest number by half a step or more, the nearest it has is infinity
    want = np.where(np.abs(want) >= torch.finfo(dtype).max * (1 + half_step(dtype) / 2), np.copysign(np.inf, want), want)
    masked = np.isneginf(want) & ~np.isneginf(x)
    same = ~touched & ~masked
    np.testing.assert_array_equal(got[same], x[same], err_msg="%s: logits that nothing is done to" % tag)
    nan = np.isnan(want)
    assert (np.isnan(got) == nan).all(), tag
    # five operations and the sum of a token's biases in fp32, on values up to `size`; then the rounding
    count = len(toks) + len(path)
    size = np.abs(np.where(np.isfinite(x), x, 0)) * 2 + abs(t["frequency"][b] if t.get("frequency") is not None else 0) * count + 2 + \
        (np.abs(t["bias"][b]).sum() if t.get("bias") is not None else 0)
    with np.errstate(invalid="ignore"):
        ok = (got == want) | nan | (np.abs(got - want) <= half_step(dtype) * np.abs(want) + (8 + (t["bias"].shape[1] if t.get("bias") is not None else 0)) * 2.0 ** -24 * size)
    assert ok.all(), "%s: token %d: %r, not %r" % (tag, int(np.argmin(ok)), got[~ok][0], want[~ok][0])


def logits_of(B, rows, V, dtype, seed, pad=0):
    per = 128 // torch.finfo(dtype).bits
    stride = -(-V // per) * per + pad * per
    x = torch.full((B, rows, stride), 55.0, dtype=dtype, device="cuda")
    x[:, :, :V] = 5 * torch.randn((B, rows, V), generator=gen(seed, "cuda"), device="cuda")
    return x


def tree_of(B, N, width, vocab, seed):
    g = gen(seed)
    made = [random_tree(N, width, g) for _ in range(B)]
    n = torch.randint(0, N + 1, (B,), generator=g, dtype=torch.int32)
    n[0] = N
    return dict(tokens=torch.randint(0, vocab, (B, N), generator=g, dtype=torch.int32).cuda(), parent=torch.stack([p for p, _ in made]).cuda(),
                mask=torch.stack([m for _, m in made]).cuda(), n_nodes=n.cuda())


def path_of(tree, b, node):
    out, parent, tokens = [], tree["parent"][b].tolist(), tree["tokens"][b].tolist()
    while node >= 0:
        out.append(tokens[node])
        node = parent[node]
    return out


def check_tree(x, tree, t, V, tag, in_place=False):
    from paper_2502_13652_amd import adjust_tree_logits
    adj, t32 = on_gpu(t)
    B, rows = x.shape[0], x.shape[1]
    before = x.double().cpu().numpy()
    out = x if in_place else torch.full_like(x, 7.0)
    print("adjust", tag, tuple(x.shape), V, x.dtype, flush=True)
    got = adjust_tree_logits(x, tree, adj, vocab=V, out=out)
    torch.cuda.synchronize()
    assert got is out
    after = out.double().cpu().numpy()
    if not in_place:
        np.testing.assert_array_equal(x.double().cpu().numpy(), before)
    n_nodes = [0] * B if tree is None else tree["n_nodes"].tolist()
    for b in range(B):
        live = 1 + n_nodes[b]
        behind = before if in_place else np.full_like(before, 7.0)
        np.testing.assert_array_equal(after[b, :, V:], behind[b, :, V:], err_msg="padding")
        np.testing.assert_array_equal(after[b, live:], behind[b, live:], err_msg="rows behind the tree")
        for r in range(live):
            check_row(before[b, r, :V], after[b, r, :V], t32, b, path_of(tree, b, r - 1) if tree is not None and r else [], r, x.dtype, "%s seq %d row %d" % (tag, b, r))
    return out


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,N,width,V,few", [(1, 1, 1, 1, 0), (2, 5, 2, 33, 0), (3, 12, 4, 1000, 50), (2, 40, 10, 8192, 100), (2, 9, 3, 8193, 0), (2, 17, 5, 20011, 30), (1, 60, 10, 32000, 0)])
def test_trees(B, N, width, V, few, dtype):
    t = make_terms(B, 1 + N, V, seed=V, few=few)
    tree = tree_of(B, N, width, few or V, V + 1)
    check_tree(logits_of(B, 1 + N, V, dtype, 3, pad=1), tree, t, V, "tree")
    check_tree(logits_of(B, 1 + N, V, dtype, 4), tree, t, V, "in place", in_place=True)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,N,width,V,few", [(3, 12, 4, 1000, 50), (2, 40, 10, 8193, 100), (1, 9, 3, 20011, 0)])
def test_in_place_without_a_mask(B, N, width, V, few, dtype):
    t = dict(make_terms(B, 1 + N, V, seed=V + 5, few=few), allowed=None)
    check_tree(logits_of(B, 1 + N, V, dtype, 4, pad=1), tree_of(B, N, width, few or V, V + 1), t, V, "in place, no mask", in_place=True)


@pytest.mark.parametrize("masked", [False, True])
def test_the_largest_tree(masked):
    """Deep paths whose tokens all lie in one stretch of the vocabulary."""
    t = make_terms(1, 1025, 300, seed=8)
    if not masked:
        t["allowed"] = None
    tree = tree_of(1, 1024, 8, 300, 3)
    check_tree(logits_of(1, 1025, 300, F32, 4), tree, t, 300, "1024 nodes")
    check_tree(logits_of(1, 1025, 300, BF, 4), tree, t, 300, "1024 nodes, in place", in_place=True)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("left_out", ["tokens", "n_prompt", "repetition", "frequency", "presence", "bias", "n_bias", "allowed", "all"])
def test_terms_that_are_left_out(left_out, dtype):
    t = make_terms(3, 7, 3001, seed=11, allowed="sequence", few=60)
    gone = {"tokens": ("tokens", "n_tokens", "n_prompt"), "bias": ("bias", "bias_tokens", "n_bias"), "all": tuple(t)}.get(left_out, (left_out,))
    for k in gone:
        t[k] = None
    x = logits_of(3, 7, 3001, dtype, 5)
    out = check_tree(x, tree_of(3, 6, 2, 60, 2) if left_out != "all" else tree_of(3, 6, 2, 60, 2), t, 3001, "without " + left_out)
    if left_out == "all":
        assert torch.equal(out[0, :, :3001].contiguous().view(torch.int16 if dtype == BF else torch.int32), x[0, :, :3001].contiguous().view(torch.int16 if dtype == BF else torch.int32))


def test_without_a_tree():
    x = logits_of(5, 1, 9001, F32, 5)
    check_tree(x, None, make_terms(5, 1, 9001, seed=3, few=40), 9001, "single rows")
    check_tree(logits_of(1, 1, 700, BF, 5), None, make_terms(1, 1, 700, seed=4), 700, "one row")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_that_are_no_ordinary_numbers(dtype):
    B, N, V = 2, 4, 500
    x = logits_of(B, 1 + N, V, dtype, 8)
    odd = torch.tensor([float("inf"), float("-inf"), float("nan"), torch.finfo(BF).min, torch.finfo(BF).max, -0.0, 0.0, 1e-30], device="cuda")
    x[:, :, :400] = odd.to(dtype)[torch.arange(400, device="cuda") % 8]
    t = make_terms(B, 1 + N, V, seed=6, few=450)
    t["frequency"][:], t["presence"][:] = 0.25, 0.5
    tree = tree_of(B, N, 2, 450, 3)
    check_tree(x, tree, t, V, "odd values")
    t["bias"][:, :5] = -np.inf                               # banned tokens
    t["n_bias"][:] = 5
    from paper_2502_13652_amd import adjust_tree_logits
    x = logits_of(B, 1 + N, V, dtype, 9)
    out = adjust_tree_logits(x, tree, on_gpu(t)[0], vocab=V)
    for b in range(B):
        for tok in t["bias_tokens"][b, :5]:
            if 0 <= tok < V:
                assert bool(torch.isneginf(out[b, :1 + int(tree["n_nodes"][b]), int(tok)]).all())


def test_long_contexts_and_one_token_many_times():
    V = 40000
    t = make_terms(2, 3, V, seed=1, ctx=70001, biases=1024, few=300)
    t["tokens"][1] = 17
    t["bias_tokens"][1, :] = 17                              # every entry biases the same token
    t["n_bias"][1] = 1024
    t["frequency"][:] = 0.001
    check_tree(logits_of(2, 3, V, F32, 2), tree_of(2, 2, 2, 300, 7), t, V, "long")


def test_trees_that_are_none():
    """Parents that point forward or outside end the path; counts out of range are cut."""
    from paper_2502_13652_amd import adjust_tree_logits
    B, N, V = 2, 6, 64
    t = dict(make_terms(B, 1 + N, V, seed=2), allowed=None)
    tree = tree_of(B, N, 2, V, 1)
    tree["parent"] = ints([[3, 0, 100, -7, 4, 2 ** 31 - 1], [-2 ** 31, 5, 1, 2, 3, 4]])
    tree["n_nodes"] = ints([N, 10 ** 9])
    tree["tokens"][0, 1] = -5
    tree["tokens"][1, 2] = V + 3
    adj, t32 = on_gpu(t)
    x = logits_of(B, 1 + N, V, F32, 1)
    out = adjust_tree_logits(x, tree, adj).double().cpu().numpy()
    for b in range(B):
        for r in range(1 + N):
            path, node, parent = [], r - 1, tree["parent"][b].tolist()
            while node >= 0:
                path.append(int(tree["tokens"][b, node]))
                node = parent[node] if parent[node] < node else -1
            check_row(x[b, r].double().cpu().numpy(), out[b, r], t32, b, path, r, F32, "seq %d row %d" % (b, r))
    tree["n_nodes"] = ints([-5, -1])
    untouched = torch.full_like(x, 3.0)
    adjust_tree_logits(x, tree, adj, out=untouched)
    assert bool((untouched[0] == 3.0).all()) and bool((untouched[1] == 3.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_frontier_rows_of_a_draft_phase(dtype):
    """Every layer's rows get the tokens of their own path; expand_layer on them equals expand_layer on the rows made by hand."""
    cfg = dict(idx=90, B=3, V=5003, dtype=dtype, D=4, F=6, K=5, h=8, beta=0.0, N=24, zipf_s=1.0, sigma=(1.0, 4.0), spike_frac=0.0, desc="adjusted frontier")
    cls = W.classifier(cfg, 1)
    a, b = make_gpu(cfg, cls), make_gpu(cfg, cls)
    t = make_terms(3, cfg["F"], cfg["V"], seed=5, few=200)
    t["allowed"][:, -1] |= np.uint32(0xff)
    adj, t32 = on_gpu(t)
    a.reset(); b.reset()
    paths = [[[]] for _ in range(3)]
    for l in range(cfg["D"]):
        x = W.logits_layer(cfg, l, device="cuda")
        per = 128 // torch.finfo(x.dtype).bits
        pad = torch.full((3, cfg["F"], -(-cfg["V"] // per) * per), 9.0, dtype=x.dtype, device="cuda")
        pad[:, :, :cfg["V"]] = x
        before = pad.clone()
        n_front = a.frontier()["n_frontier"].tolist() if l else [1] * 3
        assert a.adjust_logits(pad, adj) is pad
        after, old = pad.double().cpu().numpy(), before.double().cpu().numpy()
        for s in range(3):
            for r in range(n_front[s]):
                check_row(old[s, r, :cfg["V"]], after[s, r, :cfg["V"]], t32, s, paths[s][r], r, x.dtype, "layer %d seq %d row %d" % (l, s, r))
            np.testing.assert_array_equal(after[s, n_front[s]:], old[s, n_front[s]:])
        np.testing.assert_array_equal(after[:, :, cfg["V"]:], old[:, :, cfg["V"]:])
        other = torch.zeros_like(pad)
        b.adjust_logits(before, adj, out=other)
        a.expand_layer(pad); b.expand_layer(other)
        fa, fb = to_np(a.frontier()), to_np(b.frontier())
        for k in fa:
            np.testing.assert_array_equal(fa[k][:, :1] if k != "n_frontier" else fa[k], fb[k][:, :1] if k != "n_frontier" else fb[k])
        paths = [[paths[s][fa["parent_slot"][s, f]] + [int(fa["tokens"][s, f])] for f in range(fa["n_frontier"][s])] for s in range(3)]
    oa, ob = to_np(a.finalize_tree()), to_np(b.finalize_tree())
    for k in oa:
        np.testing.assert_array_equal(oa[k], ob[k])
    assert int(oa["n_nodes"].min()) > 8
    from paper_2502_13652_amd.binding import C2TError
    with pytest.raises(C2TError) as e:
        a.adjust_logits(pad, adj)                            # the phase is over
    assert e.value.code == -4


def test_captured_and_on_another_stream():
    from paper_2502_13652_amd import adjust_tree_logits
    B, N, V = 2, 10, 9000
    t = make_terms(B, 1 + N, V, seed=2, few=100)
    adj, _ = on_gpu(t)
    tree = tree_of(B, N, 3, 100, 3)
    x = logits_of(B, 1 + N, V, BF, 1)
    out = torch.zeros_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    adjust_tree_logits(x, tree, adj, out=out, stream=s)
    s.synchronize()
    same = lambda p, q: torch.equal(p.view(torch.int16), q.view(torch.int16))
    assert same(out, adjust_tree_logits(x, tree, adj, out=torch.zeros_like(x)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        adjust_tree_logits(x, tree, adj, out=out)
    for i in range(4):
        x.copy_(logits_of(B, 1 + N, V, BF, 10 + i))
        adj.n_tokens.copy_(ints([10 * i, 50]))
        tree["n_nodes"].copy_(ints([i, N - i]))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert same(out, adjust_tree_logits(x, tree, adj, out=torch.zeros_like(x))), i


def test_refusals():
    from paper_2502_13652_amd import LogitAdjustments, adjust_tree_logits
    from paper_2502_13652_amd.binding import C2TError
    x, tree = logits_of(2, 5, 100, F32, 1), tree_of(2, 4, 2, 100, 1)
    ok = LogitAdjustments(repetition=torch.ones(2, device="cuda"))
    for bad in (lambda: adjust_tree_logits(x.half(), tree, ok), lambda: adjust_tree_logits(x[:, :3], tree, ok), lambda: adjust_tree_logits(x, tree, ok, vocab=101),
                lambda: adjust_tree_logits(x, None, ok), lambda: adjust_tree_logits(x, dict(tree, tokens=tree["tokens"].long()), ok), lambda: adjust_tree_logits(x.cpu(), tree, ok),
                lambda: adjust_tree_logits(x, tree, ok, out=torch.zeros((2, 5, 100), dtype=BF, device="cuda")),
                lambda: adjust_tree_logits(x, tree, LogitAdjustments(tokens=ints([[1], [2]]))),
                lambda: adjust_tree_logits(x, tree, LogitAdjustments(bias=torch.zeros((2, 3), device="cuda"))),
                lambda: adjust_tree_logits(x, tree, LogitAdjustments(repetition=torch.ones(3, device="cuda"))),
                lambda: adjust_tree_logits(x, tree, LogitAdjustments(frequency=torch.ones(2, device="cuda", dtype=torch.float64))),
                lambda: adjust_tree_logits(x, tree, LogitAdjustments(allowed=torch.zeros((2, 5, 3), dtype=torch.int32, device="cuda")))):
        with pytest.raises((ValueError,)):
            bad()
    with pytest.raises(C2TError) as e:
        adjust_tree_logits(x, tree, LogitAdjustments(bias=torch.zeros((2, 1025), device="cuda"), bias_tokens=torch.zeros((2, 1025), dtype=torch.int32, device="cuda")))
    assert e.value.code == -2
    odd = torch.zeros(2 * 5 * 101, device="cuda").view(2, 5, 101)
    with pytest.raises(C2TError) as e:
        adjust_tree_logits(odd, tree, ok)
    assert e.value.code == -2
