"""A draft tree taken through its verification as a serving loop does it: adjusted draft rows, the tree, its tokens' K and V into the paged cache,
attention with the tree's mask in every layer, adjusted target logits, the accepted path committed; the cache it leaves and what later
tokens see are compared with a cache that had the accepted tokens written one after the other."""
import numpy as np
import pytest
import torch

import workloads as W
from _harness import make_gpu
from _serving import attention_reference, gen

pytestmark = pytest.mark.gpu


def accept(out, target, b):
    """Slots of the greedy path: from the root on, the child whose token the target's row of its parent has largest."""
    n, parent, tokens = int(out["n_nodes"][b]), out["parent"][b].tolist(), out["tokens"][b].tolist()
    path, at = [0], -1
    while True:
        best = int(target[b, at + 1].float().argmax())
        child = [i for i in range(n) if parent[i] == at and tokens[i] == best]
        if not child:
            return path, best
        at = child[0]
        path.append(at + 1)


@pytest.mark.parametrize("dtype,page_size", [("bf16", 16), ("f32", 64)])
def test_steps_of_a_serving_loop(dtype, page_size):
    from paper_2502_13652_amd import LogitAdjustments, PagedCache, adjust_tree_logits
    cfg = dict(idx=93, B=3, V=1009, dtype=dtype, D=3, F=6, K=4, h=6, beta=0.0, N=15, zipf_s=1.2, sigma=(0.5, 1.5), spike_frac=0.0, desc="a serving loop")
    B, V, N, F = cfg["B"], cfg["V"], cfg["N"], cfg["F"]
    layers, Hkv, Hq, D, T = 2, 2, 6, 64, 1 + cfg["N"]
    ctx = make_gpu(cfg, W.classifier(cfg, 2))
    caches = [PagedCache(B, layers, 60, page_size, Hkv, D, 12) for _ in range(2)]       # by trees; token by token
    gd = gen(77, "cuda")
    emb = torch.randn((layers, V, Hq + 2 * Hkv, D), generator=gd, device="cuda").to(torch.bfloat16)       # what a layer makes of a token
    history = torch.full((B, 400), -1, dtype=torch.int32, device="cuda")
    n_tokens = torch.tensor([5, 20, 1], dtype=torch.int32, device="cuda")
    prompt = torch.randint(0, V, (B, 20), generator=gd, device="cuda", dtype=torch.int32)
    for b in range(B):
        history[b, :n_tokens[b]] = prompt[b, :n_tokens[b]]
    one = torch.ones(B, device="cuda")
    adj = LogitAdjustments(tokens=history, n_tokens=n_tokens, n_prompt=n_tokens.clone(), repetition=1.2 * one, frequency=0.3 * one, presence=0.1 * one)
    grow = n_tokens - 1                                       # the last token of the prompt is the first step's root
    for c in caches:
        c.reserve(grow)
        for layer in range(layers):
            x = emb[layer][prompt.long()]
            c.write(layer, x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], n_new=grow)
        c.commit(torch.arange(20, dtype=torch.int32, device="cuda").repeat(B, 1), grow)
    root = torch.stack([prompt[b, int(n_tokens[b]) - 1] for b in range(B)])
    accepted_in_all = 0
    per = 128 // torch.finfo(W.torch_dtype(cfg)).bits
    stride = -(-V // per) * per
    for step in range(4):
        tree_cache, plain = caches
        ctx.reset()
        for l in range(cfg["D"]):
            x = torch.zeros((B, F, stride), dtype=W.torch_dtype(cfg), device="cuda")
            x[:, :, :V] = W.logits_layer(cfg, l, device="cuda", instance=step)
            ctx.adjust_logits(x, adj)
            ctx.expand_layer(x)
        out = ctx.finalize_tree()
        n_new = 1 + out["n_nodes"]
        tree_cache.reserve(n_new)
        ids = torch.cat([root[:, None], out["tokens"].clamp(min=0)], 1).long()
        for layer in range(layers):
            x = emb[layer][ids]
            tree_cache.write(layer, x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], n_new=n_new)
            got = tree_cache.attention(layer, x[:, :, :Hq], n_new=n_new, mask=out["mask"])
            want, _, tol, _ = attention_reference(tree_cache, layer, x[:, :, :Hq], n_new.tolist(), out["mask"], D ** -0.5)
            live = torch.isfinite(want)
            assert bool(((got.double() - want).abs() <= tol)[live].all()), (step, layer)
        # the draft's own rows stand in for the target's: its largest logits are the nodes' tokens often enough
        target = torch.zeros((B, T, stride), dtype=W.torch_dtype(cfg), device="cuda")
        target[:, :, :V] = torch.randn((B, T, V), generator=gen(step, "cuda"), device="cuda")
        for b in range(B):
            for i in range(int(out["n_nodes"][b])):
                target[b, 1 + int(out["parent"][b, i]), int(out["tokens"][b, i])] += 12.0 - i
        adjust_tree_logits(target, out, adj, vocab=V, out=target)
        paths = [accept(out, target[:, :, :V], b) for b in range(B)]
        n_path = torch.tensor([len(p) for p, _ in paths], dtype=torch.int32, device="cuda")
        path = torch.zeros((B, T), dtype=torch.int32, device="cuda")
        for b, (p, _) in enumerate(paths):
            path[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
        accepted_in_all += int(n_path.sum()) - B
        tree_cache.commit(path, n_path)
        tree_cache.truncate()
        taken = torch.gather(ids, 1, path.long())             # the same tokens, written one at a time
        for t in range(int(n_path.max())):
            now = (t < n_path).to(torch.int32)
            plain.reserve(now)
            for layer in range(layers):
                x = emb[layer][taken[:, t:t + 1]]
                plain.write(layer, x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], n_new=now)
            plain.commit(torch.zeros((B, 1), dtype=torch.int32, device="cuda"), now)
        for b, (p, best) in enumerate(paths):
            new = [int(i) for i in taken[b, 1:len(p)]] + [best]
            history[b, int(n_tokens[b]):int(n_tokens[b]) + len(new)] = torch.tensor(new, dtype=torch.int32)
            n_tokens[b] += len(new)
        root = torch.tensor([best for _, best in paths], dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        assert torch.equal(tree_cache.length, plain.length) and torch.equal(tree_cache.length, n_tokens - 1)
        for b in range(B):
            at = torch.arange(int(plain.length[b]), device="cuda")
            for name in ("k", "v"):
                rows = [getattr(c, name)[:, c.page_table[b].long()[at // page_size], :, at % page_size] for c in caches]
                assert torch.equal(*rows), (step, b, name)
        assert int((tree_cache.refcount > 0).sum()) == sum(-(-int(l) // page_size) for l in tree_cache.length)
        q = torch.randn((B, 1, Hq, D), generator=gen(step, "cuda"), device="cuda").to(torch.bfloat16)
        none = torch.zeros(B, dtype=torch.int32, device="cuda")
        for c in caches:                                      # one more token each, seen by itself and everything before it
            c.reserve(none + 1)
            c.write(1, q[:, :, :Hkv], q[:, :, Hkv:2 * Hkv])
        assert torch.equal(tree_cache.attention(1, q), plain.attention(1, q))
        assert int(sum(c.status.view(torch.int32).abs().sum() for c in caches)) == 0
    assert accepted_in_all >= 6


def test_forked_sequences_go_their_own_ways():
    """Four samples of one prompt: shared pages until each writes, and each then sees its own tokens only."""
    from paper_2502_13652_amd import PagedCache
    ps, Hkv, D, L = 16, 2, 128, 2
    c = PagedCache(5, L, 40, ps, Hkv, D, 8)
    x = torch.randn((5, 37, 4 * Hkv, D), generator=gen(1, "cuda"), device="cuda").to(torch.bfloat16)
    first = torch.tensor([37, 0, 0, 0, 0], dtype=torch.int32, device="cuda")
    c.reserve(first)
    for layer in range(L):
        c.write(layer, x[:, :, :Hkv], x[:, :, Hkv:2 * Hkv], n_new=first)
    c.commit(torch.arange(37, dtype=torch.int32, device="cuda").repeat(5, 1), first)
    c.fork(torch.zeros(4, dtype=torch.int32, device="cuda"), torch.arange(1, 5, dtype=torch.int32, device="cuda"))
    assert sorted(c.refcount.tolist())[-3:] == [5, 5, 5] and c.length.tolist() == [37] * 5
    one = torch.ones(5, dtype=torch.int32, device="cuda")
    full = c.refcount.clone()
    c.write(0, x[:, :1, :Hkv], x[:, :1, Hkv:2 * Hkv])        # nothing reserved: the shared page is not written
    assert c.status.view(torch.int32).tolist() == [PagedCache.SHARED] * 5 and torch.equal(full, c.refcount)
    c.status.view(torch.int32).zero_()
    for t in range(30):
        c.reserve(one)
        y = torch.randn((5, 1, 4 * Hkv, D), generator=gen(100 + t, "cuda"), device="cuda").to(torch.bfloat16)
        for layer in range(L):
            c.write(layer, y[:, :, :Hkv], y[:, :, Hkv:2 * Hkv])
        c.commit(torch.zeros((5, 1), dtype=torch.int32, device="cuda"), one)
    assert c.length.tolist() == [67] * 5 and int(c.status.view(torch.int32).abs().sum()) == 0
    assert sorted(c.refcount.tolist(), reverse=True)[:3] == [5, 5, 1]       # two whole pages of the prompt are still shared
    assert int((c.refcount > 0).sum()) == 2 + 5 * 3
    q = x[:, :2, :2 * Hkv]
    c.reserve(2 * one)
    c.write(0, x[:, :2, :Hkv], x[:, :2, Hkv:2 * Hkv])
    want, _, tol, _ = attention_reference(c, 0, q, [2] * 5, None, D ** -0.5)
    assert bool(((c.attention(0, q).double() - want).abs() <= tol).all())
    for layer in range(L):                                    # the prompt is what it was, for all of them
        for b in range(5):
            at = torch.arange(37, device="cuda")
            k = c.k[layer, c.page_table[b].long()[at // ps], :, at % ps]
            assert torch.equal(k, x[0, :, :Hkv])


def test_the_example_of_the_readme():
    """The README's step, line for line, on the tree of a draft phase."""
    from test_serving_host import readme_blocks
    block = [b for b in readme_blocks() if "PagedCache" in b]
    assert len(block) == 1
    cfg = dict(idx=93, B=3, V=1009, dtype="bf16", D=3, F=6, K=4, h=6, beta=0.0, N=15, zipf_s=1.2, sigma=(0.5, 1.5), spike_frac=0.0, desc="the readme")
    B, V, N, F, layers = cfg["B"], cfg["V"], cfg["N"], cfg["F"], 2
    ctx = make_gpu(cfg, W.classifier(cfg, 2))
    rows = lambda l: torch.nn.functional.pad(W.logits_layer(cfg, l, device="cuda"), (0, -V % 8))
    ctx.reset()
    for l in range(cfg["D"]):
        ctx.expand_layer(rows(l))
    out = ctx.finalize_tree()
    ctx.reset()
    x = torch.randn((B, 1 + N, 32 + 16, 128), generator=gen(1, "cuda"), device="cuda").to(torch.bfloat16)
    i32 = dict(dtype=torch.int32, device="cuda")
    before = rows(0)
    names = dict(B=B, layers=layers, pages=64, ctx=ctx, ctx_tokens=torch.randint(0, V, (B, 30), generator=gen(2, "cuda"), **i32), n=torch.full((B,), 30, **i32),
                 r=torch.full((B,), 1.3, device="cuda"), grammar_words=torch.full((B, 1, (V + 31) // 32), -2, **i32), logits=before.clone(), out=out,
                 q=x[:, :, :32], k=x[:, :, 32:40], v=x[:, :, 40:], target=torch.randn((B, 1 + N, 1016), generator=gen(3, "cuda"), device="cuda").to(torch.bfloat16)[:, :, :V],
                 path=torch.zeros((B, 1), **i32), n_path=torch.ones(B, **i32))
    exec(block[0], names)
    cache, y, target = names["cache"], names["y"], names["target"]
    assert names["logits"].data_ptr() != before.data_ptr() and bool((names["logits"][:, 0, 0:V:32] == float("-inf")).all()) and not torch.equal(names["logits"], before)
    n_new = names["n_new"].tolist()
    assert cache.length.tolist() == [1] * B and int(cache.status.view(torch.int32).abs().sum()) == 0 and int((cache.refcount > 0).sum()) == B
    # the root's key is still there: its row sees itself alone
    live = names["v"][:, 0].repeat_interleave(4, 1)
    assert torch.equal(y[:, 0], live)
    for b in range(B):
        assert bool(torch.isfinite(y[b, :n_new[b]]).all()) and bool((target[b, :n_new[b], 0:V:32] == float("-inf")).all())
