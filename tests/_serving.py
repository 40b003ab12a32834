"""Plain implementations, in 64 bits and python loops, of the cache, its attention and the logits' adjustments, and seeded inputs for them."""
import numpy as np
import torch

NEG = float("-inf")


def half_step(dtype):
    """What a rounding to the type may be off by, relative to the value."""
    return torch.finfo(dtype).eps / 2


def gen(seed, device="cpu"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def random_tree(n, width, g):
    """parent [n] (-1: the root) of a breadth-first tree and its mask [n][n] as finalize_tree writes it."""
    parent = torch.full((n,), -1, dtype=torch.int32)
    mask = torch.zeros((n, n), dtype=torch.uint8)
    for i in range(n):
        lo, hi = max(0, (i // width - 1) * width), i // width * width
        if hi > 0:
            parent[i] = int(torch.randint(lo, hi, (1,), generator=g))
            mask[i] = mask[int(parent[i])]
        mask[i, i] = 1
    return parent, mask


def make_cache(lens, room, ps, kv_heads, D, dtype, seed, layers=1, spare=2, max_pages=None, device="cuda"):
    """A cache whose sequences hold scattered pages for lens + room tokens, K and V Gaussian everywhere."""
    from paper_2502_13652_amd import PagedCache
    g = gen(seed)
    per = [-(-(l + room) // ps) for l in lens]
    pages = sum(per) + spare
    ids = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), max_pages or max(per + [1])), -1, dtype=torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = ids[at:at + n]
        refs[ids[at:at + n].long()] = 1
        at += n
    gd = gen(seed + 1, device)
    shape = (layers, pages, kv_heads, ps, D)
    k = torch.randn(shape, generator=gd, device=device).to(dtype)
    v = torch.randn(shape, generator=gd, device=device).to(dtype)
    return PagedCache.of_tensors(k, v, table.to(device), torch.tensor(lens, dtype=torch.int32, device=device), refs.to(device))


def gathered(cache, b, layer, n):
    """K and V of sequence b's first n tokens, [kv_heads][n][D] float64, and which of them lie on a page that there is."""
    at = torch.arange(n, device=cache.device)
    page = cache.page_table[b].long()[at // cache.page_size] if n else at
    ok = (page >= 0) & (page < cache.pages)
    page = torch.where(ok, page, 0)
    k = cache.k[layer, page, :, at % cache.page_size].transpose(0, 1).double()
    v = cache.v[layer, page, :, at % cache.page_size].transpose(0, 1).double()
    return k, v, ok


def attention_reference(cache, layer, q, n_new, mask, scale, lens=None):
    """out, lse, and the error that 16-bit weights and fp32 sums may make in each of them, all [B][T][H](..) float64; rows behind n_new hold NaN."""
    B, T, H, D = q.shape
    G = H // cache.kv_heads
    N = 0 if mask is None else mask.shape[-1]
    c = T - N
    dev = q.device
    out = torch.full((B, T, H, D), float("nan"), dtype=torch.float64, device=dev)
    lse = torch.full((B, T, H), float("nan"), dtype=torch.float64, device=dev)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    u = half_step(q.dtype)
    lens = cache.length.tolist() if lens is None else lens
    for b in range(B):
        n, l = int(n_new[b]), lens[b]
        if n == 0:
            continue
        k, v, ok = gathered(cache, b, layer, l + n)
        seen = torch.zeros((n, l + n), dtype=torch.bool, device=dev)
        seen[:, :l] = True
        for t in range(n):
            if t < c:
                seen[t, l:l + t + 1] = True
            else:
                seen[t, l:l + min(c, n)] = True
                seen[t, l + c:] = mask[b, t - c, :n - c] != 0
        seen &= ok
        for h in range(H):
            x = q[b, :n, h].double() @ k[h // G].T.contiguous()
            size = q[b, :n, h].double().abs() @ k[h // G].abs().T.contiguous() * scale
            x = torch.where(seen, x * scale, NEG)
            top = x.max(1).values
            ref = torch.where(top == NEG, 0.0, top)
            p = torch.where(seen, torch.exp(x - ref[:, None]), 0.0)
            total = p.sum(1)
            safe = torch.where(total == 0, 1.0, total)
            contributions = torch.where(seen[:, :, None], p[:, :, None] * v[h // G][None], 0.0) if bool((~torch.isfinite(v[h // G])).any()) else None
            o = contributions.sum(1) if contributions is not None else p @ v[h // G]
            a = contributions.abs().sum(1) if contributions is not None else p @ v[h // G].abs()
            out[b, :n, h] = o / safe[:, None]
            lse[b, :n, h] = torch.where(total == 0, NEG, ref + torch.log(safe))
            # scores: D products' sums in fp32, one more rounding by the scale, the exponent's argument and the exponential itself;
            # weights rounded to the type; sums of n terms and their rescalings in fp32
            size = torch.where(seen, size, 0.0).max(1).values
            d = (D + 4) * 2.0 ** -24 * size + 4 * 2.0 ** -23 * (1 + size)
            s = (l + n + 64) * 2.0 ** -23
            tol[b, :n, h] = u * out[b, :n, h].abs() + (a / safe[:, None]) * (u * (1 + u) + 2 * d + s)[:, None]
            tol_lse[b, :n, h] = d + s + lse[b, :n, h].abs().nan_to_num(0, 0, 0) * 2.0 ** -22
    return out, lse, tol, tol_lse


def adjust_reference(row, token_list, n_prompt, path, terms, b, allowed_row):
    """One row in float64 from the definition."""
    V = len(row)
    y = row.astype(np.float64).copy()
    ctx = [t for t in token_list]
    every, said = {}, {}
    for i, t in enumerate(ctx + list(path)):
        if 0 <= t < V:
            every[t] = every.get(t, 0) + 1
            if i >= n_prompt:
                said[t] = said.get(t, 0) + 1
    get = lambda name, default: float(terms[name][b]) if terms.get(name) is not None else default
    rep, freq, pres = get("repetition", 1.0), get("frequency", 0.0), get("presence", 0.0)
    for t in every:
        x = y[t]
        y[t] = x / rep if x > 0 else x * rep
    for t, n in said.items():
        y[t] -= freq * n + pres
    extra = {}
    if terms.get("bias") is not None:
        m = terms["bias"].shape[1] if terms.get("n_bias") is None else min(int(terms["n_bias"][b]), terms["bias"].shape[1])
        for j in range(m):
            t = int(terms["bias_tokens"][b, j])
            if 0 <= t < V:
                extra[t] = extra.get(t, 0.0) + float(terms["bias"][b, j])
    for t, x in extra.items():
        y[t] += x
    if allowed_row is not None:
        bits = np.unpackbits(allowed_row.astype(np.uint32).view(np.uint8), bitorder="little")[:V]
        y[bits == 0] = -np.inf
    touched = np.zeros(V, bool)
    touched[list(every) + list(extra)] = True
    return y, touched
