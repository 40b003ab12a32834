"""prompt_attention against its formula in 64 bits: lengths, heads, widths, strides, values that are not finite, scores of any size, starts that make no sense."""
import pytest
import torch

from _layer import prompt_reference
from _serving import gen

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def starts_of(lens, first=0):
    at = [first]
    for n in lens:
        at.append(at[-1] + n)
    return at


def inputs(rows, Hq, Hkv, D, dtype, seed, size=1.0):
    fused = torch.randn((rows, Hq + 2 * Hkv, D), generator=gen(seed, "cuda"), device="cuda")
    fused[:, :Hq] *= size
    fused = fused.to(dtype)
    return fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]


def compare(q, k, v, at, out, lse=None, scale=None, before=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    want, want_lse, tol, tol_lse = prompt_reference(q, k, v, at, scale)
    live = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    for a, z in zip(at, at[1:]):
        if 0 <= a < z <= q.shape[0]:
            live[a:z] = True
    x, y = out[live].double(), want[live]
    same = (x == y) | (x.isnan() & y.isnan()) | ((x - y).abs() <= tol[live])
    assert bool(same.all()), (int((~same).sum()), torch.nonzero(~same)[:5].tolist(), x[~same][:5].tolist(), y[~same][:5].tolist())
    if lse is not None:
        assert bool(((lse[live].double() - want_lse[live]).abs() <= tol_lse[live]).all())
    if before is not None:
        assert torch.equal(out[~live].view(torch.int16), before[~live].view(torch.int16))


# few heads: workgroups whose wavefronts divide the keys (widths 64 and 128); more: such as share them, of width 128 by two and, of most, by three a CU
@pytest.mark.parametrize("D,Hq,Hkv,dtype", [(64, 4, 2, BF), (64, 5, 1, HF), (128, 2, 2, BF), (128, 8, 2, HF), (256, 3, 1, BF), (256, 4, 4, HF), (64, 80, 40, BF), (128, 48, 24, HF), (128, 27, 27, BF), (128, 270, 90, BF)])
@pytest.mark.parametrize("lens", [[1], [2], [31], [33], [64], [127], [128], [129], [257], [300], [1000], [1, 2, 3], [0, 5, 0, 0, 64, 1, 33, 0], [200, 17, 129, 1, 512], [5] * 30])
def test_prompts(D, Hq, Hkv, dtype, lens):
    from paper_2502_13652_amd import prompt_attention
    pad = len(lens) % 3
    at = starts_of(lens, first=len(lens) % 2)
    rows = at[-1] + pad
    q, k, v = inputs(rows, Hq, Hkv, D, dtype, sum(lens) + D)
    out = torch.full((rows, Hq, D), 7.0, dtype=dtype, device="cuda")
    before = out.clone()
    lse = torch.full((rows, Hq), 7.0, device="cuda")
    starts = torch.tensor(at, dtype=torch.int32, device="cuda")
    assert prompt_attention(q, k, v, starts, out=out, lse=lse) is out
    compare(q, k, v, at, out, lse, before=before)
    alone = prompt_attention(q.contiguous(), k.contiguous(), v.contiguous(), starts)              # without lse, other strides: the same numbers
    live = slice(at[0], at[-1])
    assert torch.equal(alone[live], out[live])
    assert bool((lse[:at[0]] == 7.0).all()) and bool((lse[at[-1]:] == 7.0).all())


# width 256 with rows enough for each sequence: pairs of wavefronts that share a tile's weights
@pytest.mark.parametrize("Hq,Hkv,dtype", [(8, 1, BF), (3, 1, HF), (4, 4, BF), (64, 2, HF), (65, 1, BF)])
@pytest.mark.parametrize("lens", [[1], [31, 32, 33], [63, 64, 65], [15, 16, 17, 128, 129], [1000], [257, 0, 1, 700, 0], [450, 400, 1, 2, 3, 900]])
def test_pairs(Hq, Hkv, dtype, lens):
    from paper_2502_13652_amd import prompt_attention
    at = starts_of(lens, first=len(lens) % 2)
    rows = max(at[-1] + 2, 400 * len(lens))
    q, k, v = inputs(rows, Hq, Hkv, 256, dtype, sum(lens) + Hq)
    out, lse = torch.full((rows, Hq, 256), 7.0, dtype=dtype, device="cuda"), torch.full((rows, Hq), 7.0, device="cuda")
    before = out.clone()
    starts = torch.tensor(at, dtype=torch.int32, device="cuda")
    prompt_attention(q, k, v, starts, out=out, lse=lse)
    compare(q, k, v, at, out, lse, before=before)
    assert bool((lse[:at[0]] == 7.0).all()) and bool((lse[at[-1]:] == 7.0).all())
    again = prompt_attention(q.contiguous(), k.contiguous(), v.contiguous(), starts, out=before)
    assert again is before and torch.equal(before, out)


def test_pairs_where_the_largest_scores_come_late():
    """References move in each tile, of some rows and for one of a pair's wavefronts at a time; rows of the last tile, of which the array ends within."""
    from paper_2502_13652_amd import prompt_attention
    q, k, v = (x.clone() for x in inputs(777, 4, 1, 256, BF, 17))
    step = torch.arange(777, device="cuda")
    k *= (1 + step // 32 * 2.0).to(BF)[:, None, None]
    k[step % 96 == 5] *= 3
    lse = torch.zeros((777, 4), device="cuda")
    out = prompt_attention(q, k, v, torch.tensor([0, 777], dtype=torch.int32, device="cuda"), lse=lse)
    compare(q, k, v, [0, 777], out, lse)


@pytest.mark.parametrize("Hq,Hkv,D", [(40, 1, 64), (129, 1, 64), (33, 11, 128), (200, 1, 128), (7, 7, 256)])
def test_groups_that_do_not_fill_a_tile_evenly(Hq, Hkv, D):
    from paper_2502_13652_amd import prompt_attention
    at = starts_of([1, 70, 5, 33])
    q, k, v = inputs(at[-1], Hq, Hkv, D, BF, Hq)
    lse = torch.zeros((at[-1], Hq), device="cuda")
    out = prompt_attention(q, k, v, torch.tensor(at, dtype=torch.int32, device="cuda"), lse=lse)
    compare(q, k, v, at, out, lse)


@pytest.mark.parametrize("n,longest", [(65, 40), (130, 300), (700, 9), (4096, 3)])
def test_many_sequences(n, longest):
    from paper_2502_13652_amd import prompt_attention
    lens = torch.randint(0, longest + 1, (n,), generator=gen(n)).tolist()
    at = starts_of(lens)
    q, k, v = inputs(at[-1] + 3, 2, 1, 64, BF, n)
    out = torch.zeros((at[-1] + 3, 2, 64), dtype=BF, device="cuda")
    prompt_attention(q, k, v, torch.tensor(at, dtype=torch.int32, device="cuda"), out=out)
    compare(q, k, v, at, out, before=torch.zeros_like(out))


@pytest.mark.parametrize("dtype,D,Hq,Hkv", [(BF, 128, 2, 1), (HF, 64, 2, 1), (BF, 256, 2, 1), (BF, 128, 26, 26), (HF, 64, 45, 45), (HF, 128, 260, 260), (BF, 256, 8, 2), (HF, 256, 8, 2)])
@pytest.mark.parametrize("size,scale", [(30.0, None), (300.0, None), (1.0, 0.0), (1.0, 3.0), (2000.0, 1.0)])
def test_sharp_and_flat_rows(dtype, D, Hq, Hkv, size, scale):
    """Scores of some thousands and more: a row is then the value of its largest score."""
    from paper_2502_13652_amd import prompt_attention
    at = starts_of([150, 40])
    rows = 900 if (Hq, D) == (8, 256) else 190               # (pairs)
    q, k, v = inputs(rows, Hq, Hkv, D, dtype, 11, size)
    lse = torch.zeros((rows, Hq), device="cuda")
    out = prompt_attention(q, k, v, torch.tensor(at, dtype=torch.int32, device="cuda"), scale=scale, lse=lse)
    compare(q, k, v, at, out, lse, scale=scale)


@pytest.mark.parametrize("H", [2, 120])
def test_scores_past_what_exponents_hold(H):
    from paper_2502_13652_amd import prompt_attention
    q, k, v = inputs(200, H, 1, 64, BF, 12)
    q, k = (q.float() * 3e6).to(BF), (k.float() * 3e6).to(BF)                  # scores of 1e14, whole steps apart by millions
    out = prompt_attention(q, k, v, torch.tensor([0, 200], dtype=torch.int32, device="cuda"))
    x = torch.matmul(q.transpose(0, 1).double(), k[:, 0].double().T.contiguous())
    x.masked_fill_(torch.ones((200, 200), dtype=torch.bool, device="cuda").triu(1), float("-inf"))
    first, second = x.topk(2, -1).values.unbind(-1)
    # apart by more than fp32 sums of 64 products, rounded once more by the scale, make of the two
    size = torch.matmul(q.transpose(0, 1).double().abs(), k[:, 0].double().abs().T.contiguous()).amax(-1)
    clear = (first - second > 2 * 68 * 2.0 ** -24 * size) & (second > float("-inf"))
    assert int(clear.sum()) > 150 * H
    want = v[:, 0][x.argmax(-1)]
    assert torch.equal(out.transpose(0, 1)[clear], want[clear])


@pytest.mark.parametrize("D,dtype,Hq,Hkv", [(64, BF, 2, 1), (128, HF, 2, 1), (256, BF, 2, 1), (64, BF, 50, 50), (128, HF, 30, 30), (128, BF, 200, 200), (256, BF, 8, 2), (256, HF, 8, 2)])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_values_that_are_not_finite_count_for_the_rows_that_see_them(D, dtype, Hq, Hkv, value):
    from paper_2502_13652_amd import prompt_attention
    lens = [140, 200]
    at = starts_of(lens, 2)
    rows = 900 if (Hq, D) == (8, 256) else at[-1] + 4        # (pairs)
    q, k, v = (x.clone() for x in inputs(rows, Hq, Hkv, D, dtype, 13))
    starts = torch.tensor(at, dtype=torch.int32, device="cuda")
    clean = prompt_attention(q, k, v, starts)
    last = at[-1] - 1
    for x in (q, k, v):                                      # rows of no sequence
        x[:2], x[at[-1]:] = value, value
    v[2 + 135, :, 5] = value                                 # late tokens of the first and of the second: not seen by those ahead, nor by the other sequence
    v[last, :, 3], v[last - 40, :, D - 1] = value, -value
    k[last] = value
    got = prompt_attention(q, k, v, starts)
    untouched = torch.ones((rows, Hq, D), dtype=torch.bool, device="cuda")
    untouched[:2], untouched[at[-1]:] = False, False
    untouched[2 + 135:142, :, 5] = False
    untouched[last] = False
    untouched[last - 40:, :, D - 1] = False
    assert torch.equal(got[untouched], clean[untouched])
    assert not bool(got[2 + 135:142, :, 5].isfinite().any()) and not bool(got[last - 40:last, :, D - 1].isfinite().any())
    assert bool(got[last].isnan().all())


def test_starts_that_make_no_sense_are_left_out():
    from paper_2502_13652_amd import prompt_attention
    q, k, v = inputs(100, 2, 1, 64, BF, 14)
    for at, whole in (([-5, 20, 60, 60, 101], [(20, 60)]), ([50, 20, 90, 10], [(20, 90)]), ([100, 100], []), ([-2 ** 31, 2 ** 31 - 1, 0, 40], [(0, 40)]), ([2 ** 31 - 1, -2 ** 31], [])):
        out = torch.full((100, 2, 64), 3.0, dtype=BF, device="cuda")
        prompt_attention(q, k, v, torch.tensor(at, dtype=torch.int32, device="cuda"), out=out)
        compare(q, k, v, at, out, before=torch.full_like(out, 3.0))


def test_empty_refused_streams_and_graphs():
    from paper_2502_13652_amd import prompt_attention
    q, k, v = inputs(300, 4, 2, 64, BF, 15)
    starts = torch.tensor([0, 100, 300], dtype=torch.int32, device="cuda")
    assert prompt_attention(q[:0], k[:0], v[:0], starts).shape == (0, 4, 64)
    out = torch.ones((300, 4, 64), dtype=BF, device="cuda")
    assert bool((prompt_attention(q, k, v, starts[:1], out=out) == 1).all())
    for args in ((q, k[:200], v, starts), (q, k, v[:, :1], starts), (q.float(), k.float(), v.float(), starts), (q, k.half(), v, starts), (q, k, v, starts.long()),
                 (q, k, v, starts.cpu()), (q.transpose(0, 1), k, v, starts), (q[0], k, v, starts)):
        with pytest.raises(ValueError):
            prompt_attention(*args)
    with pytest.raises(Exception, match="invalid"):
        prompt_attention(q[:, :3], k, v, starts)
    with pytest.raises(Exception, match="unsupported"):
        prompt_attention(q[:, :, :32].contiguous(), k[:, :, :32].contiguous(), v[:, :, :32].contiguous(), starts)
    with pytest.raises(Exception, match="invalid"):
        prompt_attention(q, k, v, starts, scale=-1.0)
    contiguous = q.contiguous()
    with pytest.raises(Exception, match="invalid"):
        prompt_attention(contiguous, k, v, starts, out=contiguous)
    with pytest.raises(ValueError):
        prompt_attention(q, k, v, starts, lse=torch.zeros((300, 3), device="cuda"))
    want = prompt_attention(q, k, v, starts)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = prompt_attention(q, k, v, starts, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    out, lse = torch.zeros((300, 4, 64), dtype=BF, device="cuda"), torch.zeros((300, 4), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        prompt_attention(q, k, v, starts, out=out, lse=lse)
    for at in ([0, 100, 300], [7, 8, 290], [0, 300, 300]):   # lengths stay on the device
        starts.copy_(torch.tensor(at, dtype=torch.int32))
        out.fill_(2.0)
        graph.replay()
        torch.cuda.synchronize()
        compare(q, k, v, at, out, lse, before=torch.full_like(out, 2.0))


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 128), (16, 8, 128), (48, 24, 128), (8, 2, 256)])
def test_the_bits_are_the_same_each_time(Hq, Hkv, D):
    from paper_2502_13652_amd import prompt_attention
    q, k, v = inputs(3000, Hq, Hkv, D, BF, 16)
    starts = torch.tensor([0, 1700, 1701, 3000], dtype=torch.int32, device="cuda")
    first = prompt_attention(q, k, v, starts)
    for _ in range(5):
        assert torch.equal(prompt_attention(q, k, v, starts), first)


@pytest.mark.parametrize("D,Hq,Hkv,rows", [(64, 2, 1, 150), (128, 2, 2, 150), (128, 300, 75, 130), (256, 2, 1, 150), (256, 2, 1, 420)])
def test_rows_whose_offsets_pass_32_bits(D, Hq, Hkv, rows):
    from paper_2502_13652_amd import prompt_attention
    q, k, v = inputs(rows, Hq, Hkv, D, BF, 18)
    starts = torch.tensor([0, rows - 30, rows], dtype=torch.int32, device="cuda") if rows < 400 else torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    step = 1 << 24
    apart = torch.empty((rows - 1) * step + 3 * Hq * D + Hkv * D, dtype=BF, device="cuda")
    places, far = 0, []
    for x in (q, k, v, q):
        heads = x.shape[1]
        far.append(apart.as_strided((rows, heads, D), (step, D, 1), places))
        places += heads * D
    for to, x in zip(far, (q, k, v)):
        to.copy_(x)
    prompt_attention(far[0], far[1], far[2], starts, out=far[3])
    assert torch.equal(far[3], prompt_attention(q, k, v, starts))
