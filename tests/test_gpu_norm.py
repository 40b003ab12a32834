"""rms_norm against its formula in 64 bits: types, widths, strides, rows of any size, 8-bit outputs and their scales."""
import pytest
import torch

from _layer import F32_STEP, blocks_of, half_step, least, norm_reference, norm_tolerance
from _serving import gen

pytestmark = pytest.mark.gpu
BF, HF, F32, E4 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
EPS = 1e-5


def inputs(rows, width, dtype, residual, weight, seed):
    g = gen(seed, "cuda")
    x = torch.randn((rows, width), generator=g, device="cuda").to(dtype)
    w = (1 + 0.3 * torch.randn(width, generator=g, device="cuda")).to(weight)
    r = None if residual is None else (3 * torch.randn((rows, width), generator=g, device="cuda")).to(residual)
    return x, w, r


def check(x, w, r, out, scales, residual_out, block=None, eps=EPS):
    h, y = norm_reference(x, w, eps, r)
    if r is not None:
        assert bool(((residual_out.double() - h).abs() <= h.abs() * (half_step(residual_out.dtype) + F32_STEP) * (1 + 2.0 ** -8) + least(residual_out.dtype)).all())
    if block is None:
        assert bool(((out.double() - y).abs() <= norm_tolerance(y, out.dtype)).all())
        return
    top, each = blocks_of(y, block)
    want = torch.where(top > 0, top / 448, 1.0)
    assert scales.shape == want.shape
    assert bool(((scales.double() - want).abs() <= want * 7 * F32_STEP).all())                  # y's, and the division's
    t = y / torch.where(each > 0, each / 448, 1.0)
    got = out.float().double()
    assert bool((got.abs() <= 448).all())
    # a rounding to e4m3 of what is off by y's, the scale's, its reciprocal's and the product's
    assert bool(((got - t).abs() <= torch.maximum(t.abs() * half_step(E4), torch.full_like(t, 2.0 ** -10)) * (1 + 2.0 ** -8) + t.abs() * 20 * F32_STEP).all())


@pytest.mark.parametrize("dtype,residual,weight", [(BF, None, BF), (BF, BF, BF), (BF, F32, F32), (HF, HF, F32), (HF, F32, HF), (F32, F32, F32), (F32, None, F32)])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 7), (5, 64), (2, 505), (9, 512), (4, 1024), (7, 1111), (3, 2048), (2, 2056), (5, 4096), (2, 5000), (3, 8192), (2, 16384), (1, 30001), (2, 65536)])
def test_norm(dtype, residual, weight, rows, width):
    from paper_2502_13652_amd import rms_norm
    x, w, r = inputs(rows, width, dtype, residual, weight, rows * 7 + width)
    before = x.clone()
    to = None if r is None else torch.full_like(r, 9.0)
    kept = None if r is None else r.clone()
    out = rms_norm(x, w, EPS, residual=r, residual_out=to)
    check(x, w, r, out, None, to)
    assert torch.equal(x, before) and (r is None or torch.equal(r, kept))
    if r is not None:                                       # in place, and into x
        again = rms_norm(x, w, EPS, residual=r, out=x)
        assert again is x and torch.equal(x, out) and torch.equal(r, to)


@pytest.mark.parametrize("dtype,residual", [(BF, BF), (HF, None), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("rows,width,block", [(1, 1, 1), (3, 40, 40), (2, 40, 32), (5, 200, 64), (4, 513, 128), (3, 1000, 1000), (66, 1024, 128), (3, 2048, 2048), (2, 4096, 32),
                                              (5, 4096, 4096), (2, 8192, 128), (3, 16000, 64), (2, 30008, 30008), (1, 65535, 128)])
def test_eight_bits(dtype, residual, rows, width, block):
    from paper_2502_13652_amd import rms_norm
    x, w, r = inputs(rows, width, dtype, residual, dtype, rows + width + block)
    x[0, :width // 2] = 0.0
    if r is not None:
        r[0, :width // 2] = 0.0                              # a block of zeros
    to = None if r is None else torch.empty_like(r)
    out, scales = rms_norm(x, w, EPS, residual=r, residual_out=to, scale_block=block)
    assert out.dtype is E4 and scales.dtype is F32
    check(x, w, r, out, scales, to, block)


@pytest.mark.parametrize("width,block", [(1024, 1024), (1024, 32), (4096, 128), (333, 333), (1000, 64)])
def test_eight_bits_between_two_numbers(width, block):
    """Quotients that lie exactly between two numbers of 8 bits go to the even one.  x is 1 and -1 and eps too small to count, so y is the weight with x's sign and nothing is rounded ahead of the
    division; a block's weights are its scale times 448 and times numbers of 5 bits, 24 bits in all."""
    from paper_2502_13652_amd import rms_norm
    g = gen(width + block)
    blocks = -(-width // block)
    scale = torch.randint(2 ** 17 + 1, 2 ** 18, (blocks,), generator=g).double() * 2.0 ** -20               # 18 bits, the last one set
    scale = scale + (scale * 2 ** 20 % 2 == 0) * 2.0 ** -20
    each = scale.repeat_interleave(block)[:width]
    between = (torch.randint(8, 16, (width,), generator=g).double() + 0.5) * 2.0 ** torch.randint(-6, 5, (width,), generator=g).double()       # e4m3 has 8 .. 15 times powers of two
    first = torch.arange(0, width, block)
    between[first] = 448.0
    weight = between * each
    assert torch.equal(weight.float().double(), weight)
    x = torch.where(torch.rand((3, width), generator=g) < 0.5, -1.0, 1.0)
    out, scales = rms_norm(x.cuda(), weight.float().cuda(), 1e-30, scale_block=block)
    assert torch.equal(scales.cpu().double(), scale.expand(3, blocks))
    t = between.clone()
    t[first] = 0.0
    step = 2.0 ** torch.floor(torch.log2(torch.where(t > 0, t, 1.0))) / 8
    want = torch.where(t > 0, torch.round(t / step) * step, 448.0)                               # (torch.round: to even)
    assert torch.equal(out.float().cpu().double(), want * x.double())


def test_strides_and_what_lies_between():
    from paper_2502_13652_amd import rms_norm
    for pad, width in ((8, 256), (5, 256), (16, 250), (1, 1)):
        x, w, r = inputs(6, width, BF, BF, BF, pad)
        wide = [torch.full((6, width + pad), 5.0, dtype=d, device="cuda") for d in (BF, BF, BF, E4)]
        wide_scales = torch.full((6, 4), 5.0, device="cuda")
        xs, rs, outs, eight = (t[:, :width] for t in wide)
        xs.copy_(x), rs.copy_(r)
        rms_norm(xs, w, EPS, residual=rs, out=outs)
        check(x, w, r, outs, None, rs)
        rs.copy_(r)
        n = -(-width // 128)
        rms_norm(xs, w, EPS, residual=rs, out=eight, scale_block=128, scales=wide_scales[:, :n])
        check(x, w, r, eight, wide_scales[:, :n], rs, 128)
        for t in wide:
            assert bool((t[:, width:].float() == 5.0).all())
        assert bool((wide_scales[:, n:] == 5.0).all())
    x, w, r = inputs(12, 96, HF, F32, F32, 3)               # [2][6][96] of a padded batch, and one dimension alone
    out = rms_norm(x.view(2, 6, 96), w, EPS, residual=r.view(2, 6, 96))
    assert out.shape == (2, 6, 96)
    assert torch.equal(rms_norm(x[3], w, EPS), rms_norm(x[3:4], w, EPS)[0])
    off = torch.zeros(12 * 96 + 1, dtype=HF, device="cuda")[1:].view(12, 96)            # not 16-byte aligned
    off.copy_(x)
    assert torch.equal(rms_norm(off, w, EPS), rms_norm(x, w, EPS))


@pytest.mark.parametrize("dtype,residual,weight", [(F32, F32, F32), (BF, F32, F32), (HF, F32, HF), (F32, None, F32)])
@pytest.mark.parametrize("width,stride,shift", [(8, 12, 0), (16, 20, 4), (1024, 1028, 12), (2048, 2052, 4), (8200, 8204, 20)])
def test_32_bit_rows_aligned_to_16_bytes_and_no_more(dtype, residual, weight, width, stride, shift):
    """Such rows are taken by whole pieces; 16-bit ones beside them keep to multiples of 8 elements."""
    from paper_2502_13652_amd import rms_norm

    def place(kind):
        at, step = (shift, stride) if kind is F32 else (shift // 4 * 8, (stride + 7) // 8 * 8)
        return torch.full((at + 5 * step,), 9.0, dtype=kind, device="cuda").as_strided((5, width), (step, 1), at)

    x, w, r = inputs(5, width, dtype, residual, weight, width + shift)
    xs, outs, ws = place(dtype), place(dtype), torch.zeros(width + 4, dtype=weight, device="cuda")[4 if weight is F32 else 0:][:width]
    xs.copy_(x), ws.copy_(w)
    rs, to = (None, None) if r is None else (place(residual), place(residual))
    if r is not None:
        rs.copy_(r)
    assert xs.data_ptr() % 16 == 0 and xs.stride(0) * xs.element_size() % 16 == 0 and (r is None or rs.data_ptr() % 16 == 0 and rs.stride(0) * 4 % 16 == 0)
    rms_norm(xs, ws, EPS, residual=rs, residual_out=to, out=outs)
    check(x, w, r, outs, None, to)
    eight, scales = rms_norm(xs, ws, EPS, residual=rs, residual_out=to, scale_block=32)
    check(x, w, r, eight, scales, to, 32)
    assert torch.equal(xs, x) and (r is None or torch.equal(rs, r))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_of_any_size(dtype):
    """Squares of such numbers pass fp32; the mean does not."""
    from paper_2502_13652_amd import rms_norm
    x, w, _ = inputs(8, 1000, F32, None, F32, 5)
    for size in (1e30, 1e38 / 4, 1e-30, 1e-20, 1.0):
        y = (x * size).to(dtype)
        eps = 1e-42 if size < 1 else EPS                     # (an fp32 number: subnormal)
        eps = float(torch.tensor(eps, dtype=F32))
        check(y, w, None, rms_norm(y, w, eps), None, None, eps=eps)
    zeros = torch.zeros((3, 1000), dtype=dtype, device="cuda")
    assert bool((rms_norm(zeros, w, EPS) == 0).all())
    out, scales = rms_norm(zeros, w, EPS, scale_block=1000)
    assert bool((out.float() == 0).all()) and bool((scales == 1).all())


def test_what_is_not_finite_stays_in_its_row():
    from paper_2502_13652_amd import rms_norm
    x, w, _ = inputs(70, 640, BF, None, BF, 6)
    want = rms_norm(x, w, EPS)
    want8, scales8 = rms_norm(x, w, EPS, scale_block=640)
    bad = x.clone()
    bad[3, 100], bad[68, 5] = float("nan"), float("inf")
    got = rms_norm(bad, w, EPS)
    got8, scales = rms_norm(bad, w, EPS, scale_block=640)
    rest = [i for i in range(70) if i not in (3, 68)]
    assert torch.equal(got[rest], want[rest]) and torch.equal(got8.view(torch.uint8)[rest], want8.view(torch.uint8)[rest]) and torch.equal(scales[rest], scales8[rest])
    assert bool(got[3].isnan().all()) and bool(got[68, 5].isnan()) and bool(got8.float()[3].isnan().all()) and bool(got8.float()[68, 5].isnan())
    weight = w.clone()
    weight[7] = float("nan")                                 # one element a row: no other is touched
    got8, scales = rms_norm(x, weight, EPS, scale_block=32)
    full8, full = rms_norm(x, w, EPS, scale_block=32)
    assert bool(got8.float()[:, 7].isnan().all()) and torch.equal(got8.view(torch.uint8)[:, 32:], full8.view(torch.uint8)[:, 32:]) and bool(scales.isfinite().all())


def test_empty_refused_streams_and_graphs():
    from paper_2502_13652_amd import rms_norm
    x, w, r = inputs(5, 256, BF, BF, BF, 8)
    assert rms_norm(x[:0], w).shape == (0, 256)
    out, scales = rms_norm(x[:0], w, scale_block=32)
    assert out.shape == (0, 256) and scales.shape == (0, 8)
    for kw in (dict(residual=r[:3]), dict(residual=r.half()), dict(residual_out=r), dict(residual=r, residual_out=r.float()), dict(out=x.float()), dict(out=x[:, :128]),
               dict(scale_block=96), dict(scale_block=0), dict(scales=torch.zeros((5, 1), device="cuda")), dict(scale_block=32, scales=torch.zeros((5, 7), device="cuda")),
               dict(scale_block=32, out=x), dict(residual=r.cpu()), dict(residual=r.T.contiguous().T)):
        with pytest.raises(ValueError):
            rms_norm(x, w, EPS, **kw)
    with pytest.raises(ValueError):
        rms_norm(x, w[:128], EPS)
    with pytest.raises(ValueError):
        rms_norm(x.int(), w, EPS)
    with pytest.raises(Exception, match="invalid"):
        rms_norm(x, w, 0.0)
    with pytest.raises(Exception, match="invalid"):
        rms_norm(x, w, EPS, residual=r, out=r)               # one place for two results
    want = rms_norm(x, w, EPS, residual=r.clone())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = rms_norm(x, w, EPS, residual=r, residual_out=torch.empty_like(r), stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    to, out8 = torch.empty_like(r), torch.empty((5, 256), dtype=E4, device="cuda")
    sc = torch.empty((5, 2), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rms_norm(x, w, EPS, residual=r, residual_out=to, out=out8, scale_block=128, scales=sc)
    for seed in range(3):
        x.copy_(torch.randn((5, 256), generator=gen(seed, "cuda"), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        check(x, w, r, out8, sc, to, 128)


@pytest.mark.parametrize("width,shift", [(512, 0), (501, 3)])
def test_rows_whose_offsets_pass_32_bits(width, shift):
    from paper_2502_13652_amd import rms_norm
    x, w, r = inputs(4, width, BF, BF, BF, 21)
    apart = torch.empty(3 * 2 ** 30 + 4096, dtype=BF, device="cuda")
    far = [apart.as_strided((4, width), (2 ** 30, 1), 1024 * i + shift) for i in range(3)]
    far[0].copy_(x)
    far[1].copy_(r)
    rms_norm(far[0], w, EPS, residual=far[1], out=far[2])
    want = rms_norm(x, w, EPS, residual=r)
    assert torch.equal(far[2], want) and torch.equal(far[1], r) and torch.equal(far[0], x)
