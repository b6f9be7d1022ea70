"""Operands in 4 bits on the GPU: codes and scales exactly as defined, products against sums in 64 bits of the values that the codes stand for.

A product of two codes and their scales is exact in fp32; the sum of a row's is formed in fp32 by instructions of 64 (128) of the contraction, up to 8 sums joined afterwards: at most C / 64 + 16 additions, each off by at
most a step of fp32 of the sum of magnitudes (the instruction's own additions may cut off instead of rounding); then one rounding to the output's type."""
import math

import pytest
import torch

from paper_2412_16112_amd import clear_block as cb
from tests import more_block_util as ref

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def exact(x):
    """mx_quantize of x [rows, C] against the definition; the values (fp64, CPU)."""
    t = cb.mx_quantize(x)
    cpu = x.cpu()
    values, e = ref.quantized(cpu)
    C = cpu.shape[1]
    assert torch.equal(ref.scale_bytes(t.scales.cpu(), C), e)
    pad = t.scales.cpu().permute(1, 0, 2).reshape(cpu.shape[0], -1)[:, C // 32:]
    assert not pad.any()
    got = ref.decoded(t.codes.cpu(), t.scales.cpu())
    assert torch.equal(got.isnan(), values.isnan()) and bool(((got == values) | values.isnan()).all())
    for dtype in (F32, BF):
        back = cb.mx_dequantize(t, dtype=dtype).cpu()
        want = values.to(dtype)
        assert bool(((back == want) | (want.isnan() & back.isnan())).all())
    return values


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", [(1, 32), (3, 64), (5, 256), (33, 288), (32, 512), (77, 2400), (130, 2432), (1, 8192)], ids=str)
def test_codes_and_scales(shape, dtype):
    g = torch.Generator().manual_seed(shape[1])
    x = torch.randn(*shape, generator=g) * torch.exp(3 * torch.randn(shape[0], shape[1] // 32, 1, generator=g)).expand(-1, -1, 32).reshape(shape)
    exact(x.to(dtype).cuda())


def test_borders_of_rounding():
    # every border between two codes, a step of fp32 below, on and above it, of both signs, at several scales; the block's largest is 4, so that the scale is 1
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.5, 1.0, 2.0, 3.0, 4.0])
    near = torch.cat([borders, torch.nextafter(borders, torch.tensor(0.0)), torch.nextafter(borders, torch.tensor(9.0)), torch.tensor([0.0, 1e-30, 7.9999995])])
    near = torch.cat([near, -near])
    rows = torch.zeros(len(near), 32)
    rows[:, 3] = near
    rows[:, 17] = 4.0
    for scale in (1.0, 2.0 ** -20, 2.0 ** 30, 2.0 ** -120, 2.0 ** 120):
        exact((rows * scale).cuda())
    exact(rows.to(BF).cuda())


def test_smallest_and_largest_and_not_finite():
    tiny, least = 2.0 ** -126, 2.0 ** -149
    firsts = [0.0, -0.0, least, 3 * least, tiny / 2, tiny, 1.75 * tiny, 4 * tiny, 8 * tiny, 3.4e38, -3.4e38, math.inf, -math.inf, math.nan]
    x = torch.zeros(len(firsts), 96)
    for i, v in enumerate(firsts):
        x[i, 40] = v
        x[i, 41] = v / 2 if math.isfinite(v) else 1.0
        x[i, :32] = torch.randn(32)  # (the neighbouring blocks are as they are alone)
        x[i, 64:] = torch.randn(32)
    exact(x.cuda())
    exact(x.to(BF).cuda())


def test_every_code_at_every_scale():
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1)[:, :16 * 16].view(256, 256)  # 512 channels: every pair of codes
    scales = torch.arange(256, dtype=torch.uint8)[None, :, None].expand(2, 256, 8).contiguous()
    want = ref.decoded(codes, scales)
    for dtype in (F32, BF):
        got = cb.mx_dequantize(cb.MX4(codes.cuda(), scales.cuda()), dtype=dtype).cpu()
        w = want.to(dtype)
        assert bool(((got == w) | (got.isnan() & w.isnan())).all())


def operands(M, C, F, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    spread = lambda n: torch.exp(torch.randn(n, C // 32, 1, generator=g)).expand(-1, -1, 32).reshape(n, C)
    x = (torch.randn(M, C, generator=g) * spread(M)).to(dtype).cuda()
    w = cb.mx_quantize((torch.randn(F, C, generator=g) * spread(F) / math.sqrt(C)).cuda())
    return x, w, torch.randn(F, generator=g)


def product(values, w, bias, dtype):
    """(exact product, how far a result may be off)."""
    wv = ref.decoded(w[0].cpu(), w[1].cpu())
    want, size = values @ wv.T, values.abs() @ wv.abs().T
    if bias is not None:
        want, size = want + bias.double(), size + bias.double().abs()
    return want, (wv.shape[1] / 64 + 16) * 2 * ref.FP32 * size + ref.half_step(dtype) * want.abs()


SIZES = [(1, 32, 1), (1, 256, 16), (1, 2432, 300), (2, 96, 33), (3, 8192, 50), (4, 1056, 40), (5, 288, 17), (16, 512, 100), (17, 1056, 40), (33, 768, 65), (64, 2080, 31), (65, 2432, 300), (128, 256, 128), (130, 608, 515), (257, 2400, 777),
         (300, 4096, 256), (100, 8192, 130), (520, 96, 1030), (2100, 512, 3001), (16, 2336, 80), (30, 4640, 70), (1, 4384, 4100), (2, 4384, 4100)]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype,out,with_bias", [(BF, BF, True), (F32, F32, False), (BF, F32, True)])
def test_products(size, dtype, out, with_bias):
    x, w, bias = operands(*size, dtype)
    bias = bias.to(out if size[0] % 2 else F32) if with_bias else None
    values, _ = ref.quantized(x.cpu())
    want, off = product(values, w, bias, out)
    y = cb.mx_linear(x, w, None if bias is None else bias.cuda(), dtype=out)
    assert y.dtype == out
    ref.check(y, want, off, "product")
    assert torch.equal(cb.mx_linear(cb.mx_quantize(x), w, None if bias is None else bias.cuda(), dtype=out), y)
    assert torch.equal(cb.mx_linear(x, w, None if bias is None else bias.cuda(), dtype=out), y)


@pytest.mark.parametrize("size", [(9000, 2432, 4100), (4500, 288, 4100), (70000, 64, 50), (600, 1024, 2048), (1500, 2432, 2432), (1200, 352, 4096), (333, 2432, 7297)], ids=str)
@pytest.mark.parametrize("out,with_bias", [(BF, True), (F32, False), (F32, True)])
def test_many_tiles(size, out, with_bias):
    # every tile shape, whole and ragged, one tile and several a workgroup; the sums in 64 bits on the GPU
    M, C, F = size
    x, w, bias = operands(M, C, F, BF)
    t, bias = cb.mx_quantize(x), bias.cuda() if with_bias else None
    values, wv = (ref.decoded(a.codes.cpu(), a.scales.cpu()).cuda() for a in (t, w))
    y = cb.mx_linear(t, w, bias, dtype=out)
    want, most = torch.matmul(values, wv.t().contiguous()), torch.matmul(values.abs(), wv.abs().t().contiguous())
    if with_bias:
        want, most = want + bias.double(), most + bias.double().abs()
    ref.check(y, want, (C / 64 + 16) * 2 * ref.FP32 * most + ref.half_step(out) * want.abs(), "product")


def test_one_element_at_a_time():
    """Rows of the unit matrix: every output is one weight, wherever it lies in the tile and the contraction."""
    C, F = 672, 300
    x = torch.eye(C, device="cuda")
    w = cb.mx_quantize(torch.randn(F, C, device="cuda"))
    wv = ref.decoded(w.codes.cpu(), w.scales.cpu())
    for rows in (x, x[:64], x[600:]):
        at = 0 if rows.shape[0] in (C, 64) else 600
        assert torch.equal(cb.mx_linear(rows, w, dtype=F32).double().cpu(), wv.T[at:at + rows.shape[0]])


@pytest.mark.parametrize("M", [3, 200])
def test_layouts(M):
    C, F = 544, 210
    x, w, bias = operands(M, C, F, BF)
    y = cb.mx_linear(x, w, bias.cuda())
    # rows of X apart and off alignment, rows of Y apart, a range of W's rows, any leading axes
    wide = torch.empty(M, C + 7, dtype=BF, device="cuda")
    wide[:, 3:C + 3] = x
    into = torch.full((M, F + 5), 7.0, dtype=BF, device="cuda")
    assert cb.mx_linear(wide[:, 3:C + 3], w, bias.cuda(), out=into[:, 1:F + 1]).data_ptr() == into[:, 1:].data_ptr()
    assert torch.equal(into[:, 1:F + 1], y) and bool((into[:, 0] == 7).all()) and bool((into[:, F + 1:] == 7).all())
    assert torch.equal(cb.mx_linear(x, w.rows(17, 150), bias[17:150].cuda()), y[:, 17:150])
    assert torch.equal(cb.mx_linear(x.view(1, M, 1, C), w, bias.cuda()), y.view(1, M, 1, F))
    t = cb.mx_quantize(x)
    assert torch.equal(cb.mx_linear(t.rows(1, 3), w, bias.cuda()), y[1:3])
    assert torch.equal(cb.mx_linear(t.rows(2, 3), w, bias.cuda()), y[2:3])
    # what lies behind the last scale of a row is not looked at
    for scales in (w.scales, t.scales):
        scales.view(-1, scales.shape[1], 8)[-1, :, 1:] = 255
    assert torch.equal(cb.mx_linear(t, w, bias.cuda()), y)


def test_one_part_of_a_wider_projection():
    # [B, N, 3 C], a C of it: rows evenly spaced over both leading axes
    wide = torch.randn(2, 65, 3 * 288, dtype=BF, device="cuda")
    w = cb.mx_quantize(torch.randn(70, 288, device="cuda"))
    for part in wide.split(288, -1):
        assert torch.equal(cb.mx_quantize(part).codes, cb.mx_quantize(part.contiguous()).codes)
        into = torch.full((2, 65, 100), 7.0, dtype=BF, device="cuda")
        cb.mx_linear(part, w, out=into[..., 9:79])
        assert torch.equal(into[..., 9:79], cb.mx_linear(part.contiguous(), w)) and bool((into[..., :9] == 7).all()) and bool((into[..., 79:] == 7).all())


@pytest.mark.parametrize("M", [1, 40, 300])
def test_nan_stays_in_its_row(M):
    x, w, _ = operands(M, 512, 150, BF)
    y = cb.mx_linear(x, w)
    x[M // 2, 100] = math.nan
    z = cb.mx_linear(x, w)
    assert z[M // 2].isnan().all()
    others = [i for i in range(M) if i != M // 2]
    assert torch.equal(z[others], y[others])


def test_no_tokens():
    x, w, bias = operands(4, 64, 10, BF)
    assert cb.mx_linear(x[:0], w, bias.cuda()).shape == (0, 10)
    t = cb.mx_quantize(x[:0])
    assert t.codes.shape == (0, 32) and cb.mx_dequantize(t).shape == (0, 64) and cb.mx_linear(t, w).shape == (0, 10)
