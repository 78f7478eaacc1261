"""MXFP4: quantisation against a search over all levels, products against 64 bits.

Quantised values have to be equal.  A product sums k terms in fp32 on the
tensor cores, which cut each addition of 64 products at their largest one's
last place or better: with S = sum |a| |b|,
|got - want| <= u(type) |want| + (k / 64 + 4) 2^-23 S.
"""

from __future__ import annotations

import pytest
import torch

import exact_blocks

pytestmark = pytest.mark.gpu

DEV = "cuda"
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def mpm():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2604_05718_gb300 as pkg
    from paper_2604_05718_gb300 import build

    build.build()
    pkg.library()
    return pkg


def tokens(rows, dim, dtype=torch.bfloat16, seed=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, dim, generator=gen, dtype=torch.float64)
    x *= 2.0 ** torch.randint(-6, 7, (rows, 1), generator=gen)
    return x.to(DEV, dtype)


def same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=12345.0), torch.nan_to_num(b, nan=12345.0))


def check_quantized(mpm, x):
    q = mpm.quantize_mxfp4(x)
    want = exact_blocks.mxfp4_values(x)
    assert q.rows == x.shape[0] and q.dim == x.shape[1]
    assert same(exact_blocks.mxfp4_decode(q.codes, q.scales, q.dim), want)
    for dtype in (torch.float32, torch.bfloat16):
        assert same(mpm.dequantize_mxfp4(q, dtype).double().cpu(), want.to(dtype).double())
    # What lies past the rows and the row is zero.
    rows, dim = x.shape
    code = torch.stack([q.codes & 15, q.codes >> 4], 2).reshape(rows, -1)
    assert not code[:, dim:].any()
    t = q.scales.view(q.scales.shape[0], q.scales.shape[1], 32, 4, 4).permute(0, 3, 2, 1, 4)
    t = t.reshape(q.scales.shape[0] * 128, -1)
    assert not t[rows:].any() and not t[:, -(-dim // 32):].any()
    return q


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", [1, 2, 7, 8, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 192, 577, 768, 1030])
@pytest.mark.parametrize("rows", [1, 3, 130])
def test_quantisation(mpm, rows, dim, dtype):
    check_quantized(mpm, tokens(rows, dim, dtype, seed=rows + dim))


def test_many_rows(mpm):
    x = tokens(20011, 96, seed=4)
    q = mpm.quantize_mxfp4(x)
    for lo in (0, 127, 10000, 19900):
        part = mpm.quantize_mxfp4(x[lo:lo + 111])
        assert torch.equal(part.codes, q.codes[lo:lo + 111])
        assert torch.equal(mpm.dequantize_mxfp4(q)[lo:lo + 111], mpm.dequantize_mxfp4(part))


def test_ties_saturation_and_signs(mpm):
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.999, 6.0, 6.5, 7.99, 0.2499, 0.2501, 4.999, 5.001, 0.0]
    row = torch.tensor(ties + [-v for v in ties], dtype=torch.float64)
    x = torch.stack([row * 2.0 ** e for e in (-120, -30, -1, 0, 1, 30, 120)]).to(DEV, torch.float32)
    q = check_quantized(mpm, x)
    v = mpm.dequantize_mxfp4(q, torch.float32)[3].tolist()
    assert v[:7] == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]      # to the even code
    assert v[7:11] == [6.0, 6.0, 6.0, 6.0]                   # 6 is the largest
    assert v[16:23] == [-w for w in v[:7]]


def test_extreme_blocks(mpm):
    big = torch.finfo(torch.float32).max
    tiny = 2.0 ** -149
    x = torch.zeros(8, 64, dtype=torch.float32)
    x[0, 0], x[0, 1] = big, -1.0
    x[1, 5] = tiny                   # below half the smallest step: zero
    x[2, 0], x[2, 1] = 2.0 ** -128, 2.0 ** -129
    x[3, 40] = 2.0 ** -126
    x[4, 3] = -0.0
    x[5] = 1.0
    x[6, :32] = 2.0 ** -127
    check_quantized(mpm, x.to(DEV))
    check_quantized(mpm, x.to(DEV, torch.bfloat16)[1:])


def test_nan_and_infinity_take_their_block(mpm):
    x = tokens(40, 100, torch.float32)
    clean = mpm.dequantize_mxfp4(mpm.quantize_mxfp4(x), torch.float32)
    x[3, 40], x[7, 99], x[9, 0] = float("nan"), float("inf"), float("-inf")
    q = check_quantized(mpm, x)
    got = mpm.dequantize_mxfp4(q, torch.float32)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[3, 32:64] = bad[7, 96:] = bad[9, :32] = True
    assert got[bad].isnan().all() and torch.equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strided_and_unaligned_tokens(mpm, dtype):
    wide = tokens(50, 400, dtype)
    for view in (wide[:, :96], wide[:, 8:200], wide[:, 1:98], wide[:, 3:300]):
        a, b = mpm.quantize_mxfp4(view), mpm.quantize_mxfp4(view.contiguous())
        assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
        out = torch.full((50, view.shape[1] + 5), 9.0, dtype=dtype, device=DEV)
        mpm.dequantize_mxfp4(b, out=out[:, 2:2 + view.shape[1]])
        assert torch.equal(out[:, 2:2 + view.shape[1]], mpm.dequantize_mxfp4(b, dtype))
        assert (out[:, :2] == 9).all() and (out[:, 2 + view.shape[1]:] == 9).all()


def product_bound(a, b, want, k, dtype):
    return ROUND[dtype] * want.abs() + (k / 64 + 4) * 2.0 ** -23 * (a.abs() @ b.abs().t())


def check_product(mpm, m, n, k, dtype=torch.bfloat16, bias=True, seed=0, in_dtype=torch.bfloat16):
    a, b = mpm.quantize_mxfp4(tokens(m, k, in_dtype, seed)), mpm.quantize_mxfp4(tokens(n, k, in_dtype, seed + 1))
    gen = torch.Generator().manual_seed(seed)
    c = torch.randn(n, generator=gen).to(DEV) if bias else None
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    got = mpm.matmul_mxfp4(a, b, bias=c, out_dtype=dtype, device_status=status)
    va, vb = (mpm.dequantize_mxfp4(v, torch.float32).double() for v in (a, b))
    want = va @ vb.t()
    bound = product_bound(va, vb, want, k, dtype)
    if bias:
        want = want + c.double()
        bound = bound + (ROUND[dtype] + 2.0 ** -23) * (want.abs() + c.double().abs())
    assert got.shape == (m, n) and got.dtype == dtype and status.tolist() == [0, 0]
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all()
    assert (off <= bound).all(), f"{(off / bound.clamp(min=1e-300)).max().item():.3g} of the bound"
    return a, b, got


@pytest.mark.parametrize("m", [1, 2, 7, 8, 9, 16, 17, 33, 63, 65, 127, 128, 129, 255, 257, 400])
def test_products_of_few_and_many_rows(mpm, m):
    check_product(mpm, m, 200, 160, seed=m)
    check_product(mpm, m, 96, 1024, torch.float32, seed=m)


@pytest.mark.parametrize("n", [1, 3, 8, 31, 64, 65, 95, 96, 97, 128, 191, 192, 193, 255, 383, 385, 577])
def test_products_of_every_width(mpm, n):
    for m in (5, 300):
        check_product(mpm, m, n, 96, seed=n)
        check_product(mpm, m, n, 96, torch.float32, bias=False, seed=n)


@pytest.mark.parametrize("k", [1, 2, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 192, 255, 256, 257, 320, 384, 511, 513,
                               640, 768, 1281, 4096, 5000])
def test_products_of_every_depth(mpm, k):
    for m in (3, 260):
        check_product(mpm, m, 200, k, seed=k)
        check_product(mpm, m, 200, k, torch.float32, seed=k, in_dtype=torch.float32)


@pytest.mark.parametrize("m,n,k", [(4096, 768, 192), (2500, 2304, 768), (54208, 200, 128), (700, 9000, 320),
                                   (1, 16384, 4096), (64, 5000, 2048), (39000, 769, 65)])
def test_large_products(mpm, m, n, k):
    check_product(mpm, m, n, k, seed=m)


def test_product_into_columns_of_a_wider_matrix(mpm):
    for m, n, off, dtype in ((300, 192, 8, torch.bfloat16), (300, 200, 1, torch.bfloat16), (5, 77, 3, torch.float32),
                             (130, 64, 64, torch.float32), (5, 64, 8, torch.bfloat16)):
        a, b, want = check_product(mpm, m, n, 128, dtype, bias=False)
        wide = torch.full((m, n + 80), 5.0, dtype=dtype, device=DEV)
        mpm.matmul_mxfp4(a, b, out=wide[:, off:off + n])
        assert torch.equal(wide[:, off:off + n], want)
        assert (wide[:, :off] == 5).all() and (wide[:, off + n:] == 5).all()


@pytest.mark.parametrize("m", [9, 300])
def test_nan_rows_stay_in_their_rows(mpm, m):
    x, w = tokens(m, 200), tokens(70, 200, seed=1)
    clean = mpm.matmul_mxfp4(mpm.quantize_mxfp4(x), mpm.quantize_mxfp4(w))
    x[4, 130], w[33, 5] = float("nan"), float("inf")
    got = mpm.matmul_mxfp4(mpm.quantize_mxfp4(x), mpm.quantize_mxfp4(w))
    assert got[4].isnan().all() and got[:, 33].isnan().all()
    keep_m, keep_n = [i for i in range(m) if i != 4], [i for i in range(70) if i != 33]
    assert torch.equal(got[keep_m][:, keep_n], clean[keep_m][:, keep_n])


@pytest.mark.parametrize("m", [6, 290])
def test_scales_past_the_rows_have_no_say(mpm, m):
    a, b = mpm.quantize_mxfp4(tokens(m, 160)), mpm.quantize_mxfp4(tokens(150, 160, seed=1))
    want = mpm.matmul_mxfp4(a, b)
    for q in (a, b):
        t = q.scales.view(q.scales.shape[0], q.scales.shape[1], 32, 4, 4)
        for r in range(q.rows, q.scales.shape[0] * 128):
            t[r // 128, :, r % 32, r % 128 // 32, :] = 255
    assert torch.equal(mpm.matmul_mxfp4(a, b), want)


def test_scales_of_all_sizes_in_one_product(mpm):
    # Blocks of very different scale: 2^-40 .. 2^40.
    gen = torch.Generator().manual_seed(6)
    x = torch.randn(140, 256, generator=gen, dtype=torch.float64)
    x = x * 2.0 ** torch.randint(-40, 41, (140, 8), generator=gen).repeat_interleave(32, 1)
    w = torch.randn(130, 256, generator=gen, dtype=torch.float64)
    a, b = mpm.quantize_mxfp4(x.to(DEV, torch.float32)), mpm.quantize_mxfp4(w.to(DEV, torch.float32))
    va, vb = (mpm.dequantize_mxfp4(v, torch.float32).double() for v in (a, b))
    want = va @ vb.t()
    for rows in (140, 7):
        part = mpm.quantize_mxfp4(x[:rows].to(DEV, torch.float32))
        got = mpm.matmul_mxfp4(part, b, out_dtype=torch.float32)
        assert ((got.double() - want[:rows]).abs() <= product_bound(va, vb, want, 256, torch.float32)[:rows]).all()


def test_no_rows(mpm):
    q = mpm.quantize_mxfp4(torch.empty(0, 64, dtype=torch.bfloat16, device=DEV))
    assert q.rows == 0 and mpm.dequantize_mxfp4(q).shape == (0, 64)
    assert mpm.matmul_mxfp4(q, mpm.quantize_mxfp4(tokens(8, 64))).shape == (0, 8)


def test_same_bits_every_time_and_on_another_stream(mpm):
    x, w = tokens(1000, 768), mpm.quantize_mxfp4(tokens(400, 768, seed=1))
    for rows in (1000, 3):
        want = mpm.matmul_mxfp4(mpm.quantize_mxfp4(x[:rows]), w)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            z = x[:rows] * 0
            for _ in range(20):
                z = z + 0
            got = mpm.matmul_mxfp4(mpm.quantize_mxfp4(z + x[:rows]), w)
        s.synchronize()
        assert torch.equal(got, want)
        for _ in range(5):
            assert torch.equal(mpm.matmul_mxfp4(mpm.quantize_mxfp4(x[:rows]), w), want)


def test_refusals(mpm):
    a, b = mpm.quantize_mxfp4(tokens(8, 64)), mpm.quantize_mxfp4(tokens(16, 64))
    with pytest.raises(ValueError):
        mpm.quantize_mxfp4(torch.zeros(4, 4))
    with pytest.raises(TypeError):
        mpm.quantize_mxfp4(torch.zeros(4, 4, dtype=torch.float16, device=DEV))
    with pytest.raises(ValueError):
        mpm.quantize_mxfp4(tokens(8, 64).t())
    with pytest.raises(ValueError):
        mpm.quantize_mxfp4(tokens(8, 64), out=mpm.quantize_mxfp4(tokens(9, 64)))
    with pytest.raises(ValueError):
        mpm.matmul_mxfp4(a, mpm.quantize_mxfp4(tokens(16, 65)))
    with pytest.raises(ValueError):
        mpm.matmul_mxfp4(a, mpm.MXFP4(b.codes, b.scales, 65))
    with pytest.raises(ValueError):
        mpm.matmul_mxfp4(a, b, bias=torch.zeros(8, device=DEV))
    with pytest.raises(ValueError):
        mpm.matmul_mxfp4(a, b, out=torch.empty(16, 8, device=DEV).t())
    with pytest.raises(TypeError):
        mpm.matmul_mxfp4(a, b, out_dtype=torch.float16)
    with pytest.raises(mpm.MPMError) as e:
        mpm.matmul_mxfp4(a, b, out=b.codes.view(torch.bfloat16)[:8, :16])   # output over an operand
    assert e.value.code == 8
    with pytest.raises(mpm.MPMError) as e:
        mpm.quantize_mxfp4(torch.empty(0, (1 << 20) + 1, device=DEV))
    assert e.value.code == 2


@pytest.mark.parametrize("m,n,k", [(5000, 4096, 2048), (19500, 257, 2049), (4900, 1027, 4100), (2560, 2048, 5120)])
def test_wide_tiles_of_many_features(mpm, m, n, k):
    check_product(mpm, m, n, k, seed=m)
    check_product(mpm, m, n, k, torch.float32, bias=False, seed=m)


@pytest.mark.parametrize("m,n", [(6000, 129), (6000, 200), (5900, 257), (6144, 383), (6000, 384),      # 128 columns
                                 (19500, 1), (19500, 65), (19456, 191), (19500, 193), (19500, 385),    # 192 columns
                                 (100, 16000), (250, 18001)])                                          # 256 columns
@pytest.mark.parametrize("k", [31, 256, 300, 1280, 1400])
def test_every_tile_width(mpm, m, n, k):
    check_product(mpm, m, n, k, seed=n)
    if k == 300:
        check_product(mpm, m, n, k, torch.float32, seed=n, in_dtype=torch.float32)
