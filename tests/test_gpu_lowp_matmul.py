"""Products with a receiver's codes on the GPU against the definition in 64 bits.

The codes are the framework's own casts of FP32 weights, or drawn bytes.
Products are exact; a sum of k of them in FP32 is off by at most k * 2^-24 of
the sum of their magnitudes, and a BF16 result by another 2^-8 of itself.
"""
import numpy as np
import pytest
import torch

from paper_2602_03839_amd import head, pulse

pytestmark = pytest.mark.gpu

MX, FP8 = pulse.MXFP4, pulse.FP8_E4M3
MAGS = [0, 0.5, 1, 1.5, 2, 3, 4, 6]


def values(dtype, codes, scales, n, inv_scale=1.0):
    """The weights' values in 64 bits, from the codes."""
    c = codes.cpu().numpy()
    if dtype == MX:
        nib = np.stack([c & 15, c >> 4], 1).reshape(-1)[:n]
        mag = np.array(MAGS + [-m for m in MAGS], dtype=np.float64)[nib]
        s = scales.cpu().numpy().astype(np.float64)
        step = np.where(s == 255, np.nan, 2.0 ** (s - 127))
        return mag * np.repeat(step, 32)[:n]
    e, m = (c >> 3) & 15, (c & 7).astype(np.float64)
    v = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e.astype(np.float64) - 7))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c > 127, -v, v)[:n] / inv_scale


def weight(dtype, rows, cols, seed, inv_scale=1.0):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(rows * cols, generator=g) * torch.exp2(torch.randint(-6, 7, (rows * cols,), generator=g))
    return pulse.cast_lowp(dtype, w.cuda(), inv_scale)


def check(dtype, rows, cols, tokens, out_dtype=torch.float32, seed=0, inv_scale=1.0, make=None):
    codes, scales = (make or weight)(dtype, rows, cols, seed, inv_scale)
    x = torch.randn(tokens, cols, generator=torch.Generator().manual_seed(seed + 1)).bfloat16()
    lin = head.LowpLinear(dtype, codes, scales, rows, cols, inv_scale)
    y = lin(x.cuda(), out_dtype=out_dtype)
    assert y.shape == (tokens, rows) and y.dtype == out_dtype
    w = values(dtype, codes, scales, rows * cols, inv_scale).reshape(rows, cols)
    xd = x.double().numpy()
    want, size = xd @ w.T, np.abs(xd) @ np.abs(w.T)
    # one more rounding for the division by inv_scale
    bound = (cols + 2) * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(want) if out_dtype == torch.bfloat16 else 0)
    off = np.abs(y.cpu().double().numpy() - want)
    assert (off <= bound).all(), (off - bound).max()


@pytest.mark.parametrize("dtype", [MX, FP8])
@pytest.mark.parametrize("cols", [32, 64, 96, 128, 160, 512, 544, 896, 4864])
@pytest.mark.parametrize("rows", [1, 16, 17, 128, 200])
def test_sizes(dtype, rows, cols):
    check(dtype, rows, cols, 3, seed=rows + cols)


@pytest.mark.parametrize("dtype", [MX, FP8])
@pytest.mark.parametrize("cols", [1, 2, 7, 15, 16, 31, 33, 48, 97, 127, 129, 255, 897, 1030])
def test_rows_that_start_inside_a_block(dtype, cols):
    for rows in (1, 5, 33, 600):
        check(dtype, rows, cols, 2, seed=rows + cols)


@pytest.mark.parametrize("dtype", [MX, FP8])
@pytest.mark.parametrize("tokens", [1, 2, 15, 16, 17, 31, 32, 33, 48, 64, 65, 100, 200])
def test_token_counts(dtype, tokens):
    check(dtype, 80, 384, tokens, seed=tokens)
    check(dtype, 50, 75, tokens, torch.bfloat16, seed=tokens)


@pytest.mark.parametrize("dtype", [MX, FP8])
def test_many_rows(dtype):
    check(dtype, 66000, 128, 5, seed=3)
    check(dtype, 70001, 160, 33, torch.bfloat16, seed=4)


@pytest.mark.parametrize("dtype", [MX, FP8])
@pytest.mark.parametrize("rows,cols", [(4103, 128), (3001, 1152), (2500, 4224)])
@pytest.mark.parametrize("tokens", [17, 32, 33, 47, 64])
def test_more_tiles_than_cus_for_two_tiles_of_tokens(dtype, rows, cols, tokens):
    check(dtype, rows, cols, tokens, seed=tokens)


@pytest.mark.parametrize("dtype", [MX, FP8])
@pytest.mark.parametrize("rows,cols", [(2003, 1152), (2003, 4224), (8300, 640)])
@pytest.mark.parametrize("tokens", [33, 47, 64])
def test_two_groups_of_two_tiles_of_tokens(dtype, rows, cols, tokens):
    check(dtype, rows, cols, tokens, seed=tokens)


@pytest.mark.parametrize("dtype,cols", [(MX, 160), (MX, 224), (FP8, 80), (FP8, 208)])
@pytest.mark.parametrize("rows", [4096, 4097, 5000, 8192, 8193, 9001, 16384, 16385])
def test_tiles_of_a_block(dtype, cols, rows):
    check(dtype, rows, cols, 5, seed=rows)
    check(dtype, rows, cols, 16, torch.bfloat16, seed=rows + 1)


@pytest.mark.parametrize("inv_scale", [1.0, 3.5, 1 / 3, 3584.0])
def test_fp8_scale(inv_scale):
    check(FP8, 48, 256, 4, seed=9, inv_scale=inv_scale)


def test_every_scale_byte_and_code():
    """Each E8M0 scale that leaves the value finite, with all sixteen codes."""
    for lo in range(0, 253, 23):
        scales = torch.arange(lo, min(lo + 23, 253), dtype=torch.uint8)
        n = scales.numel()
        codes = torch.tensor([(2 * i) % 16 | ((2 * i + 1) % 16) << 4 for i in range(16)] * n,
                             dtype=torch.uint8)
        # the tokens pick single values, so nothing cancels or overflows
        x = torch.eye(32).bfloat16()
        y = head.LowpLinear(MX, codes.cuda(), scales.cuda(), n, 32)(x.cuda())
        want = values(MX, codes, scales, 32 * n).reshape(n, 32).T
        assert np.array_equal(y.cpu().double().numpy(), want), lo


def test_every_fp8_code():
    codes = torch.arange(256, dtype=torch.uint8)
    y = head.LowpLinear(FP8, codes.cuda(), None, 16, 16)(torch.eye(16).bfloat16().cuda())
    want = values(FP8, codes, None, 256).reshape(16, 16).T
    # a NaN code makes its whole row NaN, whatever it meets
    nan = np.isnan(want).any(0)
    got = y.cpu().double().numpy()
    assert np.isnan(got[:, nan]).all() and np.array_equal(got[:, ~nan], want[:, ~nan])


@pytest.mark.parametrize("dtype,cols", [(MX, 64), (MX, 75), (FP8, 64), (FP8, 75)])
def test_nan_stays_with_its_row_and_token(dtype, cols):
    rows, tokens = 70, 20
    w = torch.randn(rows * cols, generator=torch.Generator().manual_seed(1))
    w[33 * cols + cols // 2] = float("nan")
    codes, scales = pulse.cast_lowp(dtype, w.cuda())
    x = torch.randn(tokens, cols, generator=torch.Generator().manual_seed(2)).bfloat16()
    x[3, 0], x[18, cols - 1] = float("nan"), float("inf")
    got = head.LowpLinear(dtype, codes, scales, rows, cols)(x.cuda()).cpu()
    v = values(dtype, codes, scales, rows * cols).reshape(rows, cols)
    rows_nan = np.isnan(v).any(1)
    assert rows_nan[33] and rows_nan.sum() <= 2  # a block that spans two rows takes both
    bad = np.zeros((tokens, rows), bool)
    bad[:, rows_nan] = True
    bad[[3, 18]] = True
    assert np.array_equal(~torch.isfinite(got).numpy(), bad)


@pytest.mark.parametrize("cols", [16, 80, 272])
@pytest.mark.parametrize("tokens", [1, 20])
def test_fp8_nan_at_the_end_of_a_row(cols, tokens):
    codes, scales = weight(FP8, 70, cols, 3)
    codes[34 * cols - 1] = 0x7F
    x = torch.randn(tokens, cols, generator=torch.Generator().manual_seed(2)).bfloat16()
    got = head.LowpLinear(FP8, codes, scales, 70, cols)(x.cuda()).cpu()
    assert torch.isnan(got[:, 33]).all() and torch.isnan(got).sum() == tokens


def test_views_and_streams():
    """Tokens and results in wider buffers, codes that start 4 bytes into one,
    and a call on another stream."""
    rows, cols, tokens = 100, 224, 9
    g = torch.Generator().manual_seed(5)
    codes, scales = weight(MX, rows, cols, 6)
    flat = torch.zeros(codes.numel() + 64, dtype=torch.uint8, device="cuda")
    flat[4:4 + codes.numel()] = codes
    x = torch.randn(tokens, 300, generator=g).bfloat16().cuda()
    want = head.LowpLinear(MX, codes, scales, rows, cols)(x[:, :cols].contiguous())
    out = torch.full((tokens, 130), 7.0, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    lin = head.LowpLinear(MX, flat[4:4 + codes.numel()], scales, rows, cols)
    lin(x[:, :cols], out=out[:, :rows], stream=s)
    s.synchronize()
    assert torch.equal(out[:, :rows], want) and (out[:, rows:] == 7).all()
    assert lin(x[:0, :cols]).shape == (0, rows)


def test_offsets_past_32_bits():
    """A weight of more than 2^32 values: its last rows."""
    rows, cols = 2_200_000, 2048
    codes = torch.zeros(rows * cols // 2, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows * cols // 32,), 127, dtype=torch.uint8, device="cuda")
    codes[-cols // 2:] = 0x22  # ones
    scales[-cols // 32:] = 128
    x = torch.ones(1, cols, dtype=torch.bfloat16, device="cuda")
    y = head.LowpLinear(MX, codes, scales, rows, cols)(x)
    assert y[0, -1].item() == 2 * cols and (y[0, :-1] == 0).all()


def values_on_gpu(dtype, codes, scales, n, inv_scale=1.0):
    """``values`` on the GPU, for weights that take numpy seconds (without NaN)."""
    if dtype == FP8:
        c = torch.arange(256, dtype=torch.uint8)
        return torch.from_numpy(values(FP8, c, None, 256)).cuda()[codes[:n].int()] / inv_scale
    mags = torch.tensor(MAGS + [-m for m in MAGS], dtype=torch.float64, device="cuda")
    v = mags[torch.stack((codes & 15, codes >> 4), 1).flatten().int()]
    v = torch.cat([v, v.new_zeros(-v.numel() % 32)]).view(-1, 32) * torch.exp2(scales.double() - 127)[:, None]
    return v.flatten()[:n]


def check_on_gpu(dtype, rows, cols, tokens, out_dtype=torch.float32, seed=0, offset=0):
    """``check`` into an output of NaN; codes `offset` bytes into their buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.empty(rows * cols, device="cuda").normal_(generator=g)
    w *= torch.exp2(torch.randint(-6, 7, (rows * cols,), generator=g, device="cuda"))
    codes, scales = pulse.cast_lowp(dtype, w)
    del w
    flat = torch.zeros(codes.numel() + 16, dtype=torch.uint8, device="cuda")
    flat[offset:offset + codes.numel()] = codes
    x = torch.randn(tokens, cols, generator=g, device="cuda").bfloat16()
    y = torch.full((tokens, rows + 3), float("nan"), dtype=out_dtype, device="cuda")
    head.LowpLinear(dtype, flat[offset:offset + codes.numel()], scales, rows, cols)(x, out=y[:, :rows])
    assert torch.isnan(y[:, rows:]).all()
    step = max(1, (1 << 27) // cols // 32 * 32)  # rows: whole blocks of 32 values
    for r in range(0, rows, step):
        n = min(step, rows - r)
        k = r * cols
        wd = values_on_gpu(dtype, codes[k // 2 if dtype == MX else k:], None if dtype == FP8 else scales[k // 32:], n * cols).view(n, cols)
        want, size = x.double() @ wd.t(), x.double().abs() @ wd.abs().t()
        bound = (cols + 2) * 2.0 ** -24 * size + (2.0 ** -8 * want.abs() if out_dtype == torch.bfloat16 else 0)
        assert ((y[:, r:r + n].double() - want).abs() <= bound).all(), (r, n)


# more values a row than the registers of a block's waves take: the tokens in LDS, or,
# for too many of them, the kernel without slabs
@pytest.mark.parametrize("dtype,cols", [(MX, 6272), (MX, 6656), (MX, 18944), (FP8, 6160), (FP8, 7008), (FP8, 7000), (FP8, 18944)])
@pytest.mark.parametrize("rows", [17, 2003, 4103])
def test_wide_rows(dtype, cols, rows):
    for tokens in (1, 2, 5, 11, 16, 17, 33, 64):
        check_on_gpu(dtype, rows, cols, tokens, torch.bfloat16 if tokens == 11 else torch.float32, seed=rows + tokens)


# a block's runs of two groups of tiles: the waves of a tile in k, and in rows
@pytest.mark.parametrize("dtype,rows,cols", [(MX, 65551, 5120), (MX, 131099, 3584), (MX, 800003, 128), (MX, 70001, 1152),
                                             (FP8, 65551, 5120), (FP8, 800003, 208), (FP8, 70001, 1152)])
@pytest.mark.parametrize("tokens", [1, 5, 17, 33])
def test_long_weights(dtype, rows, cols, tokens):
    check_on_gpu(dtype, rows, cols, tokens, seed=tokens)


# the other kernel for rows that start a unit, with one, two and four tiles a block:
# codes that are not 16-byte aligned, or several tokens of very wide rows
@pytest.mark.parametrize("rows", [17, 2003, 4096, 4100, 8192, 8300, 16384, 17001])
def test_fp8_without_slabs(rows):
    for tokens in (1, 5, 16, 17, 40, 64):
        check_on_gpu(FP8, rows, 208, tokens, seed=rows + tokens, offset=8)
        check_on_gpu(MX, rows, 256, tokens, seed=rows + tokens, offset=4)
    check_on_gpu(FP8, min(rows, 9000), 27648, 16, seed=rows)


@pytest.mark.parametrize("dtype", [MX, FP8])
def test_more_rows_than_one_launch_has_threads(dtype):
    """2^30 rows of one value: with 4 threads a row, 2^32 threads and more.  A product
    of one term is exact."""
    rows = (1 << 30) + 77
    w = torch.empty(rows, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    codes, scales = pulse.cast_lowp(dtype, w)
    del w
    y = torch.full((1, rows), 77.0, device="cuda")
    head.LowpLinear(dtype, codes, scales, rows, 1)(torch.full((1, 1), 1.5, dtype=torch.bfloat16, device="cuda"), out=y)
    mags = torch.tensor(MAGS + [-m for m in MAGS], device="cuda")
    step = 1 << 24
    for k in range(0, rows, step):
        n = min(step, rows - k)
        if dtype == FP8:
            want = codes[k:k + n].view(torch.float8_e4m3fn).float()
        else:
            pair = codes[k // 2:(k + n + 1) // 2]
            want = mags[torch.stack((pair & 15, pair >> 4), 1).flatten().int()].view(-1)[:n]
            want = want * torch.exp2(scales[k // 32:(k + n + 31) // 32].float() - 127).repeat_interleave(32)[:n]
        assert torch.equal(y[0, k:k + n], 1.5 * want), k


@pytest.mark.parametrize("dtype", [MX, FP8])
@pytest.mark.parametrize("rows,cols", [(2, 3), (16, 128)])
def test_most_tokens(dtype, rows, cols):
    """2^20 tokens, for rows that start inside a block and for rows that do not."""
    tokens = 1 << 20
    codes, scales = weight(dtype, rows, cols, 4)
    x = torch.empty(tokens, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    y = torch.full((tokens, rows), float("nan"), device="cuda")
    head.LowpLinear(dtype, codes, scales, rows, cols)(x, out=y)
    w = torch.from_numpy(values(dtype, codes, scales, rows * cols).reshape(rows, cols)).cuda()
    off = (y.double() - x.double() @ w.t()).abs()
    assert (off <= (cols + 2) * 2.0 ** -24 * (x.double().abs() @ w.abs().t())).all()


def test_refusals():
    codes, scales = weight(MX, 16, 64, 1)
    c8, _ = weight(FP8, 16, 64, 1)
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    ok = head.LowpLinear(MX, codes, scales, 16, 64)
    ok(x)
    bad = [lambda: head.LowpLinear(9, codes, scales, 16, 64), lambda: head.LowpLinear(MX, codes, None, 16, 64),
           lambda: head.LowpLinear(MX, codes, scales, 17, 64), lambda: head.LowpLinear(MX, codes, scales[:8].clone(), 16, 64),
           lambda: head.LowpLinear(MX, codes.cpu(), scales, 16, 64), lambda: head.LowpLinear(FP8, codes, None, 16, 64),
           lambda: head.LowpLinear(FP8, c8, None, 16, 64, inv_scale=0.0)(x),
           lambda: head.LowpLinear(FP8, c8, None, 16, 64, inv_scale=float("inf"))(x),
           lambda: head.LowpLinear(FP8, torch.zeros(1028, dtype=torch.uint8, device="cuda")[4:], None, 16, 64)(x),
           lambda: head.LowpLinear(MX, codes, scales, 0, 64)(x),
           lambda: ok(x.float()), lambda: ok(x[:, :32]), lambda: ok(x.cpu()), lambda: ok(x, out_dtype=torch.float16),
           lambda: ok(x, out=torch.zeros(2, 15, device="cuda")), lambda: ok(x, out=torch.zeros(3, 16, device="cuda")),
           lambda: ok(x, out=torch.zeros(16, 2, device="cuda").t())]
    for k, call in enumerate(bad):
        with pytest.raises(pulse.PulseError):
            call()
            pytest.fail(f"call {k} was not refused")
