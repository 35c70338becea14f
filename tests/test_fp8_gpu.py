"""Eight-bit floating point (rwkvq_fp8_quantize, rwkvq_gemm_fp8) against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2505_03803_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def e4m3_table():
    """Values of the 256 codes: sign, four exponent bits (bias 7), three mantissa bits; 0x7F and 0xFF are NaN."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


TABLE = e4m3_table()


def encode_exact(x):
    """Nearest code, ties to the even one, of numbers of magnitude at most 448; NaN and infinities to 0x7F."""
    pos = TABLE[:127]
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = code | np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8)


def quantize_exact(x, block):
    """(codes, scale bytes [.., groups]) by the definition: the smallest e >= -126 with max|x| <= 448 * 2^e."""
    rows, cols = x.shape
    rb, groups = -(-rows // block), -(-cols // 128)
    codes, bytes_ = np.zeros((rows, cols), np.uint8), np.zeros((rb, groups), np.uint8)
    for i in range(rb):
        for g in range(groups):
            part = x[i * block:(i + 1) * block, g * 128:(g + 1) * 128]
            top = np.abs(np.where(np.isfinite(part), part, 0.0)).max()
            e = 0
            if top > 0:
                e = -126
                while top > 448.0 * 2.0 ** e:
                    e += 1
            codes[i * block:(i + 1) * block, g * 128:(g + 1) * 128] = encode_exact(part * 2.0 ** -e)
            bytes_[i, g] = e + 127
    return codes, bytes_


def run_quantize(x, block):
    rows, cols = x.shape
    codes = torch.full((rows, cols), 0xAA, dtype=torch.uint8, device="cuda")
    scale = torch.full((-(-rows // block), B.rwkvq_fp8_scale_pitch(cols)), 0xAA, dtype=torch.uint8, device="cuda")
    B.rwkvq_fp8_quantize(x, codes, scale, block)
    torch.cuda.synchronize()
    return codes.cpu().numpy(), scale.cpu().numpy()[:, :-(-cols // 128)]


def check_quantize(x, block):
    codes, scale = run_quantize(x, block)
    ref_codes, ref_scale = quantize_exact(x.double().cpu().numpy(), block)
    np.testing.assert_array_equal(scale, ref_scale)
    # NaN codes may carry either sign
    same = (codes == ref_codes) | (((codes & 127) == 127) & ((ref_codes & 127) == 127))
    assert same.all(), np.argwhere(~same)[:5]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("shape", [(1, 16), (1, 128), (3, 144), (127, 1040), (129, 272), (130, 2064), (257, 128)])
def test_quantize_equals_the_definition(dtype, block, shape):
    g = torch.Generator().manual_seed(shape[0] * 7 + shape[1])
    x = torch.randn(shape, generator=g) * torch.exp(3.0 * torch.randn((shape[0], 1), generator=g))
    check_quantize(x.to(TYPES[dtype]).cuda(), block)


@pytest.mark.parametrize("block", [1, 128])
def test_quantize_borders(block):
    # powers of two and 448 * 2^e with their neighbours, zeros, the ends of the range, subnormals
    one = np.float32(448.0)
    tops = [0.0, 2.0 ** -149, 2.0 ** -130, 2.0 ** -126, 448.0 * 2.0 ** -126, 1.0, 1.75, float(np.nextafter(np.float32(1.75), np.float32(2))), float(one),
            float(np.nextafter(one, np.float32(1e9))), float(np.nextafter(one, np.float32(0))), 2.0 ** 127, float(np.finfo(np.float32).max)]
    for top in tops:
        x = torch.linspace(-1.0, 1.0, 256).reshape(2, 128).double() * top
        x[0, 5] = top
        x[1, 7] = -top
        check_quantize(x.float().cuda(), block)


@pytest.mark.parametrize("block", [1, 128])
def test_quantize_ties_go_to_even(block):
    # every midpoint of two neighbouring codes, at scale 1 (a 448 in each group)
    mids = (TABLE[:126] + TABLE[1:127]) / 2
    x = torch.zeros((2, 128))
    x[0, :126] = torch.from_numpy(mids).float()
    x[1, :126] = -x[0, :126]
    x[:, 126] = 448.0
    check_quantize(x.cuda(), block)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("block", [1, 128])
def test_quantize_nonfinite(dtype, block):
    x = torch.randn((130, 272), generator=torch.Generator().manual_seed(3))
    x[0, 3], x[1, 100], x[2, 130], x[129, 271] = float("nan"), float("inf"), -float("inf"), float("nan")
    x[5, :128] = float("inf")           # nothing finite in a row's group
    check_quantize(x.to(TYPES[dtype]).cuda(), block)


@pytest.mark.parametrize("block", [1, 128])
def test_quantize_strided_rows(block):
    wide = torch.randn((70, 640), device="cuda").bfloat16()
    x = wide[:, 128:128 + 272]
    assert not x.is_contiguous()
    check_quantize(x, block)


# ---- product ------------------------------------------------------------------------------------------------
def random_codes(gen, rows, cols):
    """Random finite codes."""
    c = gen.integers(0, 256, (rows, cols)).astype(np.uint8)
    return np.where((c & 127) == 127, 0x3A, c).astype(np.uint8)


def random_scales(gen, rows, cols, lo, hi):
    s = np.full((rows, B.rwkvq_fp8_scale_pitch(cols)), 255, np.uint8)         # bytes behind the last group would show as NaN
    s[:, :-(-cols // 128)] = gen.integers(lo, hi, (rows, -(-cols // 128)))
    return s


def values(codes, scale, block):
    rows, cols = codes.shape
    s = 2.0 ** (scale.astype(np.float64) - 127.0)
    s = np.repeat(np.repeat(s, block, 0)[:rows], 128, 1)[:, :cols]
    return TABLE[codes] * s


def product_inputs(seed, M, oc, ic, lo=120, hi=134):
    gen = np.random.default_rng(seed)
    return (random_codes(gen, oc, ic), random_scales(gen, -(-oc // 128), ic, lo, hi), random_codes(gen, M, ic), random_scales(gen, M, ic, lo, hi))


def check_product(y, dtype, wc, ws, xc, xs):
    w, x = values(wc, ws, 128), values(xc, xs, 1)
    ref, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    # a product of two codes is exact in fp32; at most ic / 32 + 32 additions (instructions of 32 columns, and the sum inside one), each off by at
    # most the last place of a running sum that is never more than the sum of the magnitudes; then the output's rounding
    tol = (wc.shape[1] / 32 + 32) * 2.0 ** -23 * mag + HALF_ULP[dtype] * np.abs(ref)
    if dtype == "f16":
        tol = tol + 2.0 ** -25                       # half a step of its subnormals
    got = y.double().cpu().numpy()
    assert np.isfinite(got).all()
    err = np.abs(got - ref)
    assert (err <= tol).all(), f"max err/tol {np.max(err / np.maximum(tol, 1e-300))} at {np.argwhere(err > tol)[:4]}"


SHAPES = [(1, 64, 16), (1, 128, 128), (1, 4096, 512), (2, 128, 1024), (3, 130, 144), (8, 1, 272), (16, 384, 4096), (17, 256, 640), (33, 129, 2064),
          (77, 1000, 1152), (130, 640, 1536), (240, 128, 256), (241, 300, 528), (500, 777, 2064), (1000, 1536, 1024)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_product_against_64_bits(shape, dtype):
    M, oc, ic = shape
    # fp16 outputs stay in range: 448 * 448 * sqrt(ic) * scales
    wc, ws, xc, xs = product_inputs(M + oc + ic, M, oc, ic, *((114, 121) if dtype == "f16" else (120, 134)))
    dev = [torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)]
    y = torch.full((M, oc), float("nan"), dtype=TYPES[dtype], device="cuda")
    B.rwkvq_gemm_fp8(*dev, y)
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0
    check_product(y, dtype, wc, ws, xc, xs)
    again = torch.full_like(y, float("nan"))
    B.rwkvq_gemm_fp8(*dev, again)
    assert torch.equal(y, again)


def test_product_every_scale_has_its_place():
    # one non-zero code in each operand at a time would be slow; instead every (row, group) has its own scale and all codes are 1 (0x38): sums of powers of two
    M, oc, ic = 200, 300, 1664
    gen = np.random.default_rng(5)
    wc, xc = np.full((oc, ic), 0x38, np.uint8), np.full((M, ic), 0x38, np.uint8)
    ws, xs = random_scales(gen, 3, ic, 124, 131), random_scales(gen, M, ic, 124, 131)
    y = torch.empty((M, oc), device="cuda")
    B.rwkvq_gemm_fp8(*[torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)], y)
    ref = values(xc, xs, 1) @ values(wc, ws, 128).T
    assert np.array_equal(y.double().cpu().numpy(), ref)         # exact: small whole multiples of 2^-6


def test_product_scales_at_the_ends_of_their_range():
    wc, ws, xc, xs = product_inputs(9, 5, 130, 256)
    ws[:, :2], xs[:, :2] = [1, 254], [254, 1]        # 2^-126 * 2^127 in either order
    y = torch.empty((5, 130), device="cuda")
    B.rwkvq_gemm_fp8(*[torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)], y)
    check_product(y, "f32", wc, ws, xc, xs)


@pytest.mark.parametrize("M", [2, 40])
def test_product_strided_output_leaves_the_rest(M):
    wc, ws, xc, xs = product_inputs(11, M, 200, 384)
    wide = torch.full((M + 2, 3, 200), 7.0, dtype=torch.bfloat16, device="cuda")
    B.rwkvq_gemm_fp8(*[torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)], wide[:M, 1])
    check_product(wide[:M, 1], "bf16", wc, ws, xc, xs)
    assert (wide[:, 0] == 7).all() and (wide[:, 2] == 7).all() and (wide[M:] == 7).all()


def test_product_nan_stays_in_its_row():
    wc, ws, xc, xs = product_inputs(12, 20, 256, 512)
    xc[3, 100] = 0x7F
    y = torch.empty((20, 256), device="cuda")
    B.rwkvq_gemm_fp8(*[torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)], y)
    nan = torch.isnan(y).cpu().numpy()
    assert nan[3].all() and not np.delete(nan, 3, 0).any()


def test_quantize_then_product():
    # codes and scales as one entry point leaves them and the other reads them
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((50, 1040), generator=g, device="cuda").bfloat16()
    w = (torch.randn((260, 1040), generator=g, device="cuda") * 0.02).half()
    pitch = B.rwkvq_fp8_scale_pitch(1040)
    xc, wc = torch.empty((50, 1040), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((260, 1040), dtype=torch.float8_e4m3fn, device="cuda")
    xs, ws = torch.empty((50, pitch), dtype=torch.uint8, device="cuda"), torch.empty((3, pitch), dtype=torch.uint8, device="cuda")
    y = torch.empty((50, 260), device="cuda")
    B.rwkvq_fp8_quantize(x, xc, xs, 1)
    B.rwkvq_fp8_quantize(w, wc, ws, 128)
    B.rwkvq_gemm_fp8(wc, ws, xc, xs, y)
    check_product(y, "f32", *[t.view(torch.uint8).cpu().numpy() for t in (wc, ws, xc, xs)])


def test_product_captured_and_on_another_stream():
    wc, ws, xc, xs = product_inputs(13, 30, 512, 1024)
    dev = [torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)]
    y = torch.zeros((30, 512), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    B.rwkvq_gemm_fp8(*dev, y, stream=s)
    s.synchronize()
    first = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.rwkvq_gemm_fp8(*dev, y)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, first)
    check_product(y, "f32", wc, ws, xc, xs)


# several tiles a block, the last one ragged either way
@pytest.mark.parametrize("shape", [(224, 9472, 1024), (200, 9500, 528), (1000, 4096, 1040), (700, 5000, 2064), (1500, 2048, 640), (900, 4230, 272)], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_product_of_many_tiles_against_64_bits(shape, dtype):
    M, oc, ic = shape
    wc, ws, xc, xs = product_inputs(M + oc + ic, M, oc, ic)
    dev = [torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)]
    wide = torch.full((M + 1, oc), 7.0, dtype=TYPES[dtype], device="cuda")
    B.rwkvq_gemm_fp8(*dev, wide[:M])
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0
    rows = np.unique(np.concatenate([np.arange(0, M, 37), np.arange(max(0, M - 3), M), np.arange(220, min(M, 228))]))
    check_product(wide[:M][torch.from_numpy(rows).cuda()], dtype, wc, ws, xc[rows], xs[rows])
    assert (wide[M] == 7).all()
    again = torch.empty((M, oc), dtype=TYPES[dtype], device="cuda")
    B.rwkvq_gemm_fp8(*dev, again)
    assert torch.equal(again, wide[:M])


@pytest.mark.parametrize("block", [1, 128])
def test_quantize_more_than_32_bits_of_elements(block):
    rows, cols, last = 66000, 65536, 130
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 2 ** 32
    x[-last:] = torch.randn((last, cols), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    codes = torch.full((rows, cols), 0xAA, dtype=torch.uint8, device="cuda")
    scale = torch.zeros((-(-rows // block), B.rwkvq_fp8_scale_pitch(cols)), dtype=torch.uint8, device="cuda")
    B.rwkvq_fp8_quantize(x, codes, scale, block)
    first = (rows - last) // block * block
    part = slice(0, 1024), slice(cols - 1024, cols)
    for c in part:
        ref_codes, ref_scale = quantize_exact(x[first:, c].double().cpu().numpy(), block)
        assert np.array_equal(codes[first:, c].cpu().numpy(), ref_codes)
        assert np.array_equal(scale[first // block:, c.start // 128:c.stop // 128].cpu().numpy(), ref_scale)
    assert (codes[:first] == 0).all() and (scale[:first // block] == 127).all()


# shapes for which a block of the product takes two tiles of weights at a time: one stage and many, the second tile ragged or not there, rows of Y on and off 16 bytes
TALL = [(1500, 1604, 16), (2100, 2312, 2064), (700, 4176, 144), (2100, 1104, 128), (4000, 1604, 400), (1000, 4130, 2064)]


@pytest.mark.parametrize("shape", TALL, ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_product_of_many_tokens_against_64_bits(shape, dtype):
    M, oc, ic = shape
    wc, ws, xc, xs = product_inputs(M + oc + ic, M, oc, ic, *((114, 121) if dtype == "f16" else (120, 134)))
    dev = [torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)]
    wide = torch.full((M + 1, oc), 7.0, dtype=TYPES[dtype], device="cuda")
    B.rwkvq_gemm_fp8(*dev, wide[:M])
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0
    rows = np.unique(np.concatenate([np.arange(0, M, 61), np.arange(90, 114), np.arange(M - 3, M)]))
    check_product(wide[:M][torch.from_numpy(rows).cuda()], dtype, wc, ws, xc[rows], xs[rows])
    assert (wide[M] == 7).all()
    again = torch.empty((M, oc), dtype=TYPES[dtype], device="cuda")
    B.rwkvq_gemm_fp8(*dev, again)
    assert torch.equal(again, wide[:M])


def test_product_of_many_tokens_every_scale_has_its_place():
    # as above, sums of powers of two: 2100 tokens, nineteen blocks of weights
    M, oc, ic = 2100, 2312, 1664
    gen = np.random.default_rng(6)
    wc, xc = np.full((oc, ic), 0x38, np.uint8), np.full((M, ic), 0x38, np.uint8)
    ws, xs = random_scales(gen, 19, ic, 124, 131), random_scales(gen, M, ic, 124, 131)
    y = torch.empty((M, oc), device="cuda")
    B.rwkvq_gemm_fp8(*[torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)], y)
    ref = 2.0 ** (xs[:, :13].astype(np.float64) - 127.0) @ (128.0 * 2.0 ** (ws[:, :13].astype(np.float64) - 127.0)).T
    assert np.array_equal(y.double().cpu().numpy(), np.repeat(ref, 128, 1)[:, :oc])


# blocks that announce scales for so many pieces of 512 columns only: one token in slices whose copies are all asked for at once, a block that asks for more than it has room for, two tiles
# of weights a block; the tensor core idle, or at work on what came before
GIVEN_UP = [((1, 4096, 4096), 0), ((1, 4096, 4096), 1), ((16, 9472, 4096), 0), ((240, 256, 8192), 1), ((1500, 1604, 2064), 0), ((1500, 1604, 2064), 2)]


@pytest.mark.parametrize("shape,announced", GIVEN_UP, ids=str)
@pytest.mark.parametrize("polls", [200, 3000])
def test_blocks_that_give_up_leave_in_order(shape, announced, polls):
    """Whichever role's wait runs out, a block leaves only when what it has asked for has arrived; the status is reported once, the call after it is right."""
    M, oc, ic = shape
    wc, ws, xc, xs = product_inputs(14, M, oc, ic)
    dev = [torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)]
    want, y = torch.empty((M, oc), device="cuda"), torch.empty((M, oc), device="cuda")
    B.rwkvq_gemm_fp8(*dev, want)
    lost = torch.zeros(4, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0
    B.rwkvq_gemm_fp8_lost(*dev, y, polls, announced, lost)
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 8 and B.rwkvq_device_status() == 0
    gave_up, asked, arrived, done = lost.tolist()
    assert gave_up > 0 and asked >= 2 * gave_up and arrived == gave_up and done == gave_up
    B.rwkvq_gemm_fp8(*dev, y)
    assert torch.equal(y, want) and B.rwkvq_device_status() == 0


# (shape, rows of weights of a tile, slices).  Blocks that go from tile to tile, with fewer columns than they can have under way and with more; the last tile ragged either way
FORMS = [((2048, 4100, 272), 128, 1), ((240, 20000, 272), 128, 1), ((136, 7463, 80), 128, 1), ((1456, 5573, 672), 128, 1), ((3640, 2352, 704), 128, 1),
         ((1, 65536, 128), 256, 1), ((253, 28546, 784), 256, 1), ((1229, 9474, 928), 256, 1), ((580, 15055, 1504), 256, 1)]
# a tile for each cluster of blocks: two, four and eight slices of a tile of few tokens and of more than 32
FORMS += [((1, 5120, 2048), 128, 2), ((7, 7100, 2064), 128, 2), ((488, 648, 1808), 128, 2), ((1008, 411, 1920), 128, 2), ((624, 33, 1664), 128, 4), ((460, 350, 2224), 128, 4),
          ((200, 300, 4112), 128, 8), ((466, 34, 5424), 128, 8)]


@pytest.mark.parametrize("shape,w_rows,slices", FORMS, ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_product_in_every_form_against_64_bits(shape, w_rows, slices, dtype):
    M, oc, ic = shape
    plan = B.rwkvq_gemm_fp8_plan(M, oc, ic)
    assert plan["w_rows"] == w_rows and plan["slices"] == slices, "another form than the test is for"
    assert plan["blocks"] < plan["tiles"] if slices == 1 else plan["blocks"] == plan["tiles"] * slices
    wc, ws, xc, xs = product_inputs(M + oc + ic, M, oc, ic, *((114, 121) if dtype == "f16" else (120, 134)))
    dev = [torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)]
    wide = torch.full((M + 1, oc), 7.0, dtype=TYPES[dtype], device="cuda")
    B.rwkvq_gemm_fp8(*dev, wide[:M])
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0
    rows = np.unique(np.concatenate([np.arange(0, M, 23), np.arange(max(0, M - 3), M)]))
    check_product(wide[:M][torch.from_numpy(rows).cuda()], dtype, wc, ws, xc[rows], xs[rows])
    assert (wide[M] == 7).all()
    # the outputs in rows that are further apart, off 16 bytes: stored number by number, the same bits
    apart = torch.full((M + 1, oc + 3), 7.0, dtype=TYPES[dtype], device="cuda")
    B.rwkvq_gemm_fp8(*dev, apart[:M, :oc])
    assert torch.equal(apart[:M, :oc], wide[:M]) and (apart[M] == 7).all() and (apart[:, oc:] == 7).all()


@pytest.mark.parametrize("M,oc,ic,w_rows,slices", [(795, 7433, 1152, 128, 1), (1229, 9474, 1664, 256, 1), (1008, 411, 1920, 128, 2), (200, 300, 4224, 128, 8)])
def test_product_in_every_form_every_scale_has_its_place(M, oc, ic, w_rows, slices):
    plan = B.rwkvq_gemm_fp8_plan(M, oc, ic)
    assert plan["w_rows"] == w_rows and plan["slices"] == slices and (slices > 1 or plan["blocks"] < plan["tiles"]), plan
    gen = np.random.default_rng(7)
    groups = ic // 128
    wc, xc = np.full((oc, ic), 0x38, np.uint8), np.full((M, ic), 0x38, np.uint8)
    ws, xs = random_scales(gen, -(-oc // 128), ic, 124, 131), random_scales(gen, M, ic, 124, 131)
    y = torch.empty((M, oc), device="cuda")
    B.rwkvq_gemm_fp8(*[torch.from_numpy(a).cuda() for a in (wc, ws, xc, xs)], y)
    ref = 2.0 ** (xs[:, :groups].astype(np.float64) - 127.0) @ (128.0 * 2.0 ** (ws[:, :groups].astype(np.float64) - 127.0)).T
    assert np.array_equal(y.double().cpu().numpy(), np.repeat(ref, 128, 1)[:, :oc])         # exact: sums of few bits


# the same with several tiles a block, the first of them announced whole: the epilogue stores it, or waits for the second, while another role gives up
@pytest.mark.parametrize("shape,announced", [((2048, 4100, 272), 1), ((1456, 5573, 672), 2), ((1456, 5573, 672), 3), ((1, 65536, 128), 1), ((580, 15055, 1504), 3), ((580, 15055, 1504), 4)],
                         ids=str)
@pytest.mark.parametrize("polls", [200, 1000, 5000])
def test_blocks_that_give_up_behind_a_tile_leave_in_order(shape, announced, polls):
    plan = B.rwkvq_gemm_fp8_plan(*shape)
    assert plan["slices"] == 1 and plan["blocks"] < plan["tiles"]
    test_blocks_that_give_up_leave_in_order(shape, announced, polls)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("shape", [(1, 144), (130, 1040), (257, 272)], ids=str)
def test_quantize_strided_rows_of_every_type(dtype, block, shape):
    rows, cols = shape
    wide = torch.full((rows, cols + 48), float("inf"), device="cuda")
    wide[:, 16:16 + cols] = torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda")
    check_quantize(wide.to(TYPES[dtype])[:, 16:16 + cols], block)


def test_scales_as_exponents():
    # scales held as torch's type of eight exponent bits: the same bytes in and out
    e8 = torch.float8_e8m0fnu
    x, w = torch.randn((9, 528), device="cuda"), torch.randn((140, 528), device="cuda") * 0.02
    got = {}
    for kind in (torch.uint8, e8):
        xc, wc = (torch.empty(t.shape, dtype=torch.float8_e4m3fn, device="cuda") for t in (x, w))
        xs, ws = (torch.zeros((rows, B.rwkvq_fp8_scale_pitch(528)), dtype=torch.uint8, device="cuda").view(kind) for rows in (9, 2))
        y = torch.empty((9, 140), device="cuda")
        B.rwkvq_fp8_quantize(x, xc, xs, 1)
        B.rwkvq_fp8_quantize(w, wc, ws, 128)
        B.rwkvq_gemm_fp8(wc, ws, xc, xs, y)
        got[kind] = [t.view(torch.uint8).cpu().numpy() for t in (wc, ws, xc, xs)], y
    for a, b in zip(got[torch.uint8][0], got[e8][0]):
        assert np.array_equal(a, b)
    check_product(got[e8][1], "f32", *got[e8][0])
    assert torch.equal(got[e8][1], got[torch.uint8][1])
    # and what they stand for, as torch reads them
    assert np.array_equal(torch.from_numpy(got[e8][0][3][:, :5].copy()).view(e8).float().numpy(), 2.0 ** (got[e8][0][3][:, :5].astype(np.float32) - 127))
