"""Quantiser by rows and products of 8-bit integers against the float64 oracle (oracle.int8_rows)."""

import numpy as np
import pytest
import torch

from oracle import int8_rows

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - collected on CPU machines, skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2602_18851_amd import Int8Matrix, matmul_int8, quantize_int8  # noqa: E402
from paper_2602_18851_amd.spectral import (SN_BF16, SN_F32, SN_I8, sn_matmul_int8, spectral_matmul_int8_kernel,  # noqa: E402
                                           spectral_quantize_int8)

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": SN_F32, "bf16": SN_BF16}


def rng(*key):
    return np.random.default_rng([20261208, *key])


def wide(r, rows, cols):
    """Normal values whose rows and columns differ in size by a few octaves."""
    return r.standard_normal((rows, cols)) * np.exp2(r.integers(-6, 7, (rows, 1)) + r.integers(-3, 4, (1, cols)))


def on_gpu(x, dtype):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(TORCH[dtype]).cuda()


def host(t):
    return t.detach().cpu().double().numpy()


def check_quantized(m, x):
    codes, scale = int8_rows.quantize(x)
    assert (m.rows, m.cols) == x.shape
    np.testing.assert_array_equal(host(m.scale), scale)
    np.testing.assert_array_equal(host(m.values), codes)
    assert (m.codes[:, x.shape[1]:] == 0).all()  # code rows are filled up with zeros


# ------------------------------------------------------------------ quantiser


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 16), (3, 100), (33, 128), (17, 129), (5, 512), (5, 513), (4, 2048), (4, 2049),
                                       (3, 4097), (2, 8192), (2, 8193), (2, 20000), (300, 8)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantized_rows(rows, cols, dtype):
    x = on_gpu(wide(rng(rows, cols), rows, cols), dtype)
    check_quantized(quantize_int8(x), host(x))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantiser_at_ties_and_extremes(dtype):
    r = rng(1)
    tops = np.exp2(r.uniform(-10, 10, 40))
    x = tops[:, None] * (np.arange(-127, 128)[None, :] / 127)  # codes themselves
    halves = tops[:, None] * ((2 * np.arange(-127, 127) + 1)[None, :] / 254)  # beside every tie
    x = np.concatenate([x, halves, tops[:, None] * np.array([[1.0, 0.5, -0.5, 0.25]])], axis=1)
    extremes = np.zeros((6, x.shape[1]))
    extremes[0, :3] = 3.3e38, -1.65e38, 1e30  # the largest
    extremes[1, :3] = 2.0 ** -126, 2.0 ** -133, -2.0 ** -127  # the scale's lower limit
    extremes[2, :2] = 127 * 2.0 ** -126, 63.5 * 2.0 ** -126
    extremes[3, :3] = 127.0, 0.5, 1.5
    extremes[5, :3] = 2.0 ** -120, 2.0 ** -121, 3 * 2.0 ** -124
    x = on_gpu(np.concatenate([x, extremes]), dtype)
    check_quantized(quantize_int8(x), host(x))


@pytest.mark.parametrize("cols", [40, 300, 1000, 9000])
def test_rows_that_are_not_finite(cols):
    x = on_gpu(wide(rng(2), 5, cols), "f32")
    x[1, 3], x[2, cols - 1], x[4, 0] = float("inf"), float("nan"), -float("inf")
    m = quantize_int8(x)
    for r in (1, 2, 4):
        assert torch.isnan(m.scale[r]) and (m.codes[r] == 0).all()
    check_quantized(quantize_int8(x[[0, 3]]), host(x[[0, 3]]))
    assert torch.equal(m.codes[[0, 3]], quantize_int8(x[[0, 3]]).codes)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,ld", [(0, 208), (1, 208), (8, 203), (3, 331)])
def test_quantiser_reads_strided_rows(dtype, offset, ld):
    room = torch.full((140, ld), float("nan"), dtype=TORCH[dtype], device="cuda")
    x = room[:, offset:offset + 190]
    x.copy_(on_gpu(wide(rng(offset, ld), 140, 190), dtype))
    check_quantized(quantize_int8(x), host(x))


def test_quantiser_leaves_the_rest_of_its_rows():
    x = on_gpu(wide(rng(3), 33, 100), "f32")
    codes = torch.full((34, 160), 0x55, dtype=torch.int8, device="cuda")
    scale = torch.full((40,), -1.0, device="cuda")
    spectral_quantize_int8(x.data_ptr(), 33, 100, 100, SN_F32, codes.data_ptr(), 160, scale.data_ptr(),
                           torch.cuda.current_stream().cuda_stream)
    m = quantize_int8(x)
    assert torch.equal(codes[:33, :112], m.codes) and (codes[:33, 112:] == 0x55).all() and (codes[33] == 0x55).all()
    assert torch.equal(scale[:33], m.scale) and (scale[33:] == -1.0).all()


def test_quantiser_of_nothing():
    assert quantize_int8(torch.zeros(0, 5, device="cuda")).codes.shape == (0, 16)
    m = quantize_int8(torch.zeros(5, 0, device="cuda"))
    assert m.codes.shape == (5, 0) and (m.scale == 2.0 ** -126).all()


# ------------------------------------------------------------------ products


def matrix(key, rows, cols, scale_layout="dense", low=-4, high=4):
    """Codes of the whole range, -128 too, with scales of any value; bytes past the columns are junk."""
    r = rng(7, *key)
    codes = r.integers(-128, 128, (rows, -(-cols // 16) * 16 + 16 * int(r.integers(0, 3)))).astype(np.int8)
    scale = torch.from_numpy(np.exp2(r.uniform(low, high, rows)).astype(np.float32)).cuda()
    if scale_layout == "strided":
        scale = torch.stack([scale, torch.full_like(scale, float("nan"))], dim=1)[:, 0]
    elif scale_layout == "one":
        scale = torch.full((1,), 0.375, device="cuda").expand(rows)
    return Int8Matrix(torch.from_numpy(codes).cuda(), scale, cols=cols)


def expected(a, b, out):
    """The header's arithmetic, bit for bit: exact sums, rounded to float32, times the rounded product of the
    scales' fractions, then the powers of two."""
    sums = host(a.values) @ host(b.values).T  # whole numbers below 2^53
    fa, ea = np.frexp(a.scale.cpu().numpy())
    fb, eb = np.frexp(b.scale.cpu().numpy())
    with np.errstate(over="ignore", under="ignore"):
        v = sums.astype(np.float32) * (fa[:, None] * fb[None, :])
        v = np.ldexp(v.astype(np.float64), ea[:, None] + eb[None, :]).astype(np.float32)
    return torch.from_numpy(v).to(TORCH[out])


def same(x, y):
    return torch.equal(x.cpu(), y)


PRODUCTS = [(1, 1, 1), (1, 33, 128), (2, 128, 127), (16, 200, 129), (17, 64, 16), (33, 1, 1000), (48, 70, 4100), (64, 130, 260),
            (65, 128, 128), (128, 128, 128), (129, 300, 640), (300, 257, 384), (64, 1000, 2065), (520, 131, 257), (15, 4100, 144),
            (40, 24, 5000), (5, 20, 131071), (130, 40, 131000)]
LARGE = [(512, 512, 128), (520, 515, 130), (1000, 777, 1000), (513, 1300, 2048), (600, 4100, 257), (2050, 640, 390),
         (520, 600, 9000), (300, 520, 20000), (129, 2000, 4097), (2200, 2100, 100), (3000, 2500, 700),
         (2000, 1900, 1500), (4200, 4100, 900), (30, 4100, 3000)]


@pytest.mark.parametrize("m,n,k", PRODUCTS + LARGE)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_products(m, n, k, out):
    a, b = matrix((1, m, k), m, k), matrix((2, n, k), n, k)
    got = matmul_int8(a, b, out_dtype=TORCH[out])
    assert got.dtype == TORCH[out] and same(got, expected(a, b, out))


def test_every_kernel_is_tested():
    """The sizes above reach every kernel, and sums in parts."""
    seen = {spectral_matmul_int8_kernel(sn_matmul_int8(*size, SN_I8, CODE[out]))[:2] for size in PRODUCTS + LARGE + WIDE
            for out in ("f32", "bf16")}
    assert {name for name, _ in seen} >= {"few_rows", "small", "tile_4", "tile_8", "big"} and any(parts > 1 for _, parts in seen)


WIDE = [(8100, 8000, k) for k in (1, 100, 128, 129, 256, 300, 384, 512, 600, 1000)]


@pytest.mark.parametrize("m,n,k", WIDE)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_large_tiles_of_few_blocks(m, n, k, out):
    g = torch.Generator(device="cuda").manual_seed(k)
    mats = []
    for rows in (m, n):
        codes = torch.randint(-128, 128, (rows, -(-k // 16) * 16), generator=g, device="cuda").to(torch.int8)
        mats.append(Int8Matrix(codes, torch.full((rows,), 0.5, device="cuda"), cols=k))
    ref = (mats[0].values.float() @ mats[1].values.float().t()) * 0.25  # sums below 2^24
    assert torch.equal(matmul_int8(*mats, out_dtype=TORCH[out]), ref.to(TORCH[out]))


# sums in parts of every kind of tile, the last part's last block ragged, and few rows in blocks of 16 to 64
SPLIT = [(66, 5451, 9963), (300, 4096, 14301), (65, 5458, 7692), (70, 4506, 9750), (130, 1000, 5001), (300, 2000, 7001)]
FEW = [(16, 4000, 1000), (17, 4000, 500), (32, 8192, 1001), (49, 8000, 900), (50, 515, 1024), (64, 8192, 1000)]


@pytest.mark.parametrize("m,n,k", SPLIT + FEW)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_products_in_parts_and_of_few_rows(m, n, k, out):
    a, b = matrix((27, m, k), m, k), matrix((28, n, k), n, k, "strided")
    assert same(matmul_int8(a, b, out_dtype=TORCH[out]), expected(a, b, out))


def test_every_kernel_is_tested_in_parts():
    for out in ("f32", "bf16"):
        seen = {}
        for size in SPLIT + FEW:
            name, parts, _, _ = spectral_matmul_int8_kernel(sn_matmul_int8(*size, SN_I8, CODE[out]))
            seen.setdefault((name, parts > 1), set()).add(-(-size[0] // 16))
        assert {("tile_4", True), ("tile_8", True), ("small", True)} <= set(seen), seen
        assert seen["few_rows", False] >= {1, 2, 4}, seen  # blocks of 16 rows


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(31, 8192, 1530), (32, 8192, 1400), (17, 4000, 2700), (300, 4096, 14301), (65, 5458, 7692)])
def test_plain_operands_of_every_kernel(dtype, m, n, k):
    """Rows whose codes fill the LDS of the kernel for few, and tiles whose sums are in parts."""
    x = on_gpu(wide(rng(29, m, k), m, k), dtype)
    b = matrix((30, n, k), n, k)
    got = matmul_int8(x, b, out_dtype=torch.float32)
    assert same(got, expected(quantize_int8(x), b, "f32"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("base", [32, 496, 2032, 8192])
def test_rows_of_every_length_past_a_whole_one(dtype, base):
    """1 to 16 columns past the last whole load."""
    for cols in range(base + 1, base + 17):
        x = on_gpu(wide(rng(31, cols), 3, cols), dtype)
        check_quantized(quantize_int8(x), host(x))
        room = torch.full((3, cols + 5), float("nan"), dtype=TORCH[dtype], device="cuda")
        room[:, 3:3 + cols] = x
        check_quantized(quantize_int8(room[:, 3:3 + cols]), host(x))


@pytest.mark.parametrize("layout", ["strided", "one"])
@pytest.mark.parametrize("m,n,k", [(5, 300, 700), (300, 260, 700), (1, 1, 100), (2100, 2200, 130), (70, 300, 6000)])
def test_scales_of_any_strides(layout, m, n, k):
    a, b = matrix((5, m, k), m, k, layout), matrix((6, n, k), n, k, layout)
    assert same(matmul_int8(a, b, out_dtype=torch.float32), expected(a, b, "f32"))


@pytest.mark.parametrize("m,n,k", [(3, 40, 200), (200, 140, 200)])
def test_scales_far_apart(m, n, k):
    """Products of scales outside float32's range, whose results are inside."""
    for la, ha, lb, hb in ((100, 119, -126, -100), (-126, -90, 60, 119), (-126, -100, -60, 0), (60, 119, 0, 40)):
        a, b = matrix((8, m, k), m, k, low=la, high=ha), matrix((9, n, k), n, k, low=lb, high=hb)
        assert same(matmul_int8(a, b, out_dtype=torch.float32), expected(a, b, "f32"))


@pytest.mark.parametrize("m,n,k", [(4, 50, 300), (150, 140, 300)])
def test_rows_of_nan_stay_apart(m, n, k):
    a, b = matrix((10, m, k), m, k), matrix((11, n, k), n, k)
    ref = matmul_int8(a, b, out_dtype=torch.float32)
    a.scale[2] = float("nan")
    b.scale[7] = float("nan")
    got = matmul_int8(a, b, out_dtype=torch.float32)
    assert torch.isnan(got[2]).all() and torch.isnan(got[:, 7]).all()
    got[2], got[:, 7] = ref[2], ref[:, 7]
    assert torch.equal(got, ref)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 37, 256), (70, 37, 256), (300, 515, 4000), (2100, 2050, 200)])
@pytest.mark.parametrize("offset,extra", [(0, 8), (1, 3), (2, 2)])
def test_result_in_a_window(out, m, n, k, offset, extra):
    a, b = matrix((12, m, k), m, k), matrix((13, n, k), n, k)
    room = torch.full((m + 1, n + offset + extra), 7.0, dtype=TORCH[out], device="cuda")
    got = matmul_int8(a, b, out=room[:m, offset:offset + n])
    assert same(got, expected(a, b, out))
    room[:m, offset:offset + n] = 7.0
    assert (room == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k,offset", [(1, 200, 1000, 0), (1, 65, 40, 3), (7, 129, 257, 0), (16, 300, 2100, 1), (33, 128, 384, 0),
                                          (31, 200, 1530, 0), (32, 64, 4096, 2), (17, 700, 8200, 0), (64, 900, 1030, 0),
                                          (200, 130, 515, 0), (1, 100, 48000, 0), (1, 100, 60000, 0), (4, 33, 0, 0)])
def test_plain_operand_is_quantised_on_the_way(dtype, m, n, k, offset):
    room = torch.full((m, k + offset + 4), float("nan"), dtype=TORCH[dtype], device="cuda")
    x = room[:, offset:offset + k]
    x.copy_(on_gpu(wide(rng(m, n, k), m, max(k, 1))[:, :k], dtype))
    b, codes = matrix((14, n, k), n, k), quantize_int8(x)
    got = matmul_int8(x, b, out_dtype=torch.float32)
    assert same(got, expected(codes, b, "f32")) and torch.equal(got, matmul_int8(codes, b, out_dtype=torch.float32))


@pytest.mark.parametrize("m", [3, 100])
def test_plain_rows_that_are_not_finite(m):
    x = on_gpu(wide(rng(15), m, 500), "bf16")
    b = matrix((15, 60), 60, 500)
    ref = matmul_int8(x, b)
    x[1, 100] = float("nan")
    got = matmul_int8(x, b)
    assert torch.isnan(got[1]).all()
    got[1] = ref[1]
    assert torch.equal(got, ref)


def test_the_same_row_gives_the_same_bits_in_any_product():
    """One row alone, among few, in tiles and in sums by parts."""
    x = on_gpu(wide(rng(16), 400, 6000), "bf16")
    b = matrix((16, 300), 300, 6000)
    whole = matmul_int8(x, b, out_dtype=torch.float32)
    for rows in (slice(0, 1), slice(5, 20), slice(0, 64), slice(100, 230)):
        assert torch.equal(matmul_int8(x[rows], b, out_dtype=torch.float32), whole[rows])
        assert torch.equal(matmul_int8(quantize_int8(x[rows]), b, out_dtype=torch.float32), whole[rows])


def test_matrices_beyond_32_bits():
    """More than 2^32 elements: the bits of their last rows alone."""
    rows, k = 40000, 110000
    x = on_gpu(wide(rng(25), 1000, k), "bf16").repeat(rows // 1000, 1)
    x[-3:] *= 2
    m = quantize_int8(x)
    last = quantize_int8(x[-200:].clone())
    assert torch.equal(m.codes[-200:], last.codes) and torch.equal(m.scale[-200:], last.scale)
    del x
    b = matrix((25, 64), 64, k)
    whole = matmul_int8(m, b, out_dtype=torch.float32)
    assert torch.equal(whole[-200:], matmul_int8(last, b, out_dtype=torch.float32))
    assert torch.equal(matmul_int8(b, m, out_dtype=torch.float32)[:, -200:], whole[-200:].t())  # as the other operand


def test_products_of_nothing():
    a, b = quantize_int8(torch.zeros(3, 0, device="cuda")), quantize_int8(torch.zeros(100, 0, device="cuda"))
    assert (matmul_int8(a, b) == 0).all()
    assert matmul_int8(quantize_int8(torch.zeros(0, 9, device="cuda")), quantize_int8(torch.ones(4, 9, device="cuda"))).shape == (0, 4)


def test_refusals():
    x = torch.ones(4, 40, device="cuda")
    a, b = quantize_int8(x), quantize_int8(torch.ones(6, 40, device="cuda"))
    codes, scale = b.codes, b.scale
    for bad in (lambda: quantize_int8(x.t()), lambda: quantize_int8(x.half()), lambda: quantize_int8(x[0]),
                lambda: quantize_int8(x.clone().requires_grad_()), lambda: Int8Matrix(codes, scale[:5]),
                lambda: Int8Matrix(codes, scale.double()), lambda: Int8Matrix(codes.t(), scale),
                lambda: Int8Matrix(codes[:, 1:], scale, cols=16), lambda: Int8Matrix(codes[:, :40], scale),
                lambda: Int8Matrix(codes, scale, cols=49), lambda: matmul_int8(a, codes), lambda: matmul_int8(x[:, :39], b),
                lambda: matmul_int8(a, b, out_dtype=torch.float16), lambda: matmul_int8(a, b, out=torch.empty(4, 5, device="cuda")),
                lambda: matmul_int8(a, b, out=torch.empty(6, 4, device="cuda").t()),
                lambda: matmul_int8(quantize_int8(torch.ones(200, 40, device="cuda")), quantize_int8(torch.ones(3, 48, device="cuda"))),
                lambda: matmul_int8(torch.ones(99, 40, device="cuda"), b, workspace=torch.empty(1 << 20, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with torch.no_grad():
        quantize_int8(x.clone().requires_grad_())


@pytest.mark.parametrize("which", ["a", "b", "out"])
def test_scales_and_results_that_require_gradients_are_refused(which):
    a, b = (quantize_int8(on_gpu(wide(rng(26, i), n, 40), "f32")) for i, n in enumerate((4, 6)))
    ref = matmul_int8(a, b, out_dtype=torch.float32)
    out = torch.zeros(4, 6, device="cuda", requires_grad=which == "out")
    m = {"a": a, "b": b}.get(which)
    if m is not None:
        m.scale.requires_grad_()
    with pytest.raises(ValueError, match="gradients"):
        matmul_int8(a, b, out=out)
    assert (out == 0).all()
    with torch.no_grad():
        assert torch.equal(matmul_int8(a, b, out=out), ref)


# ------------------------------------------------------- streams and graphs


def test_calls_replay_from_a_graph():
    """One token, a few, tiles with parts, and a plain operand with a workspace: new inputs in the same memory, with eager
    work and synchronisation between replays."""
    b = matrix((20, 500), 500, 3000)
    xs = [on_gpu(wide(rng(21, m), m, 3000), "bf16") for m in (1, 40, 300)]
    outs = [torch.empty(x.shape[0], 500, dtype=torch.bfloat16, device="cuda") for x in xs]
    ws = [torch.empty(1 << 23, dtype=torch.uint8, device="cuda") for _ in xs]
    for x, o, w in zip(xs, outs, ws):
        matmul_int8(x, b, out=o, workspace=w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x, o, w in zip(xs, outs, ws):
            matmul_int8(x, b, out=o, workspace=w)
    for rep in range(4):
        for i, x in enumerate(xs):
            x.copy_(on_gpu(wide(rng(22, rep, i), *x.shape), "bf16"))
            outs[i].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for x, o in zip(xs, outs):
            assert torch.equal(o, matmul_int8(x, b))


def test_two_streams_at_once():
    b = matrix((23, 600), 600, 4000)
    xs = [on_gpu(wide(rng(24, i), 200, 4000), "bf16") for i in range(2)]
    refs = [matmul_int8(x, b) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(matmul_int8(xs[i], b))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, refs[i]) for g in got[i])
