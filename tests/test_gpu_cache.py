"""The 8-bit cache of keys and values and attention over it against the float64 oracle (oracle.cache)."""

import numpy as np
import pytest
import torch

from oracle import cache as oracle, fp8_blocks

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - collected on CPU machines, skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2602_18851_amd import Fp8Cache, Rotary, matmul_int8, quantize_int8  # noqa: E402

TORCH = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2, "f32": torch.float32, "bf16": torch.bfloat16}


def rng(*key):
    return np.random.default_rng([20261209, *key])


def on_gpu(x, dtype):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(TORCH[dtype]).cuda()


def host(t):
    return t.detach().cpu().double().numpy()


def fmt_of(cache):
    return "e4m3" if cache.k.dtype == TORCH["e4m3"] else "e5m2"


def held(cache):
    """Values of keys and values [pages, heads, page, d]."""
    out = []
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        with np.errstate(invalid="ignore"):
            out.append(fp8_blocks.decode(codes.view(torch.uint8).cpu().numpy(), fmt_of(cache)) * host(scale)[..., None])
    return out


def spread(r, *shape):
    return r.standard_normal(shape) * np.exp2(r.integers(-3, 4, (*shape[:-1], 1))) * np.exp2(r.integers(-2, 3, shape[-1]))


# ------------------------------------------------------------------ write and read


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,heads,dh,page", [(1, 1, 16, 16), (5, 3, 64, 16), (37, 8, 128, 32), (70, 2, 80, 64), (9, 5, 256, 128),
                                                  (33, 25, 96, 16), (20, 1, 48, 1024)])
def test_rows_go_to_their_slots_and_back(fmt, dtype, tokens, heads, dh, page):
    r = rng(tokens, heads, dh, page)
    pages = tokens // page + 3
    c = Fp8Cache.empty(pages, heads, page, dh, fmt)
    for t in (c.k, c.v):
        t.view(torch.uint8).fill_(0x55)
    for t in (c.k_scale, c.v_scale):
        t.fill_(-1.0)
    k, v = (on_gpu(spread(r, tokens, heads, dh), dtype) for _ in range(2))
    slots = r.permutation(pages * page)[:tokens]
    c.write(k, v, torch.from_numpy(slots).cuda())
    for x, codes, scale in ((k, c.k, c.k_scale), (v, c.v, c.v_scale)):
        ref_codes = np.full((pages, heads, page, dh), fp8_blocks.decode(np.uint8([0x55]), fmt)[0])
        ref_scale = np.full((pages, heads, page), -1.0)
        cs, ss = oracle.rows(host(x), fmt)
        ref_codes[slots // page, :, slots % page], ref_scale[slots // page, :, slots % page] = cs, ss
        np.testing.assert_array_equal(fp8_blocks.decode(codes.view(torch.uint8).cpu().numpy(), fmt), ref_codes)
        np.testing.assert_array_equal(host(scale), ref_scale)
    at = torch.from_numpy(r.permutation(slots)).cuda()
    at = torch.cat([at, at[:1]])  # a place may be read twice
    for out in ("f32", "bf16"):
        got = c.read(at, dtype=TORCH[out])
        for g, full in zip(got, held(c)):
            n = at.cpu().numpy()
            # products of a code and a power of two: exact in either type
            assert g.dtype == TORCH[out] and np.array_equal(host(g), full[n // page, :, n % page])


def test_slots_outside_are_padding():
    c = Fp8Cache.empty(3, 2, 16, 64)
    k, v = (on_gpu(spread(rng(1, i), 6, 2, 64), "bf16") for i in range(2))
    slots = torch.tensor([-1, 47, 48, 1 << 40, -(1 << 40), 5], device="cuda")
    c.write(k, v, slots)
    ref = Fp8Cache.empty(3, 2, 16, 64)
    ref.write(k[[1, 5]], v[[1, 5]], slots[[1, 5]])
    for a, b in ((c.k, ref.k), (c.v, ref.v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(c.k_scale, ref.k_scale) and torch.equal(c.v_scale, ref.v_scale)
    got = c.read(slots, out=tuple(torch.full_like(k, float("nan")) for _ in range(2)))
    for g, r in zip(got, ref.read(slots[[1, 5]])):
        assert (g[[0, 2, 3, 4]] == 0).all() and torch.equal(g[[1, 5]], r)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_rows_of_extremes(fmt):
    """Zeros, the scale's lower limit, the largest numbers, infinities and NaN."""
    x = np.zeros((7, 1, 64))
    largest = fp8_blocks.FORMATS[fmt][2]
    x[1, 0, :2], x[2, 0, :3], x[3, 0, :2] = (2.0 ** -130, -2.0 ** -140), (largest, 1.0, -3.3), (1.5e38, -1e30)
    x[4, 0, 5], x[5, 0, 63] = np.inf, np.nan
    x[6, 0] = np.nextafter(np.float32(largest), np.float32(np.inf))
    c = Fp8Cache.empty(1, 1, 16, 64, fmt)
    t = on_gpu(x, "f32")
    c.write(t, t, torch.arange(7, device="cuda"))
    with np.errstate(invalid="ignore"):
        codes, scale = oracle.rows(host(t), fmt)
    for cs, ss in ((c.k, c.k_scale), (c.v, c.v_scale)):
        np.testing.assert_array_equal(fp8_blocks.decode(cs.view(torch.uint8).cpu().numpy()[0, 0, :7], fmt), codes[:, 0])
        np.testing.assert_array_equal(host(ss)[0, 0, :7], scale[:, 0])


@pytest.mark.parametrize("fmt,first", [("e4m3", 1.9375), ("e5m2", 1.875)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_elements_that_round_to_an_infinity(fmt, first, dtype):
    """The last element that is held as a finite one, the next, and the type's largest: 2^128 from `first` 2^127 on."""
    last = torch.tensor(first * 2.0 ** 127).to(TORCH[dtype])
    below = torch.nextafter(last, torch.zeros_like(last)) if dtype == "f32" else (last.view(torch.int16) - 1).view(torch.bfloat16)
    x = torch.stack([below, last, torch.tensor(torch.finfo(TORCH[dtype]).max).to(TORCH[dtype])]).cuda()
    x = torch.stack([x, -x]).reshape(6, 1, 1).repeat(1, 1, 16)
    x[:, :, 1:] = 1.0
    c = Fp8Cache.empty(1, 1, 16, 16, fmt)
    c.write(x, x, torch.arange(6, device="cuda"))
    for got in c.read(torch.arange(6, device="cuda"), dtype=torch.float32):
        down = 2 * first - 2.0  # the mantissa below the midpoint
        want = torch.tensor([down * 2.0 ** 127, float("inf"), float("inf")])
        assert torch.equal(got[:3, 0, 0].cpu(), want) and torch.equal(got[3:, 0, 0].cpu(), -want)
    q = torch.full((1, 1, 1, 16), 2.0 ** -120, device="cuda").to(TORCH[dtype])
    table, lengths = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    assert torch.isfinite(c.attend(q, table, lengths)).all()
    assert not torch.isfinite(c.attend(q, table, lengths + 1)[..., 0]).any()


def test_rows_of_any_strides_and_pages_apart():
    """Keys and values as windows of one projection; a cache whose pages hold keys and values side by side."""
    r = rng(3)
    both = torch.zeros(4, 2, 3, 16, 80, dtype=torch.uint8, device="cuda").view(TORCH["e4m3"])
    scales = torch.zeros(4, 2, 3, 16, device="cuda")
    c = Fp8Cache(both[:, 0], scales[:, 0], both[:, 1], scales[:, 1])
    qkv = on_gpu(spread(r, 20, 1, 7 * 80 + 5)[:, 0], "bf16")
    k, v = qkv[:, 81:81 + 240].view(20, 3, 80), qkv[:, 321:321 + 240].view(20, 3, 80)
    slots = torch.from_numpy(r.permutation(64)[:20]).cuda()
    c.write(k, v, slots)
    ref = Fp8Cache.empty(4, 3, 16, 80)
    ref.write(k.contiguous(), v.contiguous(), slots)
    for a, b in ((c.k, ref.k), (c.v, ref.v)):
        assert torch.equal(a.contiguous().view(torch.uint8), b.view(torch.uint8))
    room = torch.full((2, 3, 20, 83), 7.0, device="cuda")  # tokens within heads
    out = [room[i, :, :, 1:81].transpose(0, 1) for i in range(2)]
    c.read(slots, out=out)
    for a, b in zip(out, ref.read(slots, dtype=torch.float32)):
        assert torch.equal(a, b)
    assert (room[..., 0] == 7.0).all() and (room[..., 81:] == 7.0).all()
    c.write(k.transpose(0, 1).contiguous().transpose(0, 1), v, slots)  # tokens within heads
    assert torch.equal(c.k.contiguous().view(torch.uint8), ref.k.view(torch.uint8))
    q = on_gpu(r.standard_normal((1, 2, 6, 80)), "bf16")
    table, lengths = torch.tensor([[2, 0, 3, 1]], dtype=torch.int32, device="cuda"), torch.tensor([64], dtype=torch.int32, device="cuda")
    assert torch.equal(c.attend(q, table, lengths), ref.attend(q, table, lengths))


# ------------------------------------------------------------------ attention


def setup(key, batch, drafts, heads, group, dh, page, lengths, fmt="e4m3", dtype="bf16", junk=True, spare=2):
    """A cache with the sequences' places in pages of any order; all else of it is NaN."""
    r = rng(11, *key)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + spare
    cols = max(max(need), 1)
    c = Fp8Cache.empty(pages, heads, page, dh, fmt)
    if junk:
        for t in (c.k, c.v):
            t.view(torch.uint8).fill_(0x7F)
        for t in (c.k_scale, c.v_scale):
            t.fill_(float("nan"))
    ids = r.permutation(pages)
    table = np.full((batch, cols), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
        if lengths[b]:
            t = np.arange(lengths[b])
            slots = torch.from_numpy(table[b, t // page].astype(np.int64) * page + t % page).cuda()
            c.write(*(on_gpu(spread(r, lengths[b], heads, dh), "f32") for _ in range(2)), slots)
    q = on_gpu(r.standard_normal((batch, drafts, heads * group, dh)) * 0.7, dtype)
    return c, q, torch.from_numpy(table).cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")


def trees(key, drafts, n=None):
    r = rng(12, *key)
    out = np.zeros((n or 1, drafts), np.uint64)
    for m in out:
        for i in range(drafts):
            parent = int(r.integers(-1, i)) if i else -1
            m[i] = (int(m[parent]) if parent >= 0 else 0) | (1 << i)
    return out if n else out[0]


def check(got, q, cache, table, lengths, masks=None, scale=None):
    """The rounding errors of the sums q k over d elements, in the matrix cores' order (2^-23 each of the magnitudes' sum at
    most, and float32 queries held to 2^-24), of the exponent (the factor and one product, 2^-23 of it, twice) and
    of its power (2^-22) are errors of the weights, relative to them: `off`.  They enter a result once as its weights and
    once as their sum.  Weights are held to 2^-16 (bf16) or 2^-24, sums over n places and some joins round n + 64 times."""
    dtype = "f32" if q.dtype == torch.float32 else "bf16"
    d = q.shape[3]
    ref, mag, reach = oracle.attend(host(q), *held(cache), table.cpu().numpy(), lengths.cpu().numpy(),
                                    None if masks is None else masks, scale)
    n = int(lengths.max())
    off = reach[..., None] * (d + 8) * 2.0 ** -23 + 2.0 ** -22
    tol = mag * (2 * off * (1 + off) + (2.0 ** -16 if dtype == "bf16" else 2.0 ** -24) + 2 * (n + 64) * 2.0 ** -23)
    tol += np.abs(ref) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) + 1e-37
    got = host(got)
    assert (np.isnan(got) == np.isnan(ref)).all()
    err = np.abs(got - ref)
    fine = ~np.isnan(ref)
    assert (err[fine] <= tol[fine]).all(), float((err[fine] / tol[fine]).max())


def gpu_masks(m):
    return torch.from_numpy(m.view(np.int64)).cuda()


# batch, drafts, heads, group, d_h, page, lengths
SHAPES = [
    (1, 1, 1, 1, 16, 16, [1]), (1, 1, 2, 4, 64, 16, [33]), (3, 1, 2, 8, 128, 16, [1, 31, 200]), (2, 1, 3, 5, 80, 32, [64, 65]),
    (2, 1, 2, 1, 96, 64, [100, 7]), (2, 1, 1, 16, 128, 128, [300, 129]), (1, 1, 2, 20, 64, 16, [500]), (1, 1, 1, 3, 256, 16, [77]),
    (2, 2, 2, 4, 64, 16, [50, 2]), (2, 7, 1, 8, 128, 32, [90, 600]), (1, 64, 2, 1, 64, 16, [700]), (1, 33, 1, 5, 128, 16, [40]),
    (2, 64, 1, 8, 128, 64, [64, 400]), (1, 20, 1, 3, 256, 16, [130]), (1, 64, 1, 4, 256, 32, [300]), (1, 64, 1, 5, 112, 16, [129]),
    (1, 17, 1, 2, 48, 16, [1000]), (5, 3, 2, 2, 32, 16, [3, 4, 0, 1, 60]),
]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("fmt,dtype", [("e4m3", "bf16"), ("e4m3", "f32"), ("e5m2", "bf16"), ("e5m2", "f32")])
@pytest.mark.parametrize("tree", ["chain", "one", "each"])
def test_attention(shape, fmt, dtype, tree):
    batch, drafts = shape[:2]
    c, q, table, lengths = setup(shape[:6], *shape, fmt=fmt, dtype=dtype)
    masks = None if tree == "chain" else trees(shape[:6], drafts, batch if tree == "each" else None)
    got = c.attend(q, table, lengths, tree=None if masks is None else gpu_masks(masks))
    check(got, q, c, table, lengths, masks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,drafts,heads,group,dh,page,lengths", [
    (1, 1, 1, 8, 128, 64, [9001]), (3, 1, 2, 4, 64, 16, [5000, 300, 2049]), (2, 5, 1, 8, 128, 32, [4100, 257]),
    (70, 1, 1, 2, 64, 16, [200 + 13 * i for i in range(70)]), (1, 64, 1, 8, 128, 256, [3000]), (2, 2, 1, 4, 256, 64, [2500, 2]),
    (1, 6, 2, 5, 256, 32, [7001]), (3, 9, 1, 8, 208, 64, [3100, 1, 900]), (1, 3, 2, 8, 128, 64, [6000])])
def test_sequences_in_chunks(batch, drafts, heads, group, dh, page, lengths, dtype):
    """Lengths at which workgroups share a sequence, beside short ones."""
    c, q, table, lens = setup((batch, drafts, dh), batch, drafts, heads, group, dh, page, lengths, dtype=dtype)
    got = c.attend(q, table, lens)
    check(got, q, c, table, lens)
    assert torch.equal(got, c.attend(q, table, lens))  # the same bits again


def test_a_long_sequence():
    """Equal keys, so that every weight is the same, and values that are whole numbers: the mean."""
    n, page = 131071, 256
    c = Fp8Cache.empty(512, 1, page, 64)
    c.k_scale.fill_(1.0)
    c.v_scale.fill_(1.0)
    g = torch.Generator(device="cuda").manual_seed(1)
    c.v.copy_(torch.randint(-8, 9, c.v.shape, generator=g, device="cuda").float())
    table = torch.randperm(512, generator=g, device="cuda").to(torch.int32)[None]
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    q = torch.randn(1, 1, 4, 64, generator=g, device="cuda")
    got = c.attend(q, table, lengths)
    v = c.v.float()[table[0].long()].view(-1, 64)[:n].double()
    # weights of 1 are exact; sums of whole numbers below 2^24 too; a division
    assert ((got.double() - v.mean(0)).abs() <= v.mean(0).abs() * 2.0 ** -22).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drafts", [1, 20])
def test_pages_beyond_32_bits(drafts, dtype):
    """A cache of more than 2^32 bytes of codes, its last pages in use: the bits of a small one."""
    heads, page, dh = 8, 256, 128
    pages = 17000
    big = Fp8Cache.empty(pages, heads, page, dh)
    small, q, table, lengths = setup((16, drafts), 2, drafts, heads, 8, dh, page, [1000, 300], dtype=dtype, junk=False)
    far = torch.where(table >= 0, pages - 1 - table, table)
    for b in range(2):
        at = torch.arange(int(lengths[b]), device="cuda")
        near = table[b].long()[at // page] * page + at % page
        k, v = small.read(near, dtype=torch.float32)
        slots = far[b].long()[at // page] * page + at % page
        assert int(slots.max()) * heads * dh > 1 << 32
        big.write(k, v, slots)
        for x, y in zip(big.read(slots), small.read(near)):
            assert torch.equal(x, y)
    assert torch.equal(big.attend(q, far, lengths), small.attend(q, table, lengths))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_nothing(dtype):
    c, q, table, lengths = setup((1,), 4, 3, 2, 2, 64, 16, [3, 40, 0, 3], dtype=dtype)
    masks = np.zeros((4, 3), np.uint64)
    masks[0, 1], masks[3] = 0b010, 0b111
    got = c.attend(q, table, lengths, tree=gpu_masks(masks))
    check(got, q, c, table, lengths, masks)
    assert (got[0, [0, 2]] == 0).all() and (got[2] == 0).all()


def test_masks_of_64_tokens():
    """The highest bit, and bits of later tokens."""
    c, q, table, lengths = setup((2,), 1, 64, 1, 1, 64, 16, [90])
    masks = (np.uint64(1) << np.arange(64, dtype=np.uint64))
    masks[3] = np.uint64((1 << 64) - 1)
    masks[63] = np.uint64(1 << 63)
    check(c.attend(q, table, lengths, tree=gpu_masks(masks)), q, c, table, lengths, masks)
    c, q, table, lengths = setup((3,), 2, 5, 1, 2, 64, 16, [90, 4])
    masks = np.full((2, 5), (1 << 64) - 1, np.uint64)  # bits past the tokens say nothing
    check(c.attend(q, table, lengths, tree=gpu_masks(masks)), q, c, table, lengths, masks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["written", "codes"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_drafts_that_are_not_finite_reach_who_sees_them(dtype, what, fmt):
    """A drafted token's row of NaN (or of one NaN code): NaN where it is seen, the finite result elsewhere."""
    c, q, table, lengths = setup((4,), 1, 6, 1, 2, 64, 16, [45], fmt=fmt, dtype=dtype)
    masks = np.array([0b1, 0b11, 0b101, 0b1011, 0b10101, 0b100011], np.uint64)
    place = 45 - 6 + 1  # token 1: seen by itself, 3 and 5
    page, at = int(table[0, place // 16]), place % 16
    before = c.attend(q, table, lengths, tree=gpu_masks(masks))
    check(before, q, c, table, lengths, masks)
    if what == "written":
        bad = torch.full((1, 1, 64), float("nan"), device="cuda")
        c.write(torch.zeros_like(bad), bad, torch.tensor([page * 16 + at], device="cuda"))
    else:
        c.v.view(torch.uint8)[page, 0, at, 17] = 0x7F
    got = c.attend(q, table, lengths, tree=gpu_masks(masks))
    for i in range(6):
        if masks[i] & np.uint64(2):
            assert torch.isnan(got[0, i] if what == "written" else got[0, i, :, 17]).all()
        else:
            assert torch.equal(got[0, i], before[0, i])
    if what == "codes":
        assert torch.isfinite(got[0, :, :, :17]).all() and torch.isfinite(got[0, :, :, 18:]).all()
    nan = torch.full((1, 1, 64), float("nan"), device="cuda")
    c.write(nan, torch.zeros_like(nan), torch.tensor([page * 16 + at], device="cuda"))  # and of keys
    got = c.attend(q, table, lengths, tree=gpu_masks(masks))
    for i in range(6):
        if masks[i] & np.uint64(2):
            assert torch.isnan(got[0, i]).all()
        else:
            assert torch.equal(got[0, i], before[0, i])


@pytest.mark.parametrize("drafts,group,dh", [(40, 2, 64), (40, 2, 128), (64, 4, 64), (64, 4, 128), (20, 6, 80), (30, 2, 64), (9, 2, 256)])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_trees_with_drafts_that_are_not_finite(drafts, group, dh, fmt):
    """Rows of NaN, one NaN code, pages that are not there, and tokens that see nothing, where the rows fill waves."""
    c, q, table, lengths = setup((14, drafts, dh), 2, drafts, 1, group, dh, 16, [drafts + 61, drafts + 150], fmt=fmt)
    masks = trees((14, drafts), drafts, 2)
    masks[0, 5] = masks[1, 0] = 0
    table[1, 3] = -1
    before = c.attend(q, table, lengths, tree=gpu_masks(masks))
    check(before, q, c, table, lengths, masks)
    bits = [int(m) >> 2 & 1 for m in masks[1]]  # who sees token 2 of the second sequence
    place = 150 + 2
    page, at = int(table[1, place // 16]), place % 16
    c.v.view(torch.uint8)[page, 0, at, dh - 3] = 0x7F
    got = c.attend(q, table, lengths, tree=gpu_masks(masks))
    check(got, q, c, table, lengths, masks)
    for i, sees in enumerate(bits):
        assert torch.isnan(got[1, i, :, dh - 3]).all() == bool(sees)
    other = torch.arange(dh, device="cuda") != dh - 3
    assert torch.equal(got[..., other], before[..., other])
    nan = torch.full((1, 1, dh), float("nan"), device="cuda")
    for k, v in ((torch.zeros_like(nan), nan), (nan, torch.zeros_like(nan))):
        c.write(k, v, torch.tensor([page * 16 + at], device="cuda"))
        got = c.attend(q, table, lengths, tree=gpu_masks(masks))
        for i, sees in enumerate(bits):
            assert torch.isnan(got[1, i]).all() if sees else torch.equal(got[1, i], before[1, i])
        assert torch.equal(got[0], before[0])


@pytest.mark.parametrize("batch,drafts,group,dh,lengths", [
    (66, 9, 8, 64, [20 + 3 * i for i in range(66)]), (3, 64, 3, 128, [70, 5000, 900]), (2, 64, 2, 64, [4000, 64]),
    (130, 1, 2, 64, [1 + 7 * i for i in range(130)])])
def test_many_rows_in_chunks(batch, drafts, group, dh, lengths):
    """More than 64 sequences, and trees over sequences that workgroups share."""
    c, q, table, lens = setup((15, batch, dh), batch, drafts, 1, group, dh, 32, lengths)
    masks = trees((15, batch), drafts, batch)
    got = c.attend(q, table, lens, tree=gpu_masks(masks))
    check(got, q, c, table, lens, masks)
    assert torch.equal(got, c.attend(q, table, lens, tree=gpu_masks(masks)))


LONG_CHUNKS = [
    # trees, with pairs of waves and without: chunks of 20 tiles of 128 places in windows of 8, of 35 of 64 in windows of 16
    (256, 9, 8, 64, 16, 5120, "bf16"), (128, 17, 8, 64, 32, 5120, "bf16"),
    (256, 9, 8, 128, 64, 4480, "bf16"), (128, 17, 8, 128, 16, 4480, "bf16"),
    # whole sequences of 70 and 20 tiles, whose shares are looked up
    (512, 9, 8, 128, 16, 4480, "bf16"), (272, 17, 8, 64, 16, 2560, "bf16"),
    # 137 to 140 steps a wave, with four, two and one of them to the same rows; pages are looked up 64 steps at a time
    (512, 1, 8, 128, 64, 35200, "bf16"), (512, 1, 4, 64, 16, 35200, "f32"), (256, 3, 8, 256, 16, 17920, "bf16"),
    (512, 8, 8, 64, 32, 17920, "bf16"), (256, 16, 8, 128, 16, 8960, "f32")]


@pytest.mark.parametrize("batch,drafts,group,dh,page,length,dtype", LONG_CHUNKS)
def test_long_chunks(batch, drafts, group, dh, page, length, dtype):
    """So many sequences, copies of two, that a workgroup walks through several windows of page numbers, with pages that are not
    there and a ragged end past the first window.  All copies have the same bits."""
    c, q, table, lengths = setup((29, batch, dh), 2, drafts, 1, group, dh, page, [length, length - 333], dtype=dtype)
    for b, at in ((0, 0.2), (0, 0.37), (0, 0.8), (1, 0.43), (1, 0.97)):  # parts of the sequence
        table[b, int(at * length) // page] = -1
    masks = trees((29, drafts), drafts, 2)
    copy = torch.from_numpy(np.concatenate([[0, 1], rng(29, batch).integers(0, 2, batch - 2)])).cuda()
    got = c.attend(q[copy], table[copy], lengths[copy], tree=gpu_masks(masks)[copy])
    check(got[:2], q, c, table, lengths, masks)
    assert torch.equal(got, got[:2][copy])


@pytest.mark.parametrize("batch,drafts,group,dh,page,length,dtype", LONG_CHUNKS)
def test_every_place_of_long_chunks_counts_once(batch, drafts, group, dh, page, length, dtype):
    """Keys of zeros, so that every weight is 1, and values that are whole numbers: the mean over the places that are seen, of
    exact sums below 2^24.  Rounded are the count's reciprocal, the product with it, and the result."""
    c, q, table, lengths = setup((30, batch, dh), 2, drafts, 1, group, dh, page, [length, length - 333], dtype=dtype, junk=False)
    c.k.view(torch.uint8).zero_()
    c.k_scale.fill_(1.0), c.v_scale.fill_(1.0)
    r = rng(30, batch, dh)
    c.v.copy_(torch.from_numpy(r.integers(-16, 17, tuple(c.v.shape)).astype(np.float32)).cuda())
    for b, at in ((0, 0.2), (0, 0.37), (0, 0.8), (1, 0.43), (1, 0.97)):
        table[b, int(at * length) // page] = -1
    masks = trees((30, drafts), drafts, 2)
    copy = torch.from_numpy(np.concatenate([[0, 1], r.integers(0, 2, batch - 2)])).cuda()
    got = c.attend(q[copy], table[copy], lengths[copy], tree=gpu_masks(masks)[copy])
    assert torch.equal(got, got[:2][copy])
    v = host(c.v.float())[:, 0]
    for b in range(2):
        n, ids = int(lengths[b]), table[b].cpu().numpy()
        place = np.arange(n)
        id_of = ids[place // page]
        rows = np.where((id_of >= 0)[:, None], v[id_of, place % page], 0.0)
        sees = np.concatenate([np.ones((drafts, n - drafts)), masks[b][:, None] >> np.arange(drafts, dtype=np.uint64) & np.uint64(1)], axis=1)
        sees = sees * (id_of >= 0)
        ref = (sees @ rows / sees.sum(axis=1, keepdims=True))[:, None, :]
        assert (np.abs(host(got[b]) - ref) <= np.abs(ref) * (2.0 ** -8 * (dtype == "bf16") + 2.0 ** -22)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,drafts,group,dh,page", [(257, 1, 2, 64, 16), (700, 1, 8, 128, 32), (5000, 1, 1, 16, 16),
                                                        (300, 9, 8, 64, 32), (600, 17, 8, 128, 16), (4161, 2, 2, 48, 64)])
def test_more_sequences_than_are_scanned(batch, drafts, group, dh, page, dtype):
    """Short sequences, one chunk each, have the bits of calls of 64 sequences; long ones among them are cut."""
    heads, long = 2, 3000
    c, _, rows, _ = setup((17, batch, dh), 2, 1, heads, group, dh, page, [long, 256], dtype=dtype)
    r = rng(18, batch)
    lens = r.integers(0, 257, batch)
    which = np.ones(batch, int)
    far = np.array([0, batch // 2, batch - 1])
    lens[far], which[far] = long, 0
    table = rows[torch.from_numpy(which).cuda()].contiguous()
    lengths = torch.from_numpy(lens.astype(np.int32)).cuda()
    q = on_gpu(r.standard_normal((batch, drafts, heads * group, dh)) * 0.7, dtype)
    got = c.attend(q, table, lengths)
    assert torch.equal(got, c.attend(q, table, lengths))
    at = torch.from_numpy(far).cuda()
    check(got[at], q[at], c, table[at], lengths[at])
    near = torch.from_numpy(np.delete(np.arange(batch), far)).cuda()
    for some in near.split(64):
        assert torch.equal(got[some], c.attend(q[some], table[some, :256 // page], lengths[some]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_most_sequences(dtype):
    """2^20 copies of 200, which have the bits of these."""
    r = rng(20)
    lens = r.integers(0, 65, 200)
    c, q, table, lengths = setup((32,), 200, 1, 1, 2, 16, 16, [int(n) for n in lens], dtype=dtype)
    ref = c.attend(q, table, lengths)
    copy = torch.from_numpy(r.integers(0, 200, 1 << 20)).cuda()
    assert torch.equal(c.attend(q[copy], table[copy], lengths[copy]), ref[copy])


def test_the_time_of_many_sequences_grows_as_they_do():
    """Four times the sequences take about four times as long: 16 times when every workgroup looked at every sequence."""
    c, _, rows, _ = setup((19,), 1, 1, 1, 1, 16, 16, [64])
    times = []
    for batch in (8192, 32768):
        table, lengths = rows.expand(batch, -1).contiguous(), torch.full((batch,), 64, dtype=torch.int32, device="cuda")
        q = on_gpu(rng(19, batch).standard_normal((batch, 1, 1, 16)), "bf16")
        for _ in range(5):
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            c.attend(q, table, lengths)
            end.record()
            end.synchronize()
            times.append(start.elapsed_time(end))
    assert min(times[5:]) < 9 * min(times[:5]), times


def test_a_place_that_is_not_finite_and_seen_by_all():
    c, q, table, lengths = setup((5,), 2, 2, 1, 2, 64, 16, [100, 100])
    before = c.attend(q, table, lengths)
    place = 40
    nan = torch.full((1, 1, 64), float("nan"), device="cuda")
    c.write(torch.zeros_like(nan), nan, torch.tensor([int(table[0, place // 16]) * 16 + place % 16], device="cuda"))
    got = c.attend(q, table, lengths)
    assert torch.isnan(got[0]).all() and torch.equal(got[1], before[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drafts,group,dh", [(1, 4, 64), (3, 2, 128), (40, 2, 128), (64, 4, 64), (20, 2, 256)])
@pytest.mark.parametrize("where", ["all", "drafted"])
@pytest.mark.parametrize("code", [0x7C, 0xFC])
def test_infinities_in_a_cache_written_elsewhere(drafts, group, dh, dtype, where, code):
    """An infinite code, which E5M2 has, at a place that all see or one that only some see: no finite element of who sees it as a
    value; as a key NaN, or the result without that place where its logit is minus infinity; nothing of the others changes."""
    c, q, table, lengths = setup((27, drafts, dh), 1, drafts, 1, group, dh, 16, [drafts + 100], fmt="e5m2", dtype=dtype)
    masks = trees((27, drafts), drafts)
    tree = gpu_masks(masks)
    place = 37 if where == "all" else 100 + drafts // 2
    sees = np.array([where == "all" or bool(int(m) >> (drafts // 2) & 1) for m in masks])
    sees = torch.from_numpy(sees).cuda()[:, None].expand(drafts, group)
    page, at = int(table[0, place // 16]), place % 16
    before = c.attend(q, table, lengths, tree=tree)[0]
    check(before[None], q, c, table, lengths, masks)
    kept = c.v.view(torch.uint8)[page, 0, at, 5].clone()
    c.v.view(torch.uint8)[page, 0, at, 5] = code
    got = c.attend(q, table, lengths, tree=tree)[0]
    assert torch.equal(torch.isfinite(got[..., 5]), ~sees)
    other = torch.arange(dh, device="cuda") != 5
    assert torch.equal(got[..., other], before[..., other]) and torch.equal(got[~sees], before[~sees])
    c.v.view(torch.uint8)[page, 0, at, 5] = kept
    c.k.view(torch.uint8)[page, 0, at, 5] = code
    got = c.attend(q, table, lengths, tree=tree)[0]
    assert torch.equal(got[~sees], before[~sees])
    nan = torch.isnan(got).all(dim=-1)
    up = (q[0, :, :, 5] > 0) == (code == 0x7C)  # the logit is plus infinity
    assert nan[sees & up].all() and not torch.isnan(got[~nan]).any()
    if bool((sees & ~nan).any()):  # the sums of `check` over the other places
        keys, values = c.read(table[0].long().repeat_interleave(16) * 16 + torch.arange(16, device="cuda").repeat(table.shape[1]),
                              dtype=torch.float32)
        n, t = int(lengths[0]), drafts
        k, v = keys[:n, 0].double().cpu(), values[:n, 0].double().cpu()
        for i, g in torch.nonzero(sees & ~nan).tolist()[:6]:
            see = [p for p in range(n) if p != place and (p < n - t or int(masks[i]) >> (p - n + t) & 1)]
            w = torch.softmax(k[see] @ q[0, i, g].double().cpu() * dh ** -0.5, dim=0)
            reach = float((k[see].abs() @ q[0, i, g].double().cpu().abs()).max()) * dh ** -0.5
            off = reach * (dh + 8) * 2.0 ** -23 + 2.0 ** -22
            ref, mag = w @ v[see], w @ v[see].abs()
            tol = mag * (2 * off * (1 + off) + 2.0 ** -16 + 2 * (n + 64) * 2.0 ** -23) + ref.abs() * 2.0 ** -8
            assert ((got[i, g].double().cpu() - ref).abs() <= tol).all()


def test_pages_that_are_not_there_are_not_seen():
    c, q, table, lengths = setup((6,), 2, 2, 2, 2, 64, 16, [100, 90])
    table[0, 2], table[1, 0], table[0, 6] = c.pages, -5, 1 << 30
    check(c.attend(q, table, lengths), q, c, table, lengths)
    table[1] = -1
    got = c.attend(q, table, lengths)
    assert (got[1] == 0).all()
    # lengths past the table end with it, negative ones hold nothing
    lengths = torch.tensor([1 << 30, -7], dtype=torch.int32, device="cuda")
    table[0] = torch.arange(table.shape[1], device="cuda")
    c.k.view(torch.uint8).fill_(0x30), c.v.view(torch.uint8).fill_(0x31), c.k_scale.fill_(1.0), c.v_scale.fill_(1.0)
    check(c.attend(q, table, lengths), q, c, table, lengths)


def test_scales_of_all_sizes():
    """Rows that differ by many octaves, and rows of zeros, whose scale is the least."""
    c, q, table, lengths = setup((7,), 1, 1, 1, 4, 64, 16, [80], dtype="f32")
    c.v_scale.copy_(torch.exp2(torch.randint(-60, 60, c.v_scale.shape, device="cuda").float()))
    c.k_scale.copy_(torch.exp2(torch.randint(-30, 0, c.k_scale.shape, device="cuda").float()))
    check(c.attend(q, table, lengths), q, c, table, lengths)
    zero = torch.zeros(5, 1, 64, device="cuda")
    c.write(zero, zero, int(table[0, 1]) * 16 + torch.arange(5, device="cuda"))
    check(c.attend(q, table, lengths), q, c, table, lengths)


@pytest.mark.parametrize("drafts,dtype", [(1, "bf16"), (1, "f32"), (40, "bf16")])
def test_scales_between_powers_of_two(drafts, dtype):
    """Of a cache written elsewhere: reading multiplies by them, attention takes the power of two."""
    c, q, table, lengths = setup((28, drafts), 1, drafts, 1, 4, 64, 16, [drafts + 70], dtype=dtype, junk=False)
    ref, slots = c.attend(q, table, lengths), torch.arange(c.pages * 16, device="cuda")
    k, v = c.read(slots, dtype=torch.float32)
    for t in (c.k_scale, c.v_scale):
        t.mul_(1.5)
    for got, x in zip(c.read(slots, dtype=torch.float32), (k, v)):
        assert torch.equal(got, x * 1.5)  # codes of 4 bits: exact
    assert torch.equal(c.attend(q, table, lengths), ref)


def test_logits_far_apart():
    """Weights from 1 to none, and logits in the thousands."""
    c, q, table, lengths = setup((8,), 1, 1, 2, 4, 128, 16, [300], dtype="f32")
    for factor in (30.0, 1000.0):
        check(c.attend(q * factor, table, lengths), q * factor, c, table, lengths)
    check(c.attend(q, table, lengths, scale=0.03), q, c, table, lengths, scale=0.03)


@pytest.mark.parametrize("size", [0.5, 30.0])
@pytest.mark.parametrize("drafts,group,dh,dtype", [
    (1, 1, 64, "f32"), (1, 8, 128, "f32"), (1, 16, 256, "f32"), (5, 8, 64, "f32"), (8, 8, 128, "f32"), (20, 8, 128, "f32"),
    (3, 8, 256, "f32"), (2, 4, 32, "f32"), (1, 8, 128, "bf16"), (5, 8, 64, "bf16"), (8, 8, 128, "bf16"), (4, 8, 256, "bf16"),
    (9, 8, 64, "bf16"), (9, 8, 128, "bf16"), (20, 8, 64, "bf16"), (20, 8, 128, "bf16")])
def test_weights_are_held_to_their_bits(drafts, group, dh, dtype, size):
    """32 places whose keys and values are the unit vectors, so that a result is its row's weights: within the bound of the parts
    that queries and weights are held in, which one part less exceeds."""
    n, scale, heads, batch = 32, 0.125, 2, 40
    c = Fp8Cache.empty(2, heads, 16, dh)
    unit = torch.eye(n, dh, device="cuda")[:, None].expand(n, heads, dh)
    c.write(unit, unit, torch.arange(n, device="cuda"))
    assert (c.k_scale[:, :, :] == 2.0 ** -8).all()  # 1 / 448 and up: exact
    table = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda").expand(batch, 2).contiguous()
    lengths = torch.full((batch,), n, dtype=torch.int32, device="cuda")
    q = on_gpu(rng(31, drafts, dh).uniform(-1, 1, (batch, drafts, heads * group, dh)) * size / scale, dtype)
    got = host(c.attend(q, table, lengths, scale=scale)).reshape(-1, dh)
    seen = np.broadcast_to(n - drafts + 1 + np.arange(drafts)[None, :, None], q.shape[:3]).reshape(-1)
    ref, reach = oracle.weights(host(q).reshape(-1, dh), seen, scale)
    assert (got[ref == 0] == 0).all()
    off = oracle.weights_off(reach, bf16=dtype == "bf16")[:, None]
    low, high = (on_gpu(ref * (1 + sign * off), "f32") for sign in (-1, 1))
    if dtype == "bf16":  # the result's own rounding
        low, high = low.bfloat16(), high.bfloat16()
    assert ((host(low) <= got) & (got <= host(high))).all(), float(np.abs(got / np.where(ref > 0, ref, 1) - 1)[ref > 0].max())


@pytest.mark.parametrize("batch,drafts,group,dh,length", [(512, 1, 4, 64, 35200), (256, 16, 8, 128, 8960), (256, 3, 8, 256, 17920)])
def test_many_small_weights_beside_a_large_one(batch, drafts, group, dh, length):
    """Copies of a sequence whose first place has the weight 1 and whose others have e^-16.661 = 0.4875 2^-23 each, which are
    lost beside it one by one, in chunks of 140 steps to a wave.  Values are 1, so a result is the sum of the weights over itself.
    At each step the numerator adds 32 places to 1, in eights (2^-24 off each), the sum of the first place's lane the 8 that it
    holds (2^-24).  Lost one by one, these 8 were 7.8 2^-24.  2^-20: all other roundings."""
    c = Fp8Cache.empty(-(-length // 64), 1, 64, dh)
    c.k_scale.fill_(1.0), c.v_scale.fill_(1.0)
    c.k[..., 0].view(torch.uint8).fill_(0x38), c.v.view(torch.uint8).fill_(0x38)  # 1
    c.k.view(torch.uint8)[0, 0, 0, 0] = 0
    q = torch.zeros(batch, drafts, group, dh, device="cuda")
    q[..., 0] = -16.661
    table = torch.arange(c.pages, dtype=torch.int32, device="cuda").expand(batch, -1).contiguous()
    lengths = torch.full((batch,), length, dtype=torch.int32, device="cuda")
    got = c.attend(q, table, lengths, scale=1.0)
    off = float((got.double() - 1).abs().max())
    assert off <= 140 * 5 * 2.0 ** -24 + 2.0 ** -20


def test_queries_and_results_of_any_strides():
    c, q, table, lengths = setup((9,), 3, 4, 2, 3, 64, 16, [50, 9, 80])
    ref = c.attend(q, table, lengths)
    room = torch.full((4, 6, 3, 67), 7.0, dtype=torch.bfloat16, device="cuda")  # tokens, heads, batch
    qs = room[..., 2:66].permute(2, 0, 1, 3)
    qs.copy_(q)
    wide = torch.full((3, table.shape[1] + 3), 9, dtype=torch.int32, device="cuda")
    wide[:, 1:1 + table.shape[1]] = table
    out_room = torch.full((6, 3, 4, 65), 7.0, dtype=torch.bfloat16, device="cuda")
    out = out_room[..., :64].permute(1, 2, 0, 3)
    got = c.attend(qs, wide[:, 1:1 + table.shape[1]], lengths, out=out)
    assert got is out and torch.equal(out, ref) and (out_room[..., 64] == 7.0).all()
    one = q[:1].expand(3, -1, -1, -1)  # the same queries for all
    assert torch.equal(c.attend(one, table, lengths), c.attend(one.contiguous(), table, lengths))
    masks = gpu_masks(trees((9,), 4))
    assert torch.equal(c.attend(q, table, lengths, tree=masks), c.attend(q, table, lengths, tree=masks.expand(3, 4)))


def test_a_chain_is_a_tree_of_one_branch():
    c, q, table, lengths = setup((10,), 2, 9, 2, 4, 128, 16, [500, 30])
    masks = gpu_masks((np.uint64(2) << np.arange(9, dtype=np.uint64)) - np.uint64(1))
    assert torch.equal(c.attend(q, table, lengths), c.attend(q, table, lengths, tree=masks))


def test_refusals():
    c, q, table, lengths = setup((13,), 2, 3, 2, 2, 64, 16, [50, 40])
    k = torch.zeros(4, 2, 64, device="cuda")
    slots = torch.arange(4, device="cuda")
    bad = [
        lambda: Fp8Cache(c.k.float(), c.k_scale, c.v, c.v_scale), lambda: Fp8Cache(c.k[0], c.k_scale, c.v, c.v_scale),
        lambda: Fp8Cache(c.k, c.k_scale, c.v[1:], c.v_scale), lambda: Fp8Cache(c.k, c.k_scale[:, :1], c.v, c.v_scale),
        lambda: Fp8Cache(c.k, c.k_scale.double(), c.v, c.v_scale), lambda: Fp8Cache.empty(2, 2, 48, 64),
        lambda: Fp8Cache.empty(2, 2, 16, 72), lambda: Fp8Cache.empty(2, 2, 16, 64, fmt="int8"),
        lambda: Fp8Cache(c.k[:, :, :, :32], c.k_scale, c.v[:, :, :, :32], c.v_scale),
        lambda: Fp8Cache(c.k[::2], c.k_scale[::2], c.v[::2], c.v_scale[::2].clone()) and
        Fp8Cache(c.k[:2], c.k_scale[:2], c.v[:4:2], c.v_scale[:4:2]),
        lambda: c.write(k, k[:3], slots), lambda: c.write(k, k.bfloat16(), slots), lambda: c.write(k.half(), k.half(), slots),
        lambda: c.write(k, k, slots.int()), lambda: c.write(k, k, slots[:3]), lambda: c.write(k, k, slots.cpu()),
        lambda: c.write(k.clone().requires_grad_(), k, slots), lambda: c.write(k[:, :, :32], k[:, :, :32], slots),
        lambda: c.write(k.transpose(1, 2).contiguous().transpose(1, 2), k, slots), lambda: c.write(k[0], k[0], slots),
        lambda: c.read(slots, dtype=torch.float16), lambda: c.read(slots.int()), lambda: c.read(slots[None]),
        lambda: c.read(slots, out=(k, k[:3])), lambda: c.attend(q.half(), table, lengths), lambda: c.attend(q[0], table, lengths),
        lambda: c.attend(q[:, :, :3], table, lengths), lambda: c.attend(q[:, :, :, :32], table, lengths),
        lambda: c.attend(q[:, :0], table, lengths), lambda: c.attend(q.expand(2, 3, 4, 64).repeat(1, 22, 1, 1), table, lengths),
        lambda: c.attend(q, table.long(), lengths), lambda: c.attend(q, table[:1], lengths), lambda: c.attend(q, table.t(), lengths),
        lambda: c.attend(q, table, lengths.long()), lambda: c.attend(q, table, lengths[:1]), lambda: c.attend(q, table, lengths.cpu()),
        lambda: c.attend(q, table, lengths, tree=torch.ones(2, device="cuda", dtype=torch.int64)),
        lambda: c.attend(q, table, lengths, tree=torch.ones(3, device="cuda", dtype=torch.int32)),
        lambda: c.attend(q.clone().requires_grad_(), table, lengths), lambda: c.attend(q, table, lengths, out=q.float()),
        lambda: c.attend(q, table, lengths, out=q[:, :, :2])]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("call", i)
    from paper_2602_18851_amd import SpectralError
    with pytest.raises(SpectralError):
        c.read(slots, out=(k[:1].expand(4, 2, 64), k))
    with pytest.raises(SpectralError):
        c.attend(q, table, lengths, out=q[:1].expand(2, -1, -1, -1))
    for scale in (0.0, -1.0, float("nan")):
        with pytest.raises(SpectralError):
            c.attend(q, table, lengths, scale=scale)
    assert c.attend(q[:0], table[:0], lengths[:0]).shape == (0, 3, 4, 64)
    c.write(k[:0], k[:0], slots[:0])
    assert c.read(slots[:0])[0].shape == (0, 2, 64)


@pytest.mark.parametrize("which", ["k", "k_scale", "v", "v_scale"])
def test_a_cache_that_requires_gradients_is_refused(which):
    c, q, table, lengths = setup((25,), 2, 3, 2, 2, 64, 16, [50, 40])
    ref = c.attend(q, table, lengths)
    k, slots = torch.ones(4, 2, 64, device="cuda"), torch.arange(4, device="cuda") + c.pages * 16  # padding
    getattr(c, which).requires_grad_()
    for call in (lambda: c.write(k, k, slots), lambda: c.read(slots), lambda: c.attend(q, table, lengths)):
        with pytest.raises(ValueError, match="gradients"):
            call()
        with torch.no_grad():
            call()
    with torch.no_grad():
        assert torch.equal(c.attend(q, table, lengths), ref)


def test_results_that_require_gradients_are_refused():
    c, q, table, lengths = setup((26,), 2, 3, 2, 2, 64, 16, [50, 40], dtype="f32")
    out = torch.zeros_like(q).requires_grad_()
    with pytest.raises(ValueError, match="gradients"):
        c.attend(q, table, lengths, out=out)
    assert (out == 0).all()
    with torch.no_grad():
        assert torch.equal(c.attend(q, table, lengths, out=out), c.attend(q, table, lengths))
    k, slots = torch.zeros(4, 2, 64, device="cuda"), torch.arange(4, device="cuda")
    with pytest.raises(ValueError, match="gradients"):
        c.read(slots, out=(k, k.clone().requires_grad_()))


# ------------------------------------------------------- streams and graphs


def test_calls_replay_from_a_graph():
    """A generated token after another from one graph: its slot, lengths and inputs change between replays."""
    heads, group, dh, page = 2, 4, 64, 16
    c, q, table, lengths = setup((20,), 3, 1, heads, group, dh, page, [700, 40, 16])
    eager, _, _, _ = setup((20,), 3, 1, heads, group, dh, page, [700, 40, 16])
    k, v = (torch.zeros(3, heads, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slots = torch.full((3,), -1, dtype=torch.int64, device="cuda")
    out, ws = torch.empty_like(q), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    c.write(k, v, slots)
    c.attend(q, table, lengths, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.write(k, v, slots)
        c.attend(q, table, lengths, out=out, workspace=ws)
    r = rng(21)
    last = [int(n) for n in lengths]
    for rep in range(4):
        at = []
        for b in range(3):  # the token takes the place of the last one but rep
            place = last[b] - 1 - rep
            at.append(int(table[b, place // page]) * page + place % page)
        slots.copy_(torch.tensor(at))
        lengths.copy_(torch.tensor([n - rep for n in last], dtype=torch.int32))
        for t in (k, v, q):
            t.copy_(on_gpu(r.standard_normal(t.shape), "bf16"))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        eager.write(k, v, slots)
        assert torch.equal(out, eager.attend(q, table, lengths))
        assert torch.equal(c.k.view(torch.uint8), eager.k.view(torch.uint8))


def test_many_sequences_replay_from_a_graph():
    """Their shares are formed anew at every replay, from the lengths of then."""
    c, _, rows, _ = setup((24,), 1, 1, 2, 2, 64, 16, [2000])
    r = rng(24)
    table = rows.expand(300, -1).contiguous()
    lengths = torch.zeros(300, dtype=torch.int32, device="cuda")
    q = on_gpu(r.standard_normal((300, 1, 4, 64)), "bf16")
    out, ws = torch.empty_like(q), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    c.attend(q, table, lengths, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attend(q, table, lengths, out=out, workspace=ws)
    for rep in range(4):
        lengths.copy_(torch.from_numpy(np.where(r.random(300) < 0.05 * rep, 2000, r.integers(0, 300, 300)).astype(np.int32)))
        ws.fill_(0xA5)
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, c.attend(q, table, lengths))


def test_two_streams_at_once():
    sets = [setup((22, i), 2, 2, 2, 4, 128, 32, [3000, 1500]) for i in range(2)]
    refs = [c.attend(*rest) for c, *rest in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(sets[i][0].attend(*sets[i][1:]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, refs[i]) for g in got[i])


# ------------------------------------------------------------------ all together


def test_a_prompt_and_drafted_tokens_through_a_layer():
    """An attention layer in 8 bits: projections as 8-bit integers, rotary positions, the cache, and a tree of drafted tokens,
    against the same steps with the oracle's attention."""
    d, heads, group, dh, page = 256, 2, 2, 64, 16
    r = rng(30)
    hq = heads * group
    w = {n: quantize_int8(on_gpu(r.standard_normal((rows, d)) * d ** -0.5, "bf16"))
         for n, rows in (("q", hq * dh), ("k", heads * dh), ("v", heads * dh))}
    wo = quantize_int8(on_gpu(r.standard_normal((d, hq * dh)) * d ** -0.5, "bf16"))
    rot = Rotary(dh)
    c = Fp8Cache.empty(8, heads, page, dh)
    table = torch.tensor([[5, 2, 7, 0, 1, 3]], dtype=torch.int32, device="cuda")

    def step(x, first, tree):
        n = x.shape[0]
        a = quantize_int8(x)
        q, k, v = (matmul_int8(a, w[name]).view(n, -1, dh) for name in "qkv")
        depth = torch.arange(first, first + n, device="cuda") if tree is None else \
            first - 1 + torch.tensor([bin(int(m)).count("1") for m in tree], device="cuda")
        q, k = rot.apply(q, k, positions=depth)
        place = torch.arange(first, first + n, device="cuda")
        c.write(k, v, table[0].long()[place // page] * page + place % page)
        lengths = torch.tensor([first + n], dtype=torch.int32, device="cuda")
        o = c.attend(q[None], table, lengths, tree=None if tree is None else gpu_masks(tree))
        check(o, q[None], c, table, lengths, tree)
        y = matmul_int8(o.view(n, hq * dh), wo)
        assert torch.isfinite(y).all() and y.shape == (n, d)
        return y

    for i in range(0, 64, 32):  # a prompt in pieces of chains
        step(on_gpu(r.standard_normal((32, d)), "bf16"), i, None)
    step(on_gpu(r.standard_normal((1, d)), "bf16"), 64, None)
    step(on_gpu(r.standard_normal((10, d)), "bf16"), 65, trees((30,), 10))
