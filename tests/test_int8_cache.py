"""8-bit integers and the 8-bit cache without a GPU: the oracle against hand-made values, and every refusal of the C
entry points, which come before anything touches the device."""

import math

import numpy as np
import pytest

from oracle import cache as cache_oracle, int8_rows
from paper_2602_18851_amd import spectral as sp
from test_abi import lib  # noqa: F401


def refused(code, call, *args, **kw):
    with pytest.raises(sp.SpectralError) as e:
        call(*args, **kw)
    assert e.value.code == code and sp.spectral_last_error()


# ------------------------------------------------------------------ oracle


def test_oracle_quantises_rows():
    codes, scale = int8_rows.quantize([[127.0, 0.5, 1.5, -2.5, -127.0], [0.0] * 5, [math.inf, 1, 2, 3, 4]])
    assert codes.tolist() == [[127, 0, 2, -2, -127], [0] * 5, [0] * 5]
    assert scale[0] == 1.0 and scale[1] == 2.0 ** -126 and math.isnan(scale[2])
    # half of the largest is next to a tie, on the side that the scale's rounding decides
    codes, scale = int8_rows.quantize([[1.0, 0.5], [3.0, 1.5], [5.0, 2.5]])
    for r, top in enumerate((1.0, 3.0, 5.0)):
        assert scale[r] == np.float32(top / 127)
        assert codes[r, 1] == (63 if scale[r] > top / 127 else 64)


def test_oracle_sees_places():
    table = [2, 0, -1]
    assert cache_oracle.seen(5, 2, 0, None, table, 4, 3) == [0, 1, 2, 3]
    assert cache_oracle.seen(5, 2, 1, None, table, 4, 3) == [0, 1, 2, 3, 4]
    assert cache_oracle.seen(5, 2, 1, 0b10, table, 4, 3) == [0, 1, 2, 4]
    assert cache_oracle.seen(12, 1, 0, None, table, 4, 3) == list(range(8))  # the last page is not there
    assert cache_oracle.seen(99, 1, 0, None, table, 4, 3) == list(range(8))
    assert cache_oracle.seen(1, 3, 0, None, table, 4, 3) == [] and cache_oracle.seen(1, 3, 2, None, table, 4, 3) == [0]
    assert cache_oracle.seen(0, 1, 0, None, table, 4, 3) == []


def test_oracle_attends():
    k = np.zeros((1, 1, 4, 2))
    v = np.arange(8.0).reshape(1, 1, 4, 2)
    k[0, 0, :, 0] = np.log([1.0, 2.0, 3.0, 4.0])
    out, _, _ = cache_oracle.attend([[[[1.0, 0.0]]]], k, v, [[0]], [4], scale=1.0)
    np.testing.assert_allclose(out[0, 0, 0], (np.arange(1, 5) / 10) @ v[0, 0])


def test_oracle_weighs():
    w, reach = cache_oracle.weights([[0.0, math.log(3.0), 7.0], [1.0, 2.0, 3.0]], [2, 1], 1.0)
    np.testing.assert_allclose(w, [[0.25, 0.75, 0.0], [1.0, 0.0, 0.0]])
    np.testing.assert_allclose(reach, [math.log(3.0), 1.0])


def nearest_bf16(x):
    """float32 to bf16 and back, ties to even."""
    u = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + (u >> np.uint64(16) & np.uint64(1))) & np.uint64(0xFFFF0000)).astype(np.uint32).view(np.float32)


def in_parts(x, n):
    """x as the sum of its n nearest bf16 parts."""
    rest, total = np.asarray(x, dtype=np.float32), np.zeros(np.shape(x))
    for _ in range(n):
        part = nearest_bf16(rest)
        rest = (rest - part).astype(np.float32)
        total += part
    return total


def weighed(q, n, scale, q_parts, p_parts):
    """The steps of the attention kernels for those weights: float32 between them, q and the weights in bf16 parts."""
    f = np.float32
    s = in_parts(q, q_parts).astype(f)
    c = f(f(scale) * f(1.44269504088896340736))
    there = np.arange(q.shape[1]) < n[:, None]
    top = np.where(there, s, f(-np.inf)).max(axis=1, keepdims=True)
    x = (s.astype(np.float64) * c - (top * c).astype(np.float64)).astype(f)
    p = np.where(there, np.exp2(x.astype(np.float64)).astype(f), f(0))
    total = np.zeros(q.shape[0], dtype=f)
    for j in range(q.shape[1]):
        total += p[:, j]
    return in_parts(p, p_parts).astype(f) * (f(1) / total)[:, None]


@pytest.mark.parametrize("size", [0.5, 30.0])
def test_the_bound_of_weights_tells_their_parts_apart(size):
    """float32: three parts of queries and of weights are within it, two of the queries are not, nor are two of the weights
    where logits are small.  bf16: two parts of the weights are, one is not."""
    r = np.random.default_rng(7)
    n, scale = r.integers(2, 33, 400), 0.125
    q = (r.uniform(-1, 1, (400, 64)) * size / scale).astype(np.float32)
    ref, reach = cache_oracle.weights(q, n, scale)

    def off(q_parts, p_parts, q=q, ref=ref):
        with np.errstate(divide="ignore", invalid="ignore"):
            return np.where(ref > 0, np.abs(weighed(q, n, scale, q_parts, p_parts) / ref - 1), 0.0)
    bound = cache_oracle.weights_off(reach)[:, None]
    assert (off(3, 3) <= bound).all()
    assert (off(2, 3) > bound).any()
    if size < 1:
        assert (off(3, 2) > bound).any()
    q = nearest_bf16(q)
    ref, reach = cache_oracle.weights(q, n, scale)
    bound = cache_oracle.weights_off(reach, bf16=True)[:, None]
    assert (off(1, 2, q, ref) <= bound).all() and (off(1, 1, q, ref) > bound).any()


# ------------------------------------------------------------------ refusals of the quantiser and the products


@pytest.mark.parametrize("code,kw", [
    (sp.SN_EDTYPE, dict(dtype=sp.SN_I8)), (sp.SN_EDTYPE, dict(dtype=9)), (sp.SN_EINVAL, dict(rows=-1)),
    (sp.SN_EINVAL, dict(cols=-1)), (sp.SN_EINVAL, dict(ld_x=39)), (sp.SN_EINVAL, dict(ld=32)), (sp.SN_EINVAL, dict(ld=50)),
    (sp.SN_EINVAL, dict(codes=40)), (sp.SN_EINVAL, dict(rows=(1 << 40) + 1)), (sp.SN_EINVAL, dict(ld_x=(1 << 40) + 1)),
    (sp.SN_ENULL, dict(x=0)), (sp.SN_ENULL, dict(codes=0)), (sp.SN_ENULL, dict(scale=0)), (sp.SN_EINVAL, dict(x=18)),
    (sp.SN_EINVAL, dict(scale=18))])
def test_quantiser_refuses(lib, code, kw):  # noqa: F811
    base = dict(x=16, rows=3, cols=40, ld_x=40, dtype=sp.SN_F32, codes=32, ld=48, scale=64)
    base.update(kw)
    refused(code, sp.spectral_quantize_int8, **base)


def test_quantiser_of_nothing(lib):  # noqa: F811
    sp.spectral_quantize_int8(0, 0, 40, 0, sp.SN_F32, 0, 48, 0)


def desc(**kw):
    base = dict(m=300, n=200, k=100, a_type=sp.SN_I8, c_type=sp.SN_BF16, ld_a=0, ld_b=0, ld_c=0, sa_row=0, sb_row=0)
    base.update(kw)
    return sp.sn_matmul_int8(**base)


@pytest.mark.parametrize("code,kw", [
    (sp.SN_EDTYPE, dict(a_type=sp.SN_E4M3)), (sp.SN_EDTYPE, dict(a_type=-1)), (sp.SN_EDTYPE, dict(c_type=sp.SN_I8)),
    (sp.SN_EINVAL, dict(m=-1)), (sp.SN_EINVAL, dict(n=-1)), (sp.SN_EINVAL, dict(k=-1)), (sp.SN_EINVAL, dict(k=1 << 17)),
    (sp.SN_EINVAL, dict(m=(1 << 34) + 1)), (sp.SN_EINVAL, dict(m=1 << 20, n=1 << 20)), (sp.SN_EINVAL, dict(ld_a=96)),
    (sp.SN_EINVAL, dict(ld_a=120)), (sp.SN_EINVAL, dict(ld_b=96)), (sp.SN_EINVAL, dict(ld_b=120)),
    (sp.SN_EINVAL, dict(ld_b=1 << 22)), (sp.SN_EINVAL, dict(ld_c=199)), (sp.SN_EINVAL, dict(sa_row=-1)),
    (sp.SN_EINVAL, dict(sb_row=(1 << 40) + 1)), (sp.SN_EINVAL, dict(a_type=sp.SN_F32, ld_a=99))])
def test_products_refuse_bad_descriptions(lib, code, kw):  # noqa: F811
    refused(code, sp.spectral_matmul_int8_workspace_bytes, desc(**kw))
    refused(code, sp.spectral_matmul_int8_kernel, desc(**kw))
    refused(code, sp.spectral_matmul_int8, desc(**kw), 256, 256, 256, 256, 256, 256, 1 << 40)


@pytest.mark.parametrize("code,kw,args", [
    (sp.SN_ENULL, {}, dict(a=0)), (sp.SN_ENULL, {}, dict(sa=0)), (sp.SN_ENULL, {}, dict(b=0)), (sp.SN_ENULL, {}, dict(sb=0)),
    (sp.SN_ENULL, {}, dict(c=0)), (sp.SN_EINVAL, {}, dict(a=264)), (sp.SN_EINVAL, {}, dict(b=264)),
    (sp.SN_EINVAL, {}, dict(sa=258)), (sp.SN_EINVAL, {}, dict(sb=258)), (sp.SN_EINVAL, {}, dict(c=257)),
    (sp.SN_EINVAL, dict(a_type=sp.SN_F32), dict(a=258)), (sp.SN_ENULL, dict(a_type=sp.SN_F32), dict(workspace=0)),
    (sp.SN_EINVAL, dict(a_type=sp.SN_F32), dict(workspace_bytes=100)),
    (sp.SN_EINVAL, dict(a_type=sp.SN_F32), dict(workspace=264))])
def test_products_refuse_bad_pointers(lib, code, kw, args):  # noqa: F811
    base = dict(a=256, sa=256, b=256, sb=256, c=256, workspace=256, workspace_bytes=1 << 40)
    base.update(args)
    refused(code, sp.spectral_matmul_int8, desc(**kw), **base)


def test_products_of_nothing(lib):  # noqa: F811
    for kw in (dict(m=0), dict(n=0)):
        sp.spectral_matmul_int8(desc(**kw), 0, 0, 0, 0, 0, 0, 0)
        assert sp.spectral_matmul_int8_kernel(desc(**kw)) == ("none", 0, 0, 0)


def test_rows_of_the_kernel_for_few(lib):  # noqa: F811
    """33 to 48 rows never run it; the rows on either side do somewhere."""
    def ways(m):
        return {sp.spectral_matmul_int8_kernel(desc(m=m, n=n, k=k, c_type=c))[0] for n in (1, 500, 8192, 100000, 1 << 27)
                for k in (1, 128, 1000, 1024, 1025, 8192, 131071) for c in (sp.SN_F32, sp.SN_BF16)}
    for m in (1, 16, 17, 32, 49, 64):
        assert "few_rows" in ways(m), m
    for m in (33, 40, 48, 65):
        assert "few_rows" not in ways(m), m


# ------------------------------------------------------------------ refusals of the cache


def cache(**kw):
    base = dict(k=256, k_scale=256, v=256, v_scale=256, pages=10, heads=4, page=16, head_dim=64, format=sp.SN_E4M3,
                code_page=0, scale_page=0)
    base.update(kw)
    return sp.sn_cache(**base)


BAD_CACHES = [
    (sp.SN_EDTYPE, dict(format=sp.SN_F32)), (sp.SN_EINVAL, dict(pages=-1)), (sp.SN_EINVAL, dict(pages=1 << 31)),
    (sp.SN_EINVAL, dict(heads=0)), (sp.SN_EINVAL, dict(heads=65537)), (sp.SN_EINVAL, dict(page=8)),
    (sp.SN_EINVAL, dict(page=48)), (sp.SN_EINVAL, dict(page=1 << 17)), (sp.SN_EINVAL, dict(heads=32768, page=65536)), (sp.SN_EINVAL, dict(head_dim=0)),
    (sp.SN_EINVAL, dict(head_dim=72)), (sp.SN_EINVAL, dict(head_dim=272)), (sp.SN_EINVAL, dict(code_page=4080)),
    (sp.SN_EINVAL, dict(code_page=4104)), (sp.SN_EINVAL, dict(scale_page=60)), (sp.SN_EINVAL, dict(scale_page=66)),
    (sp.SN_EINVAL, dict(k=264)), (sp.SN_EINVAL, dict(v=264)), (sp.SN_EINVAL, dict(k_scale=260)),
    (sp.SN_EINVAL, dict(v_scale=260))]
NO_MEMORY = [(sp.SN_ENULL, dict(k=0)), (sp.SN_ENULL, dict(v=0)), (sp.SN_ENULL, dict(k_scale=0)), (sp.SN_ENULL, dict(v_scale=0))]


def rows(call, c=None, **kw):
    base = dict(cache=c or cache(), dtype=sp.SN_BF16, tokens=5, k=256, k_token=256, k_head=64, v=256, v_token=256, v_head=64,
                slots=256)
    base.update(kw)
    call(**base)


@pytest.mark.parametrize("call", [sp.spectral_cache_write, sp.spectral_cache_read])
@pytest.mark.parametrize("code,kw", BAD_CACHES + NO_MEMORY)
def test_bad_caches_are_refused(lib, call, code, kw):  # noqa: F811
    refused(code, rows, call, cache(**kw))


@pytest.mark.parametrize("call", [sp.spectral_cache_write, sp.spectral_cache_read])
@pytest.mark.parametrize("code,kw", [
    (sp.SN_EDTYPE, dict(dtype=sp.SN_E4M3)), (sp.SN_EINVAL, dict(tokens=-1)), (sp.SN_EINVAL, dict(tokens=1 << 29)),
    (sp.SN_EINVAL, dict(k_token=-1)), (sp.SN_EINVAL, dict(v_head=-64)), (sp.SN_EINVAL, dict(k_head=(1 << 40) + 1)),
    (sp.SN_EINVAL, dict(k=257)), (sp.SN_EINVAL, dict(v=257)), (sp.SN_EINVAL, dict(slots=260)), (sp.SN_ENULL, dict(k=0)),
    (sp.SN_ENULL, dict(v=0)), (sp.SN_ENULL, dict(slots=0))])
def test_rows_are_refused(lib, call, code, kw):  # noqa: F811
    refused(code, rows, call, **kw)


@pytest.mark.parametrize("kw", [dict(k_head=63), dict(k_token=0), dict(v_token=255), dict(v_head=0), dict(k_token=64, k_head=319)])
def test_overlapping_results_are_refused(lib, kw):  # noqa: F811
    refused(sp.SN_EINVAL, rows, sp.spectral_cache_read, **kw)


def test_rows_of_nothing(lib):  # noqa: F811
    for call in (sp.spectral_cache_write, sp.spectral_cache_read):
        rows(call, cache(k=0, v=0, k_scale=0, v_scale=0), tokens=0, k=0, v=0, slots=0)


def attend(**kw):
    base = dict(dtype=sp.SN_BF16, batch=3, drafts=2, q_heads=8, table_cols=9, scale=0.125, q_batch=1024, q_draft=512, q_head=64,
                out_batch=1024, out_draft=512, out_head=64, table_ld=0, mask_batch=0)
    base.update(kw)
    return sp.sn_attend(**base)


BAD_CALLS = [
    (sp.SN_EDTYPE, dict(dtype=sp.SN_E4M3)), (sp.SN_EINVAL, dict(batch=-1)), (sp.SN_EINVAL, dict(batch=(1 << 20) + 1)),
    (sp.SN_EINVAL, dict(drafts=0)), (sp.SN_EINVAL, dict(drafts=65)), (sp.SN_EINVAL, dict(q_heads=0)),
    (sp.SN_EINVAL, dict(q_heads=6)), (sp.SN_EINVAL, dict(q_heads=1 << 17)), (sp.SN_EINVAL, dict(table_cols=-1)),
    (sp.SN_EINVAL, dict(table_cols=(1 << 27) - 2)), (sp.SN_EINVAL, dict(scale=0.0)), (sp.SN_EINVAL, dict(scale=-1.0)),
    (sp.SN_EINVAL, dict(scale=math.nan)), (sp.SN_EINVAL, dict(scale=math.inf)), (sp.SN_EINVAL, dict(scale=3e38)),
    (sp.SN_EINVAL, dict(table_cols=1 << 26, batch=16)), (sp.SN_EINVAL, dict(q_batch=-1)),
    (sp.SN_EINVAL, dict(q_head=(1 << 40) + 1)), (sp.SN_EINVAL, dict(out_head=63)), (sp.SN_EINVAL, dict(out_draft=0)),
    (sp.SN_EINVAL, dict(out_batch=512)), (sp.SN_EINVAL, dict(out_draft=64)), (sp.SN_EINVAL, dict(table_ld=-1)),
    (sp.SN_EINVAL, dict(mask_batch=-1)), (sp.SN_EINVAL, dict(batch=1 << 20, q_heads=64, out_draft=4096, out_batch=8192))]


@pytest.mark.parametrize("code,kw", BAD_CALLS)
def test_attention_refuses_bad_descriptions(lib, code, kw):  # noqa: F811
    refused(code, sp.spectral_cache_attend_workspace_bytes, cache(), attend(**kw))
    refused(code, sp.spectral_cache_attend, cache(), attend(**kw), 256, 256, 256, 256, 256, 256, 1 << 40)


@pytest.mark.parametrize("code,kw", BAD_CACHES + NO_MEMORY + [(sp.SN_EINVAL, dict(pages=0))])
def test_attention_refuses_bad_caches(lib, code, kw):  # noqa: F811
    refused(code, sp.spectral_cache_attend, cache(**kw), attend(), 256, 256, 256, 256, 256, 256, 1 << 40)


@pytest.mark.parametrize("code,kw", [
    (sp.SN_ENULL, dict(q=0)), (sp.SN_ENULL, dict(table=0)), (sp.SN_ENULL, dict(lengths=0)), (sp.SN_ENULL, dict(out=0)),
    (sp.SN_ENULL, dict(workspace=0)), (sp.SN_EINVAL, dict(workspace_bytes=8)), (sp.SN_EINVAL, dict(workspace=260)),
    (sp.SN_EINVAL, dict(q=257)), (sp.SN_EINVAL, dict(out=257)), (sp.SN_EINVAL, dict(table=258)), (sp.SN_EINVAL, dict(lengths=258)),
    (sp.SN_EINVAL, dict(masks=260))])
def test_attention_refuses_bad_pointers(lib, code, kw):  # noqa: F811
    base = dict(q=256, table=256, lengths=256, masks=256, out=256, workspace=256, workspace_bytes=1 << 40)
    base.update(kw)
    refused(code, sp.spectral_cache_attend, cache(), attend(table_cols=900), **base)


def test_attention_of_nothing(lib):  # noqa: F811
    sp.spectral_cache_attend(cache(k=0, v=0, k_scale=0, v_scale=0, pages=0), attend(batch=0), 0, 0, 0, 0, 0, 0, 0)


def test_attention_workspace_is_bounded(lib):  # noqa: F811
    """A short table needs none; a long one as much as the largest number of workgroups writes."""
    assert sp.spectral_cache_attend_workspace_bytes(cache(), attend(table_cols=1)) == 0
    far = sp.spectral_cache_attend_workspace_bytes(cache(), attend(table_cols=1 << 20))
    assert 0 < far < 1 << 28


def test_many_sequences_have_a_plan_in_the_workspace(lib):  # noqa: F811
    """Above 256 sequences the shares are found once, in 4 bytes for each sequence and 4 more, not by every workgroup."""
    need = {b: sp.spectral_cache_attend_workspace_bytes(cache(), attend(batch=b, drafts=1, table_cols=1)) for b in (256, 257, 1 << 20)}
    assert need == {256: 0, 257: 258 * 4 + 248, 1 << 20: 4 * (1 << 20) + 256}


def test_python_refuses_tensors_of_the_host(lib):  # noqa: F811
    import torch

    from paper_2602_18851_amd import Fp8Cache, Int8Matrix, matmul_int8, quantize_int8

    with pytest.raises(ValueError):
        quantize_int8(torch.zeros(3, 4))
    with pytest.raises(ValueError):
        Int8Matrix(torch.zeros(3, 16, dtype=torch.int8), torch.zeros(3))
    with pytest.raises(ValueError):
        matmul_int8(torch.zeros(3, 4), torch.zeros(3, 4))
    with pytest.raises(ValueError):
        Fp8Cache.empty(2, 2, 16, 64, device="cpu")
    with pytest.raises(ValueError):
        Fp8Cache.empty(2, 2, 16, 64, fmt="int8", device="cpu")
