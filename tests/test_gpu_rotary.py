"""Rotary positions against the float64 oracle (oracle.rotary), alone and inside the logit consumer."""

import math

import numpy as np
import pytest
import torch

from oracle import e4m3, rotary as rotary_oracle

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - collected on CPU machines, skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2602_18851_amd import LinearFp8, Rotary, Spectral  # noqa: E402
from paper_2602_18851_amd.spectral import SN_EINVAL, SpectralError  # noqa: E402

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SCALINGS = {"none": {}, "linear": dict(factor=3.0), "base": dict(factor=4.0),
            "index": dict(factor=8.0, trained=4096, low=1.0, high=32.0),
            "turns": dict(factor=8.0, trained=4096, low=1.0, high=4.0)}


def heads(key, t, h, d, dtype):
    r = np.random.default_rng([20260302, *key])
    return torch.from_numpy(r.standard_normal((t, h, d)).astype(np.float32)).to(DTYPES[dtype]).cuda()


def host(t):
    return t.detach().cpu().double().numpy()


def check(got, x, positions, rot, layout, freq, amp, inverse=False):
    """Cosine and sine in float: 4 ulp of the function, half an ulp of its argument times at most pi, a product with the
    amplitude; then two products and a sum, 2^-24 each, of at most |x0| + |x1|; then the rounding to the type.  The angle's own
    error is |p| 2^-48 at most."""
    ref = rotary_oracle.rotate(host(x), positions, rot, layout, freq, amp, inverse)
    xs = np.abs(host(x))
    reach = np.zeros_like(xs)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    reach[..., a] = reach[..., b] = xs[..., a] + xs[..., b]
    p = np.abs(np.asarray(positions, dtype=np.float64))[:, None, None]
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    tol = amp * reach * (12 * 2.0 ** -24 + p * 2.0 ** -48) + half * np.abs(ref) * 1.01
    err = np.abs(host(got) - ref)
    assert got.dtype == x.dtype and (err <= tol).all(), float((err - tol).max())
    assert torch.equal(got[..., rot:], x[..., rot:])


@pytest.mark.parametrize("d,rot", [(128, 128), (64, 32), (80, 80), (96, 40), (256, 256), (2, 2), (7, 6), (65, 64), (16, 12)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary(d, rot, layout, dtype, inverse):
    plan = Rotary(d, rot_dim=rot, layout=layout)
    freq, amp = rotary_oracle.frequencies(rot)
    for t, hq, hk in ((1, 1, 1), (5, 8, 2), (37, 3, 3)):
        q, k = heads((d, t, 1), t, hq, d, dtype), heads((d, t, 2), t, hk, d, dtype)
        p = torch.from_numpy(np.random.default_rng(t).integers(0, 5000, t)).cuda()
        a, b = plan.apply(q, k, positions=p, inverse=inverse)
        check(a, q, host(p), rot, layout, freq, amp, inverse)
        check(b, k, host(p), rot, layout, freq, amp, inverse)
        assert torch.equal(plan.apply(q, positions=p, inverse=inverse), a)
        first, last = plan.apply(q, k, start=11, inverse=inverse), torch.arange(11, 11 + t, device="cuda")
        for x, y in zip(first, plan.apply(q, k, positions=last, inverse=inverse)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("scaling", list(SCALINGS))
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_scaled_frequencies_and_far_positions(scaling, layout):
    plan = Rotary(64, layout=layout, base=500000.0, scaling=scaling, **SCALINGS[scaling])
    freq, amp = rotary_oracle.frequencies(64, base=500000.0, scaling=scaling, **SCALINGS[scaling])
    p = np.array([0, 1, 4095, 4096, 131071, 1 << 20, (1 << 24) + 1, (1 << 31) - 1])
    x = heads((scaling == "none", 4), len(p), 6, 64, "f32")
    check(plan.apply(x, positions=torch.from_numpy(p).cuda()), x, p, 64, layout, freq, amp)


@pytest.mark.parametrize("scaling", list(SCALINGS))
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("inverse", [False, True])
def test_cosines_and_sines_are_rounded_once(scaling, layout, inverse):
    """The pair (1, 0) turns into its cosine and sine times the amplitude, with nothing else rounded: half a unit of float32
    (2^-24 of the value) and what the double operations before it leave: the angle's p 2^-48, and 2^-34 of the value, the first
    term left out of the sine's series at an eighth of a turn, (pi / 4)^13 / 13! beside 0.7."""
    plan = Rotary(64, layout=layout, base=500000.0, scaling=scaling, **SCALINGS[scaling])
    freq, amp = rotary_oracle.frequencies(64, base=500000.0, scaling=scaling, **SCALINGS[scaling])
    p = np.concatenate([np.arange(3000), np.random.default_rng(5).integers(3000, 1 << 20, 1000)])
    x = torch.zeros(len(p), 1, 64, device="cuda")
    x[..., slice(0, 32) if layout == "half" else slice(0, 64, 2)] = 1.0
    got = plan.apply(x, positions=torch.from_numpy(p).cuda(), inverse=inverse)
    ref = rotary_oracle.rotate(host(x), p, 64, layout, freq, amp, inverse)
    tol = np.abs(ref) * (2.0 ** -24 + 2.0 ** -34) + amp * p[:, None, None] * 2.0 ** -48
    assert (np.abs(host(got) - ref) <= tol).all()


def test_turning_back_is_the_gradient():
    """<R x, g> = <x, R^T g> by differences: the map is linear, so a central difference is exact but for float32."""
    plan = Rotary(32, rot_dim=24, layout="interleaved", scaling="index", **SCALINGS["index"])
    x, g = heads((1, 1), 9, 2, 32, "f32"), heads((1, 2), 9, 2, 32, "f32")
    p = torch.arange(100, 109, device="cuda")
    dx = plan.apply(g, positions=p, inverse=True)
    for t, h, e in ((0, 0, 0), (8, 1, 23), (4, 0, 7), (3, 1, 30)):
        up, down = x.clone(), x.clone()
        up[t, h, e] += 1
        down[t, h, e] -= 1
        diff = (host(plan.apply(up, positions=p)) * host(g)).sum() - (host(plan.apply(down, positions=p)) * host(g)).sum()
        # each of the two elements that move is off by 2^-24 of values below 8, with gradients below 4
        assert abs(diff / 2 - float(dx[t, h, e])) < 64 * 2.0 ** -24 * 4
    # a rotation and back, without amplitude: the same up to the roundings of both
    plain = Rotary(32, layout="half")
    back = plain.apply(plain.apply(x, positions=p), positions=p, inverse=True)
    assert (back - x).abs().max() < 40 * 2.0 ** -24 * 4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_strided_and_shared_inputs(dtype):
    plan = Rotary(64, rot_dim=48)
    p = torch.arange(3, 24, device="cuda")
    x = heads((2, 1), 21, 5, 64, dtype)
    ref = plan.apply(x, positions=p)
    here = x.clone()
    assert plan.apply(here, positions=p, out=here) is here and torch.equal(here, ref)
    # heads before tokens, a window whose heads are not 16-byte aligned, one tensor for queries and keys
    room = torch.full((5, 21, 67), 9.0, dtype=DTYPES[dtype], device="cuda")
    view = room[:, :, 1:65].permute(1, 0, 2)
    view.copy_(x)
    assert torch.equal(plan.apply(view, positions=p), ref)
    plan.apply(view, positions=p, out=view)
    assert torch.equal(view, ref) and (room[:, :, 0] == 9).all() and (room[:, :, 65:] == 9).all()
    qkv = torch.full((21, 3, 5, 64), 1.0, dtype=DTYPES[dtype], device="cuda")
    qkv[:, 0].copy_(x)
    qkv[:, 1].copy_(x)
    a, b = plan.apply(qkv[:, 0], qkv[:, 1], positions=p, out=(qkv[:, 0], qkv[:, 1]))
    assert torch.equal(a, ref) and torch.equal(b, ref) and (qkv[:, 2] == 1).all()
    one = x[:, :1].expand(21, 5, 64)
    assert torch.equal(plan.apply(one, positions=p), plan.apply(one.contiguous(), positions=p))


def test_padding_stays():
    plan = Rotary(128)
    q, k = heads((3, 1), 40, 4, 128, "bf16"), heads((3, 2), 40, 2, 128, "bf16")
    p = torch.arange(40, device="cuda")
    ref = plan.apply(q, k, positions=p)
    p[33:] = -1
    p[7] = -(1 << 40)
    outs = torch.full_like(q, 5.0), torch.full_like(k, 6.0)
    plan.apply(q, k, positions=p, out=outs)
    live = p >= 0
    for o, r, v in zip(outs, ref, (5.0, 6.0)):
        assert torch.equal(o[live], r[live]) and (o[~live] == v).all()


@pytest.mark.parametrize("d,rot", [(128, 128), (96, 40), (7, 6), (16, 12)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("inverse", [False, True])
def test_padding_in_new_tensors_is_not_turned(d, rot, layout, dtype, inverse):
    """The new tensors take memory that held NaN; their rows of padding are the input's, whatever these hold."""
    plan = Rotary(d, rot_dim=rot, layout=layout, scaling="index", **SCALINGS["index"])
    q, k = heads((9, 1), 21, 4, d, dtype), heads((9, 2), 21, 2, d, dtype)
    q[3, 1, 0], q[3, 1, 1], q[20] = float("inf"), -0.0, 0.0
    p = torch.arange(21, device="cuda")
    p[[0, 3, 17, 20]] = torch.tensor([-1, -(1 << 40), -5, -2], device="cuda")

    def poison():
        for t in (q, k):
            torch.full_like(t, float("nan"))

    def same(a, b):  # bits, an infinity and a zero's sign among them
        return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))

    live = p >= 0
    ref = plan.apply(q[live], k[live], positions=p[live], inverse=inverse)
    torch.cuda.synchronize()
    poison()
    got = plan.apply(q, k, positions=p, inverse=inverse)
    for o, x, r in zip(got, (q, k), ref):
        assert same(o[live], r) and same(o[~live], x[~live])
    ref = plan.apply(q[6:], inverse=inverse)
    poison()
    got = plan.apply(q, start=-6, inverse=inverse)
    assert same(got[:6], q[:6]) and same(got[6:], ref)


def test_many_tokens_and_far_rows():
    """More groups of tokens than one launch takes, and rows that start past 2^32 bytes."""
    plan = Rotary(2)
    n = (1 << 24) + 100
    x = torch.ones(n, 1, 2, device="cuda")
    got = plan.apply(x)
    for t in (0, 1, 1 << 20, (1 << 24) - 1, 1 << 24, n - 1):
        assert abs(float(got[t, 0, 0]) - (math.cos(t) - math.sin(t))) < 16 * 2.0 ** -24
        assert abs(float(got[t, 0, 1]) - (math.cos(t) + math.sin(t))) < 16 * 2.0 ** -24
    del x, got
    plan = Rotary(64)
    room = torch.empty(700, 1 << 21, device="cuda")  # 5.9 GB
    far = room[:, :128].view(700, 2, 64)
    x = heads((8, 1), 700, 2, 64, "f32")
    far.copy_(x)
    ref = plan.apply(x)
    assert torch.equal(plan.apply(far), ref)
    plan.apply(far, out=far)
    assert torch.equal(far, ref)


def test_values_that_are_not_finite_stay_in_their_pair():
    plan = Rotary(64)
    x = heads((4, 1), 3, 2, 64, "f32")
    x[1, 0, 5] = float("inf")
    x[2, 1, 40] = float("nan")
    got = host(plan.apply(x, start=2))
    bad = ~np.isfinite(got)
    want = np.zeros_like(bad)
    want[1, 0, [5, 37]] = want[2, 1, [8, 40]] = True
    assert (bad == want).all()


def test_empty_and_refused_calls():
    plan = Rotary(64)
    x = heads((5, 1), 4, 2, 64, "f32")
    assert plan.apply(x[:0]).shape == (0, 2, 64) and plan.apply(x[:, :0]).shape == (4, 0, 64)
    for bad in (lambda: plan.apply(x[..., :32]), lambda: plan.apply(x.half()), lambda: plan.apply(x, x.bfloat16()),
                lambda: plan.apply(x, x[:3]), lambda: plan.apply(x, positions=torch.arange(4)),
                lambda: plan.apply(x, positions=torch.arange(4, dtype=torch.int32, device="cuda")),
                lambda: plan.apply(x, positions=torch.arange(5, device="cuda")), lambda: plan.apply(x.cpu()),
                lambda: plan.apply(x, out=x.bfloat16()), lambda: plan.apply(x, x, out=(x,)),
                lambda: plan.apply(x.transpose(1, 2).contiguous().transpose(1, 2)),
                lambda: Rotary(64, layout="other"), lambda: Rotary(64, scaling="other")):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(SpectralError) as e:
        plan.apply(x, out=x[:1].expand(4, 2, 64))
    assert e.value.code == SN_EINVAL
    with pytest.raises(SpectralError):
        Rotary(64, rot_dim=65)


def test_heads_that_require_gradients_are_refused():
    plan = Rotary(64)
    q, k = heads((10, 1), 4, 2, 64, "f32"), heads((10, 2), 4, 2, 64, "f32").requires_grad_()
    for bad in (lambda: plan.apply(k), lambda: plan.apply(q, k), lambda: plan.apply(q, k, out=(q, k.detach().clone()))):
        with pytest.raises(ValueError, match="requires gradients"):
            bad()
    with torch.no_grad():
        assert torch.equal(plan.apply(q, k)[1], plan.apply(k.detach()))


def test_rotary_replays_from_a_graph_and_on_another_stream():
    plan = Rotary(128, scaling="turns", **SCALINGS["turns"])
    q, k = heads((6, 1), 70, 8, 128, "bf16"), heads((6, 2), 70, 2, 128, "bf16")
    p = torch.arange(70, device="cuda")
    plan.apply(q, k, positions=p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = plan.apply(q, k, positions=p)
    for rep in range(4):
        q.mul_(1.25)
        p.add_(1000)
        graph.replay()
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            ref = plan.apply(q, k, positions=p)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


# ---------------------------------------------------------- logit consumer


@pytest.mark.parametrize("dh,rot,layout", [(64, 64, "half"), (128, 128, "half"), (16, 12, "interleaved"), (32, 16, "half")])
@pytest.mark.parametrize("own_positions", [False, True])
def test_logits_of_turned_queries_and_keys(dh, rot, layout, own_positions):
    """Scaled logits within 2^-14 of the products' magnitudes (the projections' hi and lo halves carry 2^-16 each, the
    rotation and its split as much again, three products of halves 2^-16) give codes between those
    of the oracle's value less and plus so much."""
    L, seq, d, nq, nkv = 2, 70, 200, 4, 2
    r = np.random.default_rng([20260303, dh, rot])
    t = lambda *s: torch.from_numpy(r.standard_normal(s).astype(np.float32)).bfloat16()  # noqa: E731
    x, wq, wk = t(L, seq, d), t(L, nq * dh, d) * 0.05, t(L, nkv * dh, d) * 0.05
    est = Spectral(L, d, nq, nkv, dh, "bf16", 0.1)
    plan = Rotary(dh, rot_dim=rot, layout=layout)
    freq, amp = rotary_oracle.frequencies(rot)
    p = np.arange(seq)
    if own_positions:
        p = r.integers(0, 30000, seq)
        p[-3:] = -1
    scale = torch.tensor([0.004, 0.01], device="cuda")
    kw = dict(positions=torch.from_numpy(p).cuda()) if own_positions else {}
    mx, over, codes = est.logits_fp8(x.cuda(), wq.cuda(), wk.cuda(), scale, want_codes=True, rotary=plan, **kw)
    mx, over, codes = host(mx), over.cpu().numpy(), codes.cpu().numpy()
    turned = np.maximum(p, 0)  # rows at negative positions are not turned
    for l in range(L):
        X = host(x[l])
        Q = rotary_oracle.rotate((X @ host(wq[l]).T).reshape(seq, nq, dh), turned, rot, layout, freq, amp)
        K = rotary_oracle.rotate((X @ host(wk[l]).T).reshape(seq, nkv, dh), turned, rot, layout, freq, amp)
        for h in range(nq):
            f = 1.0 / (math.sqrt(dh) * float(scale[l]))
            S, mag = Q[:, h] @ K[:, h // 2].T * f, np.abs(Q[:, h]) @ np.abs(K[:, h // 2]).T * f
            tol = mag * 2.0 ** -13
            low, high = (e4m3.decode(e4m3.encode(v, saturate=True)) for v in (S - tol, S + tol))
            v = e4m3.decode(codes[l, h])
            none = np.isnan(v)  # past 464
            assert (none <= (np.abs(S) + tol > 464)).all() and (none >= (np.abs(S) - tol > 464)).all()
            assert (none | ((low <= v) & (v <= high))).all()
            assert abs(mx[l, h] - np.abs(S).max()) <= tol.max()
            assert (np.abs(S) - tol > 448).sum() <= over[l, h] <= (np.abs(S) + tol > 448).sum()
    with pytest.raises(ValueError):
        est.logits_fp8(x.cuda(), wq.cuda(), wk.cuda(), scale, positions=torch.arange(seq, device="cuda"))
    with pytest.raises(SpectralError) as e:
        est.logits_fp8(x.cuda(), wq.cuda(), wk.cuda(), scale, rotary=Rotary(dh * 2))
    assert e.value.code == SN_EINVAL
    # position zero everywhere turns nothing; a lo half that was rounded up to half a step of hi can be split the other
    # way round the second time, and the sum of three products of halves then moves by 2^-16: at most to the next code
    zero = torch.zeros(seq, dtype=torch.int64, device="cuda")
    _, _, still = est.logits_fp8(x.cuda(), wq.cuda(), wk.cuda(), scale, want_codes=True, rotary=plan, positions=zero)
    _, _, plain = est.logits_fp8(x.cuda(), wq.cuda(), wk.cuda(), scale, want_codes=True)
    assert ((still.int() - plain.int()).abs() <= 1).all()
    assert (still != plain).float().mean() < 2.0 ** -8  # values within 2^-15 of a border between codes 2^-3 apart


@pytest.mark.parametrize("dh,rot,layout", [(64, 64, "half"), (16, 12, "interleaved"), (128, 96, "half")])
def test_rows_that_do_not_turn_keep_their_logits(dh, rot, layout):
    """Rows at position zero and at negative ones give the codes, maxima and counts of the call without positions; with an
    amplitude only the negative ones do.  (One value in 2^10 splits into other halves the second time, so that of 128 maxima
    over sums of d_h products some would move.)"""
    L, seq, d, nq, nkv = 4, 130, 200, 32, 8
    r = np.random.default_rng([20260306, dh, rot])
    t = lambda *s: torch.from_numpy(r.standard_normal(s).astype(np.float32)).bfloat16().cuda()  # noqa: E731
    x, wq, wk = t(L, seq, d), t(L, nq * dh, d) * 0.05, t(L, nkv * dh, d) * 0.05
    est, scale = Spectral(L, d, nq, nkv, dh, "bf16", 0.1), torch.tensor([0.004, 0.01] * 2, device="cuda")
    plain = est.logits_fp8(x, wq, wk, scale, want_codes=True)
    p = torch.zeros(seq, dtype=torch.int64, device="cuda")
    p[::3] = -4
    got = est.logits_fp8(x, wq, wk, scale, want_codes=True, rotary=Rotary(dh, rot_dim=rot, layout=layout), positions=p)
    assert all(torch.equal(a, b) for a, b in zip(plain, got))
    loud = Rotary(dh, rot_dim=rot, layout=layout, scaling="index", **SCALINGS["index"])
    got = est.logits_fp8(x, wq, wk, scale, want_codes=True, rotary=loud, positions=p)
    stay = torch.nonzero(p < 0).flatten()
    assert torch.equal(got[2][:, :, stay][..., stay], plain[2][:, :, stay][..., stay])
    assert not torch.equal(got[2], plain[2])


def test_logits_of_turned_heads_replay_from_a_graph():
    L, seq, d, nq, nkv, dh = 2, 130, 256, 4, 2, 64
    r = np.random.default_rng(20260305)
    t = lambda *s: torch.from_numpy(r.standard_normal(s).astype(np.float32)).bfloat16().cuda()  # noqa: E731
    x, wq, wk = t(L, seq, d), t(L, nq * dh, d) * 0.05, t(L, nkv * dh, d) * 0.05
    scale, p = torch.tensor([0.05, 0.1], device="cuda"), torch.arange(seq, device="cuda")
    est, plan = Spectral(L, d, nq, nkv, dh, "bf16", 0.1), Rotary(dh)

    def call():
        return est.logits_fp8(x, wq, wk, scale, want_codes=True, rotary=plan, positions=p)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for rep in range(4):
        x.mul_(0.75)
        p.add_(17)
        graph.replay()
        torch.cuda.synchronize()
        ref = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_projections_positions_and_scales_together():
    """One attention layer's front half as a program runs it: the scale from the estimator, queries and keys from 8-bit
    products, turned by their positions; the logits obey the bound of the unturned weights (Sec. 3.3), and the gradients
    go back through both operators."""
    seq, d, nq, nkv, dh = 96, 256, 4, 2, 64
    r = np.random.default_rng(20260304)
    x = r.standard_normal((seq, d))
    x = torch.from_numpy((x / np.linalg.norm(x, axis=1, keepdims=True) * math.sqrt(d)).astype(np.float32)).bfloat16().cuda()
    wq = torch.from_numpy((r.standard_normal((nq * dh, d)) * 0.05).astype(np.float32)).bfloat16().cuda()
    wk = torch.from_numpy((r.standard_normal((nkv * dh, d)) * 0.05).astype(np.float32)).bfloat16().cuda()
    est = Spectral(1, d, nq, nkv, dh, "bf16", 1.0)
    v = torch.from_numpy(r.standard_normal((1, nq, d)).astype(np.float32)).cuda()
    sigma, scale, _ = est.step(wq[None], wk[None], v, 30)
    plan = Rotary(dh)
    lq, lk = LinearFp8(wq), LinearFp8(wk)
    q, kept_q = lq.forward(x, keep=True)
    k, kept_k = lk.forward(x, keep=True)
    tq, tk = plan.apply(q.view(seq, nq, dh), k.view(seq, nkv, dh))
    S = np.stack([host(tq)[:, h] @ host(tk)[:, h // 2].T for h in range(nq)]) / math.sqrt(dh)
    # 8-bit codes are off by at most 2^-4 of their value: a few percent of the norm products at most
    bound = host(sigma)[0][:, None, None] * d / math.sqrt(dh)
    assert (np.abs(S) <= 1.2 * bound).all()
    mx, over, _ = est.logits_fp8(x[None], wq[None], wk[None], scale, rotary=plan)
    assert int(over.sum()) == 0
    # rms distance of the 8-bit logits from the consumer's: both operands rounded to 4 bits in both products
    exact = np.stack([m for m in (rotary_oracle.rotate((host(x) @ host(wq).T).reshape(seq, nq, dh), np.arange(seq), dh, "half",
                                                       *rotary_oracle.frequencies(dh))).transpose(1, 0, 2)])
    exact_k = rotary_oracle.rotate((host(x) @ host(wk).T).reshape(seq, nkv, dh), np.arange(seq), dh, "half",
                                   *rotary_oracle.frequencies(dh)).transpose(1, 0, 2)
    E = np.stack([exact[h] @ exact_k[h // 2].T for h in range(nq)]) / math.sqrt(dh)
    # each code is off by at most 2^-4 of itself, so q and k by at most (2^-3 + 2^-8) |x| |w|, summed
    xa, qa, ka = np.abs(host(x)), np.abs(host(wq)), np.abs(host(wk))
    Qa = (xa @ qa.T).reshape(seq, nq, dh).transpose(1, 0, 2) * math.sqrt(2)
    Ka = (xa @ ka.T).reshape(seq, nkv, dh).transpose(1, 0, 2) * math.sqrt(2)
    lim = np.stack([Qa[h] @ Ka[h // 2].T for h in range(nq)]) / math.sqrt(dh) * 0.3
    assert (np.abs(S - E) <= lim).all()
    assert abs(float(mx.max()) * float(scale[0]) - np.abs(E).max()) <= 2.0 ** -10 * np.abs(E).max()
    # gradients: back through the rotation, then through the products
    g = torch.from_numpy(r.standard_normal((seq, nq, dh)).astype(np.float32)).bfloat16().cuda()
    dq = plan.apply(g, inverse=True).view(seq, nq * dh)
    dx, dw = lq.backward(dq, kept_q)
    from oracle import fp8_blocks

    def f8(t, br):
        return fp8_blocks.values(*fp8_blocks.quantize(t, br, "e4m3"), br)

    want_dw, want_dx = f8(host(dq).T, 1) @ f8(host(x).T, 1).T, f8(host(dq), 1) @ f8(host(wq).T, 128).T
    assert np.abs(host(dw) - want_dw).max() <= 2.0 ** -14 * (np.abs(f8(host(dq).T, 1)) @ np.abs(f8(host(x).T, 1)).T).max()
    assert np.abs(host(dx) - want_dx).max() <= 2.0 ** -8 * np.abs(want_dx).max() * 1.01
    assert kept_k.rows == d
