"""Performance cases of the 8-bit integer products and of the 8-bit cache of keys and values with its attention.

Every case is one call of a public entry point:

  quantize  ``quantize_int8``: a matrix to 8-bit integers with a scale for each
            row (a token's, or a channel's of a weight)
  product   ``matmul_int8``: C = A B^T of two such matrices, or of a plain
            matrix A that the call quantises by rows on its way
  write     ``Fp8Cache.write``: keys and values of tokens into their places of
            a paged cache, in 8 bits with a scale for each token and head
  read      ``Fp8Cache.read``: keys and values of chosen places, as plain values
  attend    ``Fp8Cache.attend``: attention of single tokens, or of trees of
            drafted tokens, over the cache

The plain forms below compute the same from elementary operations.  A row of
integers has the scale max|x| / 127 (rounded to float32, 2^-126 at least) and
codes x / scale rounded to the nearest, ties to even.  A row of the cache has
the smallest power of two (2^-126 at least) that brings its largest magnitude to
the format's largest value or below it.
"""

import math

import numpy as np
import torch

own = False

FORMATS = {"e4m3": (torch.float8_e4m3fn, 448.0), "e5m2": (torch.float8_e5m2, 57344.0)}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one generated token against a 70B projection kept in 8 bits; quantised on the way
        dict(name="one token", op="product", m=1, n=8192, k=8192, a="bf16", out="bf16"),
        # odd sizes that fill no tile, float32 result
        dict(name="ragged product", op="product", m=1001, n=999, k=3001, a="int8", out="f32"),
        # a prompt through the 70B query projection
        dict(name="prompt product", op="product", m=8192, n=8192, k=8192, a="int8", out="bf16"),
        # activations of a prompt, a scale for each token
        dict(name="quantise tokens", op="quantize", rows=8192, cols=8192, dtype="bf16"),
        # weights of an odd width, a scale for each channel
        dict(name="quantise channels", op="quantize", rows=4097, cols=3001, dtype="f32"),
        # the next token of 64 sequences, 70B key heads: latency counts
        dict(name="write tokens", op="write", tokens=64, heads=8, dh=128, page=64, fmt="e4m3", dtype="bf16"),
        # a prompt's keys and values
        dict(name="write prompt", op="write", tokens=8191, heads=8, dh=128, page=64, fmt="e4m3", dtype="bf16"),
        # a long prefix back as plain values
        dict(name="read prefix", op="read", tokens=32768, heads=8, dh=128, page=64, fmt="e4m3", dtype="bf16"),
        # GPT-2-XL's heads, an odd number of tokens, E5M2, in float32
        dict(name="read odd", op="read", tokens=1999, heads=25, dh=64, page=16, fmt="e5m2", dtype="f32"),
        # one token at the end of a very long sequence, 70B heads
        dict(name="attend far", op="attend", batch=1, drafts=1, group=8, heads=8, dh=128, page=64, longest=131071,
             shortest=131071, tree="chain", fmt="e4m3", dtype="bf16"),
        # the next token of 64 sequences of many lengths
        dict(name="attend batch", op="attend", batch=64, drafts=1, group=8, heads=8, dh=128, page=64, longest=8192,
             shortest=200, tree="chain", fmt="e4m3", dtype="bf16"),
        # trees of 64 drafted tokens, to be checked at once
        dict(name="attend tree", op="attend", batch=16, drafts=64, group=8, heads=8, dh=128, page=64, longest=8192,
             shortest=8000, tree="each", fmt="e4m3", dtype="bf16"),
    ]


def draw(rng):
    """One more case of these ranges, at most the listed ones' bytes and operations."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["product", "product", "quantize", "write", "read", "attend", "attend"])
    if op == "product":
        m, n, k = log_int(1, 16384), log_int(64, 16384), log_int(64, 16384)
        while m * n * k > 8192 ** 3:
            m, n, k = (m + 1) // 2, n - n // 8, k - k // 8
        return dict(op=op, m=m, n=n, k=k, a=rng.choice(["bf16", "f32", "int8", "int8"]),
                    out=rng.choice(["f32", "bf16", "bf16"]))
    if op == "quantize":
        return dict(op=op, rows=log_int(1, 8192), cols=log_int(32, 8192), dtype=rng.choice(["f32", "bf16"]))
    heads, dh = log_int(1, 32), rng.choice([64, 80, 96, 128, 128, 256])
    more = dict(heads=heads, dh=dh, page=rng.choice([16, 32, 64, 128, 256]), fmt=rng.choice(["e4m3", "e4m3", "e5m2"]),
                dtype=rng.choice(["f32", "bf16", "bf16"]))
    if op != "attend":
        tokens = log_int(1, 32768)
        while tokens * heads * dh > 32768 * 8 * 128:
            tokens = (tokens + 1) // 2
        return dict(op=op, tokens=tokens, **more)
    batch, drafts, group = log_int(1, 64), rng.choice([1, 1, log_int(2, 64)]), rng.choice([1, 2, 4, 5, 8])
    longest = log_int(1, 131071)
    while batch * longest * heads * dh * max(drafts * group, 256) > 16 * 8192 * 8 * 128 * 512:
        longest = (longest + 1) // 2
    return dict(op=op, batch=batch, drafts=drafts, group=group, longest=longest,
                shortest=log_int(max(1, longest // 50), longest), tree=rng.choice(["chain", "one", "each"]), **more)


# ------------------------------------------------------------------ inputs


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + 7) % (1 << 62))
    return g


def _values(g, shape, dtype):
    """Activations as layers see them: normal values, some columns far larger than the others."""
    x = torch.randn(*shape, generator=g, device="cuda")
    x *= torch.exp(torch.randn(shape[-1], generator=g, device="cuda"))
    return x.to(DTYPES[dtype])


def _padded(codes):
    """The same codes with rows of a multiple of 16 bytes, as 8-bit matrices are stored."""
    room = torch.zeros(codes.shape[0], -(-codes.shape[1] // 16) * 16, dtype=codes.dtype, device=codes.device)
    room[:, :codes.shape[1]] = codes
    return room


def _cache(g, pages, case, filled):
    """Buffers [pages, heads, page, dh] of codes and [pages, heads, page] of scales, for keys and for values."""
    shape = (pages, case["heads"], case["page"], case["dh"])
    out = []
    for _ in range(2):
        if filled:
            codes, scale = _cache_rows(_values(g, shape, "f32"), case["fmt"])
            out += [codes, scale]
        else:
            out += [torch.zeros(shape, dtype=torch.uint8, device="cuda").view(FORMATS[case["fmt"]][0]),
                    torch.zeros(shape[:3], device="cuda")]
    return out


def _lengths(case):
    """Lengths from the shortest to the longest, in equal steps of their logarithm."""
    lo, hi, n = case["shortest"], case["longest"], case["batch"]
    return [hi if n == 1 else round(lo * (hi / lo) ** (i / (n - 1))) for i in range(n)]


def _trees(case, seed):
    """A mask for each drafted token: bit j says that it sees drafted token j; its ancestors and itself."""
    t, n = case["drafts"], case["batch"] if case["tree"] == "each" else 1
    r = np.random.default_rng([int(seed) % (1 << 32), 5])
    masks = np.zeros((n, t), dtype=np.uint64)
    for i in range(t):
        parent = r.integers(-1, i, n) if i else np.full(n, -1)
        above = np.where(parent >= 0, masks[np.arange(n), np.maximum(parent, 0)], np.uint64(0))
        masks[:, i] = above | np.uint64(1 << i)
    masks = torch.from_numpy(masks.view(np.int64)).cuda()
    return masks if case["tree"] == "each" else masks[0]


def prepare(case, seed):
    op = case["op"]
    g = _gen(seed)
    state = dict(case)
    if op == "quantize":
        state["x"] = _values(g, (case["rows"], case["cols"]), case["dtype"])
    elif op == "product":
        a = _values(g, (case["m"], case["k"]), "f32" if case["a"] == "int8" else case["a"])
        if case["a"] == "int8":
            codes, scale = _rows(a)
            a = (_padded(codes), scale)
        w = torch.randn(case["n"], case["k"], generator=g, device="cuda") * 0.02
        codes, scale = _rows(w)
        state["a"], state["b"], state["a_kind"] = a, (_padded(codes), scale), case["a"]
    elif op in ("write", "read"):
        t, page = case["tokens"], case["page"]
        pages = -(-t // page) + 3
        state["cache"] = _cache(g, pages, case, op == "read")
        order = torch.randperm(pages, generator=g, device="cuda")
        at = torch.arange(t, device="cuda")
        if t <= 64:  # tokens of as many sequences
            state["slots"] = torch.randperm(pages * page, generator=g, device="cuda")[:t]
        else:
            state["slots"] = order[at // page] * page + at % page
        if op == "write":
            state["k"], state["v"] = (_values(g, (t, case["heads"], case["dh"]), case["dtype"]) for _ in range(2))
    else:
        lengths = _lengths(case)
        need = [-(-n // case["page"]) for n in lengths]
        pages = sum(need) + 1
        state["cache"] = _cache(g, pages, case, True)
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).split(need + [1])
        table = torch.full((case["batch"], max(need)), -1, dtype=torch.int32, device="cuda")
        for i, ids in enumerate(order[:-1]):
            table[i, :need[i]] = ids
        mix = torch.randperm(case["batch"], generator=g, device="cuda")
        state["table"] = table[mix].contiguous()
        state["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")[mix].contiguous()
        shape = (case["batch"], case["drafts"], case["heads"] * case["group"], case["dh"])
        state["q"] = torch.randn(*shape, generator=g, device="cuda").to(DTYPES[case["dtype"]])
        state["masks"] = None if case["tree"] == "chain" else _trees(case, seed)
    return state


# ------------------------------------------------------------ plain forms


def _rows(x):
    """Integers [rows, cols] and scales [rows] of x."""
    x = x.double()  # quotients next to a tie
    scale = (x.abs().amax(dim=1) / 127.0).float().clamp(min=2.0 ** -126)  # a float32 quotient's last bit decides ties
    return torch.round(x / scale.double()[:, None]).to(torch.int8), scale


def _cache_rows(x, fmt):
    """Codes like x [..., dh] and scales [...]."""
    dtype, largest = FORMATS[fmt]
    x = x.float()
    mantissa, exponent = torch.frexp(x.abs().amax(dim=-1))  # mantissa in [0.5, 1)
    exponent = exponent - int(math.log2(largest / 1.75)) - 1 + (mantissa > 0.875)
    scale = ((exponent.clamp(min=-126) + 127) << 23).view(torch.float32)  # the power of two itself
    return (x / scale[..., None]).to(dtype), scale


def _sums(a, b, k):
    """Sums of products of integers, exact: in pieces whose sums stay below 2^24."""
    out = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device=a.device)
    for i in range(0, k, 1024):
        out += a[:, i:min(i + 1024, k)].float() @ b[:, i:min(i + 1024, k)].float().t()
    return out


def _plain_attend(state):
    q, table, lengths, masks = state["q"], state["table"], state["lengths"], state["masks"]
    kc, ks, vc, vs = state["cache"]
    batch, t, n_q, dh = q.shape
    heads, g = state["heads"], state["group"]
    out = torch.empty_like(q)
    pos = torch.arange(table.shape[1] * state["page"], device=q.device)
    drafted = torch.arange(t, device=q.device)
    for b in range(batch):
        ids = table[b].clamp(min=0).long()

        def values(codes, scale):
            v = codes[ids].float() * scale[ids][..., None]
            return v.transpose(0, 1).reshape(heads, -1, dh)

        k, v = values(kc, ks), values(vc, vs)
        rows = q[b].float().view(t, heads, g, dh).transpose(0, 1).reshape(heads, t * g, dh)
        s = rows @ k.transpose(1, 2) * dh ** -0.5
        at = pos - (lengths[b] - t)  # which drafted token a place holds
        if masks is None:
            sees = at[None, :] <= drafted[:, None]
        else:
            bits = (masks if masks.dim() == 1 else masks[b])[:, None] >> at.clamp(0, t - 1)[None, :] & 1
            sees = (at < 0)[None, :] | (bits == 1) & (at < t)[None, :]
        s = s.view(heads, t, g, -1).masked_fill(~sees[None, :, None, :], -math.inf)
        top = s.amax(dim=-1, keepdim=True)
        p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
        total = p.sum(dim=-1, keepdim=True)
        o = p.view(heads, t * g, -1) @ v / torch.where(total == 0, 1.0, total).view(heads, t * g, 1)
        out[b] = o.view(heads, t, g, dh).transpose(0, 1).reshape(t, n_q, dh).to(q.dtype)
    return out


def _plain(state):
    op = state["op"]
    if op == "quantize":
        return _rows(state["x"])
    if op == "product":
        a, sa = state["a"] if state["a_kind"] == "int8" else _rows(state["a"])
        b, sb = state["b"]
        return (_sums(a, b, state["k"]) * sa.double()[:, None] * sb.double()).to(DTYPES[state["out"]])
    if op == "write":
        page, at = state["page"], state["slots"]
        for i, x in enumerate((state["k"], state["v"])):
            codes, scale = _cache_rows(x, state["fmt"])
            # bytes: indexing does not know the 8-bit types
            state["cache"][2 * i].view(torch.uint8)[at // page, :, at % page] = codes.view(torch.uint8)
            state["cache"][2 * i + 1][at // page, :, at % page] = scale
        return list(state["cache"])
    if op == "read":
        page, at = state["page"], state["slots"]
        kc, ks, vc, vs = state["cache"]
        return [(c[at // page, :, at % page].float() * s[at // page, :, at % page][..., None]).to(DTYPES[state["dtype"]])
                for c, s in ((kc, ks), (vc, vs))]
    return _plain_attend(state)


# --------------------------------------------------- the framework's calls

_calls = None


def _framework():
    global _calls
    if _calls is None:
        import paper_2602_18851_amd as _calls_module

        _calls = _calls_module
    return _calls


def _own(state):
    f, op = _framework(), state["op"]
    if op == "quantize":
        m = f.quantize_int8(state["x"])
        return m.values, m.scale
    if op == "product":
        a = state["a"]
        if state["a_kind"] == "int8":
            a = f.Int8Matrix(*a, cols=state["k"])
        return f.matmul_int8(a, f.Int8Matrix(*state["b"], cols=state["k"]), out_dtype=DTYPES[state["out"]])
    if "handle" not in state:  # a program makes it once for a layer
        state["handle"] = f.Fp8Cache(*state["cache"])
    cache = state["handle"]
    if op == "write":
        cache.write(state["k"], state["v"], state["slots"])
        return [cache.k, cache.k_scale, cache.v, cache.v_scale]
    if op == "read":
        return list(cache.read(state["slots"], dtype=DTYPES[state["dtype"]]))
    return cache.attend(state["q"], state["table"], state["lengths"], tree=state["masks"])


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------- what a pass needs


def work(case):
    size = {"f32": 4, "bf16": 2, "int8": 1}
    op = case["op"]
    if op == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size[case["dtype"]] + 1) + 4 * case["rows"], "flops": 2 * n}
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k * size[case["a"]] + n * k + m * n * size[case["out"]], "flops": 2 * m * n * k}
    row = case["heads"] * (case["dh"] + 4) * 2  # a token's keys and values in the cache
    if op in ("write", "read"):
        n = case["tokens"] * case["heads"] * case["dh"] * 2
        return {"bytes": n * size[case["dtype"]] + case["tokens"] * (row + 8), "flops": 2 * n}
    places = sum(_lengths(case))
    rows = case["drafts"] * case["group"] * case["heads"]
    return {"bytes": places * row + 2 * case["batch"] * rows * case["dh"] * size[case["dtype"]],
            "flops": 4 * places * rows * case["dh"]}


# ------------------------------------------- the definitions, in 64 bits


def _power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_rows(x):
    scale = x.abs().max(dim=1, keepdim=True).values.double().div(127).float()  # a float32 by definition
    scale = torch.where(scale < 2.0 ** -126, 2.0 ** -126, scale)
    v = x.double() / scale.double()
    low = torch.floor(v)
    up = v - low  # to the nearer neighbour, ties to the even one
    v = low + ((up > 0.5) | (up == 0.5) & (low % 2 == 1))
    return v.to(torch.int8), scale[:, 0]


def _exact_cache_rows(x, fmt):
    """Values of the codes and scales, from the definition."""
    bits, low, largest = (3, -6, 448.0) if fmt == "e4m3" else (2, -14, 57344.0)
    x = x.double()
    top = x.abs().max(dim=-1).values
    scale = torch.full_like(top, 2.0 ** -126)
    at = torch.ceil(torch.log2((top / largest).clamp(min=2.0 ** -126)))
    for e in (at - 1, at, at + 1):  # the smallest power of two that is enough, whatever the logarithm rounded to
        p = _power(e)
        scale = torch.where((scale * largest < top) & (p * largest >= top), p, scale)
    v = x / scale[..., None]
    step = _power((torch.frexp(v).exponent - 1).clamp(min=low) - bits)
    return torch.round(v / step) * step, scale


def _exact_attend(state):
    """Query by query head; the places that a drafted token sees are picked out, so there is no mask."""
    q, table, masks = state["q"], state["table"], state["masks"]
    kc, ks, vc, vs = state["cache"]
    page, g = state["page"], state["group"]
    batch, t, n_q, dh = q.shape
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    for b, length in enumerate(state["lengths"].tolist()):
        at = torch.arange(length, device=q.device)
        ids, inside = table[b].long()[at // page], at % page
        before = max(length - t, 0)
        here = torch.arange(length - t, length, device=q.device)  # places of the drafted tokens
        for h in range(state["heads"]):
            k = kc[ids, h, inside].double() * ks[ids, h, inside].double()[:, None]
            v = vc[ids, h, inside].double() * vs[ids, h, inside].double()[:, None]
            rows = q[b, :, h * g:(h + 1) * g].double()  # [t, g, dh]
            e = rows.reshape(t * g, dh) @ k.t() / math.sqrt(dh)
            w = torch.zeros_like(e).view(t, g, length)
            e = e.view(t, g, length)
            for i in range(t):
                if masks is None:
                    seen = here[:i + 1]
                else:
                    m = int(masks[i] if masks.dim() == 1 else masks[b, i])
                    seen = here[[j for j in range(t) if m >> j & 1]]
                seen = torch.cat([at[:before], seen[seen >= 0]])
                if seen.numel():
                    w[i][:, seen] = torch.softmax(e[i][:, seen], dim=-1)
            out[b, :, h * g:(h + 1) * g] = (w.view(t * g, length) @ v).view(t, g, dh)
    return out


def exact(case, seed):
    op = case["op"]
    if op == "attend" and case["batch"] * case["heads"] * case["drafts"] > 8192:
        return None  # too many small steps
    state = prepare(case, seed)
    if op == "quantize":
        return _exact_rows(state["x"])
    if op == "product":
        a, sa = state["a"] if case["a"] == "int8" else _exact_rows(state["a"])
        b, sb = state["b"]
        k = case["k"]
        return (a[:, :k].double() * sa.double()[:, None]) @ (b[:, :k].double() * sb.double()[:, None]).t()
    page = case["page"]
    if op == "write":
        out = []
        for i, name in enumerate(("k", "v")):
            values = state["cache"][2 * i].double()
            scale = state["cache"][2 * i + 1].double()
            c, s = _exact_cache_rows(state[name], case["fmt"])
            at = state["slots"].tolist()
            where = torch.tensor([[n // page, n % page] for n in at], device="cuda")
            values[where[:, 0], :, where[:, 1]] = c
            scale[where[:, 0], :, where[:, 1]] = s
            out += [values, scale]
        return out
    if op == "read":
        flat = [t.double().transpose(1, 2).flatten(0, 1) for t in (state["cache"][0], state["cache"][2])]
        scale = [t.double().transpose(1, 2).flatten(0, 1) for t in (state["cache"][1], state["cache"][3])]
        return [c[state["slots"]] * s[state["slots"]].unsqueeze(-1) for c, s in zip(flat, scale)]
    return _exact_attend(state)
