"""Attention under documents, lengths, causal and prefix masks, with distance bias and capped scores, against the formula
in 64 bits.  Tolerances are bounds by the roundings that the kernels make, element by element."""
import math

import numpy as np
import pytest

F32 = 2.0 ** -24


def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def make(dtype, B, S, heads, kv, dim, seed=0, docs=None, lens=None, causal=False, prefix=None, cap=0.0, slopes=False, common=0.0,
         poison=True):
    """Inputs as views of one fused buffer; rows beyond a sequence hold NaN and infinities."""
    import torch
    g = torch.Generator().manual_seed(seed + 7 * S + dim)
    t = torch.float32 if dtype == "fp32" else torch.bfloat16
    fused = torch.randn(B, S, heads + 2 * kv, dim, generator=g)
    fused[:, :, heads:] += common * torch.randn(heads * 0 + 2 * kv, dim, generator=g)
    dc = torch.randn(B, S, heads, dim, generator=g)
    if lens is not None and poison:
        for b, n in enumerate(lens):
            fused[b, max(0, n):] = float("nan")
            fused[b, max(0, n)::2] = float("inf") if n < 0 else fused[b, max(0, n)::2]
            dc[b, max(0, n):] = float("inf")
    fused, dc = fused.to(t).cuda(), dc.to(t).cuda()
    i32 = lambda v: None if v is None else torch.tensor(np.asarray(v), dtype=torch.int32).cuda()            # noqa: E731
    return dict(q=fused[:, :, :heads], k=fused[:, :, heads:heads + kv], v=fused[:, :, heads + kv:], dc=dc, scale=1 / math.sqrt(dim),
                mask=dict(cap=cap, causal=causal, prefix=i32(prefix), docs=i32(docs), lens=i32(lens),
                          slopes=torch.exp2(-torch.arange(1.0, heads + 1)).cuda() if slopes else None))


def run(s, backward=True, rest=True):
    import torch
    from paper_2011_13635_b200 import binding as B
    q, k = s["q"], s["k"]
    nb, n, heads, dim = q.shape
    kv = k.shape[2]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx = torch.full((nb, n, heads, dim), 9.0, dtype=q.dtype, device="cuda")
    low = torch.full_like(ctx, 9.0) if rest and q.dtype == torch.bfloat16 else None
    lse = torch.full((nb, heads, n), 9.0, device="cuda")
    B.mslt_op_attention_masked(q, k, s["v"], ctx, lse, s["scale"], status, _stream(), rest=low, **s["mask"])
    out = dict(ctx=ctx, lse=lse)
    if backward:
        wide = torch.full((nb, n, heads + 2 * kv + 2, dim), 5.0, dtype=q.dtype, device="cuda")
        dq, dk, dv = wide[:, :, 1:1 + heads], wide[:, :, 1 + heads:1 + heads + kv], wide[:, :, 1 + heads + kv:-1]
        size = B.mslt_op_attention_masked_bwd_scratch_bytes(nb, n, heads)
        scratch = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        B.mslt_op_attention_masked_bwd(q, k, s["v"], ctx, lse, s["dc"], dq, dk, dv, scratch, s["scale"], status, _stream(), rest=low,
                                       **s["mask"])
        assert (wide[:, :, 0] == 5).all() and (wide[:, :, -1] == 5).all()      # neighbours are left alone
        out.update(dq=dq, dk=dk, dv=dv)
    return out


def visible(s):
    import torch
    n, m = s["q"].shape[1], s["mask"]
    nb = s["q"].shape[0]
    i = torch.arange(n)
    ok = torch.ones(nb, n, n, dtype=torch.bool)
    for b in range(nb):
        if m["causal"]:
            ok[b] = i[None] <= i[:, None]
            if m["prefix"] is not None:
                ok[b] |= (i < int(m["prefix"][b]))[None]
        if m["docs"] is not None:
            d = m["docs"][b].cpu()
            ok[b] &= d[:, None] == d
        if m["lens"] is not None:
            ok[b] &= (i < int(m["lens"][b]))[None] & (i < int(m["lens"][b]))[:, None]
    return ok


def check(s, out, rest=True):
    """Every output against the formula in 64 bits, within the bound of its roundings."""
    import torch
    bf16 = s["q"].dtype == torch.bfloat16
    u = 2.0 ** -8 if bf16 else F32
    nb, n, heads, dim = s["q"].shape
    kv, m = s["k"].shape[2], s["mask"]
    ok_all = visible(s)
    D = lambda t: t.double().cpu()                                                                          # noqa: E731
    clean = lambda t: torch.nan_to_num(D(t), 0.0, 0.0, 0.0)                                                 # noqa: E731
    Q, K, V, dC = clean(s["q"]), clean(s["k"]), clean(s["v"]), clean(s["dc"])
    i = torch.arange(n, dtype=torch.float64)
    dist = (i[:, None] - i).abs()
    for b in range(nb):
        ok = ok_all[b]
        some = ok.any(-1)
        dk = torch.zeros(kv, n, dim, dtype=torch.float64)
        dv, e_dk, e_dv = torch.zeros_like(dk), torch.zeros_like(dk), torch.zeros_like(dk)
        for h in range(heads):
            hk = h // (heads // kv)
            q, k, v, dc = Q[b, :, h], K[b, :, hk], V[b, :, hk], dC[b, :, h]
            z = q @ k.T * s["scale"]
            # dim products and sums in fp32, then a few roundings of the score as it is formed
            ez = (dim + 8) * F32 * (q.abs() @ k.abs().T) * s["scale"]
            bend = torch.ones_like(z)
            if m["cap"]:
                t = torch.tanh(z / m["cap"])
                z, bend = m["cap"] * t, 1 - t * t
                ez = ez * 1.0 + 8 * F32 * m["cap"]
            if m["slopes"] is not None:
                slope = float(m["slopes"][h])
                z = z - slope * dist
                ez = ez + 4 * F32 * slope * dist
            ez = torch.where(ok, ez + 4 * F32 * z.abs(), torch.zeros_like(z))
            zm = z.masked_fill(~ok, -math.inf)
            lse = torch.logsumexp(zm, -1)
            p = torch.exp(zm - torch.where(some, lse, torch.zeros_like(lse))[:, None]) * ok
            got = D(out["lse"])[b, h]
            top = torch.where(some, zm.amax(-1), torch.zeros_like(lse))
            # exponentials: 2^-22 of the hardware's, arguments' roundings in ez; n sums; the logarithm
            e_row = ez.amax(-1) + 2.0 ** -21 + n * F32
            e_lse = e_row + 4 * F32 * (lse.abs() + top.abs())
            assert torch.equal(got[~some], torch.full_like(got[~some], -math.inf))
            assert ((got - lse).abs()[some] <= e_lse[some]).all(), ("lse", b, h)
            o = p @ v
            # a probability's rounding, and the sum's; with rest the probabilities are held to half a step of a bf16 remainder
            up = (2 * u * u if rest else 2 * u) if bf16 else 0.0
            rel = (up + 2 * e_row)[:, None]
            e_o = rel * (p @ v.abs()) + n * F32 * (p @ v.abs()) + u * o.abs()
            diff = (D(out["ctx"])[b, :, h] - o).abs()
            assert (diff <= e_o + 1e-37).all(), ("ctx", b, h, float((diff - e_o).max()))
            if "dq" not in out:
                continue
            dp = dc @ v.T
            delta = (p * dp).sum(-1, keepdim=True)
            x = (dp - delta) * ok
            edp = (dim + 8) * F32 * (dc.abs() @ v.abs().T)
            low = (2.0 ** -16 if rest else 2.0 ** -8) if bf16 else F32
            e_delta = rel * (p * x.abs()).sum(-1, keepdim=True) + 2 * (p * edp).sum(-1, keepdim=True) + \
                (low + (dim + 8) * F32) * (dc.abs() * o.abs()).sum(-1, keepdim=True) + n * F32 * (dc.abs() * (p @ v.abs())).sum(-1, keepdim=True)
            ds = p * x * bend
            ebend = 8 * F32 if m["cap"] else 0.0
            e_ds = p * (x.abs() * (2 * e_row[:, None] + ebend) + edp + e_delta) * 1.0 + 1.0e-5 * p * x.abs() * (p > 0.9999) + u * ds.abs()
            e_ds = e_ds * 1.01
            dq = ds @ k * s["scale"]
            e_dq = s["scale"] * (e_ds @ k.abs() + n * F32 * (ds.abs() @ k.abs())) + u * dq.abs()
            diff = (D(out["dq"])[b, :, h] - dq).abs()
            assert (diff <= e_dq + 1e-37).all(), ("dq", b, h, float((diff - e_dq).max()))
            group = heads // kv
            dk[hk] += ds.T @ q * s["scale"]
            e_dk[hk] += s["scale"] * (e_ds.T @ q.abs() + group * n * F32 * (ds.abs().T @ q.abs()))
            dv[hk] += p.T @ dc
            e_dv[hk] += (p * (u * bf16 + 2 * e_row[:, None] + group * n * F32)).T @ dc.abs()
        if "dq" in out:
            for name, ref, tol in (("dk", dk, e_dk), ("dv", dv, e_dv)):
                diff = (D(out[name])[b].transpose(0, 1) - ref).abs()
                assert (diff <= 1.01 * tol + u * ref.abs() + 1e-37).all(), (name, b, float((diff - tol).max()))


def documents(B, S, n, seed=1):
    r = np.random.default_rng(seed + S)
    return np.stack([np.searchsorted(np.sort(r.integers(0, S, n - 1)), np.arange(S), side="right") for _ in range(B)])


def cases():
    out = []
    for dtype in ("fp32", "bf16"):
        for S in (1, 2, 63, 64, 65, 127, 128, 129, 200, 257):
            out.append((dtype, dict(B=2, S=S, heads=2, kv=2, dim=64)))
            out.append((dtype, dict(B=2, S=S, heads=2, kv=1, dim=64, causal=True)))
        for dim in (8, 24, 72, 96, 128):
            out.append((dtype, dict(B=1, S=150, heads=4, kv=2, dim=dim, docs=documents(1, 150, 3), slopes=True)))
        out += [
            (dtype, dict(B=3, S=130, heads=3, kv=3, dim=64, lens=[130, 0, 77])),
            (dtype, dict(B=4, S=300, heads=2, kv=1, dim=64, lens=[1, 64, 65, 299], causal=True)),
            (dtype, dict(B=2, S=129, heads=2, kv=2, dim=128, lens=[128, -3], slopes=True)),
            (dtype, dict(B=2, S=333, heads=2, kv=2, dim=64, docs=documents(2, 333, 7))),
            (dtype, dict(B=2, S=260, heads=2, kv=2, dim=64, docs=np.random.default_rng(0).integers(-2, 3, (2, 260)))),
            (dtype, dict(B=1, S=140, heads=2, kv=2, dim=64, docs=np.arange(140)[None] * 1000003 - 70000000)),  # everyone alone
            (dtype, dict(B=2, S=200, heads=2, kv=2, dim=64, docs=documents(2, 200, 4), lens=[200, 131], causal=True, prefix=[60, 500])),
            (dtype, dict(B=3, S=190, heads=2, kv=2, dim=64, causal=True, prefix=[0, 1, 150])),
            (dtype, dict(B=1, S=200, heads=4, kv=4, dim=64, cap=5.0)),
            (dtype, dict(B=1, S=200, heads=8, kv=2, dim=64, cap=30.0, slopes=True, causal=True)),
            (dtype, dict(B=1, S=700, heads=1, kv=1, dim=64, causal=True, prefix=[333], docs=documents(1, 700, 2), cap=20.0)),
            (dtype, dict(B=1, S=500, heads=6, kv=1, dim=128, slopes=True)),
            (dtype, dict(B=1, S=300, heads=2, kv=2, dim=64, common=4.0)),
        ]
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kw", cases(), ids=lambda v: v if isinstance(v, str) else "-".join(
    f"{k}{'' if isinstance(x, (np.ndarray, list)) or x is True else x}" for k, x in v.items()))
def test_against_the_formula(dtype, kw):
    s = make(dtype, **kw)
    check(s, run(s))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("how", ["rising", "falling", "steep", "uphill", "far", "negative", "zero", "capped", "capped_biased"])
def test_scores_of_every_range(dtype, dim, how):
    """Rows whose first block says nothing of what is to come: scores that rise or fall by hundreds along the keys, steep
    biases either way, keys that are all far away, scales that are not positive, caps beyond every score's range."""
    import torch
    n = 333
    kw = dict(rising={}, falling={}, steep=dict(slopes=True), uphill=dict(slopes=True, causal=True), far=dict(slopes=True, docs=(np.arange(n) % 300)[None]),
              negative=dict(causal=True), zero={}, capped=dict(cap=80.0), capped_biased=dict(cap=25.0, slopes=True, causal=True))[how]
    s = make(dtype, 1, n, 2, 1, dim, seed=9, **kw)
    if how in ("rising", "falling", "capped"):
        along = torch.linspace(0, 30, n, device="cuda")[None, :, None, None] * (-1 if how == "falling" else 1)
        s["q"] = (s["q"].float().abs() + 0.5).to(s["q"].dtype)
        s["k"] = (s["k"].float() * 0.3 + along / dim ** 0.5).to(s["k"].dtype)       # a row's scores run over some 150
    if how == "steep":
        s["mask"]["slopes"] = torch.tensor([30.0, 2.5], device="cuda")
    if how == "uphill":
        s["mask"]["slopes"] = torch.tensor([-1.0, -0.01], device="cuda")
    if how == "far":        # every document's tokens are 300 apart: all biases but the own token's are below -600
        s["mask"]["slopes"] = torch.tensor([2.0, 0.6], device="cuda")
    if how in ("negative", "zero"):
        s["scale"] = -0.2 if how == "negative" else 0.0
    # |scale| in the bounds
    sign = math.copysign(1.0, s["scale"])
    if sign < 0:
        ref = dict(s, q=-s["q"], scale=-s["scale"])
        out = run(s)
        check(ref, dict(out, dq=-out["dq"]))
    else:
        check(s, run(s))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_single_key_has_no_gradient_by_its_score(dtype, dim):
    import torch
    for kw in (dict(S=1), dict(S=150, docs=np.arange(150)[None].repeat(3, 0)), dict(S=70, lens=[1, 1, 1])):
        s = make(dtype, 3, heads=4, kv=2, dim=dim, slopes=True, **kw)
        out = run(s)
        assert not out["dq"].any() and not out["dk"].any()
        check(s, out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_layouts(dtype):
    """Heads before rows, padded rows on 16-byte boundaries only, and strides of single extents that nobody reads."""
    import torch
    s = make(dtype, 2, 140, 4, 2, 64, docs=documents(2, 140, 2))
    want = run(s)
    pad = 8 if dtype == "bf16" else 4

    def moved(x):      # [B, heads, S, dim + pad] storage, offset by 16 bytes
        b, n, h, d = x.shape
        store = torch.empty(b * h * n * (d + pad) + pad, dtype=x.dtype, device="cuda")[pad:]
        y = store.view(b, h, n, d + pad)[..., :d].transpose(1, 2)
        y.copy_(x)
        return y
    t = dict(s, **{k: moved(s[k]) for k in ("q", "k", "v", "dc")})
    got = run(t)
    for k in want:
        assert torch.equal(got[k], want[k]), k
    one = make(dtype, 1, 1, 1, 1, 64)
    odd = dict(one, **{k: one[k].as_strided((1, 1, 1, 64), (3, 5, 7, 1)) for k in ("q", "k", "v", "dc")})
    a, b = run(one), run(odd)
    for k in a:
        assert torch.equal(a[k], b[k]), k


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_many_short_and_empty_sequences(dtype, dim):
    """More row tiles than the device has SMs, most of them without a step."""
    lens = [(17 * i) % 150 if i % 3 == 0 else 0 for i in range(90)]
    s = make(dtype, 90, 140, 2, 1, dim, lens=lens, causal=True)
    check(s, run(s))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_evaluation_alone(dtype):
    """Without lse, as an evaluation calls it: the same context."""
    import torch
    from paper_2011_13635_b200 import binding as B
    s = make(dtype, 2, 300, 4, 2, 64, docs=documents(2, 300, 3), cap=20.0)
    out = run(s, backward=False, rest=False)
    check(s, out, rest=False)
    ctx = torch.empty_like(out["ctx"])
    B.mslt_op_attention_masked(s["q"], s["k"], s["v"], ctx, None, s["scale"], torch.zeros(1, dtype=torch.int32, device="cuda"), _stream(),
                               **s["mask"])
    assert torch.equal(ctx, out["ctx"])


@pytest.mark.gpu
def test_without_rest():
    s = make("bf16", 1, 200, 2, 2, 64, causal=True)
    check(s, run(s, rest=False), rest=False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_large_scores_and_lowest_values(dtype):
    """Scores of hundreds, where exponentials without the maximum overflow, and keys of the type's largest values."""
    import torch
    s = make(dtype, 1, 150, 2, 2, 64, causal=True)
    big = s["q"] * 30
    check(dict(s, q=big), run(dict(s, q=big)))
    k = s["k"].clone()
    k[:, 100:] = torch.finfo(k.dtype).max / 256           # seen by queries 100.. only
    out = run(dict(s, k=k), backward=False)
    ref = run(s, backward=False)
    assert torch.equal(out["ctx"][:, :100], ref["ctx"][:, :100])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradient_against_differences(dtype):
    """The loss sum(w ctx), moved along a direction of queries, keys and values.  bf16: two contexts within their bound
    of 2^-7 and the step's own rounding leave a few per cent of a slope that is far from zero."""
    import torch
    s = make(dtype, 1, 96, 2, 1, 64, docs=documents(1, 96, 2), slopes=True, cap=8.0)
    out = run(s)
    w = s["dc"].double()
    g = torch.Generator().manual_seed(5)
    step = 2.0 ** -7 if dtype == "fp32" else 2.0 ** -2
    for name in ("q", "k", "v"):
        d = out["d" + name].double()
        along = torch.sign(d)                                # where the loss grows fastest: its slope is sum |d|
        a = (s[name].double() + step * along).to(s[name].dtype)
        c = (s[name].double() - step * along).to(s[name].dtype)
        la, lc = ((run(dict(s, **{name: x}), backward=False)["ctx"].double() * w).sum() for x in (a, c))
        slope = float((d * (a.double() - c.double())).sum())
        assert abs(float(la - lc) - slope) < (0.02 if dtype == "fp32" else 0.08) * abs(slope), name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_same_bits_on_every_run_and_in_a_graph(dtype):
    import torch
    from paper_2011_13635_b200 import binding as B
    s = make(dtype, 2, 520, 4, 2, 64, docs=documents(2, 520, 5), lens=[520, 400], slopes=True, poison=False)
    a, b = run(s), run(s)
    for k in a:
        assert torch.equal(a[k], b[k]), k
    ctx, lse = torch.empty_like(a["ctx"]), torch.empty_like(a["lse"])
    grads = [torch.empty_like(x) for x in (s["q"], s["k"], s["v"])]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    scratch = torch.empty(B.mslt_op_attention_masked_bwd_scratch_bytes(2, 520, 4), dtype=torch.uint8, device="cuda")
    low = torch.empty_like(ctx) if dtype == "bf16" else None
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        st = torch.cuda.current_stream().cuda_stream
        B.mslt_op_attention_masked(s["q"], s["k"], s["v"], ctx, lse, s["scale"], status, st, rest=low, sync=False, **s["mask"])
        B.mslt_op_attention_masked_bwd(s["q"], s["k"], s["v"], ctx, lse, s["dc"], *grads, scratch, s["scale"], status, st, rest=low,
                                       sync=False, **s["mask"])
    for _ in range(2):
        ctx.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert int(status) == 0
        assert torch.equal(ctx, a["ctx"]) and torch.equal(lse, a["lse"])
        for got, k in zip(grads, ("dq", "dk", "dv")):
            assert torch.equal(got, a[k]), k


@pytest.mark.gpu
@pytest.mark.parametrize("dim,kw", [(64, {}), (64, dict(slopes=True, causal=True)), (128, dict(cap=15.0))])
def test_every_block_of_a_large_launch_ends(dim, kw):
    """Thousands of blocks with loops of all lengths, several times: a wait that misses its phase would run out (the call
    raises then), and one that is let through too early changes results between runs."""
    import torch
    s = make("bf16", 8, 2048, 12, 4, dim, docs=documents(8, 2048, 6), lens=[2048, 2000, 1, 64, 700, 2047, 1999, 129], **kw)
    first = run(s)
    for _ in range(5):
        again = run(s)
        for k in first:
            assert torch.equal(first[k], again[k]), k
    # the first six query heads of the first sequence by themselves: context and dq to the bit
    m = s["mask"]
    few = {k: v if not torch.is_tensor(v) else v[:6] if k == "slopes" else v[:1] for k, v in m.items()}
    got = run(dict(s, q=s["q"][:1, :, :6], dc=s["dc"][:1, :, :6], k=s["k"][:1, :, :2], v=s["v"][:1, :, :2], mask=few))
    for k in ("ctx", "dq"):
        assert torch.equal(got[k], first[k][:1, :, :6]), k


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,causal", [("fp32", False), ("bf16", False), ("bf16", True)])
def test_the_longest_row_with_offsets_beyond_32_bits(dtype, causal):
    """131072 tokens, 16416 elements apart: documents in the middle, at the end, and one of the first and last tokens."""
    import torch
    from paper_2011_13635_b200 import binding as B
    S, row, dim = 131072, 16416, 64
    t = torch.float32 if dtype == "fp32" else torch.bfloat16
    store = torch.empty(S, row, dtype=t, device="cuda")
    at = lambda i: store[:, row - (i + 1) * dim:row - i * dim].view(1, S, 1, dim)                            # noqa: E731
    names = ("q", "k", "v", "dc", "ctx", "low", "dq", "dk", "dv")
    x = {n: at(i) for i, n in enumerate(names)}
    assert (S - 1) * row > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(5)
    for n in names[:4]:
        x[n].copy_(torch.randn(1, S, 1, dim, generator=g, device="cuda"))
    docs = torch.arange(S, device="cuda", dtype=torch.int32) // 1000 + 10
    docs[:100] = docs[-72:] = 7
    low = x["low"] if dtype == "bf16" else None
    lse, status = torch.empty(1, 1, S, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    scratch = torch.empty(B.mslt_op_attention_masked_bwd_scratch_bytes(1, S, 1), dtype=torch.uint8, device="cuda")
    kw = dict(docs=docs[None], causal=causal, rest=low)
    B.mslt_op_attention_masked(x["q"], x["k"], x["v"], x["ctx"], lse, 0.125, status, _stream(), **kw)
    B.mslt_op_attention_masked_bwd(x["q"], x["k"], x["v"], x["ctx"], lse, x["dc"], x["dq"], x["dk"], x["dv"], scratch, 0.125, status,
                                   _stream(), **kw)
    for which in (75, 140, 7):
        rows = (docs == which).nonzero()[:, 0]
        part = {n: x[n][:, rows] for n in names}
        part.update(scale=0.125, mask=dict(cap=0.0, causal=causal, prefix=None, docs=None, lens=None, slopes=None))
        check(part, dict(ctx=part["ctx"], lse=lse[:, :, rows], dq=part["dq"], dk=part["dk"], dv=part["dv"]))


@pytest.mark.gpu
def test_the_longest_row_whole():
    """Every key of 131072 seen by every query: context, lse and dq of a few queries."""
    import torch
    S, dim = 131072, 64
    s = make("bf16", 1, S, 1, 1, dim)
    out = run(s)
    rows = [0, 1, 65535, 65536, S - 1]
    D = lambda v: v[0, :, 0].double()                                                                       # noqa: E731
    q, k, v, dc = D(s["q"])[rows], D(s["k"]), D(s["v"]), D(s["dc"])[rows]
    z = q @ k.T * 0.125
    p, lse = torch.softmax(z, -1), torch.logsumexp(z, -1)
    u = 2.0 ** -8
    # scores as in `check`; a row's sum has 2 x 65536 terms added one after the other
    e_row = ((dim + 8) * F32 * (q.abs() @ k.abs().T) * 0.125 + 4 * F32 * z.abs()).amax(-1) + 2.0 ** -21 + S * F32
    assert ((out["lse"][0, 0, rows] - lse).abs() <= e_row + 4 * F32 * (lse.abs() + z.amax(-1).abs())).all()
    rel = (2 * u * u + 2 * e_row)[:, None]
    o, big = p @ v, p @ v.abs()
    assert ((D(out["ctx"])[rows] - o).abs() <= (rel + S * F32) * big + u * o.abs()).all()
    dp = dc @ v.T
    delta = (p * dp).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    e_delta = ((rel + S * F32) * (dc.abs() * big).sum(-1, keepdim=True) + (2.0 ** -16 + (dim + 8) * F32) * (dc.abs() * o.abs()).sum(-1, keepdim=True))
    e_ds = p * ((dp - delta).abs() * 2 * e_row[:, None] + (dim + 8) * F32 * (dc.abs() @ v.abs().T) + e_delta) + u * ds.abs()
    dq = ds @ k * 0.125
    assert ((D(out["dq"])[rows] - dq).abs() <= 0.125 * (1.01 * e_ds @ k.abs() + S * F32 * (ds.abs() @ k.abs())) + u * dq.abs()).all()


@pytest.mark.gpu
def test_a_wait_that_runs_out_is_reported():
    """The producer of the next launch issues no copies: status after 20 ms, and the device stays usable."""
    import torch
    from paper_2011_13635_b200 import binding as B
    s = make("bf16", 2, 300, 4, 2, 64)
    want = run(s)
    B.lib.mslt_debug_starve_next_attention(1)
    with pytest.raises(B.MsltError) as e:
        run(s, backward=False)
    assert e.value.code == -5
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    grads = [torch.empty_like(s[k]) for k in ("q", "k", "v")]
    scratch = torch.empty(B.mslt_op_attention_masked_bwd_scratch_bytes(2, 300, 4), dtype=torch.uint8, device="cuda")
    B.lib.mslt_debug_starve_next_attention(1)
    with pytest.raises(B.MsltError) as e:
        B.mslt_op_attention_masked_bwd(s["q"], s["k"], s["v"], want["ctx"], want["lse"], s["dc"], *grads, scratch, s["scale"], status,
                                       _stream())
    assert e.value.code == -5
    again = run(s)
    assert all(torch.equal(again[k], want[k]) for k in want)


@pytest.mark.gpu
def test_two_streams_at_once():
    """Two calls that may run side by side, each with its own scratch."""
    import torch
    s = [make("bf16", 2, 300, 4, 4, 64, seed=i, causal=bool(i)) for i in range(2)]
    want = [run(x, backward=False, rest=False) for x in s]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    from paper_2011_13635_b200 import binding as B
    got = []
    for x, st in zip(s, streams):
        ctx, lse = torch.zeros_like(x["q"].contiguous()), torch.zeros(2, 4, 300, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        got.append((ctx, status, lse))          # the allocator knows nothing of the other stream: kept until it is done
        for _ in range(20):
            B.mslt_op_attention_masked(x["q"], x["k"], x["v"], ctx, lse, x["scale"], status, st.cuda_stream, sync=False, **x["mask"])
    torch.cuda.synchronize()
    for (ctx, status, _), w in zip(got, want):
        assert int(status) == 0 and torch.equal(ctx, w["ctx"])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_layer_from_projection_to_gradient(dtype):
    """Norm and rotation, attention under documents, and back to the gradients of the projection's output and the gains,
    as a training step runs them, against autograd in 64 bits on the same chain.  The bound is relative to each result's
    norm: bf16 rounds seven times on the way (2^-8 each at most, none of them in the same direction), fp32 at dim = 64."""
    import torch
    from paper_2011_13635_b200 import binding as B
    t = torch.float32 if dtype == "fp32" else torch.bfloat16
    nb, n, heads, kv, dim, eps = 2, 200, 4, 2, 64, 1e-6
    g = torch.Generator().manual_seed(4)
    fused = torch.randn(nb * n, heads + 2 * kv, dim, generator=g).to(t).cuda()
    gain = (1 + 0.1 * torch.randn(2, dim, generator=g)).cuda()
    dctx = torch.randn(nb, n, heads, dim, generator=g).to(t).cuda()
    docs = torch.from_numpy(documents(nb, n, 3).astype(np.int32)).cuda()
    turns, m = B.mslt_rope_turns(dim)
    turns = torch.from_numpy(turns.view(np.int64)).cuda()
    st = _stream()
    qk = torch.empty(nb * n, heads + kv, dim, dtype=t, device="cuda")
    B.mslt_op_qk_norm_rope(fused[:, :heads + kv], qk, gain, turns, heads, eps, st, seq=n, sync=False)
    view = lambda x, a, b: x.view(nb, n, -1, dim)[:, :, a:b]                                               # noqa: E731
    q, k, v = view(qk, 0, heads), view(qk, heads, heads + kv), view(fused, heads + kv, heads + 2 * kv)
    ctx, lse = torch.empty(nb, n, heads, dim, dtype=t, device="cuda"), torch.empty(nb, heads, n, device="cuda")
    low = torch.empty_like(ctx) if dtype == "bf16" else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mslt_op_attention_masked(q, k, v, ctx, lse, dim ** -0.5, status, st, docs=docs, rest=low, sync=False)
    grad = torch.empty_like(fused)
    scratch = torch.empty(max(B.mslt_op_attention_masked_bwd_scratch_bytes(nb, n, heads),
                              B.mslt_op_qk_norm_rope_bwd_scratch_bytes(nb * n, heads + kv, dim)), dtype=torch.uint8, device="cuda")
    B.mslt_op_attention_masked_bwd(q, k, v, ctx, lse, dctx, view(grad, 0, heads), view(grad, heads, heads + kv),
                                   view(grad, heads + kv, heads + 2 * kv), scratch, dim ** -0.5, status, st, docs=docs, rest=low, sync=False)
    dgain = torch.empty(2, dim, device="cuda")
    turned = grad[:, :heads + kv]
    B.mslt_op_qk_norm_rope_bwd(turned, fused[:, :heads + kv], turned, gain, dgain, turns, heads, eps, scratch, st, seq=n)
    assert int(status) == 0

    x = fused.double().requires_grad_()
    gd = gain.double().requires_grad_()
    y = x[:, :heads + kv]
    y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * gd[(torch.arange(heads + kv, device="cuda") >= heads).long()]
    f = 10000.0 ** (-2.0 * torch.arange(dim // 2, dtype=torch.float64, device="cuda") / dim)
    a = ((torch.arange(nb * n, device="cuda") % n).double()[:, None] * f)[:, None]
    u, w = y[..., :dim // 2], y[..., dim // 2:]
    y = torch.cat([u * torch.cos(a) - w * torch.sin(a), u * torch.sin(a) + w * torch.cos(a)], -1).view(nb, n, heads + kv, dim)
    K = y[:, :, heads:].repeat_interleave(heads // kv, 2)
    V = x[:, heads + kv:].view(nb, n, kv, dim).repeat_interleave(heads // kv, 2)
    z = torch.einsum("bihe,bjhe->bhij", y[:, :, :heads], K) * dim ** -0.5
    z = z.masked_fill(~(docs[:, None, :, None] == docs[:, None, None, :]), -math.inf)
    o = torch.einsum("bhij,bjhe->bihe", torch.softmax(z, -1), V)
    want = torch.autograd.grad(o, [x, gd], dctx.double())
    tol = 7 * 2.0 ** -8 if dtype == "bf16" else 1e-5
    for got, ref in ((ctx, o.detach()), (grad, want[0]), (dgain, want[1])):
        assert float((got.double() - ref).norm() / ref.norm()) < tol


def desc(bd, **change):
    h = lambda: bd.Heads(4096, 65536, 256, 64)                                                              # noqa: E731
    d = bd.AttentionDesc(dtype=1, B=2, S=128, heads=4, kv_heads=4, head_dim=64, q=h(), k=h(), v=h(), ctx=h(), lse=4096, dctx=h(), dq=h(),
                        dk=h(), dv=h(), scale=0.125)
    for k, v in change.items():
        if "." in k:
            a, b = k.split(".")
            setattr(getattr(d, a), b, v)
        else:
            setattr(d, k, v)
    return d


BAD = [dict(dtype=2), dict(B=0), dict(S=0), dict(heads=0), dict(kv_heads=3), dict(kv_heads=0), dict(head_dim=60), dict(head_dim=136),
       dict(head_dim=0), dict(scale=float("nan")), dict(cap=-1.0), dict(cap=float("inf")), dict(prefix=4096), dict(rest=4104),
       dict(dtype=0, rest=4096)] + [{f"{t}.{f}": v} for t in ("q", "k", "v", "ctx") for f, v in
                                    (("data", None), ("data", 4104), ("row", 60), ("head", 4), ("batch", -64))]


def test_refusals_before_any_device():
    from paper_2011_13635_b200 import binding as B
    fwd = lambda d: B.lib.mslt_op_attention_masked(B.C.byref(d), 4096, None, 1)                             # noqa: E731
    size = B.mslt_op_attention_masked_bwd_scratch_bytes(2, 128, 4)
    assert size >= 2 * 128 * 4 * 4
    bwd = lambda d, at=4096, n=size: B.lib.mslt_op_attention_masked_bwd(B.C.byref(d), at, n, 4096, None, 1)  # noqa: E731
    for change in BAD:
        assert fwd(desc(B, **change)) == -1, change
        assert bwd(desc(B, **change)) == -1, change
    for t in ("dctx", "dq", "dk", "dv"):
        for f, v in (("data", None), ("data", 4104), ("row", 60)):
            assert bwd(desc(B, **{f"{t}.{f}": v})) == -1
    assert bwd(desc(B, lse=None)) == -1
    assert fwd(desc(B, S=131073)) == -2 and fwd(desc(B, B=1 << 20, S=65536)) == -2
    assert bwd(desc(B), n=size - 1) == -2 and bwd(desc(B), at=None) == -2 and bwd(desc(B), at=4104) == -2
    assert B.lib.mslt_op_attention_masked(None, 4096, None, 1) == -1
    assert B.lib.mslt_op_attention_masked(B.C.byref(desc(B)), None, None, 1) == -1


def test_refusals_of_strides_and_ranges():
    """Broadcast inputs, outputs whose elements share memory, sizes past the row counters, caps that fp32 cannot turn over."""
    from paper_2011_13635_b200 import binding as B
    fwd = lambda d: B.lib.mslt_op_attention_masked(B.C.byref(d), 4096, None, 1)                             # noqa: E731
    size = B.mslt_op_attention_masked_bwd_scratch_bytes(2, 128, 4)
    bwd = lambda d: B.lib.mslt_op_attention_masked_bwd(B.C.byref(d), 4096, size, 4096, None, 1)              # noqa: E731
    for dtype in (0, 1):
        for f in ("batch", "row", "head"):
            for t in ("q", "k", "v", "ctx"):
                assert fwd(desc(B, dtype=dtype, **{f"{t}.{f}": 0})) == -1 and bwd(desc(B, dtype=dtype, **{f"{t}.{f}": 0})) == -1, (t, f)
            for t in ("dctx", "dq", "dk", "dv"):
                assert bwd(desc(B, dtype=dtype, **{f"{t}.{f}": 0})) == -1, (t, f)
            for t in ("dq", "dk", "dv"):
                assert bwd(desc(B, dtype=dtype, **{f"{t}.{f}": 56})) == -1, (t, f)
            assert fwd(desc(B, dtype=dtype, **{f"ctx.{f}": 56})) == -1, f
        for change in (dict(cap=1e-20), dict(cap=1e20), dict(cap=1e-3, scale=1e17), dict(cap=1.0, scale=1e-20), dict(cap=1.0, scale=-1e20)):
            assert fwd(desc(B, dtype=dtype, **change)) == -1, change
        assert fwd(desc(B, dtype=dtype, B=1 << 28, S=1, heads=8)) == -2


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kw", [dict(cap=1e-12), dict(cap=1e6), dict(cap=1e-12, slopes=True), dict(cap=5.0, zero_scale=True)], ids=str)
def test_caps_far_from_the_scores(dtype, kw):
    """Far below, every score but those of zero queries is at its cap; far above, the cap does nothing; scale 0: all alike."""
    kw = dict(kw)
    zero = kw.pop("zero_scale", False)
    s = make(dtype, 1, 200, 2, 1, 64, causal=True, **kw)
    s["q"][:, 5:9] = 0
    if zero:
        s["scale"] = 0.0
    check(s, run(s))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kw", [{}, dict(slopes=True), dict(cap=20.0)], ids=str)
def test_nan_that_is_seen_comes_through(dtype, dim, kw):
    """A NaN in a query or a key is not passed over as a row that sees nothing."""
    import torch
    for name in ("q", "k"):
        s = make(dtype, 2, 300, 2, 2, dim, causal=True, **kw)
        s[name][0, 150, 1, 3] = float("nan")
        out = run(s)
        bad = torch.isnan(out["ctx"]).all(-1)[0, :, 1]
        want = torch.zeros(300, dtype=torch.bool, device="cuda")
        want[150 if name == "q" else slice(150, None)] = True
        if name == "q":
            want[151:] = False
        assert torch.equal(bad, want) and torch.equal(torch.isnan(out["ctx"])[0, :, 1].any(-1), want)
        assert torch.equal(torch.isnan(out["lse"])[0, 1], want)
        assert torch.isnan(out["dq"][0, :, 1][want]).all()
        assert torch.isnan(out["dk"][0, :150, 1]).all() and torch.isnan(out["dv"][0, :150, 1]).all()
        for k in ("ctx", "dq", "dk", "dv"):
            assert not torch.isnan(out[k][1]).any() and not torch.isnan(out[k][0, :, 0]).any(), k


@pytest.mark.gpu
def test_binding_refusals():
    import torch
    from paper_2011_13635_b200 import binding as B
    s = make("bf16", 2, 32, 4, 2, 64)
    ctx, lse, status = torch.empty_like(s["q"].contiguous()), torch.empty(2, 4, 32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

    def call(q=s["q"], k=s["k"], v=s["v"], ctx=ctx, lse=lse, **kw):
        B.mslt_op_attention_masked(q, k, v, ctx, lse, 0.125, status, _stream(), **kw)
    call()
    i = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")                                # noqa: E731
    for kw in (dict(k=s["k"][:, :31]), dict(v=s["v"].float()), dict(q=s["q"].float()), dict(ctx=ctx[:1]), dict(lse=lse[:, :, :3]),
               dict(lse=lse.double()), dict(docs=i(2, 31)), dict(lens=i(3)), dict(prefix=i(2)), dict(lens=i(2).long()),
               dict(slopes=torch.zeros(3, device="cuda")), dict(rest=ctx.float()), dict(k=s["k"].repeat(1, 1, 2, 1)[:, :, :3], v=s["v"].repeat(1, 1, 2, 1)[:, :, :3]),
               dict(q=s["q"].transpose(1, 3)), dict(docs=i(2, 64)[:, ::2])):
        with pytest.raises(B.MsltError) as e:
            call(**kw)
        assert e.value.code == -1, kw.keys()
    with pytest.raises(B.MsltError) as e:
        call(q=s["q"].cpu())
    assert e.value.code == -4
