"""Rotary positions and the norm of query and key heads against their formulas in 64 bits."""
import math

import numpy as np
import pytest

U = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}   # half a step, relative


def _dt(name):
    import torch
    return torch.float32 if name == "fp32" else torch.bfloat16


def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, trained=512):
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2.0 * np.arange(rot // 2) / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":
        g = np.clip((trained * f / (2 * math.pi) - 1) / 31, 0, 1)
        f = f * g + f / factor * (1 - g)
    return f, 0.1 * math.log(factor) + 1 if scaling == "by_parts" else 1.0


def rotated(x, pos, f, m, interleaved, back=False):
    """x [rows, heads, dim] float64 tensor on the CPU."""
    import torch
    rot = 2 * len(f)
    a = torch.from_numpy(np.multiply.outer(pos.astype(np.float64), f))[:, None]
    c, s = torch.cos(a) * m, torch.sin(a) * m * (-1 if back else 1)
    y = x.clone()
    u = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    w = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    y[..., u] = x[..., u] * c - x[..., w] * s
    y[..., w] = x[..., u] * s + x[..., w] * c
    return y


def partner_size(x, rot, interleaved):
    """|x| + |its partner|: what the absolute error of a rotation is in proportion to; 0 where nothing turns."""
    import torch
    a, out = x.abs(), torch.zeros_like(x)
    u = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    w = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    out[..., u] = out[..., w] = a[..., u] + a[..., w]
    return out


# Absolute error of a cosine or sine.  fp32: the turn rounded to 24 bits (2 pi 2^-25), 2 units of the library's function,
# two products and a sum (3 x 2^-24).  bf16: the hardware's 2^-20.9 on [-pi, pi], its argument's rounding (pi 2^-23), the same.
ANGLE = {"fp32": 2 * math.pi * 2.0 ** -25 + 5 * 2.0 ** -24, "bf16": 2.0 ** -20.9 + math.pi * 2.0 ** -23 + 4 * 2.0 ** -24}


def plan(rot, **kw):
    import torch
    from paper_2011_13635_b200 import binding as B
    turns, m = B.mslt_rope_turns(rot, **kw)
    return torch.from_numpy(turns.view(np.int64)).cuda(), m


def test_turns_are_the_frequencies():
    from paper_2011_13635_b200 import binding as B
    for rot in (8, 64, 120, 128):
        for scaling, factor in (("none", 1.0), ("linear", 4.0), ("ntk", 8.0), ("by_parts", 16.0)):
            turns, m = B.mslt_rope_turns(rot, 10000.0, scaling, factor, 512)
            f, want_m = frequencies(rot, scaling=scaling, factor=factor)
            got = turns.astype(np.float64) / 2.0 ** 64 * 2 * math.pi
            # half a step of 2^-64 turn is 2^-65 2 pi of an f as small as 6e-6: more than the 1e-14 of a few roundings of a double
            assert (np.abs(got - f) <= 1e-14 * f + 2.0 ** -65 * 2 * math.pi).all()
            assert abs(m - want_m) < 1e-6


def test_turns_refusals():
    from paper_2011_13635_b200 import binding as B
    for kw in (dict(rot_dim=12), dict(rot_dim=0), dict(rot_dim=136), dict(rot_dim=64, base=1.0), dict(rot_dim=64, factor=0.5),
               dict(rot_dim=64, base=float("nan")), dict(rot_dim=64, scaling="cubic"),
               dict(rot_dim=64, scaling="by_parts", factor=2.0, trained_len=0)):
        with pytest.raises(B.MsltError) as e:
            B.mslt_rope_turns(**kw)
        assert e.value.code == -1


def test_refusals_before_any_device():
    """Descriptors that the library refuses on the host, whatever the machine."""
    from paper_2011_13635_b200 import binding as B
    good = dict(dtype=1, rows=4, heads=2, head_dim=64, x=4096, x_row=128, x_head=64, y=8192, y_row=128, y_head=64, positions=None,
                seq=4, rot_dim=64, interleaved=0, turns=16384, magnitude=1.0, inverse=0)

    def rc(fn, wrap=None, **change):
        d = B.RopeDesc(**dict(good, **change))
        if wrap is None:
            return fn(B.C.byref(d), None, 1)
        n = B.QkNormDesc(rope=d, **dict(dict(q_heads=1, center=0, eps=1e-6, gain=32768, dy=4096, dy_row=128, dy_head=64, dx=4096,
                                             dx_row=128, dx_head=64, dgain=32768), **wrap))
        return fn(n)

    bad = [dict(dtype=2), dict(rows=0), dict(heads=0), dict(head_dim=60), dict(head_dim=136), dict(rot_dim=12), dict(rot_dim=72),
           dict(rot_dim=0), dict(x=None), dict(x=4098), dict(y=None), dict(y_row=4), dict(x_head=3), dict(x_row=-8), dict(turns=None),
           dict(turns=8), dict(seq=0), dict(magnitude=float("inf"))]
    for change in bad:
        assert rc(B.lib.mslt_op_rope, **change) == -1, change
    assert rc(B.lib.mslt_op_rope, heads=5000) == -2 and rc(B.lib.mslt_op_rope, rows=(1 << 30) + 1) == -2
    assert B.lib.mslt_op_rope(None, None, 1) == -1
    size = B.mslt_op_qk_norm_rope_bwd_scratch_bytes(4, 2, 64)
    fwd = lambda n: B.lib.mslt_op_qk_norm_rope(B.C.byref(n), None, 1)                                       # noqa: E731
    bwd = lambda n: B.lib.mslt_op_qk_norm_rope_bwd(B.C.byref(n), 65536, size, None, 1)                      # noqa: E731
    for wrap in (dict(q_heads=3), dict(q_heads=-1), dict(eps=0.0), dict(eps=float("nan")), dict(gain=None)):
        assert rc(fwd, wrap) == -1 and rc(bwd, wrap) == -1, wrap
    assert rc(fwd, {}, inverse=1) == -1 and rc(fwd, {}, y=None) == -1
    for wrap in (dict(dy=None), dict(dx=None), dict(dgain=None), dict(dx_row=4), dict(dy=4098)):
        assert rc(bwd, wrap) == -1, wrap
    for at, n in ((65536, size - 1), (65544, size), (None, size)):
        assert rc(lambda d: B.lib.mslt_op_qk_norm_rope_bwd(B.C.byref(d), at, n, None, 1), {}) == -2


def test_refusals_of_outputs_that_share_memory():
    from paper_2011_13635_b200 import binding as B
    good = dict(dtype=1, rows=4, heads=2, head_dim=64, x=4096, x_row=128, x_head=64, y=8192, y_row=128, y_head=64, seq=4, rot_dim=64,
                turns=16384, magnitude=1.0)
    size = B.mslt_op_qk_norm_rope_bwd_scratch_bytes(4, 2, 64)
    for field in ("row", "head"):
        for stride in (0, 56):
            d = B.RopeDesc(**dict(good, **{f"y_{field}": stride}))
            n = B.QkNormDesc(rope=d, q_heads=1, eps=1e-6, gain=32768)
            assert B.lib.mslt_op_rope(B.C.byref(d), None, 1) == -1 and B.lib.mslt_op_qk_norm_rope(B.C.byref(n), None, 1) == -1
            n = B.QkNormDesc(rope=B.RopeDesc(**good), q_heads=1, eps=1e-6, gain=32768, dgain=32768,
                             **dict(dict(dy=4096, dy_row=128, dy_head=64, dx=4096, dx_row=128, dx_head=64), **{f"dx_{field}": stride}))
            assert B.lib.mslt_op_qk_norm_rope_bwd(B.C.byref(n), 65536, size, None, 1) == -1


CASES = [  # dtype, rows, heads, dim, rot, interleaved
    ("bf16", 1, 1, 64, 64, False), ("bf16", 5, 3, 64, 64, True), ("bf16", 33, 24, 64, 32, False), ("bf16", 700, 7, 128, 128, False),
    ("bf16", 9, 5, 96, 24, False), ("bf16", 13, 2, 8, 8, False), ("bf16", 13, 2, 72, 72, False), ("bf16", 64, 9, 40, 40, True),
    ("bf16", 3, 70, 16, 16, False), ("fp32", 1, 1, 64, 64, True), ("fp32", 31, 12, 64, 16, False), ("fp32", 257, 3, 128, 128, False),
    ("fp32", 10, 4, 24, 24, False), ("fp32", 10, 40, 8, 8, True), ("fp32", 2500, 6, 96, 48, True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,heads,dim,rot,interleaved", CASES)
@pytest.mark.parametrize("how", ["plain", "in_place", "far", "back"])
def test_rope(dtype, rows, heads, dim, rot, interleaved, how):
    import torch
    from paper_2011_13635_b200 import binding as B
    g = torch.Generator().manual_seed(rows * 31 + dim)
    wide = torch.randn(rows, heads + 2, dim, generator=g).to(_dt(dtype)).cuda()
    keep = wide.clone()
    x = wide[:, 1:1 + heads]
    turns, m = plan(rot, scaling="by_parts", factor=8.0) if how == "far" else plan(rot)
    f, want_m = frequencies(rot, scaling="by_parts", factor=8.0) if how == "far" else frequencies(rot)
    pos = np.random.default_rng(3).integers(-2 ** 31, 2 ** 31, rows) if how == "far" else np.arange(rows) % 7
    kw = dict(positions=torch.from_numpy(pos.astype(np.int32)).cuda()) if how == "far" else dict(seq=7)
    y = x if how == "in_place" else torch.full((rows, heads, dim), 7.0, dtype=x.dtype, device="cuda")
    B.mslt_op_rope(x, y, turns, _stream(), interleaved=interleaved, magnitude=m, inverse=how == "back", **kw)
    ref = rotated(keep[:, 1:1 + heads].double().cpu(), pos, f, want_m, interleaved, how == "back")
    size = partner_size(keep[:, 1:1 + heads].double().cpu(), rot, interleaved)
    # the table's frequency is a double: 2^-53 of the angle, in the reference too
    angle = ANGLE[dtype] + (np.abs(pos).max() * 2.0 ** -51 if how == "far" else 0)
    tol = (ref.abs() * U[dtype] + 1.01 * want_m * angle * size) * (1 + 1e-6)
    tol[..., rot:] = 0                                            # what is not turned is copied
    assert ((y.double().cpu() - ref).abs() <= tol).all()
    assert torch.equal(wide[:, 0], keep[:, 0]) and torch.equal(wide[:, -1], keep[:, -1])


@pytest.mark.gpu
def test_rope_back_undoes_rope_and_keeps_distances():
    """Rotation is orthogonal, and scores of rotated queries and keys depend on the distance of their positions."""
    import torch
    from paper_2011_13635_b200 import binding as B
    turns, m = plan(64)
    x = torch.randn(64, 2, 64, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    B.mslt_op_rope(x, y, turns, _stream(), seq=64)
    B.mslt_op_rope(y, z, turns, _stream(), seq=64, inverse=True)
    assert (z - x).abs().max() <= 4 * ANGLE["fp32"] * 2 * x.abs().max()
    q = x[:1, :1].expand(64, 1, 64).contiguous()
    a, b = torch.empty_like(q), torch.empty_like(q)
    p = torch.arange(64, device="cuda", dtype=torch.int32)
    B.mslt_op_rope(q, a, turns, _stream(), positions=p)
    B.mslt_op_rope(q, b, turns, _stream(), positions=p + 100000)
    d0, d1 = (a[5] * a[20]).sum(), (b[5] * b[20]).sum()
    assert abs(float(d0 - d1)) <= 64 * 4 * ANGLE["fp32"] * float((q[0] ** 2).max()) * 2


NORM = [c for c in CASES if c[1] * c[2] < 5000] + [("bf16", 50, 6, 64, 0, False), ("fp32", 4000, 3, 64, 64, False),
                                                    ("bf16", 9001, 4, 32, 16, True)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,heads,dim,rot,interleaved", NORM)
@pytest.mark.parametrize("center", [False, True])
def test_qk_norm_rope_and_gradient(dtype, rows, heads, dim, rot, interleaved, center):
    import torch
    from paper_2011_13635_b200 import binding as B
    g = torch.Generator().manual_seed(rows + heads)
    q_heads = heads // 2
    eps = 1e-6
    x = (torch.randn(rows, heads + 1, dim, generator=g) * 2 + 0.5).to(_dt(dtype)).cuda()[:, :heads]
    dy = torch.randn(rows, heads, dim, generator=g).to(_dt(dtype)).cuda()
    gain = (1 + 0.3 * torch.randn(2, dim, generator=g)).cuda()
    bias = 0.2 * torch.randn(2, dim, generator=g).cuda() if center else None
    pos = np.random.default_rng(rows).integers(0, 5000, rows)
    turns, m = plan(rot) if rot else (None, 1.0)
    f = frequencies(rot)[0] if rot else np.zeros(0)
    kw = dict(center=center, positions=torch.from_numpy(pos.astype(np.int32)).cuda(), interleaved=interleaved)
    y = torch.empty(rows, heads, dim, dtype=x.dtype, device="cuda")
    B.mslt_op_qk_norm_rope(x, y, gain, turns, q_heads, eps, _stream(), bias=bias, **kw)

    which = (torch.arange(heads) >= q_heads).long()
    xd = x.double().cpu().requires_grad_()
    gd = gain.double().cpu().requires_grad_()
    bd = bias.double().cpu().requires_grad_() if center else None
    c = xd - xd.mean(-1, keepdim=True) if center else xd
    xh = c / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
    n = xh * gd[which] + (bd[which] if center else 0)
    ref = rotated(n, pos, f, 1.0, interleaved) if rot else n
    # statistics: sums of dim terms in fp32 (dim + 4 roundings), a root and a division; a mean's error is relative to |x|
    stat = (dim + 8) * 2.0 ** -24
    large = (x.double().cpu().abs().amax(-1, keepdim=True) / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)).detach()
    e_xh = stat * (xh.detach().abs() + large)
    e_n = e_xh * gd.detach()[which].abs() + 2.0 ** -23 * n.detach().abs()
    spread = partner_size(e_n, rot, interleaved) if rot else e_n
    e_y = torch.maximum(e_n, spread) + (ANGLE[dtype] * partner_size(n.detach(), rot, interleaved) if rot else 0)
    assert ((y.double().cpu() - ref.detach()).abs() <= U[dtype] * ref.detach().abs() + 1.05 * e_y).all()

    want = torch.autograd.grad(ref, [xd, gd] + ([bd] if center else []), dy.double().cpu())
    dgain = torch.full((2, dim), 3.0, device="cuda")
    dbias = torch.full((2, dim), 3.0, device="cuda") if center else None
    scratch = torch.full((B.mslt_op_qk_norm_rope_bwd_scratch_bytes(rows, heads, dim),), 255, dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(dy)
    B.mslt_op_qk_norm_rope_bwd(dy, x, dx, gain, dgain, turns, q_heads, eps, scratch, _stream(), dbias=dbias, **kw)
    gr = rotated(dy.double().cpu(), pos, f, 1.0, interleaved, True) if rot else dy.double().cpu()
    e_g = (ANGLE[dtype] * partner_size(dy.double().cpu(), rot, interleaved) if rot else 0) + 2.0 ** -23 * gr.abs()
    r = 1 / torch.sqrt((c.detach() ** 2).mean(-1, keepdim=True) + eps)
    h = gr * gd.detach()[which]
    e_h = e_g * gd.detach()[which].abs() + 2.0 ** -23 * h.abs()
    xa = xh.detach().abs()
    mean = lambda t: t.mean(-1, keepdim=True)                                                               # noqa: E731
    e_dx = r * (e_h + mean(e_h) + stat * mean(h.abs()) + xa * (mean(e_h * xa) + mean(h.abs() * e_xh) + stat * mean(h.abs() * xa))
                + e_xh * mean(h * xh.detach()).abs() + 2 * stat * (h.abs() + xa * mean(h.abs() * xa)))
    assert ((dx.double().cpu() - want[0]).abs() <= U[dtype] * want[0].abs() + 1.05 * e_dx).all()
    # a lane adds at most rows / warps terms in a row, then 8 warps and 32 groups: below 600 roundings here
    chain = 600 * 2.0 ** -24
    by = lambda t: torch.stack([t[:, :q_heads].sum((0, 1)), t[:, q_heads:].sum((0, 1))])                    # noqa: E731
    e_gain = by(e_g * xa + gr.abs() * e_xh + chain * (gr * xh.detach()).abs())
    assert ((dgain.double().cpu() - want[1]).abs() <= 1.05 * e_gain + 1e-30).all()
    if center:
        assert ((dbias.double().cpu() - want[2]).abs() <= 1.05 * by(e_g + chain * gr.abs()) + 1e-30).all()
    # dx over dy, and the same bits
    again, dgain2 = dy.clone(), torch.empty_like(dgain)
    B.mslt_op_qk_norm_rope_bwd(again, x, again, gain, dgain2, turns, q_heads, eps, scratch, _stream(), **kw)
    assert torch.equal(again, dx) and torch.equal(dgain2, dgain)


@pytest.mark.gpu
def test_norm_gradient_against_differences():
    import torch
    from paper_2011_13635_b200 import binding as B
    rows, heads, dim = 4, 3, 16
    g = torch.Generator().manual_seed(8)
    x = torch.randn(rows, heads, dim, generator=g).cuda()
    w = torch.randn(rows, heads, dim, generator=g).cuda()
    gain = torch.ones(2, dim, device="cuda") + 0.1
    turns, _ = plan(16)
    dx, dgain = torch.empty_like(x), torch.empty(2, dim, device="cuda")
    scratch = torch.empty(B.mslt_op_qk_norm_rope_bwd_scratch_bytes(rows, heads, dim), dtype=torch.uint8, device="cuda")
    B.mslt_op_qk_norm_rope_bwd(w, x, dx, gain, dgain, turns, 2, 1e-6, scratch, _stream(), center=True, seq=4)

    def loss(x):
        y = torch.empty_like(x)
        B.mslt_op_qk_norm_rope(x, y, gain, turns, 2, 1e-6, _stream(), center=True, seq=4)
        return float((y.double() * w.double()).sum())
    step = 2.0 ** -6
    for at in [(0, 0, 0), (1, 1, 7), (2, 2, 15), (3, 0, 8)]:
        a, b = x.clone(), x.clone()
        a[at] += step
        b[at] -= step
        got = (loss(a) - loss(b)) / (2 * step)
        # third derivative of a normalised element (order 10) times step^2 / 6, and 48 fp32 roundings over 2 step
        assert abs(got - float(dx[at])) < 10 * step * step / 6 * 3 + 48 * 2.0 ** -24 * 4 / (2 * step) + 1e-3


@pytest.mark.gpu
def test_captured_on_a_side_stream_and_replayed():
    import torch
    from paper_2011_13635_b200 import binding as B
    turns, _ = plan(64)
    x = torch.randn(300, 6, 64, device="cuda").bfloat16()
    y, gain = torch.empty_like(x), torch.ones(2, 64, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.mslt_op_qk_norm_rope(x, y, gain, turns, 3, 1e-6, torch.cuda.current_stream().cuda_stream, seq=100, sync=False)
    x.copy_(torch.randn(300, 6, 64, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    z = torch.empty_like(x)
    B.mslt_op_qk_norm_rope(x, z, gain, turns, 3, 1e-6, _stream(), seq=100)
    assert torch.equal(y, z)


@pytest.mark.gpu
def test_rope_offsets_beyond_32_bits():
    """Heads that lie more than 2^31 elements apart."""
    import torch
    from paper_2011_13635_b200 import binding as B
    gap = (1 << 31) + 4096
    big = torch.empty(gap + 64 * 64, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((64, 2, 64), (64, gap, 1))
    src = torch.randn(64, 2, 64, device="cuda").bfloat16()
    x.copy_(src)
    turns, _ = plan(64)
    y, z = torch.empty_like(src), torch.empty_like(src)
    B.mslt_op_rope(x, y, turns, _stream(), seq=64)
    B.mslt_op_rope(src, z, turns, _stream(), seq=64)
    assert torch.equal(y, z)


@pytest.mark.gpu
def test_binding_refusals():
    import torch
    from paper_2011_13635_b200 import binding as B
    turns, _ = plan(64)
    x = torch.zeros(4, 2, 64, device="cuda")
    gain = torch.ones(2, 64, device="cuda")
    y = torch.empty_like(x)
    for call in (lambda: B.mslt_op_rope(x, y[:3], turns, _stream(), seq=4), lambda: B.mslt_op_rope(x, y.bfloat16(), turns, _stream(), seq=4),
                 lambda: B.mslt_op_rope(x.half(), y.half(), turns, _stream(), seq=4),
                 lambda: B.mslt_op_rope(x.transpose(1, 2), y.transpose(1, 2), turns, _stream(), seq=4),
                 lambda: B.mslt_op_rope(x, y, turns.int(), _stream(), seq=4), lambda: B.mslt_op_rope(x, y, turns, _stream()),
                 lambda: B.mslt_op_rope(x[..., :32], y[..., :32], turns, _stream(), seq=4),
                 lambda: B.mslt_op_qk_norm_rope(x, y, gain[:1], turns, 1, 1e-6, _stream(), seq=4),
                 lambda: B.mslt_op_qk_norm_rope(x, y, gain, turns, 3, 1e-6, _stream(), seq=4)):
        with pytest.raises(B.MsltError) as e:
            call()
        assert e.value.code == -1
    with pytest.raises(B.MsltError) as e:
        B.mslt_op_rope(x.cpu(), y.cpu(), turns.cpu(), 0, seq=4)
    assert e.value.code == -4
