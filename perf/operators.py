"""The position and mask operators of an encoder's attention, as measurable cases.

Three operators that follow one another between the fused projection and the context of a layer:
  rope   rotation of query and key heads by their positions, and the rotation back of their gradients
  norm   normalisation of every query and key head together with the rotation, and its backward pass
  attn   attention under document, length, causal and prefix masks, with a bias by distance or scores that
         are capped by a tanh, for any length, and its backward pass
A case names one of them with its type, sizes and options.  `prepare` makes what a training program holds before
the call; `run` is one pass; with `own` it is the calls of the package's entry points, otherwise the same
formulas in elementary torch operations.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def _rope(op, dtype, rows, heads, dim, rot, q_heads=0, interleaved=False, scaling="none", factor=1.0, far=0, backward=False,
          center=False):
    """heads: query and key heads together, side by side in a row; q_heads: how many of them are queries;
    rot: elements of a head that are rotated; far: positions are drawn below it (0: rows of 128 tokens each)."""
    return dict(op=op, dtype=dtype, rows=rows, heads=heads, dim=dim, rot=rot, q_heads=q_heads, interleaved=interleaved,
                scaling=scaling, factor=factor, far=far, backward=backward, center=center)


def _attn(dtype, batch, seq, heads, kv_heads, dim, docs=0, shortest=0, causal=False, prefix=0, cap=0.0, slopes=False, backward=False):
    """docs: documents packed into a row (0: no document mask); shortest: lengths are uniform in [shortest, seq] (0: all
    full); prefix: with causal, the largest number of leading keys that every query sees."""
    return dict(op="attn", dtype=dtype, batch=batch, seq=seq, heads=heads, kv_heads=kv_heads, dim=dim, docs=docs,
                shortest=shortest, causal=causal, prefix=prefix, cap=cap, slopes=slopes, backward=backward)


def listed():
    return [
        # queries and keys of one short sequence under evaluation: latency
        dict(_rope("rope", "bf16", 64, 24, 64, 64), name="rope_one_sequence"),
        # gradients of the benchmark's batch (128 x 128 tokens, 12 + 12 heads) turned back
        dict(_rope("rope", "bf16", 16384, 24, 64, 64, backward=True), name="rope_base_batch_back"),
        # full precision, half of each head, neighbouring pairs, positions far beyond the trained ones
        dict(_rope("rope", "fp32", 8 * 1021, 32, 64, 32, interleaved=True, scaling="by_parts", factor=16.0, far=1 << 19),
             name="rope_far_fp32"),
        # the layer's queries and keys normalised and rotated, a small ragged evaluation in full precision
        dict(_rope("norm", "fp32", 77, 6, 64, 64, q_heads=3, center=True), name="norm_ragged_fp32"),
        # training step over the benchmark's batch
        dict(_rope("norm", "bf16", 16384, 24, 64, 64, q_heads=12, backward=True), name="norm_base_batch"),
        # training step on wide heads, keys shared by groups of queries, interpolated positions
        dict(_rope("norm", "bf16", 16 * 509, 20, 128, 128, q_heads=16, interleaved=True, scaling="linear", factor=4.0, backward=True),
             name="norm_wide_shared"),
        # evaluation of one sequence, capped scores: latency
        dict(_attn("bf16", 1, 64, 12, 12, 64, cap=30.0), name="attn_one_sequence"),
        # training step on rows packed with documents
        dict(_attn("bf16", 8, 2048, 12, 12, 64, docs=6, backward=True), name="attn_documents"),
        # evaluation over one long row, prefix seen by all, capped scores
        dict(_attn("bf16", 1, 8192, 16, 16, 64, causal=True, prefix=1500, cap=50.0), name="attn_long_prefix"),
        # training step on padded rows of odd length, wide heads shared by groups, bias by distance
        dict(_attn("bf16", 4, 1999, 16, 4, 128, shortest=700, slopes=True, backward=True), name="attn_padded_wide"),
        # training step on long rows in both directions, bias by distance: the largest
        dict(_attn("bf16", 4, 4096, 12, 12, 64, slopes=True, backward=True), name="attn_long_rows"),
        # training step in full precision on packed rows of odd length
        dict(_attn("fp32", 2, 509, 12, 12, 64, docs=3, shortest=300, backward=True), name="attn_documents_fp32"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))


def draw(rng):
    op = rng.choice(["rope", "norm", "attn", "attn"])
    if op != "attn":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        dim = rng.choice([32, 64, 64, 96, 128])
        q_heads = rng.randint(1, 16)
        heads = q_heads + rng.choice([h for h in range(1, q_heads + 1) if q_heads % h == 0])
        rows = _log(rng, 1, max(2, 16384 * 24 * 64 // (heads * dim) // (2 if dtype == "fp32" else 1)))
        scaling = rng.choice(["none", "none", "linear", "ntk", "by_parts"])
        return _rope(op, dtype, rows, heads, dim, rng.choice([dim, dim // 2, dim // 4]), q_heads=q_heads,
                     interleaved=rng.random() < 0.5, scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 5.0, 16.0]),
                     far=rng.choice([0, 0, 4096, 1 << 20]), backward=rng.random() < 0.5, center=op == "norm" and rng.random() < 0.4)
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    dim = rng.choice([64, 64, 128])
    kv_heads = rng.randint(1, 6)
    heads = kv_heads * rng.choice([1, 1, 2, 4] if kv_heads < 4 else [1, 2])
    backward = rng.random() < 0.6
    seq = _log(rng, 1, 4096 if dtype == "bf16" else 700)
    most = 4 * 12 * 4096 * 4096 * 64 if dtype == "bf16" else 4 * 12 * 512 * 512 * 64
    batch = _log(rng, 1, max(1, min(32, most // (heads * dim * seq * seq))))
    causal = rng.random() < 0.4
    return _attn(dtype, batch, seq, heads, kv_heads, dim, docs=rng.choice([0, 0, 2, 7]), shortest=rng.choice([0, max(1, seq // 3)]),
                 causal=causal, prefix=rng.choice([0, seq // 2]) if causal else 0, cap=rng.choice([0.0, 0.0, 20.0, 50.0]),
                 slopes=rng.random() < 0.4, backward=backward)


# ---- what a program holds before the call ------------------------------------------------------------

def _frequencies(case):
    """Radians a position, by pair, and the factor of long contexts on cosines and sines."""
    rot, f = case["rot"], case["factor"]
    base = 10000.0
    if case["scaling"] == "ntk" and rot > 2:
        base *= f ** (rot / (rot - 2))
    inv = base ** (-2.0 * np.arange(rot // 2, dtype=np.float64) / rot)
    if case["scaling"] == "linear":
        inv = inv / f
    if case["scaling"] == "by_parts":  # pairs that turn often within the trained 4096 positions stay, slow ones are interpolated
        keep = np.clip((4096 * inv / (2 * math.pi) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        inv = inv * keep + inv / f * (1 - keep)
    return inv, (0.1 * math.log(f) + 1.0 if case["scaling"] == "by_parts" else 1.0)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)
    t = TYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(t)

    if case["op"] in ("rope", "norm"):
        n, h, d = case["rows"], case["heads"], case["dim"]
        # queries and keys lie in the output of a fused projection, with the values behind them
        s = dict(case=case, x=normal(n, h + case["heads"] - case["q_heads"], d)[:, :h])
        if case["far"]:
            s["positions"] = torch.randint(0, case["far"], (n,), generator=g, device="cuda", dtype=torch.int32)
        else:
            s["positions"] = torch.arange(n, device="cuda", dtype=torch.int32) % 128
        inv, s["magnitude"] = _frequencies(case)
        s["inv"] = torch.from_numpy(inv).cuda()
        s["y"] = torch.empty(n, h, d, device="cuda", dtype=t)
        if case["op"] == "norm":
            s["gain"] = 1.0 + 0.2 * torch.randn(2, d, generator=g, device="cuda")
            s["bias"] = 0.1 * torch.randn(2, d, generator=g, device="cuda") if case["center"] else None
            if case["backward"]:
                s["dy"] = normal(n, h, d)
                s["dx"] = torch.empty(n, h, d, device="cuda", dtype=t)
                s["dgain"] = torch.empty(2, d, device="cuda")
                s["dbias"] = torch.empty(2, d, device="cuda") if case["center"] else None
        return s

    b, n, h, kv, d = case["batch"], case["seq"], case["heads"], case["kv_heads"], case["dim"]
    common = torch.randn(2, kv, d, generator=g, device="cuda") * 0.3  # what the keys, and the values, of a head have in common
    fused = torch.randn(b, n, h + 2 * kv, d, generator=g, device="cuda")
    fused[:, :, h:h + kv] += common[0]
    fused[:, :, h + kv:] += common[1]
    fused = fused.to(t)
    s = dict(case=case, q=fused[:, :, :h], k=fused[:, :, h:h + kv], v=fused[:, :, h + kv:], scale=1.0 / math.sqrt(d))
    s["docs"] = s["lens"] = s["prefix"] = s["slopes"] = None
    if case["docs"]:
        cuts = torch.randint(0, n, (b, case["docs"] - 1), generator=g, device="cuda").sort(1).values.contiguous()
        at = torch.arange(n, device="cuda").expand(b, n).contiguous()
        s["docs"] = torch.searchsorted(cuts, at, right=True).to(torch.int32)
    if case["shortest"]:
        s["lens"] = torch.randint(case["shortest"], n + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
    if case["prefix"]:
        s["prefix"] = torch.randint(1, case["prefix"] + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
    if case["slopes"]:
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, h + 1, device="cuda", dtype=torch.float32) / h)
    s["ctx"] = torch.empty(b, n, h, d, device="cuda", dtype=t)
    s["lse"] = torch.empty(b, h, n, device="cuda")
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if case["backward"]:
        s["dctx"] = normal(b, n, h, d)
        s["rest"] = torch.empty(b, n, h, d, device="cuda", dtype=t) if t == torch.bfloat16 else None
        grads = torch.empty(b, n, h + 2 * kv, d, device="cuda", dtype=t)
        s["dq"], s["dk"], s["dv"] = grads[:, :, :h], grads[:, :, h:h + kv], grads[:, :, h + kv:]
    return s


# ---- the calls of the package --------------------------------------------------------------------------

def _plan(s, B):
    """What a program makes once: the turns of its pairs."""
    if "turns" not in s:
        c = s["case"]
        turns, s["magnitude"] = B.mslt_rope_turns(c["rot"], 10000.0, c["scaling"], c["factor"], 4096)
        s["turns"] = torch.from_numpy(turns.view(np.int64)).cuda()
    return s["turns"]


def _scratch(s, size):
    """A workspace that a program keeps from pass to pass."""
    if "scratch" not in s:
        s["scratch"] = torch.empty(max(1, size), dtype=torch.uint8, device="cuda")
    return s["scratch"]


def _run_own(s):
    from paper_2011_13635_b200 import binding as B
    c = s["case"]
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "attn":
        mask = dict(cap=c["cap"], slopes=s["slopes"], causal=c["causal"], prefix=s["prefix"], docs=s["docs"], lens=s["lens"])
        rest = s.get("rest")
        B.mslt_op_attention_masked(s["q"], s["k"], s["v"], s["ctx"], s["lse"], s["scale"], s["status"], stream, rest=rest, sync=False,
                                   **mask)
        if not c["backward"]:
            return dict(ctx=s["ctx"], lse=s["lse"])
        scratch = _scratch(s, B.mslt_op_attention_masked_bwd_scratch_bytes(c["batch"], c["seq"], c["heads"]))
        B.mslt_op_attention_masked_bwd(s["q"], s["k"], s["v"], s["ctx"], s["lse"], s["dctx"], s["dq"], s["dk"], s["dv"], scratch,
                                       s["scale"], s["status"], stream, rest=rest, sync=False, **mask)
        return dict(ctx=s["ctx"], lse=s["lse"], dq=s["dq"], dk=s["dk"], dv=s["dv"])
    turns = _plan(s, B)
    rot = dict(positions=s["positions"], interleaved=c["interleaved"], magnitude=s["magnitude"], sync=False)
    if c["op"] == "rope":
        B.mslt_op_rope(s["x"], s["y"], turns, stream, inverse=c["backward"], **rot)
        return dict(y=s["y"])
    B.mslt_op_qk_norm_rope(s["x"], s["y"], s["gain"], turns, c["q_heads"], EPS, stream, bias=s["bias"], center=c["center"], **rot)
    if not c["backward"]:
        return dict(y=s["y"])
    scratch = _scratch(s, B.mslt_op_qk_norm_rope_bwd_scratch_bytes(c["rows"], c["heads"], c["dim"]))
    B.mslt_op_qk_norm_rope_bwd(s["dy"], s["x"], s["dx"], s["gain"], s["dgain"], turns, c["q_heads"], EPS, scratch, stream,
                               dbias=s["dbias"], center=c["center"], **rot)
    return dict(y=s["y"], dx=s["dx"], dgain=s["dgain"], dbias=s["dbias"])


# ---- the plain forms ------------------------------------------------------------------------------------

def _turned(x, s, back):
    """x [rows, heads, dim] in 32 bits with the first `rot` elements of each head turned by the row's position; the
    angles of far positions need 64 bits."""
    c = s["case"]
    rot = c["rot"]
    angle = s["positions"].double()[:, None] * s["inv"][None, :]
    cos = (torch.cos(angle) * s["magnitude"]).float()[:, None, :]
    sin = (torch.sin(angle) * s["magnitude"]).float()[:, None, :]
    if back:
        sin = -sin
    y = x.clone()
    if c["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2] = a * cos - b * sin
        y[..., 1:rot:2] = a * sin + b * cos
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2] = a * cos - b * sin
        y[..., rot // 2:rot] = a * sin + b * cos
    return y


def _by_head(table, c):
    """Row 0 of a [2, dim] table for the query heads, row 1 for the key heads."""
    return torch.cat([table[0].expand(c["q_heads"], c["dim"]), table[1].expand(c["heads"] - c["q_heads"], c["dim"])])[None]


def _by_table(x, c):
    """Sums of [rows, heads, dim] over rows and over the heads that share a row of the table."""
    x = x.double()
    return torch.stack([x[:, :c["q_heads"]].sum((0, 1)), x[:, c["q_heads"]:].sum((0, 1))]).float()


def _run_norm(s):
    c = s["case"]
    t = TYPES[c["dtype"]]
    x = s["x"].float()
    if c["center"]:
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    xh = x * r
    gain = _by_head(s["gain"], c)
    n = xh * gain
    if c["center"]:
        n = n + _by_head(s["bias"], c)
    y = _turned(n, s, False).to(t)
    if not c["backward"]:
        return dict(y=y)
    g = _turned(s["dy"].float(), s, True)
    h = g * gain
    dx = h - xh * (h * xh).mean(-1, keepdim=True)
    if c["center"]:
        dx = dx - h.mean(-1, keepdim=True)
    return dict(y=y, dx=(dx * r).to(t), dgain=_by_table(g * xh, c), dbias=_by_table(g, c) if c["center"] else None)


def _allowed(s):
    """[batch, 1, seq, seq]: which keys a query sees."""
    c = s["case"]
    n = c["seq"]
    i = torch.arange(n, device="cuda")
    ok = torch.ones(c["batch"], n, n, dtype=torch.bool, device="cuda")
    if c["causal"]:
        seen = i[None, :] <= i[:, None]
        ok = ok & (seen[None] | (i[None, None, :] < s["prefix"][:, None, None]) if s["prefix"] is not None else seen[None])
    if s["docs"] is not None:
        ok = ok & (s["docs"][:, :, None] == s["docs"][:, None, :])
    if s["lens"] is not None:
        live = i[None, :] < s["lens"][:, None]
        ok = ok & live[:, :, None] & live[:, None, :]
    return ok[:, None]


def _run_attn(s):
    c = s["case"]
    t = TYPES[c["dtype"]]
    b, n, h, kv, d = c["batch"], c["seq"], c["heads"], c["kv_heads"], c["dim"]
    q = s["q"].float().permute(0, 2, 1, 3)
    k = s["k"].float().permute(0, 2, 1, 3).repeat_interleave(h // kv, 1)
    v = s["v"].float().permute(0, 2, 1, 3).repeat_interleave(h // kv, 1)
    z = (q @ k.transpose(-1, -2)) * s["scale"]
    bend = None
    if c["cap"]:
        bend = torch.tanh(z / c["cap"])
        z = bend * c["cap"]
    if c["slopes"]:
        i = torch.arange(n, device="cuda")
        z = z - s["slopes"][:, None, None] * (i[None, :] - i[:, None]).abs().float()
    ok = _allowed(s)
    z = torch.where(ok, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    del z, e
    o = p @ v
    lse = (top + torch.log(total)).squeeze(-1)
    out = dict(ctx=o.permute(0, 2, 1, 3).to(t).contiguous(), lse=lse)
    if not c["backward"]:
        return out
    g = s["dctx"].float().permute(0, 2, 1, 3)
    dv = p.transpose(-1, -2) @ g
    dp = g @ v.transpose(-1, -2)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    del dp
    if bend is not None:
        ds = ds * (1 - bend * bend)
    dq = ds @ k * s["scale"]
    dk = ds.transpose(-1, -2) @ q * s["scale"]

    def shared(x):  # gradients of a key head that several query heads read
        return x.view(b, kv, h // kv, n, d).sum(2).permute(0, 2, 1, 3).to(t)

    return dict(out, dq=dq.permute(0, 2, 1, 3).to(t), dk=shared(dk), dv=shared(dv))


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    if c["op"] == "rope":
        return dict(y=_turned(state["x"].float(), state, c["backward"]).to(TYPES[c["dtype"]]))
    return _run_norm(state) if c["op"] == "norm" else _run_attn(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------

def _pairs(case):
    """Pairs of query and key that see each other, on average over the masks that `prepare` draws."""
    n = case["seq"]
    live = 1.0
    if case["shortest"]:
        lo = case["shortest"] / n
        live = (1 + lo + lo * lo) / 3
    if case["docs"]:
        live *= 2.0 / (case["docs"] + 1)
    if case["causal"]:
        live *= 0.5 + (case["prefix"] / n) ** 2 / 6
    return case["batch"] * case["heads"] * n * n * live


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] != "attn":
        n = case["rows"] * case["heads"] * case["dim"]
        if case["op"] == "rope":
            return dict(bytes=2 * n * size, flops=3 * case["rows"] * case["heads"] * case["rot"])
        return dict(bytes=(5 if case["backward"] else 2) * n * size, flops=(20 if case["backward"] else 8) * n)
    rows = case["batch"] * case["seq"] * case["dim"]
    heads, kv = case["heads"], case["kv_heads"]
    moved = 2 * heads + 2 * kv
    if case["backward"]:  # forward: q, k, v in, context out; backward: its gradient in, dq, dk, dv out
        moved += heads + heads + 2 * kv
    return dict(bytes=rows * moved * size + 4 * case["batch"] * heads * case["seq"],
                flops=_pairs(case) * case["dim"] * (14 if case["backward"] else 4))


# ---- the definition in 64 bits ---------------------------------------------------------------------------

def _spun(x, s, sign):
    """x, double, with its pairs multiplied as complex numbers by m e^(sign i position frequency)."""
    c = s["case"]
    rot, rows = c["rot"], x.shape[0]
    lead = x[..., :rot]
    pairs = lead.reshape(rows, -1, rot // 2, 2) if c["interleaved"] else lead.reshape(rows, -1, 2, rot // 2).transpose(-1, -2)
    inv, magnitude = _frequencies(c)
    phase = sign * s["positions"].double()[:, None] * torch.from_numpy(inv).cuda()
    w = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.full_like(phase, magnitude), phase)[:, None]
    out = torch.view_as_real(w)
    out = out.reshape(lead.shape) if c["interleaved"] else out.transpose(-1, -2).reshape(lead.shape)
    return torch.cat([out, x[..., rot:]], -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return dict(y=_spun(s["x"].double(), s, -1 if case["backward"] else 1))
    if case["op"] == "norm":
        with torch.enable_grad():
            x = s["x"].double().requires_grad_()
            gain = s["gain"].double().requires_grad_()
            bias = s["bias"].double().requires_grad_() if case["center"] else None
            which = (torch.arange(case["heads"], device="cuda") >= case["q_heads"]).long()
            if case["center"]:
                n = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + EPS) * gain[which] + bias[which]
            else:
                n = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * gain[which]
            y = _spun(n, s, 1)
            if not case["backward"]:
                return dict(y=y.detach())
            wanted = [x, gain] + ([bias] if case["center"] else [])
            grads = torch.autograd.grad(y, wanted, s["dy"].double())
        return dict(y=y.detach(), dx=grads[0], dgain=grads[1], dbias=grads[2] if case["center"] else None)
    if _pairs(case) * case["dim"] > 5e11:
        return None
    b, n, h, kv, d = case["batch"], case["seq"], case["heads"], case["kv_heads"], case["dim"]
    ctx = torch.zeros(b, n, h, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(b, h, n, dtype=torch.float64, device="cuda")
    dq, dk, dv = (torch.zeros(b, n, a, d, dtype=torch.float64, device="cuda") for a in (h, kv, kv))
    rows = torch.arange(n, device="cuda")
    for ib in range(b):
        seen = torch.ones(n, n, dtype=torch.bool, device="cuda")
        if case["causal"]:
            seen = seen.tril()
            if s["prefix"] is not None:
                seen[:, :int(s["prefix"][ib])] = True
        if s["docs"] is not None:
            seen &= s["docs"][ib][:, None] == s["docs"][ib]
        if s["lens"] is not None:
            seen[int(s["lens"][ib]):] = False
            seen[:, int(s["lens"][ib]):] = False
        some = seen.any(-1)
        for ih in range(h):
            ik = ih // (h // kv)
            with torch.enable_grad():
                q, k, v = (x.double().requires_grad_() for x in (s["q"][ib, :, ih], s["k"][ib, :, ik], s["v"][ib, :, ik]))
                z = torch.einsum("ie,je->ij", q, k) * s["scale"]
                if case["cap"]:
                    z = case["cap"] * torch.tanh(z / case["cap"])
                if case["slopes"]:
                    z = z - s["slopes"][ih].double() * (rows[:, None] - rows).abs()
                z = z.masked_fill(~seen, -math.inf)
                p = torch.softmax(z.masked_fill(~some[:, None], 0.0), -1) * some[:, None]
                o = torch.einsum("ij,je->ie", p, v)
                lse[ib, ih] = torch.logsumexp(z.detach(), -1)
                ctx[ib, :, ih] = o.detach()
                if case["backward"]:
                    a, bk, bv = torch.autograd.grad(o, (q, k, v), s["dctx"][ib, :, ih].double())
                    dq[ib, :, ih] = a
                    dk[ib, :, ik] += bk
                    dv[ib, :, ik] += bv
    out = dict(ctx=ctx, lse=lse)
    return dict(out, dq=dq, dk=dk, dv=dv) if case["backward"] else out
