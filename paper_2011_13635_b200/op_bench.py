"""Bandwidth of the fused memory-bound kernels, one at a time, through the mslt_op_* entry points.

    python -m paper_2011_13635_b200.op_bench [--rows 16384] [--hidden 768] [--ffn 3072] [--heads 12]
        [--seq 128] [--batch 128] [--dtype bf16|fp32] [--only NAME[,NAME...]]

Each kernel is launched back to back on a rotation of buffers whose total size exceeds the 126 MB L2,
so that every launch reads its input from HBM; times are CUDA events on the launching stream.
Prints one JSON line per kernel: algorithmic bytes per launch, microseconds, GB/s.
"""
from __future__ import annotations

import argparse
import json


def main(argv=None, emit=print):
    """Runs the kernels and emits one JSON line per kernel; returns the list of records."""
    import torch
    from . import binding as Bd
    records = []
    ap = argparse.ArgumentParser()
    ap.add_argument("--rows", type=int, default=16384)
    ap.add_argument("--hidden", type=int, default=768)
    ap.add_argument("--ffn", type=int, default=3072)
    ap.add_argument("--heads", type=int, default=12)
    ap.add_argument("--seq", type=int, default=128)
    ap.add_argument("--batch", type=int, default=128)
    ap.add_argument("--dtype", default="bf16", choices=["bf16", "fp32"])
    ap.add_argument("--iters", type=int, default=40)
    ap.add_argument("--only", default="", help="comma-separated kernel groups: ln, colsum, softmax, attention, ce, rotary, masked")
    a = ap.parse_args(argv)
    only = set(x for x in a.only.split(",") if x)
    want = lambda group: not only or group in only
    tdt = torch.bfloat16 if a.dtype == "bf16" else torch.float32
    E = 2 if a.dtype == "bf16" else 4
    st = torch.cuda.current_stream().cuda_stream
    T, H, F = a.rows, a.hidden, a.ffn

    def rotation(shape, dtype, min_bytes=400 << 20):
        one = 1
        for s in shape:
            one *= s
        n = max(2, -(-min_bytes // (one * (2 if dtype == torch.bfloat16 else 4))))
        return [torch.randn(shape, device="cuda").to(dtype) for _ in range(int(n))]

    def run(name, nbytes, fn, nbuf):
        for i in range(3):
            fn(i % nbuf)
        torch.cuda.synchronize()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        for i in range(a.iters):
            fn(i % nbuf)
        e1.record()
        torch.cuda.synchronize()
        us = e0.elapsed_time(e1) / a.iters * 1e3
        rec = dict(kernel=name, dtype=a.dtype, bytes=nbytes, us=round(us, 2), gbs=round(nbytes / us / 1e3, 1))
        records.append(rec)
        if emit is not None:
            emit(json.dumps(rec))

    if want("attention") and a.dtype == "bf16" and a.seq <= 512:
        # fused attention of one layer: reads Q, K, V once, writes the context (and the probabilities)
        B, S, A = a.batch, a.seq, a.heads
        qs = rotation((B * S, 3 * A * 64), tdt)
        ctx = torch.empty((B * S, A * 64), device="cuda", dtype=tdt)
        probs = torch.empty((B, A, S, S), device="cuda", dtype=tdt)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        run("attention_fused", 4 * B * S * A * 64 * E,
            lambda i: Bd.mslt_op_attention(qs[i], None, ctx, None, B, S, A, 0.125, status, st, sync=False), len(qs))
        run("attention_fused_with_probs", 4 * B * S * A * 64 * E + B * A * S * S * E,
            lambda i: Bd.mslt_op_attention(qs[i], probs, ctx, None, B, S, A, 0.125, status, st, sync=False), len(qs))
        if S <= 128:
            # its backward: reads Q, K, V, the probabilities and the context gradient, writes dQ, dK, dV
            probs.copy_(torch.softmax(torch.randn((B, A, S, S), device="cuda"), -1))
            dqkv = torch.empty((B * S, 3 * A * 64), device="cuda", dtype=tdt)
            run("attention_fused_backward", 7 * B * S * A * 64 * E + B * A * S * S * E,
                lambda i: Bd.mslt_op_attention_bwd(qs[i], probs, ctx, dqkv, B, S, A, 0.125, status, st, sync=False),
                len(qs))
            del dqkv
        if int(status.item()) != 0:
            raise RuntimeError("the attention kernel reported a wait that ran out")
        del qs, ctx, probs
    if want("rotary"):
        # queries and keys in the fused projection's rows: rotation; norm and rotation; their backward
        A = a.heads
        xs = rotation((T, 3 * A, 64), tdt)
        heads = [x[:, :2 * A] for x in xs]
        y, dy = torch.empty((T, 2 * A, 64), device="cuda", dtype=tdt), torch.randn((T, 2 * A, 64), device="cuda").to(tdt)
        gain, dgain = torch.ones((2, 64), device="cuda"), torch.empty((2, 64), device="cuda")
        turns = torch.from_numpy(Bd.mslt_rope_turns(64)[0].view("int64")).cuda()
        scratch = torch.empty(Bd.mslt_op_qk_norm_rope_bwd_scratch_bytes(T, 2 * A, 64), dtype=torch.uint8, device="cuda")
        n = T * 2 * A * 64 * E
        run("rope", 2 * n, lambda i: Bd.mslt_op_rope(heads[i], y, turns, st, seq=a.seq, sync=False), len(xs))
        run("qk_norm_rope", 2 * n,
            lambda i: Bd.mslt_op_qk_norm_rope(heads[i], y, gain, turns, A, 1e-6, st, seq=a.seq, sync=False), len(xs))
        run("qk_norm_rope_backward", 3 * n,
            lambda i: Bd.mslt_op_qk_norm_rope_bwd(dy, heads[i], y, gain, dgain, turns, A, 1e-6, scratch, st, seq=a.seq, sync=False),
            len(xs))
        del xs, heads, y, dy
    if want("masked"):
        # attention under a causal mask, as a training step and as an evaluation call it
        B, S, A = a.batch, a.seq, a.heads
        qs = [x.view(B, S, 3 * A, 64) for x in rotation((B * S, 3 * A * 64), tdt)]
        parts = [(x[:, :, :A], x[:, :, A:2 * A], x[:, :, 2 * A:]) for x in qs]
        ctx, lse = torch.empty((B, S, A, 64), device="cuda", dtype=tdt), torch.empty((B, A, S), device="cuda")
        rest = torch.empty_like(ctx) if a.dtype == "bf16" else None
        grads = [torch.empty_like(ctx) for _ in range(3)]
        dctx = torch.randn(ctx.shape, device="cuda").to(tdt)
        scratch = torch.empty(Bd.mslt_op_attention_masked_bwd_scratch_bytes(B, S, A), dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        n = B * S * A * 64 * E
        run("attention_masked", 4 * n,
            lambda i: Bd.mslt_op_attention_masked(*parts[i], ctx, None, 0.125, status, st, causal=True, sync=False), len(qs))
        run("attention_masked_training", (5 if rest is not None else 4) * n,
            lambda i: Bd.mslt_op_attention_masked(*parts[i], ctx, lse, 0.125, status, st, causal=True, rest=rest, sync=False), len(qs))
        # the forward's results belong to the last buffer: the others give the same work, not gradients
        run("attention_masked_backward", (9 if rest is not None else 8) * n,
            lambda i: Bd.mslt_op_attention_masked_bwd(*parts[i], ctx, lse, dctx, *grads, scratch, 0.125, status, st, causal=True,
                                                      rest=rest, sync=False), len(qs))
        if int(status.item()) != 0:
            raise RuntimeError("the attention kernel reported a wait that ran out")
        del qs, parts, ctx, grads
    if not (want("ln") or want("colsum") or want("softmax") or want("ce")):
        return records
    gamma = torch.ones(H, device="cuda"); beta = torch.zeros(H, device="cuda")
    zs = rotation((T, H), tdt)
    y = torch.empty((T, H), device="cuda", dtype=tdt)
    # yardstick: a plain device copy of the same size (the method behind the measured HBM peak, which
    # was taken on 2 GB buffers; launches this short do not reach it)
    run("copy_same_size(reference)", 2 * T * H * E, lambda i: y.copy_(zs[i]), len(zs))
    stats = torch.empty((T, 2), device="cuda")
    run("layernorm", 2 * T * H * E,
        lambda i: Bd.mslt_op_layernorm(zs[i], gamma, beta, y, stats, 1e-12, st, sync=False), len(zs))
    dys = rotation((T, H), tdt, 200 << 20)
    dgam = torch.zeros(H, device="cuda"); dbet = torch.zeros(H, device="cuda")
    n = min(len(zs), len(dys))
    run("layernorm_bwd", 3 * T * H * E,
        lambda i: Bd.mslt_op_layernorm_bwd(dys[i], zs[i], stats, gamma, y, dgam, dbet, st, sync=False), n)
    out = torch.zeros(max(F, 3 * H), device="cuda")
    run("colsum_hidden", T * H * E, lambda i: Bd.mslt_op_colsum(zs[i], H, out, st, sync=False), len(zs))
    del dys
    gs = rotation((T, F), tdt)
    run("colsum_ffn", T * F * E, lambda i: Bd.mslt_op_colsum(gs[i], F, out, st, sync=False), len(gs))
    del gs, zs
    if not (want("softmax") or want("ce")):
        return records
    R, S = a.batch * a.heads * a.seq, a.seq
    ps = rotation((R, S), tdt)
    pout = torch.empty((R, S), device="cuda", dtype=tdt)
    run("softmax", 2 * R * S * E,
        lambda i: Bd.mslt_op_softmax(ps[i], pout, None, a.heads * S, 0.125, st, sync=False), len(ps))
    run("softmax_bwd", 3 * R * S * E,
        lambda i: Bd.mslt_op_softmax_bwd(ps[i], pout, 0.125, st, sync=False), len(ps))
    del ps
    Rm, V = a.batch * 20, 30522
    Vp = (V + 7) // 8 * 8
    logits = [torch.randn((Rm, Vp), device="cuda") for _ in range(2)]
    labels = torch.randint(0, V, (Rm,), device="cuda", dtype=torch.int32)
    dl = torch.empty((Rm, Vp), device="cuda", dtype=tdt)
    loss = torch.zeros(1, device="cuda")
    scratch = torch.empty(Bd.lib.mslt_op_cross_entropy_scratch_bytes(Rm), dtype=torch.uint8, device="cuda")
    # this entry point synchronises: its figure includes one host round trip per launch
    run("cross_entropy(sync)", Rm * Vp * (4 + E),
        lambda i: Bd.mslt_op_cross_entropy(1 if a.dtype == "bf16" else 0, logits[i], labels, V, dl, loss,
                                           scratch, st), 2)
    return records


if __name__ == "__main__":
    main()
