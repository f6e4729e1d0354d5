// Entry points of attention under masks: checks of the arguments and the choice of the kernels by type.
#include "attn_masked.h"

#include <math.h>

#include "op_check.h"

using namespace mslt;

namespace {

// The strides of a single sequence, row or head are not used; they become ones that suit a tensor map.
mslt_heads tidy(const mslt_heads& h, const mslt_attention_desc& d, int heads) {
  mslt_heads t = h;
  if (d.B == 1) t.batch = 0;
  if (d.S == 1) t.row = 128;
  if (heads == 1) t.head = 0;
  return t;
}
mslt_attention_desc tidy(const mslt_attention_desc& d) {
  mslt_attention_desc t = d;
  t.q = tidy(d.q, d, d.heads); t.ctx = tidy(d.ctx, d, d.heads); t.dctx = tidy(d.dctx, d, d.heads); t.dq = tidy(d.dq, d, d.heads);
  t.k = tidy(d.k, d, d.kv_heads); t.v = tidy(d.v, d, d.kv_heads); t.dk = tidy(d.dk, d, d.kv_heads); t.dv = tidy(d.dv, d, d.kv_heads);
  return t;
}

// h: tidied.  An input's stride of 0 has no tensor map; an output's below a head's width would have blocks write to one place.
int check_heads(const char* what, const char* name, const mslt_heads& h, const mslt_attention_desc& d, int heads, bool output) {
  const int unit = d.dtype == 1 ? 8 : 4;
  if (!h.data) return op_refuse(MSLT_ERR_ARG, "%s: %s is null", what, name);
  if ((uintptr_t)h.data & 15) return op_refuse(MSLT_ERR_ARG, "%s: %s must be 16-byte aligned", what, name);
  if (h.batch < 0 || h.row < 0 || h.head < 0 || h.batch % unit || h.row % unit || h.head % unit)
    return op_refuse(MSLT_ERR_ARG, "%s: strides of %s must be multiples of 16 bytes", what, name);
  const int64_t least = output ? d.head_dim : 1;
  if ((d.B > 1 && h.batch < least) || (d.S > 1 && h.row < least) || (heads > 1 && h.head < least))
    return op_refuse(MSLT_ERR_ARG, output ? "%s: strides of %s must be at least head_dim" : "%s: %s must not be broadcast by a stride of 0", what,
                     name);
  return 0;
}

int check_attention(const char* what, const mslt_attention_desc* d, const int32_t* status) {
  if (!status) return op_refuse(MSLT_ERR_ARG, "%s: null pointer", what);
  if (d->dtype != 0 && d->dtype != 1) return op_refuse(MSLT_ERR_ARG, "%s: dtype must be 0 or 1", what);
  if (d->B < 1 || d->S < 1 || d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads)
    return op_refuse(MSLT_ERR_ARG, "%s: needs B, S, heads >= 1 and heads a multiple of kv_heads", what);
  if (d->head_dim < 8 || d->head_dim > 128 || d->head_dim % 8)
    return op_refuse(MSLT_ERR_ARG, "%s: head_dim must be a multiple of 8 in [8, 128]", what);
  if (d->S > 131072 || (int64_t)d->B * d->heads * d->S > (1ll << 30))
    return op_refuse(MSLT_ERR_SIZE, "%s: at most 131072 rows a sequence and 2^30 rows of all heads", what);
  if (!isfinite(d->scale) || !isfinite(d->cap) || d->cap < 0)
    return op_refuse(MSLT_ERR_ARG, "%s: scale and cap must be finite, cap not negative", what);
  // 2^64 either way: products of the cap, its inverse and the scale stay within fp32
  const float most = 0x1p64f, least = 0x1p-64f, by = fabsf(d->scale) / (d->cap > 0 ? d->cap : 1.f);
  if (d->cap > 0 && (d->cap > most || d->cap < least || by > most || (d->scale != 0 && by < least)))
    return op_refuse(MSLT_ERR_ARG, "%s: cap and scale / cap must be in [2^-64, 2^64]", what);
  if (d->prefix && !d->causal) return op_refuse(MSLT_ERR_ARG, "%s: a prefix needs causal", what);
  if (d->dtype == 0 && d->rest) return op_refuse(MSLT_ERR_ARG, "%s: rest is for dtype 1", what);
  if ((uintptr_t)d->rest & 15) return op_refuse(MSLT_ERR_ARG, "%s: rest must be 16-byte aligned", what);
  int rc = 0;
  if ((rc = check_heads(what, "q", d->q, *d, d->heads, false)) || (rc = check_heads(what, "k", d->k, *d, d->kv_heads, false)) ||
      (rc = check_heads(what, "v", d->v, *d, d->kv_heads, false)) || (rc = check_heads(what, "ctx", d->ctx, *d, d->heads, true)))
    return rc;
  return 0;
}

int end_attention(const char* what, const int32_t* status, cudaStream_t st, int sync) {
  int rc = op_end(what, st, sync);
  if (rc || !sync) return rc;
  int h = 0;
  if (cudaMemcpy(&h, status, 4, cudaMemcpyDeviceToHost) != cudaSuccess)
    return op_refuse(MSLT_ERR_CUDA, "%s: reading the status word failed", what);
  if (h & 1) return op_refuse(MSLT_ERR_DEVICE, "%s: a bounded wait ran out on the device", what);
  return 0;
}

// delta of the backward call; the counters of its bf16 kernels follow
size_t delta_bytes(int32_t B, int32_t S, int32_t heads) { return ((size_t)B * S * heads * sizeof(float) + 255) / 256 * 256; }

}  // namespace

extern "C" {

int mslt_op_attention_masked(const mslt_attention_desc* caller, int32_t* d_status, void* cuda_stream, int32_t sync) {
  const char* what = "attention_masked";
  if (!caller) return op_refuse(MSLT_ERR_ARG, "%s: null pointer", what);
  const mslt_attention_desc given = tidy(*caller), *desc = &given;
  int rc = check_attention(what, desc, d_status);
  if (rc || (rc = op_need_device())) return rc;
  return op_nothrow(what, [&] {
    char err[256] = "";
    int r = desc->dtype == 1 ? attn_masked_tc_fwd(*desc, d_status, (cudaStream_t)cuda_stream, err)
                             : attn_masked_f32_fwd(*desc, (cudaStream_t)cuda_stream, err);
    if (r) return op_refuse(r, "%s", err);
    return end_attention(what, d_status, (cudaStream_t)cuda_stream, sync);
  });
}

size_t mslt_op_attention_masked_bwd_scratch_bytes(int32_t B, int32_t S, int32_t heads) {
  if (B < 1 || S < 1 || heads < 1) return 0;
  return delta_bytes(B, S, heads) + 256;
}

int mslt_op_attention_masked_bwd(const mslt_attention_desc* caller, void* d_scratch, size_t scratch_bytes, int32_t* d_status,
                                 void* cuda_stream, int32_t sync) {
  const char* what = "attention_masked_bwd";
  if (!caller) return op_refuse(MSLT_ERR_ARG, "%s: null pointer", what);
  const mslt_attention_desc given = tidy(*caller), *desc = &given;
  int rc = check_attention(what, desc, d_status);
  if (rc) return rc;
  if ((rc = check_heads(what, "dctx", desc->dctx, *desc, desc->heads, false)) ||
      (rc = check_heads(what, "dq", desc->dq, *desc, desc->heads, true)) ||
      (rc = check_heads(what, "dk", desc->dk, *desc, desc->kv_heads, true)) ||
      (rc = check_heads(what, "dv", desc->dv, *desc, desc->kv_heads, true)))
    return rc;
  if (!desc->lse) return op_refuse(MSLT_ERR_ARG, "%s: lse is null", what);
  const size_t need = mslt_op_attention_masked_bwd_scratch_bytes(desc->B, desc->S, desc->heads);
  if (!d_scratch || scratch_bytes < need || ((uintptr_t)d_scratch & 15))
    return op_refuse(MSLT_ERR_SIZE, "%s: scratch must be 16-byte aligned and hold %zu bytes", what, need);
  if ((rc = op_need_device())) return rc;
  return op_nothrow(what, [&] {
    char err[256] = "";
    int* next = (int*)((char*)d_scratch + delta_bytes(desc->B, desc->S, desc->heads));
    int r = desc->dtype == 1 ? attn_masked_tc_bwd(*desc, (float*)d_scratch, next, d_status, (cudaStream_t)cuda_stream, err)
                             : attn_masked_f32_bwd(*desc, (float*)d_scratch, (cudaStream_t)cuda_stream, err);
    if (r) return op_refuse(r, "%s", err);
    return end_attention(what, d_status, (cudaStream_t)cuda_stream, sync);
  });
}

}  // extern "C"
