// C entry points of the operators on packed sequences: argument checks, then the launchers.
#include "pf_internal.h"
#include "pf_kernels.h"

#include <algorithm>

namespace {

bool bad_dtype(int32_t dt) { return dt != PF_DTYPE_F32 && dt != PF_DTYPE_BF16; }

// Rows that fit 32-bit row numbers with a block of room behind them
constexpr int64_t MAX_ROWS = 0x7fffffff - 512;
constexpr int64_t MAX_STRIDE = 1 << 24;   // the bytes of 64 rows fit 32 bits
// A launch has at most 2^32 threads: 256 for every 32 rows of a head
constexpr int64_t MAX_BLOCKS = 1 << 22;

bool bad_sequences(const int32_t* seq_start, int32_t n_seq, int64_t tokens) {
  return n_seq < 0 || (seq_start == nullptr) != (n_seq == 0) || tokens <= 0 || tokens > MAX_ROWS || n_seq > MAX_ROWS;
}

// Checks the description; fills the launchers' form of it
int32_t attention_args(const char* who, const pf_packed_attn* d, const int32_t* seq_start, pf::PackedAttn* a) {
  if (!d || bad_dtype(d->dtype)) return pf::fail(PF_ERR_ARG, "%s: bad argument", who);
  if (bad_sequences(seq_start, d->n_seq, d->tokens))
    return pf::fail(PF_ERR_ARG, "%s: bad argument (tokens must be positive, seq_start NULL exactly when n_seq is 0)", who);
  if (!(d->d_head == 8 || d->d_head == 16 || d->d_head == 32 || d->d_head == 64 || d->d_head == 128))
    return pf::fail(PF_ERR_ARG, "%s: bad argument (d_head must be 8, 16, 32, 64 or 128)", who);
  if (d->n_heads <= 0 || d->n_kv_heads <= 0 || d->n_heads % d->n_kv_heads != 0 || d->n_heads > 65535)
    return pf::fail(PF_ERR_ARG, "%s: bad argument (n_heads must be a multiple of n_kv_heads, at most 65535)", who);
  const int64_t wq = (int64_t)d->n_heads * d->d_head, wk = (int64_t)d->n_kv_heads * d->d_head;
  a->ld_q = d->ld_q ? d->ld_q : wq;
  a->ld_k = d->ld_k ? d->ld_k : wk;
  a->ld_v = d->ld_v ? d->ld_v : wk;
  a->ld_out = d->ld_out ? d->ld_out : wq;
  if (a->ld_q < wq || a->ld_k < wk || a->ld_v < wk || a->ld_out < wq || std::max(std::max(a->ld_q, a->ld_k), std::max(a->ld_v, a->ld_out)) > MAX_STRIDE)
    return pf::fail(PF_ERR_ARG, "%s: bad argument (rows overlap, or a stride over 2^24)", who);
  if ((d->tokens + 31) / 32 * d->n_heads > MAX_BLOCKS)
    return pf::fail(PF_ERR_ARG, "%s: bad argument (ceil(tokens / 32) * n_heads is more than 2^22)", who);
  a->tokens = d->tokens;
  a->seq_start = seq_start;
  a->n_seq = d->n_seq;
  a->dtype = d->dtype;
  a->h = d->n_heads;
  a->h_kv = d->n_kv_heads;
  a->dh = d->d_head;
  a->causal = d->causal != 0;
  return PF_OK;
}

bool misaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

int32_t launched(const char* who, hipError_t e) {
  return e == hipSuccess ? PF_OK : pf::fail(PF_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}

int32_t embed_args(const char* who, int32_t dtype, const int32_t* seq_start, int32_t n_seq, int64_t tokens, int32_t S, int32_t d, int32_t V) {
  if (bad_dtype(dtype) || bad_sequences(seq_start, n_seq, tokens) || S <= 0 || d <= 0 || d % 8 != 0 || V <= 0 || tokens > (1 << 26) || tokens * (((int64_t)d + 511) / 512) > (1 << 26) ||
      V > (1 << 24) || S > (1 << 24))
    return pf::fail(PF_ERR_ARG, "%s: bad argument (d must be a multiple of 8; at most 2^24 token ids and positions, tokens times d / 512 at most 2^26; seq_start NULL exactly when n_seq is 0)", who);
  return PF_OK;
}

}  // namespace

extern "C" {

int32_t pf_op_attention_packed(const pf_packed_attn* desc, const int32_t* seq_start, const void* q, const void* k, const void* v, void* out, float* lse,
                               void* stream) {
  pf::PackedAttn a;
  const int32_t rc = attention_args("pf_op_attention_packed", desc, seq_start, &a);
  if (rc != PF_OK) return rc;
  const uintptr_t size = pf::esize(a.dtype);
  if (!q || !k || !v || !out || misaligned(q, size) || misaligned(k, size) || misaligned(v, size) || misaligned(out, size) || misaligned(lse, 4) || misaligned(seq_start, 4))
    return pf::fail(PF_ERR_ARG, "pf_op_attention_packed: bad argument (null pointer, or not aligned to its elements)");
  return launched("pf_op_attention_packed", pf::attention_packed_fwd(a, q, k, v, out, lse, (hipStream_t)stream));
}

int64_t pf_op_attention_packed_bwd_workspace(const pf_packed_attn* desc) {
  pf::PackedAttn a;
  static const int32_t some = 0;   // the sizes alone matter here
  const int32_t rc = attention_args("pf_op_attention_packed_bwd_workspace", desc, desc && desc->n_seq > 0 ? &some : nullptr, &a);
  if (rc != PF_OK) return rc;
  return pf::attention_packed_bwd_bytes(a);
}

int32_t pf_op_attention_packed_bwd(const pf_packed_attn* desc, const int32_t* seq_start, const void* q, const void* k, const void* v, const void* out,
                                   const void* dout, const float* lse, void* dq, void* dk, void* dv, void* workspace, int64_t workspace_bytes,
                                   void* stream) {
  pf::PackedAttn a;
  const int32_t rc = attention_args("pf_op_attention_packed_bwd", desc, seq_start, &a);
  if (rc != PF_OK) return rc;
  const uintptr_t size = pf::esize(a.dtype);
  for (const void* p : {q, k, v, out, dout, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!p || misaligned(p, size)) return pf::fail(PF_ERR_ARG, "pf_op_attention_packed_bwd: bad argument (null pointer, or not aligned to its elements)");
  if (!lse || misaligned(lse, 4) || misaligned(seq_start, 4) || !workspace || misaligned(workspace, 256))
    return pf::fail(PF_ERR_ARG, "pf_op_attention_packed_bwd: bad argument (null pointer, or workspace not 256-byte aligned)");
  if (workspace_bytes < pf::attention_packed_bwd_bytes(a))
    return pf::fail(PF_ERR_NOMEM, "pf_op_attention_packed_bwd: workspace of %lld bytes, %lld needed", (long long)workspace_bytes,
                    (long long)pf::attention_packed_bwd_bytes(a));
  return launched("pf_op_attention_packed_bwd", pf::attention_packed_bwd(a, q, k, v, out, dout, lse, dq, dk, dv, workspace, (hipStream_t)stream));
}

// For tests: attention_packed_route of a call (misaligned: its pointers are not aligned to 16 bytes)
int32_t pf_attention_packed_route(const pf_packed_attn* desc, int32_t misaligned) {
  pf::PackedAttn a;
  static const int32_t some = 0;
  const int32_t rc = attention_args("pf_attention_packed_route", desc, desc && desc->n_seq > 0 ? &some : nullptr, &a);
  return rc != PF_OK ? rc : pf::attention_packed_route(a, !misaligned);
}

int32_t pf_op_embed_packed(int32_t dtype, const int32_t* ids, const void* tok, const void* pos, const int32_t* seq_start, int32_t n_seq, float scale, void* x,
                           int64_t tokens, int32_t S, int32_t d, int32_t V, void* stream) {
  const int32_t rc = embed_args("pf_op_embed_packed", dtype, seq_start, n_seq, tokens, S, d, V);
  if (rc != PF_OK) return rc;
  if (!ids || !tok || !x || misaligned(ids, 4) || misaligned(tok, 16) || misaligned(pos, 16) || misaligned(x, 16) || misaligned(seq_start, 4))
    return pf::fail(PF_ERR_ARG, "pf_op_embed_packed: bad argument (null pointer, or tables or x not 16-byte aligned)");
  return launched("pf_op_embed_packed", pf::embed_packed_fwd(dtype, ids, tok, pos, seq_start, n_seq, scale, x, tokens, S, d, V, (hipStream_t)stream));
}

int64_t pf_op_embed_packed_bwd_workspace(int64_t tokens, int32_t S, int32_t d, int32_t V) {
  const int32_t rc = embed_args("pf_op_embed_packed_bwd_workspace", PF_DTYPE_F32, nullptr, 0, tokens, S, d, V);
  if (rc != PF_OK) return rc;
  return pf::embed_packed_bwd_bytes(tokens, S, d, V);
}

int32_t pf_op_embed_packed_bwd(int32_t dtype, const void* dx, const int32_t* ids, const int32_t* seq_start, int32_t n_seq, float scale, float* dtok,
                               float* dpos, int32_t accumulate, void* workspace, int64_t workspace_bytes, int64_t tokens, int32_t S, int32_t d, int32_t V,
                               void* stream) {
  const int32_t rc = embed_args("pf_op_embed_packed_bwd", dtype, seq_start, n_seq, tokens, S, d, V);
  if (rc != PF_OK) return rc;
  if (!dx || !ids || !dtok || !workspace || misaligned(dx, 16) || misaligned(ids, 4) || misaligned(dtok, 16) || misaligned(dpos, 16) || misaligned(seq_start, 4) ||
      misaligned(workspace, 256))
    return pf::fail(PF_ERR_ARG, "pf_op_embed_packed_bwd: bad argument (null pointer, dx or gradients not 16-byte or workspace not 256-byte aligned)");
  if (workspace_bytes < pf::embed_packed_bwd_bytes(tokens, S, d, V))
    return pf::fail(PF_ERR_NOMEM, "pf_op_embed_packed_bwd: workspace of %lld bytes, %lld needed", (long long)workspace_bytes,
                    (long long)pf::embed_packed_bwd_bytes(tokens, S, d, V));
  return launched("pf_op_embed_packed_bwd", pf::embed_packed_bwd(dtype, dx, ids, seq_start, n_seq, scale, dtok, dpos, accumulate, workspace, tokens, S, d, V, (hipStream_t)stream));
}

}  // extern "C"
