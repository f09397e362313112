// Attention on packed sequences for gfx950: forward and backward with fp32 products, for every type, d_head and alignment.
//
// A block of 32 rows is 32 consecutive rows of the packed buffer, whichever sequences they belong to: each row (a lane) has the
// span [lo, hi) of rows that it meets, and a block walks the union of its rows' spans.  So the number of blocks is known on the host from the
// number of rows alone, lengths stay on the device (a captured graph can be replayed with others), and many short sequences
// share a block.  In a tile that is not inside every row's span, scores outside a row's own are -inf.
//
//   forward   S^T = K Q^T, O^T = V^T P^T with the softmax's running maximum and sum: one pass over the keys
//   backward  P = exp(scale S - lse), dP = dO V^T, dS = P (dP - D), D = rowsum(dO O):
//             dV = P^T dO, dK = scale dS^T Q summed over the heads of a group in registers, dQ = scale dS K
//
// 32x32x2 fp32 MFMAs, four waves of a workgroup share the tiles that a block meets and join their sums in LDS in a fixed
// order, so results are the same every time.  Operands come straight from global memory (the caches hold a head's rows).
//  * Operand slots (lane half g, element j) of chunk kk hold column 8 kk + 4 g + j of both operands.
//  * Register r of a product holds rows 8 (r / 4) + 4 g + r % 4 of a lane's column, which is the "B" operand of the r-th MFMA
//    that contracts over those rows; its "A" operand is a row of V (K, Q, dO) read as 32 consecutive columns.
//  * A pair that is not visible has P = dS = 0, and 0 times an infinity or NaN of another sequence's row would be NaN: masked
//    tiles with such a value take their sum row by row, visible ones only.
// Large calls are bound by the fp32 matrix rate (two sequences of 2048, causal, 16 heads of 64: forward 187 us, 92 of the 154 TFLOP/s that a large
// product reaches; backward 812 us, 74 with the scores computed in both passes), small ones by one wave's chain over its tiles and the
// launch (262 rows of four sequences up to 128, 4 heads of 64: 11 us; causal backward, on 2 K/V heads, 25 to 27).
// bf16 operands that the bf16 kernels do not take (8 sequences of 512, causal, 16 heads on 4, forward / backward): d_head 32 45 / 183 us, d_head 8
// 29 / 90; rows at odd elements, d_head 64 95 / 373 (aligned: 17 / 49), d_head 128 193 / 1094 (23 / 84).
#include "attention_packed.h"

#include <algorithm>

namespace pf {
namespace {

constexpr int NW = 4;   // waves of a workgroup

// four columns from c of a row; VEC: aligned
template <bool VEC, typename T>
__device__ __forceinline__ f32x4 row4(const T* p) {
  f32x4 r;
  if constexpr (VEC) {
    float v[4];
    load4(p, v);
    r = f32x4{v[0], v[1], v[2], v[3]};
  } else {
    r = f32x4{to_f32(p[0]), to_f32(p[1]), to_f32(p[2]), to_f32(p[3])};
  }
  return r;
}
template <bool VEC, typename T>
__device__ __forceinline__ void put4(T* p, const float v[4]) {
  if constexpr (VEC) {
    store4(p, v);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = from_f32<T>(v[j]);
  }
}

// column 32 dt + lr of row `row` (d_head below 32: zero past its end)
template <int DH, typename T>
__device__ __forceinline__ float col_of(const T* base, int64_t ld, int row, int dt, int lr) {
  const float x = to_f32(base[(int64_t)row * ld + (DH < 32 ? (lr < DH ? lr : 0) : dt * 32 + lr)]);
  return DH < 32 && lr >= DH ? 0.f : x;
}

__device__ __forceinline__ int reg_row(int r, int g) { return 8 * (r >> 2) + 4 * g + (r & 3); }

// acc[dt][.] += sum over a tile's rows of w[row] X[row][.], w in registers as an MFMA left them.  seen(i): whether row i of the
// tile counts for this lane's column.  xt: X by column, as loaded; sw: 32 x 32 floats of LDS of this wave.
template <int DH, typename T, class Seen>
__device__ __forceinline__ void add_rows(f32x16* acc, const f32x16& w, const float (*xt)[16], bool masked, const T* base, int64_t ld,
                                         int row0, int row_end, Seen seen, float* sw) {
  constexpr int DT = (DH + 31) / 32;
  const int lane = threadIdx.x & 63, lr = lane & 31, g = lane >> 5;
  bool finite = true;
  if (masked) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) finite = finite && fabsf(xt[dt][r]) < INFINITY;
  }
  if (!__any(!finite)) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(xt[dt][r], w[r], acc[dt], 0, 0, 0);
    return;
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) sw[reg_row(r, g) * 32 + lr] = w[r];
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // within the wave: its LDS instructions execute in order
  for (int i = 0; i < 32 && row0 + i < row_end; ++i) {
    if (!seen(i)) continue;
    const float p = sw[i * 32 + lr];
    const T* x = base + (int64_t)(row0 + i) * ld;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int c = dt * 32 + reg_row(r, g);
        if (c < DH) acc[dt][r] = fmaf(p, to_f32(x[c]), acc[dt][r]);
      }
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

template <typename T, int DH, bool VEC>
__global__ __launch_bounds__(256) void packed_fwd_f32_kernel(PackedQkv<T> a, T* __restrict__ out, float* __restrict__ lse) {
  constexpr int KK = DH / 8, DT = (DH + 31) / 32, LD = DT * 32 + 4;
  __shared__ __align__(16) float sO[NW][32][LD];   // O of the waves; before that, probabilities of a tile taken row by row
  __shared__ float sM[NW][32], sL[NW][32];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 31, g = lane >> 5;
  const int hd = (int)(blockIdx.x % (uint32_t)a.h), T_ = a.rows.tokens;
  const int q_blk = ((T_ + 31) / 32 - 1 - (int)(blockIdx.x / (uint32_t)a.h)) * 32;   // causal: the long ones first
  const int q_row = q_blk + lr;
  const T* qh = a.q + hd * DH;
  const T* kh = a.k + hd / a.group * DH;
  const T* vh = a.v + hd / a.group * DH;
  f32x4 fq[KK];
  {
    const T* p = qh + (int64_t)min(q_row, T_ - 1) * a.ld_q + g * 4;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) fq[kk] = row4<VEC>(p + kk * 8) * a.scale;
  }
  const Span own = keys_of(a.rows, q_blk, q_row, a.causal);
  const int k_begin = lane_value(own.lo, 0), k_end = lane_value(own.hi, 31);
  const int in_lo = lane_value(own.lo, 31), in_hi = lane_value(own.hi, 0);   // inside them every row sees every key
  f32x16 accO[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) accO[i][r] = 0.f;
  float m = -INFINITY, l = 0.f;   // of the query; l: this lane's share
  for (int k0 = k_begin + wave * 32; k0 < k_end; k0 += NW * 32) {
    const T* kp = kh + (int64_t)min(k0 + lr, k_end - 1) * a.ld_k + g * 4;
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const f32x4 fk = row4<VEC>(kp + kk * 8);
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(fk[j], fq[kk][j], s, 0, 0, 0);
    }
    float fv[DT][16];
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) fv[dt][r] = col_of<DH>(vh, a.ld_v, min(k0 + reg_row(r, g), k_end - 1), dt, lr);
    const bool masked = k0 < in_lo || k0 + 31 >= in_hi;
    if (masked) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = k0 + reg_row(r, g);
        if ((key < own.lo) | (key >= own.hi)) s[r] = -INFINITY;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
    const float m_new = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32, 64)));
    const float ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __expf(m - ref);   // no reference point yet: exp(-inf) = 0
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __expf(s[r] - ref);
      l += s[r];
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) accO[dt][r] *= alpha;
    add_rows<DH>(accO, s, fv, masked, vh, a.ld_v, k0, k_end, [&](int i) { return k0 + i >= own.lo && k0 + i < own.hi; }, &sO[wave][0][0]);
  }
  l += __shfl_xor(l, 32, 64);
  if (g == 0) {
    sM[wave][lr] = m;
    sL[wave][lr] = l;
  }
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int rg = 0; rg < 4; ++rg)
      *(f32x4*)&sO[wave][lr][dt * 32 + rg * 8 + g * 4] = f32x4{accO[dt][rg * 4], accO[dt][rg * 4 + 1], accO[dt][rg * 4 + 2], accO[dt][rg * 4 + 3]};
  const uint64_t live = __ballot(own.lo < own.hi);   // rows of the block that are in a sequence (the same in every wave)
  __syncthreads();
  for (int e = tid; e < 32 * DH / 4; e += 256) {
    const int i = e / (DH / 4), c = e % (DH / 4) * 4;
    if (!((live >> i) & 1)) continue;
    float mq = sM[0][i];
#pragma unroll
    for (int w = 1; w < NW; ++w) mq = fmaxf(mq, sM[w][i]);
    float lq = 0.f;   // a query whose scores are all -inf has no softmax: 0 / 0, and log(0) = -inf for lse
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = mq == -INFINITY ? 1.f : __expf(sM[w][i] - mq);   // 0 for a wave that met no key of this query
      lq += f * sL[w][i];
      o += *(const f32x4*)&sO[w][i][c] * f;
    }
    const float inv = 1.f / lq;
    const float r4[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    put4<VEC>(out + (int64_t)(q_blk + i) * a.ld_out + hd * DH + c, r4);
    if (lse && c == 0) lse[(int64_t)hd * T_ + q_blk + i] = mq + __logf(lq);
  }
}

// the waves' sums of one 32 x DH block, in LDS, to global memory: the rows in `live`
template <int DH, bool VEC, typename T>
__device__ __forceinline__ void join_rows(const float (*sO)[32][(DH + 31) / 32 * 32 + 4], uint64_t live, T* dst, int64_t ld, float scale) {
  for (int e = threadIdx.x; e < 32 * DH / 4; e += 256) {
    const int i = e / (DH / 4), c = e % (DH / 4) * 4;
    if (!((live >> i) & 1)) continue;
    f32x4 o = *(const f32x4*)&sO[0][i][c];
#pragma unroll
    for (int w = 1; w < NW; ++w) o += *(const f32x4*)&sO[w][i][c];
    const float r4[4] = {o[0] * scale, o[1] * scale, o[2] * scale, o[3] * scale};
    put4<VEC>(dst + (int64_t)i * ld + c, r4);
  }
}
template <int DT>
__device__ __forceinline__ void put_acc(float (*s)[DT * 32 + 4], const f32x16* acc) {   // a wave's block, by lane = row
  const int lr = threadIdx.x & 31, g = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int rg = 0; rg < 4; ++rg)
      *(f32x4*)&s[lr][dt * 32 + rg * 8 + g * 4] = f32x4{acc[dt][rg * 4], acc[dt][rg * 4 + 1], acc[dt][rg * 4 + 2], acc[dt][rg * 4 + 3]};
}

template <typename T>
struct BwdF32 {
  PackedQkv<T> o;
  const T *out, *dout;
  const float* lse;
  T *dq, *dk, *dv;
  float* partial;          // [split][dK, dV][tokens][K/V heads * d_head], or null with one split
  int32_t splits, k_units;
};

// dK, dV: 32 keys of one K/V head; the waves share the tiles of 32 queries of all heads of its group, or of a split of them
template <typename T, int DH, bool VEC>
__device__ __forceinline__ void dkv_f32_block(const BwdF32<T>& b, int unit, float (*sO)[32][(DH + 31) / 32 * 32 + 4]) {
  constexpr int KK = DH / 8, DT = (DH + 31) / 32;
  const PackedQkv<T>& a = b.o;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 31, g = lane >> 5;
  const int n_kv = a.h / a.group, T_ = a.rows.tokens;
  const uint32_t per = (uint32_t)(n_kv * b.splits);
  const int hk = (int)((uint32_t)unit % per) % n_kv, split = (int)((uint32_t)unit % per) / n_kv, k_blk = (int)((uint32_t)unit / per) * 32;
  const int key = k_blk + lr;
  // the block's own rows: d_head 128 has no registers for them beside 128 of sums (239 were spilled) and reads them with every tile, from L1
  constexpr bool KEEP = DH < 128;
  constexpr int UNROLL = KEEP ? KK : 4;
  f32x4 fk[KEEP ? KK : 1], fv[KEEP ? KK : 1];
  const T* pk = a.k + (int64_t)min(key, T_ - 1) * a.ld_k + hk * DH + g * 4;
  const T* pv = a.v + (int64_t)min(key, T_ - 1) * a.ld_v + hk * DH + g * 4;
  if constexpr (KEEP) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      fk[kk] = row4<VEC>(pk + kk * 8) * a.scale;
      fv[kk] = row4<VEC>(pv + kk * 8);
    }
  }
  const Span own = queries_of(a.rows, k_blk, key, a.causal);
  const int q_begin = lane_value(own.lo, 0), q_end = lane_value(own.hi, 31);
  const int in_lo = lane_value(own.lo, 31), in_hi = lane_value(own.hi, 0);
  f32x16 accK[DT], accV[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) accK[i][r] = accV[i][r] = 0.f;
  const int tiles = (q_end - q_begin + 31) / 32;
  const int64_t all = (int64_t)(tiles > 0 ? tiles : 0) * a.group, end = all * (split + 1) / b.splits;
  for (int64_t it = all * split / b.splits + wave; it < end; it += NW) {
    const int hd = hk * a.group + (int)(it / tiles), q0 = q_begin + (int)(it % tiles) * 32;
    const T* qh = a.q + hd * DH;
    const T* dh_ = b.dout + hd * DH;
    const int q_row = min(q0 + lr, q_end - 1);
    const T* pq = qh + (int64_t)q_row * a.ld_q + g * 4;
    const T* pd = dh_ + (int64_t)q_row * a.ld_out + g * 4;
    const T* po = b.out + hd * DH + (int64_t)q_row * a.ld_out + g * 4;
    float D = 0.f;   // of row q_row
    f32x16 s, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
    if constexpr (!KEEP) asm volatile("" : "+v"(pk), "+v"(pv));   // or the compiler reads them once after all
#pragma unroll UNROLL
    for (int kk = 0; kk < KK; ++kk) {
      const f32x4 x = row4<VEC>(pq + kk * 8), y = row4<VEC>(pd + kk * 8), o = row4<VEC>(po + kk * 8);
      f32x4 xk, xv;
      if constexpr (KEEP) {
        xk = fk[kk];
        xv = fv[kk];
      } else {
        xk = row4<VEC>(pk + kk * 8) * a.scale;
        xv = row4<VEC>(pv + kk * 8);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], xk[j], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x2f32(y[j], xv[j], dp, 0, 0, 0);
        D = fmaf(y[j], o[j], D);
      }
    }
    D += __shfl_xor(D, 32, 64);
    const bool masked = q0 < in_lo || q0 + 31 >= in_hi;
    const float L = b.lse[(int64_t)hd * T_ + q_row];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int q = q0 + reg_row(r, g);   // L and D of row q are in lane q - q0
      const bool hidden = masked & hidden_at(q, own.lo, own.hi - own.lo);
      const float Lq = __shfl(L, reg_row(r, g), 64), Dq = __shfl(D, reg_row(r, g), 64);
      const float p = hidden ? 0.f : __expf(s[r] - Lq);
      dp[r] = hidden ? 0.f : p * (dp[r] - Dq);
      s[r] = p;
    }
    auto seen = [&](int i) { return q0 + i >= own.lo && q0 + i < own.hi; };
    float xt[DT][16];
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) xt[dt][r] = col_of<DH>(dh_, a.ld_out, min(q0 + reg_row(r, g), q_end - 1), dt, lr);
    add_rows<DH>(accV, s, xt, masked, dh_, a.ld_out, q0, q_end, seen, &sO[wave][0][0]);
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) xt[dt][r] = col_of<DH>(qh, a.ld_q, min(q0 + reg_row(r, g), q_end - 1), dt, lr);
    add_rows<DH>(accK, dp, xt, masked, qh, a.ld_q, q0, q_end, seen, &sO[wave][0][0]);
  }
  const uint64_t live = __ballot(own.lo < own.hi);
  put_acc<DT>(sO[wave], accK);
  __syncthreads();
  const int64_t at = (int64_t)split * 2 * T_ + k_blk, ld = n_kv * DH;
  if (b.partial) join_rows<DH, true>(sO, live, b.partial + at * ld + hk * DH, ld, 1.0f);
  else join_rows<DH, VEC>(sO, live, b.dk + (int64_t)k_blk * a.ld_k + hk * DH, a.ld_k, a.scale);
  __syncthreads();
  put_acc<DT>(sO[wave], accV);
  __syncthreads();
  if (b.partial) join_rows<DH, true>(sO, live, b.partial + (at + T_) * ld + hk * DH, ld, 1.0f);
  else join_rows<DH, VEC>(sO, live, b.dv + (int64_t)k_blk * a.ld_v + hk * DH, a.ld_v, 1.0f);
}

// dQ: 32 queries of one head; the waves share the tiles of 32 keys
template <typename T, int DH, bool VEC>
__device__ __forceinline__ void dq_f32_block(const BwdF32<T>& b, int unit, float (*sO)[32][(DH + 31) / 32 * 32 + 4]) {
  constexpr int KK = DH / 8, DT = (DH + 31) / 32;
  const PackedQkv<T>& a = b.o;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 31, g = lane >> 5;
  const int hd = (int)((uint32_t)unit % (uint32_t)a.h), T_ = a.rows.tokens;
  const int q_blk = ((T_ + 31) / 32 - 1 - (int)((uint32_t)unit / (uint32_t)a.h)) * 32;
  const int q_row = q_blk + lr, qc = min(q_row, T_ - 1);
  const T* kh = a.k + hd / a.group * DH;
  const T* vh = a.v + hd / a.group * DH;
  f32x4 fq[KK], fd[KK];
  float D = 0.f;
  {
    const T* pq = a.q + (int64_t)qc * a.ld_q + hd * DH + g * 4;
    const T* pd = b.dout + (int64_t)qc * a.ld_out + hd * DH + g * 4;
    const T* po = b.out + (int64_t)qc * a.ld_out + hd * DH + g * 4;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      fq[kk] = row4<VEC>(pq + kk * 8) * a.scale;
      fd[kk] = row4<VEC>(pd + kk * 8);
      const f32x4 o = row4<VEC>(po + kk * 8);
#pragma unroll
      for (int j = 0; j < 4; ++j) D = fmaf(fd[kk][j], o[j], D);
    }
  }
  D += __shfl_xor(D, 32, 64);
  const float L = b.lse[(int64_t)hd * T_ + qc];
  const Span own = keys_of(a.rows, q_blk, q_row, a.causal);
  const int k_begin = lane_value(own.lo, 0), k_end = lane_value(own.hi, 31);
  const int in_lo = lane_value(own.lo, 31), in_hi = lane_value(own.hi, 0);
  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
  for (int k0 = k_begin + wave * 32; k0 < k_end; k0 += NW * 32) {
    const int key_row = min(k0 + lr, k_end - 1);
    const T* pk = kh + (int64_t)key_row * a.ld_k + g * 4;
    const T* pv = vh + (int64_t)key_row * a.ld_v + g * 4;
    f32x16 s, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const f32x4 x = row4<VEC>(pk + kk * 8), y = row4<VEC>(pv + kk * 8);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], fq[kk][j], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x2f32(y[j], fd[kk][j], dp, 0, 0, 0);
      }
    }
    const bool masked = k0 < in_lo || k0 + 31 >= in_hi;
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] = __expf(s[r] - L) * (dp[r] - D);
    if (masked) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (hidden_at(k0 + reg_row(r, g), own.lo, own.hi - own.lo)) dp[r] = 0.f;
    }
    float xt[DT][16];
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) xt[dt][r] = col_of<DH>(kh, a.ld_k, min(k0 + reg_row(r, g), k_end - 1), dt, lr);
    add_rows<DH>(acc, dp, xt, masked, kh, a.ld_k, k0, k_end, [&](int i) { return k0 + i >= own.lo && k0 + i < own.hi; }, &sO[wave][0][0]);
  }
  put_acc<DT>(sO[wave], acc);
  const uint64_t live = __ballot(own.lo < own.hi);
  __syncthreads();
  join_rows<DH, VEC>(sO, live, b.dq + (int64_t)q_blk * a.ld_q + hd * DH, a.ld_q, a.scale);
}

// Both passes: the dK/dV workgroups first, they are the longer ones
template <typename T, int DH, bool VEC>
__global__ __launch_bounds__(256, 1) void packed_bwd_f32_kernel(BwdF32<T> b) {
  __shared__ __align__(16) float sO[NW][32][(DH + 31) / 32 * 32 + 4];
  const int unit = (int)blockIdx.x;
  if (unit < b.k_units) dkv_f32_block<T, DH, VEC>(b, unit, sO);
  else dq_f32_block<T, DH, VEC>(b, unit - b.k_units, sO);
}

// dK, dV from the splits' sums [split][dK, dV][tokens][width]: four columns a thread, rows that are in a sequence
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void packed_bwd_join_kernel(const float* __restrict__ partial, PackedRows rows, int32_t width, int32_t splits, T* __restrict__ dk,
                                                              T* __restrict__ dv, int64_t ld_k, int64_t ld_v, float scale) {
  const int T_ = rows.tokens, per = width / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int row = (int)(i / per), c = (int)(i % per) * 4;
  const int first = rows.start ? rows.start[0] : 0, last = rows.start ? rows.start[rows.n_seq] : T_;
  if (i >= (int64_t)T_ * per || row < first || row >= last) return;
  const bool is_v = blockIdx.y != 0;
  const float* p = partial + ((int64_t)(is_v ? T_ : 0) + row) * width + c;
  f32x4 x = *(const f32x4*)p;
  for (int s = 1; s < splits; ++s) x += *(const f32x4*)(p + (int64_t)s * 2 * T_ * width);
  if (!is_v) x *= scale;
  const float r4[4] = {x[0], x[1], x[2], x[3]};
  put4<VEC>(is_v ? dv + (int64_t)row * ld_v + c : dk + (int64_t)row * ld_k + c, r4);
}

// dsum[head][row] = dO . O: eight columns a lane, a row's lanes next to each other
__global__ __launch_bounds__(256) void packed_bwd_prep_kernel(const bf16_t* __restrict__ out, const bf16_t* __restrict__ dout, float* __restrict__ dsum,
                                                              int64_t ld, int32_t tokens, int32_t h, int32_t dh) {
  const int per = dh / 8;   // lanes of a head: 8 or 16
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)tokens * h * per;
  const int64_t at = i < n ? i : n - 1;   // lanes past the end repeat the last one
  const int64_t row = at / (h * per);
  const int hd = (int)(at / per % h), c = (int)(at % per) * 8;
  const bf16_t* po = out + row * ld + hd * dh + c;
  const bf16_t* pd = dout + row * ld + hd * dh + c;
  float x[8], y[8], s = 0.f;
  load8(po, x);
  load8(pd, y);
#pragma unroll
  for (int j = 0; j < 8; ++j) s = fmaf(x[j], y[j], s);
  for (int o = per / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (i < n && c == 0) dsum[(int64_t)hd * tokens + row] = s;
}

template <typename T>
PackedQkv<T> operands(const PackedAttn& a, const void* q, const void* k, const void* v) {
  return PackedQkv<T>{(const T*)q, (const T*)k, (const T*)v, a.ld_q, a.ld_k, a.ld_v, a.ld_out, PackedRows{a.seq_start, a.n_seq, (int32_t)a.tokens},
                      a.h, a.h / a.h_kv, a.causal, 1.0f / sqrtf((float)a.dh)};
}

bool aligned16(const PackedAttn& a, std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if ((uintptr_t)p & 15) return false;
  return a.ld_q % 8 == 0 && a.ld_k % 8 == 0 && a.ld_v % 8 == 0 && a.ld_out % 8 == 0;
}

// whether bf16 products are used: they round P and dS, as the storage type rounds the results, and are 16 times as fast
bool by_bf16(const PackedAttn& a) { return a.dtype == PF_DTYPE_BF16_ && (a.dh == 64 || a.dh == 128); }

template <typename T, bool VEC>
hipError_t join(const PackedAttn& a, const float* partial, int splits, void* dk, void* dv, hipStream_t st) {
  const int width = a.h_kv * a.dh;
  hipLaunchKernelGGL((packed_bwd_join_kernel<T, VEC>), dim3((unsigned)((a.tokens * (width / 4) + 255) / 256), 2), dim3(256), 0, st, partial,
                     PackedRows{a.seq_start, a.n_seq, (int32_t)a.tokens}, width, splits, (T*)dk, (T*)dv, a.ld_k, a.ld_v, 1.0f / sqrtf((float)a.dh));
  return hipGetLastError();
}

template <typename T, int DH, bool VEC>
hipError_t fwd(const PackedAttn& a, const void* q, const void* k, const void* v, void* out, float* lse, hipStream_t st) {
  const unsigned grid = (unsigned)((a.tokens + 31) / 32 * a.h);
  hipLaunchKernelGGL((packed_fwd_f32_kernel<T, DH, VEC>), dim3(grid), dim3(256), 0, st, operands<T>(a, q, k, v), (T*)out, lse);
  return hipGetLastError();
}
// Splits of a block's tiles in dK/dV: as many as fill the card, four tiles (one a wave) to each or more if sequences were all as long as
// they are on average.  (us in one launch, and with one split and a launch for each pass: 262 rows, 4 heads on 2 of 64, one sequence
// 22, 65 (three splits), four of 32 to 100 rows 20, 36 (one); 512 rows, causal, 4 heads of 128 43, 100 (three); two of 2048, 16 heads of 64 812, 914 (one).)
int splits_f32(const PackedAttn& a) {
  const int64_t units = (a.tokens + 31) / 32 * a.h_kv, length = a.tokens / (a.n_seq > 1 ? a.n_seq : 1);
  const int64_t tiles = ((a.causal ? length / 2 : length) + 63) / 32 * (a.h / a.h_kv);
  return (int)std::max<int64_t>(1, std::min<int64_t>({(256 + units - 1) / units, (tiles + 3) / 4, 8}));
}

template <typename T, int DH, bool VEC>
hipError_t bwd(const PackedAttn& a, const void* q, const void* k, const void* v, const void* out, const void* dout, const float* lse, void* dq,
               void* dk, void* dv, float* partial, hipStream_t st) {
  BwdF32<T> b{operands<T>(a, q, k, v), (const T*)out, (const T*)dout, lse, (T*)dq, (T*)dk, (T*)dv, nullptr, splits_f32(a), 0};
  if (b.splits > 1) b.partial = partial;
  const int64_t blocks = (a.tokens + 31) / 32;
  b.k_units = (int32_t)(blocks * a.h_kv * b.splits);
  hipLaunchKernelGGL((packed_bwd_f32_kernel<T, DH, VEC>), dim3((unsigned)(b.k_units + blocks * a.h)), dim3(256), 0, st, b);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || b.splits == 1) return e;
  return VEC ? packed_join(a, partial, b.splits, dk, dv, st) : join<T, VEC>(a, partial, b.splits, dk, dv, st);
}

#define PF_BY_SHAPE(CALL)                                                                        \
  do {                                                                                           \
    const bool f32 = a.dtype == PF_DTYPE_F32_;                                                   \
    switch (a.dh) {                                                                              \
      case 8: PF_BY_TYPE(CALL, 8);                                                               \
      case 16: PF_BY_TYPE(CALL, 16);                                                             \
      case 32: PF_BY_TYPE(CALL, 32);                                                             \
      case 64: PF_BY_TYPE(CALL, 64);                                                             \
      case 128: PF_BY_TYPE(CALL, 128);                                                           \
      default: return hipErrorInvalidValue;                                                      \
    }                                                                                            \
  } while (0)
#define PF_BY_TYPE(CALL, D)                                                                      \
  if (f32) return vec ? CALL(float, D, true) : CALL(float, D, false);                            \
  return vec ? CALL(bf16_t, D, true) : CALL(bf16_t, D, false)

}  // namespace

hipError_t allow_lds(const void* kernel, int bytes) { return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); }

hipError_t attention_packed_fwd(const PackedAttn& a, const void* q, const void* k, const void* v, void* out, float* lse, hipStream_t st) {
  const bool vec = aligned16(a, {q, k, v, out});
  if (vec && by_bf16(a)) return packed_fwd_bf16(a, operands<bf16_t>(a, q, k, v), out, lse, st);
#define PF_FWD(T, D, V) fwd<T, D, V>(a, q, k, v, out, lse, st)
  PF_BY_SHAPE(PF_FWD);
#undef PF_FWD
}

int32_t attention_packed_route(const PackedAttn& a, bool aligned) {
  if (!aligned || !aligned16(a, {}) || !by_bf16(a)) return splits_f32(a) << 16;
  const FwdPlan f = packed_fwd_plan(a);
  const BwdPlan b = packed_bwd_plan(a);
  return (1 + f.form) | (f.at_once ? 0 : 1 << 8) | (b.dkv_at_once ? 0 : 1 << 9) | (b.dq_at_once ? 0 : 1 << 10) | f.heads << 12 | b.splits << 16;
}

int64_t packed_partial_bytes(const PackedAttn& a, int splits) { return splits > 1 ? (int64_t)splits * 2 * a.tokens * a.h_kv * a.dh * 4 : 0; }

hipError_t packed_join(const PackedAttn& a, const float* partial, int splits, void* dk, void* dv, hipStream_t st) {
  return a.dtype == PF_DTYPE_F32_ ? join<float, true>(a, partial, splits, dk, dv, st) : join<bf16_t, true>(a, partial, splits, dk, dv, st);
}

static int64_t dsum_bytes(const PackedAttn& a) { return ((int64_t)a.h * a.tokens * 4 + 255) / 256 * 256; }

// enough for either kernel: which one runs depends on the alignment of the call's pointers too
int64_t attention_packed_bwd_bytes(const PackedAttn& a) {
  const int64_t f32 = packed_partial_bytes(a, splits_f32(a));
  return std::max<int64_t>(256, by_bf16(a) ? std::max(f32, dsum_bytes(a) + packed_bwd_bf16_bytes(a)) : f32);
}

hipError_t attention_packed_bwd(const PackedAttn& a, const void* q, const void* k, const void* v, const void* out, const void* dout,
                                const float* lse, void* dq, void* dk, void* dv, void* workspace, hipStream_t st) {
  const bool vec = aligned16(a, {q, k, v, out, dout, dq, dk, dv});
  if (vec && by_bf16(a)) {
    float* dsum = (float*)workspace;
    const int64_t n = a.tokens * a.h * (a.dh / 8);
    hipLaunchKernelGGL(packed_bwd_prep_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, (const bf16_t*)out, (const bf16_t*)dout, dsum, a.ld_out,
                       (int32_t)a.tokens, a.h, a.dh);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return packed_bwd_bf16(a, operands<bf16_t>(a, q, k, v), dout, lse, dsum, dq, dk, dv, (char*)workspace + dsum_bytes(a), st);
  }
#define PF_BWD(T, D, V) bwd<T, D, V>(a, q, k, v, out, dout, lse, dq, dk, dv, (float*)workspace, st)
  PF_BY_SHAPE(PF_BWD);
#undef PF_BWD
}

}  // namespace pf
