// Attention backward on packed sequences, bf16, d_head 64 or 128, on the 32x32x16 bf16 MFMA (gfx950).
//
//   P = exp(scale S - lse), dP = dO V^T, dS = P (dP - D), D = rowsum(dO O)
//   dV = P^T dO, dK = scale dS^T Q (both summed over the query heads of a group), dQ = scale dS K
//
// Two passes in one launch that each own their results (no atomics):
//  * dK/dV: a workgroup has 128 keys of a K/V head, a wave 32 of them with K and V as "B" operands in registers, and walks the
//    tiles of 64 queries of the group's heads.  S = Q K^T and dP = dO V^T put one key and 32 of a tile's 64 queries into a lane:
//    the "B" operands of dV^T += dO^T P and dK^T += Q^T dS, whose "A" operands come out of the same row-major tiles by the
//    transposing LDS load.  Where keys and K/V heads are too few for the card, the tiles are dealt out to several workgroups, whose
//    fp32 sums one more launch adds up.
//  * dQ: the forward kernel's mirror image; S^T = K Q^T and dP^T = V dO^T put one query into a lane.
// Tiles go global -> LDS directly, one tile ahead.  Bound by what a SIMD issues: matrix products, exponentials and LDS reads take about as
// long each (seven products of 2 T^2 d_head per head and pass where the formulas have five: S and dP in both passes), and two waves
// overlap them in part.  d_head 64, 16 heads on 4, one causal sequence of 8192: 480 to 500 us, 0.96 to
// 1.0 PFLOP/s of products; d_head 128: 1000 to 1050, see below.
// D = rowsum(dO O) comes from a launch before (6 us at 5000 rows of 16 heads of 64).  Rows of other sequences: see attention_packed.h.  A workgroup whose results
// hold an infinity or NaN, which rows hidden from them may have brought in, does them again with care, as a second stretch of code behind the first
// (woven into the first it cost that one registers: dK/dV of d_head 128 took 1880 us instead of 780).
#include "attention_packed.h"

#include <algorithm>

namespace pf {
namespace {

// Swizzle of tiles that are read both ways: for one chunk per lane from consecutive rows a bijection of the bank phases, and the
// 32-byte pairs of four consecutive rows apart for the transposing read.  Depends on row % 16 only.
template <int DH>
struct SwzBoth {
  static __device__ __forceinline__ int of(int r) {
    if (DH == 64) {
      const int x = (r >> 1) & 7;
      return ((x & 1) << 1) | ((x >> 1) & 1) | (x & 4);
    }
    const int x = r & 15;
    return (x & 8) | ((x & 3) << 1) | ((x >> 2) & 1);
  }
};
// byte offsets of a lane's two transposing reads, columns from 32 dt, K step 0 (tr_offset, with this swizzle: rows 8 apart differ)
template <int DH>
__device__ __forceinline__ void tr_offsets(int lane, int off[][2]) {
  const int p = lane & 15, g = lane >> 5;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int row = 8 * r + 4 * g + (p >> 2), c = dt * 4 + ((lane >> 4) & 1) * 2 + ((p & 3) >> 1);
      off[dt][r] = row * DH * 2 + ((c ^ SwzBoth<DH>::of(row)) << 4) + 8 * (p & 1) - (r ? 8 * DH * 2 : 0);   // read_tr adds the 8 rows
    }
}

template <int DT>
__device__ __forceinline__ bool not_finite(const f32x16* acc) {
  bool r_ = false;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) r_ = r_ || !(fabsf(acc[i][r]) < INFINITY);
  return r_;
}

struct BwdArgs {
  PackedQkv<bf16_t> o;
  const bf16_t* dout;
  const float *lse, *dsum;
  bf16_t *dq, *dk, *dv;
  float* partial;                              // [split][dK, dV][tokens][K/V heads * d_head], or null with one split
  int32_t k_blocks, splits;                    // dK/dV: blocks of 128 keys, parts of a block's tiles
  int32_t q_blocks, heads;                     // dQ: blocks of rows, heads of a workgroup
  int32_t k_units, q_units;                    // workgroups
  int32_t at_once;                             // they start at the same time: 1 dK/dV, 2 dQ
  float scale_log2e;
};

// ---- dK, dV ------------------------------------------------------------------------------------------------------------------
// Workgroup `unit`; whether a result is infinite or NaN.  smem: two buffers; s_span: two ints.  WANT: 1 dV, 2 dK, 3 both.
template <int DH, int WANT, bool CAREFUL>
__device__ __forceinline__ bool dkv_block(const BwdArgs& a, int unit, char* smem, int* s_span) {
  constexpr int KS = DH / 16, DT = DH / 32, ROWB = DH * 2, TILE = 64 * ROWB;
  constexpr bool DV = WANT & 1, DK = WANT & 2;
  constexpr int BUF = 2 * TILE + 512;   // Q tile | dO tile | lse (log2 units) of the 64 queries | D
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 31, g = lane >> 5;
  const int n_kv = a.o.h / a.o.group, T = a.o.rows.tokens;
  // K/V heads and splits fastest: workgroups with the same rows run at the same time
  const uint32_t per = (uint32_t)(n_kv * a.splits);
  const int hk = (int)((uint32_t)unit % per) % n_kv, split = (int)((uint32_t)unit % per) / n_kv;
  const int k_blk = block_in_order(a.o.rows, (int)((uint32_t)unit / per), a.k_blocks, 7, a.o.causal, true, a.at_once & 1) * 128;
  const int key = k_blk + wave * 32 + lr;
  bf16x8 fk[KS], fv[DK ? KS : 1];
  {
    const int row = min(key, T - 1);
    const bf16_t* pk = a.o.k + (int64_t)row * a.o.ld_k + hk * DH + g * 8;
    const bf16_t* pv = a.o.v + (int64_t)row * a.o.ld_v + hk * DH + g * 8;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      fk[kk] = as_bf16x8(*(const uint4*)(pk + kk * 16));
      if constexpr (DK) fv[kk] = as_bf16x8(*(const uint4*)(pv + kk * 16));
    }
  }
  const Span own = queries_of(a.o.rows, k_blk + wave * 32, key, a.o.causal);
  const int w_lo = lane_value(own.lo, 0), w_hi = lane_value(own.hi, 31);
  const int in_lo = lane_value(own.lo, 31), in_hi = lane_value(own.hi, 0);
  if (tid == 0) s_span[0] = w_lo;
  if (tid == 192) s_span[1] = w_hi;
  __syncthreads();
  const int q_begin = __builtin_amdgcn_readfirstlane(s_span[0]), q_end = __builtin_amdgcn_readfirstlane(s_span[1]);
  const int tiles = q_end > q_begin ? (q_end - q_begin + 63) >> 6 : 0;

  TileCopy<DH, 4, SwzBoth<DH>> copy_q, copy_d;
  copy_q.init(a.o.ld_q, wave);
  copy_d.init(a.o.ld_out, wave);
  const uint32_t lds_base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_ptr)smem) + (uint32_t)(wave * 1024);
  auto stage = [&](int buf, int hd, int q0) {
    copy_q.issue(a.o.q + hd * DH, lds_base + (uint32_t)(buf * BUF), q0, q_end);
    copy_d.issue(a.dout + hd * DH, lds_base + (uint32_t)(buf * BUF + TILE), q0, q_end);
  };
  // threads 0..63 carry lse, 64..127 carry D of the tile's queries (the others repeat them and write nothing)
  auto load_ld = [&](int hd, int q0) { return ((tid & 64) ? a.dsum : a.lse)[(int64_t)hd * T + min(q0 + (tid & 63), q_end - 1)]; };
  auto write_ld = [&](int buf, float v) {
    if (tid < 128) *(float*)(smem + buf * BUF + 2 * TILE + tid * 4) = tid < 64 ? v * LOG2E_P : v;
  };
  int t_off[DT][2];
  tr_offsets<DH>(lane, t_off);
  f32x16 accK[DK ? DT : 1], accV[DV ? DT : 1];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) {   // waited for here, once
    asm volatile("" ::"v"(fk[kk]));
    if constexpr (DK) asm volatile("" ::"v"(fv[kk]));
  }
  // the tiles of one head after the other; this split's part of them
  const int64_t all = (int64_t)tiles * a.o.group;
  const int64_t first = all * split / a.splits;
  const int steps = (int)(all * (split + 1) / a.splits - first);
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if constexpr (DK) accK[i][r] = 0.f;
      if constexpr (DV) accV[i][r] = 0.f;
    }
  float ld = 0.f;
  int hd = hk * a.o.group, q0 = q_begin;
  if (steps > 0) {
    hd += (int)(first / tiles);
    q0 += (int)(first % tiles) * 64;
    stage(0, hd, q0);
    ld = load_ld(hd, q0);
  }
  for (int it = 0; it < steps; ++it) {
    const int buf = it & 1, q_now = q0;
    write_ld(buf, ld);   // the buffer was last read before the barrier of the previous step
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    q0 += 64;
    if (q0 >= q_end) {
      q0 = q_begin;
      ++hd;
    }
    if (it + 1 < steps) {
      stage(buf ^ 1, hd, q0);
      ld = load_ld(hd, q0);
    }
    if (q_now + 64 <= w_lo || q_now >= w_hi) continue;   // none of the wave's keys is seen from the tile
    const char* sQ = smem + buf * BUF;
    const char* sdO = sQ + TILE;
    const float* sL = (const float*)(sQ + 2 * TILE);
    lds_char_ptr tQ = (lds_char_ptr)(lds_void_ptr)smem + buf * BUF;
    lds_char_ptr tdO = tQ + TILE;
    const bool masked = q_now < in_lo || q_now + 64 > in_hi;
    const int lo = own.lo - q_now, hi = own.hi - q_now;
    const bool by_element = __any(seen_in_part(lo, hi));   // of a masked tile; otherwise a lane's key is seen from all of the tile or from none
    bf16x8 fp[4], fds[4];   // P and dS, rounded to bf16 (half a step, 2^-8 of each)
#pragma unroll
    for (int qs = 0; qs < 2; ++qs) {
      f32x16 aS, aP;
#pragma unroll
      for (int r = 0; r < 16; ++r) aS[r] = aP[r] = 0.f;
      if constexpr (DH == 128) __builtin_amdgcn_s_setprio(1);   // the SIMD's other wave fills the gaps (side by side, 8192 rows, 16 heads on 4: 1081 -> 1023 us; d_head 64: 483 -> 501)
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        const int r = qs * 32 + lr;
        const int o = r * ROWB + (((kk * 2 + g) ^ SwzBoth<DH>::of(r)) << 4);
        aS = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*(const uint4*)(sQ + o)), fk[kk], aS, 0, 0, 0);
        if constexpr (DK) aP = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*(const uint4*)(sdO + o)), fv[kk], aP, 0, 0, 0);
      }
      if constexpr (DH == 128) __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        const int qi = qs * 32 + 8 * rg + 4 * g;
        const f32x4 L4 = *(const f32x4*)(sL + qi), D4 = *(const f32x4*)(sL + 64 + qi);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = rg * 4 + j;
          aS[r] = __builtin_amdgcn_exp2f(fmaf(aS[r], a.scale_log2e, -L4[j]));
          if constexpr (DK) aP[r] = aS[r] * (aP[r] - D4[j]);
        }
      }
      if (masked) {
        if (by_element) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (hidden_at(qs * 32 + 8 * (r >> 2) + (r & 3), lo - 4 * g, hi - lo)) aS[r] = aP[r] = 0.f;
        } else if (!seen_as_a_whole(lo, hi)) {
#pragma unroll
          for (int r = 0; r < 16; ++r) aS[r] = aP[r] = 0.f;
        }
      }
#pragma unroll
      for (int i = 2 * qs; i < 2 * qs + 2; ++i) {
        if constexpr (DV) fp[i] = as_operand(aS, i);
        if constexpr (DK) fds[i] = as_operand(aP, i);
        if (CAREFUL && masked) continue;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          if constexpr (DV) accV[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_tr<ROWB>(tdO, t_off[dt][0], t_off[dt][1], i), fp[i], accV[dt], 0, 0, 0);
          if constexpr (DK) accK[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_tr<ROWB>(tQ, t_off[dt][0], t_off[dt][1], i), fds[i], accK[dt], 0, 0, 0);
        }
      }
    }
    if (CAREFUL && masked) {
      auto off = [&](int dt, int r) { return t_off[dt][r]; };
      if constexpr (DV) add_with_care<DH>(accV, fp, tdO, off, lo, hi);
      if constexpr (DK) add_with_care<DH>(accK, fds, tQ, off, lo, hi);
    }
  }
  bool odd = false;
  if constexpr (!CAREFUL) {
    if constexpr (DK) odd = not_finite<DT>(accK);
    if constexpr (DV) odd = odd || not_finite<DT>(accV);
    odd = __syncthreads_or(odd && own.lo < own.hi);
  }
  if (own.lo >= own.hi) return odd;
  auto store = [&](const f32x16* acc, bf16_t* dst, int64_t ld, int64_t part, float scale) {
    if (a.partial == nullptr) {
      bf16_t* row = dst + (int64_t)key * ld + hk * DH;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
          const float v[4] = {acc[dt][rg * 4] * scale, acc[dt][rg * 4 + 1] * scale, acc[dt][rg * 4 + 2] * scale, acc[dt][rg * 4 + 3] * scale};
          store4(row + dt * 32 + rg * 8 + g * 4, v);
        }
    } else {
      float* row = a.partial + (part * T + key) * (n_kv * DH) + hk * DH;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg)
          *(f32x4*)(row + dt * 32 + rg * 8 + g * 4) = f32x4{acc[dt][rg * 4], acc[dt][rg * 4 + 1], acc[dt][rg * 4 + 2], acc[dt][rg * 4 + 3]};
    }
  };
  if constexpr (DK) store(accK, a.dk, a.o.ld_k, 2 * split, a.o.scale);
  if constexpr (DV) store(accV, a.dv, a.o.ld_v, 2 * split + 1, 1.0f);
  return odd;
}

// ---- dQ ----------------------------------------------------------------------------------------------------------------------
template <int DH, bool CAREFUL>
__device__ __forceinline__ bool dq_block(const BwdArgs& a, int unit, char* smem, int* s_span) {
  constexpr int KS = DH / 16, DT = DH / 32, ROWB = DH * 2, TILE = 64 * ROWB, BUF = 2 * TILE;   // K tile | V tile
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 31, g = lane >> 5;
  const int T = a.o.rows.tokens, groups = a.o.h / a.heads, tiles_of_rows = 4 / a.heads;
  const int hg = (int)((uint32_t)unit % (uint32_t)groups);
  const int blk = block_in_order(a.o.rows, (int)((uint32_t)unit / (uint32_t)groups), a.q_blocks, 5 + (tiles_of_rows >> 1), a.o.causal, false, a.at_once & 2);
  const int hd = hg * a.heads + wave % a.heads, q_blk = (blk * tiles_of_rows + wave / a.heads) * 32;
  const int q_row = q_blk + lr, q_cl = min(q_row, T - 1);
  bf16x8 fq[KS], fd[KS];
  {
    const bf16_t* pq = a.o.q + (int64_t)q_cl * a.o.ld_q + hd * DH + g * 8;
    const bf16_t* pd = a.dout + (int64_t)q_cl * a.o.ld_out + hd * DH + g * 8;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      fq[kk] = as_bf16x8(*(const uint4*)(pq + kk * 16));
      fd[kk] = as_bf16x8(*(const uint4*)(pd + kk * 16));
    }
  }
  const float neg_l = -a.lse[(int64_t)hd * T + q_cl] * LOG2E_P, D = a.dsum[(int64_t)hd * T + q_cl];
  const Span own = keys_of(a.o.rows, q_blk, q_row, a.o.causal);
  const int w_lo = lane_value(own.lo, 0), w_hi = lane_value(own.hi, 31);
  const int in_lo = lane_value(own.lo, 31), in_hi = lane_value(own.hi, 0);
  if (tid == 0) s_span[0] = w_lo;
  if (tid == 192) s_span[1] = w_hi;
  __syncthreads();
  const int k_begin = __builtin_amdgcn_readfirstlane(s_span[0]), k_end = __builtin_amdgcn_readfirstlane(s_span[1]);
  const int n_tiles = k_end > k_begin ? (k_end - k_begin + 63) >> 6 : 0;

  const bf16_t* kh = a.o.k + hd / a.o.group * DH;
  const bf16_t* vh = a.o.v + hd / a.o.group * DH;
  TileCopy<DH, 4, SwzBoth<DH>> copy_k;
  TileCopy<DH, 4, SwzRow<DH>> copy_v;
  copy_k.init(a.o.ld_k, wave);
  copy_v.init(a.o.ld_v, wave);
  const uint32_t lds_base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_ptr)smem) + (uint32_t)(wave * 1024);
  auto stage = [&](int buf, int k0) {
    copy_k.issue(kh, lds_base + (uint32_t)(buf * BUF), k0, k_end);
    copy_v.issue(vh, lds_base + (uint32_t)(buf * BUF + TILE), k0, k_end);
  };
  int t_off[DT][2];
  tr_offsets<DH>(lane, t_off);
  f32x16 acc[DT];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) asm volatile("" ::"v"(fq[kk]), "v"(fd[kk]));   // waited for here, once
  asm volatile("" ::"v"(neg_l), "v"(D));
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
  if (n_tiles > 0) stage(0, k_begin);
  for (int kt = 0; kt < n_tiles; ++kt) {
    const int k0 = k_begin + kt * 64, buf = kt & 1;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (kt + 1 < n_tiles) stage(buf ^ 1, k0 + 64);
    if (k0 + 64 <= w_lo || k0 >= w_hi) continue;   // none of the wave's rows sees the tile
    const char* sK = smem + buf * BUF;
    const char* sV = sK + TILE;
    lds_char_ptr tK = (lds_char_ptr)(lds_void_ptr)smem + buf * BUF;
    const bool masked = k0 < in_lo || k0 + 64 > in_hi;
    const int lo = own.lo - k0, hi = own.hi - k0;
    const bool by_element = __any(seen_in_part(lo, hi));
    bf16x8 fds[4];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      f32x16 aS, aP;
#pragma unroll
      for (int r = 0; r < 16; ++r) aS[r] = aP[r] = 0.f;
      if constexpr (DH == 128) __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        const int r = ks * 32 + lr, c = kk * 2 + g;
        aS = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*(const uint4*)(sK + r * ROWB + ((c ^ SwzBoth<DH>::of(r)) << 4))), fq[kk], aS, 0, 0, 0);
        aP = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*(const uint4*)(sV + r * ROWB + ((c ^ swz_row<DH>(r)) << 4))), fd[kk], aP, 0, 0, 0);
      }
      if constexpr (DH == 128) __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int r = 0; r < 16; ++r) aP[r] = __builtin_amdgcn_exp2f(fmaf(aS[r], a.scale_log2e, neg_l)) * (aP[r] - D);
      if (masked) {
        if (by_element) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (hidden_at(ks * 32 + 8 * (r >> 2) + (r & 3), lo - 4 * g, hi - lo)) aP[r] = 0.f;
        } else if (!seen_as_a_whole(lo, hi)) {
#pragma unroll
          for (int r = 0; r < 16; ++r) aP[r] = 0.f;
        }
      }
#pragma unroll
      for (int i = 2 * ks; i < 2 * ks + 2; ++i) {
        fds[i] = as_operand(aP, i);
        if (CAREFUL && masked) continue;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_tr<ROWB>(tK, t_off[dt][0], t_off[dt][1], i), fds[i], acc[dt], 0, 0, 0);
      }
    }
    if (CAREFUL && masked) add_with_care<DH>(acc, fds, tK, [&](int dt, int r) { return t_off[dt][r]; }, lo, hi);
  }
  const bool odd = !CAREFUL && __syncthreads_or(not_finite<DT>(acc) && own.lo < own.hi);
  if (own.lo >= own.hi) return odd;
  bf16_t* row = a.dq + (int64_t)q_row * a.o.ld_q + hd * DH;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int rg = 0; rg < 4; ++rg) {
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = acc[dt][rg * 4 + j] * a.o.scale;
      store4(row + dt * 32 + rg * 8 + g * 4, v);
    }
  return odd;
}

// Both passes in one launch, the dK/dV workgroups first, they are the longer ones.  d_head 128: dK and dV come from workgroups of their own
// (PAIR), which compute the scores twice but have half the sums each, so that two waves fit a SIMD and one's matrix products run beside the
// other's exponentials (side by side, 8 sequences of 1024, 16 heads on 4: 199 us, 241 with both in one workgroup; 20 of 300, 16 heads: 139, 186;
// d_head 64 has room for both: 8192 rows 483 us so, 594 apart at three waves a SIMD).  The two of a unit are eight apart: on the same XCD, with the same Q and dO in its L2.
template <int DH, bool CAREFUL>
__device__ __forceinline__ bool block(const BwdArgs& a, int unit, char* smem, int* s_span) {
  constexpr bool PAIR = DH == 128;
  const int k_blocks = PAIR ? (a.k_units + 7) / 8 * 16 : a.k_units;
  if (unit >= k_blocks) return dq_block<DH, CAREFUL>(a, unit - k_blocks, smem, s_span);
  if constexpr (PAIR) {
    const int k = unit / 16 * 8 + unit % 8;
    if (k >= a.k_units) return false;
    return unit & 8 ? dkv_block<DH, 1, CAREFUL>(a, k, smem, s_span) : dkv_block<DH, 2, CAREFUL>(a, k, smem, s_span);
  } else {
    return dkv_block<DH, 3, CAREFUL>(a, unit, smem, s_span);
  }
}
template <int DH>
__global__ __launch_bounds__(256, 2) void packed_bwd_bf16_kernel(BwdArgs a) {
  extern __shared__ __align__(16) char dyn_smem[];
  __shared__ int s_span[2];
  if (block<DH, false>(a, (int)blockIdx.x, dyn_smem, s_span)) {
    __syncthreads();
    block<DH, true>(a, (int)blockIdx.x, dyn_smem, s_span);
  }
}

// What the host knows of the lengths: how many sequences there are.  Rows that a row meets, on average.
double rows_met(const PackedAttn& a) {
  const double length = (double)a.tokens / (a.n_seq > 1 ? a.n_seq : 1);
  return a.causal ? length / 2 : length;
}

// Parts of a block's tiles in dK/dV: the number with the least cost, which ranks them and is no time.  A workgroup takes `start` and `tile` per tile of 64
// queries; either the card's `slots` are full, or the longest block's chain counts (its sequence `longest` times the average);
// with parts, their fp32 sums go through memory at 4 TB/s in `join` more.  Fitted to 350 sizes with 1 to 16 parts (MI355X):
// 3 % off the best number on average, 33 % at most (one part everywhere: 37 %).  us with 1 / 2 / 4 / 8 / 16 parts, causal: 16 heads of 128
// on 2, 2 sequences of 4057 1100 / 666 / 568 / 583 / 652 (the rule: 4); 16 of 64 on 4, 8 of 585 83 / 59 / 60 / 76 / 107 (3: 55).
int splits_of(const PackedAttn& a) {
  struct Cost { double start, tile, slots, join, longest; };
  const Cost c = a.dh == 64 ? Cost{3.07, 1.2, 207, 2.37, 1.93} : Cost{13.2, 1.55, 155, 2.63, 1.83};
  const double units = (double)((a.tokens + 127) / 128 * a.h_kv), group = (double)(a.h / a.h_kv), length = (double)a.tokens / (a.n_seq > 1 ? a.n_seq : 1);
  const double most = a.n_seq > 1 ? std::min((double)a.tokens, c.longest * length) : length;
  const double tiles = group * ((rows_met(a) + 128) / 64 + 0.5), chain = group * ((most + 128) / 64 + 0.5);
  int best = 1;
  double least = 0;
  for (int s = 1; s <= 16 && (s == 1 || s <= 0.75 * tiles); ++s) {
    const double full = std::max(1.0, units * s / c.slots) * (c.start + tiles / s * c.tile);
    const double us = std::max(full, c.start + chain / s * c.tile) + (s > 1 ? c.join + (double)s * a.tokens * a.h_kv * a.dh * 16 / 4e6 : 0);
    if (s == 1 || us < least) {
      best = s;
      least = us;
    }
  }
  return best;
}

// how the work is divided: a function of the sizes alone
BwdArgs plan_of(const PackedAttn& a) {
  BwdArgs b{};
  b.k_blocks = (int32_t)((a.tokens + 127) / 128);
  b.splits = splits_of(a);
  b.k_units = b.k_blocks * a.h_kv * b.splits;
  b.heads = heads_together(a);
  const int rows = 128 / b.heads;
  b.q_blocks = (int32_t)((a.tokens + rows - 1) / rows);
  b.q_units = b.q_blocks * (a.h / b.heads);
  b.at_once = (b.k_units <= (a.dh == 64 ? 512 : 256) ? 1 : 0) | (b.q_units <= 512 ? 2 : 0);
  return b;
}
template <int DH>
hipError_t run(const PackedAttn& a, const BwdArgs& b, hipStream_t st) {
  constexpr int lds = 2 * (2 * 64 * DH * 2 + 512);
  hipError_t e = allow_lds((const void*)packed_bwd_bf16_kernel<DH>, lds);
  if (e != hipSuccess) return e;
  const int k_blocks = DH == 128 ? (b.k_units + 7) / 8 * 16 : b.k_units;
  hipLaunchKernelGGL(packed_bwd_bf16_kernel<DH>, dim3((unsigned)(k_blocks + b.q_units)), dim3(256), lds, st, b);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  return b.splits > 1 ? packed_join(a, b.partial, b.splits, b.dk, b.dv, st) : hipSuccess;
}

}  // namespace

BwdPlan packed_bwd_plan(const PackedAttn& a) {
  const BwdArgs b = plan_of(a);
  return BwdPlan{b.splits, b.at_once & 1, (b.at_once >> 1) & 1};
}

int64_t packed_bwd_bf16_bytes(const PackedAttn& a) { return packed_partial_bytes(a, splits_of(a)); }

hipError_t packed_bwd_bf16(const PackedAttn& a, const PackedQkv<bf16_t>& o, const void* dout, const float* lse, const float* dsum, void* dq, void* dk,
                           void* dv, void* workspace, hipStream_t st) {
  BwdArgs b = plan_of(a);
  b.o = o;
  b.dout = (const bf16_t*)dout;
  b.lse = lse;
  b.dsum = dsum;
  b.dq = (bf16_t*)dq;
  b.dk = (bf16_t*)dk;
  b.dv = (bf16_t*)dv;
  b.partial = b.splits > 1 ? (float*)workspace : nullptr;
  b.scale_log2e = LOG2E_P * o.scale;
  return a.dh == 64 ? run<64>(a, b, st) : run<128>(a, b, st);
}

}  // namespace pf
