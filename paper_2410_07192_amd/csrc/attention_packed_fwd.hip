// Attention forward on packed sequences, bf16, d_head 64 or 128, on the 32x32x16 bf16 MFMA (gfx950).
//
// S^T = K Q^T puts 32 of a tile's 64 scores of ONE query into a lane, so that sums run in registers and a query's two lanes
// (lane ^ 32) meet only when the softmax's reference point moves and at the end; the probabilities are then the "B" operand of
// O^T = V^T P^T as they lie, and V^T comes out of the row-major tile by the transposing LDS load.  K and V tiles go global ->
// LDS directly, one tile ahead.
//
// A wave has 32 rows of the packed buffer (of any sequences, see attention_packed.h) of one head.  The waves of a workgroup
// share K/V tiles: they are `heads` heads of one group, a power of two, times the blocks of 32 rows that follow each other.
// More heads and fewer rows read the same K/V for the same products but end nearer to the causal diagonal and to the ends of sequences.
//
// Bound by what a SIMD issues: for a wave's tile of d_head 128, matrix products take 1024 cycles, its share of the CU's LDS reads as many
// and the softmax about 900, and two waves overlap them in part: two sequences up to 8192, 32 heads on 4 of 128: 836 to 880 us, 1.02 to 1.07
// PFLOP/s (a large bf16 product reaches 1.2), the matrix units busy half of the cycles at 1.8 GHz; scores one tile ahead of their softmax in program order made it 838 from 805 us at 14192 rows, because
// the products then issue together all the same.  Short calls are bound by a block's chain: launch, boundaries, Q, first tiles, about 5 us
// before the first product, then 0.8 to 1.3 us a tile.
#include "attention_packed.h"

#include <algorithm>
#include <type_traits>

namespace pf {
namespace {

// A wave's 32 rows of one head: queries, running sums and output, and the steps over a tile of 64 keys in LDS
template <int DH>
struct FwdRows {
  static constexpr int KS = DH / 16, DT = DH / 32, ROWB = DH * 2, TILE = 64 * ROWB;
  bf16x8 fq[KS];
  f32x16 accO[DT];
  // m_ref: reference point of the running sum and of O (scaled scores, log2 units).  In tiles that every row sees it follows the running
  // maximum lazily: exponentials are taken against it as it stands, and it moves only when a lane's share of the tile's sum
  // exceeds 2^7, so that most tiles compute no maximum and rescale nothing.  l_run: this lane's share of the sum, 32 of every 64 keys.
  float m_ref, l_run, scale_log2e;
  Span own;
  int lr, g, v_off0, v_off1;

  __device__ __forceinline__ void load(const PackedQkv<bf16_t>& a, int hd, int q_row) {
    const bf16_t* p = a.q + (int64_t)min(q_row, a.rows.tokens - 1) * a.ld_q + hd * DH + g * 8;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) fq[kk] = as_bf16x8(*(const uint4*)(p + kk * 16));
  }
  __device__ __forceinline__ void begin() {
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) asm volatile("" ::"v"(fq[kk]));   // waited for here, once
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) accO[i][r] = 0.f;
    m_ref = -INFINITY;
    l_run = 0.f;
  }
  __device__ __forceinline__ void scores(const char* sK, f32x16* s) const {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[ks][r] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int r = ks * 32 + lr;
        const uint4 fk = *(const uint4*)(sK + r * ROWB + (((kk * 2 + g) ^ swz_row<DH>(r)) << 4));
        s[ks] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(fk), fq[kk], s[ks], 0, 0, 0);
      }
  }
  __device__ __forceinline__ float exponentials(f32x16* s, float neg_m) const {   // their sum
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[ks][r] = __builtin_amdgcn_exp2f(fmaf(s[ks][r], scale_log2e, neg_m));
        part[r & 3] += s[ks][r];
      }
    return (part[0] + part[1]) + (part[2] + part[3]);
  }
  // Scores of the tile at key k0 into probabilities.  masked: not every row sees every key; fresh: nothing has been added yet.
  __device__ __forceinline__ void probabilities(const char* sK, f32x16* s, int k0, bool masked, bool fresh) {
    // Most tiles that are masked lie in the block's first sequence and none of its rows of the next one sees them: a lane's row sees all of
    // the tile or nothing of it (2048 rows behind 5 others, 16 heads on 2 of 128: 65 us with every such tile masked by element, 52 so).
    // A row that has met no score but -inf yet has no reference point: its sum is infinite or NaN here, and the tile is done again.
    const int lo = own.lo - k0, hi = own.hi - k0;
    if (!fresh && !(masked && __any(seen_in_part(lo, hi)))) {
      const float tot = exponentials(s, seen_as_a_whole(lo, hi) ? -m_ref : -INFINITY);
      if (!__any(!(tot <= 128.0f))) {   // (also infinite or NaN)
        l_run += tot;
        return;
      }
      scores(sK, s);
    }
    if (masked) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (hidden_at(ks * 32 + 8 * (r >> 2) + (r & 3), lo - 4 * g, hi - lo)) s[ks][r] = -INFINITY;
    }
    float mx0 = fmaxf(s[0][0], s[1][0]), mx1 = fmaxf(s[0][1], s[1][1]);
#pragma unroll
    for (int r = 2; r < 16; r += 2) {
      mx0 = fmaxf(fmaxf(mx0, s[0][r]), s[1][r]);
      mx1 = fmaxf(fmaxf(mx1, s[0][r + 1]), s[1][r + 1]);
    }
    float mx_lo, mx_hi;
    both_halves(fmaxf(mx0, mx1), mx_lo, mx_hi);
    const float m_new = fmaxf(m_ref, fmaxf(mx_lo, mx_hi) * scale_log2e);
    if (!fresh && __any(m_new > m_ref)) {
      const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_ref - m_new);   // m_ref = -inf: 0
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) accO[i][r] *= alpha;
    }
    m_ref = m_new;
    l_run += exponentials(s, m_ref == -INFINITY ? 0.f : -m_ref);
  }
  // O^T += V^T P^T.  P is rounded to bf16 (half a step, 2^-8 of each), its sum is not.
  __device__ __forceinline__ int v_off(int dt) const { return ((dt & 1) ? v_off1 : v_off0) + (dt >> 1) * 128; }
  __device__ __forceinline__ void add(lds_char_ptr sV, const f32x16* s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x8 fp = as_operand(s[i >> 1], i);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        accO[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_tr<ROWB>(sV, v_off(dt), v_off(dt), i), fp, accO[dt], 0, 0, 0);
    }
  }
  __device__ __forceinline__ void add_careful(lds_char_ptr sV, const f32x16* s, int k0) {
    bf16x8 fp[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) fp[i] = as_operand(s[i >> 1], i);
    add_with_care<DH>(accO, fp, sV, [&](int dt, int) { return v_off(dt); }, own.lo - k0, own.hi - k0);
  }
  // whether a result is infinite or NaN, which rows hidden from it may have brought in: then the block is done once more, with care
  __device__ __forceinline__ bool odd() const {
    bool r_ = false;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) r_ = r_ || !(fabsf(accO[i][r]) < INFINITY);
    return r_ && own.lo < own.hi;
  }
  __device__ __forceinline__ void sum_halves() {
    float lo, hi;
    both_halves(l_run, lo, hi);
    l_run = lo + hi;
  }
  __device__ __forceinline__ void store(const PackedQkv<bf16_t>& a, int hd, int q_row, bf16_t* out, float* lse) const {
    if (own.lo >= own.hi) return;
    const float inv = 1.f / l_run;   // a row whose scores are all -inf has no softmax: 0 / 0
    bf16_t* orow = out + (int64_t)q_row * a.ld_out + hd * DH;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        const float v[4] = {accO[dt][rg * 4] * inv, accO[dt][rg * 4 + 1] * inv, accO[dt][rg * 4 + 2] * inv, accO[dt][rg * 4 + 3] * inv};
        store4(orow + dt * 32 + rg * 8 + g * 4, v);
      }
    if (lse && g == 0) lse[(int64_t)hd * a.rows.tokens + q_row] = m_ref * LN2_P + __logf(l_run);
  }
};

struct FwdGrid {
  int32_t heads, groups, blocks, log_rows;   // of a workgroup; of the call; of rows; rows of a block
  int32_t at_once;                             // whether all workgroups start at the same time
  float scale_log2e;
};
// A workgroup's block of rows and heads: four waves share K/V tiles.  KG = 2: twice four, the second four with every other tile, so
// that a block's own chain over the keys is half as long; their sums meet in LDS.
// Registers for three waves a SIMD (d_head 64; 12 sequences of 1024, 16 heads on 4, side by side: 46.6 us, 53.0 with two; four do not fit, 108; now
// 42.2) or two.
template <int DH, int KG>
__global__ __launch_bounds__(256 * KG, DH == 64 ? 3 : 2) void packed_fwd_bf16_kernel(PackedQkv<bf16_t> a, bf16_t* __restrict__ out, float* __restrict__ lse, FwdGrid grid) {
  constexpr int NW = 4, TILE = 64 * DH * 2, BUF = KG * 2 * TILE, DT = DH / 32, LD = DH + 4;
  static_assert(KG == 1 || NW * 32 * LD * 4 <= 2 * BUF, "O of one part fits the buffers");
  extern __shared__ __align__(16) char smem[];   // two buffers of KG (K tile | V tile)
  __shared__ int s_span[2];
  __shared__ float s_ml[KG > 1 ? NW : 1][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6) % NW, part = __builtin_amdgcn_readfirstlane(tid >> 6) / NW;
  // head groups fastest: workgroups with the same rows run at the same time
  const int hg = (int)(blockIdx.x % (uint32_t)grid.groups);
  const int blk = block_in_order(a.rows, (int)(blockIdx.x / (uint32_t)grid.groups), grid.blocks, grid.log_rows, a.causal, false, grid.at_once);
  const int hd = hg * grid.heads + wave % grid.heads;
  const int q_blk = (blk * (NW / grid.heads) + wave / grid.heads) * 32;
  FwdRows<DH> w;
  w.lr = lane & 31;
  w.g = lane >> 5;
  w.scale_log2e = grid.scale_log2e;
  w.v_off0 = TILE + tr_offset<DH>(lane, 0);   // the other two of d_head 128: 128 bytes on
  w.v_off1 = TILE + tr_offset<DH>(lane, 1);
  w.load(a, hd, q_blk + w.lr);
  w.own = keys_of(a.rows, q_blk, q_blk + w.lr, a.causal);
  const int w_lo = lane_value(w.own.lo, 0), w_hi = lane_value(w.own.hi, 31);       // of the wave
  const int in_lo = lane_value(w.own.lo, 31), in_hi = lane_value(w.own.hi, 0);     // inside them every row sees every key
  if (tid == 0) s_span[0] = w_lo;
  if (tid == 64 * (NW - 1)) s_span[1] = w_hi;   // of part 0
  __syncthreads();
  const int k_begin = __builtin_amdgcn_readfirstlane(s_span[0]), k_end = __builtin_amdgcn_readfirstlane(s_span[1]);
  const int n_tiles = k_end > k_begin ? (k_end - k_begin + 63) >> 6 : 0;

  const bf16_t* kh = a.k + hd / a.group * DH;
  const bf16_t* vh = a.v + hd / a.group * DH;
  TileCopy<DH, NW, SwzRow<DH>> copy_k;
  TileCopy<DH, NW, SwzCol<DH>> copy_v;
  copy_k.init(a.ld_k, wave);
  copy_v.init(a.ld_v, wave);
  const uint32_t lds_base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_ptr)smem) + (uint32_t)(part * 2 * TILE + wave * 1024);
  auto stage = [&](int buf, int k0) {
    if (KG > 1 && k0 >= k_end) return;
    copy_k.issue(kh, lds_base + (uint32_t)(buf * BUF), k0, k_end);
    copy_v.issue(vh, lds_base + (uint32_t)(buf * BUF + TILE), k0, k_end);
  };
  auto walk = [&](auto careful_) {
    constexpr bool CAREFUL = decltype(careful_)::value;
    if (n_tiles > 0) stage(0, k_begin + part * 64);
    w.begin();
    bool fresh = true;
    for (int kt = part; kt - part < n_tiles; kt += KG) {   // as many steps in every part
      const int k0 = k_begin + kt * 64, buf = (kt / KG) & 1;
      // tile kt has landed (every wave waits for its own copies, then the barrier), and everyone has left the tile before it
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (k0 + KG * 64 < k_end) stage(buf ^ 1, k0 + KG * 64);
      if (k0 + 64 <= w_lo || k0 >= w_hi) continue;   // none of the wave's rows sees the tile
      const char* sK = smem + buf * BUF + part * 2 * TILE;
      lds_char_ptr sV = (lds_char_ptr)(lds_void_ptr)smem + buf * BUF + part * 2 * TILE;
      const bool masked = k0 < in_lo || k0 + 64 > in_hi;
      f32x16 s[2];
      __builtin_amdgcn_s_setprio(1);   // the other wave of the SIMD fills the gaps
      w.scores(sK, s);
      __builtin_amdgcn_s_setprio(0);
      w.probabilities(sK, s, k0, masked, fresh);
      fresh = false;
      if (CAREFUL && masked) {
        w.add_careful(sV, s, k0);
        continue;
      }
      __builtin_amdgcn_s_setprio(1);
      w.add(sV, s);
      __builtin_amdgcn_s_setprio(0);
    }
  };
  walk(std::false_type{});
  if (__syncthreads_or(w.odd())) walk(std::true_type{});
  w.sum_halves();
  if constexpr (KG == 2) {   // the second part's maximum, sum and O meet the first's
    __syncthreads();
    float* sO = (float*)smem + wave * 32 * LD;
    float* sML = s_ml[wave];
    if (part == 1) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg)
          *(f32x4*)(sO + w.lr * LD + dt * 32 + rg * 8 + w.g * 4) =
              f32x4{w.accO[dt][rg * 4], w.accO[dt][rg * 4 + 1], w.accO[dt][rg * 4 + 2], w.accO[dt][rg * 4 + 3]};
      if (w.g == 0) {
        sML[w.lr] = w.m_ref;
        sML[32 + w.lr] = w.l_run;
      }
    }
    __syncthreads();
    if (part == 1) return;
    const float m1 = sML[w.lr], m = fmaxf(w.m_ref, m1);
    const float f0 = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(w.m_ref - m), f1 = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m1 - m);
    w.l_run = w.l_run * f0 + sML[32 + w.lr] * f1;
    w.m_ref = m;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        const f32x4 x = *(const f32x4*)(sO + w.lr * LD + dt * 32 + rg * 8 + w.g * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) w.accO[dt][rg * 4 + j] = w.accO[dt][rg * 4 + j] * f0 + x[j] * f1;
      }
  }
  w.store(a, hd, q_blk + w.lr, out, lse);
}

// Independent waves: each has 32 rows of one head and K/V buffers of its own, so nothing waits for another wave.  KG waves share
// the keys of a unit (tile kt belongs to wave kt % KG) and join their (maximum, sum, O) in LDS.  For short sequences, whose
// tiles few rows share anyway, and for few rows, where a unit's own chain over the keys is the time.
template <int DH, int KG>
__global__ __launch_bounds__(256, DH == 64 ? 2 : 1) void packed_fwd_units_kernel(PackedQkv<bf16_t> a, bf16_t* __restrict__ out,
                                                                                 float* __restrict__ lse, int32_t blocks, int64_t units,
                                                                                 int32_t at_once, float scale_log2e) {
  constexpr int DT = DH / 32, TILE = 64 * DH * 2, NI = TILE / 1024, UNITS = 4 / KG, LD = DH + 4, CPR = DH / 8;
  constexpr int OWN = 2 * TILE + 2048;   // K tile | V tile; later O
  static_assert(32 * LD * 4 <= OWN, "O of a wave fits its buffers");
  extern __shared__ __align__(16) char dyn_smem[];
  __shared__ float sM[4][32], sL[4][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave % KG;
  const int64_t unit = (int64_t)blockIdx.x * UNITS + wave / KG;
  const bool real = unit < units;                    // heads fastest
  const int hd = real ? (int)(unit % a.h) : 0;
  const int q_blk = real ? block_in_order(a.rows, (int)(unit / a.h), blocks, 5, a.causal, false, at_once) * 32 : 0;
  FwdRows<DH> w;
  w.lr = lane & 31;
  w.g = lane >> 5;
  w.scale_log2e = scale_log2e;
  w.v_off0 = TILE + tr_offset<DH>(lane, 0);
  w.v_off1 = TILE + tr_offset<DH>(lane, 1);
  w.load(a, hd, q_blk + w.lr);
  w.own = keys_of(a.rows, q_blk, q_blk + w.lr, a.causal);
  if (!real) w.own.hi = w.own.lo;
  const int k_begin = lane_value(w.own.lo, 0), k_end = lane_value(w.own.hi, 31);
  const int in_lo = lane_value(w.own.lo, 31), in_hi = lane_value(w.own.hi, 0);
  const int n_tiles = real && k_end > k_begin ? (k_end - k_begin + 63) >> 6 : 0;

  char* const mine = dyn_smem + wave * OWN;
  lds_char_ptr sV = (lds_char_ptr)(lds_void_ptr)dyn_smem + wave * OWN;
  const uint32_t lds_base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_ptr)dyn_smem) + (uint32_t)(wave * OWN);
  const bf16_t* kh = a.k + hd / a.group * DH;
  const bf16_t* vh = a.v + hd / a.group * DH;
  TileCopy<DH, 1, SwzRow<DH>> copy_k;
  TileCopy<DH, 1, SwzCol<DH>> copy_v;
  copy_k.init(a.ld_k, 0);
  copy_v.init(a.ld_v, 0);
  auto walk = [&](auto careful_) {
    constexpr bool CAREFUL = decltype(careful_)::value;
    if (part < n_tiles) {
      copy_k.issue(kh, lds_base, k_begin + part * 64, k_end);
      copy_v.issue(vh, lds_base + TILE, k_begin + part * 64, k_end);
    }
    w.begin();
#pragma unroll 1
    for (int kt = part; kt < n_tiles; kt += KG) {
      const int k0 = k_begin + kt * 64;
      const bool more = kt + KG < n_tiles, masked = k0 < in_lo || k0 + 64 > in_hi;
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NI) : "memory");   // K of the tile has landed; V's NI copies may be on their way
      f32x16 s[2];
      w.scores(mine, s);
      w.probabilities(mine, s, k0, masked, kt == part);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // K has been read: the next tile's may come
      if (more) {
        copy_k.issue(kh, lds_base, k0 + KG * 64, k_end);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NI) : "memory");   // V has landed
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      if (CAREFUL && masked) w.add_careful(sV, s, k0);
      else w.add(sV, s);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) copy_v.issue(vh, lds_base + TILE, k0 + KG * 64, k_end);
    }
  };
  walk(std::false_type{});
  if (__any(w.odd())) walk(std::true_type{});
  w.sum_halves();
  if constexpr (KG == 1) {
    w.store(a, hd, q_blk + w.lr, out, lse);
  } else {
    if (w.g == 0) {
      sM[wave][w.lr] = w.m_ref;
      sL[wave][w.lr] = w.l_run;
    }
    float* sO = (float*)mine;   // this wave's reads of its buffers are complete
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg)
        *(f32x4*)(sO + w.lr * LD + dt * 32 + rg * 8 + w.g * 4) =
            f32x4{w.accO[dt][rg * 4], w.accO[dt][rg * 4 + 1], w.accO[dt][rg * 4 + 2], w.accO[dt][rg * 4 + 3]};
    const uint64_t live = __ballot(w.own.lo < w.own.hi);
    __syncthreads();
    const int first = wave / KG * KG;   // the unit's waves share its rows
    for (int e = part * 64 + lane; e < 32 * CPR; e += 64 * KG) {
      const int q = e / CPR, c = e % CPR * 8;
      if (!((live >> q) & 1)) continue;
      float mq = sM[first][q];
#pragma unroll
      for (int i = 1; i < KG; ++i) mq = fmaxf(mq, sM[first + i][q]);
      float lq = 0.f, o[8] = {};
#pragma unroll
      for (int i = 0; i < KG; ++i) {
        const float f = mq == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(sM[first + i][q] - mq);   // 0 for a wave that met no key
        const float* po = (const float*)(dyn_smem + (first + i) * OWN) + q * LD + c;
        const f32x4 x = *(const f32x4*)po, y = *(const f32x4*)(po + 4);
        lq += f * sL[first + i][q];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          o[j] += f * x[j];
          o[4 + j] += f * y[j];
        }
      }
      const float inv = 1.f / lq;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] *= inv;
      store8(out + (int64_t)(q_blk + q) * a.ld_out + hd * DH + c, o);
      if (lse && c == 0) lse[(int64_t)hd * a.rows.tokens + q_blk + q] = mq * LN2_P + __logf(lq);
    }
  }
}

template <int DH, int KG>
hipError_t launch_units(const PackedAttn& a, const PackedQkv<bf16_t>& o, const FwdPlan& p, void* out, float* lse, hipStream_t st) {
  constexpr int lds = 4 * (2 * 64 * DH * 2 + 2048);
  hipError_t e = allow_lds((const void*)packed_fwd_units_kernel<DH, KG>, lds);
  if (e != hipSuccess) return e;
  const int64_t blocks = (a.tokens + 31) / 32, units = blocks * a.h;
  hipLaunchKernelGGL((packed_fwd_units_kernel<DH, KG>), dim3((unsigned)((units * KG + 3) / 4)), dim3(256), lds, st, o, (bf16_t*)out, lse, (int32_t)blocks, units, p.at_once,
                     LOG2E_P * o.scale);
  return hipGetLastError();
}

template <int DH, int KG>
hipError_t launch(const PackedAttn& a, const PackedQkv<bf16_t>& o, const FwdPlan& p, void* out, float* lse, hipStream_t st) {
  constexpr int lds = 2 * KG * 2 * 64 * DH * 2;
  hipError_t e = allow_lds((const void*)packed_fwd_bf16_kernel<DH, KG>, lds);
  if (e != hipSuccess) return e;
  const int rows = 128 / p.heads, log_rows = __builtin_ctz(rows);
  const int64_t blocks = (a.tokens + rows - 1) / rows;
  const FwdGrid grid{p.heads, a.h / p.heads, (int32_t)blocks, log_rows, p.at_once, LOG2E_P * o.scale};
  hipLaunchKernelGGL((packed_fwd_bf16_kernel<DH, KG>), dim3((unsigned)(blocks * grid.groups)), dim3(256 * KG), lds, st, o, (bf16_t*)out, lse, grid);
  return hipGetLastError();
}

// Which form is fastest: shared tiles, a block's keys in one or two parts, or independent waves with 1, 2 or 4 to a unit's keys.  Each
// form's cost is the longer of two terms and some of the other: its workgroups go through the card (start + tiles x full, times
// the number of fillings of its `slots`), and its longest block's chain (start + tiles x alone).  Lengths are on the device, so the
// longest sequence is taken to be twice the average.  The costs rank the forms and are no times: 16 prompts up to 2048 are put at 36 and
// take 52 us, 2 documents up to 8192 at 1591 and take 874.  Their constants are fitted to 600 sizes timed in every form (MI355X): 2.0 % (d_head 64)
// and 1.6 % (128) off the fastest form on average, 47 % at most; the best single form would be 16 % and 26 % off.
// us in forms shared 1 / shared 2 / waves 1 / 2 / 4: 16 heads on 2 of 128, 333 rows 13.3 / 13.3 / 14.2 / 11.0 / 8.9; 16 sequences up
// to 2048 51.8 / 54.3 / 58.0 / 74.8 / 114; 2 up to 8192, 32 on 4 heads 874 / 960 / 1199 / 1331 / 1890; 12 heads of 64, 32 up to 512
// 21.1 / - / 23.7 / 24.4 / 30.0 (the rule takes one wave, 12 % off).
FwdForm fwd_form(const PackedAttn& a, int heads) {
  struct Cost { FwdForm form; int parts, slots; double start, full, alone; };
  static const Cost costs64[] = {{SHARED_1, 1, 768, 5.85, 2.14, 0.91}, {WAVES_1, 1, 512, 5.66, 1.61, 0.85}, {WAVES_2, 2, 512, 6.01, 1.43, 0.79},
                                 {WAVES_4, 4, 512, 5.49, 1.36, 0.82}};
  static const Cost costs128[] = {{SHARED_1, 1, 512, 7.24, 2.30, 1.25}, {SHARED_2, 2, 512, 8.49, 2.38, 1.63}, {WAVES_1, 1, 256, 6.96, 1.70, 1.32},
                                  {WAVES_2, 2, 256, 7.44, 1.63, 1.11}, {WAVES_4, 4, 256, 6.51, 1.72, 0.99}};
  const bool small = a.dh == 64, several = a.n_seq > 1;
  const double length = (double)a.tokens / (several ? a.n_seq : 1);
  const double longest = several ? std::min((double)a.tokens, 2 * length) : length, met = (several ? 1.5 : 1.0) * length / (a.causal ? 2 : 1);
  FwdForm best = SHARED_1;
  double least = 0;
  for (const Cost* c = small ? costs64 : costs128; c != (small ? costs64 + 4 : costs128 + 5); ++c) {
    const bool shared = c->form == SHARED_1 || c->form == SHARED_2;
    const double rows = shared ? 128.0 / heads : 32.0;
    const double workgroups = ceil(a.tokens / rows) * a.h * c->parts / (shared ? heads : 4);
    const double tiles = ((met + rows) / 64 + 0.5) / c->parts, chain = ((longest + rows) / 64 + 0.5) / c->parts;
    const double all = workgroups / c->slots * (c->start + (shared ? tiles : std::max(1.0, tiles)) * c->full);
    const double one = c->start + (shared ? chain : ceil(chain)) * c->alone;
    const double us = std::max(all, one) + 0.35 * std::min(all, one);
    if (c->form == SHARED_1 || us < least) {
      best = c->form;
      least = us;
    }
  }
  return best;
}

}  // namespace

FwdPlan packed_fwd_plan(const PackedAttn& a) {
  const int heads = heads_together(a);
  const FwdForm form = fwd_form(a, heads);
  const bool shared = form == SHARED_1 || form == SHARED_2, small = a.dh == 64;
  const int parts = form == SHARED_2 || form == WAVES_2 ? 2 : form == WAVES_4 ? 4 : 1;
  const int64_t rows = shared ? 128 / heads : 32;
  const int64_t work = (a.tokens + rows - 1) / rows * (shared ? a.h / heads : a.h) * parts;   // shared: fours of waves; else waves
  return FwdPlan{form, heads, shared ? work <= (small ? 768 : 512) : work / 4 <= (small ? 512 : 256)};
}

hipError_t packed_fwd_bf16(const PackedAttn& a, const PackedQkv<bf16_t>& o, void* out, float* lse, hipStream_t st) {
  const FwdPlan p = packed_fwd_plan(a);
  const bool small = a.dh == 64;
  switch (p.form) {
    case WAVES_1: return small ? launch_units<64, 1>(a, o, p, out, lse, st) : launch_units<128, 1>(a, o, p, out, lse, st);
    case WAVES_2: return small ? launch_units<64, 2>(a, o, p, out, lse, st) : launch_units<128, 2>(a, o, p, out, lse, st);
    case WAVES_4: return small ? launch_units<64, 4>(a, o, p, out, lse, st) : launch_units<128, 4>(a, o, p, out, lse, st);
    case SHARED_2: return small ? hipErrorInvalidValue : launch<128, 2>(a, o, p, out, lse, st);   // there is none of d_head 64, and no rule picks it
    default: return small ? launch<64, 1>(a, o, p, out, lse, st) : launch<128, 1>(a, o, p, out, lse, st);
  }
}

}  // namespace pf
