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
#include "attention_packed.h"

namespace pf {
namespace {

// O += P V for a tile that not every row sees as a whole, key by key and visible ones only: 0 (hidden) times an infinity or NaN
// of another row's V would be NaN.  p: the probabilities as the products left them; sp: 2 KiB of LDS of this wave.
template <int DH>
__device__ __forceinline__ void add_keys(f32x16* accO, const f32x16* p, const char* sV, bf16_t* sp, int k0, Span own) {
  constexpr int DT = DH / 32, ROWB = DH * 2;
  const int lane = threadIdx.x & 63, lr = lane & 31, g = lane >> 5;
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // within the wave: its LDS instructions execute in order
#pragma unroll
    for (int r = 0; r < 16; ++r) sp[(8 * (r >> 2) + 4 * g + (r & 3)) * 32 + lr] = from_f32<bf16_t>(p[ks][r]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 1
    for (int i = 0; i < 32; ++i) {
      const int key = ks * 32 + i;
      if (k0 + key < own.lo || k0 + key >= own.hi) continue;
      const float w = to_f32(sp[i * 32 + lr]);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
          asm volatile("" ::: "memory");   // a few registers are enough here
          float x[4];
          load4((const bf16_t*)(sV + key * ROWB + (((dt * 4 + rg) ^ swz_col<DH>(i)) << 4) + 8 * g), x);
#pragma unroll
          for (int j = 0; j < 4; ++j) accO[dt][rg * 4 + j] = fmaf(w, x[j], accO[dt][rg * 4 + j]);
        }
    }
  }
}

// One workgroup's block of rows and heads.  False, and nothing stored: a result is infinite or NaN, which hidden rows may have
// brought in (never so with CAREFUL).  smem: two buffers of (K tile | V tile); s_span: two ints.
struct FwdGrid {
  int32_t heads, groups, blocks;   // of a workgroup; of the call; of rows
  float scale_log2e;
};
template <int DH, int NW, bool CAREFUL>
__device__ __forceinline__ bool fwd_block(const PackedQkv<bf16_t>& a, bf16_t* out, float* lse, const FwdGrid& grid, char* smem, int* s_span) {
  constexpr int CPR = DH / 8, KS = DH / 16, DT = DH / 32, ROWB = DH * 2, TILE = 64 * ROWB, NI = TILE / 1024, RPI = 1024 / ROWB;
  constexpr int PER = NI / NW;   // copies per wave of a K or V tile
  static_assert((NW * RPI) % 16 == 0 && NI % NW == 0, "rows of one lane's copies must share their swizzle");

  const int heads = grid.heads, groups = grid.groups;
  const float scale_log2e = grid.scale_log2e;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, g = lane >> 5;
  // head groups fastest: workgroups with the same K/V and neighbouring rows run at the same time; the last rows (causal: the
  // long ones) first
  const int hg = (int)(blockIdx.x % (uint32_t)groups), blk = grid.blocks - 1 - (int)(blockIdx.x / (uint32_t)groups);
  const int hd = hg * heads + wave % heads, T = a.rows.tokens;
  const int q_blk = (blk * (NW / heads) + wave / heads) * 32, q_row = q_blk + lr;
  bf16x8 fq[KS];
  {
    const bf16_t* p = a.q + (int64_t)min(q_row, T - 1) * a.ld_q + hd * DH + g * 8;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) fq[kk] = as_bf16x8(*(const uint4*)(p + kk * 16));
  }
  const Span own = keys_of(a.rows, q_blk, q_row, a.causal);
  const int w_lo = lane_value(own.lo, 0), w_hi = lane_value(own.hi, 31);       // of the wave
  const int in_lo = lane_value(own.lo, 31), in_hi = lane_value(own.hi, 0);     // inside them every row sees every key
  if (tid == 0) s_span[0] = w_lo;
  if (tid == 64 * (NW - 1)) s_span[1] = w_hi;
  __syncthreads();
  const int k_begin = __builtin_amdgcn_readfirstlane(s_span[0]), k_end = __builtin_amdgcn_readfirstlane(s_span[1]);
  const int n_tiles = k_end > k_begin ? (k_end - k_begin + 63) >> 6 : 0;

  const int st_row = wave * RPI + lane / CPR;
  const bf16_t* kh = a.k + hd / a.group * DH + (((lane % CPR) ^ swz_row<DH>(st_row)) << 3);
  const bf16_t* vh = a.v + hd / a.group * DH + (((lane % CPR) ^ swz_col<DH>(st_row)) << 3);
  const uint32_t lds_base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_ptr)smem);
  const uint32_t ldb_k = (uint32_t)a.ld_k * 2, ldb_v = (uint32_t)a.ld_v * 2;   // bytes (strides are at most 2^30)
  auto stage = [&](int buf, int k0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_base + (uint32_t)(buf * 2 * TILE + (wave + NW * i) * 1024));
      const uint32_t row = min(k0 + st_row + NW * i * RPI, k_end - 1);   // rows past the end repeat the last one and are hidden
      lds_direct_load_1k(dst, (const char*)kh + (uint64_t)row * ldb_k);
      lds_direct_load_1k(dst + TILE, (const char*)vh + (uint64_t)row * ldb_v);
    }
  };
  const int v_off0 = TILE + tr_offset<DH>(lane, 0), v_off1 = TILE + tr_offset<DH>(lane, 1);   // the other two of d_head 128: 128 bytes on

  f32x16 accO[DT];
  // Reference point of the running sum and of O (scaled scores, log2 units).  It follows the running maximum lazily: it moves
  // only when a lane's share of a tile's sum against it exceeds 2^7, so most tiles compute no maximum and rescale nothing.
  float m_ref, l_run;   // l_run: this lane's share, 32 of every 64 keys
  static_assert(NW * 2048 <= 2 * TILE, "the second buffer holds a careful wave's probabilities");
  if (!CAREFUL && n_tiles > 0) stage(0, k_begin);
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) asm volatile("" ::"v"(fq[kk]));   // waited for here, once
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) accO[i][r] = 0.f;
  m_ref = -INFINITY;
  l_run = 0.f;
  for (int kt = 0; kt < n_tiles; ++kt) {
    const int k0 = k_begin + kt * 64, buf = CAREFUL ? 0 : kt & 1;
    if (CAREFUL) {
      __syncthreads();
      stage(0, k0);
    }
    // tile kt has landed (every wave waits for its own copies, then the barrier), and everyone has left the tile before it
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (!CAREFUL && kt + 1 < n_tiles) stage(buf ^ 1, k0 + 64);
    if (k0 + 64 <= w_lo || k0 >= w_hi) continue;   // none of the wave's rows sees the tile
    const char* sK = smem + buf * 2 * TILE;
    lds_char_ptr sV = (lds_char_ptr)(lds_void_ptr)smem + buf * 2 * TILE;
    const bool masked = k0 < in_lo || k0 + 64 > in_hi;
    f32x16 s[2];
    auto scores = [&] {
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
      if (masked) {
        const int lo = own.lo - k0 - 4 * g, hi = own.hi - k0 - 4 * g;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = ks * 32 + 8 * (r >> 2) + (r & 3);
            if (key < lo || key >= hi) s[ks][r] = -INFINITY;
          }
      }
    };
    scores();
    const float neg_m = m_ref == -INFINITY ? 0.f : -m_ref;
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[ks][r] = __builtin_amdgcn_exp2f(fmaf(s[ks][r], scale_log2e, neg_m));
        part[r & 3] += s[ks][r];
      }
    float tot = (part[0] + part[1]) + (part[2] + part[3]);
    // Rare: no reference point yet, or the sum against the old one is over 2^7 (also infinite or NaN): scores again, the reference
    // point moves to the running maximum, O and the running sum are rescaled
    if (__any(!(tot <= 128.0f) || m_ref == -INFINITY)) {
      scores();
      float mx0 = fmaxf(s[0][0], s[1][0]), mx1 = fmaxf(s[0][1], s[1][1]);
#pragma unroll
      for (int r = 2; r < 16; r += 2) {
        mx0 = fmaxf(fmaxf(mx0, s[0][r]), s[1][r]);
        mx1 = fmaxf(fmaxf(mx1, s[0][r + 1]), s[1][r + 1]);
      }
      float lo, hi;
      both_halves(fmaxf(mx0, mx1), lo, hi);
      const float m_new = fmaxf(m_ref, fmaxf(lo, hi) * scale_log2e);
      const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_ref - m_new);   // m_ref = -inf: 0
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) accO[i][r] *= alpha;
      m_ref = m_new;
      const float neg = m_ref == -INFINITY ? 0.f : -m_ref;
      tot = 0.f;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[ks][r] = __builtin_amdgcn_exp2f(fmaf(s[ks][r], scale_log2e, neg));
          tot += s[ks][r];
        }
    }
    l_run += tot;
    if (CAREFUL && masked) {
      add_keys<DH>(accO, s, sK + TILE, (bf16_t*)(smem + 2 * TILE + wave * 2048), k0, own);
      continue;
    }
    // O^T += V^T P^T: K step i covers keys 16 i .. 16 i + 15, operand slot (g, t) is key 16 i + 8 (t / 4) + 4 g + t % 4 =
    // register 8 (i % 2) + t of sub-tile i / 2.  P is rounded to bf16 (half a step, 2^-8 of each), its sum is not.
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x8 fp;
#pragma unroll
      for (int t = 0; t < 8; ++t) fp[t] = (__bf16)s[i >> 1][8 * (i & 1) + t];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const int off = ((dt & 1) ? v_off1 : v_off0) + (dt >> 1) * 128;
        accO[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_tr<ROWB>(sV, off, off, i), fp, accO[dt], 0, 0, 0);
      }
    }
  }
  if (!CAREFUL) {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) odd = odd || !(fabsf(accO[i][r]) < INFINITY);
    if (__syncthreads_or(odd && own.lo < own.hi)) return false;
  }
  float lo, hi;
  both_halves(l_run, lo, hi);
  l_run = lo + hi;
  if (own.lo < own.hi) {
    const float inv = 1.f / l_run;   // a row whose scores are all -inf has no softmax: 0 / 0
    bf16_t* orow = out + (int64_t)q_row * a.ld_out + hd * DH;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        const float v[4] = {accO[dt][rg * 4] * inv, accO[dt][rg * 4 + 1] * inv, accO[dt][rg * 4 + 2] * inv, accO[dt][rg * 4 + 3] * inv};
        store4(orow + dt * 32 + rg * 8 + g * 4, v);
      }
    if (lse && g == 0) lse[(int64_t)hd * T + q_row] = m_ref * LN2_P + __logf(l_run);
  }
  return true;
}

// apart from the kernel: its registers are not the kernel's concern
template <int DH, int NW>
__device__ __noinline__ void fwd_block_with_care(PackedQkv<bf16_t> a, bf16_t* out, float* lse, FwdGrid grid, char* smem, int* s_span) {
  fwd_block<DH, NW, true>(a, out, lse, grid, smem, s_span);
}

template <int DH, int NW>
__global__ __launch_bounds__(64 * NW, DH == 64 ? 4 : 2) void packed_fwd_bf16_kernel(PackedQkv<bf16_t> a, bf16_t* __restrict__ out,
                                                                                    float* __restrict__ lse, FwdGrid grid) {
  __shared__ __align__(16) char smem[2 * 2 * 64 * DH * 2];
  __shared__ int s_span[2];
  if (!fwd_block<DH, NW, false>(a, out, lse, grid, smem, s_span)) fwd_block_with_care<DH, NW>(a, out, lse, grid, smem, s_span);
}

template <int DH, int NW>
hipError_t launch(const PackedAttn& a, const PackedQkv<bf16_t>& o, void* out, float* lse, hipStream_t st) {
  int heads = 1;
  while (heads < NW && (a.h / a.h_kv) % (heads * 2) == 0) heads *= 2;
  const int rows = 32 * NW / heads;
  const int64_t blocks = (a.tokens + rows - 1) / rows;
  const FwdGrid grid{heads, a.h / heads, (int32_t)blocks, LOG2E_P * o.scale};
  hipLaunchKernelGGL((packed_fwd_bf16_kernel<DH, NW>), dim3((unsigned)(blocks * grid.groups)), dim3(64 * NW), 0, st, o, (bf16_t*)out, lse, grid);
  return hipGetLastError();
}

}  // namespace

hipError_t packed_fwd_bf16(const PackedAttn& a, const PackedQkv<bf16_t>& o, void* out, float* lse, hipStream_t st) {
  return a.dh == 64 ? launch<64, 8>(a, o, out, lse, st) : launch<128, 4>(a, o, out, lse, st);
}

}  // namespace pf
