// Attention on packed sequences: what its kernels share (internal).
#pragma once

#include "packed.h"
#include "pf_device.h"
#include "pf_kernels.h"

namespace pf {

// Operands of a packed attention call.  Rows of all of them are tokens; head a of Q and out, K/V head a / group of K and V.
template <typename T>
struct PackedQkv {
  const T *q, *k, *v;
  int64_t ld_q, ld_k, ld_v, ld_out;   // elements between rows
  PackedRows rows;
  int32_t h, group, causal;
  float scale;
};

// Keys that query `row` sees: its sequence, up to itself if causal.  An empty span: the row is in no sequence.
__device__ __forceinline__ Span keys_of(const PackedRows& p, int r0, int row, int causal) {
  Span s = packed_span(p, r0, row);
  if (causal && s.lo < s.hi) s.hi = row + 1;
  return s;
}
// Queries that see key `row`
__device__ __forceinline__ Span queries_of(const PackedRows& p, int r0, int row, int causal) {
  Span s = packed_span(p, r0, row);
  if (causal && s.lo < s.hi) s.lo = row;
  return s;
}
// value of lane `lane`, as a scalar
__device__ __forceinline__ int lane_value(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// A lane's row sees rows lo .. hi - 1 of a tile of 64 (either may lie outside): all of the tile; a part of it, neither all nor nothing;
// and whether row i is not among them (one comparison; length: hi - lo).
// Without short circuits, which can cost a result: `uniform && (lane test || lane test) ? a : -m` becomes a branch per lane into a block that a
// wave-uniform branch enters too, and where the value that this block computes is free (a negation, an element of a vector), the compiler's
// structurizer (ROCm 7.2) moves it to the block above and drops it for the lanes that come from the lane test; they keep a.  (In the compiler's
// output right before that pass the value is there, right after it is not; a tile's keys were lost so.)  Masks with & and | are selects.
__device__ __forceinline__ bool seen_as_a_whole(int lo, int hi) { return (lo <= 0) & (hi >= 64); }
__device__ __forceinline__ bool seen_in_part(int lo, int hi) {
  const bool all = seen_as_a_whole(lo, hi), some = max(lo, 0) < min(hi, 64);
  return some & !all;
}
__device__ __forceinline__ bool hidden_at(int i, int lo, int length) { return (uint32_t)(i - lo) >= (uint32_t)max(length, 0); }

// sum over the wave, the same in all lanes
__device__ __forceinline__ int wave_total(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr 1, 2, 4, 8: lane 15 of each row has its sum
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  return lane_value(x, 15) + lane_value(x, 31) + lane_value(x, 47) + lane_value(x, 63);
}

// Which of `blocks` blocks of 2^log_rows rows the i-th workgroup takes: those that meet most rows first, so that none of them is
// the last to start.  n_s blocks begin in sequence s.  Causal, the j-th of them meets j blocks' rows (from_end: of keys that
// queries see, counted from the sequence's end), so block i is the one at depth X, the largest with sum over s of max(0, n_s - X) > i;
// not causal, all n_s of them meet n_s blocks' rows.  (Only where not all workgroups start at once: it takes a microsecond.)  For up to 64 sequences, one a lane; more (short ones, mostly) are taken from the end on.
__device__ __forceinline__ int block_in_order(const PackedRows& p, int i, int blocks, int log_rows, int causal, bool from_end, bool at_once) {
  const int plain = causal && from_end ? i : blocks - 1 - i;
  if (at_once || p.start == nullptr || p.n_seq < 2 || p.n_seq > 64) return plain;
  const int lane = threadIdx.x & 63, up = from_end ? 0 : (1 << log_rows) - 1;   // a block of two sequences: the one that it meets more rows of
  int b0 = 0, n = 0;
  if (lane < p.n_seq) {   // rows before the first sequence count as its own, rows behind the last as the last's
    b0 = lane == 0 ? 0 : (min(max(p.start[lane], 0), p.tokens) + up) >> log_rows;
    n = (lane == p.n_seq - 1 ? blocks : (min(max(p.start[lane + 1], 0), p.tokens) + up) >> log_rows) - b0;
  }
  auto ahead = [&](int x) { return wave_total(n > x ? causal ? n - x : n : 0); };
  if (ahead(0) != blocks) return plain;   // boundaries out of order
  int lo = 0, hi = blocks;                // ahead(lo) > i >= ahead(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (ahead(mid) > i) lo = mid;
    else hi = mid;
  }
  const int rest = i - ahead(hi);
  const bool at = causal ? n > lo : n == hi;   // sequences that have such blocks: one each, or hi each
  const int nth = causal ? rest : rest / hi, x = causal ? from_end ? n - 1 - lo : lo : rest % hi;
  const uint64_t m = __ballot(at), before = ((uint64_t)1 << lane) - 1;
  const uint64_t mine = __ballot(at && __popcll(m & before) == nth);
  if (mine == 0) return plain;
  return min(max(lane_value(b0 + x, __ffsll((unsigned long long)mine) - 1), 0), blocks - 1);
}

constexpr float LN2_P = 0.6931471805599453f;
constexpr float LOG2E_P = 1.4426950408889634f;

// ---- bf16 MFMA kernels ------------------------------------------------------------------------------------------------------
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef uint16_t v8u __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4s* lds_v4s_ptr;
typedef __attribute__((address_space(3))) void* lds_void_ptr;
typedef const __attribute__((address_space(3))) char* lds_char_ptr;

// Tiles of 64 rows x d_head lie in LDS row-major, the 16-byte chunks of a row swizzled (XOR on the chunk's number).  swz_row:
// for reads of one chunk per lane from 32 consecutive rows (the operand that contracts over d_head).  swz_col: for the
// transposing read, whose 16 lanes fetch 4 rows x 32 bytes (the operand that contracts over the rows).  Both depend on row % 16 only.
template <int DH>
__device__ __forceinline__ int swz_row(int r) { return DH == 64 ? ((r >> 1) & 7) : (r & 15); }
template <int DH>
__device__ __forceinline__ int swz_col(int r) { return DH == 64 ? (((r >> 1) & 1) << 1) : ((r & 3) << 1); }

// Byte offset of a lane's transposing reads in a tile under swz_col, columns from 32 dt, K step 0: lane 16 G + p points at row
// 4 g + p / 4 (g = lane / 32; the second read is 8 rows on) and the four columns from 32 dt + 16 (G % 2) + 4 (p % 4), and receives
// column 32 dt + lane % 32 of four rows.
template <int DH>
__device__ __forceinline__ int tr_offset(int lane, int dt) {
  const int p = lane & 15, row = 4 * (lane >> 5) + (p >> 2), c = dt * 4 + ((lane >> 4) & 1) * 2 + ((p & 3) >> 1);
  return row * DH * 2 + ((c ^ swz_col<DH>(row)) << 4) + 8 * (p & 1);
}
// the "A" operand of K step i (rows 16 i .. 16 i + 15) from offsets of its two reads
template <int ROWB>
__device__ __forceinline__ bf16x8 read_tr(lds_char_ptr tile, int off0, int off1, int i) {
  const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(tile + off0 + 16 * i * ROWB));
  const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(tile + off1 + (16 * i + 8) * ROWB));
  return __builtin_bit_cast(bf16x8, v8s{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
}

// N wave-wide copies of 1 KB from a raw buffer straight into LDS: lane i's 16 bytes at byte voff[n] of the buffer land at LDS byte
// address dst + n step + 16 i; bytes past the buffer's end arrive as zeros.  dst and step are wave-uniform.  M0 holds the LDS address
// and is put back (the compiler keeps it for itself).  Asynchronous, counted by vmcnt.
template <int N>
__device__ __forceinline__ void copy_rows(uint32_t dst, uint32_t step, lds_buffer_t buf, const uint32_t* voff) {
  static_assert(N == 1 || N == 2 || N == 4, "copies of one statement");
  uint32_t saved;
#define PF_COPY_NEXT(V) "s_add_u32 m0, m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %" #V ", %3, 0 offen lds\n\t"
#define PF_COPY_FIRST "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %3, 0 offen lds\n\t"
  if constexpr (N == 1)
    asm volatile(PF_COPY_FIRST "s_mov_b32 m0, %0" : "=&s"(saved) : "s"(dst), "s"(step), "s"(buf), "v"(voff[0]) : "memory", "scc");
  else if constexpr (N == 2)
    asm volatile(PF_COPY_FIRST PF_COPY_NEXT(5) "s_mov_b32 m0, %0" : "=&s"(saved) : "s"(dst), "s"(step), "s"(buf), "v"(voff[0]), "v"(voff[1]) : "memory", "scc");
  else
    asm volatile(PF_COPY_FIRST PF_COPY_NEXT(5) PF_COPY_NEXT(6) PF_COPY_NEXT(7) "s_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "s"(dst), "s"(step), "s"(buf), "v"(voff[0]), "v"(voff[1]), "v"(voff[2]), "v"(voff[3])
                 : "memory", "scc");
#undef PF_COPY_NEXT
#undef PF_COPY_FIRST
}

// Copies of a tile of 64 rows: of the NI = 64 d_head / 512 copies, those from `first` in steps of STEP.  One copy is 512 / d_head rows;
// which chunk of a row a lane fetches undoes the swizzle (swz, of the row's number in the tile).  base: of the operand's head; rows
// row0 .. row_end - 1 are read, the rest of the tile becomes zeros.  Strides are at most 2^24 elements, so a tile's offsets fit 32 bits.
template <int DH, int STEP, class Swz>
struct TileCopy {
  static constexpr int CPR = DH / 8, RPI = 512 / DH, NI = 64 / RPI, N = NI / STEP;
  static constexpr int PERIOD = STEP * RPI >= 16 ? 1 : 16 / (STEP * RPI);   // copies after which a lane's swizzle repeats
  uint32_t off[PERIOD];
  uint32_t ldb;
  __device__ __forceinline__ void init(int64_t ld, int first) {
    const int lane = threadIdx.x & 63;
    ldb = (uint32_t)ld * 2;
#pragma unroll
    for (int i = 0; i < PERIOD; ++i) {
      const int r = (first + i * STEP) * RPI + lane / CPR;
      off[i] = (uint32_t)r * ldb + (((lane % CPR) ^ Swz::of(r)) << 4);
    }
  }
  // dst: LDS address of the tile's copy `first`
  __device__ __forceinline__ void issue(const bf16_t* base, uint32_t dst, int row0, int row_end) const {
    const lds_buffer_t buf = lds_buffer((const char*)base + (int64_t)row0 * ldb, (uint32_t)min(row_end - row0, 64) * ldb);
    constexpr int AT = N < 4 ? N : 4;
#pragma unroll
    for (int i0 = 0; i0 < N; i0 += AT) {
      uint32_t v[AT];
#pragma unroll
      for (int i = 0; i < AT; ++i) v[i] = off[(i0 + i) % PERIOD] + (uint32_t)((i0 + i) / PERIOD * PERIOD * STEP * RPI) * ldb;
      copy_rows<AT>(__builtin_amdgcn_readfirstlane(dst + (uint32_t)(i0 * STEP * 1024)), STEP * 1024, buf, v);
    }
  }
};
template <int DH>
struct SwzRow {
  static __device__ __forceinline__ int of(int r) { return swz_row<DH>(r); }
};
template <int DH>
struct SwzCol {
  static __device__ __forceinline__ int of(int r) { return swz_col<DH>(r); }
};

// the values of lanes l % 32 and l % 32 + 32, without LDS.  (Through an empty asm statement: a maximum of the two would
// otherwise be folded into the first.)
__device__ __forceinline__ void both_halves(float x, float& lo, float& hi) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  unsigned a = r[0], b = r[1];
  asm volatile("" : "+v"(a), "+v"(b));
  lo = __builtin_bit_cast(float, a);
  hi = __builtin_bit_cast(float, b);
}

// rows 16 i .. 16 i + 15 of a product's column as a "B" operand: slot (g, t) is row 16 i + 8 (t / 4) + 4 g + t % 4, which is register
// 8 (i % 2) + t of the product's 32-row half i / 2
__device__ __forceinline__ bf16x8 as_operand(const f32x16& half, int i) {
  bf16x8 f;
#pragma unroll
  for (int t = 0; t < 8; ++t) f[t] = (__bf16)half[8 * (i & 1) + t];
  return f;
}

// acc[dt] += X^T W for a tile that not every row sees as a whole, with care: 0 (hidden) times an infinity or NaN of X would be
// NaN, so those go into the product as 0 and are counted apart, over visible rows only: a row of X that is +inf, -inf or NaN
// counts 1, 2^7 or 2^14 (at most 64 rows: exact in fp32), and 2^14 times that where its weight is 0, which makes an infinity NaN as in
// a tile that is seen as a whole.  A weight below 0 meets no infinity: weights of dS have that sign alone, and an infinite element of K or
// Q makes its row's scores infinite or NaN, so P is 0 or NaN there.  NaN weights make NaN of the zeros.
// w: the "B" operands of the 64 rows' weights, visible rows lo .. hi - 1 (of the tile); off(dt, r): byte offsets of the two transposing reads.
template <int DH, class Off>
__device__ __forceinline__ void add_with_care(f32x16* acc, const bf16x8* w, lds_char_ptr tile, Off off, int lo, int hi) {
  const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt) {
    f32x16 odd;
#pragma unroll
    for (int r = 0; r < 16; ++r) odd[r] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __builtin_amdgcn_sched_barrier(0);   // one step's registers at a time
      const v8s x = __builtin_bit_cast(v8s, read_tr<DH * 2>(tile, off(dt, 0), off(dt, 1), i));
      v8s clean, mark;
      const v8u weight = __builtin_bit_cast(v8u, w[i]) & (uint16_t)0x7fff;
      v8u seen = (uint16_t)0x4680 - __builtin_elementwise_min(weight, v8u(1)) * (uint16_t)0x0700;   // weight 0: 2^14, else 1
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const bool is_odd = (x[t] & 0x7f80) == 0x7f80;
        clean[t] = is_odd ? (short)0 : x[t];
        mark[t] = !is_odd ? (short)0 : (x[t] & 0x7f) ? (short)0x4680 : x[t] < 0 ? (short)0x4300 : (short)0x3f80;   // 2^14, 2^7, 1
        if (hidden_at(16 * i + 8 * (t >> 2) + (t & 3), lo - 4 * g, hi - lo)) seen[t] = 0;
      }
      acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, clean), w[i], acc[dt], 0, 0, 0);
      odd = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, mark), __builtin_bit_cast(bf16x8, seen), odd, 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int n = (int)fminf(odd[r], 16384.f);
      const bool plus = (n & 0x7f) != 0, minus = (n & 0x3f80) != 0, nan = (n >> 14 != 0) | (plus & minus);
      acc[dt][r] += nan ? NAN : plus ? INFINITY : minus ? -INFINITY : 0.f;
    }
  }
}

// Lets `kernel` have `bytes` of dynamic LDS on the current device
hipError_t allow_lds(const void* kernel, int bytes);

// Heads of a group that a workgroup of four waves takes: a power of two
inline int heads_together(const PackedAttn& a) {
  int heads = 1;
  while (heads < 4 && (a.h / a.h_kv) % (heads * 2) == 0) heads *= 2;
  return heads;
}

// How a bf16 call (d_head 64 / 128) is run, by its sizes alone: K/V tiles shared by the waves of a workgroup, a block's keys in one part or
// two (d_head 128), or independent waves with 1, 2 or 4 to a block's keys; heads of a workgroup (shared tiles); whether all workgroups start at
// the same time, so that blocks need no order.
enum FwdForm : int32_t { SHARED_1, SHARED_2, WAVES_1, WAVES_2, WAVES_4 };
struct FwdPlan {
  FwdForm form;
  int32_t heads, at_once;
};
FwdPlan packed_fwd_plan(const PackedAttn& a);
struct BwdPlan {
  int32_t splits, dkv_at_once, dq_at_once;   // splits: parts of a block's tiles in dK/dV
};
BwdPlan packed_bwd_plan(const PackedAttn& a);

// bf16, d_head 64 / 128, all pointers 16-byte aligned, strides in eights
hipError_t packed_fwd_bf16(const PackedAttn& a, const PackedQkv<bf16_t>& o, void* out, float* lse, hipStream_t st);
hipError_t packed_bwd_bf16(const PackedAttn& a, const PackedQkv<bf16_t>& o, const void* dout, const float* lse, const float* dsum, void* dq, void* dk,
                           void* dv, void* workspace, hipStream_t st);
int64_t packed_bwd_bf16_bytes(const PackedAttn& a);   // of workspace
// fp32 sums of dK and dV of several splits, [split][dK, dV][tokens][K/V heads * d_head]: their size, and what makes dk and dv of them
int64_t packed_partial_bytes(const PackedAttn& a, int splits);
hipError_t packed_join(const PackedAttn& a, const float* partial, int splits, void* dk, void* dv, hipStream_t st);

}  // namespace pf
