// Embedding on packed sequences for gfx950, and its gradients by sorted tokens.
//
// Forward: x[t] = scale tok[ids[t]] + pos[t - start(t)], one rounding.  Bound by HBM: a wave takes two rows, 16 bytes a lane, with
// all their loads in flight at once (14500 rows of 2048, bf16: 20.7 us with all columns to a wave, 4.1 TB/s; one row a wave 21.5, four
// 24.2, eight 28.0; fp32 47).  Few rows cannot hide the four loads one after the other (sequence, id, table, store) behind each other, so each
// wave takes one slice of 512 columns then (266 rows of 1816: 8.2 us, 12.0 with all columns).
//
// Backward: dtok[v] = scale sum over rows t with ids[t] = v of dx[t], dpos[p] = sum over rows at position p of dx[t], fp32, in
// three launches and the same every time:
//   1. embed_group_kernel groups the rows by token and by position (ascending rows within a group).  Workgroup j of the tokens
//      owns ids = j modulo their number (neighbouring ids are about as frequent as each other: this deals them out) and reads all
//      ids itself, counts those of lower workgroups for its place in the order, and orders its own with a counter per wave and id:
//      no communication between workgroups.
//      Positions need no search: the rows before position p's are sum over sequences of min(length, p).
//      Other workgroups clear the last rows of a large token table meanwhile.
//   2. embed_sum_kernel adds up the grouped rows, a fixed number of them per wave however they are spread over the groups.  A
//      group inside a wave's share goes to its gradient row at once, the sums of groups that go beyond to the workspace.
//      Other waves clear the rest of the rows that no row of dx belongs to.
//   3. embed_join_kernel adds those partial sums up in order.
// Large tables are bound by writing the gradient (7250 rows of 1024, bf16, into 50257 rows: 55 us, 42 with nothing else in between, for 206 MB of it
// and 15 MB of dx read twice; added to what is there, without clearing, 30), small ones by the three launches after each other (553 rows of 512,
// fp32, into 10007: 5.6 + 7.0 + 3.9).
#include "packed.h"
#include "pf_device.h"
#include "pf_kernels.h"

#include <algorithm>

namespace pf {
namespace {

constexpr int ROWS = 2;

template <typename T>
__global__ __launch_bounds__(256) void embed_packed_kernel(const int32_t* __restrict__ ids, const T* __restrict__ tok,
                                                           const T* __restrict__ pos, PackedRows p, float scale, T* __restrict__ x,
                                                           int32_t S, int32_t d, int32_t V, int32_t parts) {
  typedef typename Raw8<T>::type raw_t;
  const int lane = threadIdx.x & 63;
  const int item = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const int r0 = item / parts * ROWS, part = item % parts;   // one of `parts` waves with these rows
  if (r0 >= p.tokens) return;
  const int row = r0 + (lane & (ROWS - 1));
  const int id = row < p.tokens ? ids[row] : -1;
  const Span s = packed_span(p, r0, row);
  const int place = s.lo < s.hi ? row - s.lo : -1;
  int idv[ROWS], plv[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    idv[i] = __builtin_amdgcn_readlane(id, i);
    plv[i] = __builtin_amdgcn_readlane(place, i);
  }
  for (uint32_t c = (uint32_t)part * 512 + lane * 8; c < (uint32_t)d; c += (uint32_t)parts * 512) {   // unsigned: c passes d
    raw_t t8[ROWS], p8[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {   // a row that is not there is read as row 0 and not used
      const bool in_t = (uint32_t)idv[i] < (uint32_t)V, in_p = (uint32_t)plv[i] < (uint32_t)S;
      t8[i] = *(const raw_t*)(tok + (int64_t)(in_t ? idv[i] : 0) * d + c);
      if (pos) p8[i] = *(const raw_t*)(pos + (int64_t)(in_p ? plv[i] : 0) * d + c);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      if (plv[i] < 0) continue;
      const bool in_t = (uint32_t)idv[i] < (uint32_t)V, in_p = pos && plv[i] < S;
      float a[8], b[8];
      unpack8(t8[i], a);
      if (pos) unpack8(p8[i], b);
#pragma unroll
      for (int j = 0; j < 8; ++j) a[j] = in_t ? in_p ? fmaf(scale, a[j], b[j]) : scale * a[j] : in_p ? b[j] : 0.f;
      store8(x + (int64_t)(r0 + i) * d + c, a);
    }
  }
}

// ---- backward --------------------------------------------------------------------------------------------------------------
// Rows of dx grouped by a key (token or position): entry e of the order is row[e] with key[e]; key k has entries
// first[k] .. first[k] + count[k] - 1.  *total: entries.
struct Grouped {
  int32_t *row, *key, *first, *count, *total;
  int32_t n_keys;
  float* grad;      // [n_keys][d]
  float* partial;   // [shares][2][d]: a share's sum of the group that began before it, and of the one that goes on behind it
  float scale;
};

constexpr int GROUP_THREADS = 1024, GROUP_WAVES = 16, GROUP_IDS = 1000;   // ids a workgroup can own (LDS: 64 bytes each, 64 KiB in all)

__global__ __launch_bounds__(GROUP_THREADS) void embed_group_kernel(const int32_t* __restrict__ ids, PackedRows p, Grouped by_id, Grouped by_pos,
                                                                    int32_t log_wgs, int32_t own, int32_t pos_wgs, int32_t d, int32_t id_cleared) {
  extern __shared__ int32_t dyn_cnt[];   // [wave][own]
  __shared__ int32_t s_below[GROUP_WAVES], s_sum[GROUP_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint64_t before = ((uint64_t)1 << lane) - 1;   // lanes below this one
  const int T = p.tokens, wgs = 1 << log_wgs;
  if ((int)blockIdx.x >= wgs + pos_wgs) {   // the table's last rows: zeros, whether a row of dx belongs to them or not
    const int64_t n = (int64_t)(by_id.n_keys - id_cleared) * d, all = (int64_t)(gridDim.x - wgs - pos_wgs) * GROUP_THREADS;
    float* to = by_id.grad + (int64_t)id_cleared * d;
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t i = (int64_t)((int)blockIdx.x - wgs - pos_wgs) * GROUP_THREADS + tid; i < n / 4; i += all) store4(to + i * 4, zero);
    return;
  }
  if ((int)blockIdx.x >= wgs) {   // positions: one per wave
    const int at = ((int)blockIdx.x - wgs) * GROUP_WAVES + wave;
    if (at >= by_pos.n_keys) return;
    const int n = p.start ? p.n_seq : 1;
    auto length = [&](int s, int& begin) {
      if (s >= n) return 0;
      if (!p.start) {
        begin = 0;
        return T;
      }
      begin = min(max(p.start[s], 0), T);
      return max(min(max(p.start[s + 1], 0), T) - begin, 0);
    };
    int rows_before = 0, begin = 0;   // at most T, unless sequences overlap: counted no further, so that no sum passes 32 bits
    for (int s = lane; s < n; s += 64) rows_before = min(rows_before + min(length(s, begin), at), T);
    for (int o = 32; o > 0; o >>= 1) rows_before = min(rows_before + __shfl_xor(rows_before, o, 64), T);
    int e = rows_before;
    for (int s0 = 0; s0 < n; s0 += 64) {
      const bool has = length(s0 + lane, begin) > at;
      const uint64_t m = __ballot(has);
      const int to = e + __popcll(m & before);
      if (has && (uint32_t)to < (uint32_t)T) {   // (sequences that overlap could be longer together than the buffer)
        by_pos.row[to] = begin + at;
        by_pos.key[to] = at;
      }
      e = min(e + __popcll(m), T);
    }
    if (lane == 0) {
      by_pos.first[at] = rows_before;
      by_pos.count[at] = e - rows_before;
      if (at == by_pos.n_keys - 1) *by_pos.total = e;
    }
    return;
  }
  const int j = blockIdx.x;
  for (int i = tid; i < GROUP_WAVES * own; i += GROUP_THREADS) dyn_cnt[i] = 0;
  const int lo = p.start ? min(max(p.start[0], 0), T) : 0, hi = p.start ? min(max(p.start[p.n_seq], 0), T) : T;
  const int chunk = ((T + GROUP_WAVES - 1) / GROUP_WAVES + 63) & ~63;
  const int t0 = wave * chunk, t1 = min(T, t0 + chunk);
  volatile int32_t* cnt = dyn_cnt + wave * own;
  auto id_of = [&](int t) { return t < t1 && t >= lo && t < hi ? ids[t] : -1; };
  __syncthreads();
  int below = 0;
  for (int t = t0; t < t1; t += 256) {
    int id[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) id[u] = id_of(t + u * 64 + lane);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool ok = (uint32_t)id[u] < (uint32_t)by_id.n_keys;
      const int b = id[u] & (wgs - 1);
      below += ok && b < j;
      if (ok && b == j) atomicAdd(&dyn_cnt[wave * own + (id[u] >> log_wgs)], 1);
    }
  }
  for (int o = 32; o > 0; o >>= 1) below += __shfl_xor(below, o, 64);
  if (lane == 0) s_below[wave] = below;
  __syncthreads();
  // counts -> first entries: thread i has id i of the workgroup's
  int mine = 0;
  if (tid < own)
    for (int w = 0; w < GROUP_WAVES; ++w) mine += dyn_cnt[w * own + tid];
  int upto = mine;   // inclusive sum over the wave's ids
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o, 64);
    if (lane >= o) upto += v;
  }
  if (lane == 63) s_sum[wave] = upto;
  __syncthreads();
  int base = 0, all = 0;
  for (int w = 0; w < GROUP_WAVES; ++w) {
    base += s_below[w] + (w < wave ? s_sum[w] : 0);
    all += s_below[w] + s_sum[w];
  }
  if (tid < own) {
    int at = base + upto - mine;
    const int64_t id = ((int64_t)tid << log_wgs) + j;
    if (id < by_id.n_keys) {
      by_id.first[id] = at;
      by_id.count[id] = mine;
    }
    for (int w = 0; w < GROUP_WAVES; ++w) {
      const int v = dyn_cnt[w * own + tid];
      dyn_cnt[w * own + tid] = at;
      at += v;
    }
  }
  if (tid == 0 && j == wgs - 1) *by_id.total = all;
  __syncthreads();
  for (int t = t0; t < t1; t += 256) {
    int id[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) id[u] = id_of(t + u * 64 + lane);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool ok = (uint32_t)id[u] < (uint32_t)by_id.n_keys && (id[u] & (wgs - 1)) == j;
      uint64_t left = __ballot(ok);
      while (left) {   // one id of the workgroup's after the other; within the wave LDS instructions execute in order
        const int leader = __ffsll((unsigned long long)left) - 1;
        const int k = __builtin_amdgcn_readlane(id[u], leader);
        const uint64_t same = __ballot(ok && id[u] == k);
        const int at = cnt[k >> log_wgs];
        if (ok && id[u] == k) {
          const int e = at + __popcll(same & before);
          by_id.row[e] = t + u * 64 + lane;
          by_id.key[e] = k;
        }
        if (lane == leader) cnt[k >> log_wgs] = at + __popcll(same);
        left &= ~same;
      }
    }
  }
}

// What a wave of the second launch does: shares of the tokens' order, shares of the positions', then runs of rows to clear
struct SumPlan {
  int32_t share;                    // entries per wave, at most 64
  int32_t slices;                   // of 512 columns
  int64_t id_end, pos_end, id_zero_end, pos_zero_end;
  int32_t id_cleared;               // token rows from here on are zeros already
};
constexpr int ZERO_RUN = 16;

template <typename T>
__global__ __launch_bounds__(256) void embed_sum_kernel(const T* __restrict__ dx, Grouped by_id, Grouped by_pos, SumPlan plan, int32_t tokens,
                                                        int32_t d, int32_t accumulate) {
  typedef typename Raw8<T>::type raw_t;
  const int lane = threadIdx.x & 63;
  int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (item >= plan.pos_zero_end) return;
  const bool tokens_ = item < plan.id_end || (item >= plan.pos_end && item < plan.id_zero_end);
  const Grouped& G = tokens_ ? by_id : by_pos;
  if (item >= plan.pos_end) {
    item -= item < plan.id_zero_end ? plan.pos_end : plan.id_zero_end;
    const int64_t k0 = item * ZERO_RUN;
    const bool none = lane < ZERO_RUN && k0 + lane < (tokens_ ? plan.id_cleared : G.n_keys) && G.count[k0 + lane] == 0;
    uint64_t left = __ballot(none);
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    while (left) {
      const int i = __ffsll((unsigned long long)left) - 1;
      left &= left - 1;
      float* to = G.grad + (k0 + i) * d;
      for (uint32_t c = lane * 4; c < (uint32_t)d; c += 256) store4(to + c, zero);
    }
    return;
  }
  if (item >= plan.id_end) item -= plan.id_end;
  const int64_t share = item / plan.slices;
  const int c = (int)(item % plan.slices) * 512 + lane * 8;
  const bool in = c < d;
  const int total = *G.total;
  const int64_t e0 = share * plan.share;
  if (e0 >= total) return;
  const int n = (int)min((int64_t)plan.share, total - e0);
  int row = 0, key = -1;
  if (lane < n) {
    row = G.row[e0 + lane];
    key = G.key[e0 + lane];
    if ((uint32_t)row >= (uint32_t)tokens || (uint32_t)key >= (uint32_t)G.n_keys) key = -1;
  }
  const int key_before = e0 > 0 ? G.key[e0 - 1] : -1;
  const int key_behind = e0 + n < total ? G.key[e0 + n] : -1;
  const T* col = dx + (in ? c : 0);
  float acc[8] = {};
  bool head = true;   // no group has ended yet
  for (int i0 = 0; i0 < n; i0 += 8) {
    raw_t x8[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + u < n ? i0 + u : n - 1;
      const int k = __builtin_amdgcn_readlane(key, i);
      x8[u] = *(const raw_t*)(col + (int64_t)(k < 0 ? 0 : __builtin_amdgcn_readlane(row, i)) * d);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + u;
      if (i >= n) break;
      const int k = __builtin_amdgcn_readlane(key, i), k_next = i + 1 < n ? __builtin_amdgcn_readlane(key, i + 1) : key_behind;
      float v[8];
      unpack8(x8[u], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += v[e];
      if (k_next == k && i + 1 < n) continue;
      if (k >= 0 && in) {
        float* to;
        if (head && k == key_before) to = G.partial + (share * 2) * d + c;
        else if (k_next == k) to = G.partial + (share * 2 + 1) * d + c;
        else {
          to = G.grad + (int64_t)k * d + c;
          float old[8] = {};
          if (accumulate) load8(to, old);
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = fmaf(acc[e], G.scale, old[e]);
        }
        store8(to, acc);
      }
      head = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    }
  }
}

// A workgroup per share and slice: if a group begins in the share and goes on behind it, its waves add up the group's sums of
// the shares that follow, a contiguous part each
__global__ __launch_bounds__(256) void embed_join_kernel(Grouped by_id, Grouped by_pos, SumPlan plan, int32_t d, int32_t accumulate) {
  __shared__ __align__(16) float s_sum[4][512];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool tokens_ = (int64_t)blockIdx.x < plan.id_end;
  const Grouped& G = tokens_ ? by_id : by_pos;
  const int64_t item = tokens_ ? blockIdx.x : blockIdx.x - plan.id_end;
  const int64_t share = item / plan.slices, e0 = share * plan.share;
  const int total = *G.total;
  if (e0 + plan.share >= total) return;
  const int k = G.key[e0 + plan.share - 1];
  if ((uint32_t)k >= (uint32_t)G.n_keys || G.key[e0 + plan.share] != k || G.first[k] < e0) return;
  const int last_e = min(G.first[k] + G.count[k], total) - 1;
  const int n = (int)(last_e / plan.share - share);   // shares that follow
  const int c = (int)(item % plan.slices) * 512 + lane * 8;
  const bool in = c < d;
  const float* part = G.partial + share * 2 * d + (in ? c : 0);
  float acc[8] = {};
  if (wave == 0) load8(part + d, acc);
  const int from = 1 + (int)((int64_t)n * wave / 4), to = 1 + (int)((int64_t)n * (wave + 1) / 4);
  for (int i0 = from; i0 < to; i0 += 4) {
    float v[4][8];
#pragma unroll
    for (int u = 0; u < 4; ++u) load8(part + (int64_t)min(i0 + u, to - 1) * 2 * d, v[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u < to)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += v[u][e];
  }
  store8(&s_sum[wave][lane * 8], acc);
  __syncthreads();
  if (wave != 0 || !in) return;
  for (int w = 1; w < 4; ++w)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += s_sum[w][lane * 8 + e];
  float* dst = G.grad + (int64_t)k * d + c;
  float old[8] = {};
  if (accumulate) load8(dst, old);
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = fmaf(acc[e], G.scale, old[e]);
  store8(dst, acc);
}

// Where everything lies in the workspace, and how the work is divided: functions of the sizes alone
struct BwdLayout {
  int32_t log_wgs, own, share, slices;
  int64_t shares;
  int64_t id_row, id_key, id_first, id_count, pos_row, pos_key, pos_first, pos_count, totals, id_partial, pos_partial, bytes;
};
BwdLayout bwd_layout(int64_t tokens, int64_t S, int64_t d, int64_t V) {
  BwdLayout L{};
  L.log_wgs = 8;
  while ((((int64_t)GROUP_IDS) << L.log_wgs) < V) ++L.log_wgs;
  L.own = (int32_t)((V + ((int64_t)1 << L.log_wgs) - 1) >> L.log_wgs);
  L.slices = (int32_t)((d + 511) / 512);
  // Entries per wave.  Eight are loaded at a time, so few waves are done earlier with eight each, many carry fewer partial sums and read
  // less about their groups with 16 (553 rows of 512, fp32: 18.6 us with 16, 16.8 with 8; 4000 of 680: 18.9, 17.8; 7250 of 1024:
  // 45.4, 48.4; 12400 of 400: 27.5, 28.7).  Positions have as many waves as tokens.
  L.share = (tokens + 15) / 16 * L.slices * 2 < 1280 ? 8 : 16;
  L.shares = (tokens + L.share - 1) / L.share;
  int64_t at = 0;
  auto take = [&](int64_t n) {
    const int64_t here = at;
    at += (n * 4 + 255) / 256 * 256;
    return here;
  };
  L.id_row = take(tokens);
  L.id_key = take(tokens);
  L.pos_row = take(tokens);
  L.pos_key = take(tokens);
  L.id_first = take(V);
  L.id_count = take(V);
  L.pos_first = take(S);
  L.pos_count = take(S);
  L.totals = take(2);
  L.id_partial = take(L.shares * 2 * d);
  L.pos_partial = take(L.shares * 2 * d);
  L.bytes = at;
  return L;
}

}  // namespace

hipError_t embed_packed_fwd(int32_t dtype, const int32_t* ids, const void* tok, const void* pos, const int32_t* seq_start, int32_t n_seq, float scale,
                            void* x, int64_t tokens, int32_t S, int32_t d, int32_t V, hipStream_t stream) {
  const PackedRows p{seq_start, n_seq, (int32_t)tokens};
  const int64_t pairs = (tokens + ROWS - 1) / ROWS;
  const int parts = pairs < 2048 ? (int)(((int64_t)d + 511) / 512) : 1;   // 2048 waves: two a SIMD
  const dim3 grid((unsigned)((pairs * parts + 3) / 4)), block(256);
  if (dtype == PF_DTYPE_BF16_)
    hipLaunchKernelGGL(embed_packed_kernel<bf16_t>, grid, block, 0, stream, ids, (const bf16_t*)tok, (const bf16_t*)pos, p, scale, (bf16_t*)x, S, d, V, parts);
  else
    hipLaunchKernelGGL(embed_packed_kernel<float>, grid, block, 0, stream, ids, (const float*)tok, (const float*)pos, p, scale, (float*)x, S, d, V, parts);
  return hipGetLastError();
}

int64_t embed_packed_bwd_bytes(int64_t tokens, int32_t S, int32_t d, int32_t V) { return bwd_layout(tokens, S, d, V).bytes; }

hipError_t embed_packed_bwd(int32_t dtype, const void* dx, const int32_t* ids, const int32_t* seq_start, int32_t n_seq, float scale, float* dtok,
                            float* dpos, int32_t accumulate, void* workspace, int64_t tokens, int32_t S, int32_t d, int32_t V, hipStream_t stream) {
  const BwdLayout L = bwd_layout(tokens, S, d, V);
  const PackedRows p{seq_start, n_seq, (int32_t)tokens};
  char* w = (char*)workspace;
  auto ints = [&](int64_t at) { return (int32_t*)(w + at); };
  Grouped by_id{ints(L.id_row), ints(L.id_key), ints(L.id_first), ints(L.id_count), ints(L.totals), V, dtok, (float*)(w + L.id_partial), scale};
  Grouped by_pos{ints(L.pos_row), ints(L.pos_key), ints(L.pos_first), ints(L.pos_count), ints(L.totals) + 1, dpos ? S : 0, dpos, (float*)(w + L.pos_partial), 1.0f};
  const int wgs = 1 << L.log_wgs, pos_wgs = dpos ? (S + GROUP_WAVES - 1) / GROUP_WAVES : 0;
  // Grouping leaves the memory idle: of a large table it clears the rows of the second half (rare tokens, where ids go by frequency) beside
  // it, the few of them that have a gradient are written twice.  (50257 rows of 1024: 46.0 us without, 45.2 / 43.8 / 42.2 / 41.7 / 43.8
  // with the last 16 / 32 / 64 / 96 / 128 MB; tables of 20 MB and less: no difference.)
  const int clear_rows = !accumulate && (int64_t)V * d * 4 >= (64 << 20) ? V / 2 : 0;
  const int id_cleared = V - clear_rows;
  const int clear_wgs = clear_rows > 0 ? (int)std::min<int64_t>(512, ((int64_t)clear_rows * d / 4 + GROUP_THREADS - 1) / GROUP_THREADS) : 0;
  hipLaunchKernelGGL(embed_group_kernel, dim3((unsigned)(wgs + pos_wgs + clear_wgs)), dim3(GROUP_THREADS), (size_t)GROUP_WAVES * L.own * 4, stream, ids, p, by_id, by_pos,
                     L.log_wgs, L.own, pos_wgs, d, id_cleared);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  SumPlan plan{L.share, L.slices, 0, 0, 0, 0, id_cleared};
  plan.id_end = L.shares * L.slices;
  plan.pos_end = plan.id_end + (dpos ? L.shares * L.slices : 0);
  plan.id_zero_end = plan.pos_end + (accumulate ? 0 : ((int64_t)id_cleared + ZERO_RUN - 1) / ZERO_RUN);
  plan.pos_zero_end = plan.id_zero_end + (accumulate || !dpos ? 0 : ((int64_t)S + ZERO_RUN - 1) / ZERO_RUN);
  const dim3 sum_grid((unsigned)((plan.pos_zero_end + 3) / 4)), block(256);
  if (dtype == PF_DTYPE_BF16_) hipLaunchKernelGGL(embed_sum_kernel<bf16_t>, sum_grid, block, 0, stream, (const bf16_t*)dx, by_id, by_pos, plan, (int32_t)tokens, d, accumulate);
  else hipLaunchKernelGGL(embed_sum_kernel<float>, sum_grid, block, 0, stream, (const float*)dx, by_id, by_pos, plan, (int32_t)tokens, d, accumulate);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)plan.pos_end), block, 0, stream, by_id, by_pos, plan, d, accumulate);
  return hipGetLastError();
}

}  // namespace pf
