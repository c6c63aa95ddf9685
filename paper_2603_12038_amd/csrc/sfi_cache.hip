// What writes the rows of a cache and what drops them: rotary positions with the append of new rows, and the move of the
// kept rows behind an eviction.
#include "sfi_internal.h"

namespace sfi {

// ---- rotary positions and append ------------------------------------------------------------------------------
// Pair i of a head is turned by the angle pos * f_i.  The table holds f_i / 2 pi as a fraction of 2^64 of a turn, so
// pos * entry mod 2^64 is the angle mod one turn, exact in integers up to the entry's own rounding (pos * 2^-53 turns: 1e-10 at a
// million), where the product in fp32 would be off by pos * 2^-24 radians.  The fraction of a turn goes on as 24 bits of fp32 (2^-25 of half a turn, 1e-7 radians at
// most), and sine, cosine and products are in fp32: 2^-21 of the terms, hidden behind the one rounding to bf16 (up to 2^-8).
//
// A wave has one new row at a time (a token): lane i computes the sine and cosine of pair i once, through LDS they go to the lanes
// that need them, and the row's heads (query, key, value) follow four at a time, 16 lanes of 16 bytes to a head.
// Bound by the rows read and written: a prompt of 8192 rows of 48 heads, 201 MB in 36.5 us; 16 prompts of 700 to 2011 rows of 56 heads into a paged
// cache, 622 MB in 130 us, 4.8 TB/s (a large copy reaches 5.1); four rows 4.0 us, a launch and three round trips.
__global__ void rope_table_kernel(const RopeTable t, uint64_t* table) {
  if (threadIdx.x < kHeadDim / 2) table[threadIdx.x] = t.turn[threadIdx.x];
}
hipError_t launch_rope_table(const RopeTable& t, uint64_t* table, hipStream_t s) {
  hipLaunchKernelGGL(rope_table_kernel, dim3(1), dim3(64), 0, s, t, table);
  return hipGetLastError();
}

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / 64;
constexpr int kRopeAhead = 4;

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// fp32 -> bf16, nearest even; what is no number stays none
__device__ __forceinline__ uint32_t bf16_any(float v) {
  return v != v ? 0x7fc0u | (__float_as_uint(v) >> 31 << 15) : bf16_rne(v);
}

// AHEAD groups of four heads of a new row (heads behind the last one repeat it), `there` or not.
struct NewRow {
  const uint16_t *q, *k, *v;
  int Hq, Hkv;
};
template <int AHEAD>
__device__ __forceinline__ void request_heads(u32x4 (&x)[AHEAD], const NewRow w, int h0, int step, int sub, int c, bool there) {
#pragma unroll
  for (int r = 0; r < AHEAD; ++r) {
    const int h = min(h0 + r * step + sub, w.Hq + 2 * w.Hkv - 1);
    const bool is_q = h < w.Hq, is_k = !is_q && h < w.Hq + w.Hkv;
    const int hk = is_q ? h : is_k ? h - w.Hq : h - w.Hq - w.Hkv;
    x[r] = u32x4{0u, 0u, 0u, 0u};
    if (there) x[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>((is_q ? w.q : is_k ? w.k : w.v) + hk * kHeadDim + 8 * c));
  }
}

// AHEAD: groups of four heads a wave requests together; one where it has no more than a few.  Then the first
// are on their way while sines are made (four rows 4.25 -> 4.0 us; with four groups a prompt of 8192 rows 36.7 -> 38.5).
template <int AHEAD>
__global__ __launch_bounds__(kRopeThreads) void rope_append_kernel(const RopeArgs a) {
  __shared__ float2 s_cs[kRopeWaves][kHeadDim / 2];  // cosine, sine
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t token = (int64_t)blockIdx.x * kRopeWaves + wave;
  const int64_t n_tokens = (int64_t)a.B * a.max_new;
  const int b = (int)((token < n_tokens ? token : n_tokens - 1) / a.max_new), t = (int)((token < n_tokens ? token : n_tokens - 1) % a.max_new);
  const int c = lane & 15, sub = lane >> 4;  // elements 8 c .. 8 c + 7 of head sub of each four
  const NewRow in = {a.q + (int64_t)b * a.q_in_b + (int64_t)t * a.q_in_t, a.k + (int64_t)b * a.k_in_b + (int64_t)t * a.k_in_t,
                     a.v + (int64_t)b * a.v_in_b + (int64_t)t * a.v_in_t, a.Hq, a.Hkv};
  const int heads = a.Hq + 2 * a.Hkv, step = 4 * (int)gridDim.y;
  int bad = 0;
  const int L0 = a.ctx_len[b];
  const int L = min(max(L0, 0), a.len_cap);
  bad |= L != L0 ? kGuardCtxLen : 0;
  int n = a.max_new;
  if (a.n_new != nullptr) {
    const int n0 = a.n_new[b];
    n = min(max(n0, 0), a.max_new);
    bad |= n != n0 ? kGuardNNew : 0;
  }
  if (n > L) {
    bad |= a.n_new != nullptr || L > 0 ? kGuardNNew : 0;  // (max_new for every sequence: none for an unused slot)
    n = L;
  }
  const int row = L - n + t;
  const bool live = token < n_tokens && t < n;
  u32x4 x[AHEAD];
  if (AHEAD == 1) request_heads<AHEAD>(x, in, 4 * (int)blockIdx.y, step, sub, c, live);
  const int64_t pos = a.pos != nullptr ? (int64_t)a.pos[b] + t : (int64_t)row;
  const int half = a.rot / 2;
  {
    float sn = 0.f, cs = 1.f;
    if (lane < half) {
      const uint64_t phase = (uint64_t)pos * a.table[lane];
      sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &sn, &cs);
    }
    s_cs[wave][lane] = make_float2(cs * a.magnitude, sn * a.magnitude);
  }
  __syncthreads();
  // Half layout: element e < half goes with e + half; the partner's chunk is half / 8 lanes away.  Interleaved: 2 i with 2 i + 1.
  const bool turned = 8 * c < a.rot, upper = !a.interleaved && 8 * c >= half;
  const int partner = upper ? lane - half / 8 : lane + half / 8;
  float cs[8], sn[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int i = a.interleaved ? 4 * c + j / 2 : 8 * c + j - (upper ? half : 0);
    const float2 v = s_cs[wave][turned ? i : 0];
    cs[j] = v.x;
    sn[j] = v.y;
  }
  int64_t k_row, v_row;  // element offsets of the cache row
  bool in_pool = true;
  if (a.block_table != nullptr) {
    const int page0 = live ? a.block_table[(int64_t)b * a.table_stride + (row >> a.page_lg)] : 0;
    in_pool = page0 >= 0 && page0 < a.n_blocks;
    bad |= in_pool ? 0 : kGuardBlock;
    const int64_t r = (int64_t)page0 * a.page_rpb + (row & ((1 << a.page_lg) - 1));
    k_row = r * a.k_st;
    v_row = r * a.v_st;
  } else {
    k_row = (int64_t)b * a.k_sb + (int64_t)row * a.k_st;
    v_row = (int64_t)b * a.v_sb + (int64_t)row * a.v_st;
  }
  uint16_t* q_out = a.q_out + ((int64_t)b * a.max_new + t) * a.Hq * kHeadDim;
  for (int h0 = 4 * (int)blockIdx.y; h0 < heads; h0 += AHEAD * step) {
    if (AHEAD > 1 || h0 != 4 * (int)blockIdx.y) request_heads<AHEAD>(x, in, h0, step, sub, c, live);
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) {
      const int h = h0 + r * step + sub;
      const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
      const int hk = is_q ? h : is_k ? h - a.Hq : h - a.Hq - a.Hkv;
      const u32x4 w = x[r];
      u32x4 o = w;
      if (a.interleaved) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = lo_f(w[j]), s = hi_f(w[j]);
          o[j] = bf16_any(p * cs[2 * j] - s * sn[2 * j]) | bf16_any(s * cs[2 * j] + p * sn[2 * j]) << 16;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t z = (uint32_t)__shfl((int)w[j], partner & 63);
          const float s0 = upper ? sn[2 * j] : -sn[2 * j], s1 = upper ? sn[2 * j + 1] : -sn[2 * j + 1];
          o[j] = bf16_any(lo_f(w[j]) * cs[2 * j] + lo_f(z) * s0) | bf16_any(hi_f(w[j]) * cs[2 * j + 1] + hi_f(z) * s1) << 16;
        }
      }
      const bool turn = turned && (is_q || is_k);
      if (live && h < heads && (is_q || in_pool)) {
        uint16_t* dst = is_q ? q_out + h * kHeadDim : is_k ? a.K + k_row + (int64_t)hk * a.k_sh : a.V + v_row + (int64_t)hk * a.v_sh;
        *reinterpret_cast<u32x4*>(dst + 8 * c) = turn ? o : w;
      }
    }
  }
  if (bad != 0 && a.guard != nullptr && lane == 0) atomicOr(a.guard, bad);
}
hipError_t launch_rope_append(const RopeArgs& a, int n_cu, hipStream_t s) {
  const int64_t tokens = (int64_t)a.B * a.max_new;
  const int quads = (a.Hq + 2 * a.Hkv + 3) / 4;
  const unsigned gx = (unsigned)((tokens + kRopeWaves - 1) / kRopeWaves);
  // Heads split over workgroups until every unit has eight.  8192 rows of 48 heads, one group of heads at a time / four: 44 / 36.5 us (201 MB, 5.5 TB/s);
  // four rows, a group each: 4.0 / 5.8.
  int parts = (int)((8 * (int64_t)n_cu + gx - 1) / gx);
  if (parts > quads) parts = quads;
  if (parts < 1) parts = 1;
  const dim3 grid(gx, parts), block(kRopeThreads);
  if (quads >= kRopeAhead * parts) hipLaunchKernelGGL(rope_append_kernel<kRopeAhead>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(rope_append_kernel<1>, grid, block, 0, s, a);
  return hipGetLastError();
}

// ---- eviction: the kept rows, in their order, to the front ----------------------------------------------------------
// Row r of what is left was row
//   r                          for the sink rows,
//   kept[r - n_sink]           for the n_kept rows of J that stay (ascending),
//   r + (rows that went)       for the recent rows.
struct MoveSpan {
  int L, sinks, kept, gone, after;  // rows before; sink rows; rows of J that stay / go; rows afterwards
  const int32_t* list;
  __device__ __forceinline__ int source(int r) const {  // (a word of the list is read whatever r is: several rows' reads go out together)
    const int v = list[min(max(r - sinks, 0), max(kept - 1, 0))];
    return r < sinks ? r : r < sinks + kept ? v : r + gone;
  }
};
__device__ __forceinline__ MoveSpan span_of(const MoveArgs& a, int bh) {
  MoveSpan m;
  m.L = (int)a.state[(int64_t)bh * kStateWords + ST_LEN];  // as the selecting launch read it: ctx_len may be overwritten here
  m.sinks = min(a.n_sink, m.L);
  m.kept = a.n_kept[bh];
  m.gone = max(0, m.L - a.recent - a.n_sink) - m.kept;
  m.after = m.L - m.gone;
  m.list = a.budget > 0 ? a.kept + (int64_t)bh * a.budget : a.n_kept;
  return m;
}
// Row numbers in the cache of N logical rows of sequence b; bit i of the result: row i's block id is in the pool.
template <int N>
__device__ __forceinline__ unsigned rows_in_pool(int64_t (&at)[N], const int (&row)[N], const int32_t* table, int64_t table_stride, int lg, int rpb,
                                                 int n_blocks, int b, int& bad) {
  unsigned ok = (1u << N) - 1;
  if (table == nullptr) {
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = row[i];
    return ok;
  }
  int page[N];
#pragma unroll
  for (int i = 0; i < N; ++i) page[i] = table[(int64_t)b * table_stride + (row[i] >> lg)];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int pc = min(max(page[i], 0), n_blocks - 1);
    if (pc != page[i]) {
      bad |= kGuardBlock;
      ok &= ~(1u << i);
    }
    at[i] = (int64_t)pc * rpb + (row[i] & ((1 << lg) - 1));
  }
  return ok;
}

constexpr int kMoveThreads = 256;
constexpr int kMoveItems = kMoveRows / (kMoveThreads / 16);
static_assert(kMoveRows % (kMoveThreads / 16) == 0, "whole rounds of 16 lanes a row");

// The first `pairs` workgroups: a pair's weights and positions, its lengths (the longest way).  The others: kMoveRows rows of K and V of a pair each.
// IN_PLACE: source and target are the same rows.  A row only ever moves down, so a chunk's target is the source of its own and
// of lower chunks: a workgroup holds its rows in registers, says so, and stores once the lower chunks whose sources it overwrites have
// said so.  Chunks are dealt by a counter, lower ones first, and nobody waits before having said its own: every wait ends.
template <bool IN_PLACE, bool STREAM>
__global__ __launch_bounds__(kMoveThreads) void move_rows_kernel(const MoveArgs a) {
  const int tid = threadIdx.x;
  __shared__ int s_ticket;
  int unit = blockIdx.x;
  if (IN_PLACE) {
    if (tid == 0) s_ticket = (int)atomicAdd(a.ticket, 1u);
    __syncthreads();
    unit = s_ticket;
  }
  const int pairs = a.B * a.Hkv;
  const int bh = unit % pairs, chunk = unit / pairs - 1;
  const int b = bh / a.Hkv, h = bh % a.Hkv;
  const MoveSpan m = span_of(a, bh);

  if (chunk < 0) {
    // One workgroup per pair, front to back: what it reads of a trip lies at or behind what it writes, and behind all it wrote before.
    constexpr int kPer = 8;
    const float* w_in = a.w_in + (int64_t)bh * a.w_in_rows;
    float* w_out = a.w_out != nullptr ? a.w_out + (int64_t)bh * a.w_out_rows : nullptr;
    const int32_t* p_in = a.pos_in != nullptr ? a.pos_in + (int64_t)bh * a.w_in_rows : nullptr;
    int32_t* p_out = a.pos_out != nullptr ? a.pos_out + (int64_t)bh * a.w_out_rows : nullptr;
    for (int r0 = 0; r0 < m.after; r0 += kPer * kMoveThreads) {
      float w[kPer];
      int32_t p[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int r = r0 + i * kMoveThreads + tid;
        const int src = r < m.after ? m.source(r) : 0;
        w[i] = r < m.after && w_out != nullptr ? w_in[src] : 0.f;
        p[i] = r < m.after && p_out != nullptr ? p_in[src] : 0;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int r = r0 + i * kMoveThreads + tid;
        if (r >= m.after) continue;
        if (w_out != nullptr) w_out[r] = w[i];
        if (p_out != nullptr) p_out[r] = p[i];
      }
      __syncthreads();
    }
    if (w_out != nullptr)  // rows appended later start without weight
      for (int r = m.after + tid; r < a.w_out_rows; r += kMoveThreads) w_out[r] = 0.f;
    if (h == 0 && tid == 0) {
      a.len_out[b] = m.after;
      if (a.recent_out != nullptr) a.recent_out[b] = max(a.n_sink, m.after - a.recent);
    }
    return;
  }

  const int r0 = chunk * kMoveRows;
  if (r0 >= m.after) return;
  const int last = min(r0 + kMoveRows, m.after) - 1;
  if (IN_PLACE && a.same_rows && m.source(last) == last) return;  // sources ascend: nothing up to here has moved
  int bad = 0;
  const int c = tid & 15, rr = tid >> 4;
  // (rows behind the last one repeat it: no branch between the requests)
  int from[kMoveItems];
  int64_t src[kMoveItems];
#pragma unroll
  for (int i = 0; i < kMoveItems; ++i) from[i] = m.source(min(r0 + rr + i * (kMoveThreads / 16), last));
  rows_in_pool<kMoveItems>(src, from, a.table, a.table_stride, a.page_lg, a.page_rpb, a.n_blocks, b, bad);
  const uint16_t* Kb = a.K + (int64_t)b * a.k_sb + (int64_t)h * a.k_sh + 8 * c;
  const uint16_t* Vb = a.V + (int64_t)b * a.v_sb + (int64_t)h * a.v_sh + 8 * c;
  u32x4 k4[kMoveItems], v4[kMoveItems];
#pragma unroll
  for (int i = 0; i < kMoveItems; ++i) {
    k4[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(Kb + src[i] * a.k_st));
    v4[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(Vb + src[i] * a.v_st));
  }
  int to[kMoveItems];
  int64_t dst[kMoveItems];
#pragma unroll
  for (int i = 0; i < kMoveItems; ++i) to[i] = min(r0 + rr + i * (kMoveThreads / 16), last);
  const unsigned ok = rows_in_pool<kMoveItems>(dst, to, a.table_out, a.table_out_stride, a.page_out_lg, a.page_out_rpb, a.n_blocks_out, b, bad);
  if (IN_PLACE) {
    // all of the workgroup's rows have arrived before it says so
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    uint32_t* flag = a.flags + (int64_t)bh * a.flag_stride;
    if (tid == 0) __hip_atomic_store(flag + chunk, 1u, __ATOMIC_RELEASE, __HIP_MEMORY_SCOPE_AGENT);
    if (tid < 64) {
      // first row whose source lies at or behind this chunk's first target (source(r) >= r: at most r0), 64 places a trip
      int lo = 0, hi = r0;
      while (lo < hi) {
        const int stride = (hi - lo + 63) / 64, at = lo + tid * stride;
        const uint64_t from_here = __ballot(at >= hi || m.source(min(at, hi - 1)) >= r0);
        const int f = from_here != 0ull ? __builtin_ctzll(from_here) : 64;
        const int up = min(lo + f * stride, hi);
        lo = f == 0 ? lo : lo + (f - 1) * stride + 1;  // the place before was too early
        hi = f == 0 ? lo : up;
      }
      // chunks from its place on have sources in what is overwritten here
      for (int d0 = lo / kMoveRows; d0 < chunk; d0 += 64) {
        const int d = min(d0 + tid, chunk - 1);
        while (!__all(__hip_atomic_load(flag + d, __ATOMIC_ACQUIRE, __HIP_MEMORY_SCOPE_AGENT) != 0u)) __builtin_amdgcn_s_sleep(2);
      }
    }
    __syncthreads();
  }
  uint16_t* Ko = a.K_out + (int64_t)b * a.ko_sb + (int64_t)h * a.ko_sh + 8 * c;
  uint16_t* Vo = a.V_out + (int64_t)b * a.vo_sb + (int64_t)h * a.vo_sh + 8 * c;
#pragma unroll
  for (int i = 0; i < kMoveItems; ++i)
    if (r0 + rr + i * (kMoveThreads / 16) <= last && (ok >> i & 1u) != 0) {  // a block that is not in the pool is not written
      if (STREAM) {
        __builtin_nontemporal_store(k4[i], reinterpret_cast<u32x4*>(Ko + dst[i] * a.ko_st));
        __builtin_nontemporal_store(v4[i], reinterpret_cast<u32x4*>(Vo + dst[i] * a.vo_st));
      } else {
        *reinterpret_cast<u32x4*>(Ko + dst[i] * a.ko_st) = k4[i];
        *reinterpret_cast<u32x4*>(Vo + dst[i] * a.vo_st) = v4[i];
      }
    }
  if (bad != 0 && a.guard != nullptr) atomicOr(a.guard, bad);
}
// Rows are read past the caches (nobody reads them again: 38 -> 32 us for 4 caches of 60000 rows cut to 4261), and written past them where
// the new caches would not stay there for the next step anyway: 16 x 4092 rows (268 MB) 113 -> 107 us, the 4 x 4261 (70 MB) 32 -> 36.
// In place: 16 x 5800..6200 rows of 8 KV heads cut to 4092 557 us (into another cache 107), 4 x 30011..60000 cut to 4261, paged, 176 (31), one of 4096 rows of 2 KV heads cut to 1028 5.6
// (4.0).  What bounds it has not been measured; unlike the copy it stores and reads a flag per workgroup, with release and acquire for the device.
hipError_t launch_move_rows(const MoveArgs& a, bool in_place, hipStream_t s) {
  const dim3 grid((unsigned)(a.n_chunks + 1) * (unsigned)(a.B * a.Hkv)), block(kMoveThreads);
  const int64_t bytes = (int64_t)a.B * a.Hkv * a.n_chunks * kMoveRows * (4 * kHeadDim);
  if (in_place) hipLaunchKernelGGL((move_rows_kernel<true, false>), grid, block, 0, s, a);
  else if (bytes > kCacheBytes / 2) hipLaunchKernelGGL((move_rows_kernel<false, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((move_rows_kernel<false, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace sfi
