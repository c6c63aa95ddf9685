// Dense decode attention of a batch whose sequences hold the same first rows: those are read once for all.
//
// For a KV head the B x G queries of the batch are columns of one matrix product against the shared rows, masked by how many of them
// each sequence shares; the rows that a sequence has of its own are a product with its G queries alone.  Both are cut into splits that leave flash
// records (running maximum, sum and accumulator, log2 domain: weights 2^(y - m), y = log2(e) * logit) in the layout of the dense kernel,
// [query head][split], and the merge launch joins them.
//
// Matrix instructions (16x16x32 bf16, fp32 accumulation), a tile of 32 rows, blocks A and B of 16:
//   S   = K (16 rows x 128) Q^T (128 x 16 columns): lane (jg = lane / 16, n = lane % 16) has logits of column n, rows 4 jg + i of a block
//   O^T += V^T (16 dims x 32 rows) P (32 rows x 16 columns): contraction slot (jg, i) is row 4 jg + i of block A (i < 4) or
//         4 jg + i - 4 of block B, where the first product left this lane's weights.  Product e of eight takes dim 8 m + e as its row m, so
//         lane (jg, n) loads 16 bytes of a V row as they lie (dims 8 n .. + 7), and has dims 8 (4 jg + i) + e of column n in the end:
//         maximum, sum and accumulator of a column stay in the lanes that have its logits.
// A weight goes into the second product as the sum of two bf16 (what is lost is below 2^-17 of it): with one the output would
// carry the weights' 2^-9, with two it has fp32's accuracy but for the order of the sums.
#include "sfi_internal.h"

namespace sfi {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;

namespace {

__device__ __forceinline__ uint32_t pack_lo(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t pack_hi(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ float across_max(float v) {  // over lanes n, n + 16, n + 32, n + 48
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const float t = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(t), __float_as_uint(t), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float across_sum(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const float t = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(t), __float_as_uint(t), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// two fp32 -> two bf16, nearest even
__device__ __forceinline__ uint32_t round2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Where a tile's rows lie.  Rows outside [lo, hi] are replaced by one of the same block of 16 inside, or by the nearest row if the block has
// none: nothing else is read, and what a replacement contributes is masked.
struct Rows {
  const char* K;    // KV head's base (of the sequence, or of the pool)
  const char* V;
  uint64_t k_st, v_st;  // bytes
  const int32_t* table;
  int lg, rpb, n_blocks;
  int lo, hi;
};
struct Block {
  int first, last, base;  // rows of the block that may be read; what to add to a row for its number in the pool
};
template <bool PAGED>
__device__ __forceinline__ Block block_of(const Rows& R, int r0, int& bad) {
  Block b;
  b.first = max(R.lo, r0);
  b.last = min(R.hi, r0 + 15);
  if (b.first > b.last) b.first = b.last = min(max(r0, R.lo), R.hi);
  b.base = 0;
  if (PAGED) {
    const int at = b.first >> R.lg;
    const int page = R.table[at], pc = min(max(page, 0), R.n_blocks - 1);
    bad |= pc != page ? kGuardBlock : 0;
    b.base = pc * R.rpb - (at << R.lg);
  }
  return b;
}
__device__ __forceinline__ uint4 load16(const char* p) { return *reinterpret_cast<const uint4*>(p); }

struct Tile {
  uint4 ka[4], kb[4], v[8];
};
template <bool PAGED>
__device__ __forceinline__ void issue(Tile& T, const Rows& R, int r0, int jg, int n, int& bad) {
  const Block A = block_of<PAGED>(R, r0, bad), B = block_of<PAGED>(R, r0 + 16, bad);
  const char* pa = R.K + (uint64_t)(uint32_t)(min(max(r0 + n, A.first), A.last) + A.base) * R.k_st + jg * 16;
  const char* pb = R.K + (uint64_t)(uint32_t)(min(max(r0 + 16 + n, B.first), B.last) + B.base) * R.k_st + jg * 16;
#pragma unroll
  for (int kb = 0; kb < 4; ++kb) {
    T.ka[kb] = load16(pa + kb * 64);
    T.kb[kb] = load16(pb + kb * 64);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    T.v[i] = load16(R.V + (uint64_t)(uint32_t)(min(max(r0 + 4 * jg + i, A.first), A.last) + A.base) * R.v_st + n * 16);
    T.v[4 + i] = load16(R.V + (uint64_t)(uint32_t)(min(max(r0 + 16 + 4 * jg + i, B.first), B.last) + B.base) * R.v_st + n * 16);
  }
}
// vt[e]: element e of each of the eight rows, the operand of product e.
__device__ __forceinline__ void turn_v(const uint4 (&v)[8], bf16x8 (&vt)[8]) {
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = d == 0 ? v[i].x : d == 1 ? v[i].y : d == 2 ? v[i].z : v[i].w;
    vt[2 * d] = __builtin_bit_cast(bf16x8, make_uint4(pack_lo(w[0], w[1]), pack_lo(w[2], w[3]), pack_lo(w[4], w[5]), pack_lo(w[6], w[7])));
    vt[2 * d + 1] = __builtin_bit_cast(bf16x8, make_uint4(pack_hi(w[0], w[1]), pack_hi(w[2], w[3]), pack_hi(w[4], w[5]), pack_hi(w[6], w[7])));
  }
}

// NCB blocks of 16 columns of a wave.
template <int NCB>
struct Cols {
  bf16x8 q[NCB][4];
  f32x4 acc[NCB][8];
  float m[NCB], l[NCB];  // l: of this lane's rows
  int lo[NCB], hi[NCB];  // rows this column sees
};
// The running maximum is let lag behind by up to kLag octaves before accumulators are rescaled (weights up to 2^kLag: nothing is lost in fp32).
constexpr float kLag = 8.f;
template <int NCB>
__device__ __forceinline__ void step(Cols<NCB>& C, const bf16x8 (&ka)[4], const bf16x8 (&kb)[4], const bf16x8 (&vt)[8], int r0, int jg, bool masked,
                                     float c2) {
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      s[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[k], C.q[cb][k], s[0], 0, 0, 0);
      s[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb[k], C.q[cb][k], s[1], 0, 0, 0);
    }
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = s[i >> 2][i & 3] * c2;
    if (masked) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * (i >> 2) + 4 * jg + (i & 3);
        y[i] = r >= C.lo[cb] && r < C.hi[cb] ? y[i] : kNeg;
      }
    }
    float mx = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
    mx = across_max(mx);
    if (__any(mx > C.m[cb] + kLag)) {
      const float m1 = fmaxf(mx, C.m[cb]);
      const float f = __builtin_amdgcn_exp2f(C.m[cb] - m1);
      C.m[cb] = m1;
      C.l[cb] *= f;
#pragma unroll
      for (int e = 0; e < 8; ++e) C.acc[cb][e] *= f;
    }
    float p[8], rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(y[i] - C.m[cb]);
    if (masked) {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = y[i] == kNeg ? 0.f : p[i];
    }
    C.l[cb] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      hi[i] = round2(p[2 * i], p[2 * i + 1]);
      rest[2 * i] = p[2 * i] - __uint_as_float(hi[i] << 16);
      rest[2 * i + 1] = p[2 * i + 1] - __uint_as_float(hi[i] & 0xffff0000u);
      lo[i] = round2(rest[2 * i], rest[2 * i + 1]);
    }
    const bf16x8 ph = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
    const bf16x8 pl = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      C.acc[cb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[e], ph, C.acc[cb][e], 0, 0, 0);
      C.acc[cb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[e], pl, C.acc[cb][e], 0, 0, 0);
    }
  }
}
template <int NCB>
__device__ __forceinline__ void start(Cols<NCB>& C) {
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    C.m[cb] = kNeg;
    C.l[cb] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) C.acc[cb][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
}
__device__ __forceinline__ void load_query(bf16x8 (&q)[4], const uint16_t* row, bool live, int jg) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint4 t = *reinterpret_cast<const uint4*>(row + 32 * k + 8 * jg);
    if (!live) t = make_uint4(0u, 0u, 0u, 0u);
    q[k] = __builtin_bit_cast(bf16x8, t);
  }
}

// Tiles [t0, t1) of 32 rows, wave w of the workgroup takes t0 + w, t0 + w + 4, ...; whole: no column masks anything in tiles below it.
template <int NCB, bool PAGED>
__device__ __forceinline__ void walk(Cols<NCB>& C, const Rows& R, int t0, int t1, int whole_from, int whole_to, int wave, int jg, int n, float c2, int& bad) {
  Tile T;
  int t = t0 + wave;
  if (t < t1) issue<PAGED>(T, R, t * kTile, jg, n, bad);
  for (; t < t1; t += kWaves) {
    bf16x8 ka[4], kb[4], vt[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      ka[k] = __builtin_bit_cast(bf16x8, T.ka[k]);
      kb[k] = __builtin_bit_cast(bf16x8, T.kb[k]);
    }
    turn_v(T.v, vt);
    if (t + kWaves < t1) issue<PAGED>(T, R, (t + kWaves) * kTile, jg, n, bad);
    step<NCB>(C, ka, kb, vt, t * kTile, jg, t * kTile < whole_from || (t + 1) * kTile > whole_to, c2);
  }
}

// The four waves' columns joined and written as one record each: rows(col) gives the record's address, nullptr: no such column.
template <int NCB, typename F>
__device__ __forceinline__ void join(Cols<NCB>& C, int wave, int jg, int n, float* lds, F record) {
  constexpr int kCols = 16 * NCB, kPitch = kHeadDim + 4;
  float* s_m = lds;                      // [kWaves][kCols]
  float* s_l = lds + kWaves * kCols;
  float* s_acc = lds + 2 * kWaves * kCols;  // [2][kCols][kPitch]
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    const float l = across_sum(C.l[cb]);
    if (jg == 0) {
      s_m[wave * kCols + 16 * cb + n] = C.m[cb];
      s_l[wave * kCols + 16 * cb + n] = l;
    }
  }
  __syncthreads();
  float M[NCB], Z[NCB];
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    const int c = 16 * cb + n;
    M[cb] = fmaxf(fmaxf(s_m[c], s_m[kCols + c]), fmaxf(s_m[2 * kCols + c], s_m[3 * kCols + c]));
    Z[cb] = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) Z[cb] += s_l[w * kCols + c] * __builtin_amdgcn_exp2f(s_m[w * kCols + c] - M[cb]);
    const float f = __builtin_amdgcn_exp2f(C.m[cb] - M[cb]);
#pragma unroll
    for (int e = 0; e < 8; ++e) C.acc[cb][e] *= f;
  }
  for (int left = kWaves / 2; left >= 1; left >>= 1) {  // the upper half hands over to the lower one
    if (wave >= left && wave < 2 * left) {
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float* p = s_acc + ((wave - left) * kCols + 16 * cb + n) * kPitch + 8 * (4 * jg + i);
          *reinterpret_cast<float4*>(p) = make_float4(C.acc[cb][0][i], C.acc[cb][1][i], C.acc[cb][2][i], C.acc[cb][3][i]);
          *reinterpret_cast<float4*>(p + 4) = make_float4(C.acc[cb][4][i], C.acc[cb][5][i], C.acc[cb][6][i], C.acc[cb][7][i]);
        }
    }
    __syncthreads();
    if (wave < left) {
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float* p = s_acc + (wave * kCols + 16 * cb + n) * kPitch + 8 * (4 * jg + i);
#pragma unroll
          for (int e = 0; e < 8; ++e) C.acc[cb][e][i] += p[e];
        }
    }
    __syncthreads();
  }
  if (wave != 0) return;
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    float* rec = record(16 * cb + n);
    if (rec == nullptr) continue;
    if (jg == 0) *reinterpret_cast<float4*>(rec) = make_float4(M[cb], Z[cb], kNeg, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float4* p = reinterpret_cast<float4*>(rec + 4 + 8 * (4 * jg + i));
      p[0] = make_float4(C.acc[cb][0][i], C.acc[cb][1][i], C.acc[cb][2][i], C.acc[cb][3][i]);
      p[1] = make_float4(C.acc[cb][4][i], C.acc[cb][5][i], C.acc[cb][6][i], C.acc[cb][7][i]);
    }
  }
}
template <int NCB>
constexpr int join_floats() { return 2 * kWaves * 16 * NCB + 2 * 16 * NCB * (kHeadDim + 4); }

__device__ __forceinline__ Rows rows_of(const SharedArgs& a, int b, int h) {
  Rows R;
  R.K = reinterpret_cast<const char*>(a.K + (a.table == nullptr ? (int64_t)b * a.k_sb : 0) + (int64_t)h * a.k_sh);
  R.V = reinterpret_cast<const char*>(a.V + (a.table == nullptr ? (int64_t)b * a.v_sb : 0) + (int64_t)h * a.v_sh);
  R.k_st = (uint64_t)a.k_st * 2;
  R.v_st = (uint64_t)a.v_st * 2;
  R.table = a.table != nullptr ? a.table + (int64_t)b * a.table_stride : nullptr;
  R.lg = a.page_lg;
  R.rpb = a.page_rpb;
  R.n_blocks = a.n_blocks;
  R.lo = 0;
  R.hi = 0;
  return R;
}
__device__ __forceinline__ int len_of(const SharedArgs& a, int b) { return min(max(a.ctx_len[b], 0), a.len_cap); }
__device__ __forceinline__ int shared_of(const SharedArgs& a, int b, int L, int L_lead) {
  return min(max(a.shared_len[b], 0), min(min(L, L_lead), a.max_shared));
}

// The shared rows: a workgroup per KV head, split and group of 16 NCB columns (column c = query head c % G of the KV head's group in sequence c / G).
template <int NCB, bool PAGED>
__global__ __launch_bounds__(kAttnThreads, 1) void shared_rows_kernel(const SharedArgs a) {
  __shared__ __align__(16) float lds[join_floats<NCB>()];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, jg = lane >> 4, n = lane & 15;
  const int h = blockIdx.x, split = blockIdx.y, c0 = blockIdx.z * (16 * NCB);
  const int n_cols = a.B * a.G;
  const int L_lead = len_of(a, a.lead);
  Cols<NCB> C;
  start(C);
  int most = 0, least = 0x7fffffff;
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    const int c = c0 + 16 * cb + n, cc = min(c, n_cols - 1), b = cc / a.G, g = cc % a.G;
    C.lo[cb] = 0;
    C.hi[cb] = c < n_cols ? shared_of(a, b, len_of(a, b), L_lead) : 0;
    most = max(most, C.hi[cb]);
    least = min(least, c < n_cols ? C.hi[cb] : 0x7fffffff);
    load_query(C.q[cb], a.q + ((int64_t)b * a.Hq + h * a.G + g) * kHeadDim, c < n_cols, jg);
  }
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) {
    most = max(most, __shfl_xor(most, d));
    least = min(least, __shfl_xor(least, d));
  }
  most = __builtin_amdgcn_readfirstlane(most);
  least = __builtin_amdgcn_readfirstlane(least);
  int bad = 0;
  if (most > 0) {
    Rows R = rows_of(a, a.lead, h);
    R.hi = most - 1;
    const int tiles = (most + kTile - 1) / kTile;
    walk<NCB, PAGED>(C, R, (int)((int64_t)tiles * split / a.n_shared), (int)((int64_t)tiles * (split + 1) / a.n_shared), 0, least, wave, jg, n, a.scale_log2, bad);
  }
  join<NCB>(C, wave, jg, n, lds, [&](int col) -> float* {
    const int c = c0 + col;
    if (c >= n_cols) return nullptr;
    return a.part + (((int64_t)(c / a.G) * a.Hq + h * a.G + c % a.G) * kSlotCap + split) * kPartStride;
  });
  if (bad != 0 && a.guard != nullptr) atomicOr(a.guard, bad);
}

// A sequence's own rows: a workgroup per KV head, split and sequence.
template <bool PAGED>
__global__ __launch_bounds__(kAttnThreads, 2) void own_rows_kernel(const SharedArgs a) {
  __shared__ __align__(16) float lds[join_floats<1>()];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, jg = lane >> 4, n = lane & 15;
  const int h = blockIdx.x, split = blockIdx.y, b = blockIdx.z;
  const int L = len_of(a, b), S = shared_of(a, b, L, len_of(a, a.lead));
  Cols<1> C;
  start(C);
  C.lo[0] = S;
  C.hi[0] = L;
  load_query(C.q[0], a.q + ((int64_t)b * a.Hq + h * a.G + min(n, a.G - 1)) * kHeadDim, n < a.G, jg);
  int bad = (a.ctx_len[b] != L ? kGuardCtxLen : 0) | (a.shared_len[b] != S ? kGuardShared : 0);
  if (S < L) {
    Rows R = rows_of(a, b, h);
    R.lo = S;
    R.hi = L - 1;
    const int first = S / kTile, tiles = (L + kTile - 1) / kTile - first;
    walk<1, PAGED>(C, R, first + tiles * split / a.n_own, first + tiles * (split + 1) / a.n_own, S, L, wave, jg, n, a.scale_log2, bad);
  }
  join<1>(C, wave, jg, n, lds, [&](int col) -> float* {
    if (col >= a.G) return nullptr;
    return a.part + (((int64_t)b * a.Hq + h * a.G + col) * kSlotCap + a.n_shared + split) * kPartStride;
  });
  if (bad != 0 && a.guard != nullptr) atomicOr(a.guard, bad);
}

template <int NCB>
void launch_shared_t(const SharedArgs& a, hipStream_t s) {
  const dim3 grid(a.Hkv, a.n_shared, (a.B * a.G + 16 * NCB - 1) / (16 * NCB));
  if (a.table != nullptr) hipLaunchKernelGGL((shared_rows_kernel<NCB, true>), grid, dim3(kAttnThreads), 0, s, a);
  else hipLaunchKernelGGL((shared_rows_kernel<NCB, false>), grid, dim3(kAttnThreads), 0, s, a);
}

}  // namespace

int shared_cols(int n_cols) { return n_cols <= 16 ? 16 : n_cols <= 32 ? 32 : 64; }

hipError_t launch_shared_rows(const SharedArgs& a, hipStream_t s) {
  switch (shared_cols(a.B * a.G)) {
    case 16: launch_shared_t<1>(a, s); break;
    case 32: launch_shared_t<2>(a, s); break;
    default: launch_shared_t<4>(a, s);
  }
  return hipGetLastError();
}
hipError_t launch_own_rows(const SharedArgs& a, hipStream_t s) {
  const dim3 grid(a.Hkv, a.n_own, a.B);
  if (a.table != nullptr) hipLaunchKernelGGL(own_rows_kernel<true>, grid, dim3(kAttnThreads), 0, s, a);
  else hipLaunchKernelGGL(own_rows_kernel<false>, grid, dim3(kAttnThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace sfi
