// Dense decode attention of a batch whose sequences hold the same first rows: those are read once for all.
//
// For a KV head the B x G queries of the batch are columns of one matrix product against the shared rows, masked by how many of them
// each sequence shares; the rows that a sequence has of its own are a product with its G queries alone.  Both are cut into splits that leave flash
// records (running maximum, sum and accumulator, log2 domain: weights 2^(y - m), y = log2(e) * logit) in the layout of the dense kernel,
// [query head][split], and the own rows' launch, the second of two, joins them.
//
// Matrix instructions (16x16x32 bf16, fp32 accumulation), a tile of 32 rows, blocks A and B of 16:
//   S   = K (16 rows x 128) Q^T (128 x 16 columns): lane (jg = lane / 16, n = lane % 16) has logits of column n, rows 4 jg + i of a block
//   O^T += V^T (16 dims x 32 rows) P (32 rows x 16 columns): contraction slot (jg, i) is row 4 jg + i of block A (i < 4) or
//         4 jg + i - 4 of block B, where the first product left this lane's weights.  Product e of eight takes dim 8 m + e as its row m, so
//         lane (jg, n) loads 16 bytes of a V row as they lie (dims 8 n .. + 7), and has dims 8 (4 jg + i) + e of column n in the end:
//         maximum, sum and accumulator of a column stay in the lanes that have its logits.
// A weight goes into the second product as the sum of bf16 terms, each to nearest: with one the output would carry the weights' 2^-8.
// Three hold all 24 bits; two lose up to 2^-17, 2.4e-6 of the outputs' norm where the weights are alike (three: 2e-7 at 200 rows, 3e-7 at 16384,
// 4e-7 at 32768).  Two are taken for many columns behind a bf16 output alone, which rounds by up to 2^-8 itself: what an fp32 output holds does
// not depend on how many columns or rows a launch has room for.  Time with two / three terms, one row of their own:
// 64 sequences of 64 heads over 32768 rows 93 / 122 us, over 2048 17.2 / 18.4; 16 of 32 over 16384 15.6 / 16.1.
#include "sfi_internal.h"
#include "sfi_wave.h"

namespace sfi {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

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
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
// STREAM: past the caches, for rows that no other workgroup reads.
template <bool STREAM>
__device__ __forceinline__ uint4 load16(const char* p) {
  const u32x4 v = STREAM ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)) : *reinterpret_cast<const u32x4*>(p);
  return make_uint4(v.x, v.y, v.z, v.w);
}

// A tile in registers.  A K row leaves as requests of 64 bytes, so the other half of a cache line comes from the L2 if it is left there: K through the caches, V (whole
// lines at once) past them.  Own rows of 100 to 1201 and 300 rows 23.0 / 20.9 us (K past them too 27.4 / 23.0, V through them too 22.2 / 21.0), 1200 rows each
// 29.7 (29.8, 36); 16 columns over 32768 / 65536 rows 23.5 / 44.9 (25.2 / 44.8, 23.4 / 50).  (Two caches in turn: the last-level cache has part of the rows.)
struct Tile {
  uint4 ka[4], kb[4], v[8];
};
template <bool PAGED>
__device__ __forceinline__ void issue_k(Tile& T, const Rows& R, const Block& A, const Block& B, int r0, int jg, int n) {
  const char* pa = R.K + (uint64_t)(uint32_t)(min(max(r0 + n, A.first), A.last) + A.base) * R.k_st + jg * 16;
  const char* pb = R.K + (uint64_t)(uint32_t)(min(max(r0 + 16 + n, B.first), B.last) + B.base) * R.k_st + jg * 16;
#pragma unroll
  for (int kb = 0; kb < 4; ++kb) {
    T.ka[kb] = load16<false>(pa + kb * 64);
    T.kb[kb] = load16<false>(pb + kb * 64);
  }
}
template <bool PAGED>
__device__ __forceinline__ void issue_v(Tile& T, const Rows& R, const Block& A, const Block& B, int r0, int jg, int n) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    T.v[i] = load16<true>(R.V + (uint64_t)(uint32_t)(min(max(r0 + 4 * jg + i, A.first), A.last) + A.base) * R.v_st + n * 16);
    T.v[4 + i] = load16<true>(R.V + (uint64_t)(uint32_t)(min(max(r0 + 16 + 4 * jg + i, B.first), B.last) + B.base) * R.v_st + n * 16);
  }
}
// Element e of each of the eight rows: the operand of product e.
__device__ __forceinline__ bf16x8 turn_v(const uint4 (&v)[8], int e) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = (e >> 1) == 0 ? v[i].x : (e >> 1) == 1 ? v[i].y : (e >> 1) == 2 ? v[i].z : v[i].w;
  return __builtin_bit_cast(bf16x8, (e & 1) == 0 ? make_uint4(pack_lo(w[0], w[1]), pack_lo(w[2], w[3]), pack_lo(w[4], w[5]), pack_lo(w[6], w[7]))
                                                 : make_uint4(pack_hi(w[0], w[1]), pack_hi(w[2], w[3]), pack_hi(w[4], w[5]), pack_hi(w[6], w[7])));
}

// NCB blocks of 16 columns of a wave.
template <int NCB>
struct Cols {
  bf16x8 q[NCB][4];
  f32x4 acc[NCB][8];
  float m[NCB], l[NCB];  // l: of this lane's rows
  int lo[NCB], hi[NCB];  // rows this column sees
};
// The parts of a tile.  Products with K:
template <int NCB>
__device__ __forceinline__ void scores(const Cols<NCB>& C, const bf16x8 (&ka)[4], const bf16x8 (&kb)[4], f32x4 (&s)[NCB][2]) {
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) s[cb][0] = s[cb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb) {
      s[cb][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[k], C.q[cb][k], s[cb][0], 0, 0, 0);
      s[cb][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb[k], C.q[cb][k], s[cb][1], 0, 0, 0);
    }
}
// What a column does not see.
template <int NCB>
__device__ __forceinline__ void mask(const Cols<NCB>& C, f32x4 (&s)[NCB][2], int r0, int jg) {
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + 16 * (i >> 2) + 4 * jg + (i & 3);
      s[cb][i >> 2][i & 3] = r >= C.lo[cb] && r < C.hi[cb] ? s[cb][i >> 2][i & 3] : -__builtin_inff();
    }
}
// The weights of a block of columns in bf16 terms, and their sum over the lane's rows.
struct Weights {
  bf16x8 hi, lo, rest;
};
template <bool THREE>
__device__ __forceinline__ float weights_of(const f32x4 (&s)[2], float m, float c2, Weights& w) {
  float p[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], c2, -m));  // a masked row: 2^-inf = 0
  uint32_t hi[4], lo[4], rest[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    hi[i] = round2(p[2 * i], p[2 * i + 1]);
    const float r0 = p[2 * i] - __uint_as_float(hi[i] << 16), r1 = p[2 * i + 1] - __uint_as_float(hi[i] & 0xffff0000u);
    lo[i] = round2(r0, r1);
    if (THREE) rest[i] = round2(r0 - __uint_as_float(lo[i] << 16), r1 - __uint_as_float(lo[i] & 0xffff0000u));
  }
  if (THREE) w.rest = __builtin_bit_cast(bf16x8, make_uint4(rest[0], rest[1], rest[2], rest[3]));
  w.hi = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
  w.lo = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
  return ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
}
// All blocks' weights.  The running maximum may lag behind the rows: only when a lane's weights add up to more than kLag (they are then far
// from what fp32 or bf16 lose anything at) is it brought up, accumulators and sums rescaled and the weights made again.  That
// happens in the first tile, whose maximum is kNeg, and rarely later; the common way looks for no maximum at all.  c2 > 0.
constexpr float kLag = 256.f;
template <int NCB, bool THREE>
__device__ __forceinline__ void soften(Cols<NCB>& C, const f32x4 (&s)[NCB][2], Weights (&w)[NCB], float c2) {
  float sum[NCB];
  bool up = false;
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    sum[cb] = weights_of<THREE>(s[cb], C.m[cb], c2, w[cb]);
    up |= sum[cb] > kLag;
  }
  if (__builtin_expect(__any(up), 0)) {
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb) {
      const float mx = fmaxf(fmaxf(fmaxf(s[cb][0][0], s[cb][0][1]), fmaxf(s[cb][0][2], s[cb][0][3])),
                             fmaxf(fmaxf(s[cb][1][0], s[cb][1][1]), fmaxf(s[cb][1][2], s[cb][1][3]))) * c2;
      const float m1 = fmaxf(across_max(mx), C.m[cb]);  // (not below kNeg: finite)
      const float f = __builtin_amdgcn_exp2f(C.m[cb] - m1);
      C.m[cb] = m1;
      C.l[cb] *= f;
#pragma unroll
      for (int e = 0; e < 8; ++e) C.acc[cb][e] *= f;
      sum[cb] = weights_of<THREE>(s[cb], m1, c2, w[cb]);
    }
  }
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) C.l[cb] += sum[cb];
}
// Products with V.
template <bool THREE>
__device__ __forceinline__ void add_rows(f32x4 (&acc)[8], const bf16x8 (&vt)[8], const Weights& w) {
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[e], w.hi, acc[e], 0, 0, 0);
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[e], w.lo, acc[e], 0, 0, 0);
  if (THREE) {
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[e], w.rest, acc[e], 0, 0, 0);
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

// Tiles [t0, t1) of 32 rows, wave w of NW takes t0 + w, t0 + w + NW, ...; no column masks anything from row whole_from to whole_to.  DEPTH tile
// buffers; the rows of a later tile are requested into each half of a buffer as soon as its consumer is done with it.
template <bool PAGED>
struct Walker {
  Tile T;
  Block A, B;
  __device__ __forceinline__ void place(const Rows& R, int t, int& bad) {
    A = block_of<PAGED>(R, t * kTile, bad);
    B = block_of<PAGED>(R, t * kTile + 16, bad);
  }
};
template <int NCB, int NW, int DEPTH, bool PAGED>
__device__ __forceinline__ void walk(Cols<NCB>& C, const Rows& R, int t0, int t1, int whole_from, int whole_to, int wave, int jg, int n, float c2, int& bad) {
  Walker<PAGED> W[DEPTH];
  int t = t0 + wave;
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) {
    const int td = t + d * NW;
    if (td < t1) {
      W[d].place(R, td, bad);
      issue_k<PAGED>(W[d].T, R, W[d].A, W[d].B, td * kTile, jg, n);
      issue_v<PAGED>(W[d].T, R, W[d].A, W[d].B, td * kTile, jg, n);
    }
  }
  // Tile td out of buffer d, and the one that takes its place.
  auto tile = [&](int d, int td, bool refill) {
    const int next = td + DEPTH * NW, r0 = td * kTile;
    f32x4 s[NCB][2];
    {
      bf16x8 ka[4], kb[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        ka[k] = __builtin_bit_cast(bf16x8, W[d].T.ka[k]);
        kb[k] = __builtin_bit_cast(bf16x8, W[d].T.kb[k]);
      }
      scores<NCB>(C, ka, kb, s);
    }
    if (refill) {
      W[d].place(R, next, bad);
      issue_k<PAGED>(W[d].T, R, W[d].A, W[d].B, next * kTile, jg, n);
    }
    if (r0 < whole_from || r0 + kTile > whole_to) mask<NCB>(C, s, r0, jg);
    Weights w[NCB];
    soften<NCB, true>(C, s, w, c2);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bf16x8 vt = turn_v(W[d].T.v, e);
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb) {
        C.acc[cb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, w[cb].hi, C.acc[cb][e], 0, 0, 0);
        C.acc[cb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, w[cb].lo, C.acc[cb][e], 0, 0, 0);
        C.acc[cb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, w[cb].rest, C.acc[cb][e], 0, 0, 0);
      }
    }
    if (refill) issue_v<PAGED>(W[d].T, R, W[d].A, W[d].B, next * kTile, jg, n);
  };
  if (DEPTH == 1) {
    for (; t < t1; t += NW) tile(0, t, t + NW < t1);
    return;
  }
  // A loop in which every request is made, and the last tiles behind it: with a branch around requests the compiler waits for all that are on
  // their way (16 columns, 8 heads, 32768 rows: 26.3 us, without the branch 25.1; 65536 rows, paged: 47 / 45 us, 6.0 TB/s).
  for (; t + (2 * DEPTH - 1) * NW < t1; t += DEPTH * NW) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) tile(d, t + d * NW, true);
  }
#pragma unroll
  for (int d = 0; d < 2 * DEPTH - 1; ++d)
    if (t + d * NW < t1) tile(d % DEPTH, t + d * NW, t + (d + DEPTH) * NW < t1);
}

// Joins the columns of the NR waves that had other rows of the same columns (rank: which of them this wave is, 0 .. NR - 1; cols: the columns of all
// of the workgroup's waves, c0: this wave's first) and writes them as one record each: record(col) gives its address, nullptr: no such column.
// lds: join_floats.
template <int NR>
constexpr int join_floats(int cols) { return 2 * NR * cols + (NR > 1 ? NR / 2 * cols * (kHeadDim + 4) : 0); }
template <int NCB, int NR, bool TURNED, typename F>
__device__ __forceinline__ void join(Cols<NCB>& C, int rank, int cols, int c0, int jg, int n, float* lds, F record) {
  constexpr int kPitch = kHeadDim + 4;
  float M[NCB], Z[NCB];
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    M[cb] = C.m[cb];
    Z[cb] = across_sum(C.l[cb]);
  }
  if (NR > 1) {
    float* s_m = lds;               // [NR][cols]
    float* s_l = lds + NR * cols;
    float* s_acc = lds + 2 * NR * cols;  // [NR / 2][cols][kPitch]
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb)
      if (jg == 0) {
        s_m[rank * cols + c0 + 16 * cb + n] = C.m[cb];
        s_l[rank * cols + c0 + 16 * cb + n] = Z[cb];
      }
    __syncthreads();
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb) {
      const int c = c0 + 16 * cb + n;
#pragma unroll
      for (int w = 0; w < NR; ++w) M[cb] = fmaxf(M[cb], s_m[w * cols + c]);
      Z[cb] = 0.f;
#pragma unroll
      for (int w = 0; w < NR; ++w) Z[cb] += s_l[w * cols + c] * __builtin_amdgcn_exp2f(s_m[w * cols + c] - M[cb]);
      const float f = __builtin_amdgcn_exp2f(C.m[cb] - M[cb]);
#pragma unroll
      for (int e = 0; e < 8; ++e) C.acc[cb][e] *= f;
    }
#pragma unroll
    for (int left = NR / 2; left >= 1; left >>= 1) {  // the upper half hands over to the lower one
      if (rank >= left && rank < 2 * left) {
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<f32x4*>(s_acc + ((rank - left) * cols + c0 + 16 * cb + n) * kPitch + 16 * e + 4 * jg) = C.acc[cb][e];
      }
      __syncthreads();
      if (rank < left) {
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            C.acc[cb][e] += *reinterpret_cast<const f32x4*>(s_acc + (rank * cols + c0 + 16 * cb + n) * kPitch + 16 * e + 4 * jg);
      }
      if (left > 1) __syncthreads();
    }
  }
  if (rank != 0) return;
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    float* rec = record(c0 + 16 * cb + n);
    if (rec == nullptr) continue;
    if (jg == 0) *reinterpret_cast<float4*>(rec) = make_float4(M[cb], Z[cb], kNeg, 0.f);
    if (TURNED) {  // acc[e][i]: dim 8 (4 jg + i) + e
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float4* p = reinterpret_cast<float4*>(rec + 4 + 8 * (4 * jg + i));
        p[0] = make_float4(C.acc[cb][0][i], C.acc[cb][1][i], C.acc[cb][2][i], C.acc[cb][3][i]);
        p[1] = make_float4(C.acc[cb][4][i], C.acc[cb][5][i], C.acc[cb][6][i], C.acc[cb][7][i]);
      }
    } else {  // dim 16 e + 4 jg + i
#pragma unroll
      for (int e = 0; e < 8; ++e) *reinterpret_cast<f32x4*>(rec + 4 + 16 * e + 4 * jg) = C.acc[cb][e];
    }
  }
}

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

// What a workgroup's columns are: column c = query head c % G of the KV head's group in sequence c / G, and how many of the lead's rows it sees.
struct Seen {
  int most, least;  // over the wave's columns
};
template <int NCB>
__device__ __forceinline__ Seen load_columns(const SharedArgs& a, Cols<NCB>& C, int c0, int h, int jg, int n) {
  const int n_cols = a.B * a.G, L_lead = len_of(a, a.lead);
  int most = 0, least = 0x7fffffff;
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    const int c = c0 + 16 * cb + n, cc = min(c, n_cols - 1), b = cc / a.G, g = cc % a.G;
    load_query(C.q[cb], a.q + ((int64_t)b * a.Hq + h * a.G + g) * kHeadDim, c < n_cols, jg);
    C.lo[cb] = 0;
    C.hi[cb] = c < n_cols ? shared_of(a, b, len_of(a, b), L_lead) : 0;
    most = max(most, C.hi[cb]);
    least = min(least, c < n_cols ? C.hi[cb] : 0x7fffffff);
  }
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) {
    most = max(most, __shfl_xor(most, d));
    least = min(least, __shfl_xor(least, d));
  }
  return {__builtin_amdgcn_readfirstlane(most), __builtin_amdgcn_readfirstlane(least)};
}
__device__ __forceinline__ float* shared_record(const SharedArgs& a, int c, int h, int split) {
  return c < a.B * a.G ? a.part + (((int64_t)(c / a.G) * a.Hq + h * a.G + c % a.G) * kSlotCap + split) * kPartStride : nullptr;
}

// The shared rows for few columns (16): a workgroup per KV head and split, every wave with rows of its own in registers.
template <bool PAGED>
__global__ __launch_bounds__(kAttnThreads, 1) void shared_few_kernel(const SharedArgs a) {
  __shared__ __align__(16) float lds[join_floats<kWaves>(16)];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, jg = lane >> 4, n = lane & 15;
  const int h = blockIdx.x, split = blockIdx.y;
  Cols<1> C;
  start(C);
  const Seen seen = load_columns(a, C, 0, h, jg, n);
  int bad = 0;
  if (seen.most > 0) {
    Rows R = rows_of(a, a.lead, h);
    R.hi = seen.most - 1;
    const int tiles = (seen.most + kTile - 1) / kTile;
    walk<1, kWaves, 2, PAGED>(C, R, (int)((int64_t)tiles * split / a.n_shared), (int)((int64_t)tiles * (split + 1) / a.n_shared), 0, seen.least, wave, jg, n, a.scale_log2, bad);
  }
  join<1, kWaves, true>(C, wave, 16, 0, jg, n, lds, [&](int col) { return shared_record(a, col, h, split); });
  if (bad != 0 && a.guard != nullptr) atomicOr(a.guard, bad);
}

// The shared rows for many columns: the tiles go through LDS, where all waves of the workgroup read them.  CG groups of 16 NCB columns,
// and RG groups of waves that take a tile each of a stage of RG tiles.
// - Every thread requests kAhead stages in front, as 16 bytes of a row each, and stores a stage into one of two buffers: one barrier per
//   stage.  In LDS the 16-byte pieces of K row r stand at piece ^ (r & 15), the 32-byte pieces of V row r at piece ^ (r & 7): what 16 lanes read
//   together, one piece of 16 rows of K, or of 4 rows of V (transposed on the way: ds_read_b64_tr_b16 gives a lane one dim of
//   four rows), lies in different banks.
// - Eight waves, two on each SIMD.  64 sequences of 64 heads over 32768 rows of 8 KV heads: three terms 122 us, 69.3 GFLOP and as many again for the second
//   and third terms, 1140 TFLOP/s of matrix instructions where a library's 8192^3 product reaches 1200.  Two terms 93 to 106 us for 104 GFLOP; there
//   the matrix pipe is busy 46 % of the time, the vector pipe as long, and other orders did not bring them closer together: waves of a SIMD in turn 111, stage t's
//   products with V beside stage t + 1's weights and stage t + 2's products with K in steps of four 112, one wave per SIMD with 64 columns (spills) 214.
//   32 sequences of 32 heads over 16384 rows, paged (two groups of 64 columns), two terms: 26 us for 67 MB, 8.6 GFLOP.
template <bool PAGED, int NCB, int CG, int RG, bool THREE>
__global__ __launch_bounds__(64 * CG * RG, 1) void shared_many_kernel(const SharedArgs a) {
  constexpr int kThreads = 64 * CG * RG, kRowsHere = kTile * RG, kCols = 16 * NCB * CG;
  constexpr int kLoads = kRowsHere * 16 / kThreads;  // of K, and as many of V, per thread and stage
  constexpr int kRowStep = kThreads / 16;
  constexpr int kAhead = 2;  // stages on their way, and buffers
  static_assert(kLoads * kThreads == kRowsHere * 16, "whole rounds");
  static_assert(kThreads == 512 && RG <= 2, "eight waves, two on each SIMD");
  constexpr int kStage = kRowsHere * 512;
  constexpr int kLds = 2 * kStage > 4 * join_floats<RG>(kCols) ? 2 * kStage : 4 * join_floats<RG>(kCols);
  __shared__ __align__(16) unsigned char lds[kLds];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, jg = lane >> 4, n = lane & 15;
  const int cg = wave % CG, rg = wave / CG;
  const int h = blockIdx.x, split = blockIdx.y, c_first = blockIdx.z * kCols, c0 = 16 * NCB * cg;
  __shared__ int s_most[CG * RG];
  Cols<NCB> C;
  start(C);
  const Seen seen = load_columns(a, C, c_first + c0, h, jg, n);
  if (lane == 0) s_most[wave] = seen.most;
  __syncthreads();
  int most = 0;
#pragma unroll
  for (int w = 0; w < CG; ++w) most = max(most, s_most[w]);
  most = __builtin_amdgcn_readfirstlane(most);
  const float c2 = a.scale_log2;
  int bad = 0;
  const int stages = (most + kRowsHere - 1) / kRowsHere;
  const int t0 = (int)((int64_t)stages * split / a.n_shared), t1 = (int)((int64_t)stages * (split + 1) / a.n_shared);
  if (t0 < t1) {
    const Rows R = rows_of(a, a.lead, h);
    const int last = most - 1;
    const int my_row = tid >> 4, piece = tid & 15;
    uint4 pk[kAhead][kLoads], pv[kAhead][kLoads];
    // A wave's 64 pieces are of four rows, which lie in one page.
    auto row_of = [&](int t, int j) { return min(t * kRowsHere + 4 * wave + j * kRowStep, last); };
    int page[kLoads];  // of the stage that is requested next
    auto look_up = [&](int t) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) page[j] = PAGED ? R.table[row_of(t, j) >> R.lg] : 0;
    };
    auto request = [&](int slot, int t) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        int row = row_of(t, j);
        const uint32_t more = (uint32_t)min(lane >> 4, last - row);
        if (PAGED) {
          const int pc = min(max(page[j], 0), R.n_blocks - 1);
          bad |= pc != page[j] ? kGuardBlock : 0;
          row = pc * R.rpb + (row & ((1 << R.lg) - 1));
        }
        pk[slot][j] = load16<false>(R.K + (uint64_t)(uint32_t)row * R.k_st + (more * (uint32_t)R.k_st + piece * 16));
        pv[slot][j] = load16<false>(R.V + (uint64_t)(uint32_t)row * R.v_st + (more * (uint32_t)R.v_st + piece * 16));
      }
    };
    auto stash = [&](int slot, int buf) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int r = my_row + j * kRowStep;
        *reinterpret_cast<uint4*>(lds + buf + r * 256 + ((piece ^ (r & 15)) << 4)) = pk[slot][j];
        *reinterpret_cast<uint4*>(lds + buf + kRowsHere * 256 + r * 256 + (((piece >> 1) ^ (r & 7)) << 5) + ((piece & 1) << 4)) = pv[slot][j];
      }
    };
    const unsigned char* k_at = lds + (rg * kTile + n) * 256;
    const unsigned char* v_at = lds + kRowsHere * 256 + (rg * kTile + 4 * jg + (n >> 2)) * 256 + 8 * (n & 3);
    const int v_turn = (4 * jg + (n >> 2)) & 7;
    auto read_k = [&](int buf, bf16x8 (&ka)[4], bf16x8 (&kb)[4]) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        ka[k] = *reinterpret_cast<const bf16x8*>(k_at + buf + (((4 * k + jg) ^ n) << 4));
        kb[k] = *reinterpret_cast<const bf16x8*>(k_at + buf + 16 * 256 + (((4 * k + jg) ^ n) << 4));
      }
    };
    auto read_v = [&](int buf, bf16x8 (&vt)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned char* p = v_at + buf + ((e ^ v_turn) << 5);
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * 256));
        vt[e] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    };
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      look_up(min(t0 + s, t1 - 1));
      request(s, min(t0 + s, t1 - 1));
      __builtin_amdgcn_sched_barrier(0);  // in this order: the loop's wait for the first stage is not one for all of them
    }
    look_up(min(t0 + kAhead, t1 - 1));
    f32x4 s[NCB][2];
    bf16x8 ka[4], kb[4], vt[8];
    Weights w[NCB];
    auto stage = [&](int t, int u) {
      const int r0 = t * kRowsHere + rg * kTile, buf = u * kStage;
      stash(u, buf);
      request(u, min(t + kAhead, t1 - 1));
      look_up(min(t + kAhead + 1, t1 - 1));
      __syncthreads();
      read_k(buf, ka, kb);
      read_v(buf, vt);
      scores<NCB>(C, ka, kb, s);
      if (r0 + kTile > seen.least) mask<NCB>(C, s, r0, jg);
      soften<NCB, THREE>(C, s, w, c2);
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb) add_rows<THREE>(C.acc[cb], vt, w[cb]);
    };
    int t = t0;
    for (; t + 1 < t1; t += kAhead) {  // (no way out in the middle: it would make the compiler wait for both stages at the head)
      stage(t, 0);
      stage(t + 1, 1);
    }
    if (t < t1) stage(t, 0);
  }
  if (RG > 1) __syncthreads();  // the buffers are read no more
  join<NCB, RG, false>(C, rg, kCols, c0, jg, n, reinterpret_cast<float*>(lds), [&](int col) { return shared_record(a, c_first + col, h, split); });
  if (bad != 0 && a.guard != nullptr) atomicOr(a.guard, bad);
}

constexpr int kOwnWaves = 4;
constexpr int kOwnThreads = 64 * kOwnWaves;
constexpr int kOwnAhead = 8;  // records a thread requests together
constexpr int kDeviceScope = 16;  // cache-policy bit sc1 of the buffer instructions

// Where own rows are shared out (shared_splits), sequences that differ are evened out: 16 sequences of 100 to 1201 rows, 8 KV heads, 19.1 us, one workgroup per pair 21.8; and
// one that shares nothing among others that share 16384 rows is read by as many workgroups as it has records left.
// Which part of whose own rows workgroup `slot` of a KV head has, of own_wgs: tiles shared out evenly over the batch, as few to a workgroup as
// the workgroups allow (at least one for each wave), every sequence at least one workgroup and at most as many as it has records.
struct OwnShare {
  int b, part, parts;  // b = B: nothing
};
constexpr int kOwnPlan = kMaxOwnPlan / 64;  // sequences per lane
__device__ __forceinline__ OwnShare own_share(const SharedArgs& a, int slot, int lane) {
  const int L_lead = len_of(a, a.lead);
  uint32_t tiles[kOwnPlan], total = 0u;
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < kOwnPlan; ++i) {
    tiles[i] = 0u;
    const int b = 64 * i + lane;
    if (64 * i >= a.B || b >= a.B) continue;
    const int L = len_of(a, b), S = shared_of(a, b, L, L_lead);
    tiles[i] = S < L ? (uint32_t)((L + kTile - 1) / kTile - S / kTile) : 0u;
    total += tiles[i];
    most = fmaxf(most, (float)tiles[i]);
  }
  total = wave_sum(total);  // (the workspace has four bytes per row: below 2^32 tiles)
  const uint32_t cap = kSlotCap - a.n_shared, longest = (uint32_t)(wave_max(most) * 1.000001f) + 1u;  // a float is off by 2^-24 of itself
  const uint32_t lo = max(max((uint32_t)kOwnWaves, total / (uint32_t)a.own_wgs), longest / cap + 1u);
  const uint32_t hi = total / (uint32_t)(a.own_wgs - a.B) + 1u;
  auto parts_of = [&](uint32_t n, uint32_t per) { return max((n + per - 1u) / per, 1u); };
  auto needed = [&](uint32_t per) {
    uint32_t n = 0u;
#pragma unroll
    for (int i = 0; i < kOwnPlan; ++i)
      if (64 * i < a.B) n += 64 * i + lane < a.B ? parts_of(tiles[i], per) : 0u;
    return wave_sum(n);
  };
  uint32_t per = max(lo, hi);
  constexpr int kTries = 6;
  if (hi > lo) {
    uint32_t n[kTries];
#pragma unroll
    for (int k = 0; k < kTries; ++k) n[k] = needed(lo + (hi - lo) * k / kTries);
#pragma unroll
    for (int k = kTries - 1; k >= 0; --k) per = n[k] <= (uint32_t)a.own_wgs ? lo + (hi - lo) * k / kTries : per;
  }
  // (hi is enough: the sum of the rounded-up quotients is below total / hi + B)
  uint32_t base = 0u;
#pragma unroll
  for (int i = 0; i < kOwnPlan; ++i) {
    if (64 * i >= a.B) break;
    const uint32_t mine = 64 * i + lane < a.B ? parts_of(tiles[i], per) : 0u, upto = base + wave_incl_scan(mine);
    const uint64_t past = __ballot(upto > (uint32_t)slot);
    if (past != 0ull) {
      const int at = __builtin_ctzll(past);
      const int parts = __builtin_amdgcn_readlane((int)mine, at);
      return {64 * i + at, slot - (__builtin_amdgcn_readlane((int)upto, at) - parts), parts};
    }
    base = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  }
  return {a.B, 0, 0};
}

// A sequence's own rows, one (ALONE) or several workgroups per KV head and sequence, and the merge.  Bound by the rows and the records: 32 sequences of
// 8 KV heads with 1200 rows each, 157 MB from memory, in 34.5 us, 4.6 TB/s; 100 to 1201 rows, paged, 85 MB and 9 MB of the shared rows' records, 27.9, and 23.5 where
// the last-level cache has part of the rows (two such caches in turn); one row each 6.5.
// A tile per wave on its way: with two, two workgroups fit a unit in place of three, 40 -> 48 us.  The last of a pair's workgroups to finish merges the
// records of all and those of the shared rows, which the launch before has left, into the output; records go from workgroup to workgroup at
// device scope (stores and loads that name it, a count once the stores have been performed; the counter is zero between launches).
// A pair with one workgroup keeps its record in LDS, and requests the shared rows' records before its waves are joined.
template <bool PAGED, bool ALONE>
__global__ __launch_bounds__(kOwnThreads, 3) void own_rows_kernel(const SharedArgs a) {
  __shared__ __align__(16) float lds[join_floats<kOwnWaves>(16)];
  __shared__ __align__(16) float s_own[16][kPartStride];
  __shared__ float s_w[16][kSlotCap];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, jg = lane >> 4, n = lane & 15;
  const int h = blockIdx.x;
  const OwnShare own = ALONE ? OwnShare{(int)blockIdx.y, 0, 1} : own_share(a, blockIdx.y, lane);
  const int b = own.b;
  if (!ALONE && b == a.B) return;
  const int64_t head0 = (int64_t)b * a.Hq + h * a.G;
  Cols<1> C;
  start(C);
  load_query(C.q[0], a.q + (head0 + min(n, a.G - 1)) * kHeadDim, n < a.G, jg);
  const int L = len_of(a, b), S = shared_of(a, b, L, len_of(a, a.lead));
  C.lo[0] = S;
  C.hi[0] = L;
  int bad = (a.ctx_len[b] != L ? kGuardCtxLen : 0) | (a.shared_len[b] != S ? kGuardShared : 0);
  if (S < L) {
    Rows R = rows_of(a, b, h);
    R.lo = S;
    R.hi = L - 1;
    const int first = S / kTile, tiles = (L + kTile - 1) / kTile - first;
    walk<1, kOwnWaves, 1, PAGED>(C, R, first + (int)((int64_t)tiles * own.part / own.parts), first + (int)((int64_t)tiles * (own.part + 1) / own.parts), S, L, wave, jg, n,
                                 a.scale_log2, bad);
  }
  if (bad != 0 && a.guard != nullptr) atomicOr(a.guard, bad);

  // headers of a wave's heads, a record per lane; four output dims of every lanes-th record per thread, up to kRound heads at a time
  constexpr int kRec = kPartStride * (int)sizeof(float), kHeads = 16 / kOwnWaves, kRound = kOwnThreads / (kHeadDim / 4);
  const int n_rec = a.n_shared + (ALONE ? 0 : own.parts);  // in memory
  float* const pair = a.part + head0 * kSlotCap * kPartStride;
  const __amdgpu_buffer_rsrc_t recs = __builtin_amdgcn_make_buffer_rsrc(pair, 0, a.G * kSlotCap * kRec, 0x00020000);
  struct Share {
    int quads, lanes, rl, item, g, c;
  };
  auto share_of = [&](int g0) {
    Share r;
    r.quads = min(kRound, a.G - g0) * (kHeadDim / 4);
    r.lanes = kOwnThreads / r.quads;
    r.rl = tid / r.quads;
    r.item = tid % r.quads;
    r.g = g0 + r.item / (kHeadDim / 4);
    r.c = r.item % (kHeadDim / 4);
    return r;
  };
  float2 hd[kHeads];
  auto request_headers = [&]() {
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      const int g = wave + i * kOwnWaves;
      const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(recs, (min(g, a.G - 1) * kSlotCap + min(lane, max(n_rec - 1, 0))) * kRec, 0, ALONE ? 0 : kDeviceScope);
      hd[i] = lane < n_rec ? make_float2(__uint_as_float(v.x), __uint_as_float(v.y)) : make_float2(kNeg, 0.f);
    }
  };
  f32x4 pre[kOwnAhead];
  auto request = [&](const Share& r, int s0) {  // (records behind the last one repeat it)
#pragma unroll
    for (int i = 0; i < kOwnAhead; ++i) {
      const int s = max(min(s0 + i * r.lanes, n_rec - 1), 0);
      pre[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(recs, (min(r.g, a.G - 1) * kSlotCap + s) * kRec + 16 + 16 * r.c, 0,
                                                                               ALONE ? 0 : kDeviceScope));
    }
  };
  const Share first = share_of(0);
  if (ALONE && n_rec > 0) {
    request_headers();
    request(first, first.rl);
  }
  join<1, kOwnWaves, true>(C, wave, 16, 0, jg, n, lds, [&](int col) { return s_own[col]; });
  __syncthreads();
  if (!ALONE) {
    for (int i = tid; i < a.G * (kPartStride / 4); i += kOwnThreads) {
      const int g = i / (kPartStride / 4), c4 = i % (kPartStride / 4);
      __builtin_amdgcn_raw_buffer_store_b128(*reinterpret_cast<const u32x4*>(&s_own[g][4 * c4]), recs, (g * kSlotCap + a.n_shared + own.part) * kRec + 16 * c4, 0,
                                             kDeviceScope);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's record stores have been performed
    __shared__ uint32_t s_before;
    __syncthreads();
    uint32_t* const arrive = a.arrive + ((int64_t)b * a.Hkv + h) * kWaves * kArriveStride;
    if (tid == 0) s_before = __hip_atomic_fetch_add(arrive, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (s_before != (uint32_t)own.parts - 1) return;
    if (tid == 0) __hip_atomic_store(arrive, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    request_headers();
    request(first, first.rl);
  }
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int g = wave + i * kOwnWaves;
    if (g >= a.G) break;
    float2 ml = n_rec > 0 ? hd[i] : make_float2(kNeg, 0.f);
    if (ALONE && lane == n_rec) ml = make_float2(s_own[g][0], s_own[g][1]);
    const float w = __builtin_amdgcn_exp2f(ml.x - wave_max(ml.x));
    const float Z = wave_sum_f(w * ml.y);
    s_w[g][lane] = Z > 0.f ? w / Z : 0.f;
  }
  __syncthreads();
  f32x4* s_o = reinterpret_cast<f32x4*>(lds);  // [lanes][quads]
  bool odd = false;
  for (int g0 = 0; g0 < a.G; g0 += kRound) {
    const Share r = g0 == 0 ? first : share_of(g0);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (r.rl < r.lanes) {
      for (int s0 = r.rl; s0 < n_rec; s0 += kOwnAhead * r.lanes) {
        if (g0 > 0 || s0 > r.rl) request(r, s0);
#pragma unroll
        for (int i = 0; i < kOwnAhead; ++i) {
          const int s = s0 + i * r.lanes;
          if (s < n_rec) o += s_w[r.g][s] * pre[i];
        }
      }
      if (ALONE && r.rl == 0) o += s_w[r.g][n_rec] * *reinterpret_cast<const f32x4*>(&s_own[r.g][4 + 4 * r.c]);
      if (r.rl > 0) s_o[r.rl * r.quads + r.item] = o;
    }
    __syncthreads();
    if (r.rl == 0) {
      for (int k = 1; k < r.lanes; ++k) o += s_o[k * r.quads + r.item];
      store_out4(a.out, (head0 + r.g) * kHeadDim + 4 * r.c, make_float4(o[0], o[1], o[2], o[3]), a.out_bf16 != 0);
      odd |= !(fabsf(o[0]) + fabsf(o[1]) + fabsf(o[2]) + fabsf(o[3]) < __builtin_inff());
    }
    __syncthreads();
  }
  // A column of the shared rows' launch takes the lead's rows behind those that its sequence shares with a weight of zero, which a V row with
  // infinities or NaN turns into NaN.  An output that is not finite is therefore made again from the rows it sees alone, where others see more.
  if (__builtin_expect(!__syncthreads_or(odd), 1)) return;
  bool more = false;
  for (int i = tid; i < a.B; i += kOwnThreads) more |= shared_of(a, i, len_of(a, i), len_of(a, a.lead)) > S;
  if (!__syncthreads_or(more)) return;
  start(C);
  load_query(C.q[0], a.q + (head0 + min(n, a.G - 1)) * kHeadDim, n < a.G, jg);
  for (int part = S > 0 ? 0 : 1; part < (S < L ? 2 : 1); ++part) {  // the lead's rows, then its own
    Rows R = rows_of(a, part == 0 ? a.lead : b, h);
    R.lo = C.lo[0] = part == 0 ? 0 : S;
    C.hi[0] = part == 0 ? S : L;
    R.hi = C.hi[0] - 1;
    int reported = 0;
    walk<1, kOwnWaves, 1, PAGED>(C, R, R.lo / kTile, R.hi / kTile + 1, R.lo, R.hi + 1, wave, jg, n, a.scale_log2, reported);
  }
  join<1, kOwnWaves, true>(C, wave, 16, 0, jg, n, lds, [&](int col) { return s_own[col]; });
  __syncthreads();
  for (int g0 = 0; g0 < a.G; g0 += kRound) {
    const Share r = share_of(g0);  // the threads that stored before
    if (r.rl != 0) continue;
    const float4 v = *reinterpret_cast<const float4*>(&s_own[r.g][4 + 4 * r.c]);
    const float z = s_own[r.g][1], f = z == 0.f ? 0.f : 1.0f / z;  // no row: 0; a NaN that was seen is in z or v, and stays
    store_out4(a.out, (head0 + r.g) * kHeadDim + 4 * r.c, make_float4(v.x * f, v.y * f, v.z * f, v.w * f), a.out_bf16 != 0);
  }
}

}  // namespace

#define SFI_LAUNCH_PAGED(kernel, grid, threads, ...)                                                                        \
  do {                                                                                                                      \
    if (a.table != nullptr) hipLaunchKernelGGL((kernel<true __VA_OPT__(, ) __VA_ARGS__>), grid, dim3(threads), 0, s, a);    \
    else hipLaunchKernelGGL((kernel<false __VA_OPT__(, ) __VA_ARGS__>), grid, dim3(threads), 0, s, a);                      \
  } while (0)

// Columns (us of the shared rows' launch, 8 KV heads, three weight terms where not said otherwise):
//   up to 16 in registers: 2048 rows 7.7, 16384 rows 15.9, 65536 rows 45 (the kernel for many columns with 64: 7.5, 16.2, with two terms 56);
//   up to 256 by 64, which read the rows from the caches again: 32 columns 7.8 / 16.8 (32 in registers 9.4 / 18.8); 128 columns, 2048 / 16384 rows, 10.8 / 26.2
//   (all 128 at once 14.9 / 28.6); 256 columns, 4096 / 16384 rows 16.5 / 34.8 (256 at once 20 / 34.8);
//   above by 256: 512 columns, 16384 / 32768 rows 63 / 122 (by 64 69 / 145; two terms 51 / 93, by 64 59 / 114), though 4096 rows 24.8 (22.5).
int shared_cols(int n_cols) { return n_cols <= 16 ? 16 : n_cols <= 256 ? 64 : 256; }

hipError_t launch_shared_rows(const SharedArgs& a, hipStream_t s) {
  const int cols = shared_cols(a.B * a.G);
  const dim3 grid(a.Hkv, a.n_shared, (a.B * a.G + cols - 1) / cols);
  const bool three = a.out_bf16 == 0;
  if (cols == 16) SFI_LAUNCH_PAGED(shared_few_kernel, grid, kAttnThreads);
  else if (cols == 64 && three) SFI_LAUNCH_PAGED(shared_many_kernel, grid, 512, 1, 4, 2, true);
  else if (cols == 64) SFI_LAUNCH_PAGED(shared_many_kernel, grid, 512, 1, 4, 2, false);
  else if (three) SFI_LAUNCH_PAGED(shared_many_kernel, grid, 512, 2, 8, 1, true);
  else SFI_LAUNCH_PAGED(shared_many_kernel, grid, 512, 2, 8, 1, false);
  return hipGetLastError();
}
hipError_t launch_own_rows(const SharedArgs& a, hipStream_t s) {
  const bool alone = a.own_wgs == 0;
  const dim3 grid(a.Hkv, alone ? a.B : a.own_wgs), block(kOwnThreads);
  if (alone && a.table != nullptr) hipLaunchKernelGGL((own_rows_kernel<true, true>), grid, block, 0, s, a);
  else if (alone) hipLaunchKernelGGL((own_rows_kernel<false, true>), grid, block, 0, s, a);
  else if (a.table != nullptr) hipLaunchKernelGGL((own_rows_kernel<true, false>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((own_rows_kernel<false, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace sfi
