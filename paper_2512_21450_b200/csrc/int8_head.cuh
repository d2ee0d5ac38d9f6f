// Rows in 8-bit integers with a scale each, and the head's products on them: z_tv = a_t b_v sum_k A_tk B_vk, A the tokens' hidden states
// and B the rows of W.  The sums are exact (32-bit integers); one rounding to fp32, two multiplications, and where asked for one
// rounding to 16 bits follow.
//
// A row x becomes q = rint(x r), half to even, r = 127 / max|x| in fp32, and stands for s q, s = max|x| / 127.  The product x r is not
// rounded before it is rounded to an integer: fma(x, r, 1.5 * 2^23) rounds once, to a float whose last place is 1 and whose low byte
// is q.  A row whose largest magnitude is below 2^-100 (127 / it may overflow) counts as zero: s = 0.  A row with an infinity or a NaN
// has s = NaN and q = 0, so that everything it enters is NaN.
#pragma once
#include <cuda_fp16.h>

#include "epilogues.cuh"

namespace rlh {

constexpr float kSmallestRow = 7.888609052210118e-31f;   // 2^-100

struct RowScale {
  float s, r;
};
// From the bits of the largest magnitude (as integers they order as the values do, NaN above all).
__device__ __forceinline__ RowScale row_scale(uint32_t most_bits) {
  const float most = __uint_as_float(most_bits);
  if (most_bits >= 0x7f800000u) return {CUDART_NAN_F, 0.f};
  if (most < kSmallestRow) return {0.f, 0.f};
  return {__fdiv_rn(most, 127.f), __fdiv_rn(127.f, most)};
}
__device__ __forceinline__ uint32_t pack4(const RowScale& c, float x0, float x1, float x2, float x3) {
  constexpr float kMagic = 12582912.f;
  const uint32_t a = __float_as_uint(__fmaf_rn(x0, c.r, kMagic)), b = __float_as_uint(__fmaf_rn(x1, c.r, kMagic));
  const uint32_t d = __float_as_uint(__fmaf_rn(x2, c.r, kMagic)), e = __float_as_uint(__fmaf_rn(x3, c.r, kMagic));
  const uint32_t w = __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(d, e, 0x0040), 0x5410);
  return c.r == 0.f ? 0u : w;
}
// Eight elements of a row as they were loaded: the running maximum of their magnitudes (two 16-bit words, or the bits of a float),
// the bits of the float that it is, and the eight bytes that they become.
template <class T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ uint32_t most(uint32_t m) const {
    constexpr uint32_t k = 0x7fff7fffu;
    return __vmaxu2(m, __vmaxu2(__vmaxu2(v.x & k, v.y & k), __vmaxu2(v.z & k, v.w & k)));
  }
  __device__ static __forceinline__ uint32_t larger(uint32_t m) { return max(m & 0xffffu, m >> 16); }
  __device__ static __forceinline__ uint32_t bits(uint32_t m) { return m << 16; }
  __device__ __forceinline__ uint2 pack(const RowScale& c) const {
    auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
    auto hi = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
    return make_uint2(pack4(c, lo(v.x), hi(v.x), lo(v.y), hi(v.y)), pack4(c, lo(v.z), hi(v.z), lo(v.w), hi(v.w)));
  }
};
template <>
struct Eight<__half> : Eight<__nv_bfloat16> {
  __device__ __forceinline__ void load(const __half* p) { v = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ static __forceinline__ uint32_t bits(uint32_t m) { return __float_as_uint(__half2float(__ushort_as_half((unsigned short)m))); }
  __device__ __forceinline__ uint2 pack(const RowScale& c) const {
    auto of = [](uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); };
    const float2 a = of(v.x), b = of(v.y), d = of(v.z), e = of(v.w);
    return make_uint2(pack4(c, a.x, a.y, b.x, b.y), pack4(c, d.x, d.y, e.x, e.y));
  }
};
template <>
struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __ldg(reinterpret_cast<const float4*>(p));
    b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ uint32_t most(uint32_t m) const {
    auto u = [](float x) { return __float_as_uint(x) & 0x7fffffffu; };
    return max(m, max(max(max(u(a.x), u(a.y)), max(u(a.z), u(a.w))), max(max(u(b.x), u(b.y)), max(u(b.z), u(b.w)))));
  }
  __device__ static __forceinline__ uint32_t larger(uint32_t m) { return m; }
  __device__ static __forceinline__ uint32_t bits(uint32_t m) { return m; }
  __device__ __forceinline__ uint2 pack(const RowScale& c) const {
    return make_uint2(pack4(c, a.x, a.y, a.z, a.w), pack4(c, b.x, b.y, b.z, b.w));
  }
};
__device__ __forceinline__ uint32_t warp_max(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }
// What is stored in 8 bits, as the bf16 that the products of the loss take: 16 bytes to 16 values.
__device__ __forceinline__ void unpack16(const uint4& q, float s, uint4& lo, uint4& hi) {
  auto two = [&](uint32_t w, int i) {
    const float a = (float)(int8_t)(w >> (8 * i)) * s, b = (float)(int8_t)(w >> (8 * i + 8)) * s;
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  };
  lo = make_uint4(two(q.x, 0), two(q.x, 2), two(q.y, 0), two(q.y, 2));
  hi = make_uint4(two(q.z, 0), two(q.z, 2), two(q.w, 0), two(q.w, 2));
}
// One row of 8 * vecs elements, 16-byte aligned, by one warp: put(v, bytes of elements 8 v to 8 v + 7); the scale.  What does not fit
// HELD loads per lane is read twice.
template <int HELD, class T, class Put>
__device__ __forceinline__ float quantize_row(const T* src, int vecs, int lane, Put put) {
  Eight<T> h[HELD];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (lane + 32 * i < vecs) h[i].load(src + (lane + 32 * i) * 8);
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (lane + 32 * i < vecs) m = h[i].most(m);
  for (int v = lane + 32 * HELD; v < vecs; v += 32) {
    Eight<T> x;
    x.load(src + v * 8);
    m = x.most(m);
  }
  const RowScale c = row_scale(Eight<T>::bits(warp_max(Eight<T>::larger(m))));
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (lane + 32 * i < vecs) put(lane + 32 * i, h[i].pack(c));
  for (int v = lane + 32 * HELD; v < vecs; v += 32) {
    Eight<T> x;
    x.load(src + v * 8);
    put(v, x.pack(c));
  }
  return c.s;
}

// Any rows, a warp each.  HELD > 0: 16-byte aligned rows of a multiple of 8 elements, quantize_row<HELD>; else one element after the other.
// As many loads per lane as a row has, no more: bf16, 65536 rows of 896 elements 29.8 us with 4, 37.6 with 8, 60.9 with 16; of 3584 118 with 8, 113
// with 16 (6.2 TB/s).  151936 rows of 2048: bf16 135 us, fp16 135, fp32 217 (6.9-7.2 TB/s; read twice, in fp16 214 and in fp32 331).  Rows
// of 999: fp16 2.8, fp32 3.8 TB/s.
template <class T, int HELD>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* X, int64_t ldX, int64_t rows, int64_t d, int8_t* Q, int64_t ldQ,
                                                            float* scale) {
  chain_begin();
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  for (int64_t r = (int64_t)blockIdx.x * warps + (threadIdx.x >> 5); r < rows; r += (int64_t)gridDim.x * warps) {
    const T* src = X + r * ldX;
    int8_t* dst = Q + r * ldQ;
    float s;
    if constexpr (HELD > 0) {
      s = quantize_row<HELD>(src, (int)(d / 8), lane, [&](int v, uint2 w) { reinterpret_cast<uint2*>(dst)[v] = w; });
    } else {
      uint32_t m = 0;
      for (int64_t k = lane; k < d; k += 32) m = max(m, __float_as_uint((float)src[k]) & 0x7fffffffu);
      const RowScale c = row_scale(warp_max(m));
      for (int64_t k = lane; k < d; k += 32) dst[k] = (int8_t)pack4(c, (float)src[k], 0.f, 0.f, 0.f);   // what lies behind the row stays
      s = c.s;
    }
    if (lane == 0) scale[r] = s;
  }
}

// ---------------------------------------------------------------------------------------------
// Scales of a warp's columns.  Lane i holds those of columns i of the warp's chunks of a tile, and of the unit's next tile, loaded before
// the accumulator is waited for: while the ring streams B, a load takes microseconds even where it hits L2 (a uniform load per four
// columns at each chunk made a 128 x 256 tile's epilogue 13 us).  Every chunk's 32 then go through shared memory to all lanes.
template <int W>
struct ColumnScales {
  static constexpr int kChunks = BN / 32 / (W / 4);
  float now[kChunks], ahead[kChunks];
  int tile_ahead;   // whose scales `ahead` has
  __device__ __forceinline__ void init() { tile_ahead = -1; }
  __device__ __forceinline__ void load(float (&x)[kChunks], const float* b, int V, int n_tile, int chunk0) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int col = n_tile * BN + (chunk0 + i) * 32 + lane;
      x[i] = col < V ? __ldg(b + col) : 0.f;
    }
  }
  __device__ __forceinline__ void begin_tile(const float* b, int V, int n_tile, int next, int chunk0) {
    if (tile_ahead == n_tile) {
#pragma unroll
      for (int i = 0; i < kChunks; ++i) now[i] = ahead[i];
    } else {
      load(now, b, V, n_tile, chunk0);
    }
    if (next >= 0) load(ahead, b, V, next, chunk0);
    tile_ahead = next;
  }
  // 32 integer sums of one row, whose scale is a -> logits; columns past V become 0.  Chunks come in order.
  __device__ __forceinline__ void apply(const float (&v)[32], float a, float (&z)[32]) {
    __shared__ __align__(16) float scale_s[W][32];
    const int lane = threadIdx.x & 31;
    float* mine = scale_s[(threadIdx.x >> 5) - 2];
    __syncwarp();   // the chunk before has been read
    mine[lane] = now[0];
    __syncwarp();
#pragma unroll
    for (int i = 0; i + 1 < kChunks; ++i) now[i] = now[i + 1];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float4 q = reinterpret_cast<const float4*>(mine)[j];
      z[4 * j] = (float)__float_as_int(v[4 * j]) * a * q.x;
      z[4 * j + 1] = (float)__float_as_int(v[4 * j + 1]) * a * q.y;
      z[4 * j + 2] = (float)__float_as_int(v[4 * j + 2]) * a * q.z;
      z[4 * j + 3] = (float)__float_as_int(v[4 * j + 3]) * a * q.w;
    }
  }
};

// Eight epilogue warps in place of four up to these widths: the products take half the time that bf16's do, so the epilogue shows to
// twice the width, less where it has a box to wait for.  8192 rows x 151936 words, four / eight, d = 512 / 1024 / 1536 / 2048 / 2560:
// statistics 1209 / 1454 / 1728 / 1900 / 2155 us, 953 / 1207 / 1456 / 1846 / 2255; bf16 logits 972 / 1277 / 1591 / 1910 / 2283 us, 856 / 1262 /
// 1682 / 2114 / 2486; fp32 logits 1211 / 1637 / 2113 / 2408 / 2835, 1080 / 1619 / 2087 / 2527 / 2966.  At d = 1024 eight take 1 to 5 % less time
// (on another box bf16 1226 / 1187, fp16 1348 / 1283, fp32 1673 / 1592): the line for logits lies on the safe side, below it.
constexpr int kEightWarpsStatsI8 = 2048;
constexpr int kEightWarpsScale = 768;
// Row by row (no TMA): 50257 words, four / eight warps, 2048 rows at d = 1024 bf16 136 / 135 us, fp16 137 / 135, fp32 163 / 182; 599 rows 80 / 66, 76 / 64,
// 77 / 77; 2048 rows at d = 2048 171 / 178, 182 / 194, 225 / 252.
template <int OUT>
constexpr int kWarpsByRow = OUT == 1 ? 4 : 8;

// Statistics of RowStats over those logits: scoring under a head held in 8 bits.
struct Int8StatsParams : RowStats::Params {
  const float* row_scale;   // compact rows
  const float* col_scale;   // [V]
};
template <int W>
struct EpiStatsI8 {
  static constexpr bool kParts = false;
  static constexpr int kSideWarps = 0;
  static constexpr bool kFeeds = false, kAhead = false, kInt8 = true;
  static constexpr int kStagingBytes = 0;
  static constexpr int kWarps = W;
  using Params = Int8StatsParams;
  struct State : RowStats::State {
    float scale;
    ColumnScales<W> cols;
  };
  __device__ static __forceinline__ void init(State& st) { st.cols.init(); }
  __device__ static __forceinline__ void finish(State&) {}
  __device__ static __forceinline__ void begin_tile(const Params& p, State& st, int n_tile, int next, int chunk0) {
    st.cols.begin_tile(p.col_scale, p.V, n_tile, next, chunk0);
  }
  __device__ static __forceinline__ void begin_unit(const Params& p, State& st, int m_tile, int nr, int row_in_tile, int m_rows,
                                                    int slab_off, int ks) {
    RowStats::begin_unit(p, st, m_tile, nr, row_in_tile, m_rows, slab_off, ks);
    const int row = m_tile * BM + row_in_tile;
    st.scale = row < m_rows ? p.row_scale[row] : 0.f;
  }
  __device__ static __forceinline__ void chunk(const Params& p, State& st, int m_tile, int n_tile, int c, int row_in_tile, int m_rows,
                                               const float (&v)[32], const CUtensorMap* map, uint32_t staging) {
    float z[32];
    st.cols.apply(v, st.scale, z);
    RowStats::chunk(p, st, m_tile, n_tile, c, row_in_tile, m_rows, z, map, staging);
  }
  static constexpr int kMerge = RowStats::kMerge;
  __device__ static __forceinline__ void pack(const State& st, float (&x)[kMerge]) { RowStats::pack(st, x); }
  __device__ static __forceinline__ void merge(State& st, const float (&x)[kMerge]) { RowStats::merge(st, x); }
  __device__ static __forceinline__ void end_unit(const Params& p, State& st, int m_tile, int nr, int row_in_tile, int m_rows) {
    RowStats::end_unit(p, st, m_tile, nr, row_in_tile, m_rows);
  }
};

// The logits themselves.  OUT as in the ABI (0 bf16, 1 fp32, 2 fp16).  TMA: C's rows start and end on 16 bytes and boxes go through the
// TMA unit, which clips them at the edges; else each warp writes its 32 x 32 values row by row.
enum OutType { kOutBf16 = 0, kOutF32 = 1, kOutF16 = 2 };
template <int OUT>
__device__ __forceinline__ uint32_t two_halves(float a, float b) {
  if constexpr (OUT == kOutF16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}
template <int OUT>
__device__ __forceinline__ void store_one(void* C, size_t at, float x) {
  if constexpr (OUT == kOutF32) static_cast<float*>(C)[at] = x;
  else if constexpr (OUT == kOutF16) static_cast<__half*>(C)[at] = __float2half_rn(x);
  else static_cast<__nv_bfloat16*>(C)[at] = __float2bfloat16_rn(x);
}
struct ScaleParams {
  const float* row_scale;
  const float* col_scale;
  int V;
  void* C;                  // not TMA
  long long ldC;
};
template <int OUT, bool TMA, int W>
struct EpiScale {
  static constexpr bool kParts = false;
  static constexpr int kSideWarps = 0;
  static constexpr bool kFeeds = false, kAhead = false, kInt8 = true;
  static constexpr int kWarps = W;
  static constexpr int kMerge = 0;
  static constexpr int kStagingBytes = kEpiStaging;
  using Params = ScaleParams;
  struct State {
    float scale;
    uint32_t n_issued;
    ColumnScales<W> cols;
  };
  __device__ static __forceinline__ void init(State& st) {
    st.n_issued = 0;
    st.cols.init();
  }
  __device__ static __forceinline__ void begin_tile(const Params& p, State& st, int n_tile, int next, int chunk0) {
    st.cols.begin_tile(p.col_scale, p.V, n_tile, next, chunk0);
  }
  __device__ static __forceinline__ void finish(State& st) {
    if ((threadIdx.x & 31) == 0 && st.n_issued) bulk_wait_group_all();
    __syncwarp();
  }
  __device__ static __forceinline__ void begin_unit(const Params& p, State& st, int m_tile, int, int row_in_tile, int m_rows, int, int) {
    const int row = m_tile * BM + row_in_tile;
    st.scale = row < m_rows ? p.row_scale[row] : 0.f;
  }
  __device__ static __forceinline__ void chunk(const Params& p, State& st, int m_tile, int n_tile, int c, int row_in_tile, int m_rows,
                                               const float (&v)[32], const CUtensorMap* map, uint32_t staging) {
    const int lane = threadIdx.x & 31;
    const int row0 = m_tile * BM + (row_in_tile - lane), col0 = n_tile * BN + c * 32;
    constexpr bool kPairs = TMA && OUT != kOutF32;   // a box holds two chunks: its second half may lie past V, and is clipped
    if (row0 >= m_rows || (kPairs ? col0 & ~63 : col0) >= p.V) return;   // warp-uniform
    float z[32];
    st.cols.apply(v, st.scale, z);
    constexpr int kBufs = kStagingBytes / kWarps / kBoxBytes;
    if constexpr (kPairs) {
      uint32_t w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = two_halves<OUT>(z[2 * i], z[2 * i + 1]);
      stage_half_box<kBufs>(w, c, staging, st.n_issued, map, col0, row0);
    } else {
      const uint32_t buf = staging + (TMA ? st.n_issued % kBufs : 0) * kBoxBytes;
      if (TMA && lane == 0) bulk_wait_group_read<kBufs - 1>();
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t addr = buf + lane * 128u + (uint32_t((j ^ (lane & 7)) << 4));
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(z[4 * j]), "f"(z[4 * j + 1]), "f"(z[4 * j + 2]),
                     "f"(z[4 * j + 3])
                     : "memory");
      }
      if constexpr (TMA) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          tma_store_3d(map, buf, col0, row0, 0);
          bulk_commit_group();
        }
        st.n_issued++;
      } else {
        __syncwarp();
        const int rows = min(32, m_rows - row0);
        if (col0 + lane < p.V) {
          size_t at = (size_t)row0 * p.ldC + col0 + lane;
          auto value = [&](int r) {
            float x;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(buf + r * 128u + ((uint32_t(lane >> 2) ^ uint32_t(r & 7)) << 4) + (lane & 3) * 4u) : "memory");
            return x;
          };
          if (rows == 32) {
            // sixteen loads on their way at a time, no row asked for: 2048 rows x 27931 words, d = 416 80 us asking for each, 78 so; 599 rows 33.5, 28.9
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += 16) {
              float x[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) x[i] = value(r0 + i);
#pragma unroll
              for (int i = 0; i < 16; ++i, at += p.ldC) store_one<OUT>(p.C, at, x[i]);
            }
          } else {
            for (int r0 = 0; r0 < rows; r0 += 8) {
              float x[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) x[i] = value(r0 + i);
#pragma unroll
              for (int i = 0; i < 8; ++i, at += p.ldC)
                if (r0 + i < rows) store_one<OUT>(p.C, at, x[i]);
            }
          }
        }
        __syncwarp();   // before the next chunk takes the buffer
      }
    }
  }
  __device__ static __forceinline__ void end_unit(const Params&, State&, int, int, int, int) {}
};

// ---------------------------------------------------------------------------------------------
// Up to N tokens (at most 128) as a stream of B on the tensor cores, the operands' roles exchanged: 128 rows of B are the M side of a tile, the tokens
// its N side.  All of the tokens lie in shared memory for the whole kernel.  (As the M side of the engine's tiles they were read again
// for every tile by every CTA, which made the L2 slices of a few lines the bottleneck: 9 to 32 tokens took 110 to 140 us at
// d = 3584 and 152 K rows, 40 to 128 took 97 to 101; a dp4a kernel took 95 us for one token and 139 for eight.)  Every CTA takes an equal share of the rows in tiles of `rows`.
//   warp 0: TMA producer;  warp 1: allocates tensor memory, issues the products;  warps 2 to 9: a thread per row of B and half of the tokens.
constexpr int kStreamStageBytes = 128 * 128;   // 128 rows, a k-block of 128 bytes
constexpr int kStreamMaxStages = 12;
constexpr int kStreamSmem = 224 * 1024;        // of it 1 KB to start on a multiple of 1024
constexpr int kStreamThreads = 64 + 8 * 32;
// Stages that fit beside the tokens.
__host__ __device__ constexpr int stream_stages(int n_tokens, int k_blocks) {
  const long long left = kStreamSmem - 1024 - (long long)n_tokens * 128 * k_blocks;
  const long long s = left < 0 ? 0 : left / kStreamStageBytes;
  return (int)(s < kStreamMaxStages ? s : kStreamMaxStages);
}
// Fewer stages than these and the engine's tiles are faster.  151936 rows, 65 / 96 tokens, stream / engine: d = 448 17.1 / 17.9 us, 20.9 / 22.9; d = 1024
// 32.3 / 34.0, 37.2 / 37.5; d = 1280 (six stages) 39.2 / 41.3, 46.7 / 43.8; d = 1664 (four) 54.0 / 55.8, 60.6 / 53.8.  128 tokens: d = 448 21.2, 23.6;
// d = 1024 36.9, 38.9; d = 1152 (four) 43.0, 43.2.  64 tokens at d = 2560 (three) 83, 73-88; 48 at d = 2560 (six) 69, 88.
constexpr int stream_min_stages(int n_tokens) { return n_tokens > 64 ? 5 : 4; }
// Up to kStreamOwn tokens in bf16 the kernel quantises itself, in four warps more and before these eight turn to their rows, while the ring
// fills: a launch less.  1 / 4 / 8 / 13 / 16 tokens, 151936 rows, d = 2048 52.8 / 54.3 / 55.5 / 55.8 / 56.0 us with the launch, 50.0 / 51.7 / 52.7 / 53.1 /
// 53.6 without; d = 3584 88.0 / 90.5 / 92.4 / 93.4 / 93.5, 83.3 / 85.3 / 86.4 / 88.6 / 89.4.
constexpr int kStreamOwn = 16, kStreamOwnWarps = 4;
struct StreamParams {
  const __nv_bfloat16* X;   // OWN: the tokens, d a multiple of 8, rows 16-byte aligned
  long long ldX;
  int d;
  const float* a_scale;
  const float* b_scale;
  int T, V, k_blocks, rows, stages;   // rows of B per tile, at most 128
  void* C;
  long long ldC;
};
// What both kernels of the stream share: barriers, the producer, the issuer of the products.
struct StreamBars {
  uint64_t full[kStreamMaxStages], empty[kStreamMaxStages], acc_full[2], acc_empty[2], tokens, drain;
  uint32_t tmem_base;
  int abort_flag;
};
template <int N>
constexpr uint32_t kStreamCols = 2 * N <= 32 ? 32 : 2 * N <= 64 ? 64 : 2 * N <= 128 ? 128 : 256;   // two accumulators; a power of two from 32 on
// Before the launch's memory is touched.  acc_warps: warps that read an accumulator; token_arrivals: on the barrier of the tokens.
template <int N>
__device__ __forceinline__ void stream_begin(StreamBars& s, const CUtensorMap* tmTokens, const CUtensorMap* tmRows, int acc_warps, int token_arrivals) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStreamMaxStages; ++i) { mbar_init(smem_u32(&s.full[i]), 1); mbar_init(smem_u32(&s.empty[i]), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(smem_u32(&s.acc_full[a]), 1); mbar_init(smem_u32(&s.acc_empty[a]), acc_warps); }
    mbar_init(smem_u32(&s.tokens), token_arrivals);
    mbar_init(smem_u32(&s.drain), 1);
    s.abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(tmTokens);
    prefetch_tmap(tmRows);
  }
  if (threadIdx.x >> 5 == 1) {
    tmem_alloc(smem_u32(&s.tmem_base), kStreamCols<N>);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  chain_wait();
}
template <int N>
__device__ __forceinline__ void stream_end(StreamBars& s) {
  chain_release();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x >> 5 == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(s.tmem_base, kStreamCols<N>);
  }
}
// One thread.  tmTokens NULL: others put the tokens where they belong.
template <int N>
__device__ __forceinline__ void stream_produce(StreamBars& s, const CUtensorMap* tmTokens, const CUtensorMap* tmRows, const StreamParams& p, uint32_t tokens,
                                               uint32_t ring, int r0, int tiles, DevStatus* status) {
  const uint32_t tok_bar = smem_u32(&s.tokens);
  if (tmTokens) {
    mbar_arrive_expect_tx(tok_bar, (uint32_t)p.k_blocks * N * 128u);
    for (int kb = 0; kb < p.k_blocks; ++kb) tma_load_2d(tokens + (uint32_t)kb * N * 128u, tmTokens, tok_bar, kb * 128, 0);
  }
  int stage = 0;
  uint32_t phase = 0;
  bool ok = true;
  for (int t = 0; t < tiles && ok; ++t) {
    for (int kb = 0; kb < p.k_blocks; ++kb) {
      if (!mbar_wait_bounded(smem_u32(&s.empty[stage]), phase ^ 1u, &s.abort_flag)) {
        latch_status(status, kStatusTimeout, (1 << 28) | (blockIdx.x << 8) | stage);
        ok = false;
        break;
      }
      const uint32_t full = smem_u32(&s.full[stage]);
      mbar_arrive_expect_tx(full, (uint32_t)p.rows * 128u);
      tma_load_2d(ring + (uint32_t)stage * kStreamStageBytes, tmRows, full, kb * 128, r0 + t * p.rows);
      if (++stage == p.stages) { stage = 0; phase ^= 1u; }
    }
  }
  if (!ok) {
    // copies already issued land before the block's shared memory goes away
    for (int i = 0; i < p.stages; ++i) {
      const uint32_t ph = i < stage ? phase : (phase ^ 1u);
      for (int it = 0; it < 4096 && !mbar_try_wait(smem_u32(&s.full[i]), ph); ++it) {}
    }
    for (int it = 0; tmTokens && it < 4096 && !mbar_try_wait(tok_bar, 0); ++it) {}
  }
}
// One thread.
template <int N>
__device__ __forceinline__ void stream_multiply(StreamBars& s, const StreamParams& p, uint32_t tokens, uint32_t ring, int tiles, DevStatus* status) {
  constexpr uint32_t idesc = make_idesc_s8(128, N);
  constexpr uint64_t hi = make_smem_desc_hi(16, 1024);
  constexpr uint32_t hi32 = uint32_t(hi >> 32), lo_const = uint32_t(hi);
  const uint32_t ring_lo = (ring & 0x3FFFFu) >> 4, tok_lo = (tokens & 0x3FFFFu) >> 4, tmem_base = s.tmem_base;
  int stage = 0;
  uint32_t phase = 0;
  bool ok = tiles == 0 || mbar_wait_bounded(smem_u32(&s.tokens), 0, &s.abort_flag);
  if (!ok) latch_status(status, kStatusTimeout, (3 << 28) | (blockIdx.x << 8) | 0xff);
  for (int t = 0; t < tiles && ok; ++t) {
    const uint32_t a = t & 1u;
    if (!mbar_wait_bounded(smem_u32(&s.acc_empty[a]), ((t >> 1) & 1u) ^ 1u, &s.abort_flag)) {
      latch_status(status, kStatusTimeout, (2 << 28) | (blockIdx.x << 8) | a);
      ok = false;
      break;
    }
    tc_fence_after();
    for (int kb = 0; kb < p.k_blocks; ++kb) {
      if (!mbar_wait_bounded(smem_u32(&s.full[stage]), phase, &s.abort_flag)) {
        latch_status(status, kStatusTimeout, (3 << 28) | (blockIdx.x << 8) | stage);
        ok = false;
        break;
      }
      tc_fence_after();
      const uint32_t w = lo_const | (ring_lo + (uint32_t)stage * (kStreamStageBytes >> 4)), x = lo_const | (tok_lo + (uint32_t)kb * (N * 128 >> 4));
#pragma unroll
      for (int k = 0; k < 4; ++k) umma_i8_words<1>(tmem_base + a * N, w + 2 * k, hi32, x + 2 * k, hi32, idesc, (kb > 0 || k > 0) ? 1u : 0u);
      umma_commit(smem_u32(&s.empty[stage]));
      if (++stage == p.stages) { stage = 0; phase ^= 1u; }
    }
    if (ok) umma_commit(smem_u32(&s.acc_full[a]));
  }
  umma_commit(smem_u32(&s.drain));
  bool drained = false;
  for (int it = 0; it < (1 << 22) && !drained; ++it) drained = mbar_try_wait(smem_u32(&s.drain), 0) != 0;
  if (!drained) latch_status(status, kStatusTimeout, (4 << 28) | (blockIdx.x << 8));
}
// The accumulators of this block's tiles, one after the other, by one warp: load(accumulator's address), which is then free for the next
// but one tile, and use(row of B or -1, its scale).  Scales of rows are loaded four tiles early: while the ring streams B such a load
// takes as long as a tile or two.
template <int N, class Load, class Use>
__device__ __forceinline__ void stream_consume(StreamBars& s, const StreamParams& p, int r0, int r1, int tiles, DevStatus* status, Load load, Use use) {
  const int q = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, at = q * 32 + lane;   // tensor-memory lanes 32 q and on are this warp's
  auto row_of = [&](int t) { const int r = r0 + t * p.rows + at; return t < tiles && at < p.rows && r < r1 ? r : -1; };
  auto scale_of = [&](int r) { return r >= 0 ? __ldg(p.b_scale + r) : 0.f; };
  constexpr int kAhead = 4;
  float b[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) b[u] = scale_of(row_of(u));
  bool ok = true;
  for (int t0 = 0; t0 < tiles && ok; t0 += kAhead) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int t = t0 + u;
      if (t >= tiles) break;
      const uint32_t a = u & 1u;
      if (!mbar_wait_bounded(smem_u32(&s.acc_full[a]), (t >> 1) & 1u, &s.abort_flag)) {
        latch_status(status, kStatusTimeout, (5 << 28) | (blockIdx.x << 8) | a);
        ok = false;
      }
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      load(s.tmem_base + a * N + (uint32_t(q * 32) << 16));
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&s.acc_empty[a]));
      use(row_of(t), b[u]);
      b[u] = scale_of(row_of(t + kAhead));
    }
  }
}

template <int N, int OUT, bool OWN = false>
__global__ void __launch_bounds__(kStreamThreads + (OWN ? 32 * kStreamOwnWarps : 0), 1)
int8_stream_kernel(const __grid_constant__ CUtensorMap tmTokens, const __grid_constant__ CUtensorMap tmRows, const StreamParams p, DevStatus* status) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) StreamBars bars;
  __shared__ float a_s[8][N / 2];   // a copy of its half per warp; OWN: the first two, of all
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t tokens = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t ring = tokens + (uint32_t)p.k_blocks * N * 128u;
  stream_begin<N>(bars, OWN ? &tmRows : &tmTokens, &tmRows, 8, OWN ? 8 + kStreamOwnWarps : 1);
  const int r0 = (int)((long long)p.V * blockIdx.x / gridDim.x), r1 = (int)((long long)p.V * (blockIdx.x + 1) / gridDim.x);
  const int tiles = (r1 - r0 + p.rows - 1) / p.rows;

  if (warp == 0) {
    if (lane == 0) stream_produce<N>(bars, OWN ? nullptr : &tmTokens, &tmRows, p, tokens, ring, r0, tiles, status);
  } else if (warp == 1) {
    if (lane == 0) stream_multiply<N>(bars, p, tokens, ring, tiles, status);
  } else {
    constexpr int kMine = N / 2;
    const int first = (warp - 2) / 4 * kMine;   // of this warp's tokens
    float* scales = a_s[OWN ? 0 : warp - 2];
    bool ok = true;
    if constexpr (OWN) {
      // rows of the swizzled operand: 128 bytes of a k-block, 16-byte chunk j of row t at position j ^ (t & 7).  What lies behind the
      // tokens, and behind d (where B reads as zeros), may hold anything
      for (int t = warp - 2; t < p.T; t += 8 + kStreamOwnWarps) {
        const float sc = quantize_row<16>(p.X + t * p.ldX, p.d / 8, lane, [&](int v, uint2 w) {
          const uint32_t to = tokens + (uint32_t)(v >> 4) * (N * 128u) + t * 128u + ((uint32_t(v >> 1 & 7) ^ uint32_t(t & 7)) << 4) + (v & 1) * 8u;
          asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(w.x), "r"(w.y) : "memory");
        });
        if (lane == 0) scales[t] = sc;
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.tokens));
      if (warp < 10) {
        ok = mbar_wait_bounded(smem_u32(&bars.tokens), 0, &bars.abort_flag);   // every lane: the scales are then visible to it
        ok = __all_sync(0xffffffffu, ok);
      }
      scales += first;
    } else {
      for (int t = lane; t < kMine; t += 32) scales[t] = first + t < p.T ? p.a_scale[first + t] : 0.f;
      __syncwarp();
    }
    if (warp < 10 && ok && first < p.T) {
      uint32_t x[kMine / 8][8];
      stream_consume<N>(bars, p, r0, r1, tiles, status,
        [&](uint32_t taddr) {
#pragma unroll
          for (int c = 0; c < kMine / 8; ++c) tmem_ld_32x8(taddr + first + c * 8, x[c]);
        },
        [&](int r, float b) {
          if (r < 0) return;
          size_t out = (size_t)r + (size_t)first * p.ldC;
#pragma unroll
          for (int c = 0; c < kMine / 8; ++c) {
            const int left = p.T - first - c * 8;   // of the tokens
            if (left <= 0) break;
            float z[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = (float)(int)x[c][i] * scales[c * 8 + i] * b;
            if (left >= 8) {
#pragma unroll
              for (int i = 0; i < 8; ++i, out += p.ldC) store_one<OUT>(p.C, out, z[i]);
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i, out += p.ldC)
                if (i < left) store_one<OUT>(p.C, out, z[i]);
            }
          }
        });
    } else if (warp < 10 && ok) {
      stream_consume<N>(bars, p, r0, r1, tiles, status, [](uint32_t) {}, [](int, float) {});   // no token is this warp's
    }
  }
  stream_end<N>(bars);
}

// Statistics of RowStats over the same logits: scoring of up to N tokens.  Eight warps, two per 32 rows of B with half of the tokens
// each; a thread keeps maximum, sum and weighted sum of every token over its own rows of all tiles, so that a logit costs one
// exponential and no exchange; the threads' numbers are merged once, at the end, in a fixed order.  One float4 per (block, token).
// For kStreamScores tokens: a call with this / with the engine's statistics, 151936 rows, d = 256 / 1024 / 2048: 1 token 18.5 / 39.6 / 60.7 us, 30.5 /
// 45.0 / 68.4; 32 tokens 21.1 / 38.8 / 61.4, 28.9 / 42.3 / 65.3; but 48 tokens 26.7 / 47.3 / 67.5, 28.9 / 42.0 / 65.2, and 64 slower throughout.
constexpr int kStreamScores = 32;
template <int N>
__global__ void __launch_bounds__(kStreamThreads, 1)
int8_stream_stats_kernel(const __grid_constant__ CUtensorMap tmTokens, const __grid_constant__ CUtensorMap tmRows, const StreamParams p,
                         const int* tokens_c, float4* partials, int part_stride, DevStatus* status) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) StreamBars bars;
  constexpr int kMine = N / 2;
  __shared__ float a_s[N], zy_s[N];
  __shared__ int y_s[N];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t tokens = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t ring = tokens + (uint32_t)p.k_blocks * N * 128u;
  // [4][N] in the tokens' place: a warp that is through its last tile knows that every product has read them
  float4* part_s = reinterpret_cast<float4*>(smem_raw + (tokens - smem_u32(smem_raw)));
  static_assert(4 * sizeof(float4) <= 128, "four per token, where a token has 128 bytes at least");
  stream_begin<N>(bars, &tmTokens, &tmRows, 8, 1);
  const int n = min(status->n_valid, N);
  const int r0 = (int)((long long)p.V * blockIdx.x / gridDim.x), r1 = (int)((long long)p.V * (blockIdx.x + 1) / gridDim.x);
  const int tiles = n > 0 ? (r1 - r0 + p.rows - 1) / p.rows : 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) status->n_ranges = gridDim.x;
  for (int t = threadIdx.x; t < N; t += kStreamThreads) {
    a_s[t] = t < n ? p.a_scale[t] : 0.f;
    y_s[t] = t < n ? tokens_c[t] : -1;
    zy_s[t] = 0.f;
  }
  __syncthreads();

  if (warp == 0) {
    if (lane == 0 && tiles > 0) stream_produce<N>(bars, &tmTokens, &tmRows, p, tokens, ring, r0, tiles, status);
  } else if (warp == 1) {
    if (lane == 0) stream_multiply<N>(bars, p, tokens, ring, tiles, status);
  } else {
    const int first = (warp - 2) / 4 * kMine;   // first of this warp's tokens
    float m[kMine], s[kMine], a[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) { m[i] = -CUDART_INF_F; s[i] = a[i] = 0.f; }
    uint32_t x[kMine / 8][8];
    stream_consume<N>(bars, p, r0, r1, tiles, status,
      [&](uint32_t taddr) {
#pragma unroll
        for (int c = 0; c < kMine / 8; ++c) tmem_ld_32x8(taddr + first + c * 8, x[c]);
      },
      [&](int r, float b) {
        if (r < 0) return;
#pragma unroll
        for (int t = 0; t < kMine; ++t) {
          const float z = (float)(int)x[t / 8][t % 8] * a_s[first + t] * b;
          if (r == y_s[first + t]) zy_s[first + t] = z;
          // the smaller of the two exponents is 0
          const float d = z - m[t], e = ex2_approx(-fabsf(d) * kLog2e);
          const bool up = d > 0.f;
          s[t] = up ? fmaf(s[t], e, 1.f) : s[t] + e;
          a[t] = up ? fmaf(a[t], e, z) : fmaf(e, z, a[t]);
          m[t] = fmaxf(m[t], z);
        }
      });
    // over the warp's rows; a thread without a row has m = -inf and sums of 0
#pragma unroll
    for (int t = 0; t < kMine; ++t) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m[t], o), s2 = __shfl_xor_sync(0xffffffffu, s[t], o), a2 = __shfl_xor_sync(0xffffffffu, a[t], o);
        const float mx = fmaxf(m[t], m2);
        const float f = m[t] == mx ? 1.f : ex2_approx((m[t] - mx) * kLog2e), f2 = m2 == mx ? 1.f : ex2_approx((m2 - mx) * kLog2e);
        s[t] = s[t] * f + s2 * f2;
        a[t] = a[t] * f + a2 * f2;
        m[t] = mx;
      }
      if (lane == 0) part_s[(warp & 3) * N + first + t] = make_float4(m[t], s[t], a[t], 0.f);
    }
  }
  __syncthreads();
  for (int t = threadIdx.x; t < n; t += kStreamThreads) {
    float4 x = part_s[t];
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      const float4 y = part_s[w * N + t];
      const float mx = fmaxf(x.x, y.x);
      const float f = x.x == mx ? 1.f : ex2_approx((x.x - mx) * kLog2e), f2 = y.x == mx ? 1.f : ex2_approx((y.x - mx) * kLog2e);
      x = make_float4(mx, x.y * f + y.y * f2, x.z * f + y.z * f2, 0.f);
    }
    x.w = zy_s[t];
    partials[(size_t)blockIdx.x * part_stride + t] = x;
  }
  stream_end<N>(bars);
}

// Merge of a few rows' statistics, a warp per row: all its column ranges are on their way at once, in the lanes, and added up over them in
// a fixed order.  (combine_loss_kernel, which also knows losses, takes a block per 32 rows and loads a few
// ranges at a time.)
struct ScoreParams {
  const float4* partials;
  int part_stride;
  const int* row_map;
  float *logp, *entropy, *lse;   // [T]; the latter two may be NULL
};
__global__ void __launch_bounds__(256) merge_scores_kernel(const ScoreParams p, const DevStatus* st) {
  chain_begin();
  const int n = st->n_valid, n_ranges = st->n_ranges, lane = threadIdx.x & 31;
  for (int i = blockIdx.x * 8 + (threadIdx.x >> 5); i < n; i += gridDim.x * 8) {
    const int row = p.row_map[i];
    float M = -CUDART_INF_F, S = 0.f, A = 0.f, zy = 0.f;
    auto add = [&](float m2, float s2, float a2) {
      const float m = fmaxf(M, m2);
      const float f = M == m ? 1.f : exp2f((M - m) * kLog2e), f2 = m2 == m ? 1.f : exp2f((m2 - m) * kLog2e);   // (-inf: nothing there)
      S = S * f + s2 * f2;
      A = A * f + a2 * f2;
      M = m;
    };
    for (int r0 = 0; r0 < n_ranges; r0 += 128) {
      float4 q[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = r0 + k * 32 + lane;
        q[k] = r < n_ranges ? p.partials[(size_t)r * p.part_stride + i] : make_float4(-CUDART_INF_F, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        add(q[k].x, q[k].y, q[k].z);
        zy += q[k].w;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float m2 = __shfl_xor_sync(0xffffffffu, M, o), s2 = __shfl_xor_sync(0xffffffffu, S, o), a2 = __shfl_xor_sync(0xffffffffu, A, o);
      zy += __shfl_xor_sync(0xffffffffu, zy, o);
      add(m2, s2, a2);
    }
    if (lane == 0) {
      const float lse = M + logf(S);
      p.logp[row] = zy - lse;
      if (p.entropy) p.entropy[row] = lse - A / S;
      if (p.lse) p.lse[row] = lse;
    }
  }
}

}  // namespace rlh
