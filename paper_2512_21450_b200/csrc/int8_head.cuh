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
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// Eight bf16 values to eight bytes.
__device__ __forceinline__ uint2 pack8_bf16(const RowScale& c, const uint4& v) {
  return make_uint2(pack4(c, bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)),
                    pack4(c, bf16_lo(v.z), bf16_hi(v.z), bf16_lo(v.w), bf16_hi(v.w)));
}
__device__ __forceinline__ uint32_t most_bf16(const uint4& v) {   // two maxima, as 16-bit words
  constexpr uint32_t k = 0x7fff7fffu;
  return __vmaxu2(__vmaxu2(v.x & k, v.y & k), __vmaxu2(v.z & k, v.w & k));
}
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
// One bf16 row of d elements (a multiple of 8, 16-byte aligned) by one warp; what does not fit kHeld words per lane is read twice.
__device__ __forceinline__ float quantize_row_bf16(const uint4* src, int vecs, uint2* dst, int lane) {
  constexpr int kHeld = 8;
  uint4 h[kHeld];
  uint32_t m2 = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    h[i] = lane + 32 * i < vecs ? __ldg(src + lane + 32 * i) : make_uint4(0, 0, 0, 0);
    m2 = __vmaxu2(m2, most_bf16(h[i]));
  }
  for (int v = lane + 32 * kHeld; v < vecs; v += 32) m2 = __vmaxu2(m2, most_bf16(__ldg(src + v)));
  const RowScale c = row_scale(warp_max(max(m2 & 0xffffu, m2 >> 16)) << 16);
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (lane + 32 * i < vecs) dst[lane + 32 * i] = pack8_bf16(c, h[i]);
  for (int v = lane + 32 * kHeld; v < vecs; v += 32) dst[v] = pack8_bf16(c, __ldg(src + v));
  return c.s;
}

// Any rows: a warp per row, eight elements per lane and step.  VEC: rows start on 16 bytes; else, and at a row's ragged end, one
// element after the other.
template <class T>
__device__ __forceinline__ float as_float(T x) {
  if constexpr (sizeof(T) == 4) return x;
  else return (float)x;
}
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int64_t k, int64_t d, float (&x)[8]) {
  if (VEC && k + 8 <= d) {
    if constexpr (sizeof(T) == 4) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(row + k)), b = __ldg(reinterpret_cast<const float4*>(row + k) + 1);
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(row + k));
      const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = as_float(e[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = k + i < d ? as_float(row[k + i]) : 0.f;
  }
}
template <class T, bool VEC>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* X, int64_t ldX, int64_t rows, int64_t d, int8_t* Q, int64_t ldQ,
                                                            float* scale) {
  chain_begin();
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  for (int64_t r = (int64_t)blockIdx.x * warps + (threadIdx.x >> 5); r < rows; r += (int64_t)gridDim.x * warps) {
    const T* src = X + r * ldX;
    int8_t* dst = Q + r * ldQ;
    if constexpr (VEC && std::is_same<T, __nv_bfloat16>::value) {
      if (d % 8 == 0) {
        const float s = quantize_row_bf16(reinterpret_cast<const uint4*>(src), (int)(d / 8), reinterpret_cast<uint2*>(dst), lane);
        if (lane == 0) scale[r] = s;
        continue;
      }
    }
    uint32_t m = 0;
    for (int64_t k = lane * 8; k < d; k += 256) {
      float x[8];
      load8<T, VEC>(src, k, d, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    }
    const RowScale c = row_scale(warp_max(m));
    for (int64_t k = lane * 8; k < d; k += 256) {
      float x[8];
      load8<T, VEC>(src, k, d, x);
      const uint2 w = make_uint2(pack4(c, x[0], x[1], x[2], x[3]), pack4(c, x[4], x[5], x[6], x[7]));
      if (k + 8 <= d) {
        *reinterpret_cast<uint2*>(dst + k) = w;
      } else {
        for (int i = 0; k + i < d; ++i) dst[k + i] = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));   // what lies behind the row stays
      }
    }
    if (lane == 0) scale[r] = c.s;
  }
}

// ---------------------------------------------------------------------------------------------
// 32 integer sums of one row -> logits.  b: scales of columns from col0 on, 16-byte aligned at multiples of 4.
__device__ __forceinline__ void scale_chunk(const float (&v)[32], float a, const float* b, int nvalid, float (&z)[32]) {
  if (nvalid >= 32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float4 q = __ldg(reinterpret_cast<const float4*>(b) + j);
      z[4 * j] = (float)__float_as_int(v[4 * j]) * a * q.x;
      z[4 * j + 1] = (float)__float_as_int(v[4 * j + 1]) * a * q.y;
      z[4 * j + 2] = (float)__float_as_int(v[4 * j + 2]) * a * q.z;
      z[4 * j + 3] = (float)__float_as_int(v[4 * j + 3]) * a * q.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) z[i] = i < nvalid ? (float)__float_as_int(v[i]) * a * __ldg(b + i) : 0.f;
  }
}

// Statistics of RowStats over those logits: scoring under a head held in 8 bits.
struct Int8StatsParams : RowStats::Params {
  const float* row_scale;   // compact rows
  const float* col_scale;   // [V], 16-byte aligned
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
  };
  __device__ static __forceinline__ void init(State&) {}
  __device__ static __forceinline__ void finish(State&) {}
  __device__ static __forceinline__ void begin_unit(const Params& p, State& st, int m_tile, int nr, int row_in_tile, int m_rows,
                                                    int slab_off, int ks) {
    RowStats::begin_unit(p, st, m_tile, nr, row_in_tile, m_rows, slab_off, ks);
    const int row = m_tile * BM + row_in_tile;
    st.scale = row < m_rows ? p.row_scale[row] : 0.f;
  }
  __device__ static __forceinline__ void chunk(const Params& p, State& st, int m_tile, int n_tile, int c, int row_in_tile, int m_rows,
                                               const float (&v)[32], const CUtensorMap* map, uint32_t staging) {
    const int col0 = n_tile * BN + c * 32;
    if (col0 >= p.V) return;
    float z[32];
    scale_chunk(v, st.scale, p.col_scale + col0, p.V - col0, z);
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
  const float* col_scale;   // 16-byte aligned
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
  };
  __device__ static __forceinline__ void init(State& st) { st.n_issued = 0; }
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
    scale_chunk(v, st.scale, p.col_scale + col0, p.V - col0, z);
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
          for (int r = 0; r < rows; ++r, at += p.ldC) {
            float x;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(buf + r * 128u + ((uint32_t(lane >> 2) ^ uint32_t(r & 7)) << 4) + (lane & 3) * 4u) : "memory");
            store_one<OUT>(p.C, at, x);
          }
        }
        __syncwarp();   // before the next chunk takes the buffer
      }
    }
  }
  __device__ static __forceinline__ void end_unit(const Params&, State&, int, int, int, int) {}
};

// ---------------------------------------------------------------------------------------------
// A few tokens: a stream of B.  A warp takes kRows rows of B at a time, 16 bytes of each per lane and step, and multiplies them with the
// tokens, which lie in shared memory; the sums over the lanes are formed by halving, so that every lane ends up with one of them.
constexpr int kFewTokens = 8;
constexpr int kFewSmem = 64 * 1024;
struct FewParams {
  const int8_t* A;
  const float* a_scale;
  const int8_t* B;
  const float* b_scale;
  long long ldA, ldB, ldC;
  int T, d, V, out;
  void* C;
};
__device__ __forceinline__ int dot16(const uint4& a, const uint4& b, int acc) {
  acc = __dp4a((int)a.x, (int)b.x, acc);
  acc = __dp4a((int)a.y, (int)b.y, acc);
  acc = __dp4a((int)a.z, (int)b.z, acc);
  return __dp4a((int)a.w, (int)b.w, acc);
}
template <int T, int R>
__global__ void __launch_bounds__(512) int8_few_kernel(const FewParams p) {
  chain_begin();
  extern __shared__ __align__(16) uint8_t few_smem[];
  const int vecs = (p.d + 15) / 16;
  uint4* x_s = reinterpret_cast<uint4*>(few_smem);   // [T][vecs], zero past d and past the tokens there are
  for (int i = threadIdx.x; i < T * vecs; i += blockDim.x) {
    const int t = i / vecs, v = i - t * vecs;
    uint4 q = make_uint4(0, 0, 0, 0);
    if (t < p.T) {
      const int8_t* src = p.A + t * p.ldA + v * 16;
      if (v * 16 + 16 <= p.d) {
        q = *reinterpret_cast<const uint4*>(src);
      } else {
        uint32_t w[4] = {0, 0, 0, 0};
        for (int k = 0; v * 16 + k < p.d; ++k) w[k / 4] |= (uint32_t)(uint8_t)src[k] << (8 * (k & 3));
        q = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    x_s[i] = q;
  }
  __syncthreads();
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int groups = (p.V + R - 1) / R;
  for (int g = blockIdx.x * warps + (threadIdx.x >> 5); g < groups; g += gridDim.x * warps) {
    const int v0 = g * R;
    int n[R * T];   // sum of (row r, token t) at r * T + t
#pragma unroll
    for (int i = 0; i < R * T; ++i) n[i] = 0;
    const uint4* row[R];
#pragma unroll
    for (int r = 0; r < R; ++r) row[r] = reinterpret_cast<const uint4*>(p.B + (long long)min(v0 + r, p.V - 1) * p.ldB);
#pragma unroll 2
    for (int k = lane; k < vecs; k += 32) {
      uint4 w[R];
#pragma unroll
      for (int r = 0; r < R; ++r) w[r] = __ldcs(row[r] + k);
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const uint4 x = x_s[t * vecs + k];
#pragma unroll
        for (int r = 0; r < R; ++r) n[r * T + t] = dot16(w[r], x, n[r * T + t]);
      }
    }
    // halving: after the step over lanes `o` apart a lane keeps one half of the sums, the other half is its partner's
    constexpr int N = R * T;
    int left = N, first = 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      if (left > 1) {
        const int half = left / 2;
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
          if (i < half) {
            const int keep = up ? n[i + half] : n[i], give = up ? n[i] : n[i + half];
            n[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
          }
        first += up ? half : 0;
        left = half;
      } else {
        n[0] += __shfl_xor_sync(0xffffffffu, n[0], o);
      }
    }
    const int v = v0 + first / T, t = first % T;
    constexpr int kCopies = 32 / N;   // lanes that have the same sum
    if (lane % kCopies == 0 && v < p.V && t < p.T) {
      const float z = (float)n[0] * p.a_scale[t] * p.b_scale[v];
      const size_t at = (size_t)t * p.ldC + v;
      if (p.out == kOutF32) store_one<kOutF32>(p.C, at, z);
      else if (p.out == kOutF16) store_one<kOutF16>(p.C, at, z);
      else store_one<kOutBf16>(p.C, at, z);
    }
  }
}

}  // namespace rlh
