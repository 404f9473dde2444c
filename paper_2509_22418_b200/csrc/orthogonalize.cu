// Orthogonalised update of matrices: momentum, then products that bring every singular value to about one
// (a polynomial applied `steps` times, Newton-Schulz), on tcgen05 tensor cores:
//
//   m' = beta m + w G   u = nesterov ? w G + beta m' : m'   (without a momentum: u = G)
//   X = u / (|u|_F + eps);   steps times:  A = X X^T,  P = b A + c A A,  X = a X + P X;   O = scale X
//
// for matrices with more rows than columns A = X^T X and X = a X + X P, so that A and P are of the shorter side.
//
// Numbers.  The products' operands are fp16 (11 bits; bf16 has 8) times powers of two that keep |X| <= 2.8 below the
// largest and 2^-26 above the smallest normal number; sums are fp32.  X itself is carried as a pair of fp16 (22 bits), and
// a X is formed from the pair: rounding X leaves noise in directions whose singular values are small, and the polynomial multiplies
// those by a = 3.4 a step, noise included.  Root mean square error of O relative to O's (5 steps, CPU model): bf16
// operands and X 1e-2 for random matrices, 0.16 to 0.35 for those with a few large directions; fp16 operands and X 1.3e-3
// and 2e-2 to 4e-2; with the pair 1.4e-3 and 2e-4 to 5e-4.  P X needs no pair: b A + c A A is small where X is.
//
// A and A A are symmetric: tiles on and below the diagonal are worked and stored on both sides.
#include <algorithm>
#include <cmath>
#include <cuda_fp16.h>
#include "../../include/ppu.h"
#include "gemm_epilogue.cuh"

int ppu_fail(int code, const char* fmt, ...);

namespace {
using namespace tc;
using gemm_tc_detail::BK;
using gemm_tc_detail::UMMA_K;
using gemm_tc_detail::ld_v8;
using gemm_tc_detail::st_v8;

constexpr int X_EXP = 12, A_EXP = 12, LO_EXP = 11;      // powers of two: X, A as stored; the pair's second number over its first
constexpr int SMS = 148, MAX_STEPS = 32, MAX_SIDE = 1 << 16;
enum Mode { GRAM = 0, POLY = 1, UPDATE = 2 };

struct GemmP {
  int M, N, K, batch;
  int tiles_m, tiles_n, tiles;       // tiles of a matrix (on and below the diagonal where the product is symmetric)
  __half* C; int64_t ldc, stride;    // GRAM, POLY: the symmetric result
  const __half* A; float b, c;       // POLY: C = b A + c acc, factors with the powers of two
  const __half *hi; __half* lo;      // UPDATE: X as a pair (its second number is replaced in place)
  float a, f;                        // X' = a X + f acc
  __half* hi_out;                    // null: the last step, O = scale X'
  bf16* O; int64_t ldo; float scale;
  int* flags;
};

// ---- the tile kernel: one CTA, 128 x 128 ----------------------------------------------------------
constexpr int TM = 128, TN = 128, STAGES = 6, EPI = 8;
constexpr int A_BYTES = TM * BK * 2, STAGE_BYTES = A_BYTES + TN * BK * 2;
constexpr int SMEM = STAGES * STAGE_BYTES + 1024 + 256;

__device__ __forceinline__ uint32_t half2_bits(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 half2_floats(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }

// unit -> matrix and tile; symmetric products count (row, column <= row)
struct Place { int b, i, j; };
__device__ __forceinline__ Place place(int u, const GemmP& p, bool symmetric) {
  Place w;
  w.b = u / p.tiles;
  const int t = u - w.b * p.tiles;
  if (symmetric) {
    int i = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    while (i * (i + 1) / 2 > t) --i;
    w.i = i; w.j = t - i * (i + 1) / 2;
  } else {
    w.i = t % p.tiles_m; w.j = t / p.tiles_m;
  }
  return w;
}

// 32 columns from n on of row m (one to a lane)
template <int MODE>
__device__ __forceinline__ void finish(const GemmP& p, int b, int m, int n, bool mirror, const uint32_t* r) {
  if (m >= p.M) return;
  if constexpr (MODE != UPDATE) {
    __half* row = p.C + b * p.stride + m * p.ldc + n;
    uint32_t o[16];
    if (MODE == GRAM) {
#pragma unroll
      for (int j = 0; j < 16; ++j) o[j] = half2_bits(p.c * __uint_as_float(r[2 * j]), p.c * __uint_as_float(r[2 * j + 1]));
    } else {
      uint32_t x[16];
      const __half* src = p.A + b * p.stride + m * p.ldc + n;
      ld_v8(x, src); ld_v8(x + 8, src + 16);
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float2 v = half2_floats(x[j]);
        o[j] = half2_bits(fmaf(p.c, __uint_as_float(r[2 * j]), p.b * v.x), fmaf(p.c, __uint_as_float(r[2 * j + 1]), p.b * v.y));
      }
    }
    st_v8(row, o); st_v8(row + 16, o + 8);
    if (mirror) {
      __half* col = p.C + b * p.stride + m;
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (n + j < p.N) col[(int64_t)(n + j) * p.ldc] = __ushort_as_half((unsigned short)(o[j / 2] >> (16 * (j & 1))));
    }
  } else {
    const int64_t at = b * p.stride + m * p.ldc + n;
    uint32_t h[16], l[16];
    ld_v8(h, p.hi + at); ld_v8(h + 8, p.hi + at + 16);
    ld_v8(l, p.lo + at); ld_v8(l + 8, p.lo + at + 16);
    float y[32];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float2 a = half2_floats(h[j]), d = half2_floats(l[j]);
      constexpr float s = 1.f / (1 << LO_EXP);
      y[2 * j] = fmaf(p.f, __uint_as_float(r[2 * j]), p.a * fmaf(s, d.x, a.x));
      y[2 * j + 1] = fmaf(p.f, __uint_as_float(r[2 * j + 1]), p.a * fmaf(s, d.y, a.y));
    }
    if (p.hi_out) {
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        h[j] = half2_bits(y[2 * j], y[2 * j + 1]);
        const float2 a = half2_floats(h[j]);
        l[j] = half2_bits((y[2 * j] - a.x) * (1 << LO_EXP), (y[2 * j + 1] - a.y) * (1 << LO_EXP));
      }
      st_v8(p.hi_out + at, h); st_v8(p.hi_out + at + 16, h + 8);
      st_v8(p.lo + at, l); st_v8(p.lo + at + 16, l + 8);
    } else {
      bf16* o = p.O + ((int64_t)b * p.M + m) * p.ldo + n;
#pragma unroll
      for (int j = 0; j < 32; ++j) y[j] *= p.scale;
      if (p.N % 8 == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (n + 8 * j < p.N) *reinterpret_cast<uint4*>(o + 8 * j) = gemm_tc_detail::pack8_bf16(y + 8 * j);
      } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) if (n + j < p.N) o[j] = __float2bfloat16_rn(y[j]);
      }
    }
  }
}

template <bool A_K, bool B_K, int MODE>
__global__ void __launch_bounds__(64 + 32 * EPI, 1)
ortho_tile_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ GemmP p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + STAGES * STAGE_BYTES);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (STAGES + s); };
  auto tfull_bar = [&](int a) { return bar0 + 8u * (2 * STAGES + a); };
  auto tempty_bar = [&](int a) { return bar0 + 8u * (2 * STAGES + 2 + a); };
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), EPI); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), 2 * TN);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait(); pdl_trigger();

  const int units = p.tiles * p.batch, k_blocks = (p.K + BK - 1) / BK;
  if (warp == 0) {
    if (lane == 0) {
      // ---------------- TMA producer ----------------
      asm volatile("fence.proxy.async.global;" ::: "memory");      // (the operands were written by plain stores)
      int s = 0; uint32_t ph = 0;
      bool ok = true;
      for (int u = blockIdx.x; u < units && ok; u += gridDim.x) {
        const Place w = place(u, p, MODE != UPDATE);
        for (int kb = 0; kb < k_blocks; ++kb) {
          ok = mbar_wait(empty_bar(s), ph ^ 1u, abort_flag, p.flags);
          if (!ok) break;
          const uint32_t a_dst = smem_u32(smem + s * STAGE_BYTES), b_dst = a_dst + A_BYTES;
          mbar_expect_tx(full_bar(s), STAGE_BYTES);
          if (A_K) {
            tma_load_3d(a_dst, &mapA, full_bar(s), kb * BK, w.i * TM, w.b);
          } else {
#pragma unroll
            for (int j = 0; j < TM / 64; ++j) tma_load_3d(a_dst + j * 8192, &mapA, full_bar(s), w.i * TM + 64 * j, kb * BK, w.b);
          }
          if (B_K) {
            tma_load_3d(b_dst, &mapB, full_bar(s), kb * BK, w.j * TN, w.b);
          } else {
#pragma unroll
            for (int j = 0; j < TN / 64; ++j) tma_load_3d(b_dst + j * 8192, &mapB, full_bar(s), w.j * TN + 64 * j, kb * BK, w.b);
          }
          if (++s == STAGES) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      // ---------------- MMA issuer: D fp32, A and B fp16 ----------------
      const uint32_t idesc = (1u << 4) | ((A_K ? 0u : 1u) << 15) | ((B_K ? 0u : 1u) << 16) | ((uint32_t)(TN >> 3) << 17) | ((uint32_t)(TM >> 4) << 24);
      int s = 0; uint32_t ph = 0;
      int acc = 0; uint32_t acc_ph = 0;
      for (int u = blockIdx.x; u < units; u += gridDim.x) {
        if (!mbar_wait(tempty_bar(acc), acc_ph ^ 1u, abort_flag, p.flags)) break;
        tc_fence_after();
        bool ok = true;
        for (int kb = 0; kb < k_blocks; ++kb) {
          ok = mbar_wait(full_bar(s), ph, abort_flag, p.flags);
          if (!ok) break;
          tc_fence_after();
          const uint32_t a_addr = smem_u32(smem + s * STAGE_BYTES), b_addr = a_addr + A_BYTES;
#pragma unroll
          for (int k = 0; k < BK / UMMA_K; ++k) {
            const uint64_t adesc = A_K ? make_desc(a_addr + k * 32, 16, 1024) : make_desc(a_addr + k * 2048, 8192, 1024);
            const uint64_t bdesc = B_K ? make_desc(b_addr + k * 32, 16, 1024) : make_desc(b_addr + k * 2048, 8192, 1024);
            umma_bf16(tmem_base + acc * TN, adesc, bdesc, idesc, (kb > 0 || k > 0) ? 1u : 0u);
          }
          umma_commit(empty_bar(s));
          if (++s == STAGES) { s = 0; ph ^= 1u; }
        }
        if (!ok) break;
        umma_commit(tfull_bar(acc));
        if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
      }
    }
  } else {
    // ---------------- epilogue warps: a quarter of the rows, half of the columns each ----------------
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    int acc = 0; uint32_t acc_ph = 0;
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
      const Place w = place(u, p, MODE != UPDATE);
      if (!mbar_wait(tfull_bar(acc), acc_ph, abort_flag, p.flags)) break;
      tc_fence_after();
      const int m = w.i * TM + quarter * 32 + lane;
#pragma unroll 1
      for (int c = half * (TN / 2); c < (half + 1) * (TN / 2); c += 32) {
        const int n = w.j * TN + c;
        if (n >= p.N) break;
        uint32_t r[32];
        tmem_ld32(tmem_base + acc * TN + c + ((uint32_t)(quarter * 32) << 16), r);
        tmem_ld_wait();
        finish<MODE>(p, w.b, m, n, MODE != UPDATE && w.i != w.j, r);
        __syncwarp();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(tempty_bar(acc));
      if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
    }
  }
  // ---------------- common exit ----------------
  if (*abort_flag) {
    for (int i = 0; i < 64; ++i) __nanosleep(2000);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 2 * TN);
  }
}

// ---- momentum, norm and the first X ----------------------------------------------------------------
struct PrepP {
  const void* G; int64_t ldg, stride_g;
  const float* m; int64_t ldm, stride_m;           // null: no momentum
  float* m_out; int64_t ldm_out, stride_m_out;
  int rows, cols, nesterov, f32;
  float beta, w, eps, scale;
  double* partial;                                 // [batch][blocks]
  __half *hi, *lo; int64_t ld;
  bf16* O;                                         // no steps: scale X
};

// four columns of a row from column c on; what lies behind the row's end is 0.  VEC: rows are whole fours, aligned
template <int VEC> __device__ __forceinline__ float4 load4(const float* p, int left) {
  if (VEC) return *reinterpret_cast<const float4*>(p);
  return make_float4(p[0], left > 1 ? p[1] : 0.f, left > 2 ? p[2] : 0.f, left > 3 ? p[3] : 0.f);
}
template <int VEC> __device__ __forceinline__ float4 load4(const bf16* p, int left) {
  if (VEC) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x)), b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
    return make_float4(a.x, a.y, b.x, b.y);
  }
  return make_float4(__bfloat162float(p[0]), left > 1 ? __bfloat162float(p[1]) : 0.f, left > 2 ? __bfloat162float(p[2]) : 0.f, left > 3 ? __bfloat162float(p[3]) : 0.f);
}
__device__ __forceinline__ float4 weigh(float s, const float4 a, float t, const float4 b) {
  return make_float4(fmaf(s, a.x, t * b.x), fmaf(s, a.y, t * b.y), fmaf(s, a.z, t * b.z), fmaf(s, a.w, t * b.w));
}

// the new momentum, and the sum of the squares of u in 64 bits (whose range holds any)
template <typename TG, int VEC>
__global__ void __launch_bounds__(256) ortho_norm_kernel(const PrepP p) {
  pdl_wait(); pdl_trigger();
  const int b = blockIdx.y;
  const uint32_t chunks = (p.cols + 3) / 4;
  const uint64_t n = (uint64_t)p.rows * chunks;
  double sum = 0.0;
  for (uint64_t e = (uint64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (uint64_t)gridDim.x * 256) {
    const uint32_t row = n <= 0xffffffffu ? (uint32_t)e / chunks : (uint32_t)(e / chunks), c = 4 * (uint32_t)(e - (uint64_t)row * chunks);
    const int left = p.cols - c;
    float4 u = load4<VEC>((const TG*)p.G + b * p.stride_g + row * p.ldg + c, left);
    if (p.m) {
      const float4 m = load4<VEC>(p.m + b * p.stride_m + row * p.ldm + c, left), g = u;
      const float4 v = weigh(p.beta, m, p.w, g);
      float* o = p.m_out + b * p.stride_m_out + row * p.ldm_out + c;
      if (VEC) *reinterpret_cast<float4*>(o) = v;
      else { o[0] = v.x; if (left > 1) o[1] = v.y; if (left > 2) o[2] = v.z; if (left > 3) o[3] = v.w; }
      u = p.nesterov ? weigh(p.beta, v, p.w, g) : v;
    }
    sum = fma((double)u.x, (double)u.x, sum); sum = fma((double)u.y, (double)u.y, sum);
    sum = fma((double)u.z, (double)u.z, sum); sum = fma((double)u.w, (double)u.w, sum);
  }
  __shared__ double s_sum[8];
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) sum += s_sum[w];
    p.partial[(int64_t)b * gridDim.x + blockIdx.x] = sum;
  }
}

// X as a pair of fp16, its rows filled up with zeros
template <typename TG, int VEC>
__global__ void __launch_bounds__(256) ortho_scale_kernel(const PrepP p, int blocks) {
  pdl_wait(); pdl_trigger();
  const int b = blockIdx.y;
  __shared__ double s_inv;
  if (threadIdx.x < 32) {
    double s = 0.0;
    for (int i = threadIdx.x; i < blocks; i += 32) s += p.partial[(int64_t)b * blocks + i];
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const double d = sqrt(s) + (double)p.eps;
    if (threadIdx.x == 0) s_inv = d > 0.0 ? 1.0 / d : d == 0.0 ? 0.0 : d;      // (a matrix of zeros stays one; NaN stays NaN)
  }
  __syncthreads();
  const double inv = s_inv;
  const uint32_t chunks = p.ld / 4;
  const uint64_t n = (uint64_t)p.rows * chunks;
  for (uint64_t e = (uint64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (uint64_t)gridDim.x * 256) {
    const uint32_t row = n <= 0xffffffffu ? (uint32_t)e / chunks : (uint32_t)(e / chunks), c = 4 * (uint32_t)(e - (uint64_t)row * chunks);
    const int left = p.cols - (int)c;
    float4 u = make_float4(0.f, 0.f, 0.f, 0.f);
    if (left > 0) {
      u = load4<VEC>((const TG*)p.G + b * p.stride_g + row * p.ldg + c, left);
      if (p.m) {
        const float4 m = load4<VEC>(p.m_out + b * p.stride_m_out + row * p.ldm_out + c, left);
        u = p.nesterov ? weigh(p.beta, m, p.w, u) : m;
      }
    }
    const float x[4] = {(float)(u.x * inv), (float)(u.y * inv), (float)(u.z * inv), (float)(u.w * inv)};
    if (p.O) {
#pragma unroll
      for (int j = 0; j < 4; ++j) if (j < left) p.O[((int64_t)b * p.rows + row) * p.cols + c + j] = __float2bfloat16_rn(p.scale * x[j]);
      continue;
    }
    uint32_t h[2], l[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float s = 1 << X_EXP, y0 = x[2 * j] * s, y1 = x[2 * j + 1] * s;
      h[j] = half2_bits(y0, y1);
      const float2 a = half2_floats(h[j]);
      l[j] = half2_bits((y0 - a.x) * (1 << LO_EXP), (y1 - a.y) * (1 << LO_EXP));
    }
    const int64_t at = ((int64_t)b * p.rows + row) * p.ld + c;
    *reinterpret_cast<uint2*>(p.hi + at) = make_uint2(h[0], h[1]);
    *reinterpret_cast<uint2*>(p.lo + at) = make_uint2(l[0], l[1]);
  }
}

// ---- host ------------------------------------------------------------------------------------------
struct Plan { int side, blocks; int64_t ld, lds; size_t partial, hi[2], lo, a, p, bytes; };

Plan make_plan(int batch, int m, int n, int steps) {
  Plan q = {};
  q.side = std::min(m, n);
  q.ld = ((int64_t)n + 63) / 64 * 64;
  q.lds = ((int64_t)q.side + 63) / 64 * 64;
  const int64_t chunks = (int64_t)m * ((n + 3) / 4);
  q.blocks = (int)std::max<int64_t>(1, std::min<int64_t>((chunks + 1023) / 1024, SMS * 8 / std::min(batch, SMS * 8)));
  size_t at = 0;
  auto take = [&](size_t k) { const size_t was = at; at += (k + 255) / 256 * 256; return was; };
  q.partial = take((size_t)batch * q.blocks * 8);
  if (steps > 0) {
    const size_t x = (size_t)batch * m * q.ld * 2, s = (size_t)batch * q.side * q.lds * 2;
    q.hi[0] = take(x); q.hi[1] = take(steps > 1 ? x : 0); q.lo = take(x);
    q.a = take(s); q.p = take(s);
  }
  q.bytes = at;
  return q;
}

int check_ortho(int batch, int m, int n, int steps) {
  if (batch < 0 || m < 0 || n < 0) return ppu_fail(PPU_EINVAL, "negative size");
  if (m > MAX_SIDE || n > MAX_SIDE || batch > 65535) return ppu_fail(PPU_ESHAPE, "at most 65535 matrices of sides up to %d", MAX_SIDE);
  if (steps < 0 || steps > MAX_STEPS) return ppu_fail(PPU_EINVAL, "steps must be 0 to %d", MAX_STEPS);
  // tiles are counted in 32 bits
  const int64_t tiles = (((int64_t)m + 127) / 128) * (((int64_t)n + 127) / 128) * batch;
  if (tiles > (1 << 30)) return ppu_fail(PPU_ESHAPE, "too many matrices of this size");
  return PPU_OK;
}

// largest |a x + b x^3 + c x^5| for 0 <= x <= top, and of |b y + c y^2| for 0 <= y <= top^2
double largest_value(double a, double b, double c, double top) {
  auto f = [&](double x) { return std::fabs(x * (a + x * x * (b + x * x * c))); };
  double best = f(top);
  auto at = [&](double y) { if (y > 0 && y < top * top) best = std::max(best, f(std::sqrt(y))); };
  if (c != 0) {
    const double disc = 9 * b * b - 20 * a * c;
    if (disc >= 0) { at((-3 * b + std::sqrt(disc)) / (10 * c)); at((-3 * b - std::sqrt(disc)) / (10 * c)); }
  } else if (b != 0) {
    at(-a / (3 * b));
  }
  return best;
}
double largest_poly(double b, double c, double top) {
  const double y = top * top;
  double best = std::fabs(y * (b + c * y));
  if (c != 0) { const double z = -b / (2 * c); if (z > 0 && z < y) best = std::max(best, std::fabs(z * (b + c * z))); }
  return best;
}

#define CUDA_OK(call)                                                                    \
  do {                                                                                   \
    cudaError_t e_ = (call);                                                             \
    if (e_ != cudaSuccess)                                                               \
      return ppu_fail(PPU_ECUDA, "%s failed: %s", #call, cudaGetErrorString(e_));        \
  } while (0)

// boxes of 64 x rows over [batch][rows][inner]
bool encode(CUtensorMap* map, const __half* base, int64_t ld, int inner, int rows, int batch, int box_rows) {
  const cuuint64_t dim[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)batch}, stride[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * rows * 2};
  const cuuint32_t box[3] = {(cuuint32_t)BK, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
  return get_encoder()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, (void*)base, dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
struct Operand { const __half* p; int64_t ld; int rows, inner; };      // as stored: [batch][rows][ld], `inner` columns of it

template <bool A_K, bool B_K, int MODE>
int product(const Operand& A, const Operand& B, GemmP p, cudaStream_t st) {
  static PerDeviceFlag attr;
  if (!ppu_set_smem_once(attr, ortho_tile_kernel<A_K, B_K, MODE>, SMEM)) return ppu_fail(PPU_ECUDA, "shared memory limit not accepted");
  CUtensorMap mapA, mapB;
  if (!encode(&mapA, A.p, A.ld, A.inner, A.rows, p.batch, A_K ? TM : 64) || !encode(&mapB, B.p, B.ld, B.inner, B.rows, p.batch, B_K ? TN : 64))
    return ppu_fail(PPU_ECUDA, "tensor map not accepted");
  p.tiles_m = (p.M + TM - 1) / TM; p.tiles_n = (p.N + TN - 1) / TN;
  p.tiles = MODE == UPDATE ? p.tiles_m * p.tiles_n : p.tiles_m * (p.tiles_m + 1) / 2;
  const int64_t units = (int64_t)p.tiles * p.batch;
  CUDA_OK(ppu_launch_dependent(ortho_tile_kernel<A_K, B_K, MODE>, (unsigned)std::min<int64_t>(units, ppu_sm_count()), 64 + 32 * EPI, SMEM, st, mapA, mapB, p));
  return PPU_OK;
}

template <typename TG>
int prepare(const PrepP& p, const Plan& q, int batch, bool vec, cudaStream_t st) {
  const dim3 grid(q.blocks, batch);
  if (vec) {
    CUDA_OK(ppu_launch_dependent(ortho_norm_kernel<TG, 1>, grid, 256, 0, st, p));
    CUDA_OK(ppu_launch_dependent(ortho_scale_kernel<TG, 1>, grid, 256, 0, st, p, q.blocks));
  } else {
    CUDA_OK(ppu_launch_dependent(ortho_norm_kernel<TG, 0>, grid, 256, 0, st, p));
    CUDA_OK(ppu_launch_dependent(ortho_scale_kernel<TG, 0>, grid, 256, 0, st, p, q.blocks));
  }
  return PPU_OK;
}
// whether rows may be read four values (of `bytes` together) at a time
bool aligned(const void* p, int64_t ld, int64_t stride, int bytes) {
  return !p || (!(reinterpret_cast<uintptr_t>(p) & (bytes - 1)) && ld % 4 == 0 && stride % 4 == 0);
}

}  // namespace

extern "C" int ppu_orthogonalize_query_bytes(int batch, int m, int n, int steps, size_t* bytes) {
  if (!bytes) return ppu_fail(PPU_EINVAL, "bytes is null");
  const int rc = check_ortho(batch, m, n, steps);
  if (rc) return rc;
  *bytes = batch && m && n ? make_plan(batch, m, n, steps).bytes : 0;
  return PPU_OK;
}

extern "C" int ppu_orthogonalize(const void* G, int64_t ldg, int64_t stride_g, int g_type, const float* momentum, int64_t ldm, int64_t stride_m, float* momentum_out,
                                 int64_t ldmo, int64_t stride_mo, float beta, float weight, int nesterov, const float* coef, int n_coef, int steps, float eps, float scale,
                                 void* O, int batch, int m, int n, void* workspace, size_t workspace_bytes, int32_t* flags, void* cuda_stream) {
  const int rc = check_ortho(batch, m, n, steps);
  if (rc) return rc;
  if (g_type != PPU_BF16 && g_type != PPU_F32) return ppu_fail(PPU_EINVAL, "unknown type");
  if (!(eps >= 0.f)) return ppu_fail(PPU_EINVAL, "eps must not be negative");
  if ((momentum == nullptr) != (momentum_out == nullptr)) return ppu_fail(PPU_EINVAL, "momentum and momentum_out go together");
  if (steps > 0 && (!coef || (n_coef != 1 && n_coef != steps))) return ppu_fail(PPU_EINVAL, "coefficients: one triple, or one for each step");
  double top = 1.0;                                // bound of the singular values
  int p_exp[MAX_STEPS];
  for (int k = 0; k < steps; ++k) {
    const float* c = coef + (n_coef == 1 ? 0 : 3 * k);
    const double poly = largest_poly(c[1], c[2], top);
    top = 1.01 * largest_value(c[0], c[1], c[2], top);
    if (!(top <= 2.8) || !(poly <= 1024.0) || !(std::fabs((double)c[0]) <= 1024.0))
      return ppu_fail(PPU_EINVAL, "the coefficients of step %d take singular values up to %g, above 2.8", k, top);
    p_exp[k] = std::min(12, (int)std::floor(std::log2(32768.0 / std::max(poly, 1e-30))));
  }
  if (batch == 0 || m == 0 || n == 0) return PPU_OK;
  if (!G || !O || !workspace) return ppu_fail(PPU_EINVAL, "null operand");
  if (ldg < n || (momentum && (ldm < n || ldmo < n))) return ppu_fail(PPU_EINVAL, "row strides must be at least n");
  if (batch > 1 && (stride_g < 0 || (momentum && (stride_m < 0 || stride_mo < (m - 1) * ldmo + n)))) return ppu_fail(PPU_EINVAL, "matrices written must not overlap");
  if (momentum_out == momentum && momentum && (ldm != ldmo || (batch > 1 && stride_m != stride_mo)))
    return ppu_fail(PPU_EINVAL, "momentum_out in the place of momentum needs its strides");
  const int g_bytes = g_type == PPU_BF16 ? 2 : 4;
  if ((reinterpret_cast<uintptr_t>(G) % g_bytes) || (reinterpret_cast<uintptr_t>(momentum) & 3) || (reinterpret_cast<uintptr_t>(momentum_out) & 3) ||
      (reinterpret_cast<uintptr_t>(O) & 15) || (reinterpret_cast<uintptr_t>(workspace) & 255))
    return ppu_fail(PPU_EINVAL, "O must be 16-byte, workspace 256-byte aligned, G and momentum as their types are");
  const Plan q = make_plan(batch, m, n, steps);
  if (workspace_bytes < q.bytes) return ppu_fail(PPU_ENOMEM, "workspace has %zu bytes, %zu needed", workspace_bytes, q.bytes);
  if (steps > 0 && gemm_tc_init() != 0) return ppu_fail(PPU_ECUDA, "no tensor-map encoder");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  uint8_t* ws = (uint8_t*)workspace;
  __half *hi[2] = {(__half*)(ws + q.hi[0]), (__half*)(ws + q.hi[1])}, *lo = (__half*)(ws + q.lo), *A = (__half*)(ws + q.a), *P = (__half*)(ws + q.p);
  PrepP pp = {};
  pp.G = G; pp.ldg = ldg; pp.stride_g = stride_g; pp.m = momentum; pp.ldm = ldm; pp.stride_m = stride_m;
  pp.m_out = momentum_out; pp.ldm_out = ldmo; pp.stride_m_out = stride_mo; pp.rows = m; pp.cols = n; pp.nesterov = nesterov != 0;
  pp.beta = beta; pp.w = weight; pp.eps = eps; pp.scale = scale; pp.partial = (double*)(ws + q.partial); pp.hi = hi[0]; pp.lo = lo; pp.ld = q.ld;
  pp.O = steps == 0 ? (bf16*)O : nullptr;
  const bool vec = n % 4 == 0 && aligned(G, ldg, stride_g, 4 * g_bytes) && aligned(momentum, ldm, stride_m, 16) && aligned(momentum_out, ldmo, stride_mo, 16);
  int rc2 = g_type == PPU_BF16 ? prepare<bf16>(pp, q, batch, vec, st) : prepare<float>(pp, q, batch, vec, st);
  const bool left = m <= n;
  for (int k = 0; k < steps && !rc2; ++k) {
    const float* c = coef + (n_coef == 1 ? 0 : 3 * k);
    const Operand X = {hi[k & 1], q.ld, m, n}, SA = {A, q.lds, q.side, q.side}, SP = {P, q.lds, q.side, q.side};
    GemmP g = {};
    g.batch = batch; g.flags = flags;
    // A = X X^T or X^T X
    g.M = g.N = q.side; g.K = left ? n : m; g.C = A; g.ldc = q.lds; g.stride = q.side * q.lds;
    g.c = std::ldexp(1.f, A_EXP - 2 * X_EXP);
    rc2 = left ? product<true, true, GRAM>(X, X, g, st) : product<false, false, GRAM>(X, X, g, st);
    if (rc2) break;
    // P = b A + c A A
    g.K = q.side; g.C = P; g.A = A;
    g.b = std::ldexp(c[1], p_exp[k] - A_EXP); g.c = std::ldexp(c[2], p_exp[k] - 2 * A_EXP);
    rc2 = product<true, true, POLY>(SA, SA, g, st);
    if (rc2) break;
    // X = a X + P X or X P
    g.M = m; g.N = n; g.K = q.side; g.hi = hi[k & 1]; g.lo = lo; g.hi_out = k + 1 < steps ? hi[(k + 1) & 1] : nullptr;
    g.ldc = q.ld; g.stride = (int64_t)m * q.ld; g.a = c[0]; g.f = std::ldexp(1.f, -p_exp[k]);
    g.O = (bf16*)O; g.ldo = n; g.scale = scale;
    if (k + 1 == steps) { g.a = std::ldexp(c[0], -X_EXP); g.f = std::ldexp(1.f, -p_exp[k] - X_EXP); }
    rc2 = left ? product<true, false, UPDATE>(SP, X, g, st) : product<true, true, UPDATE>(X, SP, g, st);
  }
  return rc2;
}
