// Pieces shared by the tcgen05 GEMM kernels: launch parameters, the fused-epilogue arithmetic and
// the routine that drains one accumulator tile from tensor memory to global memory.
#pragma once
#include "tc_common.cuh"

namespace gemm_tc_detail {
using namespace tc;

constexpr int BM = 128;
constexpr int BK = 64;            // 64 bf16 = 128 bytes = one swizzle row
constexpr int UMMA_K = 16;
constexpr int EPI_WARPS = 8;      // two per TMEM lane quarter, each draining half the columns
// (a block: warp 0: TMA, warp 1: MMA + TMEM owner, then epilogue)

// hardware tanh (relative error about 2^-11, below the bf16 rounding of the stored result)
__device__ __forceinline__ float tanh_fast(float x) {
  float y;
  asm("tanh.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float gelu_dev(float x) {
  const float u = 0.7978845608028654f * (x + 0.044715f * x * x * x);
  const float t = tanh_fast(u);
  return 0.5f * x * (1.f + t);
}
__device__ __forceinline__ float gelu_grad_dev(float x) {
  const float u = 0.7978845608028654f * (x + 0.044715f * x * x * x);
  const float t = tanh_fast(u);
  const float du = 0.7978845608028654f * (1.f + 3.f * 0.044715f * x * x);
  return 0.5f * (1.f + t) + 0.5f * x * (1.f - t * t) * du;
}
__device__ __forceinline__ uint4 pack8_bf16(const float* f) {
  uint4 u;
  __nv_bfloat162* p = reinterpret_cast<__nv_bfloat162*>(&u);
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
  return u;
}

// 32-byte global accesses (one full sector per lane and instruction)
__device__ __forceinline__ void st_v8(void* p, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]),
               "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void ld_v8(uint32_t* v, const void* p) {
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
                 "=r"(v[7])
               : "l"(p));
}
__device__ __forceinline__ uint32_t pack2_bf16(float a, float b) {
  __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&v);
}

// rotary positions on `pairs` adjacent pairs of f starting at column n0 of a [.., heads x dh] row
__device__ __forceinline__ void rope_pairs(float* f, int pairs, const float2* cs_row, int n0, int dh) {
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    if (q >= pairs) break;
    const float2 w = __ldg(cs_row + ((n0 + 2 * q) % dh) / 2);
    const float a = f[2 * q], b = f[2 * q + 1];
    f[2 * q] = a * w.x - b * w.y;
    f[2 * q + 1] = a * w.y + b * w.x;
  }
}

struct TcParams {
  int M, N, K;
  int epilogue;
  void* C; long long ldc;
  void* C2;
  const void* aux; long long ldaux;
  int* flags;
  int tiles_m, tiles_n;
  int tail_from;   // SM-pair kernel: tiles from this index on are worked as two 128-column halves
  int n_fastest;   // SM-pair kernel: consecutive tile indices walk along N (else along M)
  int splits; long long split_stride;
  // Boxes no larger than the operands need: rows of A (K-major, one CTA to a tile: M below 128), k rows of MN-major
  // operands and products along k (K below 64).  Rows outside a tensor cost the TMA unit more than rows inside:
  // 24 x 32768 x 2048 took 42 us with 104 of 128 rows filled in, 36 us with 128 real rows,
  // 34 us with a box of 24.
  int a_rows, k_rows;
  int wide;   // every output / auxiliary row start is 32-byte aligned: use 32-byte accesses
  int rope_S, rope_dh, rope_cols;
  void* C3; long long ldc3; int c3_lo, c3_hi;
  float piece_scale; float2* piece_stats; long long ld_pieces;
  PieceEntries entries;
  const float* row_scale; unsigned* zero_word;
  int dependent;   // launched as a programmatic dependent
  // Epilogue warps.  0: all drain each tile, a part of its columns each.  1: half of them drain one accumulator, half the
  // other, so that one tile is read from tensor memory (600 cycles of latency for 64 columns) while the other
  // is stored (900 cycles of the load/store pipe): for blocks that work several tiles (dE of
  // 24 x 32768 x 768: 18.7 -> 16.7 us, of 90 x 6300 x 360: 11 -> 8).
  int alternate;
};

// what a kernel's epilogue warps do with an accumulator: the epilogues of drain_cols, or one of
// those that have instantiations of their own: drain_cols keeps its registers, and these have 32 KB of
// shared memory behind the operand stages, through which they store 64-column groups
enum DrainMode { DRAIN_COLS = 0, DRAIN_PIECES = 1, DRAIN_TWO = 2 };
// DRAIN_PIECES has twice the warps on 256-wide tiles: its 64 columns take a warp 1500 cycles, of which the exponentials are 512 of the SM
// quarter's unit for them (logits of 4096 x 32768 x 64: 110 us with 8 warps, 88 with 16; x 768: 160 and 153).
constexpr int epi_warps(int mode, int bn) { return mode == DRAIN_PIECES && bn == 256 ? 2 * EPI_WARPS : EPI_WARPS; }
constexpr int gemm_threads(int mode, int bn) { return 64 + 32 * epi_warps(mode, bn); }
constexpr int store_bytes(int mode) { return mode == DRAIN_PIECES ? 32 * 64 : 32 * 128; }    // a warp's 32 rows x 32 or 64 bf16 columns
template <int MODE> struct Second {};
// DRAIN_TWO: a launch works the units of two products (launch_gemm_tc_two), the one with the longer units
// first; A's order may differ between the two.  This holds the second product.
template <> struct Second<DRAIN_TWO> { CUtensorMap a, b; TcParams p; int a_k, a_k2, units, units2, fill; };
// The i-th unit of block (pair) b of n: the first product's are dealt round; blocks that got one less then
// have `fill` of the second's, as many as make up for it; the rest are dealt round again.
__device__ __forceinline__ int two_unit(int i, int b, int n, int units, int units2, int fill) {
  constexpr int NONE = 0x7fffffff;
  const int own = units > b ? (units - b - 1) / n + 1 : 0;
  if (i < own) return b + i * n;
  i -= own;
  const int heavy = units % n;
  int v = 0;
  if (heavy > 0) {
    const int light = n - heavy;
    if (b >= heavy) {
      if (i < fill) { v = b - heavy + i * light; return v < units2 ? units + v : NONE; }
      i -= fill;
    }
    v = light * fill;
  }
  v += n - 1 - b + i * n;
  return v < units2 ? units + v : NONE;
}

template <int MODE, int BN> constexpr int store_smem() { return MODE == DRAIN_COLS ? 0 : epi_warps(MODE, BN) * store_bytes(MODE); }

// Columns of a tile of bn that a set of four warps (one for each quarter of the rows) drains: an equal part, of the whole
// tile or, where the sets take turns, of every other tile's; pieces are not divided, so sets may be left without.
template <int MODE, int BN> __device__ __forceinline__ void set_columns(int set, int alternate, int bn, int& begin, int& end) {
  constexpr int SETS = epi_warps(MODE, BN) / 4;
  const int sub = alternate ? set % (SETS / 2) : set;
  int cols = alternate ? bn / (SETS / 2) : bn / SETS;
  if (MODE == DRAIN_PIECES && cols < PIECE) cols = PIECE;
  begin = sub * cols;
  end = begin + cols < bn ? begin + cols : bn;
}

// host side (gemm_tc.cu / gemm_tc_pair.cu)
bool encode_map(CUtensorMap* map, const bf16* base, long long ld, bool kmajor, int rows, int K, int box_rows,
                bool transient = false, int k_rows = BK);
TcParams make_params(const GemmArgs& g);
int launch_gemm_tc_pair(const GemmArgs& g, const TcParams& p, int bn, cudaStream_t st);   // bn: 256 or 128
int launch_gemm_tc_pair_pieces(const GemmArgs& g, const TcParams& p, cudaStream_t st);
int launch_gemm_tc_pair_two(const GemmArgs& g, const GemmArgs* g2, cudaStream_t st);
// units of the second product that take the time of one of the first (overhead: of a unit, in k)
inline int two_fill(const GemmArgs& g, const GemmArgs& g2, int overhead) {
  const int k1 = g.K / (g.splits > 1 ? g.splits : 1), k2 = g2.K / (g2.splits > 1 ? g2.splits : 1);
  return (k1 + overhead) / (k2 + overhead);
}

// Drains rows [m0 + 32 quarter, +32) x columns [n0 + half BN/2, + BN/2) of the accumulator at
// TMEM column t_acc through registers into global memory, applying the epilogue p.epilogue.
// One row per lane; `sp` is the split-K slice (offsets the output by sp * split_stride).
// (drain_cols: the same for an explicit range [c_begin, c_end) of the tile's columns, both
// multiples of 32)
__device__ __forceinline__ void drain_cols(const TcParams& p, int m0, int n0, int sp, uint32_t t_acc,
                                           int quarter, int c_begin, int c_end, int lane) {
  const int m = m0 + quarter * 32 + lane;
  const bool row_ok = m < p.M;
  const uint32_t t_row = t_acc + ((uint32_t)(quarter * 32) << 16);
  float head_dot = 0.f;   // EPI_DELTA_BF16: running sum over the current head's columns
#pragma unroll 1
  for (int c0 = c_begin; c0 < c_end; c0 += 32) {
    const int nb = n0 + c0;
    if (nb >= p.N) break;                  // warp-uniform
    uint32_t r[32];
    tmem_ld32(t_row + c0, r);              // asynchronous until tmem_ld_wait
    const long long ci = (long long)m * p.ldc + nb + (long long)sp * p.split_stride;
    const bool full = nb + 32 <= p.N;
    if (p.wide && full) {
      // whole 32-column chunk with 32-byte accesses
      if (p.epilogue == EPI_RESID_F32) {
        uint32_t x[32];
        const float* rs = (const float*)p.aux + (long long)m * p.ldaux + nb;
        if (row_ok) {
#pragma unroll
          for (int j = 0; j < 4; ++j) ld_v8(x + 8 * j, rs + 8 * j);
        }
        tmem_ld_wait();
        if (row_ok) {
#pragma unroll
          for (int j = 0; j < 32; ++j) x[j] = __float_as_uint(__uint_as_float(x[j]) + __uint_as_float(r[j]));
#pragma unroll
          for (int j = 0; j < 4; ++j) st_v8((float*)p.C + ci + 8 * j, x + 8 * j);
        }
      } else if (p.epilogue == EPI_DGELU) {
        uint32_t hv[16];
        const bf16* hs = (const bf16*)p.aux + (long long)m * p.ldaux + nb;
        if (row_ok) { ld_v8(hv, hs); ld_v8(hv + 8, hs + 16); }
        tmem_ld_wait();
        if (row_ok) {
          uint32_t o[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float2 h2 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&hv[j]));
            o[j] = pack2_bf16(__uint_as_float(r[2 * j]) * gelu_grad_dev(h2.x),
                              __uint_as_float(r[2 * j + 1]) * gelu_grad_dev(h2.y));
          }
          st_v8((bf16*)p.C + ci, o);
          st_v8((bf16*)p.C + ci + 16, o + 8);
        }
      } else if (p.epilogue == EPI_STORE_F32) {
        tmem_ld_wait();
        if (row_ok) {
#pragma unroll
          for (int j = 0; j < 4; ++j) st_v8((float*)p.C + ci + 8 * j, r + 8 * j);
        }
      } else {
        uint32_t uv[16];
        if (p.epilogue == EPI_DELTA_BF16 && row_ok) {
          const bf16* us = (const bf16*)p.aux + (long long)m * p.ldaux + nb;
          ld_v8(uv, us); ld_v8(uv + 8, us + 16);
        }
        tmem_ld_wait();
        if (row_ok) {
          if (p.epilogue == EPI_ROPE_BF16 && nb < p.rope_cols) {
            const float2* cs_row = (const float2*)p.aux + (long long)(m % p.rope_S) * (p.rope_dh / 2);
            if (p.rope_dh % 32 == 0) {
              // the chunk lies inside one head: its 16 (cos, sin) pairs are 128 contiguous bytes
              uint32_t w[32];
              const float2* src = cs_row + (nb % p.rope_dh) / 2;
#pragma unroll
              for (int j = 0; j < 4; ++j) ld_v8(w + 8 * j, src + 4 * j);
#pragma unroll
              for (int q = 0; q < 16; ++q) {
                const float cw = __uint_as_float(w[2 * q]), sw = __uint_as_float(w[2 * q + 1]);
                const float a = __uint_as_float(r[2 * q]), b = __uint_as_float(r[2 * q + 1]);
                r[2 * q] = __float_as_uint(a * cw - b * sw);
                r[2 * q + 1] = __float_as_uint(a * sw + b * cw);
              }
            } else {
              rope_pairs(reinterpret_cast<float*>(r), 16, cs_row, nb, p.rope_dh);
            }
          }
          uint32_t o[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) o[j] = pack2_bf16(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
          if (p.C) {       // (the pre-activation store of EPI_GELU_DUAL is optional)
            st_v8((bf16*)p.C + ci, o);
            st_v8((bf16*)p.C + ci + 16, o + 8);
          }
          if (p.epilogue == EPI_DELTA_BF16) {
            // the product uses the stored (rounded) values, as the attention kernels will
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float2 gv = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&o[j]));
              const float2 u2 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&uv[j]));
              head_dot = fmaf(gv.x, u2.x, fmaf(gv.y, u2.y, head_dot));
            }
            if ((nb + 32) % p.rope_dh == 0) {
              const int heads = p.N / p.rope_dh;
              ((float*)p.C3)[((long long)(m / p.rope_S) * heads + nb / p.rope_dh) * p.rope_S + m % p.rope_S] = head_dot;
              head_dot = 0.f;
            }
          }
          if (p.epilogue == EPI_GELU_DUAL) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              o[j] = pack2_bf16(gelu_dev(__uint_as_float(r[2 * j])), gelu_dev(__uint_as_float(r[2 * j + 1])));
            st_v8((bf16*)p.C2 + ci, o);
            st_v8((bf16*)p.C2 + ci + 16, o + 8);
            if (p.C3 && nb < p.c3_hi && nb + 32 > p.c3_lo) {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const int col = nb + 8 * j;
                if (col >= p.c3_lo && col + 8 <= p.c3_hi)
                  *reinterpret_cast<uint4*>((bf16*)p.C3 + (long long)m * p.ldc3 + (col - p.c3_lo)) =
                      make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
              }
            }
          }
        }
      }
      continue;
    }
    if (p.epilogue == EPI_RESID_F32) {
      float4 x[8];
      const float4* rs = reinterpret_cast<const float4*>((const float*)p.aux + (long long)m * p.ldaux + nb);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        x[j] = (row_ok && (full || nb + 4 * j < p.N)) ? rs[j] : make_float4(0.f, 0.f, 0.f, 0.f);
      tmem_ld_wait();
      if (row_ok) {
        float4* o = reinterpret_cast<float4*>((float*)p.C + ci);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (full || nb + 4 * j < p.N)
            o[j] = make_float4(x[j].x + __uint_as_float(r[4 * j]), x[j].y + __uint_as_float(r[4 * j + 1]),
                               x[j].z + __uint_as_float(r[4 * j + 2]), x[j].w + __uint_as_float(r[4 * j + 3]));
      }
    } else if (p.epilogue == EPI_DGELU) {
      uint4 hv[4];
      const uint4* hs = reinterpret_cast<const uint4*>((const bf16*)p.aux + (long long)m * p.ldaux + nb);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        hv[j] = (row_ok && (full || nb + 8 * j < p.N)) ? hs[j] : make_uint4(0, 0, 0, 0);
      tmem_ld_wait();
      if (row_ok) {
        uint4* o = reinterpret_cast<uint4*>((bf16*)p.C + ci);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (!(full || nb + 8 * j < p.N)) break;
          const __nv_bfloat162* hp = reinterpret_cast<const __nv_bfloat162*>(&hv[j]);
          float a[8];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float2 h2 = __bfloat1622float2(hp[q]);
            a[2 * q] = __uint_as_float(r[8 * j + 2 * q]) * gelu_grad_dev(h2.x);
            a[2 * q + 1] = __uint_as_float(r[8 * j + 2 * q + 1]) * gelu_grad_dev(h2.y);
          }
          o[j] = pack8_bf16(a);
        }
      }
    } else {
      tmem_ld_wait();
      if (row_ok) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (!(full || nb + 8 * j < p.N)) break;
          float f[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) f[q] = __uint_as_float(r[8 * j + q]);
          if (p.epilogue == EPI_ROPE_BF16 && nb + 8 * j < p.rope_cols)
            rope_pairs(f, 4, (const float2*)p.aux + (long long)(m % p.rope_S) * (p.rope_dh / 2), nb + 8 * j,
                       p.rope_dh);
          if (p.epilogue == EPI_STORE_F32) {
            float4* o = reinterpret_cast<float4*>((float*)p.C + ci + 8 * j);
            o[0] = make_float4(f[0], f[1], f[2], f[3]);
            o[1] = make_float4(f[4], f[5], f[6], f[7]);
          } else {
            if (p.C) *reinterpret_cast<uint4*>((bf16*)p.C + ci + 8 * j) = pack8_bf16(f);
            if (p.epilogue == EPI_GELU_DUAL) {
#pragma unroll
              for (int q = 0; q < 8; ++q) f[q] = gelu_dev(f[q]);
              const uint4 gv = pack8_bf16(f);
              *reinterpret_cast<uint4*>((bf16*)p.C2 + ci + 8 * j) = gv;
              const int col = nb + 8 * j;
              if (p.C3 && col >= p.c3_lo && col + 8 <= p.c3_hi)
                *reinterpret_cast<uint4*>((bf16*)p.C3 + (long long)m * p.ldc3 + (col - p.c3_lo)) = gv;
            }
          }
        }
      }
    }
  }
}

__device__ __forceinline__ float ex2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A warp's 32 rows x COLS (64 or 32) columns, packed by its lanes (one row each), to global memory through its
// shared memory, so that a store covers four rows' whole 128-byte lines, or eight rows' halves.  (From the
// registers, a lane 32 bytes of its own row at a time, a store touches 32 lines: 2304 x 32000 x 768 took 95 us
// against 70 without the store and 85 this way.  By TMA from the same shared memory it took 90: the buffer is free
// again only when the copy has read it; the dE of 256 x 2048 x 32768, all stores, 111 us by TMA and 73 this way.)
// Row r of the buffer has its 16-byte pieces in other places than its neighbours: no bank conflicts either
// way.  rows, cols: of the output, from here on.
template <int COLS>
__device__ __forceinline__ void store_group(bf16* out, long long ld, uint32_t buf, const uint32_t* o, int rows, int cols, int lane) {
  constexpr int P = COLS / 8, ROWS = 32 / P;     // pieces of a row, rows of a store
  auto place = [](int r, int j) { return (uint32_t)(r * COLS * 2 + ((j ^ (COLS == 64 ? r & 7 : r >> 1 & 3)) << 4)); };
  __syncwarp();                     // (the group before has been read)
#pragma unroll
  for (int j = 0; j < P; ++j)
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(buf + place(lane, j)), "r"(o[4 * j]), "r"(o[4 * j + 1]), "r"(o[4 * j + 2]),
                 "r"(o[4 * j + 3])
                 : "memory");
  __syncwarp();
  const int piece = lane % P;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int r = ROWS * i + lane / P;
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(buf + place(r, piece)) : "memory");
    if (r < rows && 8 * piece < cols) *reinterpret_cast<uint4*>(out + r * ld + 8 * piece) = v;
  }
}

// EPI_PIECES.  A lane holds 64 logits of its row at a time: x = acc * piece_scale (the scale holds
// log2(e) and the temperature), e = 2^(x - ref).  The powers are stored in bf16 - a relative
// rounding of half a step (2^-8) whatever the logit, where a bf16 logit of 16 would be off by 2^-4
// absolutely - and {ref, sum e} in fp32, the sum over the unrounded powers, so the log-sum-exp keeps fp32
// accuracy.  bf16 has fp32's exponents, so with ordinary logits (|x| <= 60: 41 nats) one reference, 0,
// serves the whole row, and its softmax is the stored powers times one factor, which the gradient
// products apply to their other operand and to their result: no pass over the powers.  Pieces beyond that
// are kept relative to their own maximum and brought into line afterwards.  That is by a power of two, and exact, because ref
// is a whole number: with the maximum itself the powers were rounded to bf16 a second time (rms error of dX 2.88e-3, now 2.4e-3).
// The exponent is one fused multiply-add on the accumulator, exact but for its own rounding.
// The entries' own x are taken from tensor memory a column at a time: a warp's 32 rows have two in a
// piece with 32 entries in 32768 columns.  (As dot products in the row kernel they were a gather of 4 KB of E
// for each entry: 106 of 1200 us at 4096 x 2048 x 32768.)
// (Of 16 warps a thread has 112 registers: 64 logits, and powers of 32 at a time.)
template <typename F>
__device__ __forceinline__ void drain_pieces(const TcParams& p, uint32_t buf, int m0, int n0,
                                             uint32_t t_acc, int quarter, int c_begin, int c_end, int lane, F release) {
  const int mw = m0 + quarter * 32, m = mw + lane;
  const uint32_t t_row = t_acc + ((uint32_t)(quarter * 32) << 16);
  if (c_begin >= c_end || n0 + c_begin >= p.N || mw >= p.M) { release(); return; }
#pragma unroll 1
  for (int c0 = c_begin; c0 < c_end; c0 += PIECE) {
    const int nb = n0 + c0;
    if (nb >= p.N) break;                  // warp-uniform
    uint32_t r[PIECE];
    tmem_ld32(t_row + c0, r);
    tmem_ld32(t_row + c0 + 32, r + 32);
    int at = 0, end = 0, id = -1;          // this row's entries in the piece, and the first one's column
    if (m < p.M) {
      if (p.entries.k > 1) {
        const uint8_t* off = p.entries.off + (long long)m * p.entries.ld_off + nb / PIECE;
        at = off[0]; end = off[1];
      } else {
        end = 1;
      }
      if (at < end) id = p.entries.ids[(long long)m * p.entries.ld + at];
      if (id < nb || id >= nb + PIECE) id = -1;
    }
    tmem_ld_wait();
    if (nb + PIECE > p.N) {                // columns past the vocabulary: nothing
#pragma unroll
      for (int j = 0; j < PIECE; ++j)
        if (nb + j >= p.N) r[j] = 0xff800000u;
    }
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < PIECE; ++j) mx[j & 3] = fmaxf(mx[j & 3], __uint_as_float(r[j]));
    mx[0] = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
    float top = mx[0] * p.piece_scale;
    top = fabsf(top) <= PIECE_RANGE || top == -INFINITY ? 0.f : rintf(top);      // (-inf: all powers are 0)
    float less = top, off = 0.f;
    const bool far = fabsf(top) > 16777216.f;
    if (far) { less = 0.f; off = mx[0]; }  // 2^24: the rounding of top would be an exponent of more than 1 (the largest is taken off first)
    for (unsigned any = __ballot_sync(0xffffffffu, id >= 0); any; any = __ballot_sync(0xffffffffu, id >= 0)) {
      const int col = __shfl_sync(0xffffffffu, id, __ffs(any) - 1);
      const float x = __uint_as_float(tmem_ld1(t_row + c0 + (col - nb)));
      while (id == col) {                  // an id may be given several times
        p.entries.x[(long long)m * p.entries.k + at] = make_float2(fmaf(x - off, p.piece_scale, -less), top);
        ++at;
        id = at < end ? p.entries.ids[(long long)m * p.entries.ld + at] : -1;
      }
      __syncwarp();
    }
    if (c0 + PIECE >= c_end || nb + PIECE >= p.N) release();
    if (far) {
#pragma unroll
      for (int j = 0; j < PIECE; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) - off);
    }
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < PIECE; h += 32) {
      uint32_t o[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float e0 = ex2_fast(fmaf(__uint_as_float(r[h + 2 * j]), p.piece_scale, -less));
        const float e1 = ex2_fast(fmaf(__uint_as_float(r[h + 2 * j + 1]), p.piece_scale, -less));
        sum[(2 * j) & 3] += e0;
        sum[(2 * j + 1) & 3] += e1;
        o[j] = pack2_bf16(e0, e1);
      }
      // (columns up to the next multiple of 64 belong to the row too)
      if (p.C) store_group<32>((bf16*)p.C + (long long)mw * p.ldc + nb + h, p.ldc, buf, o, p.M - mw, 32, lane);
    }
    if (m < p.M)
      p.piece_stats[(long long)m * p.ld_pieces + nb / PIECE] = make_float2(top, (sum[0] + sum[1]) + (sum[2] + sum[3]));
  }
}

// EPI_OUT_BF16: row_scale * (aux + acc), rounded once.  aux: fp32 partial sums, rows 32-byte aligned;
// N is a multiple of 8.
template <typename F>
__device__ __forceinline__ void drain_out_bf16(const TcParams& p, uint32_t buf, int m0, int n0,
                                               uint32_t t_acc, int quarter, int c_begin, int c_end, int lane, F release) {
  const int mw = m0 + quarter * 32, m = mw + lane;
  const bool row_ok = m < p.M;
  const uint32_t t_row = t_acc + ((uint32_t)(quarter * 32) << 16);
  if (n0 + c_begin >= p.N || mw >= p.M) { release(); return; }
  const float f = p.row_scale && row_ok ? p.row_scale[m] : 1.f;
#pragma unroll 1
  for (int c0 = c_begin; c0 < c_end; c0 += 64) {
    const int nb = n0 + c0;
    if (nb >= p.N) break;                  // warp-uniform
    uint32_t o[32];
#pragma unroll
    for (int h = 0; h < 2; ++h) {          // 32 columns at a time: with the partial sums, 64 do not fit the registers
      uint32_t r[32];
      tmem_ld32(t_row + c0 + 32 * h, r);
      if (p.aux) {
        const float* src = (const float*)p.aux + (long long)m * p.ldaux + nb + 32 * h;
        uint32_t x[32];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (row_ok && nb + 32 * h + 8 * j < p.N) ld_v8(x + 8 * j, src + 8 * j);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (row_ok && nb + 32 * h + (j & ~7) < p.N) r[j] = __float_as_uint(__uint_as_float(x[j]) + __uint_as_float(r[j]));
      } else {
        tmem_ld_wait();
      }
      if (h == 1 && (c0 + 64 >= c_end || nb + 64 >= p.N)) release();
#pragma unroll
      for (int j = 0; j < 16; ++j) o[16 * h + j] = pack2_bf16(f * __uint_as_float(r[2 * j]), f * __uint_as_float(r[2 * j + 1]));
    }
    store_group<64>((bf16*)p.C + (long long)mw * p.ldc + nb, p.ldc, buf, o, p.M - mw, p.N - nb, lane);
  }
}

// fp32 partial sums of a split product, or the running sum of several chunks (EPI_RESID_F32, aux may be C): N is
// a multiple of 8, rows are 32-byte aligned
template <typename F>
__device__ __forceinline__ void drain_f32(const TcParams& p, int m0, int n0, int sp, uint32_t t_acc, int quarter, int c_begin, int c_end,
                                          int lane, F release) {
  const int m = m0 + quarter * 32 + lane;
  const bool row_ok = m < p.M;
  const uint32_t t_row = t_acc + ((uint32_t)(quarter * 32) << 16);
  const bool add = p.epilogue == EPI_RESID_F32;
  if (n0 + c_begin >= p.N) { release(); return; }
#pragma unroll 1
  for (int c0 = c_begin; c0 < c_end; c0 += 32) {
    const int nb = n0 + c0;
    if (nb >= p.N) break;                  // warp-uniform
    uint32_t r[32], x[32];
    tmem_ld32(t_row + c0, r);
    float* dst = (float*)p.C + (long long)sp * p.split_stride + (long long)m * p.ldc + nb;
    const float* src = (const float*)p.aux + (long long)m * p.ldaux + nb;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (add && row_ok && nb + 8 * j < p.N) ld_v8(x + 8 * j, src + 8 * j);
    tmem_ld_wait();
    if (c0 + 32 >= c_end || nb + 32 >= p.N) release();
    if (!row_ok) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (nb + 8 * j >= p.N) break;
      if (add) {
#pragma unroll
        for (int q = 0; q < 8; ++q) r[8 * j + q] = __float_as_uint(__uint_as_float(r[8 * j + q]) + __uint_as_float(x[8 * j + q]));
      }
      st_v8(dst + 8 * j, r + 8 * j);
    }
  }
}
// Drains an accumulator as MODE says; release() hands it back, once its last columns are in registers.  (After the last
// store instead, a block's next product but one waited: 4099 x 32003 x 768 163 us, 158 now.)
template <int MODE, typename F>
__device__ __forceinline__ void drain(const TcParams& p, uint32_t buf, int m0, int n0, int sp, uint32_t t_acc, int quarter,
                                      int c_begin, int c_end, int lane, F release) {
  if constexpr (MODE == DRAIN_COLS) {
    drain_cols(p, m0, n0, sp, t_acc, quarter, c_begin, c_end, lane);
    release();
  } else if constexpr (MODE == DRAIN_PIECES) {
    drain_pieces(p, buf, m0, n0, t_acc, quarter, c_begin, c_end, lane, release);
  } else {
    if (p.epilogue == EPI_OUT_BF16) drain_out_bf16(p, buf, m0, n0, t_acc, quarter, c_begin, c_end, lane, release);
    else drain_f32(p, m0, n0, sp, t_acc, quarter, c_begin, c_end, lane, release);
  }
}

}  // namespace gemm_tc_detail
