// The pair of norms around a block's end, fused with its gate and the residual scale:
//
//   n = N(y) g1 + b1      norm of the block's output y
//   r' = a r + gate * n   gated, onto the scaled residual stream
//   h = N(r') g2 + b2     norm that the next block (or the head) reads
//
// N is LayerNorm or RMSNorm; gate has a row for every `gate_rows` consecutive rows of y.  Backward,
// with dh and the residual's gradient dr':
//
//   G = dr' + N'(dh g2; r')     dr = a G     dy = N'(gate G g1; y)
//   dgate = sum G n   dg1 = sum gate G yhat   db1 = sum gate G   dg2 = sum dh rhat   db2 = sum dh
//
// Both passes read each input once and write each output once: 12 and 18 bytes per element, so HBM
// bounds them.  A "unit" of LANES threads owns a contiguous range of rows; a thread owns CH chunks of 4
// columns of all of them (16 bytes of fp32, 8 of bf16: neighbours are adjacent in both).  So gains,
// shifts and gate stay in registers over the rows, and the parameter sums of the backward pass are
// running sums in registers, which the units of a block add up in shared memory and a second small kernel over
// the blocks, in a fixed order (no atomics).  (With a unit's sums written by itself, 16384 x 64 took 17.7 us where
// it takes 9.5, and 2041 x 768 with 13 gates 14.1 where it takes 11.6.)
// Rows arrive through a ring of cp.async copies in shared memory: a unit works on one row at a time, two to four
// sums over its threads one after the other, and loads for it would wait as long again.
// LANES is a compile-time constant: with the loops over lanes and warps left to run time the same
// kernel issued 675 instructions per warp and row and took 84 us at 8192 x 2048 where it takes 38.
#include <algorithm>
#include "../../include/ppu.h"
#include "common.cuh"

int ppu_fail(int code, const char* fmt, ...);

namespace {

constexpr int MAX_D = 4096;
// 8 columns a thread, and as many threads on an SM as the registers then allow.  8192 x 2048, inputs and outputs beyond
// the L2: forward 38.2 us with 768 threads of 80 registers, 42.9 with 1024 of 64 (spilling), 49 with 16 columns
// a thread (384 threads of 145 registers); backward 55.3 us with 512 threads of 128 registers, 68 with 256, 76 with
// 4 columns a thread.  Three rows in flight do as well as four.
constexpr int CH = 2, FWD_THREADS = 768, BWD_THREADS = 512;

struct NormArgs {
  const bf16 *y, *dh;
  const float *r, *dr;               // forward: residual in; backward: r' (saved) and its gradient (may be null)
  const float *gate, *g1, *b1, *g2, *b2;
  float* r_out; bf16 *h, *dy; float* dr_out;
  float4* stats;                     // {mean1, rstd1, mean2, rstd2} per row
  float scale, eps;
  int T, d, gate_rows, layer;
  int deal_rows;                     // rows dealt to the units as one (1, or the rows of a group)
  int units, blocks;
  int per_group;                     // units that share a group of gate rows (0: units own whole groups / plain rows)
  int join_gate;                     // the units of a block share a group
  float* partial;                    // [4][blocks][d]: dg1, db1, dg2, db2; then dgate: [blocks or units][d]
  float* dgate;
};

__device__ __forceinline__ void cp16(uint32_t smem, const void* gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(gmem) : "memory");
}
__device__ __forceinline__ void cp8(uint32_t smem, const void* gmem) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem), "l"(gmem) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void from_bf4(const uint2 u, float* f) {
  const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x));
  const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
  f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
}
__device__ __forceinline__ uint2 to_bf4(const float* f) {
  __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
  return make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
}
__device__ __forceinline__ void from_f4(const float4& v, float* f) { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
__device__ __forceinline__ float4 to_f4(const float* f) { return make_float4(f[0], f[1], f[2], f[3]); }

// Units of a block: about 128 threads forward, 256 backward, where they share their sums (with 512 throughout 16
// rows of 2048 take 7.0 us for 5.5), or 480 of 96, five units to an SM.
constexpr int units_of(int lanes, bool bwd) { return !bwd ? (lanes <= 128 ? 128 / lanes : 1) : lanes == 96 ? 5 : lanes <= 128 ? 256 / lanes : 1; }
template <int LANES, bool BWD> struct Layout {
  static constexpr int UNITS = units_of(LANES, BWD);
  static constexpr int BLOCK = LANES * UNITS;
  static constexpr int WARPS = LANES > 32 ? LANES / 32 : 1;
};

// Sums of a unit's threads.  Within a warp by shuffles; a unit of several warps then through shared
// memory and the unit's own named barrier.  Two buffers in turn: a thread that is back for the next sum
// writes the other one, and the one after that lies behind a barrier that all readers of this have passed.
template <int LANES, int N> struct UnitSum {
  static constexpr int W = LANES > 32 ? LANES / 32 : 1;
  float* buf;                       // [2][W][N] of this unit
  int bar, lane, warp, turn;
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int o = LANES < 32 ? LANES / 2 : 16; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if constexpr (W > 1) {
      float* b = buf + turn;
      turn ^= W * N;
      if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) b[warp * N + i] = v[i];
      asm volatile("bar.sync %0, %1;" ::"r"(bar), "n"(LANES) : "memory");
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += b[w * N + i];
    }
  }
};

// where a unit's threads stand and which rows are its own
struct Unit {
  int tid, unit;                    // thread of the unit, index of the unit
  int lo, hi;                       // rows
  int group;                        // gate row of all of them (units that share a group)
};
template <int LANES, bool BWD>
__device__ __forceinline__ Unit my_unit(const NormArgs& a) {
  Unit u;
  u.tid = threadIdx.x % LANES;
  // (rows that are not shared out by groups go to all blocks before a block gets a second unit's)
  if (BWD && a.per_group == 0) u.unit = blockIdx.x + threadIdx.x / LANES * a.blocks;
  else u.unit = blockIdx.x * Layout<LANES, BWD>::UNITS + threadIdx.x / LANES;
  u.group = u.lo = u.hi = 0;
  if (u.unit >= a.units) return u;
  if (a.per_group > 0) {            // a share of one group's rows
    u.group = u.unit / a.per_group;
    const int part = u.unit % a.per_group, g0 = u.group * a.gate_rows;
    const int64_t n = min(a.gate_rows, a.T - g0);
    u.lo = g0 + (int)(n * part / a.per_group);
    u.hi = g0 + (int)(n * (part + 1) / a.per_group);
  } else {                          // whole groups (of one row where there is no sum over a group)
    const int64_t rows = a.deal_rows, groups = (a.T + rows - 1) / rows;
    u.lo = (int)(groups * u.unit / a.units * rows);
    u.hi = (int)min(groups * (u.unit + 1) / a.units * rows, (int64_t)a.T);
  }
  return u;
}
// rows that a unit's turns cover: threads of several units in a warp go on together, shuffles need all lanes
template <int LANES> __device__ __forceinline__ int turns_of(const Unit& u) {
  if constexpr (LANES < 32) return __reduce_max_sync(0xffffffffu, u.hi - u.lo);
  return u.hi - u.lo;
}

// a vector's chunks of this thread
template <int LANES>
__device__ __forceinline__ void load_vector(const float* p, int tid, int d, float (&f)[CH][4]) {
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int col = 4 * (tid + LANES * c);
    if (col < d) from_f4(*reinterpret_cast<const float4*>(p + col), f[c]);
  }
}

// A row in flight: per thread and chunk 8 bytes of each bf16 and 16 of each fp32 operand.  A thread
// copies and reads its own columns alone, so there is no barrier.
template <bool BWD, int GATE> struct Ring {
  static constexpr int NB = BWD ? 2 : 1, NF = (BWD ? 2 : 1) + (GATE == 2 ? 1 : 0);
  static constexpr int BYTES = CH * (8 * NB + 16 * NF);      // per thread
  static constexpr int STAGES = 3;
};

// GATE: 0 none, 1 one row for all rows, 2 read with each row
template <int LANES, int GATE>
__global__ void __launch_bounds__(Layout<LANES, false>::BLOCK, FWD_THREADS / Layout<LANES, false>::BLOCK) norm_gate_fwd_kernel(const NormArgs a) {
  pdl_wait(); pdl_trigger();
  constexpr int BLOCK = Layout<LANES, false>::BLOCK;
  using R = Ring<false, GATE>;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float s_sum[Layout<LANES, false>::UNITS][2 * Layout<LANES, false>::WARPS];
  const Unit u = my_unit<LANES, false>(a);
  const int slot = threadIdx.x / LANES;
  UnitSum<LANES, 1> sum{s_sum[slot], 1 + slot, (int)threadIdx.x & 31, u.tid >> 5, 0};
  bool on[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) on[c] = 4 * (u.tid + LANES * c) < a.d;
  // stage s: [NF * CH][BLOCK] of 16 bytes (r, then the gate), then [CH][BLOCK] of 8 bytes (y)
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem);
  auto f_off = [&](int s, int i) { return s * (R::BYTES * BLOCK) + (i * BLOCK + (int)threadIdx.x) * 16; };
  auto b_off = [&](int s, int i) { return s * (R::BYTES * BLOCK) + R::NF * CH * BLOCK * 16 + (i * BLOCK + (int)threadIdx.x) * 8; };
  auto fetch = [&](int t, int s) {
    if (t < u.hi) {
      const int64_t e = (int64_t)t * a.d + 4 * u.tid;
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (on[c]) {
          cp8(ring + b_off(s, c), a.y + e + 4 * LANES * c);
          cp16(ring + f_off(s, c), a.r + e + 4 * LANES * c);
        }
      if (GATE == 2) {
        const float* g = a.gate + (int64_t)(t / a.gate_rows) * a.d + 4 * u.tid;
#pragma unroll
        for (int c = 0; c < CH; ++c) if (on[c]) cp16(ring + f_off(s, CH + c), g + 4 * LANES * c);
      }
    }
    cp_commit();
  };
#pragma unroll
  for (int s = 0; s < R::STAGES - 1; ++s) fetch(u.lo + s, s);
  float g1[CH][4] = {}, b1[CH][4] = {}, g2[CH][4] = {}, b2[CH][4] = {};
  if (u.lo < u.hi) {
    load_vector<LANES>(a.g1, u.tid, a.d, g1);
    if (a.b1) load_vector<LANES>(a.b1, u.tid, a.d, b1);
    load_vector<LANES>(a.g2, u.tid, a.d, g2);
    if (a.b2) load_vector<LANES>(a.b2, u.tid, a.d, b2);
    if (GATE == 1) {
      float gt[CH][4] = {};
      load_vector<LANES>(a.gate, u.tid, a.d, gt);
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) { g1[c][j] *= gt[c][j]; b1[c][j] *= gt[c][j]; }
    }
  }
  const float inv_d = 1.f / a.d;
  // mean, then the squares about it: one pass over the squares alone would lose digits where the mean is large
  auto moments = [&](const float (&x)[CH][4], float& mean, float& rstd) {
    mean = 0.f;
    if (a.layer) {
      float v[1] = {0.f};
#pragma unroll
      for (int c = 0; c < CH; ++c) v[0] += (x[c][0] + x[c][1]) + (x[c][2] + x[c][3]);
      sum(v);
      mean = v[0] * inv_d;
    }
    float v[1] = {0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float q = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) { const float e = x[c][j] - mean; q = fmaf(e, e, q); }
      if (on[c]) v[0] += q;
    }
    sum(v);
    rstd = rsqrtf(v[0] * inv_d + a.eps);
  };
  const int turns = turns_of<LANES>(u);
  int s = 0;
  for (int i = 0; i < turns; ++i) {
    const int t = u.lo + i;
    const bool row = t < u.hi;
    cp_wait<R::STAGES - 2>();
    float y[CH][4] = {}, r[CH][4] = {}, gt[CH][4] = {};
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (on[c] && row) {
        from_bf4(*reinterpret_cast<const uint2*>(smem + b_off(s, c)), y[c]);
        from_f4(*reinterpret_cast<const float4*>(smem + f_off(s, c)), r[c]);
        if (GATE == 2) from_f4(*reinterpret_cast<const float4*>(smem + f_off(s, CH + c)), gt[c]);
      }
    fetch(t + R::STAGES - 1, s == 0 ? R::STAGES - 1 : s - 1);
    s = s == R::STAGES - 1 ? 0 : s + 1;
    float m1, r1, m2, r2;
    moments(y, m1, r1);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float n = fmaf((y[c][j] - m1) * r1, g1[c][j], b1[c][j]);
        if (GATE == 2) n *= gt[c][j];
        r[c][j] = fmaf(a.scale, r[c][j], n);
      }
    // (columns past the row's end have zero gains and shifts: r' = 0 there)
    moments(r, m2, r2);
    if (row) {
      const int64_t e = (int64_t)t * a.d + 4 * u.tid;
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (on[c]) {
          *reinterpret_cast<float4*>(a.r_out + e + 4 * LANES * c) = to_f4(r[c]);
#pragma unroll
          for (int j = 0; j < 4; ++j) r[c][j] = fmaf((r[c][j] - m2) * r2, g2[c][j], b2[c][j]);
          *reinterpret_cast<uint2*>(a.h + e + 4 * LANES * c) = to_bf4(r[c]);
        }
      if (u.tid == 0) a.stats[t] = make_float4(m1, r1, m2, r2);
    }
  }
}

// GATE: 0 none, 1 one row for all of the unit's rows, 2 read with each row, its gradient written at the end of each group
template <int LANES, int GATE>
__global__ void __launch_bounds__(Layout<LANES, true>::BLOCK, BWD_THREADS / Layout<LANES, true>::BLOCK) norm_gate_bwd_kernel(const NormArgs a) {
  pdl_wait(); pdl_trigger();
  constexpr int BLOCK = Layout<LANES, true>::BLOCK;
  using R = Ring<true, GATE>;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float s_sum[Layout<LANES, true>::UNITS][2 * 2 * Layout<LANES, true>::WARPS];
  const Unit u = my_unit<LANES, true>(a);
  const int slot = threadIdx.x / LANES;
  UnitSum<LANES, 2> sum{s_sum[slot], 1 + slot, (int)threadIdx.x & 31, u.tid >> 5, 0};
  bool on[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) on[c] = 4 * (u.tid + LANES * c) < a.d;
  // stage s: [NF * CH][BLOCK] of 16 bytes (r', dr', the gate), then [2 CH][BLOCK] of 8 bytes (dh, y)
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem);
  auto f_off = [&](int s, int i) { return s * (R::BYTES * BLOCK) + (i * BLOCK + (int)threadIdx.x) * 16; };
  auto b_off = [&](int s, int i) { return s * (R::BYTES * BLOCK) + R::NF * CH * BLOCK * 16 + (i * BLOCK + (int)threadIdx.x) * 8; };
  auto fetch = [&](int t, int s) {
    if (t < u.hi) {
      const int64_t e = (int64_t)t * a.d + 4 * u.tid;
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (on[c]) {
          cp8(ring + b_off(s, c), a.dh + e + 4 * LANES * c);
          cp8(ring + b_off(s, CH + c), a.y + e + 4 * LANES * c);
          cp16(ring + f_off(s, c), a.r + e + 4 * LANES * c);
          if (a.dr) cp16(ring + f_off(s, CH + c), a.dr + e + 4 * LANES * c);
        }
      if (GATE == 2) {
        const float* g = a.gate + (int64_t)(t / a.gate_rows) * a.d + 4 * u.tid;
#pragma unroll
        for (int c = 0; c < CH; ++c) if (on[c]) cp16(ring + f_off(s, 2 * CH + c), g + 4 * LANES * c);
      }
    }
    cp_commit();
  };
#pragma unroll
  for (int s = 0; s < R::STAGES - 1; ++s) fetch(u.lo + s, s);
  float gg[CH][4] = {}, g2[CH][4] = {};                      // gate g1 (g1 where the gate comes with each row)
  if (u.lo < u.hi) {
    load_vector<LANES>(a.g1, u.tid, a.d, gg);
    load_vector<LANES>(a.g2, u.tid, a.d, g2);
    if (GATE == 1) {
      float gt[CH][4] = {};
      load_vector<LANES>(a.gate + (int64_t)u.group * a.d, u.tid, a.d, gt);
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) gg[c][j] *= gt[c][j];
    }
  }
  // running sums: A = sum G yhat, B = sum G (of the group, where the gate comes with each row),
  // C = sum dh rhat, D = sum dh, and there PA, PB = sums of gate G yhat, gate G
  float A[CH][4] = {}, B[CH][4] = {}, C[CH][4] = {}, D[CH][4] = {}, PA[CH][4] = {}, PB[CH][4] = {};
  const float inv_d = 1.f / a.d;
  const int turns = turns_of<LANES>(u);
  int s = 0;
  float4 st = u.lo < u.hi ? a.stats[u.lo] : make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < turns; ++i) {
    const int t = u.lo + i;
    const bool row = t < u.hi;
    cp_wait<R::STAGES - 2>();
    // columns past the row's end, and turns past the unit's rows: zeros throughout
    float dh[CH][4] = {}, y[CH][4] = {}, r[CH][4] = {}, G[CH][4] = {}, gt[CH][4] = {};
    const float4 now = row ? st : make_float4(0.f, 0.f, 0.f, 0.f);
    if (t + 1 < u.hi) st = a.stats[t + 1];
    float v[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (on[c] && row) {
        from_bf4(*reinterpret_cast<const uint2*>(smem + b_off(s, c)), dh[c]);
        from_bf4(*reinterpret_cast<const uint2*>(smem + b_off(s, CH + c)), y[c]);
        from_f4(*reinterpret_cast<const float4*>(smem + f_off(s, c)), r[c]);
        if (a.dr) from_f4(*reinterpret_cast<const float4*>(smem + f_off(s, CH + c)), G[c]);
        if (GATE == 2) from_f4(*reinterpret_cast<const float4*>(smem + f_off(s, 2 * CH + c)), gt[c]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          r[c][j] = (r[c][j] - now.z) * now.w;                // rhat
          y[c][j] = (y[c][j] - now.x) * now.y;                // yhat
          C[c][j] = fmaf(dh[c][j], r[c][j], C[c][j]);
          D[c][j] += dh[c][j];
          dh[c][j] *= g2[c][j];
          v[0] += dh[c][j];
          v[1] = fmaf(dh[c][j], r[c][j], v[1]);
        }
      }
    fetch(t + R::STAGES - 1, s == 0 ? R::STAGES - 1 : s - 1);
    s = s == R::STAGES - 1 ? 0 : s + 1;
    sum(v);
    const float mean = a.layer ? v[0] * inv_d : 0.f, dot = v[1] * inv_d;
    float w[2] = {0.f, 0.f};
    const int64_t e = (int64_t)t * a.d + 4 * u.tid;
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (on[c] && row) {
        float o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          G[c][j] = fmaf(now.w, fmaf(-r[c][j], dot, dh[c][j] - mean), G[c][j]);
          o[j] = a.scale * G[c][j];
          A[c][j] = fmaf(G[c][j], y[c][j], A[c][j]);
          B[c][j] += G[c][j];
          G[c][j] *= gg[c][j];
          if (GATE == 2) G[c][j] *= gt[c][j];
          w[0] += G[c][j];
          w[1] = fmaf(G[c][j], y[c][j], w[1]);
        }
        *reinterpret_cast<float4*>(a.dr_out + e + 4 * LANES * c) = to_f4(o);
      }
    sum(w);
    const float mean1 = a.layer ? w[0] * inv_d : 0.f, dot1 = w[1] * inv_d;
    const bool last = GATE == 2 && row && ((t + 1) % a.gate_rows == 0 || t + 1 == a.T);      // the group's last row
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (on[c] && row) {
        float o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = now.y * fmaf(-y[c][j], dot1, G[c][j] - mean1);
        *reinterpret_cast<uint2*>(a.dy + e + 4 * LANES * c) = to_bf4(o);
        if (last) {
          const int col = 4 * (u.tid + LANES * c);
          float b1[4] = {};
          if (a.b1) from_f4(*reinterpret_cast<const float4*>(a.b1 + col), b1);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            o[j] = fmaf(gg[c][j], A[c][j], b1[j] * B[c][j]);
            PA[c][j] = fmaf(gt[c][j], A[c][j], PA[c][j]);
            PB[c][j] = fmaf(gt[c][j], B[c][j], PB[c][j]);
            A[c][j] = B[c][j] = 0.f;
          }
          *reinterpret_cast<float4*>(a.dgate + (int64_t)(t / a.gate_rows) * a.d + col) = to_f4(o);
        }
      }
  }
  // the sums of the block's units, added up in order: across a warp's by shuffles, then through shared memory
  constexpr int PLANES = GATE == 1 ? 5 : 4, WIDE = LANES * CH, PARTS = LANES < 32 ? BLOCK / 32 : Layout<LANES, true>::UNITS;
  static_assert(PLANES * PARTS * WIDE * 16 <= R::BYTES * R::STAGES * BLOCK, "sums in the ring's place");
  const int part = LANES < 32 ? (int)threadIdx.x >> 5 : slot;
  const bool writes = LANES >= 32 || (threadIdx.x & 31) < LANES;
  float4* joined = reinterpret_cast<float4*>(smem);          // [plane][part][column / 4]
  if (PARTS > 1) __syncthreads();                            // (the ring has been read)
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float o[4] = {};
    if (GATE == 1 && on[c]) {
      const int col = 4 * (u.tid + LANES * c);
      float gt[4], g1[4], b1[4] = {};
      from_f4(*reinterpret_cast<const float4*>(a.gate + (int64_t)u.group * a.d + col), gt);
      from_f4(*reinterpret_cast<const float4*>(a.g1 + col), g1);
      if (a.b1) from_f4(*reinterpret_cast<const float4*>(a.b1 + col), b1);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        o[j] = fmaf(g1[j], A[c][j], b1[j] * B[c][j]);
        A[c][j] *= gt[j];
        B[c][j] *= gt[j];
      }
      if (!a.join_gate && u.unit < a.units) *reinterpret_cast<float4*>(a.partial + ((int64_t)4 * a.blocks + u.unit) * a.d + col) = to_f4(o);
    }
#pragma unroll
    for (int q = 0; q < PLANES; ++q) {
      float (&v)[4] = q == 0 ? (GATE == 2 ? PA[c] : A[c]) : q == 1 ? (GATE == 2 ? PB[c] : B[c]) : q == 2 ? C[c] : q == 3 ? D[c] : o;
#pragma unroll
      for (int w = LANES; w < 32; w *= 2)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += __shfl_xor_sync(0xffffffffu, v[j], w);
      if (PARTS == 1) {                                      // a block is one unit
        if (on[c] && (q < 4 || a.join_gate))
          *reinterpret_cast<float4*>(a.partial + ((int64_t)q * a.blocks + blockIdx.x) * a.d + 4 * (u.tid + LANES * c)) = to_f4(v);
      } else if (writes) joined[(q * PARTS + part) * WIDE + u.tid + LANES * c] = to_f4(v);
    }
  }
  if (PARTS == 1) return;
  __syncthreads();
  const int n4 = a.d / 4, planes = GATE == 1 && a.join_gate ? 5 : 4;
  for (int i = threadIdx.x; i < planes * n4; i += BLOCK) {
    const int q = i / n4, c4 = i - q * n4;
    float4 v = joined[q * PARTS * WIDE + c4];
#pragma unroll
    for (int w = 1; w < PARTS; ++w) {
      const float4 x = joined[(q * PARTS + w) * WIDE + c4];
      v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    }
    *reinterpret_cast<float4*>(a.partial + ((int64_t)q * a.blocks + blockIdx.x) * a.d + 4 * c4) = v;
  }
}

// parameter gradients from the blocks' partial sums: blockIdx.y = 0..3 the norms' gains and shifts over
// all blocks, 4 + g the gate's row g over its group's parts.  A block takes 128 columns (4 to a lane), a warp
// adds a 32nd of the parts in order, and the 32 sums are added in order.
struct ParamOut { float* out[4]; float* dgate; };
__global__ void __launch_bounds__(1024) norm_gate_params_kernel(const float* partial, const ParamOut po, int blocks, int group_parts, int d) {
  pdl_wait(); pdl_trigger();
  __shared__ float4 sh[32][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int c = blockIdx.x * 128 + 4 * lane;
  const int which = min((int)blockIdx.y, 4), g = (int)blockIdx.y - 4;
  float* out = which == 0 ? po.out[0] : which == 1 ? po.out[1] : which == 2 ? po.out[2] : which == 3 ? po.out[3] : po.dgate + (int64_t)g * d;
  if (!out) return;
  const int n = which < 4 ? blocks : group_parts;
  const int64_t first = which < 4 ? 0 : (int64_t)g * group_parts;
  const float* p = partial + ((int64_t)which * blocks + first) * d + c;
  const int per = (n + 31) / 32, b0 = w * per, b1 = min(n, b0 + per);
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < d) {
#pragma unroll 8
    for (int b = b0; b < b1; ++b) {
      const float4 v = *reinterpret_cast<const float4*>(p + (int64_t)b * d);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  sh[w][lane] = s;
  __syncthreads();
  if (threadIdx.x < 128 && blockIdx.x * 128 + threadIdx.x < d) {
    const float* col = reinterpret_cast<const float*>(sh) + threadIdx.x;
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < 32; ++q) t += col[128 * q];
    out[blockIdx.x * 128 + threadIdx.x] = t;
  }
}

// ---- host ---------------------------------------------------------------------------------------
constexpr int SMS = 148;                      // work is split for a B200 (also where sizes are asked without a device)

struct Shape { int lanes, slots, units, blocks, per_group, join_gate, gate_mode; size_t partial; };

// threads of a unit: the fewest that hold a row, of the sizes that are compiled (with 320 and 384 the forward pass of 8192 x
// 2056 takes 48 us, with 512 79: two units to an SM instead of one)
int lanes_for(int d) {
  for (int l : {4, 8, 16, 32, 64, 96, 128, 192, 256, 320, 384}) if (4 * CH * l >= d) return l;
  return 512;
}
// rows are dealt to as many threads per SM as are resident there
Shape make_shape(int T, int d, int has_gate, int gate_rows, bool backward) {
  Shape s = {};
  s.lanes = lanes_for(d);
  const int64_t groups = has_gate ? ((int64_t)T + gate_rows - 1) / gate_rows : 1;
  s.gate_mode = !has_gate ? 0 : groups == 1 ? 1 : 2;
  if (!backward) {
    s.units = (int)std::min<int64_t>(T, (int64_t)SMS * (FWD_THREADS / s.lanes));
    return s;
  }
  const int64_t slots = units_of(s.lanes, true), target = SMS * (BWD_THREADS / s.lanes);     // units of a block, of the machine
  if (has_gate && groups < target) {                   // several units to a group, whole blocks of them where it has that many
    s.gate_mode = 1;
    int64_t per = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(gate_rows, T), target / groups));
    s.join_gate = per % slots <= per / 8;              // (else too many units would be left without rows)
    if (s.join_gate) per = per / slots * slots;
    s.per_group = (int)per;
    s.units = (int)(groups * per);
    s.blocks = (int)((s.units + slots - 1) / slots);
  } else {                                             // whole groups (more groups than units) or plain rows
    const int64_t n = has_gate ? groups : T;
    s.blocks = (int)std::min<int64_t>(target / slots, n);
    s.units = (int)(s.blocks * std::min<int64_t>(slots, (n + s.blocks - 1) / s.blocks));
  }
  s.slots = (int)slots;
  s.partial = (4 * (size_t)s.blocks + (s.gate_mode == 1 ? (s.join_gate ? s.blocks : s.units) : 0)) * d * 4;
  return s;
}

int check_norm(int T, int d, const float* gate, int gate_rows, int kind, float eps) {
  if (T < 0 || d < 1) return ppu_fail(PPU_EINVAL, "negative or empty size");
  if (d % 8 || d > MAX_D) return ppu_fail(PPU_ESHAPE, "d must be a multiple of 8 up to %d (got %d)", MAX_D, d);
  if (T > (1 << 24)) return ppu_fail(PPU_ESHAPE, "at most 2^24 rows");
  if (gate && gate_rows < 1) return ppu_fail(PPU_EINVAL, "a gate needs gate_rows >= 1");
  if (kind != PPU_NORM_LAYER && kind != PPU_NORM_RMS) return ppu_fail(PPU_EINVAL, "unknown norm kind %d", kind);
  if (!(eps >= 0.f)) return ppu_fail(PPU_EINVAL, "eps must not be negative");
  return PPU_OK;
}
bool misaligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps) if (reinterpret_cast<uintptr_t>(p) & 15) return true;
  return false;
}

#define CUDA_OK(call)                                                                    \
  do {                                                                                   \
    cudaError_t e_ = (call);                                                             \
    if (e_ != cudaSuccess)                                                               \
      return ppu_fail(PPU_ECUDA, "%s failed: %s", #call, cudaGetErrorString(e_));        \
  } while (0)

template <int LANES, int GATE, bool BWD>
int launch_norm(const NormArgs& a, cudaStream_t st) {
  using L = Layout<LANES, BWD>;
  using R = Ring<BWD, GATE>;
  constexpr int bytes = R::BYTES * R::STAGES * L::BLOCK;
  static_assert(bytes <= 220 * 1024, "shared memory of a block");
  static PerDeviceFlag attr;
  void (*kernel)(NormArgs);
  if constexpr (BWD) kernel = norm_gate_bwd_kernel<LANES, GATE>;
  else kernel = norm_gate_fwd_kernel<LANES, GATE>;
  if (!ppu_set_smem_once(attr, kernel, bytes)) return ppu_fail(PPU_ECUDA, "shared memory limit not accepted");
  CUDA_OK(ppu_launch_dependent(kernel, BWD ? a.blocks : (a.units + L::UNITS - 1) / L::UNITS, L::BLOCK, bytes, st, a));
  return PPU_OK;
}
template <int LANES, bool BWD>
int launch_gate(const NormArgs& a, int gate_mode, cudaStream_t st) {
  if (gate_mode == 0) return launch_norm<LANES, 0, BWD>(a, st);
  if (gate_mode == 1) return launch_norm<LANES, 1, BWD>(a, st);
  return launch_norm<LANES, 2, BWD>(a, st);
}
template <bool BWD>
int dispatch(const NormArgs& a, const Shape& s, cudaStream_t st) {
  switch (s.lanes) {
#define LANES_CASE(L) case L: return launch_gate<L, BWD>(a, s.gate_mode, st);
    LANES_CASE(4) LANES_CASE(8) LANES_CASE(16) LANES_CASE(32) LANES_CASE(64) LANES_CASE(96) LANES_CASE(128) LANES_CASE(192)
    LANES_CASE(256) LANES_CASE(320) LANES_CASE(384)
#undef LANES_CASE
    default: break;
  }
  return launch_gate<512, BWD>(a, s.gate_mode, st);
}

}  // namespace

extern "C" int ppu_norm_gate_fwd(const void* y, const float* r, const float* gate, int gate_rows,
                                 const float* post_gain, const float* post_shift, const float* pre_gain,
                                 const float* pre_shift, int kind, float res_scale, float eps, float* r_out,
                                 void* h, float* stats, int T, int d, void* cuda_stream) {
  const int rc = check_norm(T, d, gate, gate_rows, kind, eps);
  if (rc) return rc;
  if (T == 0) return PPU_OK;
  if (!y || !r || !post_gain || !pre_gain || !r_out || !h || !stats) return ppu_fail(PPU_EINVAL, "null operand");
  if (misaligned({y, r, gate, post_gain, post_shift, pre_gain, pre_shift, r_out, h, stats}))
    return ppu_fail(PPU_EINVAL, "operands must be 16-byte aligned");
  const Shape s = make_shape(T, d, gate != nullptr, gate_rows, false);
  NormArgs a = {};
  a.y = (const bf16*)y; a.r = r; a.gate = gate; a.g1 = post_gain; a.b1 = post_shift; a.g2 = pre_gain; a.b2 = pre_shift;
  a.r_out = r_out; a.h = (bf16*)h; a.stats = (float4*)stats; a.scale = res_scale; a.eps = eps;
  a.T = T; a.d = d; a.gate_rows = gate ? gate_rows : 1; a.layer = kind == PPU_NORM_LAYER; a.units = s.units; a.per_group = 0;
  a.deal_rows = 1;                             // (no sums over a group)
  return dispatch<false>(a, s, (cudaStream_t)cuda_stream);
}

extern "C" int ppu_norm_gate_query_bytes(int T, int d, int gate_rows, size_t* bytes) {
  if (!bytes) return ppu_fail(PPU_EINVAL, "bytes is null");
  const int rc = check_norm(T, d, nullptr, 0, PPU_NORM_LAYER, 0.f);
  if (rc) return rc;
  if (gate_rows < 0) return ppu_fail(PPU_EINVAL, "negative gate_rows");
  *bytes = T ? make_shape(T, d, gate_rows > 0, gate_rows, true).partial : 0;
  return PPU_OK;
}

extern "C" int ppu_norm_gate_bwd(const void* dh, const float* dr_out, const void* y, const float* r_out,
                                 const float* stats, const float* gate, int gate_rows, const float* post_gain,
                                 const float* post_shift, const float* pre_gain, int kind, float res_scale,
                                 void* dy, float* dr, float* dpost_gain, float* dpost_shift, float* dpre_gain,
                                 float* dpre_shift, float* dgate, int T, int d, void* workspace,
                                 size_t workspace_bytes, void* cuda_stream) {
  const int rc = check_norm(T, d, gate, gate_rows, kind, 0.f);
  if (rc) return rc;
  if (!dpost_gain || !dpre_gain) return ppu_fail(PPU_EINVAL, "null operand");
  if ((gate == nullptr) != (dgate == nullptr)) return ppu_fail(PPU_EINVAL, "gate and dgate go together");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (T == 0) {                                // sums over nothing
    for (float* p : {dpost_gain, dpost_shift, dpre_gain, dpre_shift})
      if (p) CUDA_OK(cudaMemsetAsync(p, 0, (size_t)d * 4, st));
    return PPU_OK;
  }
  if (!dh || !y || !r_out || !stats || !post_gain || !pre_gain || !dy || !dr || !workspace) return ppu_fail(PPU_EINVAL, "null operand");
  if (misaligned({dh, dr_out, y, r_out, stats, gate, post_gain, post_shift, pre_gain, dy, dr, dgate, workspace}))
    return ppu_fail(PPU_EINVAL, "operands must be 16-byte aligned");
  const Shape s = make_shape(T, d, gate != nullptr, gate_rows, true);
  if (workspace_bytes < s.partial) return ppu_fail(PPU_ENOMEM, "workspace has %zu bytes, %zu needed", workspace_bytes, s.partial);
  NormArgs a = {};
  a.dh = (const bf16*)dh; a.dr = dr_out; a.y = (const bf16*)y; a.r = r_out; a.stats = (float4*)stats;
  a.gate = gate; a.g1 = post_gain; a.b1 = post_shift; a.g2 = pre_gain; a.dy = (bf16*)dy; a.dr_out = dr;
  a.scale = res_scale; a.T = T; a.d = d; a.gate_rows = gate ? gate_rows : 1; a.layer = kind == PPU_NORM_LAYER; a.units = s.units;
  a.deal_rows = s.gate_mode == 2 ? gate_rows : 1; a.per_group = s.per_group; a.blocks = s.blocks; a.join_gate = s.join_gate; a.partial = (float*)workspace; a.dgate = dgate;
  const int rc2 = dispatch<true>(a, s, st);
  if (rc2) return rc2;
  const int groups = s.gate_mode == 1 ? s.units / s.per_group : 0;      // gate rows still to be summed
  const int parts = s.join_gate ? s.per_group / s.slots : s.per_group;
  const ParamOut po = {{dpost_gain, dpost_shift, dpre_gain, dpre_shift}, dgate};
  CUDA_OK(ppu_launch_dependent(norm_gate_params_kernel, dim3((d + 127) / 128, 4 + groups), 1024, 0, st, a.partial, po, s.blocks, parts, d));
  return PPU_OK;
}
