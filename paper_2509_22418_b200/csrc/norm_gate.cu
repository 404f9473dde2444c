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
// bounds them.  A "unit" of 8 to 512 threads owns a contiguous range of rows; a thread owns 8 columns
// of all of them.  So gains, shifts and gate stay in registers over the rows, and the five parameter
// sums of the backward pass are running sums in registers, written once per unit and added in a fixed
// order by a second small kernel (no atomics).  Rows arrive through a ring of cp.async copies in shared
// memory, three rows ahead: a unit works on one row at a time and would otherwise wait for each.
// A unit's threads meet at a barrier of their own, so a block may hold several units (short rows).
#include <algorithm>
#include "../../include/ppu.h"
#include "common.cuh"

int ppu_fail(int code, const char* fmt, ...);

namespace {

constexpr int MAX_D = 4096;
// rows in flight of a unit: with two blocks of 256 threads on an SM (one of 512) what fits its shared memory
template <bool BWD, int GATE> struct Ring {
  static constexpr int BYTES = (BWD ? 96 : 48) + (GATE == 2 ? 32 : 0);   // per thread and row
  static constexpr int STAGES = BWD && GATE == 2 ? 3 : 4;
};

struct NormArgs {
  const bf16 *y, *dh;
  const float *r, *dr;               // forward: residual in; backward: r' (saved) and its gradient (may be null)
  const float *gate, *g1, *b1, *g2, *b2;
  float* r_out; bf16 *h, *dy; float* dr_out;
  float4* stats;                     // {mean1, rstd1, mean2, rstd2} per row
  float scale, eps;
  int T, d, gate_rows;
  int deal_rows;                     // rows dealt to the units as one (1, or the rows of a group)
  int tpr;                           // threads of a unit
  int units;
  int per_group;                     // units that share a group of gate rows (0: units own whole groups / plain rows)
  float* partial;                    // [5][units][d]: dg1, db1, dg2, db2, dgate
  float* dgate;
};

__device__ __forceinline__ void cp16(void* smem, const void* gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem)
               : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void bf8(const void* p, float* f) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const __nv_bfloat162* q = reinterpret_cast<const __nv_bfloat162*>(&u);
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 t = __bfloat1622float2(q[i]); f[2 * i] = t.x; f[2 * i + 1] = t.y; }
}
__device__ __forceinline__ void put_bf8(bf16* p, const float* f) {
  uint4 u;
  __nv_bfloat162* q = reinterpret_cast<__nv_bfloat162*>(&u);
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = u;
}
__device__ __forceinline__ void f8(const float* p, float* f) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void put_f8(float* p, const float* f) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

// Sums of a unit's threads.  Within a warp by shuffles; a unit of several warps then through shared
// memory and the unit's own named barrier.  Two buffers in turn: a thread that is back for the next sum
// writes the other one, and the one after that lies behind a barrier that all readers of this have passed.
struct UnitSum {
  float2* buf;                      // [2][16] of this unit
  int tpr, bar, lane, warp, turn;
  __device__ float2 operator()(float2 v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (o < tpr) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
      }
    if (tpr <= 32) return v;
    float2* b = buf + 16 * turn;
    turn ^= 1;
    if (lane == 0) b[warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(tpr) : "memory");
    float2 s = b[0];
    for (int w = 1; w < (tpr >> 5); ++w) { s.x += b[w].x; s.y += b[w].y; }
    return s;
  }
};

// where a unit's threads stand and which rows are its own
struct Unit {
  int tid, unit;                    // thread of the unit, index of the unit
  int64_t lo, hi;                   // rows
  int group;                        // gate row of all of them (units that share a group)
};
__device__ __forceinline__ Unit my_unit(const NormArgs& a) {
  Unit u;
  u.tid = threadIdx.x % a.tpr;
  u.unit = blockIdx.x * (blockDim.x / a.tpr) + threadIdx.x / a.tpr;
  u.group = 0;
  if (u.unit >= a.units) { u.lo = u.hi = 0; return u; }
  if (a.per_group > 0) {            // a share of one group's rows
    u.group = u.unit / a.per_group;
    const int part = u.unit % a.per_group;
    const int64_t g0 = (int64_t)u.group * a.gate_rows, n = min((int64_t)a.gate_rows, a.T - g0);
    u.lo = g0 + n * part / a.per_group;
    u.hi = g0 + n * (part + 1) / a.per_group;
  } else {                          // whole groups (of one row where there is no sum over a group)
    const int64_t rows = a.deal_rows, groups = (a.T + rows - 1) / rows;
    u.lo = groups * u.unit / a.units * rows;
    u.hi = min(groups * (u.unit + 1) / a.units * rows, (int64_t)a.T);
  }
  return u;
}

// GATE: 0 none, 1 one row for all of the unit's rows, 2 read with each row
template <bool LAYER, int GATE>
__global__ void __launch_bounds__(MAX_D / 8) norm_gate_fwd_kernel(const NormArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float2 s_sum[4][2 * 16];
  const Unit u = my_unit(a);
  const int lane = threadIdx.x & 31, slot = threadIdx.x / a.tpr;
  UnitSum sum{s_sum[a.tpr > 32 ? slot : 0], a.tpr, 1 + slot, lane, (int)u.tid >> 5, 0};
  const int col = u.tid * 8;
  const bool on = col < a.d;
  constexpr int BYTES = Ring<false, GATE>::BYTES, STAGES = Ring<false, GATE>::STAGES;   // y, r, gate
  // a thread copies and reads its own 8 columns: no other thread's data, so no barrier
  auto at = [&](int s, int off) { return smem + ((size_t)(s * BYTES + off) * blockDim.x); };
  auto fetch = [&](int64_t t, int s) {
    if (t < u.hi && on) {
      const int64_t e = t * a.d + col;
      cp16(at(s, 0) + 16 * threadIdx.x, a.y + e);
      cp16(at(s, 16) + 16 * threadIdx.x, a.r + e);
      cp16(at(s, 32) + 16 * threadIdx.x, a.r + e + 4);
      if (GATE == 2) {
        const float* g = a.gate + t / a.gate_rows * a.d + col;
        cp16(at(s, 48) + 16 * threadIdx.x, g);
        cp16(at(s, 64) + 16 * threadIdx.x, g + 4);
      }
    }
    cp_commit();
  };
  for (int s = 0; s < STAGES - 1; ++s) fetch(u.lo + s, s);
  float g1[8] = {}, b1[8] = {}, g2[8] = {}, b2[8] = {};
  if (on && u.lo < u.hi) {
    f8(a.g1 + col, g1);
    if (a.b1) f8(a.b1 + col, b1);
    f8(a.g2 + col, g2);
    if (a.b2) f8(a.b2 + col, b2);
    if (GATE == 1) {
      float gt[8];
      f8(a.gate + col, gt);
#pragma unroll
      for (int j = 0; j < 8; ++j) { g1[j] *= gt[j]; b1[j] *= gt[j]; }
    }
  }
  const float inv_d = 1.f / a.d;
  int s = 0;
  // (units of one warp or less run as many turns as the longest of their warp: shuffles need all lanes)
  int64_t turns = u.hi - u.lo;
  if (a.tpr < 32) turns = __reduce_max_sync(0xffffffffu, (int)turns);
  for (int64_t i = 0; i < turns; ++i) {
    const int64_t t = u.lo + i;
    const bool row = on && t < u.hi;
    cp_wait<STAGES - 2>();
    float y[8] = {}, r[8] = {}, gt[8];
    if (row) {
      bf8(at(s, 0) + 16 * threadIdx.x, y);
      const float4 p = *reinterpret_cast<const float4*>(at(s, 16) + 16 * threadIdx.x);
      const float4 q = *reinterpret_cast<const float4*>(at(s, 32) + 16 * threadIdx.x);
      r[0] = p.x; r[1] = p.y; r[2] = p.z; r[3] = p.w; r[4] = q.x; r[5] = q.y; r[6] = q.z; r[7] = q.w;
      if (GATE == 2) {
        const float4 v = *reinterpret_cast<const float4*>(at(s, 48) + 16 * threadIdx.x);
        const float4 w = *reinterpret_cast<const float4*>(at(s, 64) + 16 * threadIdx.x);
        gt[0] = v.x; gt[1] = v.y; gt[2] = v.z; gt[3] = v.w; gt[4] = w.x; gt[5] = w.y; gt[6] = w.z; gt[7] = w.w;
      }
    }
    fetch(t + STAGES - 1, (s + STAGES - 1) % STAGES);
    s = (s + 1) % STAGES;
    // mean, then the squares about it: one pass over the squares alone would lose digits where the mean is large
    auto moments = [&](const float* x, float& mean, float& rstd) {
      mean = 0.f;
      if (LAYER) {
        float v = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) v += x[j];
        mean = sum(make_float2(v, 0.f)).x * inv_d;
      }
      float v = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) { const float e = x[j] - mean; v += e * e; }
      rstd = rsqrtf(sum(make_float2(row ? v : 0.f, 0.f)).x * inv_d + a.eps);
    };
    float m1, r1, m2, r2;
    moments(y, m1, r1);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float n = (y[j] - m1) * r1 * g1[j] + b1[j];
      if (GATE == 2) n *= row ? gt[j] : 0.f;
      r[j] = row ? fmaf(a.scale, r[j], n) : 0.f;
    }
    moments(r, m2, r2);
    if (row) {
      const int64_t e = t * a.d + col;
      put_f8(a.r_out + e, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j] = (r[j] - m2) * r2 * g2[j] + b2[j];
      put_bf8(a.h + e, r);
      if (u.tid == 0) a.stats[t] = make_float4(m1, r1, m2, r2);
    }
  }
}

// GATE: 0 none, 1 one row for all of the unit's rows, 2 read with each row, its gradient written at the end of each group
template <bool LAYER, int GATE>
__global__ void __launch_bounds__(MAX_D / 8) norm_gate_bwd_kernel(const NormArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float2 s_sum[4][2 * 16];
  const Unit u = my_unit(a);
  const int lane = threadIdx.x & 31, slot = threadIdx.x / a.tpr;
  UnitSum sum{s_sum[a.tpr > 32 ? slot : 0], a.tpr, 1 + slot, lane, (int)u.tid >> 5, 0};
  const int col = u.tid * 8;
  const bool on = col < a.d;
  constexpr int BYTES = Ring<true, GATE>::BYTES, STAGES = Ring<true, GATE>::STAGES;     // dh, y, r', dr', gate
  auto at = [&](int s, int off) { return smem + ((size_t)(s * BYTES + off) * blockDim.x) + 16 * threadIdx.x; };
  auto fetch = [&](int64_t t, int s) {
    if (t < u.hi && on) {
      const int64_t e = t * a.d + col;
      cp16(at(s, 0), a.dh + e);
      cp16(at(s, 16), a.y + e);
      cp16(at(s, 32), a.r + e);
      cp16(at(s, 48), a.r + e + 4);
      if (a.dr) { cp16(at(s, 64), a.dr + e); cp16(at(s, 80), a.dr + e + 4); }
      if (GATE == 2) {
        const float* g = a.gate + t / a.gate_rows * a.d + col;
        cp16(at(s, 96), g);
        cp16(at(s, 112), g + 4);
      }
    }
    cp_commit();
  };
  auto get = [&](int s, int off, float* f) {
    const float4 p = *reinterpret_cast<const float4*>(at(s, off)), q = *reinterpret_cast<const float4*>(at(s, off + 16));
    f[0] = p.x; f[1] = p.y; f[2] = p.z; f[3] = p.w; f[4] = q.x; f[5] = q.y; f[6] = q.z; f[7] = q.w;
  };
  for (int s = 0; s < STAGES - 1; ++s) fetch(u.lo + s, s);
  float gg[8] = {}, g2[8] = {};                              // gate g1 (g1 where the gate comes with each row)
  if (on && u.lo < u.hi) {
    f8(a.g1 + col, gg);
    f8(a.g2 + col, g2);
    if (GATE == 1) {
      float gt[8];
      f8(a.gate + (int64_t)u.group * a.d + col, gt);
#pragma unroll
      for (int j = 0; j < 8; ++j) gg[j] *= gt[j];
    }
  }
  // running sums: A = sum G yhat, B = sum G (of the group, where the gate comes with each row),
  // C = sum dh rhat, D = sum dh, and there PA, PB = sums of gate G yhat, gate G
  float A[8] = {}, B[8] = {}, C[8] = {}, D[8] = {}, PA[8] = {}, PB[8] = {};
  const float inv_d = 1.f / a.d;
  int s = 0;
  int64_t turns = u.hi - u.lo;
  if (a.tpr < 32) turns = __reduce_max_sync(0xffffffffu, (int)turns);
  float4 st = u.lo < u.hi ? a.stats[u.lo] : make_float4(0.f, 0.f, 0.f, 0.f);
  for (int64_t i = 0; i < turns; ++i) {
    const int64_t t = u.lo + i;
    const bool row = on && t < u.hi;
    cp_wait<STAGES - 2>();
    float dh[8] = {}, y[8] = {}, r[8] = {}, G[8] = {}, gt[8] = {};
    if (row) {
      bf8(at(s, 0), dh);
      bf8(at(s, 16), y);
      get(s, 32, r);
      if (a.dr) get(s, 64, G);
      if (GATE == 2) get(s, 96, gt);
    }
    fetch(t + STAGES - 1, (s + STAGES - 1) % STAGES);
    s = (s + 1) % STAGES;
    const float4 now = st;
    if (t + 1 < u.hi) st = a.stats[t + 1];
    float2 v = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      r[j] = (r[j] - now.z) * now.w;                          // rhat
      if (row) { C[j] = fmaf(dh[j], r[j], C[j]); D[j] += dh[j]; }
      dh[j] *= g2[j];
      if (LAYER) v.x += dh[j];
      v.y = fmaf(dh[j], r[j], v.y);
    }
    v = sum(v);
    v.x *= inv_d; v.y *= inv_d;
    float2 w = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float x = fmaf(-r[j], v.y, dh[j]);
      if (LAYER) x -= v.x;
      G[j] = row ? fmaf(now.w, x, G[j]) : 0.f;
      y[j] = (y[j] - now.x) * now.y;                          // yhat
      A[j] = fmaf(G[j], y[j], A[j]);
      B[j] += G[j];
      float q = G[j] * gg[j];
      if (GATE == 2) q *= gt[j];
      if (LAYER) w.x += q;
      w.y = fmaf(q, y[j], w.y);
    }
    w = sum(w);
    w.x *= inv_d; w.y *= inv_d;
    if (row) {
      const int64_t e = t * a.d + col;
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = a.scale * G[j];
      put_f8(a.dr_out + e, o);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float q = G[j] * gg[j];
        if (GATE == 2) q *= gt[j];
        q = fmaf(-y[j], w.y, q);
        if (LAYER) q -= w.x;
        o[j] = now.y * q;
      }
      put_bf8(a.dy + e, o);
      if (GATE == 2 && ((t + 1) % a.gate_rows == 0 || t + 1 == a.T)) {   // the group's last row
        float b1[8] = {};
        if (a.b1) f8(a.b1 + col, b1);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          o[j] = fmaf(gg[j], A[j], b1[j] * B[j]);
          PA[j] = fmaf(gt[j], A[j], PA[j]);
          PB[j] = fmaf(gt[j], B[j], PB[j]);
          A[j] = B[j] = 0.f;
        }
        put_f8(a.dgate + t / a.gate_rows * a.d + col, o);
      }
    }
  }
  if (on && u.unit < a.units) {
    const int64_t plane = (int64_t)a.units * a.d, e = (int64_t)u.unit * a.d + col;
    if (GATE == 2) {
      put_f8(a.partial + e, PA);
      put_f8(a.partial + plane + e, PB);
    } else if (GATE == 1) {
      float gt[8], o[8], b1[8] = {};
      f8(a.gate + (int64_t)u.group * a.d + col, gt);
      f8(a.g1 + col, gg);
      if (a.b1) f8(a.b1 + col, b1);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = fmaf(gg[j], A[j], b1[j] * B[j]);
        A[j] *= gt[j]; B[j] *= gt[j];
      }
      put_f8(a.partial + e, A);
      put_f8(a.partial + plane + e, B);
      put_f8(a.partial + 4 * plane + e, o);
    } else {
      put_f8(a.partial + e, A);
      put_f8(a.partial + plane + e, B);
    }
    put_f8(a.partial + 2 * plane + e, C);
    put_f8(a.partial + 3 * plane + e, D);
  }
}

// parameter gradients from the units' partial sums: blockIdx.y = 0..3 the norms' gains and shifts over
// all units, 4 + g the gate's row g over the units of its group; a warp adds a 32nd of them in order, and
// the 32 sums are added in order
struct ParamOut { float* out[4]; float* dgate; };
__global__ void __launch_bounds__(1024) norm_gate_params_kernel(const float* partial, ParamOut po, int units, int per_group, int d) {
  __shared__ float sh[32][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  const int which = min((int)blockIdx.y, 4), g = (int)blockIdx.y - 4;
  float* out = which < 4 ? po.out[which] : po.dgate + (int64_t)g * d;
  if (which < 4 && !out) return;
  const int n = which < 4 ? units : per_group, first = which < 4 ? 0 : g * per_group;
  const float* p = partial + ((int64_t)which * units + first) * d + c;
  const int per = (n + 31) / 32, b0 = w * per, b1 = min(n, b0 + per);
  float s = 0.f;
  if (c < d) {
#pragma unroll 8
    for (int b = b0; b < b1; ++b) s += p[(int64_t)b * d];
  }
  sh[w][lane] = s;
  __syncthreads();
  if (w == 0 && c < d) {
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < 32; ++q) t += sh[q][lane];
    out[c] = t;
  }
}

// ---- host ---------------------------------------------------------------------------------------
constexpr int SMS = 148;                      // work is split for a B200 (also where sizes are asked without a device)

struct Shape { int tpr, block, units, per_group, blocks, gate_mode; size_t partial; };
// threads per row, rows dealt to about 512 threads per SM (two blocks of 256)
Shape make_shape(int T, int d, int has_gate, int gate_rows, bool backward) {
  Shape s;
  const int need = d / 8;
  s.tpr = 8;
  if (need <= 32) while (s.tpr < need) s.tpr *= 2;
  else s.tpr = (need + 31) / 32 * 32;
  const int64_t target = std::min<int64_t>(16 * SMS, std::max<int64_t>(SMS, (int64_t)SMS * 512 / s.tpr));
  const int64_t groups = has_gate ? ((int64_t)T + gate_rows - 1) / gate_rows : 1;
  s.per_group = 0;
  s.gate_mode = !has_gate ? 0 : groups == 1 ? 1 : 2;
  if (backward && has_gate && groups < target) {       // several units to a group
    s.gate_mode = 1;
    const int64_t rows = std::min<int64_t>(gate_rows, T);
    s.per_group = (int)std::max<int64_t>(1, std::min<int64_t>(rows, target / groups));
    s.units = (int)(groups * s.per_group);
  } else {
    // whole groups (backward, more groups than units) or plain rows
    s.units = (int)std::min<int64_t>(target, backward && has_gate ? groups : T);
  }
  const int fit = s.tpr <= 32 ? 128 / s.tpr : std::max(1, 256 / s.tpr);
  s.block = s.tpr * fit;
  s.blocks = (s.units + fit - 1) / fit;
  s.partial = backward ? 5 * (size_t)s.units * d * 4 : 0;
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

template <bool LAYER, int GATE, bool BWD>
int launch_norm(const NormArgs& a, const Shape& s, cudaStream_t st) {
  constexpr int per_thread = Ring<BWD, GATE>::BYTES * Ring<BWD, GATE>::STAGES;
  static PerDeviceFlag attr;
  auto kernel = BWD ? norm_gate_bwd_kernel<LAYER, GATE> : norm_gate_fwd_kernel<LAYER, GATE>;
  if (!ppu_set_smem_once(attr, kernel, per_thread * (MAX_D / 8))) return ppu_fail(PPU_ECUDA, "shared memory limit not accepted");
  kernel<<<s.blocks, s.block, per_thread * s.block, st>>>(a);
  CUDA_OK(cudaGetLastError());
  return PPU_OK;
}
template <bool BWD>
int dispatch(const NormArgs& a, const Shape& s, int kind, cudaStream_t st) {
  const bool layer = kind == PPU_NORM_LAYER;
  switch (s.gate_mode) {
    case 0: return layer ? launch_norm<true, 0, BWD>(a, s, st) : launch_norm<false, 0, BWD>(a, s, st);
    case 1: return layer ? launch_norm<true, 1, BWD>(a, s, st) : launch_norm<false, 1, BWD>(a, s, st);
    default: return layer ? launch_norm<true, 2, BWD>(a, s, st) : launch_norm<false, 2, BWD>(a, s, st);
  }
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
  a.T = T; a.d = d; a.gate_rows = gate ? gate_rows : 1; a.tpr = s.tpr; a.units = s.units; a.per_group = 0;
  a.deal_rows = 1;                             // (no sums over a group)
  return dispatch<false>(a, s, kind, (cudaStream_t)cuda_stream);
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
  a.scale = res_scale; a.T = T; a.d = d; a.gate_rows = gate ? gate_rows : 1; a.tpr = s.tpr; a.units = s.units;
  a.deal_rows = s.gate_mode == 2 ? gate_rows : 1; a.per_group = s.per_group; a.partial = (float*)workspace; a.dgate = dgate;
  const int rc2 = dispatch<true>(a, s, kind, st);
  if (rc2) return rc2;
  const int groups = s.gate_mode == 1 ? s.units / s.per_group : 0;      // gate rows still to be summed
  const ParamOut po = {{dpost_gain, dpost_shift, dpre_gain, dpre_shift}, dgate};
  norm_gate_params_kernel<<<dim3((d + 31) / 32, 4 + groups), 1024, 0, st>>>(a.partial, po, s.units, s.per_group, d);
  CUDA_OK(cudaGetLastError());
  return PPU_OK;
}
