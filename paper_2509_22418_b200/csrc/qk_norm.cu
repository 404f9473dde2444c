// Norms of the queries' and keys' heads with the rotation by position in the same pass, between the QKV product and
// attention, on rows [q heads | k heads | v heads] of d_head columns each:
//
//   xh = N(x)   y = R(position) (xh gain)          for each q and k head x; v heads are copied
//   g = R(-position) dy   dgain = sum g xh   w = g gain   dx = rstd (w - xh mean(w xh) [- mean w])
//
// N is RMSNorm, or LayerNorm with the terms in brackets; R turns the pairs of the first rot columns.  The backward pass
// forms N again from the heads it is given (a head is in registers anyway), so nothing else is saved.
//
// HBM bounds both passes: 4 bytes an element forward, 6 backward.  A slot of LANES threads holds a head, 8 columns a thread,
// and keeps that head (its gain, its gain's gradient) while it goes through tokens; the slots of a block work on the same
// tokens, so that an angle's sine and cosine are formed once for all heads of a block, in shared memory.  The angle is formed
// in 64 bits as a fraction of a turn: at position 1e6 its rounding to 32 bits would be 0.06.
// A thread's columns are four pairs: 8 neighbours, or twice 4 neighbours half the rotated part apart.
#include <algorithm>
#include <cmath>
#include "../../include/ppu.h"
#include "common.cuh"

int ppu_fail(int code, const char* fmt, ...);

namespace {

constexpr int MAX_DH = 256, BLOCK = 256, SMS = 148;
// Tokens of a slot at a time (and as many on their way), blocks on an SM.  8192 x 48 heads of 128, us: forward 38.1; with 4 blocks (64 registers,
// spilling) 42.3, with 2 tokens and 4 blocks 40.7, 8 and 2 46.6, without the group on its way 41.9.  Backward 60.2; 1 token and 4 blocks 66, 3 and 2 60.9, 4 and
// 2 62.0.
constexpr int FWD_ROWS = 4, BWD_ROWS = 2;
constexpr int FWD_BLOCKS = 3, BWD_BLOCKS = 3;
constexpr int MOST_GROUPS = 4;                       // groups of rows whose angles are formed together

struct QkArgs {
  const bf16 *x, *dy;                // forward: x; backward: x and the gradient of the result
  bf16* out; int64_t ldx, ldy, ldo;
  const float *q_gain, *k_gain;      // null: ones
  const int32_t* positions; int seq; // null: t % seq
  const float* inv_freq;             // null: turns
  int n_q, n_k, heads, dh, rot;      // heads: those worked (q, k and copied ones)
  int per_head, layer;
  float eps;
  int T, slots, tokens;              // slots of a block that hold different heads, tokens at a time
  int groups_of_rows;                // of ROWS * tokens tokens each whose angles are formed together
  float* partial; int groups;        // backward: [rows][groups][dh]
  double turns[MAX_DH / 2];          // inverse frequencies / (2 pi)
};

// Two values in one instruction (half of the arithmetic's issue slots: with one value each the forward pass issued 194 instructions for a warp's two
// heads and took 48 us at 8192 x 48 heads of 128, where memory allows 31).
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 ra, rb, rd;\nmov.b64 ra, {%2, %3};\nmov.b64 rb, {%4, %5};\nmul.rn.f32x2 rd, ra, rb;\nmov.b64 {%0, %1}, rd;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n.reg .b64 ra, rb, rc, rd;\nmov.b64 ra, {%2, %3};\nmov.b64 rb, {%4, %5};\nmov.b64 rc, {%6, %7};\nfma.rn.f32x2 rd, ra, rb, rc;\nmov.b64 {%0, %1}, rd;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// The 8 columns of a thread are four pairs (a_i, b_i); v[0] = a_0 a_1, v[1] = a_2 a_3, v[2] = b_0 b_1, v[3] = b_2 b_3.
// HALVES 0: 8 neighbours from c0 on, a_0 b_0 a_1 b_1 ...; 1: the a's from c0 on, the b's from c1 on.
template <int HALVES> __device__ __forceinline__ uint4 load_row(const bf16* p, int c0, int c1) {
  if (!HALVES) return *reinterpret_cast<const uint4*>(p + c0);
  const uint2 a = *reinterpret_cast<const uint2*>(p + c0), b = *reinterpret_cast<const uint2*>(p + c1);
  return make_uint4(a.x, a.y, b.x, b.y);
}
template <int HALVES> __device__ __forceinline__ void store_row(bf16* p, int c0, int c1, const uint4 v) {
  if (!HALVES) { *reinterpret_cast<uint4*>(p + c0) = v; return; }
  *reinterpret_cast<uint2*>(p + c0) = make_uint2(v.x, v.y);
  *reinterpret_cast<uint2*>(p + c1) = make_uint2(v.z, v.w);
}
__device__ __forceinline__ float low(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float high(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
template <int HALVES> __device__ __forceinline__ void unpack(const uint4 u, float2 (&v)[4]) {
  if (HALVES) {
    v[0] = make_float2(low(u.x), high(u.x)); v[1] = make_float2(low(u.y), high(u.y)); v[2] = make_float2(low(u.z), high(u.z)); v[3] = make_float2(low(u.w), high(u.w));
  } else {
    v[0] = make_float2(low(u.x), low(u.y)); v[1] = make_float2(low(u.z), low(u.w)); v[2] = make_float2(high(u.x), high(u.y)); v[3] = make_float2(high(u.z), high(u.w));
  }
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <int HALVES> __device__ __forceinline__ uint4 pack(const float2 (&v)[4]) {
  if (HALVES) return make_uint4(pack2(v[0].x, v[0].y), pack2(v[1].x, v[1].y), pack2(v[2].x, v[2].y), pack2(v[3].x, v[3].y));
  return make_uint4(pack2(v[0].x, v[2].x), pack2(v[0].y, v[2].y), pack2(v[1].x, v[3].x), pack2(v[1].y, v[3].y));
}
// column of value j of v[i]
template <int HALVES> __device__ __forceinline__ int column(int i, int j, int c0, int c1) {
  const int pr = 2 * (i & 1) + j;
  return HALVES ? (i < 2 ? c0 : c1) + pr : c0 + 2 * pr + (i < 2 ? 0 : 1);
}
// (a, b) -> (a cos - b sin, a sin + b cos); back: by the negative angle
template <bool BACK> __device__ __forceinline__ void turn(float2 (&v)[4], const float4 c, const float4 s) {
  const float2 co[2] = {make_float2(c.x, c.y), make_float2(c.z, c.w)}, si[2] = {make_float2(s.x, s.y), make_float2(s.z, s.w)};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 a = v[i], b = v[2 + i], n = make_float2(-si[i].x, -si[i].y);
    v[i] = fma2(a, co[i], mul2(b, BACK ? si[i] : n));
    v[2 + i] = fma2(b, co[i], mul2(a, BACK ? n : si[i]));
  }
}
__device__ __forceinline__ float total(const float2 a) { return a.x + a.y; }

template <int LANES, int N> __device__ __forceinline__ void slot_sum(float (&v)[N]) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

template <int LANES, int HALVES, int LAYER, bool BWD>
__global__ void __launch_bounds__(BLOCK, BWD ? BWD_BLOCKS : FWD_BLOCKS) qk_norm_kernel(const __grid_constant__ QkArgs a) {
  constexpr int ROWS = BWD ? BWD_ROWS : FWD_ROWS;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ double s_turns[MAX_DH / 2];
  const int pairs = a.rot / 2, group = a.tokens * ROWS, tile = group * a.groups_of_rows;
  float* angles = reinterpret_cast<float*>(smem);          // [2][tile][pairs / 4][4 cosines, 4 sines]
  pdl_wait(); pdl_trigger();
  for (int i = threadIdx.x; i < pairs; i += BLOCK) s_turns[i] = a.inv_freq ? (double)a.inv_freq[i] * 0.15915494309189535 : a.turns[i];
  __syncthreads();

  const int slot = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  // this slot's head (dealt round to the blocks: each has its share of the values, which are less work), its first token of a group
  const int head = slot % a.slots * gridDim.y + blockIdx.y, mine = slot / a.slots;
  const bool on = mine < a.tokens && head < a.heads && 8 * lane < a.dh;
  const bool turned = 8 * lane < a.rot, normed = on && head < a.n_q + a.n_k;
  const bool work = __any_sync(0xffffffffu, normed);       // (a warp of values copies them)
  const int c0 = HALVES ? (turned ? 4 * lane : 8 * lane) : 8 * lane, c1 = HALVES && turned ? pairs + 4 * lane : c0 + 4;
  const int64_t at = (int64_t)head * a.dh;
  float2 gain[4], dgain[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) { gain[i] = both(1.f); dgain[i] = both(0.f); }
  if (normed) {
    const bool q = head < a.n_q;
    const float* g = q ? a.q_gain : a.k_gain;
    if (g) {
      if (a.per_head) g += (int64_t)(q ? head : head - a.n_q) * a.dh;
#pragma unroll
      for (int i = 0; i < 4; ++i) gain[i] = make_float2(g[column<HALVES>(i, 0, c0, c1)], g[column<HALVES>(i, 1, c0, c1)]);
    }
  }
  const float inv_dh = 1.f / (float)a.dh;
  const int tiles = (a.T + tile - 1) / tile;
  uint4 next[ROWS], next_grad[BWD ? ROWS : 1];
  auto load = [&](int first) {                       // the group of rows from token `first` on
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int64_t t = (int64_t)first + r * a.tokens + mine;
      next[r] = make_uint4(0, 0, 0, 0);
      if (BWD) next_grad[BWD ? r : 0] = make_uint4(0, 0, 0, 0);
      if (on && t < a.T) {
        if (!BWD || normed) next[r] = load_row<HALVES>(a.x + t * a.ldx + at, c0, c1);
        if (BWD) next_grad[BWD ? r : 0] = load_row<HALVES>(a.dy + t * a.ldy + at, c0, c1);
      }
    }
  };
  load(blockIdx.x * tile);
  int buf = 0;
  for (int it = blockIdx.x; it < tiles; it += gridDim.x, buf ^= 1) {
    const int t0 = it * tile;
    float* cs = angles + buf * tile * a.rot;
    const int n = min(tile, a.T - t0) * pairs;
    for (int e = threadIdx.x; e < n; e += BLOCK) {
      const int row = e / pairs, pr = e - row * pairs, t = t0 + row;
      const int pos = a.positions ? a.positions[t] : a.seq > 0 ? t % a.seq : t;
      const double turns = (double)pos * s_turns[pr];
      float s, c;
      sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
      float* to = cs + row * a.rot + (pr & ~3) * 2 + (pr & 3);
      to[0] = c; to[4] = s;
    }
    __syncthreads();
    for (int g0 = 0; g0 < tile && t0 + g0 < a.T; g0 += group) {
      uint4 raw[ROWS], grad[BWD ? ROWS : 1];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) { raw[r] = next[r]; if (BWD) grad[BWD ? r : 0] = next_grad[BWD ? r : 0]; }
      // the next group is on its way while this one is worked
      load(g0 + group < tile ? t0 + g0 + group : (int)min((int64_t)a.T, ((int64_t)it + gridDim.x) * tile));
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const int row = g0 + r * a.tokens + mine, t = t0 + row;
        const bool there = on && t < a.T;
        uint4 out = BWD ? grad[BWD ? r : 0] : raw[r];
        if (work) {
          float2 x[4];
          unpack<HALVES>(raw[r], x);
          float4 co = make_float4(1.f, 1.f, 1.f, 1.f), si = make_float4(0.f, 0.f, 0.f, 0.f);      // of the pairs 4 lane ..
          if (there && turned && normed) {
            const float4* p = reinterpret_cast<const float4*>(cs + row * a.rot + 8 * lane);
            co = p[0]; si = p[1];
          }
          if constexpr (!BWD) {
            if (LAYER) {
              float v[1] = {total(x[0]) + total(x[1]) + total(x[2]) + total(x[3])};
              slot_sum<LANES>(v);
              const float mean = v[0] * inv_dh;
#pragma unroll
              for (int i = 0; i < 4; ++i) { x[i].x -= mean; x[i].y -= mean; }
            }
            float v[1] = {total(fma2(x[0], x[0], mul2(x[1], x[1]))) + total(fma2(x[2], x[2], mul2(x[3], x[3])))};
            if (LAYER && 8 * lane >= a.dh) v[0] = 0.f;                       // (threads without columns)
            slot_sum<LANES>(v);
            const float2 rstd = both(rsqrtf(fmaf(v[0], inv_dh, a.eps)));
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = mul2(x[i], mul2(rstd, gain[i]));
            turn<false>(x, co, si);
            if (normed) out = pack<HALVES>(x);
          } else {
            float2 y[4], w[4];
            unpack<HALVES>(out, y);
            turn<true>(y, co, si);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = mul2(y[i], gain[i]);
            float mean_w = 0.f;
            if (LAYER) {
              float v[2] = {total(x[0]) + total(x[1]) + total(x[2]) + total(x[3]), total(w[0]) + total(w[1]) + total(w[2]) + total(w[3])};
              slot_sum<LANES>(v);
              const float mean = v[0] * inv_dh;
              mean_w = v[1] * inv_dh;
#pragma unroll
              for (int i = 0; i < 4; ++i) { x[i].x -= mean; x[i].y -= mean; }
            }
            // sums of (x - mean)^2 and w (x - mean)
            float v[2] = {total(fma2(x[0], x[0], mul2(x[1], x[1]))) + total(fma2(x[2], x[2], mul2(x[3], x[3]))),
                          total(fma2(w[0], x[0], mul2(w[1], x[1]))) + total(fma2(w[2], x[2], mul2(w[3], x[3])))};
            if (LAYER && 8 * lane >= a.dh) v[0] = v[1] = 0.f;
            slot_sum<LANES>(v);
            const float rs = rsqrtf(fmaf(v[0], inv_dh, a.eps));
            const float2 rstd = both(rs), dot = both(-(v[1] * rs * inv_dh)), less = both(-mean_w);      // (minus) the means of w xh and of w
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 xh = mul2(x[i], rstd);
              if (there) dgain[i] = fma2(y[i], xh, dgain[i]);                // (without eps, the zeros in the place of a row that is not there give NaN)
              if (LAYER) { w[i].x += less.x; w[i].y += less.y; }
              x[i] = mul2(rstd, fma2(xh, dot, w[i]));
            }
            if (normed) out = pack<HALVES>(x);
          }
        }
        if (there) store_row<HALVES>(a.out + t * a.ldo + at, c0, c1, out);
      }
    }
  }
  if constexpr (BWD) {
    if (!a.partial) return;
    // sums of the block's slots that share a gain, in the order of the slots
    __syncthreads();                                 // (the angles have been read)
    float* sums = reinterpret_cast<float*>(smem);    // [slots of the block][dh]
    if (8 * lane < a.dh)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sums[slot * a.dh + column<HALVES>(i, 0, c0, c1)] = normed ? dgain[i].x : 0.f;
        sums[slot * a.dh + column<HALVES>(i, 1, c0, c1)] = normed ? dgain[i].y : 0.f;
      }
    __syncthreads();
    const int all = a.slots * a.tokens;              // slots in use: head slot % slots, token slot / slots
    if (a.per_head) {
      for (int e = threadIdx.x; e < a.slots * a.dh; e += BLOCK) {
        const int h = e / a.dh, c = e - h * a.dh, hd = h * gridDim.y + blockIdx.y;
        if (hd >= a.n_q + a.n_k) break;
        float s = 0.f;
        for (int k = h; k < all; k += a.slots) s += sums[k * a.dh + c];
        a.partial[((int64_t)blockIdx.x * a.groups + hd) * a.dh + c] = s;
      }
    } else {
      for (int e = threadIdx.x; e < 2 * a.dh; e += BLOCK) {
        const int g = e / a.dh, c = e - g * a.dh;
        float s = 0.f;
        for (int k = 0; k < all; ++k) {
          const int h = k % a.slots * gridDim.y + blockIdx.y;
          if (h < a.n_q + a.n_k && (h >= a.n_q) == (g == 1)) s += sums[k * a.dh + c];
        }
        a.partial[((int64_t)(blockIdx.x * gridDim.y + blockIdx.y) * 2 + g) * a.dh + c] = s;
      }
    }
  }
}

// gain gradients from the blocks' partial sums [rows][columns]: a warp adds a 32nd of the rows in order for 32 columns, and the 32 sums
// are added in order.  Columns below q_columns are dq_gain's.
__global__ void __launch_bounds__(1024) qk_norm_gains_kernel(const float* partial, int rows, int columns, int q_columns, float* dq_gain, float* dk_gain) {
  pdl_wait(); pdl_trigger();
  __shared__ float sh[32][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  const int r0 = (int)((int64_t)rows * w / 32), r1 = (int)((int64_t)rows * (w + 1) / 32);
  float s = 0.f;
  if (c < columns)
#pragma unroll 8
    for (int r = r0; r < r1; ++r) s += partial[(int64_t)r * columns + c];
  sh[w][lane] = s;
  __syncthreads();
  if (w == 0 && c < columns) {
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < 32; ++q) t += sh[q][lane];
    float* out = c < q_columns ? dq_gain : dk_gain;
    if (out) out[c < q_columns ? c : c - q_columns] = t;
  }
}

// ---- host ------------------------------------------------------------------------------------------
struct Plan { int lanes, slots, tokens, many, grid_x, grid_y, rows, groups; size_t bytes; };

Plan make_plan(int T, int heads, int normed, int dh, int per_head, bool backward) {
  Plan p = {};
  p.lanes = 2;
  while (p.lanes * 8 < dh) p.lanes *= 2;
  const int all = BLOCK / p.lanes;
  p.grid_y = (heads + all - 1) / all;
  p.slots = (heads + p.grid_y - 1) / p.grid_y;
  p.tokens = all / p.slots;
  const int group = p.tokens * (backward ? BWD_ROWS : FWD_ROWS), resident = SMS * (backward ? BWD_BLOCKS : FWD_BLOCKS);
  // several groups of rows between two barriers where every block then still has several turns, and 32 KB hold their angles
  p.many = 1;
  while (p.many < MOST_GROUPS && group * p.many * 2 * dh <= 4096 && (int64_t)T * p.grid_y >= (int64_t)group * p.many * 2 * 4 * resident) p.many *= 2;
  const int tile = group * p.many, tiles = (T + tile - 1) / tile;
  p.grid_x = std::max(1, std::min(tiles, resident / std::min(p.grid_y, resident)));
  p.groups = per_head ? normed : 2;
  p.rows = per_head ? p.grid_x : p.grid_x * p.grid_y;
  p.bytes = backward ? (size_t)p.rows * p.groups * dh * 4 : 0;
  return p;
}

int check_qk(int T, int n_q, int n_k, int n_v, int dh) {
  if (T < 0 || n_q < 0 || n_k < 0 || n_v < 0 || dh < 1) return ppu_fail(PPU_EINVAL, "negative or empty size");
  if (n_q + (int64_t)n_k < 1) return ppu_fail(PPU_EINVAL, "no heads of queries or keys");
  if (dh % 8 || dh > MAX_DH) return ppu_fail(PPU_ESHAPE, "d_head must be a multiple of 8 up to %d (got %d)", MAX_DH, dh);
  if (n_q > 4096 || n_k > 4096 || n_v > 4096) return ppu_fail(PPU_ESHAPE, "at most 4096 heads of a kind");
  if (T > (1 << 24)) return ppu_fail(PPU_ESHAPE, "at most 2^24 rows");
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

// arguments common to both passes
int fill_args(QkArgs& a, int kind, int pairs, int rot, float rope_base, const float* inv_freq, const float* q_gain, const float* k_gain, int gain_per_head,
              const int32_t* positions, int seq, float eps, int T, int n_q, int n_k, int dh) {
  if (kind != PPU_NORM_LAYER && kind != PPU_NORM_RMS) return ppu_fail(PPU_EINVAL, "unknown norm kind %d", kind);
  if (pairs != PPU_PAIRS_ADJACENT && pairs != PPU_PAIRS_HALVES) return ppu_fail(PPU_EINVAL, "unknown pairs %d", pairs);
  if (rot < 0 || rot > dh || rot % 8) return ppu_fail(PPU_ESHAPE, "rot_dim must be a multiple of 8 up to d_head (got %d)", rot);
  if (rot && !inv_freq && !(rope_base > 0.f && std::isfinite(rope_base))) return ppu_fail(PPU_EINVAL, "rope_base must be positive");
  if (!(eps >= 0.f)) return ppu_fail(PPU_EINVAL, "eps must not be negative");
  if (seq < 0) return ppu_fail(PPU_EINVAL, "seq must not be negative");
  if (misaligned({q_gain, k_gain}) || (reinterpret_cast<uintptr_t>(positions) | reinterpret_cast<uintptr_t>(inv_freq)) & 3)
    return ppu_fail(PPU_EINVAL, "gains must be 16-byte aligned, positions and frequencies 4-byte");
  a.q_gain = q_gain; a.k_gain = k_gain; a.positions = positions; a.seq = seq; a.inv_freq = rot ? inv_freq : nullptr;
  a.n_q = n_q; a.n_k = n_k; a.dh = dh; a.rot = rot; a.per_head = gain_per_head != 0; a.layer = kind == PPU_NORM_LAYER; a.eps = eps; a.T = T;
  for (int i = 0; i < rot / 2 && !inv_freq; ++i) a.turns[i] = std::pow((double)rope_base, -2.0 * i / rot) * 0.15915494309189535;
  return PPU_OK;
}

template <int LANES, int HALVES, int LAYER, bool BWD>
int launch_qk(const QkArgs& a, const Plan& p, cudaStream_t st) {
  static PerDeviceFlag attr;
  constexpr int most = 2 * BLOCK * (BWD ? BWD_ROWS : FWD_ROWS) * 8 * 4;      // one head to a block, all of it rotated: 64 KB forward
  int bytes = 2 * p.tokens * (BWD ? BWD_ROWS : FWD_ROWS) * p.many * a.rot * 4;
  if (BWD) bytes = std::max(bytes, BLOCK / LANES * a.dh * 4);
  auto kernel = qk_norm_kernel<LANES, HALVES, LAYER, BWD>;
  if (!ppu_set_smem_once(attr, kernel, most)) return ppu_fail(PPU_ECUDA, "shared memory limit not accepted");
  CUDA_OK(ppu_launch_dependent(kernel, dim3(p.grid_x, p.grid_y), BLOCK, bytes, st, a));
  return PPU_OK;
}
template <int LANES, bool BWD>
int launch_form(const QkArgs& a, const Plan& p, int pairs, cudaStream_t st) {
  if (pairs == PPU_PAIRS_HALVES) return a.layer ? launch_qk<LANES, 1, 1, BWD>(a, p, st) : launch_qk<LANES, 1, 0, BWD>(a, p, st);
  return a.layer ? launch_qk<LANES, 0, 1, BWD>(a, p, st) : launch_qk<LANES, 0, 0, BWD>(a, p, st);
}
template <bool BWD>
int dispatch(const QkArgs& a, const Plan& p, int pairs, cudaStream_t st) {
  switch (p.lanes) {
    case 2: return launch_form<2, BWD>(a, p, pairs, st);
    case 4: return launch_form<4, BWD>(a, p, pairs, st);
    case 8: return launch_form<8, BWD>(a, p, pairs, st);
    case 16: return launch_form<16, BWD>(a, p, pairs, st);
    default: return launch_form<32, BWD>(a, p, pairs, st);
  }
}

}  // namespace

extern "C" int ppu_qk_norm_fwd(const void* qkv, int64_t ldx, const float* q_gain, const float* k_gain, int gain_per_head, const int32_t* positions, int seq, int kind,
                               float eps, float rope_base, const float* inv_freq, int rot_dim, int pairs, void* out, int64_t ldo, int T, int n_q, int n_k, int n_v,
                               int d_head, void* cuda_stream) {
  int rc = check_qk(T, n_q, n_k, n_v, d_head);
  if (rc) return rc;
  QkArgs a = {};
  rc = fill_args(a, kind, pairs, rot_dim, rope_base, inv_freq, q_gain, k_gain, gain_per_head, positions, seq, eps, T, n_q, n_k, d_head);
  if (rc) return rc;
  if (T == 0) return PPU_OK;
  const int64_t cols = ((int64_t)n_q + n_k + n_v) * d_head;
  if (!qkv || !out) return ppu_fail(PPU_EINVAL, "null operand");
  if (ldx < cols || ldo < cols || ldx % 8 || ldo % 8) return ppu_fail(PPU_EINVAL, "row strides must be multiples of 8 that hold all heads");
  if (misaligned({qkv, out})) return ppu_fail(PPU_EINVAL, "qkv and out must be 16-byte aligned");
  if (out == qkv && ldo != ldx) return ppu_fail(PPU_EINVAL, "out in the place of qkv needs its row stride");
  a.x = (const bf16*)qkv; a.ldx = ldx; a.out = (bf16*)out; a.ldo = ldo;
  a.heads = n_q + n_k + (out == qkv ? 0 : n_v);
  const Plan p = make_plan(T, n_q + n_k + n_v, n_q + n_k, d_head, a.per_head, false);
  a.slots = p.slots; a.tokens = p.tokens; a.groups_of_rows = p.many;
  return dispatch<false>(a, p, pairs, (cudaStream_t)cuda_stream);
}

extern "C" int ppu_qk_norm_query_bytes(int T, int n_q, int n_k, int n_v, int d_head, int gain_per_head, size_t* bytes) {
  if (!bytes) return ppu_fail(PPU_EINVAL, "bytes is null");
  const int rc = check_qk(T, n_q, n_k, n_v, d_head);
  if (rc) return rc;
  *bytes = T ? make_plan(T, n_q + n_k + n_v, n_q + n_k, d_head, gain_per_head != 0, true).bytes : 0;
  return PPU_OK;
}

extern "C" int ppu_qk_norm_bwd(const void* dout, int64_t ldy, const void* qkv, int64_t ldx, const float* q_gain, const float* k_gain, int gain_per_head,
                               const int32_t* positions, int seq, int kind, float eps, float rope_base, const float* inv_freq, int rot_dim, int pairs, void* dqkv,
                               int64_t ldo, float* dq_gain, float* dk_gain, int T, int n_q, int n_k, int n_v, int d_head, void* workspace, size_t workspace_bytes,
                               void* cuda_stream) {
  int rc = check_qk(T, n_q, n_k, n_v, d_head);
  if (rc) return rc;
  QkArgs a = {};
  rc = fill_args(a, kind, pairs, rot_dim, rope_base, inv_freq, q_gain, k_gain, gain_per_head, positions, seq, eps, T, n_q, n_k, d_head);
  if (rc) return rc;
  if ((dq_gain && !q_gain) || (dk_gain && !k_gain)) return ppu_fail(PPU_EINVAL, "a gradient of a gain that is not there");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const size_t q_size = (size_t)d_head * (a.per_head ? n_q : 1), k_size = (size_t)d_head * (a.per_head ? n_k : 1);
  if (T == 0) {                                      // sums over nothing
    if (dq_gain) CUDA_OK(cudaMemsetAsync(dq_gain, 0, q_size * 4, st));
    if (dk_gain) CUDA_OK(cudaMemsetAsync(dk_gain, 0, k_size * 4, st));
    return PPU_OK;
  }
  const int64_t cols = ((int64_t)n_q + n_k + n_v) * d_head;
  const bool gains = dq_gain || dk_gain;
  if (!dout || !qkv || !dqkv || (gains && !workspace)) return ppu_fail(PPU_EINVAL, "null operand");
  if (ldx < cols || ldy < cols || ldo < cols || ldx % 8 || ldy % 8 || ldo % 8) return ppu_fail(PPU_EINVAL, "row strides must be multiples of 8 that hold all heads");
  if (misaligned({dout, qkv, dqkv, workspace})) return ppu_fail(PPU_EINVAL, "operands must be 16-byte aligned");
  if (dqkv == dout && ldo != ldy) return ppu_fail(PPU_EINVAL, "dqkv in the place of dout needs its row stride");
  a.x = (const bf16*)qkv; a.ldx = ldx; a.dy = (const bf16*)dout; a.ldy = ldy; a.out = (bf16*)dqkv; a.ldo = ldo;
  // (the work is split as if the values were copied in any case: the order of the gains' sums does not depend on it)
  a.heads = n_q + n_k + (dqkv == dout ? 0 : n_v);
  const Plan p = make_plan(T, n_q + n_k + n_v, n_q + n_k, d_head, a.per_head, true);
  if (gains && workspace_bytes < p.bytes) return ppu_fail(PPU_ENOMEM, "workspace has %zu bytes, %zu needed", workspace_bytes, p.bytes);
  a.slots = p.slots; a.tokens = p.tokens; a.groups_of_rows = p.many; a.partial = gains ? (float*)workspace : nullptr; a.groups = p.groups;
  rc = dispatch<true>(a, p, pairs, st);
  if (rc || !gains) return rc;
  const int columns = p.groups * d_head, q_columns = (a.per_head ? n_q : 1) * d_head;
  CUDA_OK(ppu_launch_dependent(qk_norm_gains_kernel, (columns + 31) / 32, 1024, 0, st, a.partial, p.rows, columns, q_columns, dq_gain, dk_gain));
  return PPU_OK;
}
