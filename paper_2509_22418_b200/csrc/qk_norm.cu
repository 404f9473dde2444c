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
constexpr int FWD_ROWS = 4, BWD_ROWS = 2;            // tokens of a slot in flight
constexpr int FWD_BLOCKS = 4, BWD_BLOCKS = 3;        // blocks on an SM

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
  float* partial; int groups;        // backward: [rows][groups][dh]
  int norm_y;                        // blocks (y) with heads of queries and keys
  double turns[MAX_DH / 2];          // inverse frequencies / (2 pi)
};

__device__ __forceinline__ void unpack4(const uint2 u, float* f) {
  const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x));
  const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
  f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
}
__device__ __forceinline__ uint2 pack4(const float* f) {
  __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
  return make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
}
// the 8 columns of a thread: at c0 and c1 = c0 + 4 (HALVES 0), or at c0 and c1
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
__device__ __forceinline__ void unpack8(const uint4 u, float* f) { unpack4(make_uint2(u.x, u.y), f); unpack4(make_uint2(u.z, u.w), f + 4); }
__device__ __forceinline__ uint4 pack8(const float* f) {
  const uint2 a = pack4(f), b = pack4(f + 4);
  return make_uint4(a.x, a.y, b.x, b.y);
}
// pair j of a thread's columns
template <int HALVES> __device__ __forceinline__ constexpr int pair_a(int j) { return HALVES ? j : 2 * j; }
template <int HALVES> __device__ __forceinline__ constexpr int pair_b(int j) { return HALVES ? 4 + j : 2 * j + 1; }

template <int LANES, int N> __device__ __forceinline__ void slot_sum(float (&v)[N]) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

template <int LANES, int HALVES, bool BWD>
__global__ void __launch_bounds__(BLOCK, BWD ? BWD_BLOCKS : FWD_BLOCKS) qk_norm_kernel(const __grid_constant__ QkArgs a) {
  constexpr int ROWS = BWD ? BWD_ROWS : FWD_ROWS;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ double s_turns[MAX_DH / 2];
  const int pairs = a.rot / 2, tile = a.tokens * ROWS;
  float2* angles = reinterpret_cast<float2*>(smem);        // [2][tile][pairs] (cos, sin)
  pdl_wait(); pdl_trigger();
  for (int i = threadIdx.x; i < pairs; i += BLOCK) s_turns[i] = a.inv_freq ? (double)a.inv_freq[i] * 0.15915494309189535 : a.turns[i];
  __syncthreads();

  const int slot = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int head = blockIdx.y * a.slots + slot % a.slots, mine = slot / a.slots;      // this slot's head, its first token of a tile
  const bool on = mine < a.tokens && head < a.heads && 8 * lane < a.dh;
  const bool turned = 8 * lane < a.rot, normed = head < a.n_q + a.n_k;
  const int c0 = HALVES ? (turned ? 4 * lane : 8 * lane) : 8 * lane, c1 = HALVES && turned ? pairs + 4 * lane : c0 + 4;
  const int64_t at = (int64_t)head * a.dh;
  float gain[8], dgain[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) { gain[j] = 1.f; dgain[j] = 0.f; }
  if (on && normed) {
    const bool q = head < a.n_q;
    const float* g = q ? a.q_gain : a.k_gain;
    if (g) {
      if (a.per_head) g += (int64_t)(q ? head : head - a.n_q) * a.dh;
#pragma unroll
      for (int j = 0; j < 8; ++j) gain[j] = g[j < 4 ? c0 + j : c1 + j - 4];
    }
  }
  const float inv_dh = 1.f / (float)a.dh;
  const int tiles = (a.T + tile - 1) / tile;
  int buf = 0;
  for (int i = blockIdx.x; i < tiles; i += gridDim.x, buf ^= 1) {
    const int t0 = i * tile;
    uint4 raw[ROWS], grad[BWD ? ROWS : 1];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int t = t0 + r * a.tokens + mine;
      raw[r] = make_uint4(0, 0, 0, 0);
      if (BWD) grad[BWD ? r : 0] = make_uint4(0, 0, 0, 0);
      if (on && t < a.T) {
        raw[r] = load_row<HALVES>(a.x + t * a.ldx + at, c0, c1);
        if (BWD) grad[BWD ? r : 0] = load_row<HALVES>(a.dy + t * a.ldy + at, c0, c1);
      }
    }
    float2* cs = angles + buf * tile * pairs;
    const int n = min(tile, a.T - t0) * pairs;
    for (int e = threadIdx.x; e < n; e += BLOCK) {
      const int row = e / pairs, pr = e - row * pairs, t = t0 + row;
      const int pos = a.positions ? a.positions[t] : a.seq > 0 ? t % a.seq : t;
      const double turn = (double)pos * s_turns[pr];
      float s, c;
      sincospif(2.f * (float)(turn - rint(turn)), &s, &c);
      cs[e] = make_float2(c, s);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int row = r * a.tokens + mine, t = t0 + row;
      const bool there = on && t < a.T;
      float x[8], y[8];
      unpack8(raw[r], x);
      float4 w0 = make_float4(1.f, 0.f, 1.f, 0.f), w1 = w0;                   // (cos, sin) of the pairs 4 lane ..
      if (there && turned) {
        const float4* p = reinterpret_cast<const float4*>(cs + (int64_t)row * pairs + 4 * lane);
        w0 = p[0]; w1 = p[1];
      }
      const float co[4] = {w0.x, w0.z, w1.x, w1.z}, si[4] = {w0.y, w0.w, w1.y, w1.w};
      if constexpr (!BWD) {
        float mean = 0.f;
        if (a.layer) {
          float v[1] = {0.f};
#pragma unroll
          for (int j = 0; j < 8; ++j) v[0] += x[j];
          slot_sum<LANES>(v);
          mean = v[0] * inv_dh;
        }
        float v[1] = {0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) { y[j] = x[j] - mean; v[0] = fmaf(y[j], y[j], v[0]); }
        if (a.layer && 8 * lane >= a.dh) v[0] = 0.f;                         // (threads without columns)
        slot_sum<LANES>(v);
        const float rstd = 1.f / sqrtf(fmaf(v[0], inv_dh, a.eps));
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] *= rstd * gain[j];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = y[pair_a<HALVES>(j)], q = y[pair_b<HALVES>(j)];
          x[pair_a<HALVES>(j)] = p * co[j] - q * si[j];
          x[pair_b<HALVES>(j)] = p * si[j] + q * co[j];
        }
        if (there) store_row<HALVES>(a.out + t * a.ldo + at, c0, c1, normed ? pack8(x) : raw[r]);
      } else {
        unpack8(grad[r], y);
#pragma unroll
        for (int j = 0; j < 4; ++j) {                                        // turned back
          const float p = y[pair_a<HALVES>(j)], q = y[pair_b<HALVES>(j)];
          y[pair_a<HALVES>(j)] = p * co[j] + q * si[j];
          y[pair_b<HALVES>(j)] = q * co[j] - p * si[j];
        }
        float mean = 0.f, mean_w = 0.f;
        if (a.layer) {
          float v[2] = {0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 8; ++j) { v[0] += x[j]; v[1] = fmaf(y[j], gain[j], v[1]); }
          slot_sum<LANES>(v);
          mean = v[0] * inv_dh; mean_w = v[1] * inv_dh;
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] -= mean;
        }
        float v[2] = {0.f, 0.f};                                             // sums of (x - mean)^2 and w (x - mean)
#pragma unroll
        for (int j = 0; j < 8; ++j) { v[0] = fmaf(x[j], x[j], v[0]); v[1] = fmaf(y[j] * gain[j], x[j], v[1]); }
        if (8 * lane >= a.dh) v[0] = v[1] = 0.f;
        slot_sum<LANES>(v);
        const float rstd = 1.f / sqrtf(fmaf(v[0], inv_dh, a.eps));
        const float dot = v[1] * rstd * inv_dh;                              // mean of w xh
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float xh = x[j] * rstd;
          if (there) dgain[j] = fmaf(y[j], xh, dgain[j]);                     // (without eps, the zeros in the place of a row that is not there give NaN)
          x[j] = rstd * (fmaf(y[j], gain[j], -mean_w) - xh * dot);
        }
        if (there) store_row<HALVES>(a.out + t * a.ldo + at, c0, c1, normed ? pack8(x) : grad[r]);
      }
    }
  }
  if constexpr (BWD) {
    if (!a.partial || (int)blockIdx.y >= a.norm_y) return;
    // sums of the block's slots that share a gain, in the order of the slots
    __syncthreads();                                 // (the angles have been read)
    float* sums = reinterpret_cast<float*>(smem);    // [slots of the block][dh]
    if (8 * lane < a.dh)
#pragma unroll
      for (int j = 0; j < 8; ++j) sums[slot * a.dh + (j < 4 ? c0 + j : c1 + j - 4)] = on && normed ? dgain[j] : 0.f;
    __syncthreads();
    const int all = a.slots * a.tokens;              // slots in use: head slot % slots, token slot / slots
    if (a.per_head) {
      const int here = min(a.slots, a.n_q + a.n_k - (int)blockIdx.y * a.slots);
      for (int e = threadIdx.x; e < here * a.dh; e += BLOCK) {
        const int h = e / a.dh, c = e - h * a.dh;
        float s = 0.f;
        for (int k = h; k < all; k += a.slots) s += sums[k * a.dh + c];
        a.partial[((int64_t)blockIdx.x * a.groups + blockIdx.y * a.slots + h) * a.dh + c] = s;
      }
    } else {
      for (int e = threadIdx.x; e < 2 * a.dh; e += BLOCK) {
        const int g = e / a.dh, c = e - g * a.dh;
        float s = 0.f;
        for (int k = 0; k < all; ++k) {
          const int h = blockIdx.y * a.slots + k % a.slots;
          if (h < a.n_q + a.n_k && (h >= a.n_q) == (g == 1)) s += sums[k * a.dh + c];
        }
        a.partial[((int64_t)(blockIdx.x * a.norm_y + blockIdx.y) * 2 + g) * a.dh + c] = s;
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
struct Plan { int lanes, slots, tokens, grid_x, grid_y, rows, groups; size_t bytes; };

Plan make_plan(int T, int heads, int normed, int dh, int per_head, bool backward) {
  Plan p = {};
  p.lanes = 2;
  while (p.lanes * 8 < dh) p.lanes *= 2;
  const int all = BLOCK / p.lanes;
  p.grid_y = (heads + all - 1) / all;
  p.slots = (heads + p.grid_y - 1) / p.grid_y;
  p.tokens = all / p.slots;
  const int tile = p.tokens * (backward ? BWD_ROWS : FWD_ROWS);
  const int tiles = (T + tile - 1) / tile, resident = SMS * (backward ? BWD_BLOCKS : FWD_BLOCKS);
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

template <int LANES, int HALVES, bool BWD>
int launch_qk(const QkArgs& a, const Plan& p, cudaStream_t st) {
  static PerDeviceFlag attr;
  constexpr int most = 2 * BLOCK / LANES * (BWD ? BWD_ROWS : FWD_ROWS) * LANES * 4 * 8;      // one head to a block, all of it rotated
  int bytes = 2 * p.tokens * (BWD ? BWD_ROWS : FWD_ROWS) * (a.rot / 2) * 8;
  if (BWD) bytes = std::max(bytes, BLOCK / LANES * a.dh * 4);
  if (!ppu_set_smem_once(attr, qk_norm_kernel<LANES, HALVES, BWD>, most)) return ppu_fail(PPU_ECUDA, "shared memory limit not accepted");
  CUDA_OK(ppu_launch_dependent(qk_norm_kernel<LANES, HALVES, BWD>, dim3(p.grid_x, p.grid_y), BLOCK, bytes, st, a));
  return PPU_OK;
}
template <bool BWD>
int dispatch(const QkArgs& a, const Plan& p, int pairs, cudaStream_t st) {
  const bool h = pairs == PPU_PAIRS_HALVES;
  switch (p.lanes) {
    case 2: return h ? launch_qk<2, 1, BWD>(a, p, st) : launch_qk<2, 0, BWD>(a, p, st);
    case 4: return h ? launch_qk<4, 1, BWD>(a, p, st) : launch_qk<4, 0, BWD>(a, p, st);
    case 8: return h ? launch_qk<8, 1, BWD>(a, p, st) : launch_qk<8, 0, BWD>(a, p, st);
    case 16: return h ? launch_qk<16, 1, BWD>(a, p, st) : launch_qk<16, 0, BWD>(a, p, st);
    default: return h ? launch_qk<32, 1, BWD>(a, p, st) : launch_qk<32, 0, BWD>(a, p, st);
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
  Plan p = make_plan(T, n_q + n_k + n_v, n_q + n_k, d_head, a.per_head, false);
  p.grid_y = (a.heads + p.slots - 1) / p.slots;
  a.slots = p.slots; a.tokens = p.tokens;
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
  Plan p = make_plan(T, n_q + n_k + n_v, n_q + n_k, d_head, a.per_head, true);
  if (gains && workspace_bytes < p.bytes) return ppu_fail(PPU_ENOMEM, "workspace has %zu bytes, %zu needed", workspace_bytes, p.bytes);
  p.grid_y = (n_q + n_k + p.slots - 1) / p.slots;      // blocks that hold heads of queries and keys
  p.rows = a.per_head ? p.grid_x : p.grid_x * p.grid_y;
  a.norm_y = p.grid_y;
  p.grid_y = (a.heads + p.slots - 1) / p.slots;
  a.slots = p.slots; a.tokens = p.tokens; a.partial = gains ? (float*)workspace : nullptr; a.groups = p.groups;
  rc = dispatch<true>(a, p, pairs, st);
  if (rc || !gains) return rc;
  const int columns = p.groups * d_head, q_columns = (a.per_head ? n_q : 1) * d_head;
  CUDA_OK(ppu_launch_dependent(qk_norm_gains_kernel, (columns + 31) / 32, 1024, 0, st, a.partial, p.rows, columns, q_columns, dq_gain, dk_gain));
  return PPU_OK;
}
