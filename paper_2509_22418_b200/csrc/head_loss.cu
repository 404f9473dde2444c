// Losses of hidden states against a large vocabulary that never hold the [T, V] logits: softmax
// cross entropy and distillation from a teacher's top logits, with the gradients of the hidden
// states and of the vocabulary matrix.
//
//   s = X E^T / temperature,  lse_t = log sum_v exp(s_tv),  p = softmax(s)
//   row loss = sum_j q_tj (log q_tj - s_t,id(j) + lse_t)        (cross entropy: one entry, q = 1)
//   ds_tv = w_t (Q_t p_tv - sum_{j: id(j) = v} q_tj),  Q_t = sum_j q_tj
//   dX = ds E / temperature,  dE = ds^T X / temperature
//
// Three matrix products cannot be avoided (6 T V d operations), and a backward pass that forms the
// logits again would make it four.  So rows are worked in chunks, whose softmax is kept only until
// the chunk's two gradient products are done: a [rows, V] buffer of bounded size, not [T, V].
//   1. tcgen05 product of the chunk's rows with E^T.  Its epilogue works the vocabulary in pieces
//      of 64 columns: bf16 powers relative to the piece's own maximum, and {maximum, sum} in fp32.
//   2. one block per row joins the pieces to the row's log-sum-exp, computes the entries' logits as
//      fp32 dot products of their own (k of them, d long: the stored powers would be too coarse for
//      the loss and for p - 1 next to p = 1), the row loss, and turns the powers into ds in place: one
//      factor for each piece, the entries' places overwritten with their exact values.
//   3. dX and dE products of ds; dE over several chunks is a running fp32 sum, rounded once by the last.
// Steps 1 and 2 go over sub-chunks that fit the L2 (64 MiB), so step 2 does not read HBM.
// Roundings: the powers and ds are bf16 (the tensor cores' operand type; each off by at most half a
// step, 2^-8 of its own value, independently), dX and dE are rounded once from fp32; statistics,
// losses and running sums are fp32.
#include <algorithm>
#include "../../include/ppu.h"
#include "common.cuh"

int ppu_fail(int code, const char* fmt, ...);

namespace {

constexpr int ROW_THREADS = 256;
constexpr int MAX_ENTRIES = PPU_MAX_TEACHER_ENTRIES;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Targets {             // q_tj
  const int32_t* ids; int64_t ld_ids; int k;
  const float* z; int64_t ld_z;          // teacher logits; null: every present entry has q = 1 (k = 1)
  const float* teacher_lse;              // or null: softmax over the present entries
  float inv_temp;
};

struct RowArgs {
  Targets tg;
  bf16* u; int64_t ldu;                  // powers in, ds out (this sub-chunk's rows); null without gradients
  const float2* stats; int64_t ld_pieces; int n_pieces;
  const bf16* X; int64_t ldx; const bf16* E; int64_t lde; int d, V;
  int64_t row0;                          // first row of the sub-chunk
  float scale2;                          // log2(e) / temperature
  const float* weight; const int* count; // weight null: 1 / *count
  float *row_loss, *lse, *weighted;      // per row; the first two may be null
  int* flags;
};

// an id outside [0, V): negative entries are absent, others are left out and reported
__device__ __forceinline__ bool present_id(int id, int V, int* flags) {
  if (id >= V && flags) atomicExch(flags + PPU_FLAG_TOKEN, 1);
  return id >= 0 && id < V;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ void unpack8(const uint4& u, float* f) {
  const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&u);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 t = __bfloat1622float2(p[i]);
    f[2 * i] = t.x; f[2 * i + 1] = t.y;
  }
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  uint4 u;
  __nv_bfloat162* p = reinterpret_cast<__nv_bfloat162*>(&u);
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
  return u;
}

// sum s 2^m over {m, s} pairs, kept relative to the largest m; an empty pair is {-inf, 0}
struct Piece { float m, s; };
__device__ __forceinline__ Piece join(Piece a, Piece b) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return {m, a.s + b.s};     // (keeps a NaN)
  return {m, a.s * exp2f(a.m - m) + b.s * exp2f(b.m - m)};
}

// rows with at least one present entry (integer atomics: any order gives the same count)
__global__ void __launch_bounds__(256) count_rows_kernel(Targets tg, int T, int V, int* count) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  bool any = false;
  if (t < T)
    for (int j = 0; j < tg.k && !any; ++j) {
      const int id = tg.ids[t * tg.ld_ids + j];
      any = id >= 0 && id < V && !(tg.z && tg.z[t * tg.ld_z + j] * tg.inv_temp == -INFINITY);
    }
  const int n = __syncthreads_count(any);
  if (threadIdx.x == 0 && n) atomicAdd(count, n);
}

template <bool GRAD>
__global__ void __launch_bounds__(ROW_THREADS) head_rows_kernel(const RowArgs a) {
  __shared__ int s_id[MAX_ENTRIES];
  __shared__ float s_q[MAX_ENTRIES], s_l[MAX_ENTRIES];
  __shared__ float s_total, s_entropy;
  __shared__ int s_any;
  __shared__ Piece s_piece[ROW_THREADS / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t row = blockIdx.x, t = a.row0 + row;
  const int k = a.tg.k;

  // the row's entries and their q (warp 0), while every thread joins its share of the pieces
  if (warp == 0) {
    constexpr int PER = MAX_ENTRIES / 32;
    float zs[PER]; int id[PER]; bool in[PER];
    float top = -INFINITY;
    bool any = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int j = lane + 32 * i;
      id[i] = -1; zs[i] = 0.f; in[i] = false;
      if (j < k) {
        id[i] = a.tg.ids[t * a.tg.ld_ids + j];
        in[i] = present_id(id[i], a.V, a.flags);
        if (in[i] && a.tg.z) {
          zs[i] = a.tg.z[t * a.tg.ld_z + j] * a.tg.inv_temp;
          in[i] = !(zs[i] == -INFINITY);
        }
      }
      if (in[i]) { top = fmaxf(top, zs[i]); any = true; }
    }
    any = __any_sync(0xffffffffu, any);
    float norm = 0.f;                      // a hard target: q = exp(0)
    if (a.tg.z) {
      if (a.tg.teacher_lse) norm = a.tg.teacher_lse[t];
      else {
        top = warp_max(top);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) if (in[i]) s += expf(zs[i] - top);
        norm = top + logf(warp_sum(s));
      }
    }
    float total = 0.f, entropy = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int j = lane + 32 * i;
      float q = 0.f;
      if (in[i]) {
        q = expf(zs[i] - norm);
        if (q != 0.f) entropy += q * (zs[i] - norm);
        total += q;
      }
      if (j < k) { s_id[j] = in[i] ? id[i] : -1; s_q[j] = q; }
    }
    total = warp_sum(total); entropy = warp_sum(entropy);
    if (lane == 0) { s_total = total; s_entropy = entropy; s_any = any; }
  }
  const float2* st = a.stats + row * a.ld_pieces;
  Piece mine = {-INFINITY, 0.f};
  for (int i = threadIdx.x; i < a.n_pieces; i += ROW_THREADS) {
    const float2 v = st[i];
    if (v.y != 0.f) mine = join(mine, {v.x, v.y});
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Piece other = {__shfl_xor_sync(0xffffffffu, mine.m, o), __shfl_xor_sync(0xffffffffu, mine.s, o)};
    mine = join(mine, other);
  }
  if (lane == 0) s_piece[warp] = mine;
  __syncthreads();
  Piece all = s_piece[0];
#pragma unroll
  for (int w = 1; w < ROW_THREADS / 32; ++w) all = join(all, s_piece[w]);
  const float lse2 = all.m + log2f(all.s);          // base 2
  if (threadIdx.x == 0 && a.lse) a.lse[t] = lse2 * LN2;

  if (!s_any) {                                     // block-uniform: the row has no loss and no gradient
    if (threadIdx.x == 0) { if (a.row_loss) a.row_loss[t] = 0.f; a.weighted[t] = 0.f; }
    if (GRAD)
      for (int i = threadIdx.x; i < a.ldu / 8; i += ROW_THREADS)
        reinterpret_cast<uint4*>(a.u + row * a.ldu)[i] = make_uint4(0, 0, 0, 0);
    return;
  }
  // the entries' logits, one warp each
  const uint4* xr = reinterpret_cast<const uint4*>(a.X + t * a.ldx);
  for (int j = warp; j < k; j += ROW_THREADS / 32) {
    if (s_id[j] < 0) continue;
    const uint4* er = reinterpret_cast<const uint4*>(a.E + (int64_t)s_id[j] * a.lde);
    float acc = 0.f;
    for (int i = lane; i < a.d / 8; i += 32) {
      float x[8], e[8];
      unpack8(xr[i], x); unpack8(er[i], e);
#pragma unroll
      for (int c = 0; c < 8; ++c) acc = fmaf(x[c], e[c], acc);
    }
    acc = warp_sum(acc);
    if (lane == 0) s_l[j] = acc * a.scale2;
  }
  __syncthreads();
  const float w = a.weight ? a.weight[t] : 1.f / (float)*a.count;
  if (threadIdx.x == 0) {
    float x = 0.f;
    for (int j = 0; j < k; ++j)
      if (s_id[j] >= 0 && s_q[j] != 0.f) x = fmaf(s_q[j], lse2 - s_l[j], x);
    const float l = s_entropy + x * LN2;
    if (a.row_loss) a.row_loss[t] = l;
    a.weighted[t] = w * l;
  }
  if (!GRAD) return;
  const float c = w * a.tg.inv_temp, cq = c * s_total;
  uint4* ur = reinterpret_cast<uint4*>(a.u + row * a.ldu);
  const int nvec = (int)(a.ldu / 8);
#pragma unroll 4
  for (int i = threadIdx.x; i < nvec; i += ROW_THREADS) {
    const float f = cq * exp2f(st[i / (PIECE / 8)].x - lse2);
    float v[8];
    unpack8(ur[i], v);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] *= f;
    ur[i] = pack8(v);
  }
  __syncthreads();                                  // the entries' places have been written: overwrite them
  for (int j = threadIdx.x; j < k; j += ROW_THREADS) {
    const int id = s_id[j];
    if (id < 0) continue;
    float q = 0.f;
    bool first = true;                              // an id given twice: its first entry writes for all
    for (int i = 0; i < k; ++i)
      if (s_id[i] == id) { if (i < j) first = false; q += s_q[i]; }
    // Q p - q with p = exp(x): Q (exp(x) - 1) + (Q - q) keeps its digits where p is next to 1
    if (first) a.u[row * a.ldu + id] = __float2bfloat16_rn(c * (s_total * expm1f((s_l[j] - lse2) * LN2) + (s_total - q)));
  }
}

__global__ void __launch_bounds__(1024) sum_rows_kernel(const float* __restrict__ v, int T, float* out) {
  __shared__ float red[32];
  float s = 0.f;
#pragma unroll 4
  for (int i = threadIdx.x; i < T; i += 1024) s += v[i];
  s = warp_sum(s);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x < 32) {
    s = warp_sum(red[threadIdx.x]);
    if (threadIdx.x == 0) *out = s;
  }
}

// out bf16 [rows, n] = sum of `splits` fp32 partial products, in index order
__global__ void __launch_bounds__(256)
join_partials_kernel(const float* __restrict__ part, int splits, int64_t stride, bf16* __restrict__ out, int64_t ldo, int rows, int n8) {
  const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
  if (i >= (int64_t)rows * n8) return;
  float s[8] = {};
#pragma unroll 4
  for (int q = 0; q < splits; ++q) {
    const float4* p = reinterpret_cast<const float4*>(part + q * stride + i * 8);
    const float4 x = p[0], y = p[1];
    s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
    s[4] += y.x; s[5] += y.y; s[6] += y.z; s[7] += y.w;
  }
  *reinterpret_cast<uint4*>(out + (i / n8) * ldo + (i % n8) * 8) = pack8(s);
}

// ---- host ---------------------------------------------------------------------------------------
constexpr int64_t U_BYTES = 256ll << 20;      // default bound of a chunk's powers
constexpr int64_t L2_BYTES = 64ll << 20;      // a sub-chunk's powers, re-read while in the L2 (126 MB)
constexpr int SMS = 148;                      // work is split for a B200 (also where sizes are asked without a device)

int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// slices of the reduction for a [M, N] product over K: as many as bring the output's tiles near one
// wave, each at least 256 long
int splits_for(int64_t M, int64_t N, int64_t K) {
  const int64_t pair = ((M + 255) / 256) * ((N + 255) / 256);
  int64_t tiles = pair, units = SMS / 2;
  if (M <= 128 || N <= 128 || pair < 16) { tiles = ((M + 127) / 128) * ((N + 127) / 128); units = SMS; }
  return (int)std::max<int64_t>(1, std::min<int64_t>(units / tiles, K / 256));
}

struct Plan {
  int64_t ldu, n_pieces, chunk, sub;
  int chunks, sx, se;                          // split-K factors of dX and dE
  size_t off_weighted, off_stats, off_u, off_acc, off_part, bytes;
};
Plan make_plan(int T, int d, int V, int want, int chunk_rows) {
  Plan p;
  p.ldu = round_up(V, PIECE);
  p.n_pieces = p.ldu / PIECE;
  const int64_t row_bytes = want ? p.ldu * 2 : p.n_pieces * 8;     // (without gradients only the pieces' statistics)
  T = std::max(T, 1);
  int64_t c = chunk_rows > 0 ? round_up(chunk_rows, 256) : std::max<int64_t>(256, U_BYTES / row_bytes / 256 * 256);
  p.chunks = (int)std::max<int64_t>(1, (T + c - 1) / c);
  p.chunk = p.chunks == 1 ? T : round_up((T + p.chunks - 1) / p.chunks, 256);
  p.sub = want ? std::min<int64_t>(p.chunk, std::max<int64_t>(256, L2_BYTES / row_bytes / 256 * 256)) : p.chunk;
  p.sx = (want & 1) ? splits_for(p.chunk, d, V) : 1;
  p.se = (want & 2) && p.chunks == 1 ? splits_for(V, d, p.chunk) : 1;
  size_t off = 256;                            // the row count
  auto take = [&off](int64_t bytes) { const size_t at = off; off += (size_t)round_up(bytes, 256); return at; };
  p.off_weighted = take(4ll * T);
  p.off_stats = take(8ll * p.sub * p.n_pieces);
  p.off_u = take(want ? p.chunk * row_bytes : 0);
  p.off_acc = take((want & 2) && p.chunks > 1 ? 4ll * V * d : 0);
  int64_t part = 0;
  if (p.sx > 1) part = 4ll * p.sx * p.chunk * d;
  if (p.se > 1) part = std::max<int64_t>(part, 4ll * p.se * V * d);
  p.off_part = take(part);
  p.bytes = off;
  return p;
}

int check_sizes(int T, int d, int V, int chunk_rows) {
  if (T < 0 || d < 1 || V < 1 || chunk_rows < 0) return ppu_fail(PPU_EINVAL, "negative or empty size");
  if (d % 8 || d > 16384) return ppu_fail(PPU_ESHAPE, "d must be a multiple of 8 up to 16384 (got %d)", d);
  if (T > (1 << 20) || V > (1 << 22)) return ppu_fail(PPU_ESHAPE, "at most 2^20 rows and 2^22 vocabulary entries");
  return PPU_OK;
}

struct HeadCall {
  const void *X, *E; int64_t ldx, lde;
  Targets tg;
  const float* weight;
  int T, d, V;
  float temp;
  float *loss, *row_loss, *lse;
  void *dX, *dE; int64_t lddx, ldde;
  int chunk_rows;
  void* ws; size_t ws_bytes;
  int* flags;
  cudaStream_t st;
};

#define CUDA_OK(call)                                                                    \
  do {                                                                                   \
    cudaError_t e_ = (call);                                                             \
    if (e_ != cudaSuccess)                                                               \
      return ppu_fail(PPU_ECUDA, "%s failed: %s", #call, cudaGetErrorString(e_));        \
  } while (0)
#define GEMM_OK(call)                                                                    \
  do {                                                                                   \
    const int r_ = (call);                                                               \
    if (r_) return ppu_fail(r_ == -4 ? PPU_ESHAPE : PPU_ECUDA, "head product failed (%d)", r_); \
  } while (0)

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// bf16 C = A . B^T, split over K into fp32 partials where that fills the machine
int product_bf16(GemmArgs g, int splits, float* part, cudaStream_t st) {
  if (splits <= 1) { g.epilogue = EPI_STORE_BF16; GEMM_OK(launch_gemm_tc(g, st)); return PPU_OK; }
  bf16* out = (bf16*)g.C; const int64_t ldo = g.ldc;
  g.epilogue = EPI_STORE_F32; g.C = part; g.ldc = g.N; g.splits = splits; g.split_stride = (int64_t)g.M * g.N;
  GEMM_OK(launch_gemm_tc(g, st));
  const int64_t n = (int64_t)g.M * (g.N / 8);
  join_partials_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(part, splits, g.split_stride, out, ldo, g.M, g.N / 8);
  return PPU_OK;
}

int run_head(const HeadCall& c) {
  const int want = (c.dX ? 1 : 0) | (c.dE ? 2 : 0);
  int rc = check_sizes(c.T, c.d, c.V, c.chunk_rows);
  if (rc) return rc;
  if (!c.loss || !c.ws || !c.E || (c.T && (!c.X || !c.tg.ids))) return ppu_fail(PPU_EINVAL, "null operand");
  if (c.ldx < c.d || c.lde < c.d || (c.dX && c.lddx < c.d) || (c.dE && c.ldde < c.d) || c.ldx % 8 || c.lde % 8 ||
      (c.dX && c.lddx % 8) || (c.dE && c.ldde % 8))
    return ppu_fail(PPU_EINVAL, "row strides must be multiples of 8 and at least d");
  if (!aligned16(c.X) || !aligned16(c.E) || !aligned16(c.dX) || !aligned16(c.dE))
    return ppu_fail(PPU_EINVAL, "operands must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(c.ws) & 255) return ppu_fail(PPU_EINVAL, "workspace not 256-byte aligned");
  const Plan p = make_plan(c.T, c.d, c.V, want, c.chunk_rows);
  if (c.ws_bytes < p.bytes) return ppu_fail(PPU_ENOMEM, "workspace has %zu bytes, %zu needed", c.ws_bytes, p.bytes);

  uint8_t* ws = (uint8_t*)c.ws;
  int* count = (int*)ws;
  float* weighted = (float*)(ws + p.off_weighted);
  float2* stats = (float2*)(ws + p.off_stats);
  bf16* u = want ? (bf16*)(ws + p.off_u) : nullptr;
  float* acc = (float*)(ws + p.off_acc);
  float* part = (float*)(ws + p.off_part);

  if (c.T == 0) {                              // a mean over nothing: no loss, no gradient
    CUDA_OK(cudaMemsetAsync(c.loss, 0, 4, c.st));
    if (c.dE) CUDA_OK(cudaMemset2DAsync(c.dE, (size_t)c.ldde * 2, 0, (size_t)c.d * 2, (size_t)c.V, c.st));
    return PPU_OK;
  }
  if (!c.weight) {
    CUDA_OK(cudaMemsetAsync(count, 0, 4, c.st));
    count_rows_kernel<<<(c.T + 255) / 256, 256, 0, c.st>>>(c.tg, c.T, c.V, count);
  }
  RowArgs r;
  r.tg = c.tg; r.ldu = p.ldu; r.ld_pieces = p.n_pieces; r.n_pieces = (int)p.n_pieces; r.stats = stats;
  r.X = (const bf16*)c.X; r.ldx = c.ldx; r.E = (const bf16*)c.E; r.lde = c.lde; r.d = c.d; r.V = c.V;
  r.scale2 = LOG2E / c.temp; r.weight = c.weight; r.count = count;
  r.row_loss = c.row_loss; r.lse = c.lse; r.weighted = weighted; r.flags = c.flags;

  GemmArgs g0;
  g0.C2 = nullptr; g0.aux = nullptr; g0.ldaux = 0; g0.flags = c.flags; g0.transient = true;
  for (int ch = 0; ch < p.chunks; ++ch) {
    const int64_t c0 = ch * p.chunk, rows = std::min<int64_t>(p.chunk, c.T - c0);
    if (rows <= 0) break;
    for (int64_t s0 = 0; s0 < rows; s0 += p.sub) {
      const int64_t n = std::min<int64_t>(p.sub, rows - s0);
      GemmArgs g = g0;
      g.A = r.X + (c0 + s0) * c.ldx; g.lda = c.ldx; g.a_kmajor = 1;
      g.B = r.E; g.ldb = c.lde; g.b_kmajor = 1;
      g.M = (int)n; g.N = c.V; g.K = c.d; g.epilogue = EPI_PIECES;
      g.C = u ? u + s0 * p.ldu : nullptr; g.ldc = p.ldu;
      g.piece_scale = r.scale2; g.piece_stats = stats; g.ld_pieces = p.n_pieces;
      GEMM_OK(launch_gemm_tc_pieces(g, c.st));
      r.row0 = c0 + s0; r.u = u ? u + s0 * p.ldu : nullptr;
      if (want) head_rows_kernel<true><<<(unsigned)n, ROW_THREADS, 0, c.st>>>(r);
      else head_rows_kernel<false><<<(unsigned)n, ROW_THREADS, 0, c.st>>>(r);
    }
    if (c.dX) {
      GemmArgs g = g0;
      g.A = u; g.lda = p.ldu; g.a_kmajor = 1; g.B = r.E; g.ldb = c.lde; g.b_kmajor = 0;
      g.M = (int)rows; g.N = c.d; g.K = c.V; g.C = (bf16*)c.dX + c0 * c.lddx; g.ldc = c.lddx;
      rc = product_bf16(g, p.sx, part, c.st);
      if (rc) return rc;
    }
    if (c.dE) {
      GemmArgs g = g0;
      g.A = u; g.lda = p.ldu; g.a_kmajor = 0; g.B = r.X + c0 * c.ldx; g.ldb = c.ldx; g.b_kmajor = 0;
      g.M = c.V; g.N = c.d; g.K = (int)rows; g.C = c.dE; g.ldc = c.ldde;
      const bool last = ch == p.chunks - 1 || c0 + p.chunk >= c.T;
      if (ch == 0 && last) {
        rc = product_bf16(g, p.se, part, c.st);
        if (rc) return rc;
      } else if (last) {
        g.epilogue = EPI_RESID_BF16; g.aux = acc; g.ldaux = c.d;
        GEMM_OK(launch_gemm_tc_resid_bf16(g, c.st));
      } else {
        g.epilogue = ch == 0 ? EPI_STORE_F32 : EPI_RESID_F32;
        g.C = acc; g.ldc = c.d; g.aux = acc; g.ldaux = c.d;
        GEMM_OK(launch_gemm_tc(g, c.st));
      }
    }
  }
  sum_rows_kernel<<<1, 1024, 0, c.st>>>(weighted, c.T, c.loss);
  CUDA_OK(cudaGetLastError());
  return PPU_OK;
}

}  // namespace

extern "C" int ppu_head_query_bytes(int T, int d, int V, int grads, int chunk_rows, size_t* bytes) {
  if (!bytes) return ppu_fail(PPU_EINVAL, "bytes is null");
  if (grads < 0 || grads > 3) return ppu_fail(PPU_EINVAL, "grads is a sum of 1 (dX) and 2 (dE)");
  const int rc = check_sizes(T, d, V, chunk_rows);
  if (rc) return rc;
  *bytes = make_plan(T, d, V, grads, chunk_rows).bytes;
  return PPU_OK;
}

extern "C" int ppu_head_xent(const void* X, int64_t ldx, const void* E, int64_t lde, const int32_t* target,
                             const float* row_weight, int T, int d, int V, float* loss, float* row_loss,
                             float* lse, void* dX, int64_t lddx, void* dE, int64_t ldde, int chunk_rows,
                             void* workspace, size_t workspace_bytes, int32_t* flags, void* cuda_stream) {
  HeadCall c;
  c.X = X; c.E = E; c.ldx = ldx; c.lde = lde;
  c.tg = Targets{target, 1, 1, nullptr, 0, nullptr, 1.f};
  c.weight = row_weight; c.T = T; c.d = d; c.V = V; c.temp = 1.f;
  c.loss = loss; c.row_loss = row_loss; c.lse = lse; c.dX = dX; c.dE = dE; c.lddx = lddx; c.ldde = ldde;
  c.chunk_rows = chunk_rows; c.ws = workspace; c.ws_bytes = workspace_bytes; c.flags = flags;
  c.st = (cudaStream_t)cuda_stream;
  return run_head(c);
}

extern "C" int ppu_head_distill(const void* X, int64_t ldx, const void* E, int64_t lde, const int32_t* teacher_ids,
                                int64_t ld_ids, const float* teacher_logits, int64_t ld_logits, int k,
                                const float* teacher_lse, float temperature, const float* row_weight, int T,
                                int d, int V, float* loss, float* row_loss, float* lse, void* dX, int64_t lddx,
                                void* dE, int64_t ldde, int chunk_rows, void* workspace,
                                size_t workspace_bytes, int32_t* flags, void* cuda_stream) {
  if (k < 1 || k > PPU_MAX_TEACHER_ENTRIES)
    return ppu_fail(PPU_ESHAPE, "k must lie in 1..%d (got %d)", PPU_MAX_TEACHER_ENTRIES, k);
  if (!(temperature > 0.f) || !(temperature < 1e6f)) return ppu_fail(PPU_EINVAL, "temperature must be positive");
  if (ld_ids < k || ld_logits < k) return ppu_fail(PPU_EINVAL, "teacher row strides must be at least k");
  if (T && !teacher_logits) return ppu_fail(PPU_EINVAL, "null operand");
  HeadCall c;
  c.X = X; c.E = E; c.ldx = ldx; c.lde = lde;
  c.tg = Targets{teacher_ids, ld_ids, k, teacher_logits, ld_logits, teacher_lse, 1.f / temperature};
  c.weight = row_weight; c.T = T; c.d = d; c.V = V; c.temp = temperature;
  c.loss = loss; c.row_loss = row_loss; c.lse = lse; c.dX = dX; c.dE = dE; c.lddx = lddx; c.ldde = ldde;
  c.chunk_rows = chunk_rows; c.ws = workspace; c.ws_bytes = workspace_bytes; c.flags = flags;
  c.st = (cudaStream_t)cuda_stream;
  return run_head(c);
}

// error words of the operators above: waits for the stream, reports and clears them
extern "C" int ppu_op_status(int32_t* flags, void* cuda_stream) {
  if (!flags) return ppu_fail(PPU_EINVAL, "flags is null");
  int h[PPU_FLAG_COUNT];
  CUDA_OK(cudaMemcpyAsync(h, flags, sizeof(h), cudaMemcpyDeviceToHost, (cudaStream_t)cuda_stream));
  CUDA_OK(cudaStreamSynchronize((cudaStream_t)cuda_stream));
  if (!h[PPU_FLAG_TOKEN] && !h[PPU_FLAG_TIMEOUT]) return PPU_OK;
  CUDA_OK(cudaMemsetAsync(flags, 0, sizeof(h), (cudaStream_t)cuda_stream));
  if (h[PPU_FLAG_TIMEOUT]) return ppu_fail(PPU_ETIMEOUT, "a bounded wait inside a kernel expired");
  return ppu_fail(PPU_ETOKEN, "an id outside [0, vocab) was left out");
}
