// Losses of hidden states against a large vocabulary, worked in chunks of rows: softmax cross entropy and
// distillation from a teacher's top logits, with the gradients of the hidden states and of the vocabulary
// matrix.
//
//   s = X E^T / temperature,  lse_t = log sum_v exp(s_tv),  p = softmax(s)
//   row loss = sum_j q_tj (log q_tj - s_t,id(j) + lse_t)        (cross entropy: one entry, q = 1)
//   ds_tv = w_t (Q_t p_tv - sum_{j: id(j) = v} q_tj),  Q_t = sum_j q_tj
//   dX = ds E / temperature,  dE = ds^T X / temperature
//
// Three matrix products cannot be avoided (6 T V d operations), and a backward pass that forms the
// logits again would make it four.  So rows are worked in chunks, whose softmax is kept only until
// the chunk's two gradient products are done: a [rows, V] buffer of bounded size, not [T, V].  (Where one chunk is all, up
// to 6144 rows, that is what bf16 logits would take, and with the running dE of two chunks 8192 x 2048 x 32768 takes
// 571 MB where its logits are 537.  From there on it grows no further than to 726 MB, for 2^20 rows whose logits are 69 GB;
// without dE 8192 rows take 285 MB, for the loss alone 17.)
//   1. tcgen05 product of the chunk's rows with E^T.  Its epilogue works the vocabulary in pieces of 64
//      columns: bf16 powers u = 2^(x - ref), x = s log2(e), and {ref, sum} in fp32; ref is 0 for ordinary
//      logits (within 41 nats of 0), else the piece's maximum, as a whole number.  The entries' own x are kept in fp32 (the powers
//      would be too coarse for the loss and for p - 1 next to p = 1); for that a kernel before it has
//      sorted each row's entries and counted how many lie before each piece (not needed for one entry a row).
//   2. a warp or a block per row joins the pieces to the row's log-sum-exp and forms the row loss.  Then
//      ds_tv = f_t u_tv with one factor per row: the powers stay as they are, but for the entries'
//      places, which are overwritten, and for pieces (rows) beyond the range of the common reference,
//      which are rescaled.
//   3. dX = f (u E), the factor applied in the product's epilogue, and dE = u^T (f X) with f X formed in
//      step 2, both in one launch; dE over several chunks is a running fp32 sum, rounded once by the last.
// Step 2 once rewrote the whole buffer as ds: 27 us per 1024 rows of 32768 (L2-resident), 7 % of the
// call at 8192 rows of d = 2048.
// Roundings: u and f X are bf16 (the tensor cores' operand type; each off by at most half a step, 2^-8 of
// its own value; f is off by as much for all but the entries' places, see there), dX and dE are rounded
// once from fp32; statistics, losses and running sums are fp32.  Powers below 2^-126 are 0: probabilities below 2^-66 at
// worst, in a row whose logits all lie 41 nats below 0.  (The tensor cores' fp32 sums drop what
// lies below the last bit, so logits come out low: by 1.2e-6 of the log-sum-exp at d = 2048.)
#include <algorithm>
#include <climits>
#include "../../include/ppu.h"
#include "common.cuh"

int ppu_fail(int code, const char* fmt, ...);

namespace {

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
  bf16* u; int64_t ldu;                  // powers of this chunk's rows; null without gradients
  const float2* stats; int64_t ld_pieces; int n_pieces;
  const bf16* X; int64_t ldx; int d, V;
  const float2* x;                       // the entries' {x - ref, ref} [rows][k]
  int sorted;                            // tg is the chunk's own (sorted) copy: its rows are the chunk's
  int64_t row0;                          // first row of the chunk
  int T;
  float scale2;                          // log2(e) / temperature
  const float* weight; const int* count; // weight null: 1 / *count, or where that is null too, the blocks count the rows themselves
  float *row_loss, *lse, *weighted;      // per row; the first two may be null
  float* factor;                         // f, of this chunk's rows
  bf16* fx;                              // f X [rows][d], or null
  unsigned *done, blocks; float* loss;   // blocks finished so far, and all there will be; sum of `weighted`, by the last of them
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
__device__ __forceinline__ void unpack8(const uint4 u, float* f) {
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

__device__ __forceinline__ bool row_counts(const Targets& tg, int64_t t, int V) {
  for (int j = 0; j < tg.k; ++j) {
    const int id = tg.ids[t * tg.ld_ids + j];
    if (id >= 0 && id < V && !(tg.z && tg.z[t * tg.ld_z + j] * tg.inv_temp == -INFINITY)) return true;
  }
  return false;
}
// rows with at least one present entry (integer atomics: any order gives the same count)
__global__ void __launch_bounds__(256) count_rows_kernel(Targets tg, int T, int V, int* count) {
  pdl_wait(); pdl_trigger();
  const int64_t t = blockIdx.x * 256 + threadIdx.x;
  const int n = __syncthreads_count(t < T && row_counts(tg, t, V));
  if (threadIdx.x == 0 && n) atomicAdd(count, n);
}
// the same by one block, which needs no zeroed count: one launch less
__global__ void __launch_bounds__(1024) count_rows_block_kernel(Targets tg, int T, int V, int* count) {
  __shared__ int s_n[32];
  pdl_wait(); pdl_trigger();
  int n = 0;
#pragma unroll 4
  for (int64_t t = threadIdx.x; t < T; t += 1024) n += row_counts(tg, t, V);
  n = __reduce_add_sync(0xffffffffu, n);
  if ((threadIdx.x & 31) == 0) s_n[threadIdx.x >> 5] = n;
  __syncthreads();
  if (threadIdx.x < 32) {
    n = __reduce_add_sync(0xffffffffu, s_n[threadIdx.x]);
    if (threadIdx.x == 0) *count = n;
  }
}

// scales 64 stored powers (by a power of two: no rounding)
__device__ __forceinline__ void scale_piece(bf16* p, float f) {
#pragma unroll
  for (int i = 0; i < PIECE / 8; ++i) {
    float v[8];
    unpack8(reinterpret_cast<const uint4*>(p)[i], v);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] *= f;
    reinterpret_cast<uint4*>(p)[i] = pack8(v);
  }
}

// A chunk's entries, each row's in ascending order of id (the rank of each by comparing it with all: k is at most
// 128), absent ones as -1 behind them; and off[p] = entries before piece p.  One warp to a row.
__global__ void __launch_bounds__(128) sort_entries_kernel(Targets tg, int64_t row0, int rows, int V, int n_pieces, int32_t* ids, float* zs, uint8_t* off,
                                                           int64_t ld_off, int* flags) {
  __shared__ int s_key[4][MAX_ENTRIES], s_id[4][MAX_ENTRIES];
  pdl_wait(); pdl_trigger();
  const int lane = threadIdx.x & 31, g = threadIdx.x >> 5;
  const int64_t row = (int64_t)blockIdx.x * 4 + g, t = row0 + row;
  if (row >= rows) return;
  constexpr int PER = MAX_ENTRIES / 32;
  float z[PER];
  int key[PER], present = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = lane + 32 * i;
    key[i] = INT_MAX; z[i] = 0.f;
    if (j < tg.k) {
      const int id = tg.ids[t * tg.ld_ids + j];
      z[i] = tg.z[t * tg.ld_z + j];
      if (present_id(id, V, flags) && !(z[i] * tg.inv_temp == -INFINITY)) { key[i] = id; ++present; }
      s_key[g][j] = key[i];
    }
  }
  present = __reduce_add_sync(0xffffffffu, present);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = lane + 32 * i;
    if (j >= tg.k) continue;
    int rank = 0;
    for (int q = 0; q < tg.k; ++q) rank += s_key[g][q] < key[i] || (s_key[g][q] == key[i] && q < j);
    const int id = key[i] == INT_MAX ? -1 : key[i];
    s_id[g][rank] = id;
    ids[row * tg.k + rank] = id;
    zs[row * tg.k + rank] = z[i];
  }
  __syncwarp();
  // a lane goes through a 32nd of the pieces, four to a store; where it starts it searches
  const int n4 = (int)(ld_off / 4), per = (n4 + 31) / 32;
  int at = 0;
  {
    int hi = present;
    const int first = 4 * per * lane * PIECE;
    while (at < hi) {
      const int mid = (at + hi) / 2;
      if (s_id[g][mid] < first) at = mid + 1; else hi = mid;
    }
  }
  for (int w = per * lane; w < min(n4, per * (lane + 1)); ++w) {
    uint32_t word = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      while (at < present && s_id[g][at] < (4 * w + b) * PIECE) ++at;
      word |= (uint32_t)at << (8 * b);
    }
    *reinterpret_cast<uint32_t*>(off + row * ld_off + 4 * w) = word;
  }
}

// Step 2 for W warps to a row: one (four rows to a block, no barrier) where the rows alone fill the
// machine, 4 or 16 for few rows with many pieces or entries to go through.
template <bool GRAD, int W>
__global__ void __launch_bounds__(W == 1 ? 128 : 32 * W) head_rows_kernel(const RowArgs a, int rows) {
  constexpr int R = W == 1 ? 4 : 1, THREADS = W == 1 ? 128 : 32 * W, N = 32 * W;     // rows and threads of a block, threads of a row
  __shared__ int s_id[R][MAX_ENTRIES];
  __shared__ float s_q[R][MAX_ENTRIES], s_v[R][MAX_ENTRIES];
  __shared__ float2 s_x[R][MAX_ENTRIES];
  __shared__ float s_total[R], s_entropy[R], s_f[R], s_inv[R], s_sum[16];
  __shared__ int s_any[R], s_last, s_count[THREADS / 32];
  __shared__ Piece s_piece[W];
  const int lane = threadIdx.x & 31, warp = W == 1 ? 0 : threadIdx.x >> 5, tid = W == 1 ? lane : threadIdx.x;   // of the row
  const int g = W == 1 ? threadIdx.x >> 5 : 0;
  const int64_t row = (int64_t)blockIdx.x * R + g, t = a.row0 + row;        // row of the chunk, of the call
  const int k = a.tg.k;
  const int64_t te = a.sorted ? row : t;                                     // row of the entries
  auto sync = [] { if constexpr (W == 1) __syncwarp(); else __syncthreads(); };

  pdl_wait(); pdl_trigger();
  if (!a.weight && !a.count) {
    int n = 0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < a.T; i += THREADS) n += row_counts(a.tg, i, a.V);
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) s_count[threadIdx.x >> 5] = n;
    __syncthreads();
  }
  if (row < rows) {
    // what the row needs from global memory is asked for first: the rest is a chain of short steps
    const float2* st = a.stats + row * a.ld_pieces;
    const uint4* xr = reinterpret_cast<const uint4*>(a.X + t * a.ldx);
    const float2 st0 = tid < a.n_pieces ? st[tid] : make_float2(0.f, 0.f);
    uint4 x0 = make_uint4(0, 0, 0, 0);
    if (GRAD && a.fx && tid < a.d / 8) x0 = xr[tid];
    const float row_weight = a.weight ? a.weight[t] : 0.f;
    // the row's entries and their q
    if (warp == 0) {
      constexpr int PER = MAX_ENTRIES / 32;
      float zs[PER]; float2 ex[PER]; int id[PER]; bool in[PER];
      float top = -INFINITY;
      bool any = false;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int j = lane + 32 * i;
        id[i] = -1; zs[i] = 0.f; ex[i] = make_float2(0.f, 0.f); in[i] = false;
        if (j < k) {
          id[i] = a.tg.ids[te * a.tg.ld_ids + j];
          ex[i] = a.x[row * k + j];                 // (of an absent entry: whatever is there, and not used)
          if (a.tg.z) zs[i] = a.tg.z[te * a.tg.ld_z + j] * a.tg.inv_temp;
        }
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if (lane + 32 * i < k) in[i] = present_id(id[i], a.V, a.flags) && !(zs[i] == -INFINITY);
        if (in[i]) { top = fmaxf(top, zs[i]); any = true; }
      }
      any = __any_sync(0xffffffffu, any);
      float norm = 0.f;                    // a hard target: q = exp(0)
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
        if (j < k) { s_id[g][j] = in[i] ? id[i] : -1; s_q[g][j] = q; s_x[g][j] = ex[i]; }
      }
      total = warp_sum(total); entropy = warp_sum(entropy);
      if (lane == 0) { s_total[g] = total; s_entropy[g] = entropy; s_any[g] = any; }
    }
    // the pieces: with the common reference throughout, a plain sum
    Piece all = {0.f, st0.y};
    bool plain = st0.x == 0.f;
#pragma unroll 4
    for (int i = tid + N; i < a.n_pieces; i += N) {
      const float2 v = st[i];
      plain &= v.x == 0.f;
      all.s += v.y;
    }
    if constexpr (W == 1) plain = __all_sync(0xffffffffu, plain);
    else plain = __syncthreads_and(plain);
    if (plain) {
      all.s = warp_sum(all.s);
    } else {
      all = {-INFINITY, 0.f};
      for (int i = tid; i < a.n_pieces; i += N) {
        const float2 v = st[i];
        if (v.y != 0.f) all = join(all, {v.x, v.y});
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        all = join(all, {__shfl_xor_sync(0xffffffffu, all.m, o), __shfl_xor_sync(0xffffffffu, all.s, o)});
    }
    if constexpr (W > 1) {
      if (lane == 0) s_piece[warp] = all;
      __syncthreads();
      all = s_piece[0];
      for (int w = 1; w < W; ++w) all = join(all, s_piece[w]);
    } else {
      __syncwarp();
    }
    // The row's powers are relative to the largest of its pieces' references (0 for ordinary logits) and add up to
    // all.s: p = u / all.s.  What follows uses the two apart: far from 0 their sum, the log-sum-exp, is rounded to
    // more than the powers are (at 2^20 to 2^-4, an error of 4 % of p).
    const float ref = all.m, log_s = log2f(all.s);       // base 2
    if (tid == 0 && a.lse) a.lse[t] = (ref + log_s) * LN2;
    bf16* ur = a.u + row * a.ldu;
    uint4* fx = GRAD && a.fx ? reinterpret_cast<uint4*>(a.fx + row * a.d) : nullptr;
    if (!s_any[g]) {                                // the row has no loss and no gradient
      if (tid == 0) {
        if (a.row_loss) a.row_loss[t] = 0.f;
        a.weighted[t] = 0.f;
        if (GRAD) a.factor[row] = 0.f;
      }
      if (GRAD) {
        if (!isfinite(all.s))                       // (0 times the powers has to be 0)
          for (int i = tid; i < a.ldu / 8; i += N) reinterpret_cast<uint4*>(ur)[i] = make_uint4(0, 0, 0, 0);
        if (fx)
          for (int i = tid; i < a.d / 8; i += N) fx[i] = make_uint4(0, 0, 0, 0);
      }
    } else {
      const int n8 = a.d / 8;
      float w;
      if (a.weight) {
        w = row_weight;
      } else if (a.count) {
        w = 1.f / (float)*a.count;
      } else {
        int n = 0;
        for (int i = 0; i < THREADS / 32; ++i) n += s_count[i];
        w = 1.f / (float)n;
      }
      const float total = s_total[g];
      if (warp == 0) {
        float x = 0.f;
        for (int j = lane; j < k; j += 32) {
          const float2 e = s_x[g][j];
          if (s_id[g][j] >= 0 && s_q[g][j] != 0.f) x = fmaf(s_q[g][j], ((ref - e.y) - e.x) + log_s, x);
        }
        x = warp_sum(x);
        if (lane == 0) {
          const float l = s_entropy[g] + x * LN2;
          if (a.row_loss) a.row_loss[t] = l;
          a.weighted[t] = w * l;
        }
        if (GRAD) {
          // what the entries' places are to hold: (p - q / Q) all.s.  With p = 2^x: (2^x - 1) + (1 - q / Q) keeps its
          // digits where p is next to 1, the difference itself where p and q are small (formed through 1, it was off by 6e-8 of
          // the row: more than entries of 1e-7 have).  An id given twice: its first entry stands for all.
          for (int j = lane; j < k; j += 32) {
            const int id = s_id[g][j];
            const float2 e = s_x[g][j];
            float v = 0.f;
            if (id >= 0 && total != 0.f && !(j > 0 && s_id[g][j - 1] == id)) {
              float q = 0.f;
              for (int i = j; i < k && s_id[g][i] == id; ++i) q += s_q[g][i];
              const float u = (e.y - ref) + e.x, x = u - log_s;
              if (x < -1.f) v = fmaf(-q / total, all.s, exp2f(u));
              else v = (expm1f(x * LN2) + (total - q) / total) * all.s;
            }
            s_v[g][j] = v;
          }
          __syncwarp();
          // These carry most of the gradient, and rounded to bf16 they would be off by up to 2^-8.  So the row's factor
          // is moved by as much, to where they round best: a lane tries the factor that makes one of them
          // exact (the largest of its share; the last lane leaves it), the least sum of squares is taken.
          // (relative errors at 8192 x 2048 x 32768 against 64 bits, 1.7e-3 of them the results' own rounding: dE 2.9e-3
          // without, 2.4e-3 with; dX 2.4e-3 and 1.7e-3)
          float ratio = 1.f;
          if (lane < 31) {
            float top = 0.f;
            for (int j = lane; j < k; j += 31) if (fabsf(s_v[g][j]) > fabsf(top)) top = s_v[g][j];
            const float r = __bfloat162float(__float2bfloat16_rn(top));
            if (r != 0.f) ratio = top / r;
          }
          const float inv = 1.f / ratio;
          float err = 0.f;
          for (int j = 0; j < k; ++j) {
            const float v = s_v[g][j], e = fmaf(-__bfloat162float(__float2bfloat16_rn(v * inv)), ratio, v);
            err = fmaf(e, e, err);
          }
          if (!(err < INFINITY)) err = INFINITY;
          float best = err;
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) best = fminf(best, __shfl_xor_sync(0xffffffffu, best, o));
          const unsigned who = __ballot_sync(0xffffffffu, err == best);
          const int from = best < INFINITY ? __ffs(who) - 1 : 31;
          const float use = __shfl_sync(0xffffffffu, ratio, from), use_inv = __shfl_sync(0xffffffffu, inv, from);
          if (lane == 0) {
            const float f = w * a.tg.inv_temp * total * exp2f(-log_s) * use;
            s_f[g] = f; s_inv[g] = use_inv;
            a.factor[row] = f;
          }
        }
      }
      if (GRAD) {
        sync();
        const float f = s_f[g], inv = s_inv[g];
        if (fx)
#pragma unroll 4
          for (int i = tid; i < n8; i += N) {
            const uint4 xv = i == tid ? x0 : xr[i];
            float v[8];
            unpack8(xv, v);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] *= f;
            fx[i] = pack8(v);
          }
        if (!plain) {                               // (seldom) powers that are relative to something else
          for (int i = tid; i < a.n_pieces; i += N) {
            const float2 v = st[i];
            if (v.x != ref && v.y != 0.f) scale_piece(ur + (int64_t)i * PIECE, ldexpf(1.f, (int)(v.x - ref)));
          }
          sync();
        }
        for (int j = tid; j < k; j += N) {          // those stand: overwrite the entries' places
          const int id = s_id[g][j];
          if (id >= 0 && total != 0.f && !(j > 0 && s_id[g][j - 1] == id)) ur[id] = __float2bfloat16_rn(s_v[g][j] * inv);
        }
      }
    }
  }
  // the last block adds up the losses, in the same order whichever block that is
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    s_last = atomicAdd(a.done, 1u) == a.blocks - 1u;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  float s = 0.f;
#pragma unroll 4
  for (int i = threadIdx.x; i < a.T; i += THREADS) s += __ldcg(a.weighted + i);
  s = warp_sum(s);
  if (lane == 0) s_sum[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.f;
    for (int i = 0; i < THREADS / 32; ++i) s += s_sum[i];
    *a.loss = s;
  }
}

// out bf16 [rows, 4 n4] = sum of `splits` fp32 partial products times the row's factor.  A block takes 32
// places of 4 values; each of its 8 warps adds an eighth of the partial products in index order, and the 8 sums are
// added in order (one thread for all of them: 41 us for 148 products of [120, 128], a chain of loads).
__global__ void __launch_bounds__(256)
join_partials_kernel(const float* part, int splits, int64_t stride, const float* row_scale, bf16* out, int64_t ldo, int rows, int n4) {
  __shared__ float4 s_sum[8][32];
  pdl_wait(); pdl_trigger();
  const int lane = threadIdx.x & 31, g = threadIdx.x >> 5;
  const int64_t i = blockIdx.x * (int64_t)32 + lane;
  const bool on = i < (int64_t)rows * n4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (on) {
    const int q1 = (g + 1) * splits / 8;
#pragma unroll 4
    for (int q = g * splits / 8; q < q1; ++q) {
      const float4 x = *reinterpret_cast<const float4*>(part + q * stride + i * 4);
      s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
    }
  }
  s_sum[g][lane] = s;
  __syncthreads();
  if (g || !on) return;
#pragma unroll
  for (int w = 1; w < 8; ++w) {
    const float4 x = s_sum[w][lane];
    s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
  }
  const int64_t r = i / n4;
  const float f = row_scale ? row_scale[r] : 1.f;
  __nv_bfloat162 a = __floats2bfloat162_rn(f * s.x, f * s.y), b = __floats2bfloat162_rn(f * s.z, f * s.w);
  *reinterpret_cast<uint2*>(out + r * ldo + (i - r * n4) * 4) =
      make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
}

// ---- host ---------------------------------------------------------------------------------------
// A chunk by default: 6144 rows (8192 are worked as two of 4096), at most 1 GiB of powers, but no fewer than 256 rows (2 GiB
// for 2^22 ids).  The gradient
// products lose efficiency below 4096 rows: 8192 x 2048 x 131072 takes 13.7 ms in chunks of 1024, 11.4 of
// 2048, 10.5 of 4096 and of 8192.
// (A few more than 6144 rows are two chunks of half as many: 3 % of 6400 x 2048 x 32768, 1.67 ms in one chunk and 1.72, and 2 %
// of 8191 rows; 6144 take 1.60 in one, 1.67 in two.)
constexpr int64_t USUAL_ROWS = 6144, U_BYTES = 1ll << 30;
constexpr int SMS = 148;                      // work is split for a B200 (also where sizes are asked without a device)

int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// Slices of the reductions of dX [rows, d] over V and dE [V, d] over the rows, which one launch works, from a
// model of its time: units of (k + overhead), 6 ns for each k (an SM pair's 256 x 256 tile; one SM's 128 x 128
// tile takes the same), shared out evenly or as long as the longest unit; then for a split product its
// partial sums, read at 3.3 TB/s by a launch of its own (3 us).  Slices are at least 1024 long (at 512 the join of 24 rows and
// of 1001 costs more than it saves: 66 us against 62, 56 against 52).
void choose_splits(int64_t rows, int64_t d, int64_t V, int want, bool split_e, int* sx, int* se) {
  GemmArgs gx, ge;
  gx.M = (int)rows; gx.N = (int)d; ge.M = (int)V; ge.N = (int)d;
  const bool pairs = want == 3 ? gemm_tc_pairs_two(gx, &ge) : gemm_tc_pairs_two(want & 1 ? gx : ge, nullptr);
  const int64_t tile = pairs ? 256 : 128, units = pairs ? SMS / 2 : SMS;
  const double overhead = pairs ? 330. : 190.;
  const int64_t tx = (want & 1) ? ((rows + tile - 1) / tile) * ((d + tile - 1) / tile) : 0;
  const int64_t te = (want & 2) ? ((V + tile - 1) / tile) * ((d + tile - 1) / tile) : 0;
  auto ns = [&](int a, int b) {
    const double ux = (double)V / a + overhead, ue = (double)rows / b + overhead;
    const double work = (tx * a * ux + te * b * ue) / units;
    const double longest = std::max(tx ? ux : 0., te ? ue : 0.);
    return 6. * std::max(work, longest) + (a > 1 ? 3000. + a * 4. * rows * d / 3300. : 0.) + (b > 1 ? 3000. + b * 4. * V * d / 3300. : 0.);
  };
  *sx = *se = 1;
  double best = ns(1, 1);
  const int most = (int)std::max<int64_t>(32, units / std::max<int64_t>(tx, 1));     // (a single tile's reduction goes to all SMs)
  for (int s = 2; tx && s <= most && s <= V / 1024; ++s)
    if (const double t = ns(s, 1); t < 0.95 * best) { best = t; *sx = s; }
  for (int s = 2; te && split_e && s <= 32 && s <= rows / 1024; ++s)
    if (const double t = ns(*sx, s); t < 0.95 * best) { best = t; *se = s; }
}

struct Plan {
  // usual: rows of a chunk by default.  They decide the warps to a row, and so the order of a row's and of the loss's sums:
  // loss, row losses and lse do not depend on chunk_rows.  (The gradients do, by the order of their sums: dE is added
  // up over chunks, and the slices of dX go by the chunk's rows and by whether dE is wanted too.)
  int64_t ldu, n_pieces, chunk, usual;
  int chunks, sx, se;                          // split-K factors of dX and dE
  int64_t ld_off;
  size_t off_weighted, off_factor, off_stats, off_x, off_ids, off_z, off_before, off_u, off_fx, off_acc, off_part_x, off_part_e, bytes;
};
Plan make_plan(int T, int d, int V, int want, int chunk_rows, int k) {
  Plan p;
  p.ldu = round_up(V, PIECE);
  p.n_pieces = p.ldu / PIECE;
  const int64_t row_bytes = want ? p.ldu * 2 : p.n_pieces * 8;     // (without gradients only the pieces' statistics)
  T = std::max(T, 1);
  p.usual = std::max<int64_t>(256, std::min<int64_t>(USUAL_ROWS, U_BYTES / row_bytes / 256 * 256));
  int64_t c = chunk_rows > 0 ? round_up(chunk_rows, 256) : p.usual;
  p.usual = std::min<int64_t>(p.usual, T);
  p.chunks = (int)std::max<int64_t>(1, (T + c - 1) / c);
  p.chunk = p.chunks == 1 ? T : round_up((T + p.chunks - 1) / p.chunks, 256);
  choose_splits(p.chunk, d, V, want, p.chunks == 1, &p.sx, &p.se);
  size_t off = 256;                            // the row count, the rows finished
  auto take = [&off](int64_t bytes) { const size_t at = off; off += (size_t)round_up(bytes, 256); return at; };
  p.off_weighted = take(4ll * T);
  p.off_factor = take(4ll * p.chunk);
  p.off_stats = take(8ll * p.chunk * p.n_pieces);
  p.ld_off = round_up(p.n_pieces + 1, 4);
  p.off_x = take(8ll * p.chunk * k);
  p.off_ids = take(k > 1 ? 4ll * p.chunk * k : 0);
  p.off_z = take(k > 1 ? 4ll * p.chunk * k : 0);
  p.off_before = take(k > 1 ? p.chunk * p.ld_off : 0);
  p.off_u = take(want ? p.chunk * row_bytes : 0);
  p.off_fx = take((want & 2) ? 2ll * p.chunk * d : 0);
  p.off_acc = take((want & 2) && p.chunks > 1 ? 4ll * V * d : 0);
  p.off_part_x = take(p.sx > 1 ? 4ll * p.sx * p.chunk * d : 0);
  p.off_part_e = take(p.se > 1 ? 4ll * p.se * V * d : 0);
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

// warps to a row: one where the rows fill the machine or have little to go through (64 pieces are two a lane)
int warps_for(int64_t rows, int64_t n_pieces) {
  const int64_t share = n_pieces / 64;
  if (rows >= 16 * SMS || share < 4) return 1;
  return rows >= 2 * SMS || share < 16 ? 4 : 16;
}
template <bool GRAD>
cudaError_t launch_rows(const RowArgs& r, int64_t rows, int warps, cudaStream_t st) {
  if (warps == 1) return ppu_launch_dependent(head_rows_kernel<GRAD, 1>, (unsigned)((rows + 3) / 4), 128, 0, st, r, (int)rows);
  if (warps == 4) return ppu_launch_dependent(head_rows_kernel<GRAD, 4>, (unsigned)rows, 128, 0, st, r, (int)rows);
  return ppu_launch_dependent(head_rows_kernel<GRAD, 16>, (unsigned)rows, 512, 0, st, r, (int)rows);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// a split product's epilogue: fp32 partial sums, which join() adds up after the launch
void split_product(GemmArgs& g, int splits, float* part) {
  g.epilogue = EPI_STORE_F32; g.C = part; g.ldc = g.N; g.splits = splits; g.split_stride = (int64_t)g.M * g.N;
}
cudaError_t join(const GemmArgs& g, void* out, int64_t ldo, cudaStream_t st) {
  const int64_t n = (int64_t)g.M * (g.N / 4);
  return ppu_launch_dependent(join_partials_kernel, (unsigned)((n + 31) / 32), 256, 0, st, (const float*)g.C, g.splits, g.split_stride, g.row_scale,
                              (bf16*)out, ldo, g.M, g.N / 4);
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
  const int k = c.tg.k;
  const Plan p = make_plan(c.T, c.d, c.V, want, c.chunk_rows, k);
  if (c.ws_bytes < p.bytes) return ppu_fail(PPU_ENOMEM, "workspace has %zu bytes, %zu needed", c.ws_bytes, p.bytes);

  uint8_t* ws = (uint8_t*)c.ws;
  int* count = (int*)ws;
  unsigned* done = (unsigned*)ws + 1;
  float* factor = (float*)(ws + p.off_factor);
  float2* stats = (float2*)(ws + p.off_stats);
  bf16* u = want ? (bf16*)(ws + p.off_u) : nullptr;
  bf16* fx = c.dE ? (bf16*)(ws + p.off_fx) : nullptr;
  float* acc = (float*)(ws + p.off_acc);
  float *part_x = (float*)(ws + p.off_part_x), *part_e = (float*)(ws + p.off_part_e);

  if (c.T == 0) {                              // a mean over nothing: no loss, no gradient
    CUDA_OK(cudaMemsetAsync(c.loss, 0, 4, c.st));
    if (c.dE) CUDA_OK(cudaMemset2DAsync(c.dE, (size_t)c.ldde * 2, 0, (size_t)c.d * 2, (size_t)c.V, c.st));
    return PPU_OK;
  }
  // the rows that count, for a mean: up to 2^10 rows by every block of the row kernel for itself (a launch
  // costs more; its entries have to be those of all rows), up to 2^14 by one block
  const bool by_rows = c.T <= (1 << 10) && (k == 1 || p.chunks == 1);
  if (!c.weight && c.T > (1 << 14)) {
    CUDA_OK(cudaMemsetAsync(count, 0, 4, c.st));
    CUDA_OK(ppu_launch_dependent(count_rows_kernel, (c.T + 255) / 256, 256, 0, c.st, c.tg, c.T, c.V, count));
  } else if (!c.weight && !by_rows) {
    CUDA_OK(ppu_launch_dependent(count_rows_block_kernel, 1, 1024, 0, c.st, c.tg, c.T, c.V, count));
  }
  RowArgs r;
  r.tg = c.tg; r.u = u; r.ldu = p.ldu; r.ld_pieces = p.n_pieces; r.n_pieces = (int)p.n_pieces; r.stats = stats;
  r.X = (const bf16*)c.X; r.ldx = c.ldx; r.d = c.d; r.V = c.V; r.T = c.T;
  r.scale2 = LOG2E / c.temp; r.weight = c.weight; r.count = by_rows ? nullptr : count;
  r.row_loss = c.row_loss; r.lse = c.lse; r.weighted = (float*)(ws + p.off_weighted); r.factor = factor; r.fx = fx;
  r.done = done; r.loss = c.loss; r.flags = c.flags;
  float2* ex = (float2*)(ws + p.off_x);
  int32_t* sorted_ids = (int32_t*)(ws + p.off_ids);
  float* sorted_z = (float*)(ws + p.off_z);
  uint8_t* before = ws + p.off_before;
  r.x = ex; r.sorted = k > 1;
  if (k > 1) { r.tg.ids = sorted_ids; r.tg.ld_ids = k; r.tg.z = sorted_z; r.tg.ld_z = k; }
  const bf16* E = (const bf16*)c.E;
  const int warps = warps_for(p.usual, p.n_pieces);
  const int64_t per_block = warps == 1 ? 4 : 1;
  r.blocks = 0;
  for (int64_t c0 = 0; c0 < c.T; c0 += p.chunk) r.blocks += (unsigned)((std::min<int64_t>(p.chunk, c.T - c0) + per_block - 1) / per_block);

  GemmArgs g0;
  g0.C2 = nullptr; g0.aux = nullptr; g0.ldaux = 0; g0.flags = c.flags; g0.transient = true;
  for (int64_t c0 = 0; c0 < c.T; c0 += p.chunk) {
    const int64_t rows = std::min<int64_t>(p.chunk, c.T - c0);
    if (k > 1)
      CUDA_OK(ppu_launch_dependent(sort_entries_kernel, (unsigned)((rows + 3) / 4), 128, 0, c.st, c.tg, c0, (int)rows, c.V, (int)p.n_pieces, sorted_ids,
                                   sorted_z, before, p.ld_off, c.flags));
    {
      GemmArgs g = g0;
      g.A = r.X + c0 * c.ldx; g.lda = c.ldx; g.a_kmajor = 1;
      g.B = E; g.ldb = c.lde; g.b_kmajor = 1;
      g.M = (int)rows; g.N = c.V; g.K = c.d; g.epilogue = EPI_PIECES; g.C = u; g.ldc = p.ldu;
      if (c0 == 0) g.zero_word = done;
      if (k > 1) g.entries = {sorted_ids, k, k, before, p.ld_off, ex};
      else g.entries = {c.tg.ids + c0 * c.tg.ld_ids, c.tg.ld_ids, 1, nullptr, 0, ex};
      g.piece_scale = r.scale2; g.piece_stats = stats; g.ld_pieces = p.n_pieces;
      GEMM_OK(launch_gemm_tc_pieces(g, c.st));
    }
    r.row0 = c0;
    CUDA_OK(want ? launch_rows<true>(r, rows, warps, c.st) : launch_rows<false>(r, rows, warps, c.st));
    // both gradient products in one launch
    GemmArgs gx = g0, ge = g0;
    bf16* dX = c.dX ? (bf16*)c.dX + c0 * c.lddx : nullptr;
    if (c.dX) {
      gx.A = u; gx.lda = p.ldu; gx.a_kmajor = 1; gx.B = E; gx.ldb = c.lde; gx.b_kmajor = 0; gx.row_scale = factor;
      gx.M = (int)rows; gx.N = c.d; gx.K = c.V; gx.epilogue = EPI_OUT_BF16; gx.C = dX; gx.ldc = c.lddx;
      if (p.sx > 1) split_product(gx, p.sx, part_x);
    }
    if (c.dE) {
      const bool first = c0 == 0, last = c0 + p.chunk >= c.T;
      ge.A = u; ge.lda = p.ldu; ge.a_kmajor = 0; ge.B = fx; ge.ldb = c.d; ge.b_kmajor = 0;
      ge.M = c.V; ge.N = c.d; ge.K = (int)rows; ge.epilogue = EPI_OUT_BF16; ge.C = c.dE; ge.ldc = c.ldde;
      if (p.se > 1) split_product(ge, p.se, part_e);
      if (!first) { ge.aux = acc; ge.ldaux = c.d; }
      if (!last) { ge.epilogue = first ? EPI_STORE_F32 : EPI_RESID_F32; ge.C = acc; ge.ldc = c.d; }
    }
    if (want) GEMM_OK(launch_gemm_tc_two(c.dX ? gx : ge, want == 3 ? &ge : nullptr, c.st));
    if (c.dX && p.sx > 1) CUDA_OK(join(gx, dX, c.lddx, c.st));
    if (c.dE && p.se > 1) CUDA_OK(join(ge, c.dE, c.ldde, c.st));
  }
  CUDA_OK(cudaGetLastError());
  return PPU_OK;
}

}  // namespace

extern "C" int ppu_head_query_bytes(int T, int d, int V, int grads, int chunk_rows, int k, size_t* bytes) {
  if (!bytes) return ppu_fail(PPU_EINVAL, "bytes is null");
  if (grads < 0 || grads > 3) return ppu_fail(PPU_EINVAL, "grads is a sum of 1 (dX) and 2 (dE)");
  const int rc = check_sizes(T, d, V, chunk_rows);
  if (rc) return rc;
  if (k < 1 || k > PPU_MAX_TEACHER_ENTRIES)
    return ppu_fail(PPU_ESHAPE, "k must lie in 1..%d (got %d)", PPU_MAX_TEACHER_ENTRIES, k);
  *bytes = make_plan(T, d, V, grads, chunk_rows, k).bytes;
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
  if (!(temperature >= 1e-4f) || !(temperature <= 1e4f)) return ppu_fail(PPU_EINVAL, "temperature must lie in 1e-4..1e4");
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
