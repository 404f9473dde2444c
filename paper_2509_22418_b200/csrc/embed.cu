// Embedding lookup with a scale, and the table's gradient from tokens sorted by id.
//
//   out[t] = scale E[id_t]        dE[v] = add[v] + scale sum over t with id_t = v of dout[t]
//
// Negative ids are absent (a row of zeros, no gradient); ids >= V too, and are reported.  HBM bounds both: the rows
// read and written once.
//
// The gradient has no atomics.  Token ids are sorted (stable, so the tokens of an id stay in order), the sorted
// list is cut into pieces of `piece` tokens, and a group of lanes sums the rows of each id of its piece for its own
// columns in registers.  An id that lies within one piece is finished there; one that crosses pieces leaves a
// sum for each of them, which a further kernel adds up in order.  A frequent id (padding, or a word that is a tenth of a text)
// is so shared out over many groups, but for its pieces' sums, which one block for 256 columns adds up (16384 tokens x 256 of one id 81 us, of mixed
// ids 33; 2^20 x 256 595 and 283, of fp32 gradients).  All rows are filled first (zeros, or `add`; in the place of `add` none is), by the blocks that would otherwise idle
// beside the sort, which for up to SORT_TOKENS tokens is the work of one block; those with tokens are then written again.
#include <algorithm>
#include "../../include/ppu.h"
#include "common.cuh"

int ppu_fail(int code, const char* fmt, ...);

namespace {

constexpr int MAX_D = 16384, MAX_T = 1 << 20, MAX_V = 1 << 22;
constexpr int SORT_THREADS = 1024, SORT_TOKENS = 8192;       // one block, 8 tokens a thread (16384 so take 43 us, in tiles 32)
constexpr int TILE = 256, TILE_WARPS = 8;                    // longer lists: tokens of a warp, warps of a block
constexpr int MAX_DIGITS = 256;
constexpr int SMS = 148;                                     // work is split for a B200

struct F8 { float f[8]; };
// eight values as they were read: they are converted when all of a thread's loads have been issued (a conversion waits for its load)
template <typename T> struct Raw8;
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
  __device__ __forceinline__ F8 get() const { return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}}; }
};
template <> struct Raw8<bf16> {
  uint4 u;
  __device__ __forceinline__ void load(const bf16* p) { u = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ F8 get() const {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&u);
    F8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 x = __bfloat1622float2(h[i]); r.f[2 * i] = x.x; r.f[2 * i + 1] = x.y; }
    return r;
  }
};
template <typename T> __device__ __forceinline__ F8 load8(const T* p) { Raw8<T> r; r.load(p); return r.get(); }
__device__ __forceinline__ void store8(float* p, const F8& v) {
  *reinterpret_cast<float4*>(p) = make_float4(v.f[0], v.f[1], v.f[2], v.f[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v.f[4], v.f[5], v.f[6], v.f[7]);
}
__device__ __forceinline__ void store8(bf16* p, const F8& v) {
  uint4 u;
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&u);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v.f[2 * i], v.f[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = u;
}

// ---- lookup: a thread takes 8 columns of a row at a time -----------------------------------------
template <typename TE, typename TO>
__global__ void __launch_bounds__(256) embed_lookup_kernel(const int32_t* ids, const TE* E, int64_t lde, TO* out, int64_t ldo, float scale, uint32_t n, uint32_t chunks,
                                                           int V, int32_t* flags) {
  pdl_wait(); pdl_trigger();
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    const uint32_t t = i / chunks, c = i - t * chunks;
    const int id = ids[t];
    F8 v = {};
    if (id >= 0 && id < V) {
      v = load8(E + (int64_t)id * lde + 8 * c);
#pragma unroll
      for (int j = 0; j < 8; ++j) v.f[j] *= scale;
    } else if (id >= V && flags && c == 0) {
      atomicExch(flags + PPU_FLAG_TOKEN, 1);
    }
    store8(out + (int64_t)t * ldo + 8 * c, v);
  }
}

// ---- sorting tokens by id ------------------------------------------------------------------------
// Least significant digit first, `bits` bits a pass.  A warp owns consecutive tokens and takes 32 at a time: lanes
// with the same digit find each other by a vote for each bit, so that a token's rank among its warp's tokens of that digit
// needs no atomics and the order is kept.  Absent tokens have the key V, which sorts behind all ids.
__device__ __forceinline__ uint32_t key_of(int id, int V) { return id < 0 || id >= V ? (uint32_t)V : (uint32_t)id; }

// ranks 32 tokens; counter: the warp's own, one for each digit
__device__ __forceinline__ uint32_t warp_rank(uint32_t digit, int bits, bool valid, uint32_t* counter, int lane) {
  uint32_t peers = __ballot_sync(0xffffffffu, valid);
  for (int k = 0; k < bits; ++k) {
    const bool bit = digit >> k & 1;
    const uint32_t v = __ballot_sync(0xffffffffu, bit);
    peers &= bit ? v : ~v;
  }
  uint32_t before = 0;
  const int leader = valid ? __ffs(peers) - 1 : lane;
  if (valid && lane == leader) { before = counter[digit]; counter[digit] = before + __popc(peers); }
  before = __shfl_sync(0xffffffffu, before, leader);
  __syncwarp();
  return before + __popc(peers & ((1u << lane) - 1u));
}

struct Fill { void* dE; int64_t ldde; const void* add; int64_t ldadd; uint32_t rows, chunks; int mode; };   // mode 0: nothing, 1: zeros, 2: copy add; chunks of 16 bytes

// AT_ONCE: 16 bytes in flight of a thread
template <int AT_ONCE, bool COPY> __device__ __forceinline__ void fill_loop(const Fill& f, uint32_t block, uint32_t blocks, int bytes_log2) {
  const uint64_t n = (uint64_t)f.rows * f.chunks, step = (uint64_t)blocks * blockDim.x;
  for (uint64_t i0 = (uint64_t)block * blockDim.x + threadIdx.x; i0 < n; i0 += AT_ONCE * step) {
    uint4 x[AT_ONCE];
    uint64_t v[AT_ONCE];
    uint32_t c[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const uint64_t i = i0 + j * step;
      v[j] = n <= 0xffffffffu ? (uint32_t)i / f.chunks : i / f.chunks;
      c[j] = (uint32_t)(i - v[j] * f.chunks);
      x[j] = make_uint4(0, 0, 0, 0);
      if (COPY && i < n) x[j] = *reinterpret_cast<const uint4*>((const uint8_t*)f.add + ((v[j] * f.ldadd) << bytes_log2) + 16 * c[j]);
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j)
      if (i0 + j * step < n) *reinterpret_cast<uint4*>((uint8_t*)f.dE + ((v[j] * f.ldde) << bytes_log2) + 16 * c[j]) = x[j];
  }
}
// (a copy of 32003 x 768 in fp32, with sums of 4099 tokens: 43.6 us with four in flight, 50 with one; zeros, 32768 x 2048 in bf16, 44.5 and 43.5)
__device__ __forceinline__ void fill_rows(const Fill& f, uint32_t block, uint32_t blocks, int bytes_log2) {
  if (f.mode == 2) fill_loop<4, true>(f, block, blocks, bytes_log2);
  else fill_loop<1, false>(f, block, blocks, bytes_log2);
}

// Block 0 sorts, the others fill.  ITEMS: tokens a thread.
template <int ITEMS>
__global__ void __launch_bounds__(SORT_THREADS) embed_sort_fill_kernel(const int32_t* ids, int T, int V, int bits, int passes, uint32_t* keys, uint32_t* order, Fill fill,
                                                                       int bytes_log2, int32_t* flags) {
  pdl_wait(); pdl_trigger();
  if (blockIdx.x > 0) { fill_rows(fill, blockIdx.x - 1, gridDim.x - 1, bytes_log2); return; }
  extern __shared__ uint32_t sh[];
  const int D = 1 << bits, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t* counter = sh;                          // [32 warps][D]
  uint32_t* s_key = sh + 32 * D;                   // [ITEMS * 1024]
  uint32_t* s_order = s_key + ITEMS * SORT_THREADS;
  __shared__ uint32_t s_sum[32];
  uint32_t key[ITEMS], ord[ITEMS];
  bool wrong = false;
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    const int t = (warp * ITEMS + j) * 32 + lane;
    const int id = t < T ? ids[t] : -1;
    wrong |= id >= V;
    key[j] = key_of(id, V); ord[j] = t;
  }
  if (wrong && flags) atomicExch(flags + PPU_FLAG_TOKEN, 1);
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * bits;
    for (int i = threadIdx.x; i < 32 * D; i += SORT_THREADS) counter[i] = 0;
    __syncthreads();
    uint32_t rank[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) rank[j] = warp_rank((key[j] >> shift) & (D - 1), bits, true, counter + warp * D, lane);
    __syncthreads();
    // exclusive sums of the counters in the order (digit, warp): a thread takes a digit's warps (or some of them)
    const int per = 32 * D >= SORT_THREADS ? 32 * D / SORT_THREADS : 1;      // entries a thread (D <= 256: 8 at most)
    uint32_t own[8], total = 0;
    const int first = threadIdx.x * per;
    for (int e = 0; e < 8; ++e) {
      if (e >= per || first + e >= 32 * D) break;
      const int digit = (first + e) >> 5, w = (first + e) & 31;
      own[e] = counter[w * D + digit]; total += own[e];
    }
    uint32_t scan = total;
    for (int o = 1; o < 32; o <<= 1) { const uint32_t x = __shfl_up_sync(0xffffffffu, scan, o); if (lane >= o) scan += x; }
    if (lane == 31) s_sum[warp] = scan;
    __syncthreads();
    if (warp == 0) {
      uint32_t s = s_sum[lane];
      for (int o = 1; o < 32; o <<= 1) { const uint32_t x = __shfl_up_sync(0xffffffffu, s, o); if (lane >= o) s += x; }
      s_sum[lane] = s;
    }
    __syncthreads();
    uint32_t at = scan - total + (warp ? s_sum[warp - 1] : 0);
    for (int e = 0; e < 8; ++e) {
      if (e >= per || first + e >= 32 * D) break;
      const int digit = (first + e) >> 5, w = (first + e) & 31;
      counter[w * D + digit] = at; at += own[e];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const uint32_t to = counter[warp * D + ((key[j] >> shift) & (D - 1))] + rank[j];
      s_key[to] = key[j]; s_order[to] = ord[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int i = (warp * ITEMS + j) * 32 + lane;
      key[j] = s_key[i]; ord[j] = s_order[i];
    }
  }
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    const int i = (warp * ITEMS + j) * 32 + lane;
    if (i < T) { keys[i] = key[j]; order[i] = ord[j]; }      // (what stands in for tokens beyond T sorts behind all of them: key V, in order)
  }
}

// Longer lists, three launches a pass: a warp counts its tile's digits; a block for each digit sums over the tiles;
// tokens go to their places.  ids non-null: the first pass, which reads the ids themselves (and fills the table's rows
// with the blocks behind the first `blocks`).
__device__ __forceinline__ uint32_t tile_key(const int32_t* ids, const uint32_t* keys, int i, int V) { return ids ? key_of(ids[i], V) : keys[i]; }

__global__ void __launch_bounds__(TILE_WARPS * 32) embed_count_kernel(const int32_t* ids, const uint32_t* keys, int T, int V, int shift, int bits, uint32_t* hist, int tiles,
                                                                      int blocks, Fill fill, int bytes_log2, int32_t* flags) {
  pdl_wait(); pdl_trigger();
  if ((int)blockIdx.x >= blocks) { fill_rows(fill, blockIdx.x - blocks, gridDim.x - blocks, bytes_log2); return; }
  __shared__ uint32_t counter[TILE_WARPS][MAX_DIGITS];
  const int D = 1 << bits, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tile = blockIdx.x * TILE_WARPS + warp;
  for (int i = lane; i < D; i += 32) counter[warp][i] = 0;
  __syncwarp();
  bool wrong = false;
  uint32_t key[TILE / 32];
#pragma unroll
  for (int j = 0; j < TILE / 32; ++j) {
    const int i = tile * TILE + j * 32 + lane;
    key[j] = 0;
    if (i < T) { key[j] = tile_key(ids, keys, i, V); if (ids) wrong |= ids[i] >= V; }
  }
#pragma unroll
  for (int j = 0; j < TILE / 32; ++j) warp_rank((key[j] >> shift) & (D - 1), bits, tile * TILE + j * 32 + lane < T, counter[warp], lane);
  if (wrong && flags) atomicExch(flags + PPU_FLAG_TOKEN, 1);
  if (tile < tiles)
    for (int i = lane; i < D; i += 32) hist[(int64_t)i * tiles + tile] = counter[warp][i];
}

__global__ void __launch_bounds__(1024) embed_offsets_kernel(uint32_t* hist, uint32_t* totals, int tiles) {
  pdl_wait(); pdl_trigger();
  __shared__ uint32_t s_sum[32];
  const int warps = blockDim.x / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t* row = hist + (int64_t)blockIdx.x * tiles;
  uint32_t carry = 0;
  for (int base = 0; base < tiles; base += blockDim.x) {
    const int i = base + threadIdx.x;
    const uint32_t x = i < tiles ? row[i] : 0;
    uint32_t s = x;
    for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(0xffffffffu, s, o); if (lane >= o) s += y; }
    if (lane == 31) s_sum[warp] = s;
    __syncthreads();
    uint32_t before = carry, all = 0;
    for (int w = 0; w < warps; ++w) { if (w < warp) before += s_sum[w]; all += s_sum[w]; }
    if (i < tiles) row[i] = before + s - x;
    carry += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) totals[blockIdx.x] = carry;
}

__global__ void __launch_bounds__(TILE_WARPS * 32) embed_place_kernel(const int32_t* ids, const uint32_t* keys, const uint32_t* order, int T, int V, int shift, int bits,
                                                                      const uint32_t* hist, const uint32_t* totals, int tiles, uint32_t* keys_out, uint32_t* order_out) {
  pdl_wait(); pdl_trigger();
  __shared__ uint32_t counter[TILE_WARPS][MAX_DIGITS];
  __shared__ uint32_t s_base[MAX_DIGITS];
  const int D = 1 << bits, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tile = blockIdx.x * TILE_WARPS + warp;
  if (warp == 0) {                                 // exclusive sums of the digits' totals
    uint32_t carry = 0;
    for (int base = 0; base < D; base += 32) {
      const uint32_t x = base + lane < D ? totals[base + lane] : 0;
      uint32_t s = x;
      for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(0xffffffffu, s, o); if (lane >= o) s += y; }
      if (base + lane < D) s_base[base + lane] = carry + s - x;
      carry += __shfl_sync(0xffffffffu, s, 31);
    }
  }
  __syncthreads();
  if (tile >= tiles) return;
  uint32_t key[TILE / 32], ord[TILE / 32];
#pragma unroll
  for (int j = 0; j < TILE / 32; ++j) {
    const int i = tile * TILE + j * 32 + lane;
    key[j] = ord[j] = 0;
    if (i < T) { key[j] = tile_key(ids, keys, i, V); ord[j] = ids ? (uint32_t)i : order[i]; }
  }
  for (int i = lane; i < D; i += 32) counter[warp][i] = s_base[i] + hist[(int64_t)i * tiles + tile];
  __syncwarp();
#pragma unroll
  for (int j = 0; j < TILE / 32; ++j) {
    const bool valid = tile * TILE + j * 32 + lane < T;
    const uint32_t to = warp_rank((key[j] >> shift) & (D - 1), bits, valid, counter[warp], lane);
    if (valid) { keys_out[to] = key[j]; order_out[to] = ord[j]; }
  }
}

// ---- sums over the tokens of each id ---------------------------------------------------------------
struct SumArgs {
  const uint32_t *keys, *order;
  const void* dout; int64_t ldd;
  void* dE; int64_t ldde;
  const void* add; int64_t ldadd;                  // null: nothing is added
  float* head; float* last;                        // [pieces][d]: sums of ids that began in an earlier piece, of ids that go on in the next
  float scale;
  int T, d, V, piece, pieces, slices, lanes;       // lanes: of a group, which covers 8 * lanes columns
};

// dE's row of an id, from its sum and, where there is something to add to, that row's columns `x`
template <typename TG>
__device__ __forceinline__ void finish_row(const SumArgs& a, uint32_t id, int col, F8 v, const F8& x) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v.f[j] = a.add ? fmaf(a.scale, v.f[j], x.f[j]) : a.scale * v.f[j];
  store8((TG*)a.dE + (int64_t)id * a.ldde + col, v);
}
template <typename TG>
__device__ __forceinline__ F8 add_row(const SumArgs& a, uint32_t id, int col) { return load8((const TG*)a.add + (int64_t)id * a.ldadd + col); }

// Rows in flight of a group.  The rows to add to are read with the tokens that end their ids: read when a sum is done, one after another, they made
// 4099 x 768 onto an fp32 table take 40 us.
constexpr int AHEAD = 4;
template <typename TD, typename TG, bool ADD>
__global__ void __launch_bounds__(256) embed_sum_kernel(const SumArgs a) {
  pdl_wait(); pdl_trigger();
  const int group = (blockIdx.x * 256 + threadIdx.x) / a.lanes;
  const int p = group / a.slices, slice = group - p * a.slices;
  const int col = 8 * (slice * a.lanes + (int)threadIdx.x % a.lanes);
  if (p >= a.pieces || col >= a.d) return;
  const int lo = p * a.piece, hi = min(a.T, lo + a.piece);
  const uint32_t V = a.V, NONE = 0xffffffffu;
  bool begun = lo > 0 && a.keys[lo - 1] == a.keys[lo];      // the first id began in an earlier piece
  F8 sum = {};
  const TD* dout = (const TD*)a.dout + col;
  bool ended = true;
  // ids and tokens of the rows AHEAD further are on their way while rows are
  uint32_t id[AHEAD + 1], token[AHEAD];
  auto ids_from = [&](int i, uint32_t (&k)[AHEAD + 1], uint32_t (&o)[AHEAD]) {
#pragma unroll
    for (int j = 0; j <= AHEAD; ++j) k[j] = i + j < min(hi + 1, a.T) ? a.keys[i + j] : NONE;
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) o[j] = i + j < hi ? a.order[i + j] : 0;
  };
  ids_from(lo, id, token);
  for (int i0 = lo; i0 < hi; i0 += AHEAD) {
    Raw8<TD> x[AHEAD];
    Raw8<TG> y[AHEAD];
    uint32_t next_id[AHEAD + 1], next_token[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      if (i0 + j < hi && id[j] < V) {
        x[j].load(dout + (int64_t)token[j] * a.ldd);
        if (ADD && id[j + 1] != id[j]) y[j].load((const TG*)a.add + (int64_t)id[j] * a.ldadd + col);
      }
    ids_from(i0 + AHEAD, next_id, next_token);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (i0 + j >= hi || id[j] >= V) break;        // (nothing but absent tokens follows)
      const F8 v = x[j].get();
#pragma unroll
      for (int e = 0; e < 8; ++e) sum.f[e] += v.f[e];
      ended = id[j + 1] != id[j];
      if (ended) {
        if (begun) store8(a.head + (int64_t)p * a.d + col, sum);
        else finish_row<TG>(a, id[j], col, sum, ADD ? y[j].get() : F8{});
        begun = false; sum = F8{};
      }
    }
#pragma unroll
    for (int j = 0; j <= AHEAD; ++j) id[j] = next_id[j];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) token[j] = next_token[j];
  }
  if (!ended) store8((begun ? a.head : a.last) + (int64_t)p * a.d + col, sum);      // the id goes on in the next piece
}

// One block for each piece in which an id begins that goes on behind it, and 256 columns: its warps add up consecutive shares
// of the pieces' sums, and the shares are added in order.  (A warp for each piece and blocks of 32 or 8 warps for the longest: 3 to 6 us more for up
// to 8192 tokens.)
constexpr int JOIN_WARPS = 8;
template <typename TG>
__global__ void __launch_bounds__(32 * JOIN_WARPS) embed_join_kernel(const SumArgs a) {
  pdl_wait(); pdl_trigger();
  __shared__ float s_sum[JOIN_WARPS][256];
  const int p = blockIdx.x;
  const int64_t lo = (int64_t)p * a.piece, hi = lo + a.piece;
  if (hi >= a.T) return;
  const uint32_t id = a.keys[hi - 1];
  if (id >= (uint32_t)a.V || a.keys[hi] != id || (a.keys[lo] == id && lo > 0 && a.keys[lo - 1] == id)) return;
  int n = 0;                                        // pieces p + 1 .. p + n begin with this id (keys are sorted)
  for (int more = 32 * JOIN_WARPS; more == 32 * JOIN_WARPS; n += more) {
    const int64_t at = hi + (int64_t)(n + (int)threadIdx.x) * a.piece;
    more = __syncthreads_count(at < a.T && a.keys[at] == id);
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = blockIdx.y * 256 + 8 * lane;
  F8 sum = {};
  if (col < a.d) {
    if (warp == 0) sum = load8(a.last + (int64_t)p * a.d + col);
    const float* head = a.head + (int64_t)(p + 1) * a.d + col;
    const int end = (int)((int64_t)n * (warp + 1) / JOIN_WARPS);
#pragma unroll 8
    for (int i = (int)((int64_t)n * warp / JOIN_WARPS); i < end; ++i) {
      const F8 x = load8(head + (int64_t)i * a.d);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum.f[j] += x.f[j];
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) s_sum[warp][8 * lane + j] = sum.f[j];
  __syncthreads();
  if (warp > 0 || col >= a.d) return;
  for (int w = 1; w < JOIN_WARPS; ++w)
#pragma unroll
    for (int j = 0; j < 8; ++j) sum.f[j] += s_sum[w][8 * lane + j];
  finish_row<TG>(a, id, col, sum, a.add ? add_row<TG>(a, id, col) : F8{});
}

// ---- host ------------------------------------------------------------------------------------------
struct Plan { int bits, passes, tiles, piece, pieces, slices, lanes; size_t keys, order, hist, totals, head, last, bytes; };

Plan make_plan(int T, int d, int V) {
  Plan p = {};
  int bits = 1;
  while ((1ll << bits) <= V) ++bits;                // keys 0..V
  p.passes = (bits + 7) / 8;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.tiles = (T + TILE - 1) / TILE;
  p.lanes = 1;
  while (p.lanes < 32 && p.lanes * 8 < d) p.lanes *= 2;
  p.slices = (d + 8 * p.lanes - 1) / (8 * p.lanes);
  // Pieces of 32 tokens; shorter (4 at least) where they would not give an eighth of the machine's threads something to do, longer where they
  // would be more than its threads (each leaves up to two sums).
  const int64_t threads = (int64_t)p.slices * p.lanes;
  p.piece = 32;
  while (p.piece > 4 && T / p.piece * threads < (int64_t)SMS * 256) p.piece /= 2;
  while (T / p.piece * threads > (int64_t)SMS * 2048) p.piece *= 2;
  p.pieces = (T + p.piece - 1) / p.piece;
  size_t at = 0;
  auto take = [&](size_t n) { const size_t was = at; at += (n + 255) / 256 * 256; return was; };
  const int copies = T > SORT_TOKENS ? 2 : 1;
  p.keys = take((size_t)copies * T * 4);
  p.order = take((size_t)copies * T * 4);
  p.hist = take(copies > 1 ? (size_t)(1 << p.bits) * p.tiles * 4 : 0);
  p.totals = take(copies > 1 ? MAX_DIGITS * 4 : 0);
  p.head = take((size_t)p.pieces * d * 4);
  p.last = take((size_t)p.pieces * d * 4);
  p.bytes = at;
  return p;
}

int check_embed(int T, int d, int V) {
  if (T < 0 || d < 1 || V < 1) return ppu_fail(PPU_EINVAL, "negative or empty size");
  if (d % 8 || d > MAX_D) return ppu_fail(PPU_ESHAPE, "d must be a multiple of 8 up to %d (got %d)", MAX_D, d);
  if (T > MAX_T || V > MAX_V) return ppu_fail(PPU_ESHAPE, "at most 2^20 tokens and 2^22 ids");
  return PPU_OK;
}
bool misaligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps) if (reinterpret_cast<uintptr_t>(p) & 15) return true;
  return false;
}
bool bad_type(int t) { return t != PPU_BF16 && t != PPU_F32; }

#define CUDA_OK(call)                                                                    \
  do {                                                                                   \
    cudaError_t e_ = (call);                                                             \
    if (e_ != cudaSuccess)                                                               \
      return ppu_fail(PPU_ECUDA, "%s failed: %s", #call, cudaGetErrorString(e_));        \
  } while (0)

template <typename TE, typename TO>
int lookup(const int32_t* ids, const void* E, int64_t lde, void* out, int64_t ldo, float scale, int T, int d, int V, int32_t* flags, cudaStream_t st) {
  const uint32_t chunks = d / 8, n = (uint32_t)T * chunks;
  const int blocks = (int)std::min<uint32_t>((n + 255) / 256, SMS * 32);
  CUDA_OK(ppu_launch_dependent(embed_lookup_kernel<TE, TO>, blocks, 256, 0, st, ids, (const TE*)E, lde, (TO*)out, ldo, scale, n, chunks, V, flags));
  return PPU_OK;
}

template <typename TD, typename TG>
int sums(const SumArgs& a, cudaStream_t st) {
  const int64_t groups = (int64_t)a.pieces * a.slices;
  const int per_block = 256 / a.lanes;
  const unsigned blocks = (unsigned)((groups + per_block - 1) / per_block);
  if (a.add) CUDA_OK(ppu_launch_dependent(embed_sum_kernel<TD, TG, true>, blocks, 256, 0, st, a));
  else CUDA_OK(ppu_launch_dependent(embed_sum_kernel<TD, TG, false>, blocks, 256, 0, st, a));
  if (a.pieces > 1) CUDA_OK(ppu_launch_dependent(embed_join_kernel<TG>, dim3(a.pieces, (a.d + 255) / 256), 32 * JOIN_WARPS, 0, st, a));
  return PPU_OK;
}

template <int ITEMS>
int sort_fill(const int32_t* ids, int T, int V, const Plan& p, uint8_t* ws, const Fill& f, int fill_blocks, int bytes_log2, int32_t* flags, cudaStream_t st) {
  static PerDeviceFlag attr;
  const int smem = 32 * (1 << p.bits) * 4 + ITEMS * SORT_THREADS * 8;
  if (!ppu_set_smem_once(attr, embed_sort_fill_kernel<ITEMS>, 32 * MAX_DIGITS * 4 + ITEMS * SORT_THREADS * 8)) return ppu_fail(PPU_ECUDA, "shared memory limit not accepted");
  CUDA_OK(ppu_launch_dependent(embed_sort_fill_kernel<ITEMS>, 1 + fill_blocks, SORT_THREADS, smem, st, ids, T, V, p.bits, p.passes, (uint32_t*)(ws + p.keys),
                               (uint32_t*)(ws + p.order), f, bytes_log2, flags));
  return PPU_OK;
}

}  // namespace

extern "C" int ppu_embed_fwd(const int32_t* ids, const void* E, int64_t lde, int e_type, float scale, void* out, int64_t ldo, int out_type, int T, int d, int V,
                             int32_t* flags, void* cuda_stream) {
  const int rc = check_embed(T, d, V);
  if (rc) return rc;
  if (bad_type(e_type) || bad_type(out_type)) return ppu_fail(PPU_EINVAL, "unknown type");
  if (T == 0) return PPU_OK;
  if (!ids || !E || !out) return ppu_fail(PPU_EINVAL, "null operand");
  if (lde < d || ldo < d || lde % 8 || ldo % 8) return ppu_fail(PPU_EINVAL, "row strides must be multiples of 8, at least d");
  if (misaligned({E, out}) || reinterpret_cast<uintptr_t>(ids) & 3) return ppu_fail(PPU_EINVAL, "E and out must be 16-byte aligned");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (e_type == PPU_BF16)
    return out_type == PPU_BF16 ? lookup<bf16, bf16>(ids, E, lde, out, ldo, scale, T, d, V, flags, st) : lookup<bf16, float>(ids, E, lde, out, ldo, scale, T, d, V, flags, st);
  return out_type == PPU_BF16 ? lookup<float, bf16>(ids, E, lde, out, ldo, scale, T, d, V, flags, st) : lookup<float, float>(ids, E, lde, out, ldo, scale, T, d, V, flags, st);
}

extern "C" int ppu_embed_query_bytes(int T, int d, int V, size_t* bytes) {
  if (!bytes) return ppu_fail(PPU_EINVAL, "bytes is null");
  const int rc = check_embed(T, d, V);
  if (rc) return rc;
  *bytes = T ? make_plan(T, d, V).bytes : 0;
  return PPU_OK;
}

extern "C" int ppu_embed_bwd(const int32_t* ids, const void* dout, int64_t ldd, int dout_type, float scale, const void* add, int64_t ldadd, void* dE, int64_t ldde,
                             int grad_type, int T, int d, int V, void* workspace, size_t workspace_bytes, int32_t* flags, void* cuda_stream) {
  const int rc = check_embed(T, d, V);
  if (rc) return rc;
  if (bad_type(dout_type) || bad_type(grad_type)) return ppu_fail(PPU_EINVAL, "unknown type");
  if (!dE || (T && (!ids || !dout || !workspace))) return ppu_fail(PPU_EINVAL, "null operand");
  if ((T && (ldd < d || ldd % 8)) || ldde < d || ldde % 8 || (add && (ldadd < d || ldadd % 8))) return ppu_fail(PPU_EINVAL, "row strides must be multiples of 8, at least d");
  if (misaligned({dout, add, dE}) || reinterpret_cast<uintptr_t>(ids) & 3) return ppu_fail(PPU_EINVAL, "dout, add and dE must be 16-byte aligned");
  if (add == dE && add && ldadd != ldde) return ppu_fail(PPU_EINVAL, "dE in the place of add needs its row stride");
  if (reinterpret_cast<uintptr_t>(workspace) & 255) return ppu_fail(PPU_EINVAL, "workspace must be 256-byte aligned");
  const Plan p = make_plan(T, d, V);
  if (T && workspace_bytes < p.bytes) return ppu_fail(PPU_ENOMEM, "workspace has %zu bytes, %zu needed", workspace_bytes, p.bytes);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  uint8_t* ws = (uint8_t*)workspace;
  const int log2 = grad_type == PPU_BF16 ? 1 : 2;
  Fill f = {dE, ldde, add, ldadd, (uint32_t)V, (uint32_t)((d << log2) / 16), add == dE ? 0 : add ? 2 : 1};
  // (one block an SM beside the sorting one)
  const int64_t pieces16 = (int64_t)f.rows * f.chunks;
  const int fill_blocks = f.mode == 0 ? 0 : (int)std::min<int64_t>(SMS - 1, (pieces16 + SORT_THREADS - 1) / SORT_THREADS);
  uint32_t *keys = (uint32_t*)(ws + p.keys), *order = (uint32_t*)(ws + p.order);
  if (T <= SORT_TOKENS) {
    int rc2 = PPU_OK;
    if (T <= 1024) rc2 = sort_fill<1>(ids, T, V, p, ws, f, fill_blocks, log2, flags, st);
    else if (T <= 4096) rc2 = sort_fill<4>(ids, T, V, p, ws, f, fill_blocks, log2, flags, st);
    else rc2 = sort_fill<8>(ids, T, V, p, ws, f, fill_blocks, log2, flags, st);
    if (rc2) return rc2;
  } else {
    uint32_t *hist = (uint32_t*)(ws + p.hist), *totals = (uint32_t*)(ws + p.totals);
    uint32_t *k_in = keys, *o_in = order, *k_out = keys + T, *o_out = order + T;
    const int blocks = (p.tiles + TILE_WARPS - 1) / TILE_WARPS;
    const int more = f.mode == 0 ? 0 : (int)std::min<int64_t>(SMS * 8, (pieces16 + 255) / 256);
    for (int pass = 0; pass < p.passes; ++pass) {
      const int32_t* from = pass == 0 ? ids : nullptr;
      const int shift = pass * p.bits;
      CUDA_OK(ppu_launch_dependent(embed_count_kernel, blocks + (pass == 0 ? more : 0), TILE_WARPS * 32, 0, st, from, k_in, T, V, shift, p.bits, hist, p.tiles, blocks, f,
                                   log2, pass == 0 ? flags : nullptr));
      CUDA_OK(ppu_launch_dependent(embed_offsets_kernel, 1 << p.bits, std::min(1024, (p.tiles + 31) / 32 * 32), 0, st, hist, totals, p.tiles));
      CUDA_OK(ppu_launch_dependent(embed_place_kernel, blocks, TILE_WARPS * 32, 0, st, from, k_in, o_in, T, V, shift, p.bits, hist, totals, p.tiles, k_out, o_out));
      std::swap(k_in, k_out); std::swap(o_in, o_out);
    }
    keys = k_in; order = o_in;
  }
  if (T == 0) return PPU_OK;
  SumArgs a = {};
  a.keys = keys; a.order = order; a.dout = dout; a.ldd = ldd; a.dE = dE; a.ldde = ldde; a.add = add; a.ldadd = ldadd;
  a.head = (float*)(ws + p.head); a.last = (float*)(ws + p.last); a.scale = scale;
  a.T = T; a.d = d; a.V = V; a.piece = p.piece; a.pieces = p.pieces; a.slices = p.slices; a.lanes = p.lanes;
  if (dout_type == PPU_BF16) return grad_type == PPU_BF16 ? sums<bf16, bf16>(a, st) : sums<bf16, float>(a, st);
  return grad_type == PPU_BF16 ? sums<float, bf16>(a, st) : sums<float, float>(a, st);
}
