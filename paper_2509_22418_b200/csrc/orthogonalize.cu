// Orthogonalised update of matrices: momentum, then products that bring every singular value to about one
// (a polynomial applied `steps` times, Newton-Schulz), on tcgen05 tensor cores:
//
//   m' = beta m + w G   u = nesterov ? w G + beta m' : m'   (without a momentum: u = G)
//   X = u / (|u|_F + eps);   steps times:  A = X X^T,  P = b A + c A A,  X = a X + P X;   O = scale X
//
// for matrices with more rows than columns A = X^T X and X = a X + X P, so that A and P are of the shorter side.
//
// Numbers.  The products' operands are fp16 (11 bits; bf16 has 8) times powers of two that keep |X| <= 2.8 below the
// largest and 2^-26 above the smallest normal number; sums are fp32.  X itself is carried as that fp16 copy and a second fp16 number, what the
// first leaves of it (22 bits; fp32 on chip), and a X is formed from both: rounding X leaves noise in directions whose singular values are small, and the polynomial multiplies
// those by a = 3.4 a step, noise included.  For sides below DIAG_SIDE P's diagonal is kept in fp32 and multiplies the same fp16 copy of X as the rest of
// P (so that what P annuls it annuls as a whole): it comes to -2.7 where singular values come to one, and half a step of fp16 there is 2^-10 of X.
// Root mean square error of O relative to O's (5 steps, CPU model; the rounding of O to bf16 is 1.66e-3): bf16 operands and X 1e-2 for random matrices, 0.16 to
// 0.35 for those with a few large directions; fp16 operands and X 1.3e-3 and 2e-2 to 4e-2; with X carried so 1.4e-3 (sides of 768), 1.7e-3 (256), 2.4e-3 (33)
// and 2e-4 to 7e-4; with P's diagonal too 1.3e-3 (256), 1.5e-3 (130) and 2e-4 to 6e-4.  Sides up to 128 are mostly worked on chip, below.
// Measured, O's rounding included, without P's diagonal and with it, and five steps' time: 24 x 33 x 2100 3.3e-3 and 2.4e-3, 131 and 148 us; 24 x 64 x 2100 2.5e-3 and
// 2.1e-3, 138 and 155; 24 x 255 x 2100 2.4e-3 and 2.1e-3, 268 and 304; 24 x 256 x 2048 2.35e-3 and 2.06e-3, 241 and 271; 40 x 448 x 4096 2.6e-3 and 2.1e-3, 1292 and 1502;
// 12 x 768 x 768 2.2e-3 and 2.0e-3, 206 and 217; 8192 x 2048 2.1e-3 and 1.9e-3, 586 and 609.  So it pays for short sides, whose error would else be the largest of all;
// from 256 on the time is left as it is at an error of 2.8e-3 at most (sides of 350 to 450 of random matrices 12000 long).
//
// A and A A are symmetric: only tiles on and below the diagonal are worked and stored; a block above it is read as its
// mirror image, which tensor cores take in the other order of its elements.  (With the tiles stored on both sides, two bytes at a time down
// the columns, a tile of 128 x 128 took 7 us more.)
//
// What bounds it.  8192 x 2048: 112 GFLOP a step in 104 to 107 us (1060 TFLOP/s).  At the rate of one large product the three parts would take 24 us (72 slices of
// A on 74 pairs), 12 (36 tiles of A A) and 43 (256 tiles of X, in three waves and a half); the rest is the ends of the parts, each of which reads what the last warps
// of the one before it store (5 to 9 us each).  24 x 256 x 2048: 36 to 43 us a step (by where its buffers lie) for 10 GFLOP and 12 bytes a value of X (151 MB, through the L2): 8 of them, 100 MB, in the
// pass over X's tiles, which is most of a step, 2 as A's operand and 2 as that of P X.
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

constexpr int X_EXP = 12, A_EXP = 12;                 // powers of two of X and A as stored
constexpr int SMS = 148, MAX_STEPS = 32, MAX_SIDE = 1 << 16, DIAG_SIDE = 256;
enum Mode { GRAM = 0, POLY = 1, UPDATE = 2 };

// epilogue warps, columns they take at a time (8192 x 2048, a step: 8 and 16 110 us, 8 and 32 112, 16 and 16 115: more of them delay the copies' and products' own threads)
constexpr int EPI = 8, W = 16;
constexpr int KH = 2, BOX = 128 * BK * 2;             // 64-k slabs of a stage; bytes of a box of 64 x 128
constexpr int STAGES = 3, STAGE_BYTES = 2 * KH * BOX; // a CTA's share of a stage: 128 rows of A, 128 of B, 128 k
constexpr int GO = 8;                               // barriers that tell the epilogues that what a unit reads is there
constexpr int BUF_WORDS = 32 * 9;                     // an epilogue warp's
constexpr int SMEM = STAGES * STAGE_BYTES + EPI * BUF_WORDS * 4 + 1024 + 256;
constexpr int BLOCK = 64 + 32 * EPI;
constexpr unsigned long long WAIT_NS = 2000000000ull; // a wait gives up after two seconds

struct KernelP {
  int m, n, side, batch, steps, left;
  int tiles_s, sym;                  // tiles along the shorter side, on and below the diagonal
  int tiles_m, tiles_n, n_fast;      // of X
  int splits;                        // slices of the sum of A
  int units[3];                      // units of a matrix
  int tail_from;                     // tiles of X from here on are worked in two halves of their columns
  int per_step;
  __half *A, *P, *hi[2]; int64_t ld, lds;      // operands, by rows
  __half *lo, *A2;                   // what X's fp16 copy leaves of it, and A once more, as their epilogues read and write them: 32 x 32 blocks (block_at)
  int rows32, cols32, side32;        // blocks along X's sides, along the shorter one
  bf16* O; float scale;
  float gram;                        // A = gram * its accumulator
  float a[MAX_STEPS], b[MAX_STEPS], c[MAX_STEPS], f[MAX_STEPS], d[MAX_STEPS];
  float* diag;                       // [batch][side] P's diagonal, times d; null: it stays in P
  float* partial;                    // slices' sums
  unsigned *done, *arrived;          // [3][batch] warps that have finished; [batch][sym][CTAs][EPI] slices that have left their sums
  unsigned* along; int tiles_l;      // [batch][tiles_l] and of them, for X, those of each tile along the longer side: 2 each, 1 for half a tile
  int* flags;
};

__device__ __forceinline__ uint32_t half2_bits(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 half2_floats(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }

__device__ __forceinline__ unsigned load_acquire(const unsigned* p) {
  unsigned v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ unsigned long long now_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// waits with a limit in time: until a barrier's phase is over, until a counter has come to a value
template <typename F>
__device__ __forceinline__ bool wait_for(volatile int* abort_flag, int* flags, F ready) {
  if (ready()) return true;
  const unsigned long long t0 = now_ns();
  for (uint32_t it = 1;; ++it) {
    if (ready()) return true;
    if ((it & 255u) == 0) {
      if (*abort_flag) return false;
      if (now_ns() - t0 > WAIT_NS) break;
    }
  }
  *abort_flag = 1;
  if (flags) atomicExch(flags + PPU_FLAG_TIMEOUT, 1);
  return false;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t saddr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// (PAIR: the two CTAs of a cluster on one 256 x 256 tile; else a CTA on 128 x 128)
template <bool PAIR> __device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  if constexpr (PAIR)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst), "l"(map), "r"(bar),
                 "r"(x), "r"(y), "r"(z) : "memory");
  else tma_load_3d(dst, map, bar, x, y, z);
}
template <bool PAIR> __device__ __forceinline__ void umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (PAIR) {
    const uint32_t z = 0;
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5, %5, %5, %5, %5}, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(z)
                 : "memory");
  } else {
    umma_bf16(d, a, b, idesc, accumulate);
  }
}
template <bool PAIR> __device__ __forceinline__ void commit(uint32_t bar) {
  if constexpr (PAIR) {
    const uint16_t mask = 3;
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(mask) : "memory");
  } else {
    umma_commit(bar);
  }
}

// ---- units -----------------------------------------------------------------------------------------
// A step's units are all matrices' of A, then of P, then of X; CTAs (or pairs) take every n-th of them, step after step.
// A unit waits for what it reads to be finished: P of the matrix for its A, X for its P, each a counter, A for its X, tile by tile
// along the longer side, over which it sums.
// A unit waits only for units that come before it (and slices of a tile of A for one another), and all CTAs are resident (a cooperative launch) and work in
// order: so there is always one that can go on.  (A tile's slices are consecutive units of different workers, and each leaves its sums before it waits: the first
// unit that has not come so far waits for nothing behind it, and nor does its worker, whose unit before is finished or of a tile all of whose slices have.)  The same waits order what is overwritten: A's tiles are written when X has been begun, and so P of
// the step before is done, P's when A is, X's other buffer when P is.
struct Unit { int mode, b, i, j, split, splits, kb0, kb1, K, bn; };
template <bool PAIR>
__device__ __forceinline__ Unit unit_at(const KernelP& p, int r) {
  constexpr int TILE = PAIR ? 256 : 128;
  Unit w;
  w.mode = GRAM;
  if (r >= p.units[GRAM] * p.batch) { r -= p.units[GRAM] * p.batch; w.mode = POLY; }
  if (w.mode == POLY && r >= p.units[POLY] * p.batch) { r -= p.units[POLY] * p.batch; w.mode = UPDATE; }
  const int per = w.mode == GRAM ? p.units[GRAM] : w.mode == POLY ? p.units[POLY] : p.units[UPDATE];
  w.b = r / per;
  int t = r - w.b * per;
  w.bn = TILE; w.split = 0; w.splits = 1;
  w.K = w.mode == GRAM ? (p.left ? p.n : p.m) : p.side;
  const int k_blocks = (w.K + KH * BK - 1) / (KH * BK);
  w.kb0 = 0; w.kb1 = k_blocks;
  if (w.mode != UPDATE) {
    if (w.mode == GRAM) {
      w.splits = p.splits;
      w.split = t % w.splits; t /= w.splits;
      w.kb0 = (int)((int64_t)w.split * k_blocks / w.splits); w.kb1 = (int)((int64_t)(w.split + 1) * k_blocks / w.splits);
    }
    int i = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    while (i * (i + 1) / 2 > t) --i;
    w.i = i * TILE; w.j = (t - i * (i + 1) / 2) * TILE;
  } else {
    int half = 0;
    if (PAIR && t >= p.tail_from) { const int v = t - p.tail_from; t = p.tail_from + (v >> 1); half = v & 1; w.bn = TILE / 2; }
    w.i = (p.n_fast ? t / p.tiles_n : t % p.tiles_m) * TILE;
    w.j = (p.n_fast ? t % p.tiles_n : t / p.tiles_m) * TILE + half * (TILE / 2);
  }
  return w;
}
// the counter a unit waits for, and the value of it
template <bool PAIR>
__device__ __forceinline__ const unsigned* awaited(const KernelP& p, const Unit& w, int step, unsigned& value) {
  constexpr unsigned EACH = (PAIR ? 2 : 1) * EPI;
  const unsigned before = w.mode == GRAM ? (unsigned)step * p.units[UPDATE] : (unsigned)(step + 1) * p.units[w.mode - 1];
  value = before * EACH;
  return p.done + (w.mode == GRAM ? UPDATE : w.mode - 1) * p.batch + w.b;
}

// ---- 16 columns from n on of row m (one to a lane) ---------------------------------------------------
// What the epilogues alone read and write again lies in blocks: 32 x 32 values in 1024 consecutive places, sixteen columns of row 0, of row 1, ... of row
// 31, then the other sixteen.  A lane takes 32 bytes and the warp 1 KB.
__device__ __forceinline__ int64_t block_at(int b, int rows32, int cols32, int m, int n) {
  return (((int64_t)b * rows32 + m / 32) * cols32 + n / 32) * 1024 + (n & 16) * 32;
}
// P's diagonal for this lane's row (left), or for column n + lane % 16
__device__ __forceinline__ float diagonal(const KernelP& p, const Unit& w, int m0, int n, int lane) {
  const int i = p.left ? m0 + lane : n + (lane & 15);
  return i < p.side ? __ldcg(p.diag + (int64_t)w.b * p.side + i) : 0.f;
}
// A, or P with x of A
template <bool DIAG>
__device__ __forceinline__ void finish_product(const KernelP& p, const Unit& w, int step, int m0, int n, const uint32_t* r, const uint32_t* x, int lane) {
  const int m = m0 + lane;
  uint32_t o[8];
  if (w.mode == GRAM) {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = half2_bits(p.gram * __uint_as_float(r[2 * j]), p.gram * __uint_as_float(r[2 * j + 1]));
    st_v8(p.A2 + block_at(w.b, p.side32, p.side32, m0, n) + 16 * lane, o);
  } else {
    const float b = p.b[step], c = p.c[step];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 v = half2_floats(x[j]);
      float2 y = make_float2(fmaf(c, __uint_as_float(r[2 * j]), b * v.x), fmaf(c, __uint_as_float(r[2 * j + 1]), b * v.y));
      if (DIAG && n - m0 == (lane & 16) && (lane & 15) / 2 == j) {      // the diagonal
        if (m < p.side) p.diag[(int64_t)w.b * p.side + m] = p.d[step] * (lane & 1 ? y.y : y.x);
        (lane & 1 ? y.y : y.x) = 0.f;
      }
      o[j] = half2_bits(y.x, y.y);
    }
  }
  if (m < p.side) st_v8((w.mode == GRAM ? p.A : p.P) + ((int64_t)w.b * p.side + m) * p.lds + n, o);
}
// X, with x: X's two numbers of before.  buf: 32 x 9 words of the warp, through which rows of O that are not whole 16 bytes are stored;
// pd: P's diagonal of this lane's row (left) or of column n + lane % 16
template <bool DIAG>
__device__ __forceinline__ void finish_x(const KernelP& p, const Unit& w, int step, int m0, int n, const uint32_t* r, const uint32_t* x, float pd, uint32_t* buf, int lane) {
  const int m = m0 + lane;
  const float a = p.a[step], f = p.f[step];
  // a X + (P's diagonal) (X in fp16) + f (the rest of P X)
  float y[W];
#pragma unroll
  for (int j = 0; j < W; j += 2) {
    const float2 h = half2_floats(x[j / 2]), l = half2_floats(x[8 + j / 2]);
    float2 ax = make_float2(a * (h.x + l.x), a * (h.y + l.y));
    if constexpr (DIAG) {
      const float d0 = p.left ? pd : __shfl_sync(0xffffffffu, pd, j), d1 = p.left ? pd : __shfl_sync(0xffffffffu, pd, j + 1);
      ax.x = fmaf(d0, h.x, ax.x); ax.y = fmaf(d1, h.y, ax.y);
    }
    y[j] = fmaf(f, __uint_as_float(r[j]), ax.x); y[j + 1] = fmaf(f, __uint_as_float(r[j + 1]), ax.y);
  }
  uint32_t o[8];
  if (step + 1 < p.steps) {
    uint32_t l[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      o[j] = half2_bits(y[2 * j], y[2 * j + 1]);
      const float2 v = half2_floats(o[j]);
      l[j] = half2_bits(y[2 * j] - v.x, y[2 * j + 1] - v.y);
    }
    st_v8(p.lo + block_at(w.b, p.rows32, p.cols32, m0, n) + 16 * lane, l);
    if (m < p.m) st_v8(p.hi[(step + 1) & 1] + ((int64_t)w.b * p.m + m) * p.ld + n, o);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = gemm_tc_detail::pack2_bf16(p.scale * y[2 * j], p.scale * y[2 * j + 1]);
  if (p.n % 8 == 0) {
    if (m >= p.m) return;
    bf16* to = p.O + ((int64_t)w.b * p.m + m) * p.n + n;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (n + 8 * j < p.n) *reinterpret_cast<uint4*>(to + 8 * j) = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
  } else {
    const int col = lane & 15, c = n + col;
#pragma unroll
    for (int j = 0; j < 8; ++j) buf[lane * 9 + j] = o[j];
    __syncwarp();
    if (c < p.n)
      for (int i = lane >> 4; i < 32 && m0 + i < p.m; i += 2)
        reinterpret_cast<unsigned short*>(p.O)[((int64_t)w.b * p.m + m0 + i) * p.n + c] = (unsigned short)(buf[i * 9 + col / 2] >> (16 * (col & 1)));
    __syncwarp();
  }
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                 "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr)
               : "memory");
}

// ---- all steps -----------------------------------------------------------------------------------------
template <bool PAIR, bool DIAG>
__device__ __forceinline__ void ortho_steps(const CUtensorMap* maps, const KernelP& p) {
  constexpr int CTAS = PAIR ? 2 : 1, TILE = 128 * CTAS;
  constexpr int PIECES = 4;                     // of W columns, fetched ahead (203 x 333, a step, when this was chosen: one 19.7 us, two 18.1, four 17.2; 24 x 256 x 2048 on pairs: 45, 42.3, 41.6)
  extern __shared__ uint8_t smem_raw[];
  // (the window starts at the same offset in both CTAs of a pair, so aligned offsets match too)
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint32_t* bufs = reinterpret_cast<uint32_t*>(smem + STAGES * STAGE_BYTES);
  uint64_t* bars = reinterpret_cast<uint64_t*>(bufs + EPI * BUF_WORDS);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 4 + GO);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_rank() : 0;
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (STAGES + s); };
  auto tfull_bar = [&](int a) { return bar0 + 8u * (2 * STAGES + a); };
  auto tempty_bar = [&](int a) { return bar0 + 8u * (2 * STAGES + 2 + a); };
  // (the copying thread is up to five units ahead of the epilogues: the one they work on, the next, finished, and one in each stage lie between)
  auto go_bar = [&](int u) { return bar0 + 8u * (2 * STAGES + 4 + (u & (GO - 1))); };
  auto leaders = [&](uint32_t bar) { return PAIR ? map_to_rank(bar, 0) : bar; };
  auto wait_bar = [&](uint32_t bar, uint32_t parity) { return wait_for(abort_flag, p.flags, [&] { return mbar_try(bar, parity); }); };
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), CTAS * EPI); }
    for (int u = 0; u < GO; ++u) mbar_init(go_bar(u), 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      tmem_alloc(smem_u32(tmem_slot), 2 * TILE);
    }
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) cluster_sync_all();       // the peer's barriers are set up before anything signals them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();

  const int workers = gridDim.x / CTAS, worker = blockIdx.x / CTAS;
  // calls f(step, unit) for this worker's units in order until it returns false
  auto each_unit = [&](auto f) {
    int r = worker;
    for (int step = 0; step < p.steps;) {
      if (r >= p.per_step) { r -= p.per_step; ++step; continue; }
      if (!f(step, unit_at<PAIR>(p, r))) return;
      r += workers;
    }
  };
  // which operand's 128 x 128 blocks from k0 on are read in the order [k][rows]: X in A = X^T X and as the second operand of P X, and
  // blocks of A and P above the diagonal
  auto a_mn = [&](const Unit& w, int k0) { return w.mode == GRAM ? !p.left : (w.mode == POLY || p.left) && k0 / TILE > w.i / TILE; };
  // (a tile on the diagonal of A or A A: both operands are the same)
  auto same = [&](const Unit& w) { return w.mode != UPDATE && w.i == w.j; };
  auto b_mn = [&](const Unit& w, int k0) { return w.mode == GRAM ? !p.left : w.mode == UPDATE && p.left ? true : k0 / TILE > w.j / TILE; };
  if (warp == 0) {
    if (lane == 0) {
      // ---------------- TMA producer (each CTA: 128 rows of A, its half of B's) ----------------
      int s = 0, u = 0; uint32_t ph = 0;
      const unsigned tiles_short = p.left ? p.tiles_m : p.tiles_n;
      each_unit([&](int step, const Unit& w) {
        unsigned value;
        const unsigned* counter = awaited<PAIR>(p, w, step, value);
        // A's products need not wait for all of X: they are over the longer side, whose tiles are finished in that order
        bool all = w.mode != GRAM;
        if (all && !wait_for(abort_flag, p.flags, [&] { return load_acquire(counter) >= value; })) return false;
        if (all) mbar_arrive(go_bar(u));
        asm volatile("fence.proxy.async.global;" ::: "memory");      // (the operands were written by plain stores)
        const CUtensorMap* X = maps + (step & 1);
        const CUtensorMap *mA = w.mode == GRAM ? X : w.mode == POLY ? maps + 2 : p.left ? maps + 3 : X;
        const CUtensorMap *mB = w.mode == GRAM ? X : w.mode == POLY ? maps + 2 : p.left ? X : maps + 3;
        const int a0 = w.i + (int)rank * 128, b_rows = w.bn / CTAS, b0 = w.j + (int)rank * b_rows;
        for (int kb = w.kb0; kb < w.kb1; ++kb) {
          const int k0 = kb * KH * BK, slabs = k0 + BK < w.K ? KH : 1;      // (the second slab may lie past the end of the sum)
          if (!all && (kb == w.kb0 || k0 % TILE == 0)) {
            all = load_acquire(counter) >= value;
            const unsigned *tile = p.along + (int64_t)w.b * p.tiles_l + k0 / TILE, there = 2u * step * tiles_short * CTAS * EPI;
            if (!all && !wait_for(abort_flag, p.flags, [&] { return load_acquire(tile) >= there; })) return false;
            asm volatile("fence.proxy.async.global;" ::: "memory");
          }
          if (!wait_bar(empty_bar(s), ph ^ 1u)) return false;
          const uint32_t a_dst = smem_u32(smem + s * STAGE_BYTES), b_dst = a_dst + KH * BOX;
          const uint32_t fb = leaders(full_bar(s));
          // blocks [rows][k] come in a box for each slab of 64 k, blocks [k][rows] in one for each 64 rows, of 128 k
          const bool amn = a_mn(w, k0), bmn = b_mn(w, k0);
          const int a_boxes = amn ? 2 : slabs, b_boxes = same(w) ? 0 : bmn ? b_rows / 64 : slabs;
          if (rank == 0) mbar_expect_tx(full_bar(s), CTAS * (a_boxes + b_boxes) * BOX);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if (j >= a_boxes) break;
            if (amn) load_box<PAIR>(a_dst + j * BOX, mA, fb, a0 + 64 * j, k0, w.b);
            else load_box<PAIR>(a_dst + j * BOX, mA, fb, k0 + BK * j, a0, w.b);
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if (j >= b_boxes) break;
            if (bmn) load_box<PAIR>(b_dst + j * BOX, mB, fb, b0 + 64 * j, k0, w.b);
            else load_box<PAIR>(b_dst + j * BOX, mB, fb, k0 + BK * j, b0, w.b);
          }
          if (++s == STAGES) { s = 0; ph ^= 1u; }
        }
        if (w.mode == GRAM) mbar_arrive(go_bar(u));
        ++u;
        return true;
      });
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      // ---------------- MMA issuer: D fp32, A and B fp16 ----------------
      int s = 0; uint32_t ph = 0;
      int acc = 0; uint32_t acc_ph = 0;
      each_unit([&](int, const Unit& w) {
        const uint32_t idesc0 = (1u << 4) | ((uint32_t)(w.bn >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
        if (!wait_bar(tempty_bar(acc), acc_ph ^ 1u)) return false;
        tc_fence_after();
        for (int kb = w.kb0; kb < w.kb1; ++kb) {
          if (!wait_bar(full_bar(s), ph)) return false;
          tc_fence_after();
          const uint32_t a_addr = smem_u32(smem + s * STAGE_BYTES), b_addr = same(w) ? a_addr : a_addr + KH * BOX;
          const int k0 = kb * KH * BK, slabs = k0 + BK < w.K ? KH : 1;
          const bool amn = a_mn(w, k0), bmn = b_mn(w, k0);
          const uint32_t idesc = idesc0 | ((amn ? 1u : 0u) << 15) | ((bmn ? 1u : 0u) << 16);
          const uint64_t ad = make_desc(a_addr, amn ? BOX : 16, 1024), bd = make_desc(b_addr, bmn ? BOX : 16, 1024);
          // (steps of the descriptors' addresses, which stay below 2^14: from 16 k to 16 k, from slab to slab)
          const uint32_t a_step = (amn ? 2048 : 32) >> 4, b_step = (bmn ? 2048 : 32) >> 4, a_slab = (amn ? 8192 : BOX) >> 4, b_slab = (bmn ? 8192 : BOX) >> 4;
#pragma unroll
          for (int kh = 0; kh < KH; ++kh) {
            if (kh >= slabs) break;
#pragma unroll
            for (int k = 0; k < BK / UMMA_K; ++k)
              umma<PAIR>(tmem_base + (uint32_t)(acc * TILE), ad + kh * a_slab + k * a_step, bd + kh * b_slab + k * b_step, idesc, (kb > w.kb0 || kh > 0 || k > 0) ? 1u : 0u);
          }
          commit<PAIR>(empty_bar(s));
          if (++s == STAGES) { s = 0; ph ^= 1u; }
        }
        commit<PAIR>(tfull_bar(acc));
        if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
        return true;
      });
    }
  } else {
    // ---------------- epilogue warps: a quarter of a CTA's rows, half of the columns each ----------------
    const int quarter = warp & 3, set = (warp - 2) >> 2, me = warp - 2;
    int acc = 0, u = 0; uint32_t acc_ph = 0;
    uint32_t* buf = bufs + me * BUF_WORDS;
    each_unit([&](int step, const Unit& w) {
      const int m0 = w.i + (int)rank * 128 + quarter * 32;
      const int c0 = set * (w.bn / 2), c1 = min(c0 + w.bn / 2, (w.mode == UPDATE ? p.n : p.side) - w.j);      // columns of the tile
      uint32_t x[PIECES][W];
      float pd[PIECES];
      // what other CTAs have written is read from here on (the copying thread has seen the counter), while the products run
      if (!__all_sync(0xffffffffu, wait_bar(go_bar(u), u / GO & 1))) return false;
      ++u;
      const bool rows = m0 < (w.mode == UPDATE ? p.m : p.side);
      const __half* x_hi = p.hi[step & 1] + ((int64_t)w.b * p.m + min(m0 + lane, p.m - 1)) * p.ld;
      auto fetch_x = [&](int q, int c) {           // (no branches on what is loaded where: values would be moved, and waited for)
        if (c >= c1) return;
        ld_v8(x[q], x_hi + w.j + c);
        ld_v8(x[q] + 8, p.lo + block_at(w.b, p.rows32, p.cols32, m0, w.j + c) + 16 * lane);
        if (DIAG) pd[q] = diagonal(p, w, m0, w.j + c, lane);
      };
      auto fetch_a = [&](int q, int c) {
        if (c < c1) ld_v8(x[q], p.A2 + block_at(w.b, p.side32, p.side32, m0, w.j + c) + 16 * lane);
      };
      if (rows && w.mode == UPDATE) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) fetch_x(q, c0 + q * W);
      }
      if (rows && w.mode == POLY) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) fetch_a(q, c0 + q * W);
      }
      if (!__all_sync(0xffffffffu, wait_bar(tfull_bar(acc), acc_ph))) return false;
      tc_fence_after();
      const uint32_t t_row = tmem_base + (uint32_t)(acc * TILE) + ((uint32_t)(quarter * 32) << 16);
      // A tile of A in slices: each slice leaves its sums of the columns that are others' to finish, laid out as the lanes read them, and adds
      // up those of its own columns in the order of the slices.  (The slices of a tile are consecutive units, so that they are worked at the same time.)
      auto mine = [&](int c) { return w.splits == 1 || (c - c0) / W * w.splits / (w.bn / 2 / W) == w.split; };
      const int tile = w.i / TILE * (w.i / TILE + 1) / 2 + w.j / TILE;
      const int64_t place = ((int64_t)w.b * p.sym + tile) * CTAS + rank;
      const int64_t slice = (int64_t)128 * TILE / 4;      // in float4
      float4* sums = reinterpret_cast<float4*>(p.partial) + place * w.splits * slice + me * (32 * (TILE / 2) / 4) + lane;
      if (w.splits > 1) {
        unsigned* arrived = p.arrived + place * EPI + me;
        bool some = false;
#pragma unroll 1
        for (int c = c0; c < c1; c += W) {
          if (mine(c)) { some = true; continue; }
          uint32_t r[W];
          tmem_ld16(t_row + c, r);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < W / 4; ++j)
            sums[w.split * slice + ((c - c0) / 4 + j) * 32] =
                make_float4(__uint_as_float(r[4 * j]), __uint_as_float(r[4 * j + 1]), __uint_as_float(r[4 * j + 2]), __uint_as_float(r[4 * j + 3]));
        }
        __syncwarp();
        bool ok = true;
        if (lane == 0) {
          asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(arrived) : "memory");
          const unsigned all = (unsigned)(step + 1) * w.splits;
          if (some) ok = wait_for(abort_flag, p.flags, [&] { return load_acquire(arrived) >= all; });
        }
        if (!__all_sync(0xffffffffu, ok)) return false;
      }
      // the tile's pieces, q of every PIECES: fn(q, column); the lanes come together before each, which reads tensor memory
      auto each_piece = [&](auto fn) {
#pragma unroll 1
        for (int from = c0; from < c1; from += PIECES * W) {
#pragma unroll
          for (int q = 0; q < PIECES; ++q)
            if (from + q * W < c1) { __syncwarp(); fn(q, from + q * W); }
        }
      };
      if (!rows) {
      } else if (w.mode == UPDATE) {
        each_piece([&](int q, int c) {
          uint32_t r[W];
          tmem_ld16(t_row + c, r);
          tmem_ld_wait();
          finish_x<DIAG>(p, w, step, m0, w.j + c, r, x[q], pd[q], buf, lane);
          fetch_x(q, c + PIECES * W);
        });
      } else if (w.splits == 1) {
        each_piece([&](int q, int c) {
          uint32_t r[W];
          tmem_ld16(t_row + c, r);
          tmem_ld_wait();
          finish_product<DIAG>(p, w, step, m0, w.j + c, r, x[q], lane);
          if (w.mode == POLY) fetch_a(q, c + PIECES * W);
        });
      } else {
        const int first = w.split == 0;            // what this slice has left of a piece is in flight ahead
        auto fetch_sums = [&](int q, int c) {
          if (c >= c1 || !mine(c)) return;
#pragma unroll
          for (int j = 0; j < W / 4; ++j) {
            const float4 v = __ldcg(sums + first * slice + ((c - c0) / 4 + j) * 32);
            x[q][4 * j] = __float_as_uint(v.x); x[q][4 * j + 1] = __float_as_uint(v.y); x[q][4 * j + 2] = __float_as_uint(v.z); x[q][4 * j + 3] = __float_as_uint(v.w);
          }
        };
#pragma unroll
        for (int q = 0; q < PIECES; ++q) fetch_sums(q, c0 + q * W);
        each_piece([&](int piece, int c) {
          if (mine(c)) {
            uint32_t r[W];
            tmem_ld16(t_row + c, r);
            tmem_ld_wait();
            float all[W];
#pragma unroll
            for (int j = 0; j < W; ++j) all[j] = 0.f;
#pragma unroll 1
            for (int q = 0; q < w.splits; ++q) {
#pragma unroll
              for (int j = 0; j < W / 4; ++j) {
                float4 v = make_float4(__uint_as_float(r[4 * j]), __uint_as_float(r[4 * j + 1]), __uint_as_float(r[4 * j + 2]), __uint_as_float(r[4 * j + 3]));
                if (q == first) v = make_float4(__uint_as_float(x[piece][4 * j]), __uint_as_float(x[piece][4 * j + 1]), __uint_as_float(x[piece][4 * j + 2]), __uint_as_float(x[piece][4 * j + 3]));
                else if (q != w.split) v = __ldcg(sums + q * slice + ((c - c0) / 4 + j) * 32);
                all[4 * j] += v.x; all[4 * j + 1] += v.y; all[4 * j + 2] += v.z; all[4 * j + 3] += v.w;
              }
            }
#pragma unroll
            for (int j = 0; j < W; ++j) r[j] = __float_as_uint(all[j]);
            finish_product<DIAG>(p, w, step, m0, w.j + c, r, x[piece], lane);      // (of x only a tile of P reads)
          }
          fetch_sums(piece, c + PIECES * W);
        });
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (PAIR) asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(leaders(tempty_bar(acc))) : "memory");
        else mbar_arrive(tempty_bar(acc));
      }
      asm volatile("fence.proxy.async.global;" ::: "memory");      // (read by copies of other CTAs)
      __syncwarp();
      if (lane == 0) {
        asm volatile("fence.acq_rel.gpu;" ::: "memory");
        if (w.mode == UPDATE)
          asm volatile("red.relaxed.gpu.global.add.u32 [%0], %1;" ::"l"(p.along + (int64_t)w.b * p.tiles_l + (p.left ? w.j : w.i) / TILE), "r"(w.bn == TILE ? 2 : 1) : "memory");
        asm volatile("red.relaxed.gpu.global.add.u32 [%0], 1;" ::"l"(p.done + w.mode * p.batch + w.b) : "memory");
      }
      if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
      return true;
    });
  }
  // ---------------- common exit ----------------
  __syncwarp();
  if (*abort_flag) {
    for (int i = 0; i < 64; ++i) __nanosleep(2000);      // copies and products in flight
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) cluster_sync_all();       // neither CTA leaves while its peer may still signal it
  if (warp == 1) {
    tc_fence_after();
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    else tmem_dealloc(tmem_base, 2 * TILE);
  }
}

struct Maps { CUtensorMap m[4]; };                 // X (even steps), X (odd steps), A, P
template <bool DIAG> __global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(BLOCK, 1) ortho_pair_kernel(const __grid_constant__ Maps maps, const __grid_constant__ KernelP p) {
  ortho_steps<true, DIAG>(maps.m, p);
}
template <bool DIAG> __global__ void __launch_bounds__(BLOCK, 1) ortho_single_kernel(const __grid_constant__ Maps maps, const __grid_constant__ KernelP p) {
  ortho_steps<false, DIAG>(maps.m, p);
}

// ---- momentum, norm and the first X ----------------------------------------------------------------
struct PrepP {
  const void* G; int64_t ldg, stride_g;
  const float* m; int64_t ldm, stride_m;           // null: no momentum
  float* m_out; int64_t ldm_out, stride_m_out;
  int rows, cols, nesterov, f32;
  float beta, w, eps, scale;
  double* partial;                                 // [batch][blocks]
  __half *hi, *lo; int64_t ld; int rows32, cols32;
  bf16* O;                                         // no steps: scale X
  unsigned* counters; int n_counters;              // set to 0
};

// four columns of a row from column c on; what lies behind the row's end is 0.  VEC: rows are whole fours, aligned
template <int VEC> __device__ __forceinline__ float4 load4(const float* p, int left) {
  if (VEC) return *reinterpret_cast<const float4*>(p);
  return make_float4(p[0], left > 1 ? p[1] : 0.f, left > 2 ? p[2] : 0.f, left > 3 ? p[3] : 0.f);
}
// bf16 as they were read: they are converted when all of a thread's loads have been issued (a conversion waits for its load)
struct Bf4 {
  uint2 u;
  __device__ __forceinline__ operator float4() const {
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x)), b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
    return make_float4(a.x, a.y, b.x, b.y);
  }
};
template <int VEC> __device__ __forceinline__ Bf4 load4(const bf16* p, int left) {
  if (VEC) return {*reinterpret_cast<const uint2*>(p)};
  const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
  const uint32_t x = h[0], y = left > 1 ? h[1] : 0, z = left > 2 ? h[2] : 0, w = left > 3 ? h[3] : 0;
  return {make_uint2(x | y << 16, z | w << 16)};
}
__device__ __forceinline__ void clear(float4& v) { v = make_float4(0.f, 0.f, 0.f, 0.f); }
__device__ __forceinline__ void clear(Bf4& v) { v.u = make_uint2(0, 0); }
template <typename T> struct FourOf { typedef float4 type; };
template <> struct FourOf<bf16> { typedef Bf4 type; };
__device__ __forceinline__ float4 weigh(float s, const float4 a, float t, const float4 b) {
  return make_float4(fmaf(s, a.x, t * b.x), fmaf(s, a.y, t * b.y), fmaf(s, a.z, t * b.z), fmaf(s, a.w, t * b.w));
}

// 1 / (|u| + eps) from the sum of u's squares.  A matrix of zeros stays one; one with a value that is not finite becomes NaN throughout (1 / infinity would
// leave its finite values zeros).  The sum of finite fp32 squares is finite in 64 bits.
__device__ __forceinline__ double inverse_norm(double squares, float eps) {
  const double d = sqrt(squares) + (double)eps;
  return !isfinite(squares) ? nan("") : d > 0.0 ? 1.0 / d : 0.0;
}

constexpr int AHEAD = 4;                            // fours of a thread in flight
// the new momentum, and the sum of the squares of u in 64 bits (whose range holds any)
template <typename TG, int VEC>
__global__ void __launch_bounds__(256, 4) ortho_norm_kernel(const PrepP p) {
  pdl_wait(); pdl_trigger();
  const int b = blockIdx.y;
  const uint32_t chunks = (p.cols + 3) / 4;
  const uint64_t n = (uint64_t)p.rows * chunks, stride = (uint64_t)gridDim.x * 256;
  double sum = 0.0;
  for (uint64_t e0 = (uint64_t)blockIdx.x * 256 + threadIdx.x; e0 < n; e0 += AHEAD * stride) {
    typename FourOf<TG>::type raw[AHEAD];
    float4 m[AHEAD];
    int64_t row[AHEAD]; int c[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const uint64_t e = e0 + i * stride;
      row[i] = n <= 0xffffffffu ? (uint32_t)e / chunks : e / chunks;
      c[i] = 4 * (int)(e - (uint64_t)row[i] * chunks);
      clear(raw[i]); clear(m[i]);
      if (e < n) {
        raw[i] = load4<VEC>((const TG*)p.G + b * p.stride_g + row[i] * p.ldg + c[i], p.cols - c[i]);
        if (p.m) m[i] = load4<VEC>(p.m + b * p.stride_m + row[i] * p.ldm + c[i], p.cols - c[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (e0 + i * stride >= n) break;
      const int left = p.cols - c[i];
      float4 u = raw[i];
      if (p.m) {
        const float4 g = u, v = weigh(p.beta, m[i], p.w, g);
        float* o = p.m_out + b * p.stride_m_out + row[i] * p.ldm_out + c[i];
        if (VEC) *reinterpret_cast<float4*>(o) = v;
        else { o[0] = v.x; if (left > 1) o[1] = v.y; if (left > 2) o[2] = v.z; if (left > 3) o[3] = v.w; }
        u = p.nesterov ? weigh(p.beta, v, p.w, g) : v;
      }
      sum = fma((double)u.x, (double)u.x, sum); sum = fma((double)u.y, (double)u.y, sum);
      sum = fma((double)u.z, (double)u.z, sum); sum = fma((double)u.w, (double)u.w, sum);
    }
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

// X in fp16 by rows, and what that leaves of it by blocks, filled up with zeros.  A warp takes one 32 x 32 block, 4 rows of 8 fours at a time, and has it in
// flight while the norm is put together.
template <typename TG, int VEC>
__global__ void __launch_bounds__(256) ortho_scale_kernel(const PrepP p, int blocks) {
  pdl_wait(); pdl_trigger();
  const int b = blockIdx.y;
  if (b == 0)
    for (int i = blockIdx.x * 256 + threadIdx.x; i < p.n_counters; i += gridDim.x * 256) p.counters[i] = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r0 = lane >> 3, c0 = 4 * (lane & 7);
  const int n = p.rows32 * p.cols32, e = n - 1 - (blockIdx.x * 8 + warp);      // (from the end: what was read last is still in the L2)
  const int rb = e / p.cols32, cb = e - rb * p.cols32, c = cb * 32 + c0, left = p.cols - c;
  typename FourOf<TG>::type raw[8];
  float4 m[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = rb * 32 + 4 * i + r0;
    const bool there = e >= 0 && left > 0 && row < p.rows;
    clear(raw[i]); clear(m[i]);
    if (there) raw[i] = load4<VEC>((const TG*)p.G + b * p.stride_g + row * p.ldg + c, left);
    if (there && p.m) m[i] = load4<VEC>(p.m_out + b * p.stride_m_out + row * p.ldm_out + c, left);
  }
  __shared__ double s_sum[8], s_inv;
  double sum = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < blocks; i += 256) sum += p.partial[(int64_t)b * blocks + i];
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) sum += s_sum[w];
    s_inv = inverse_norm(sum, p.eps) * (p.O ? 1.0 : (double)(1 << X_EXP));
  }
  __syncthreads();
  if (e < 0) return;
  const double inv = s_inv;
  __half* block = p.lo + ((int64_t)b * n + e) * 1024 + (c0 / 16) * 512 + c0 % 16;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = rb * 32 + 4 * i + r0;
    float4 u = raw[i];
    if (p.m) u = p.nesterov ? weigh(p.beta, m[i], p.w, u) : m[i];
    const float4 x = make_float4((float)(u.x * inv), (float)(u.y * inv), (float)(u.z * inv), (float)(u.w * inv));
    if (p.O) {
      if (row < p.rows) {
        bf16* o = p.O + ((int64_t)b * p.rows + row) * p.cols + c;
        if (left > 0) o[0] = __float2bfloat16_rn(p.scale * x.x);
        if (left > 1) o[1] = __float2bfloat16_rn(p.scale * x.y);
        if (left > 2) o[2] = __float2bfloat16_rn(p.scale * x.z);
        if (left > 3) o[3] = __float2bfloat16_rn(p.scale * x.w);
      }
      continue;
    }
    const uint2 h = make_uint2(half2_bits(x.x, x.y), half2_bits(x.z, x.w));
    const float2 v0 = half2_floats(h.x), v1 = half2_floats(h.y);
    *reinterpret_cast<uint2*>(block + 16 * (4 * i + r0)) = make_uint2(half2_bits(x.x - v0.x, x.y - v0.y), half2_bits(x.z - v1.x, x.w - v1.y));
    if (row < p.rows) *reinterpret_cast<uint2*>(p.hi + ((int64_t)b * p.rows + row) * p.ld + c) = h;
  }
}

// ---- matrices whose shorter side is at most 128: all of it on chip, in one launch ---------------------------
// A cluster works a matrix, each CTA up to 256 columns of it (of the transpose, where it has more rows): X in tensor memory, its fp16 copy
// in shared memory, where both products read it.  The CTAs add up their parts of A through each other's shared memory,
// each a share of its columns, in the order of their ranks; P is formed by each for itself, and multiplies X as a pair of fp16 (the product
// costs little here, and small random matrices would lose more than others: 20 x 30 2.1e-3, with the pair 1.3e-3).  A step is a chain of short dependent works (a product, a pass over its result, a
// barrier): 4 us for 100 x 100, 6 for 128 x 256, 12 where eight CTAs join their sums, against 18 and more through global memory (100 x 100 105 -> 33 us).
// 512 threads: no change.
constexpr int SMALL_SIDE = 128, SMALL_COLS = 256, SMALL_CTAS = 8;
constexpr int SMALL_THREADS = 256, SMALL_WARPS = SMALL_THREADS / 32, PARTS = SMALL_WARPS / 4;      // warps of a quarter of the rows
constexpr int SLAB = 128 * BK * 2;                   // 128 rows x 64 columns of fp16
constexpr int SMALL_X = 4 * SLAB, SMALL_A = 2 * SLAB;
constexpr int SMALL_SMEM = 2 * SMALL_X + 2 * SMALL_A + 1024;
static_assert(128 * 128 * 4 <= SMALL_X, "the sums of A lie where X's second numbers do later");

struct SmallP {
  PrepP in;                          // G, momentum, norm
  int side, length, left, chunk, steps;      // chunk: columns of a CTA, a multiple of 32
  bf16* O; float scale, gram;
  float a[MAX_STEPS], b[MAX_STEPS], c[MAX_STEPS], f[MAX_STEPS];      // X = (a + f P's diagonal) X + f (P X)
  int* flags;
};

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const bf16* p) { return __bfloat162float(*p); }
// elements (i, j .. j + 31) of the matrix (of its transpose, where it has more rows than columns); `have` of them are there
template <typename T> __device__ __forceinline__ void load32(const T* base, int64_t ld, bool left, bool vec, int i, int j, int have, float (&u)[32]) {
  if (left && vec) {
    const T* p = base + i * ld + j;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float4 v = 4 * q < have ? load4<1>(p + 4 * q, 4) : make_float4(0.f, 0.f, 0.f, 0.f);
      u[4 * q] = v.x; u[4 * q + 1] = v.y; u[4 * q + 2] = v.z; u[4 * q + 3] = v.w;
    }
  } else {
    const T* p = left ? base + i * ld + j : base + j * ld + i;
    const int64_t step = left ? 1 : ld;
#pragma unroll
    for (int q = 0; q < 32; ++q) u[q] = q < have ? load1(p + q * step) : 0.f;
  }
}
__device__ __forceinline__ void store32(float* base, int64_t ld, bool left, bool vec, int i, int j, int have, const float (&u)[32]) {
  if (left && vec) {
    float* p = base + i * ld + j;
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (4 * q < have) *reinterpret_cast<float4*>(p + 4 * q) = make_float4(u[4 * q], u[4 * q + 1], u[4 * q + 2], u[4 * q + 3]);
  } else {
    float* p = left ? base + i * ld + j : base + j * ld + i;
    const int64_t step = left ? 1 : ld;
#pragma unroll
    for (int q = 0; q < 32; ++q) if (q < have) p[q * step] = u[q];
  }
}
// 8 fp16 of row r from column c (a multiple of 8) on, in slabs of 64 columns with 128-byte swizzle
__device__ __forceinline__ uint32_t slab_at(int r, int c) { return (c >> 6) * SLAB + r * 128 + ((((c >> 3) & 7) ^ (r & 7)) << 4); }
__device__ __forceinline__ float4 load_peer(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

template <typename TG, int VEC>
__global__ void __launch_bounds__(SMALL_THREADS, 1) ortho_small_kernel(const __grid_constant__ SmallP p) {
  extern __shared__ uint8_t smem_raw[];
  // (the window starts at the same offset in all CTAs of a cluster)
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t *sX = smem, *sL = smem + SMALL_X, *sA = sL + SMALL_X, *sP = sA + SMALL_A;      // X in fp16, what that leaves, A, P
  float4* sums = reinterpret_cast<float4*>(sL);      // [32 fours of columns][128 rows], before sL is written
  __shared__ uint64_t s_bar;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  __shared__ double s_part[SMALL_WARPS], s_total;
  __shared__ float s_diag[128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3, part = warp >> 2, row = quarter * 32 + lane;
  uint32_t rank, ctas;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
  const int b = blockIdx.x / ctas;
  volatile int* abort_flag = &s_abort;
  const uint32_t bar = smem_u32(&s_bar);
  if (threadIdx.x == 0) {
    mbar_init(bar, 1);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  if (warp == 0) tmem_alloc(smem_u32(&s_tmem), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tX = s_tmem + ((uint32_t)(quarter * 32) << 16), tAcc = tX + SMALL_COLS;      // X, and the products' sums
  pdl_wait(); pdl_trigger();

  const int col0 = (int)rank * p.chunk, own = max(0, min(p.chunk, p.length - col0)), chunks = p.chunk / 32;
  uint32_t parity = 0;
  // fn() issues one thread's products; all do what they can meanwhile and wait for them
  auto products = [&](auto fn, auto meanwhile) {
    asm volatile("fence.proxy.async;" ::: "memory");       // (the operands in shared memory were written by plain stores)
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0) {
      tc_fence_after();
      asm volatile("fence.proxy.async;" ::: "memory");
      fn();
      umma_commit(bar);
    }
    __syncwarp();
    meanwhile();
    wait_for(abort_flag, p.flags, [&] { return mbar_try(bar, parity); });      // (where it gives up the results are not valid, and flags say so)
    __syncwarp();                                    // (each lane has left the wait by itself)
    parity ^= 1;
    tc_fence_after();
  };
  // All lanes of a warp take part in a barrier of the cluster, and in a copy to or from tensor memory, together: they are joined before, wherever they may
  // have gone different ways.
  auto cluster_barrier = [&] { __syncwarp(); asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory"); };

  // u, the new momentum and the sum of squares
  double sum = 0.0;
  for (int c = part; c < chunks; c += PARTS) {
    const int j = col0 + 32 * c, have = row < p.side ? min(32, col0 + own - j) : 0;
    float u[32];
    load32((const TG*)p.in.G + b * p.in.stride_g, p.in.ldg, p.left, VEC, row, j, have, u);
    if (p.in.m) {
      float m[32];
      load32(p.in.m + b * p.in.stride_m, p.in.ldm, p.left, VEC, row, j, have, m);
#pragma unroll
      for (int q = 0; q < 32; ++q) m[q] = fmaf(p.in.beta, m[q], p.in.w * u[q]);
      store32(p.in.m_out + b * p.in.stride_m_out, p.in.ldm_out, p.left, VEC, row, j, have, m);
#pragma unroll
      for (int q = 0; q < 32; ++q) u[q] = p.in.nesterov ? fmaf(p.in.beta, m[q], p.in.w * u[q]) : m[q];
    }
    uint32_t bits[32];
#pragma unroll
    for (int q = 0; q < 32; ++q) { sum = fma((double)u[q], (double)u[q], sum); bits[q] = __float_as_uint(u[q]); }
    __syncwarp();
    tmem_st32(tX + 32 * c, bits);
  }
  __syncwarp();
  tmem_st_wait();
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_part[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < SMALL_WARPS; ++w) sum += s_part[w];
    s_total = sum;
  }
  cluster_barrier();
  double norm = 0.0;
  for (uint32_t r = 0; r < ctas; ++r) {
    double d;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(d) : "r"(map_to_rank(smem_u32(&s_total), r)));
    norm += d;
  }
  const double inv = inverse_norm(norm, p.in.eps) * (double)(1 << X_EXP);

  for (int step = 0; step <= p.steps; ++step) {
    // X (after the last step O), and its fp16 copy
    for (int c = part; c < chunks; c += PARTS) {
      uint32_t r[32], y[32];
      __syncwarp();
      tmem_ld32(tX + 32 * c, r);
      if (step > 0) tmem_ld32(tAcc + 32 * c, y);
      tmem_ld_wait();
      float x[32];
      const float f = step > 0 ? p.f[step - 1] : 0.f, a = step > 0 ? fmaf(f, s_diag[row], p.a[step - 1]) : 0.f;
#pragma unroll
      for (int q = 0; q < 32; ++q) x[q] = step == 0 ? (float)(__uint_as_float(r[q]) * inv) : fmaf(f, __uint_as_float(y[q]), a * __uint_as_float(r[q]));
      if (step < p.steps) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<uint4*>(sX + slab_at(row, 32 * c + 8 * q)) =
              make_uint4(half2_bits(x[8 * q], x[8 * q + 1]), half2_bits(x[8 * q + 2], x[8 * q + 3]), half2_bits(x[8 * q + 4], x[8 * q + 5]), half2_bits(x[8 * q + 6], x[8 * q + 7]));
#pragma unroll
        for (int q = 0; q < 32; ++q) r[q] = __float_as_uint(x[q]);
        tmem_st32(tX + 32 * c, r);
      } else {
        const int j = col0 + 32 * c, have = row < p.side ? min(32, col0 + own - j) : 0;
        const int m = p.left ? p.side : p.length, n = p.left ? p.length : p.side;
        bf16* O = p.O + (int64_t)b * m * n;
        if (p.left) {                                // (rows that are not whole 16 bytes go through shared memory)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = p.scale * x[8 * q + e];
            const uint4 v = gemm_tc_detail::pack8_bf16(y);
            if (n % 8) *reinterpret_cast<uint4*>(sX + slab_at(row, 32 * c + 8 * q)) = v;
            else if (8 * q < have) *reinterpret_cast<uint4*>(O + (int64_t)row * n + j + 8 * q) = v;
          }
        } else {
          bf16* o = O + (int64_t)j * n + row;
#pragma unroll
          for (int q = 0; q < 32; ++q) if (q < have) o[(int64_t)q * n] = __float2bfloat16_rn(p.scale * x[q]);
        }
      }
    }
    if (step == p.steps) {
      if (p.left && p.length % 8) {
        __syncthreads();
        for (int r = warp; r < p.side; r += SMALL_WARPS)
          for (int c = lane; c < own; c += 32)
            p.O[((int64_t)b * p.side + r) * p.length + col0 + c] = *reinterpret_cast<const bf16*>(sX + slab_at(r, c & ~7) + (c & 7) * 2);
      }
      break;
    }
    tmem_st_wait();
    // A = X X^T of this CTA's columns
    const uint32_t idesc = (1u << 4) | ((uint32_t)(128 >> 4) << 24);
    const uint32_t aX = smem_u32(sX), aL = smem_u32(sL), aA = smem_u32(sA), aP = smem_u32(sP), tBase = s_tmem;
    products([&] {
      for (int k = 0; k < p.chunk / UMMA_K; ++k) {
        const uint64_t d = make_desc(aX + (k >> 2) * SLAB + (k & 3) * 32, 16, 1024);
        umma_bf16(tBase + SMALL_COLS, d, d, idesc | (uint32_t)(128 >> 3) << 17, k > 0);
      }
    }, [] {});
    // A in fp16, of all CTAs' sums
#pragma unroll 1
    for (int c = 128 / PARTS * part; c < 128 / PARTS * (part + 1); c += 32) {
      uint32_t r[32];
      tmem_ld32(tAcc + c, r);
      tmem_ld_wait();
      if (ctas == 1) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint4 v;
          uint32_t* o = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = half2_bits(p.gram * __uint_as_float(r[8 * q + 2 * e]), p.gram * __uint_as_float(r[8 * q + 2 * e + 1]));
          *reinterpret_cast<uint4*>(sA + slab_at(row, c + 8 * q)) = v;
        }
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          sums[(c / 4 + q) * 128 + row] = make_float4(__uint_as_float(r[4 * q]), __uint_as_float(r[4 * q + 1]), __uint_as_float(r[4 * q + 2]), __uint_as_float(r[4 * q + 3]));
      }
    }
    if (ctas > 1) {
      cluster_barrier();
      const int share = 32 * 128 / (int)ctas;        // fours of columns x rows
      for (int e = threadIdx.x; e < share; e += SMALL_THREADS) {
        const int at = (int)rank * share + e, r = at & 127, c = 4 * (at >> 7);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f), x[SMALL_CTAS];
        const uint32_t from = smem_u32(sums + at);
#pragma unroll
        for (uint32_t q = 0; q < SMALL_CTAS; ++q) x[q] = q < ctas ? load_peer(map_to_rank(from, q)) : v;
#pragma unroll
        for (uint32_t q = 0; q < SMALL_CTAS; ++q) { v.x += x[q].x; v.y += x[q].y; v.z += x[q].z; v.w += x[q].w; }
        const uint32_t h0 = half2_bits(p.gram * v.x, p.gram * v.y), h1 = half2_bits(p.gram * v.z, p.gram * v.w);
        const uint32_t to = aA + slab_at(r, c & ~7) + (c & 4) * 2;
        for (uint32_t q = 0; q < ctas; ++q) asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(map_to_rank(to, q)), "r"(h0), "r"(h1) : "memory");
      }
      asm volatile("fence.proxy.async;" ::: "memory");
      cluster_barrier();
    }
    // P = b A + c A A
    products([&] {
      for (int k = 0; k < 128 / UMMA_K; ++k) {
        const uint64_t d = make_desc(aA + (k >> 2) * SLAB + (k & 3) * 32, 16, 1024);
        umma_bf16(tBase + SMALL_COLS, d, d, idesc | (uint32_t)(128 >> 3) << 17, k > 0);
      }
    }, [&] {
      for (int c = part; c < chunks; c += PARTS) {      // what X's fp16 copy leaves of it
        uint32_t r[32];
        tmem_ld32(tX + 32 * c, r);
        tmem_ld_wait();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t o[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x0 = __uint_as_float(r[8 * q + 2 * e]), x1 = __uint_as_float(r[8 * q + 2 * e + 1]);
            const float2 h = half2_floats(half2_bits(x0, x1));
            o[e] = half2_bits(x0 - h.x, x1 - h.y);
          }
          *reinterpret_cast<uint4*>(sL + slab_at(row, 32 * c + 8 * q)) = make_uint4(o[0], o[1], o[2], o[3]);
        }
      }
    });
#pragma unroll 1
    for (int c = 128 / PARTS * part; c < 128 / PARTS * (part + 1); c += 32) {
      uint32_t r[32];
      __syncwarp();
      tmem_ld32(tAcc + c, r);
      tmem_ld_wait();
      const float fb = p.b[step], fc = p.c[step];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint4 a = *reinterpret_cast<const uint4*>(sA + slab_at(row, c + 8 * q));
        const uint32_t* h = reinterpret_cast<const uint32_t*>(&a);
        uint4 v;
        uint32_t* o = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 x = half2_floats(h[e]);
          float2 y = make_float2(fmaf(fc, __uint_as_float(r[8 * q + 2 * e]), fb * x.x), fmaf(fc, __uint_as_float(r[8 * q + 2 * e + 1]), fb * x.y));
          if (c == 32 * quarter && lane / 2 == 4 * q + e) {      // the diagonal
            s_diag[row] = lane & 1 ? y.y : y.x;
            (lane & 1 ? y.y : y.x) = 0.f;
          }
          o[e] = half2_bits(y.x, y.y);
        }
        *reinterpret_cast<uint4*>(sP + slab_at(row, c + 8 * q)) = v;
      }
    }
    // P X
    products([&] {
      for (int k = 0; k < 2 * 128 / UMMA_K; ++k) {
        const int j = k & 7;                         // (X, then what it leaves)
        umma_bf16(tBase + SMALL_COLS, make_desc(aP + (j >> 2) * SLAB + (j & 3) * 32, 16, 1024), make_desc((k < 8 ? aX : aL) + j * 2048, SLAB, 1024),
                  idesc | (1u << 16) | (uint32_t)(p.chunk >> 3) << 17, k > 0);
      }
    }, [] {});
  }
  __syncwarp();
  if (*abort_flag)
    for (int i = 0; i < 64; ++i) __nanosleep(2000);  // products in flight
  tc_fence_before();
  __syncthreads();
  cluster_barrier();                                 // no CTA leaves while another may still read its shared memory
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(s_tmem, 512);
  }
}

// ---- host ------------------------------------------------------------------------------------------
struct Plan {
  int side, blocks; int64_t ld, lds;
  bool pair;
  int ctas, chunk;                   // on chip: CTAs of a matrix (0: not so), columns of each
  int tiles_s, sym, tiles_m, tiles_n, splits, workers;
  size_t partial, hi[2], lo, a, a2, p, diag, sums, counters, bytes;
  int rows32, cols32, side32;
  int n_counters;
};

Plan make_plan(int batch, int m, int n, int steps) {
  Plan q = {};
  q.side = std::min(m, n);
  q.ld = ((int64_t)n + 63) / 64 * 64;
  q.lds = ((int64_t)q.side + 63) / 64 * 64;
  q.rows32 = (m + 31) / 32; q.cols32 = (n + 31) / 32; q.side32 = (q.side + 31) / 32;
  const int64_t chunks = (int64_t)m * ((n + 3) / 4);
  q.blocks = (int)std::max<int64_t>(1, std::min<int64_t>((chunks + 1023) / 1024, SMS * 4 / std::min(batch, SMS * 4)));
  auto tiles = [](int64_t x, int t) { return (int)((x + t - 1) / t); };
  // SM pairs on 256 x 256 tiles, or single SMs on 128 x 128.  Pairs read half as much for a product, singles have four times the units to share out and shorter
  // ones to wait for.  So pairs where the products bound a step, from 28 GFLOP on, unless a good part of their tiles is empty (less than 3.5 tiles of 128 x 128
  // to one of 256 x 256).  Five steps, us, pairs and singles; in brackets where calls follow one another for half a second (the clock then falls under large products):
  //   full tiles   8192 x 2048 (112 GFLOP) 590 and 740 (653, 810), 101 x 509 x 481 (47) 702 and 738 (776, 820), 2 x 1700 x 2000 (45) 283 and 354, 4 x 1300 x 1300 (35) 280 and 312,
  //                2048 x 2048 (34) 269 and 282, 4 x 1024 x 2048 (30) 252 and 255 (267, 281), 7 x 1024 x 1024 (30) 233 and 242, 8 x 900 x 1200 (29) 259 and 303,
  //                2300 x 1800 (28) 266 and 282;   below: 6 x 1024 x 1024 (26) 222 and 217 (235, 241), 60 x 256 x 2048 (25) 524 and 509 (542, 536), 3 x 1024 x 2048 (23) 240 and 220,
  //                12 x 768 x 768 (22) 210 and 202 (226, 227), 12 x 512 x 2048 (21) 262 and 264, 48 x 256 x 2048 (20) 435 and 407, 6 x 512 x 4096 (20) 296 and 275, 2 x 1300 x 1300 (18)
  //                229 and 211, 24 x 256 x 2048 (10) 241 and 239, 24 x 256 x 1024 (5) 167 and 141; but 60 x 200 x 2048 (15) 552 and 591
  //   others       96 x 384 x 2048 (92) 1532 and 1221, 128 x 260 x 2500 (67) 2443 and 2032, 80 x 300 x 2600 (58) 1497 and 1263, 32 x 384 x 2048 (31) 503 and 421
  const double flop = (double)batch * q.side * q.side * (3.0 * std::max(m, n) + q.side);
  const int64_t singles = (int64_t)tiles(m, 128) * tiles(n, 128) * batch, pairs = (int64_t)tiles(m, 256) * tiles(n, 256) * batch;
  q.pair = q.side > 128 && flop >= 28e9 && 2 * singles >= 7 * pairs;
  const int t = q.pair ? 256 : 128;
  q.workers = q.pair ? SMS / 2 : SMS;
  q.tiles_s = tiles(q.side, t); q.sym = q.tiles_s * (q.tiles_s + 1) / 2;
  q.tiles_m = tiles(m, t); q.tiles_n = tiles(n, t);
  // The sums of A in slices where there are fewer tiles than workers.  Pairs: of 4096 products at least, since joining slices takes about 7 us, and
  // 2048 products 10 (8192 x 2048: A in two slices 30 us, in one 48).  Single SMs: of 1024 (8 x 64 x 4096: a step 20.9 us, in one slice 34.3, in eight 23.3).
  // (A A's sums are of the shorter side; by the same rule it has more tiles than workers before they are long enough.)
  const int64_t k_blocks = ((int64_t)std::max(m, n) + KH * BK - 1) / (KH * BK);
  q.splits = (int)std::max<int64_t>(1, std::min<int64_t>({8, q.workers / std::max<int64_t>(1, (int64_t)q.sym * batch), k_blocks / (q.pair ? 32 : 8)}));
  // on chip where a cluster of up to 8 CTAs holds the matrix
  const int length = std::max(m, n);
  if (steps > 0 && q.side <= SMALL_SIDE && length <= SMALL_COLS * SMALL_CTAS) {
    q.ctas = 1;
    while (q.ctas * SMALL_COLS < length) q.ctas *= 2;
    q.chunk = ((length + q.ctas - 1) / q.ctas + 31) / 32 * 32;
    q.bytes = 256;                                 // (nothing is kept in it; checked as any workspace)
    return q;
  }
  size_t at = 0;
  auto take = [&](size_t k) { const size_t was = at; at += (k + 255) / 256 * 256; return was; };
  q.partial = take((size_t)batch * q.blocks * 8);
  if (steps > 0) {
    const size_t x = (size_t)batch * m * q.ld * 2, s = (size_t)batch * q.side * q.lds * 2;
    q.hi[0] = take(x); q.hi[1] = take(steps > 1 ? x : 0); q.lo = take((size_t)batch * q.rows32 * q.cols32 * 2048);
    q.a = take(s); q.a2 = take((size_t)batch * q.side32 * q.side32 * 2048); q.p = take(s);
    q.diag = take(q.side < DIAG_SIDE ? (size_t)batch * q.side * 4 : 0);
    const int ctas = q.pair ? 2 : 1;
    q.sums = take(q.splits > 1 ? (size_t)batch * q.sym * q.splits * t * t * 4 : 0);
    q.n_counters = (3 + std::max(q.tiles_m, q.tiles_n)) * batch + (q.splits > 1 ? batch * q.sym * ctas * EPI : 0);
    q.counters = take((size_t)q.n_counters * 4);
  }
  q.bytes = at;
  return q;
}

int check_ortho(int batch, int m, int n, int steps) {
  if (batch < 0 || m < 0 || n < 0) return ppu_fail(PPU_EINVAL, "negative size");
  if (m > MAX_SIDE || n > MAX_SIDE || batch > 65535) return ppu_fail(PPU_ESHAPE, "at most 65535 matrices of sides up to %d", MAX_SIDE);
  if (steps < 0 || steps > MAX_STEPS) return ppu_fail(PPU_EINVAL, "steps must be 0 to %d", MAX_STEPS);
  // (16 warps report each tile in each of 32 steps: counted in 32 bits)
  const int64_t tiles = (((int64_t)m + 127) / 128) * (((int64_t)n + 127) / 128) * batch;
  if (tiles > (1 << 20)) return ppu_fail(PPU_ESHAPE, "too many matrices of this size");
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

// boxes of 64 x 128 over [batch][rows][inner]
bool encode(CUtensorMap* map, const __half* base, int64_t ld, int inner, int rows, int batch) {
  const cuuint64_t dim[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)batch}, stride[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * rows * 2};
  const cuuint32_t box[3] = {(cuuint32_t)BK, 128, 1}, one[3] = {1, 1, 1};
  return get_encoder()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, (void*)base, dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// how many CTAs (or pairs) are resident together on the current device
int resident(bool pair) {
  static int known[2][PPU_MAX_DEVICES];
  int& n = known[pair][ppu_current_device()];
  if (n > 0) return n;
  int got = 0;
  if (pair) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2); cfg.blockDim = dim3(BLOCK); cfg.dynamicSmemBytes = SMEM;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&got, ortho_pair_kernel<true>, &cfg) != cudaSuccess) return -1;
    n = std::min(got, ppu_sm_count() / 2);
  } else {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&got, ortho_single_kernel<true>, BLOCK, SMEM) != cudaSuccess) return -1;
    n = got > 0 ? ppu_sm_count() : 0;
  }
  return n;
}

int launch_steps(const Maps& maps, const KernelP& p, bool pair, cudaStream_t st) {
  static PerDeviceFlag attr_set[4];
  void (*kernels[4])(Maps, KernelP) = {ortho_single_kernel<false>, ortho_single_kernel<true>, ortho_pair_kernel<false>, ortho_pair_kernel<true>};
  for (int i = 0; i < 4; ++i)
    if (!ppu_set_smem_once(attr_set[i], kernels[i], SMEM)) return ppu_fail(PPU_ECUDA, "shared memory limit not accepted");
  auto kernel = kernels[2 * pair + (p.diag != nullptr)];
  const int most = resident(pair);
  if (most < p.splits) return ppu_fail(PPU_ECUDA, "the kernel does not fit on this device");
  const int units = p.batch * std::max(p.units[GRAM], std::max(p.units[POLY], p.units[UPDATE]));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((pair ? 2 : 1) * std::min(most, units)); cfg.blockDim = dim3(BLOCK); cfg.dynamicSmemBytes = SMEM; cfg.stream = st;
  cudaLaunchAttribute attr[1];                     // CTAs wait for one another: all of them are resident
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, maps, p));
  return PPU_OK;
}

int launch_small(const SmallP& p, int batch, int ctas, bool vec, bool f32, cudaStream_t st) {
  static PerDeviceFlag attr_set[4];
  void (*kernel)(SmallP) = f32 ? (vec ? ortho_small_kernel<float, 1> : ortho_small_kernel<float, 0>) : vec ? ortho_small_kernel<bf16, 1> : ortho_small_kernel<bf16, 0>;
  if (!ppu_set_smem_once(attr_set[2 * f32 + vec], kernel, SMALL_SMEM)) return ppu_fail(PPU_ECUDA, "shared memory limit not accepted");
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)batch * ctas); cfg.blockDim = dim3(SMALL_THREADS); cfg.dynamicSmemBytes = SMALL_SMEM; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas; attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, p));
  return PPU_OK;
}

template <typename TG>
int prepare(const PrepP& p, const Plan& q, int batch, bool vec, cudaStream_t st) {
  const dim3 grid(q.blocks, batch), blocks32((q.rows32 * q.cols32 + 7) / 8, batch);
  if (vec) {
    CUDA_OK(ppu_launch_dependent(ortho_norm_kernel<TG, 1>, grid, 256, 0, st, p));
    CUDA_OK(ppu_launch_dependent(ortho_scale_kernel<TG, 1>, blocks32, 256, 0, st, p, q.blocks));
  } else {
    CUDA_OK(ppu_launch_dependent(ortho_norm_kernel<TG, 0>, grid, 256, 0, st, p));
    CUDA_OK(ppu_launch_dependent(ortho_scale_kernel<TG, 0>, blocks32, 256, 0, st, p, q.blocks));
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
    // (X's second number loses its digits with X: at 2^-10 values of 2^-13 of the norm keep 14 bits; zeros are exact)
    if (top > 0.0 && top < 0x1p-10) return ppu_fail(PPU_EINVAL, "the coefficients of step %d leave no singular value above %g, below 2^-10", k, top);
    p_exp[k] = std::min(12, (int)std::floor(std::log2(32768.0 / std::max(poly, 1e-30))));
  }
  if (batch == 0 || m == 0 || n == 0) return PPU_OK;
  if (!G || !O || !workspace) return ppu_fail(PPU_EINVAL, "null operand");
  if (ldg < n || (momentum && (ldm < n || ldmo < n))) return ppu_fail(PPU_EINVAL, "row strides must be at least n");
  if (batch > 1 && (stride_g < 0 || (momentum && stride_m < 0))) return ppu_fail(PPU_EINVAL, "strides must not be negative");
  // one matrix behind another, or the rows of all matrices beside one another
  if (batch > 1 && momentum && !(stride_mo >= (m - 1) * ldmo + n || (stride_mo >= n && ldmo >= (batch - 1) * stride_mo + n)))
    return ppu_fail(PPU_EINVAL, "matrices written must not overlap");
  if (momentum_out == momentum && momentum && (ldm != ldmo || (batch > 1 && stride_m != stride_mo)))
    return ppu_fail(PPU_EINVAL, "momentum_out in the place of momentum needs its strides");
  if (momentum_out && (const void*)momentum_out == G) return ppu_fail(PPU_EINVAL, "G is read again after momentum_out is written: they must not overlap");
  const int g_bytes = g_type == PPU_BF16 ? 2 : 4;
  if ((reinterpret_cast<uintptr_t>(G) % g_bytes) || (reinterpret_cast<uintptr_t>(momentum) & 3) || (reinterpret_cast<uintptr_t>(momentum_out) & 3) ||
      (reinterpret_cast<uintptr_t>(O) & 15) || (reinterpret_cast<uintptr_t>(workspace) & 255))
    return ppu_fail(PPU_EINVAL, "O must be 16-byte, workspace 256-byte aligned, G and momentum as their types are");
  const Plan q = make_plan(batch, m, n, steps);
  if (workspace_bytes < q.bytes) return ppu_fail(PPU_ENOMEM, "workspace has %zu bytes, %zu needed", workspace_bytes, q.bytes);
  if (steps > 0 && gemm_tc_init() != 0) return ppu_fail(PPU_ECUDA, "no tensor-map encoder");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  uint8_t* ws = (uint8_t*)workspace;
  __half *hi[2] = {(__half*)(ws + q.hi[0]), (__half*)(ws + q.hi[1])}, *A = (__half*)(ws + q.a), *P = (__half*)(ws + q.p);
  PrepP pp = {};
  pp.G = G; pp.ldg = ldg; pp.stride_g = stride_g; pp.m = momentum; pp.ldm = ldm; pp.stride_m = stride_m;
  pp.m_out = momentum_out; pp.ldm_out = ldmo; pp.stride_m_out = stride_mo; pp.rows = m; pp.cols = n; pp.nesterov = nesterov != 0;
  pp.beta = beta; pp.w = weight; pp.eps = eps; pp.scale = scale; pp.partial = (double*)(ws + q.partial); pp.hi = hi[0]; pp.ld = q.ld;
  pp.lo = (__half*)(ws + q.lo); pp.rows32 = q.rows32; pp.cols32 = q.cols32;
  pp.O = steps == 0 ? (bf16*)O : nullptr;
  pp.counters = (unsigned*)(ws + q.counters); pp.n_counters = q.n_counters;
  const bool vec = n % 4 == 0 && aligned(G, ldg, stride_g, 4 * g_bytes) && aligned(momentum, ldm, stride_m, 16) && aligned(momentum_out, ldmo, stride_mo, 16);
  if (q.ctas > 0) {
    SmallP p = {};
    p.in = pp; p.side = q.side; p.length = std::max(m, n); p.left = m <= n; p.chunk = q.chunk; p.steps = steps;
    p.O = (bf16*)O; p.scale = std::ldexp(scale, -X_EXP); p.gram = std::ldexp(1.f, A_EXP - 2 * X_EXP); p.flags = flags;
    for (int k = 0; k < steps; ++k) {
      const float* c = coef + (n_coef == 1 ? 0 : 3 * k);
      p.b[k] = std::ldexp(c[1], p_exp[k] - A_EXP); p.c[k] = std::ldexp(c[2], p_exp[k] - 2 * A_EXP);
      p.a[k] = c[0]; p.f[k] = std::ldexp(1.f, -p_exp[k]);
    }
    return launch_small(p, batch, q.ctas, vec, g_type == PPU_F32, st);
  }
  const int rc2 = g_type == PPU_BF16 ? prepare<bf16>(pp, q, batch, vec, st) : prepare<float>(pp, q, batch, vec, st);
  if (rc2 || steps == 0) return rc2;
  Maps maps;
  if (!encode(&maps.m[0], hi[0], q.ld, n, m, batch) || !encode(&maps.m[1], steps > 1 ? hi[1] : hi[0], q.ld, n, m, batch) ||
      !encode(&maps.m[2], A, q.lds, q.side, q.side, batch) || !encode(&maps.m[3], P, q.lds, q.side, q.side, batch))
    return ppu_fail(PPU_ECUDA, "tensor map not accepted");
  KernelP p = {};
  p.m = m; p.n = n; p.side = q.side; p.batch = batch; p.steps = steps; p.left = m <= n;
  p.tiles_s = q.tiles_s; p.sym = q.sym; p.tiles_m = q.tiles_m; p.tiles_n = q.tiles_n; p.n_fast = m > n;
  p.splits = q.splits;
  const int tiles = q.tiles_m * q.tiles_n, rem = tiles % q.workers;
  p.tail_from = 1 << 30;
  p.units[GRAM] = q.sym * q.splits; p.units[POLY] = q.sym; p.units[UPDATE] = tiles;
  if (q.pair && batch == 1 && tiles > q.workers && rem > 0 && 2 * rem <= q.workers) {      // a last wave of halves instead of one of few tiles
    p.tail_from = tiles - rem;
    p.units[UPDATE] = tiles + rem;
  }
  p.per_step = batch * (p.units[GRAM] + p.units[POLY] + p.units[UPDATE]);
  p.A = A; p.P = P; p.hi[0] = hi[0]; p.hi[1] = hi[1]; p.lo = pp.lo; p.A2 = (__half*)(ws + q.a2); p.diag = q.side < DIAG_SIDE ? (float*)(ws + q.diag) : nullptr; p.rows32 = q.rows32; p.cols32 = q.cols32; p.side32 = q.side32; p.ld = q.ld; p.lds = q.lds; p.O = (bf16*)O; p.scale = scale;
  p.gram = std::ldexp(1.f, A_EXP - 2 * X_EXP);
  for (int k = 0; k < steps; ++k) {
    const float* c = coef + (n_coef == 1 ? 0 : 3 * k);
    const int out = k + 1 < steps ? 0 : -X_EXP;    // O has no power of two
    p.b[k] = std::ldexp(c[1], p_exp[k] - A_EXP); p.c[k] = std::ldexp(c[2], p_exp[k] - 2 * A_EXP);
    p.a[k] = std::ldexp(c[0], out); p.f[k] = p.d[k] = std::ldexp(1.f, out - p_exp[k]);
  }
  p.partial = (float*)(ws + q.sums); p.done = pp.counters; p.tiles_l = p.left ? q.tiles_n : q.tiles_m; p.along = p.done + 3 * batch; p.arrived = p.along + (int64_t)batch * p.tiles_l; p.flags = flags;
  return launch_steps(maps, p, q.pair, st);
}
