// tcgen05 GEMM for sm_100a: C[M,N] = A . B^T with bf16 operands and fp32 accumulation in
// tensor memory.  One persistent CTA per SM walks 128 x BN output tiles; a producer thread
// streams 64-deep operand slabs into a shared-memory ring with TMA (128-byte swizzle), one
// thread issues tcgen05.mma (M=128, N=BN, K=16) into one of two TMEM accumulators, and four
// epilogue warps drain the other accumulator through registers into global memory, so the
// epilogue of tile i overlaps the main loop of tile i+1.  Both operands may be K-major
// (row-major [rows, K]) or MN-major (stored [K, rows]) - forward products are K/K, input
// gradients K/MN, subset weight gradients MN/MN (the reduction runs over tokens).
//
// Every mbarrier wait is bounded: on expiry the CTA raises a shared abort flag and a device
// error word, all roles leave their loops, tensor memory is released and the kernel returns.
#include <mutex>
#include <unordered_map>
#include "gemm_epilogue.cuh"

namespace tc {
static EncodeTiledFn g_encode = nullptr;
EncodeTiledFn get_encoder() { return g_encode; }
}  // namespace tc

namespace {
using namespace tc;
using namespace gemm_tc_detail;

template <int BN> struct Cfg {
  static constexpr int STAGES = BN == 256 ? 4 : 6;
  static constexpr int A_BYTES = BM * BK * 2;
  static constexpr int B_BYTES = BN * BK * 2;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int SMEM = STAGES * STAGE_BYTES + 1024 /*align*/ + 256 /*barriers*/;
  static constexpr int TMEM_COLS = 2 * BN;
};

template <int BN, bool A_K, bool B_K, int MODE>
__global__ void __launch_bounds__(gemm_threads(MODE, BN), 1)
gemm_tc_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
               const __grid_constant__ Second<MODE> two, const __grid_constant__ TcParams p) {
  using C = Cfg<BN>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~(uintptr_t)1023);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::STAGES * C::STAGE_BYTES + store_smem<MODE, BN>());
  // bars[0..ST): full, [ST..2ST): empty, [2ST..2ST+2): tmem_full, [2ST+2..2ST+4): tmem_empty
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * C::STAGES + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
  auto tfull_bar = [&](int a) { return bar0 + 8u * (2 * C::STAGES + a); };
  auto tempty_bar = [&](int a) { return bar0 + 8u * (2 * C::STAGES + 2 + a); };

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), MODE != DRAIN_COLS && p.alternate ? epi_warps(MODE, BN) / 2 : epi_warps(MODE, BN)); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), (uint32_t)C::TMEM_COLS);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  if (p.dependent) { pdl_wait(); pdl_trigger(); }
  if (MODE == DRAIN_PIECES && blockIdx.x == 0 && threadIdx.x == 0 && p.zero_word) *p.zero_word = 0;

  const int tiles_mn = p.tiles_m * p.tiles_n;
  int num_tiles = tiles_mn * p.splits;
  const int k_blocks = (p.K + BK - 1) / BK;
  // units of a DRAIN_TWO launch: those of p, then those of two.p
  constexpr bool TWO = MODE == DRAIN_TWO, FIT = MODE != DRAIN_COLS;   // FIT: boxes may be smaller than a stage
  if constexpr (TWO) num_tiles = two.units + two.units2;
  auto unit_of = [&](int i) {
    if constexpr (TWO) return two_unit(i, blockIdx.x, gridDim.x, two.units, two.units2, two.fill);
    else return (int)(blockIdx.x + i * gridDim.x);
  };
  auto second = [&](int u) { if constexpr (TWO) return u >= two.units; else return false; };
  auto params = [&](bool sec) { if constexpr (TWO) return sec ? &two.p : &p; else return &p; };
  auto a_kmajor = [&](bool sec) { if constexpr (TWO) return (sec ? two.a_k2 : two.a_k) != 0; else return A_K; };
  struct Place { int sp, m0, n0, kb0, kb1; };
  auto locate = [&](int u, bool sec) {
    const TcParams& q = *params(sec);
    int per = tiles_mn, kbs = k_blocks;
    if constexpr (TWO) {
      per = q.tiles_m * q.tiles_n; kbs = (q.K + BK - 1) / BK;
      if (sec) u -= two.units;
    }
    Place w;
    w.sp = u / per;
    const int t2 = u - w.sp * per;
    w.m0 = (t2 % q.tiles_m) * BM; w.n0 = (t2 / q.tiles_m) * BN;
    w.kb0 = (int)((long long)w.sp * kbs / q.splits);
    w.kb1 = (int)((long long)(w.sp + 1) * kbs / q.splits);
    return w;
  };

  if (warp == 0) {
    if (lane == 0) {
      // ---------------- TMA producer ----------------
      int s = 0; uint32_t ph = 0;
      for (int i = 0, u = unit_of(0); u < num_tiles; u = unit_of(++i)) {
        const bool sec = second(u), ak = a_kmajor(sec);
        const Place w = locate(u, sec);
        uint32_t stage_bytes = C::STAGE_BYTES;
        if constexpr (FIT)
          stage_bytes = (ak ? params(sec)->a_rows * 128 : (BM / 64) * params(sec)->k_rows * 128) +
                        (B_K ? C::B_BYTES : (BN / 64) * params(sec)->k_rows * 128);
        const CUtensorMap *mA = &mapA, *mB = &mapB;
        if constexpr (TWO) if (sec) { mA = &two.a; mB = &two.b; }
        bool ok = true;
        for (int kb = w.kb0; kb < w.kb1 && ok; ++kb) {
          ok = mbar_wait(empty_bar(s), ph ^ 1u, abort_flag, p.flags);
          if (!ok) break;
          const uint32_t a_dst = smem_u32(smem + s * C::STAGE_BYTES);
          const uint32_t b_dst = a_dst + C::A_BYTES;
          mbar_expect_tx(full_bar(s), stage_bytes);
          if (ak) {
            tma_load_2d(a_dst, mA, full_bar(s), kb * BK, w.m0);
          } else {
#pragma unroll
            for (int j = 0; j < BM / 64; ++j)
              tma_load_2d(a_dst + j * 8192, mA, full_bar(s), w.m0 + 64 * j, kb * BK);
          }
          if (B_K) {
            tma_load_2d(b_dst, mB, full_bar(s), kb * BK, w.n0);
          } else {
#pragma unroll
            for (int j = 0; j < BN / 64; ++j)
              tma_load_2d(b_dst + j * 8192, mB, full_bar(s), w.n0 + 64 * j, kb * BK);
          }
          if (++s == C::STAGES) { s = 0; ph ^= 1u; }
        }
        if (!ok) break;
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      // ---------------- MMA issuer ----------------
      // instruction descriptor: D fp32, A/B bf16, majors, N >> 3, M >> 4
      const uint32_t idesc0 = (1u << 4) | (1u << 7) | (1u << 10) | ((B_K ? 0u : 1u) << 16) | ((uint32_t)(BN >> 3) << 17) |
                              ((uint32_t)(BM >> 4) << 24);
      int s = 0; uint32_t ph = 0;
      int acc = 0; uint32_t acc_ph = 0;
      for (int i = 0, u = unit_of(0); u < num_tiles; u = unit_of(++i)) {
        const bool sec = second(u), ak = a_kmajor(sec);
        const int k_rows = FIT ? params(sec)->k_rows : BK;
        const Place w = locate(u, sec);
        const uint32_t idesc = idesc0 | ((ak ? 0u : 1u) << 15);
        if (!mbar_wait(tempty_bar(acc), acc_ph ^ 1u, abort_flag, p.flags)) break;
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + (uint32_t)(acc * BN);
        bool ok = true;
        for (int kb = w.kb0; kb < w.kb1; ++kb) {
          ok = mbar_wait(full_bar(s), ph, abort_flag, p.flags);
          if (!ok) break;
          tc_fence_after();
          // (rows of A past a smaller box are what was there before: rows of the accumulator that are not stored)
          const uint32_t a_addr = smem_u32(smem + s * C::STAGE_BYTES);
          const uint32_t b_addr = a_addr + C::A_BYTES;
          auto product = [&](int k) {
            const uint64_t adesc = ak ? make_desc(a_addr + k * 32, 16, 1024)
                                      : make_desc(a_addr + k * 2048, 8192, 1024);
            const uint64_t bdesc = B_K ? make_desc(b_addr + k * 32, 16, 1024)
                                       : make_desc(b_addr + k * 2048, 8192, 1024);
            umma_bf16(d_tmem, adesc, bdesc, idesc, (kb > w.kb0 || k > 0) ? 1u : 0u);
          };
          if (k_rows == BK) {
#pragma unroll
            for (int k = 0; k < BK / UMMA_K; ++k) product(k);
          } else {
#pragma unroll 1
            for (int k = 0; k * UMMA_K < k_rows; ++k) product(k);
          }
          umma_commit(empty_bar(s));           // slot is free once these MMAs have read it
          if (++s == C::STAGES) { s = 0; ph ^= 1u; }
        }
        if (!ok) break;
        umma_commit(tfull_bar(acc));           // accumulator complete
        if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
      }
    }
  } else {
    // ---------------- epilogue warps ----------------
    const int quarter = warp & 3;              // TMEM lanes [32 q, 32 q + 32) belong to this warp
    const int set = (warp - 2) >> 2;           // four warps that drain the same columns
    const int turn = MODE != DRAIN_COLS && p.alternate ? set / (epi_warps(MODE, BN) / 8) : -1;
    const uint32_t store_buf = smem_u32(smem + C::STAGES * C::STAGE_BYTES) + (warp - 2) * store_bytes(MODE);
    int acc = 0; uint32_t acc_ph = 0;
    for (int i = 0, u = unit_of(0); u < num_tiles; u = unit_of(++i)) {
      if (turn >= 0 && acc != turn) {            // the other warps' accumulator
        if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
        continue;
      }
      int c_begin, c_end;
      set_columns<MODE, BN>(set, turn >= 0, BN, c_begin, c_end);
      const bool sec = second(u);
      const Place w = locate(u, sec);
      if (!mbar_wait(tfull_bar(acc), acc_ph, abort_flag, p.flags)) break;
      tc_fence_after();
      const uint32_t t_acc = tmem_base + (uint32_t)(acc * BN);
      drain<MODE>(*params(sec), store_buf, w.m0, w.n0, w.sp, t_acc, quarter, c_begin, c_end, lane, [&] {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty_bar(acc));
      });
      if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
    }
  }

  // ---------------- common exit ----------------
  if (*abort_flag) {
    // give copies and MMAs already in flight time to land before memory is released
    for (int i = 0; i < 64; ++i) __nanosleep(2000);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, (uint32_t)C::TMEM_COLS);
  }
}

}  // namespace

namespace gemm_tc_detail {
// Tensor maps are cached per (address, leading dimension, order, extents, box): a training step
// issues the same few hundred products every time, and encoding is a driver call.
namespace mapcache {
struct MapKey {
  const void* base; long long ld; int kmajor, rows, K, box_rows;
  bool operator==(const MapKey& o) const {
    return base == o.base && ld == o.ld && kmajor == o.kmajor && rows == o.rows && K == o.K && box_rows == o.box_rows;
  }
};
struct MapKeyHash {
  size_t operator()(const MapKey& k) const {
    size_t h = std::hash<const void*>()(k.base);
    auto mix = [&h](size_t v) { h ^= v + 0x9e3779b97f4a7c15ull + (h << 6) + (h >> 2); };
    mix((size_t)k.ld); mix((size_t)k.kmajor); mix((size_t)k.rows); mix((size_t)k.K); mix((size_t)k.box_rows);
    return h;
  }
};
std::unordered_map<MapKey, CUtensorMap, MapKeyHash> g_maps;
std::mutex g_maps_lock;
constexpr size_t MAP_CACHE_LIMIT = 1 << 16;
}  // namespace mapcache
using namespace mapcache;

bool encode_map(CUtensorMap* map, const bf16* base, long long ld, bool kmajor, int rows, int K,
                int box_rows, bool transient, int k_rows) {
  const MapKey key{base, ld, kmajor ? 1 : 0, rows, K, box_rows};
  if (!transient) {
    std::lock_guard<std::mutex> lk(g_maps_lock);
    auto it = g_maps.find(key);
    if (it != g_maps.end()) { *map = it->second; return true; }
  }
  // kmajor: memory is [rows, K] (inner = K).  else: memory is [K, rows] (inner = rows).
  cuuint64_t gdim[2];
  cuuint64_t gstride[1] = {(cuuint64_t)ld * 2};
  cuuint32_t box[2];
  cuuint32_t estr[2] = {1, 1};
  if (kmajor) {
    gdim[0] = (cuuint64_t)K; gdim[1] = (cuuint64_t)rows;
    box[0] = BK; box[1] = (cuuint32_t)box_rows;
  } else {
    gdim[0] = (cuuint64_t)rows; gdim[1] = (cuuint64_t)K;
    box[0] = 64; box[1] = (cuuint32_t)k_rows;
  }
  CUresult r = tc::g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, (void*)base, gdim, gstride, box,
                        estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return false;
  if (transient) return true;
  std::lock_guard<std::mutex> lk(g_maps_lock);
  if (g_maps.size() >= MAP_CACHE_LIMIT) g_maps.clear();
  g_maps.emplace(key, *map);
  return true;
}

// launch parameters common to every tile shape (tile counts and split-K are set by the launcher)
TcParams make_params(const GemmArgs& g) {
  TcParams p;
  p.M = g.M; p.N = g.N; p.K = g.K; p.epilogue = g.epilogue;
  p.C = g.C; p.ldc = g.ldc; p.C2 = g.C2; p.aux = g.aux; p.ldaux = g.ldaux; p.flags = g.flags;
  p.a_rows = BM;
  p.k_rows = g.K < BK && !(g.a_kmajor && g.b_kmajor) ? (g.K + UMMA_K - 1) / UMMA_K * UMMA_K : BK;
  p.tiles_m = p.tiles_n = 0; p.tail_from = 1 << 30; p.n_fastest = 0; p.splits = 1; p.split_stride = 0;
  p.C3 = g.C3; p.ldc3 = g.ldc3; p.c3_lo = g.c3_lo; p.c3_hi = g.c3_hi;
  p.piece_scale = g.piece_scale; p.piece_stats = g.piece_stats; p.ld_pieces = g.ld_pieces;
  p.entries = g.entries; p.row_scale = g.row_scale; p.zero_word = g.zero_word; p.dependent = g.transient ? 1 : 0; p.alternate = 0;
  p.rope_S = g.rope_S > 0 ? g.rope_S : 1; p.rope_dh = g.rope_dh > 0 ? g.rope_dh : 2; p.rope_cols = g.rope_cols;
  const bool f32 = g.epilogue == EPI_STORE_F32 || g.epilogue == EPI_RESID_F32;
  const long long out_unit = f32 ? 8 : 16;   // elements per 32 bytes
  bool w = (reinterpret_cast<uintptr_t>(g.C) % 32 == 0) && (g.ldc % out_unit == 0) &&
           (g.split_stride % out_unit == 0);
  if (g.epilogue == EPI_GELU_DUAL) w = w && (reinterpret_cast<uintptr_t>(g.C2) % 32 == 0);
  if (g.epilogue == EPI_RESID_F32) w = w && (reinterpret_cast<uintptr_t>(g.aux) % 32 == 0) && (g.ldaux % 8 == 0);
  if (g.epilogue == EPI_DGELU) w = w && (reinterpret_cast<uintptr_t>(g.aux) % 32 == 0) && (g.ldaux % 16 == 0);
  if (g.epilogue == EPI_DELTA_BF16) w = w && (reinterpret_cast<uintptr_t>(g.aux) % 32 == 0) && (g.ldaux % 16 == 0);
  p.wide = w ? 1 : 0;
  return p;
}
}  // namespace gemm_tc_detail

namespace {
template <int BN, bool A_K, bool B_K, int MODE = DRAIN_COLS>
int launch_t(const GemmArgs& g, cudaStream_t st) {
  using C = Cfg<BN>;
  static PerDeviceFlag attr;
  if (!ppu_set_smem_once(attr, gemm_tc_kernel<BN, A_K, B_K, MODE>, C::SMEM + store_smem<MODE, BN>())) return -1;
  CUtensorMap mapA, mapB;
  TcParams p = make_params(g);
  if (MODE == DRAIN_COLS) p.k_rows = BK;
  else if (A_K && g.M < BM) p.a_rows = (g.M + 7) / 8 * 8;
  if (!encode_map(&mapA, g.A, g.lda, A_K, g.M, g.K, p.a_rows, g.transient, p.k_rows)) return -2;
  if (!encode_map(&mapB, g.B, g.ldb, B_K, g.N, g.K, BN, g.transient, p.k_rows)) return -2;
  p.tiles_m = (g.M + BM - 1) / BM;
  p.tiles_n = (g.N + BN - 1) / BN;
  const int k_blocks = (g.K + BK - 1) / BK;
  p.splits = g.splits < 1 ? 1 : (g.splits > k_blocks ? k_blocks : g.splits);
  p.split_stride = g.split_stride;
  const int tiles = p.tiles_m * p.tiles_n * p.splits;
  const int n_sm = ppu_sm_count();
  const int grid = tiles < n_sm ? tiles : n_sm;
  p.alternate = MODE != DRAIN_COLS && tiles >= 2 * grid;
  constexpr int smem = C::SMEM + store_smem<MODE, BN>();
  if (g.transient)
    return ppu_launch_dependent(gemm_tc_kernel<BN, A_K, B_K, MODE>, grid, gemm_threads(MODE, BN), smem, st, mapA, mapB, Second<MODE>{}, p) == cudaSuccess ? 0 : -3;
  gemm_tc_kernel<BN, A_K, B_K, MODE><<<grid, gemm_threads(MODE, BN), smem, st>>>(mapA, mapB, Second<MODE>{}, p);
  return cudaGetLastError() == cudaSuccess ? 0 : -3;
}

template <int BN>
int launch_bn(const GemmArgs& g, cudaStream_t st) {
  if (g.a_kmajor && g.b_kmajor) return launch_t<BN, true, true>(g, st);
  if (g.a_kmajor && !g.b_kmajor) return launch_t<BN, true, false>(g, st);
  if (!g.a_kmajor && g.b_kmajor) return launch_t<BN, false, true>(g, st);
  return launch_t<BN, false, false>(g, st);
}

}  // namespace

int gemm_tc_init() {
  if (tc::g_encode) return 0;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess ||
      q != cudaDriverEntryPointSuccess || !fn)
    return -1;
  tc::g_encode = (tc::EncodeTiledFn)fn;
  return 0;
}

namespace {
// the SM-pair kernel on 256 x 256 tiles is chosen for this product: from 16 tiles up it is at
// least as fast as one CTA per 128 x 128 tile even though it then leaves SM pairs idle
// (2048 x 2048 x 8192, 64 tiles: 0.053 ms against 0.092; 512 x 2048 x 8192, 16 tiles: equal)
bool picks_pair256(const GemmArgs& g) {
  const long long tiles_pair = (long long)((g.M + 255) / 256) * ((g.N + 255) / 256);
  // (a split product needs as many 128-k blocks as slices, or the pair kernel would write fewer
  // partial outputs than the caller adds up)
  const bool split_ok = g.splits <= 1 || g.splits <= (g.K + 127) / 128;
  return split_ok && (g.tile_shape == 2 || g.tile_shape == 4 ||
                      (g.tile_shape == 0 && g.M > 128 && g.N > 128 && tiles_pair >= 16));
}
}  // namespace

bool gemm_tc_fuses_delta(const GemmArgs& g) {
  // a thread drains 128 consecutive columns of its row in 32-column chunks with 32-byte accesses:
  // heads must be whole multiples of a chunk and must not straddle the 128-column boundary
  GemmArgs probe = g;
  probe.epilogue = EPI_DELTA_BF16;
  const int dh = g.rope_dh;
  return picks_pair256(g) && (dh == 32 || dh == 64 || dh == 128) && g.N % dh == 0 && g.N % 32 == 0 &&
         g.rope_S > 0 && g.M % g.rope_S == 0 && g.aux && g.C3 && gemm_tc_detail::make_params(probe).wide;
}

int launch_gemm_tc(const GemmArgs& g, cudaStream_t st) {
  if (g.M <= 0 || g.N <= 0 || g.K <= 0) return 0;
  if (gemm_tc_init() != 0) return -1;
  if (g.epilogue == EPI_DELTA_BF16 && !gemm_tc_fuses_delta(g)) return -4;
  if ((g.lda % 8) || (g.ldb % 8) || (g.ldc % 8) || (g.N % 8) ||
      (reinterpret_cast<uintptr_t>(g.A) & 15) || (reinterpret_cast<uintptr_t>(g.B) & 15) ||
      (reinterpret_cast<uintptr_t>(g.C) & 15))
    return -4;
  // Wide tiles when the grid still fills the machine; narrow ones for small outputs.
  // SM pairs on 256 x 256 tiles from 16 tiles up when the product is not split.
  // (256 x 128 pair tiles throughout would fill the last wave of the N = 2048 products better -
  // 512 tiles instead of 256 on the 74 pairs of a B200 - but the narrower product measured 25 %
  // slower, so only a half-empty last wave is worked that way, inside the 256-wide kernel;
  // tile_shape 3 keeps the narrow kernel testable, 4 is the 256-wide kernel without narrow units.)
  if (g.splits > 1 && (g.tile_shape == 3 || g.epilogue != EPI_STORE_F32)) return -4;
  if (g.tile_shape == 3) return launch_gemm_tc_pair(g, make_params(g), 128, st);
  if (picks_pair256(g)) return launch_gemm_tc_pair(g, make_params(g), 256, st);
  const long long tiles256 = (long long)((g.M + BM - 1) / BM) * ((g.N + 255) / 256) * (g.splits > 1 ? g.splits : 1);
  if (g.N > 128 && tiles256 >= ppu_sm_count()) return launch_bn<256>(g, st);
  return launch_bn<128>(g, st);
}

namespace {
bool operands_ok(const GemmArgs& g) {
  return !((g.lda % 8) || (g.ldb % 8) || (reinterpret_cast<uintptr_t>(g.A) & 15) || (reinterpret_cast<uintptr_t>(g.B) & 15));
}
}  // namespace

int launch_gemm_tc_pieces(const GemmArgs& g, cudaStream_t st) {
  if (g.M <= 0 || g.N <= 0 || g.K <= 0) return 0;
  if (gemm_tc_init() != 0) return -1;
  if (!operands_ok(g) || !g.a_kmajor || !g.b_kmajor || g.splits > 1 || !g.piece_stats ||
      (g.C && ((g.ldc % PIECE) || (reinterpret_cast<uintptr_t>(g.C) & 31))))
    return -4;
  const TcParams p = make_params(g);
  if (picks_pair256(g)) return launch_gemm_tc_pair_pieces(g, p, st);
  const long long tiles256 = (long long)((g.M + BM - 1) / BM) * ((g.N + 255) / 256);
  if (g.N > 128 && tiles256 >= ppu_sm_count()) return launch_t<256, true, true, DRAIN_PIECES>(g, st);
  return launch_t<128, true, true, DRAIN_PIECES>(g, st);
}

bool gemm_tc_pairs_two(const GemmArgs& g, const GemmArgs* g2) {
  // SM pairs where neither product is narrower than a tile half and there are 16 units or more between them
  const GemmArgs& h = g2 ? *g2 : g;
  const long long tiles = (long long)((g.M + 255) / 256) * ((g.N + 255) / 256) + (g2 ? (long long)((h.M + 255) / 256) * ((h.N + 255) / 256) : 0);
  return g.M > 128 && g.N > 128 && h.M > 128 && h.N > 128 && tiles >= 16;
}

namespace {
int one_units(const GemmArgs& g, TcParams& p) {
  p = make_params(g);
  if (g.a_kmajor && g.M < BM) p.a_rows = (g.M + 7) / 8 * 8;
  p.tiles_m = (g.M + BM - 1) / BM;
  p.tiles_n = (g.N + 127) / 128;
  const int k_blocks = (g.K + BK - 1) / BK;
  p.splits = g.splits < 1 ? 1 : (g.splits > k_blocks ? k_blocks : g.splits);
  p.split_stride = g.split_stride;
  return p.tiles_m * p.tiles_n * p.splits;
}
bool two_ok(const GemmArgs& g) {
  const bool f32 = g.epilogue == EPI_STORE_F32 || g.epilogue == EPI_RESID_F32;
  return operands_ok(g) && g.transient && !g.b_kmajor && (f32 || g.epilogue == EPI_OUT_BF16) && (g.splits <= 1 || g.epilogue == EPI_STORE_F32) &&
         !(g.N % 8) && !(g.ldc % 8) && !(g.aux && (g.ldaux % 8)) && !(reinterpret_cast<uintptr_t>(g.C) & (f32 ? 31 : 15)) &&
         !(reinterpret_cast<uintptr_t>(g.aux) & 31) && g.M > 0 && g.N > 0 && g.K > 0;
}
}  // namespace

int launch_gemm_tc_two(const GemmArgs& g, const GemmArgs* g2, cudaStream_t st) {
  if (gemm_tc_init() != 0) return -1;
  if (!two_ok(g) || (g2 && !two_ok(*g2))) return -4;
  // the product with the longer units first
  const int k1 = g.K / (g.splits > 1 ? g.splits : 1), k2 = g2 ? g2->K / (g2->splits > 1 ? g2->splits : 1) : 0;
  if (k2 > k1) return launch_gemm_tc_two(*g2, &g, st);
  if (gemm_tc_pairs_two(g, g2)) return launch_gemm_tc_pair_two(g, g2, st);
  using C = Cfg<128>;
  static PerDeviceFlag attr;
  constexpr int smem = C::SMEM + store_smem<DRAIN_TWO, 128>();
  auto kernel = gemm_tc_kernel<128, true, false, DRAIN_TWO>;
  if (!ppu_set_smem_once(attr, kernel, smem)) return -1;
  CUtensorMap mapA, mapB;
  Second<DRAIN_TWO> m = {};
  TcParams p;
  m.units = one_units(g, p);
  m.a_k = g.a_kmajor;
  if (!encode_map(&mapA, g.A, g.lda, g.a_kmajor, g.M, g.K, p.a_rows, true, p.k_rows)) return -2;
  if (!encode_map(&mapB, g.B, g.ldb, false, g.N, g.K, 128, true, p.k_rows)) return -2;
  if (g2) {
    m.units2 = one_units(*g2, m.p);
    m.a_k2 = g2->a_kmajor;
    if (!encode_map(&m.a, g2->A, g2->lda, g2->a_kmajor, g2->M, g2->K, m.p.a_rows, true, m.p.k_rows)) return -2;
    if (!encode_map(&m.b, g2->B, g2->ldb, false, g2->N, g2->K, 128, true, m.p.k_rows)) return -2;
  }
  m.fill = g2 ? two_fill(g, *g2, 190) : 0;
  const int units = m.units + m.units2, n_sm = ppu_sm_count();
  p.alternate = units >= 2 * n_sm;
  return ppu_launch_dependent(kernel, units < n_sm ? units : n_sm, gemm_threads(DRAIN_TWO, 128), smem, st, mapA, mapB, m, p) == cudaSuccess ? 0 : -3;
}
