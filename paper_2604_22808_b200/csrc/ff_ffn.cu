// The gated feed-forward block, forward and backward, bf16 with fp32 accumulation:
//   G = X Wg, U = X Wu, H = act(G) * U, out = H Wd                                      X [M][D], Wg, Wu [D][F], Wd [F][D]
//   dH = dout Wd^T, dG = dH U act'(G), dU = dH act(G), dX = dG Wg^T + dU Wu^T,
//   dWg = X^T dG, dWu = X^T dU, dWd = H^T dout
//
// One kernel makes all products: forward in two launches (gate and up; out), backward in two (dH; all gradients together), and where K
// was cut a small one joins the parts.  It is a persistent GEMM on CTA pairs (tcgen05, cta_group::2) with tiles of 256 x 256 (128 rows of
// A and 128 columns of B in either CTA's shared memory), K in chunks of 64, a ring of six stages filled by TMA, and two accumulators of
// 256 tensor-memory columns, so that the epilogue of a tile overlaps the main loop of the next.  Operands are read as they lie in memory,
// K-major or MN-major, so nothing is transposed.
//   gate and up   one tile is 128 columns of G (the even CTA's half of B) beside the same 128 columns of U (the odd CTA's), so
//                 that both values of an element lie in one lane of tensor memory and H leaves without G and U reaching memory
//   dH            its epilogue reads G and U and writes dG, dU and H (needed for dWd; made again rather than kept)
//   gradients     dX, dWg and dWu, dWd in one launch, whose items go to the pairs one after another (in a launch each: 4000 tokens, dim
//                 1024, hidden 2816 150 us instead of 124, 64 tokens 35 instead of 24); dX: K runs over the columns of dG, then those of
//                 dU;  dWg, dWu: the matrices side by side along N, K runs over the tokens
// H, dG and dU are rounded to bf16 between the products: they are operands of the next one.
// Products with few tiles are cut along K (split_of, splits_of); with few tokens the weights are the rows (ffn_few_kernel).
//
//   warp 0      TMA producer          warp 1      tcgen05.mma issuer of the pair (even CTA), owns the tensor memory
//   warps 2..9  epilogue: a thread owns one row of the tile and half its columns, which reach memory by TMA from a staging area of
//               the warp (stored from registers, every thread a row of its own, dH took 343 us instead of 266, G and U kept 141
//               instead of 111)
#include <cuda.h>
#include <stdio.h>

#include <initializer_list>
#include <new>

#include "ff_internal.h"
#include "ff_sm100.cuh"

using namespace sm100;

struct ff_ffn {
  ff_ffn_config_t cfg;
  int device, sm_count;
  int room[2][2][9];       // few-token kernel: blocks that run at the same time, [matrices - 1][tiles of 128 tokens][blocks of a cluster]
  int* status;             // device status word (plan-like: raised by an expired wait)
  mutable FFMapCache maps; // tensor maps by matrix and box; every use puts in its address
  char err[512];
};

namespace {

constexpr int TM = 256, TN = 256, TK = 64;     // (a narrow tile: 128 columns)
constexpr int PIECE = 64 * 128;                  // 64 rows of 128 bytes
constexpr int OPERAND = 2 * PIECE;               // one CTA's 128 rows (or columns) of a K chunk
__host__ __device__ constexpr int stage_bytes(int nt) { return OPERAND + nt / 2 * 128; }
constexpr int EPI_WARPS = 8;
constexpr int THREADS = 64 + 32 * EPI_WARPS;

enum { PRODUCTS = 0, GATE = 1, DGATE = 2 };      // what a launch makes
// Stages of the ring, and staging areas of an epilogue warp: 32 rows of 64 columns each, on their way to or from memory by TMA
constexpr int AREA = 32 * 128;
__host__ __device__ constexpr int ring_stages(int epi) { return epi == DGATE ? 5 : 6; }
__host__ __device__ constexpr int areas(int epi) { return epi == DGATE ? 2 : 1; }

// One product of a launch.
struct Sub {
  long long rows;                  // output rows
  int cols;                        // output columns of one matrix
  int m_tiles, n_tiles, mats;      // tiles; matrices side by side
  int kchunks, sources;            // K chunks of one source, sources one after the other
  int split;                       // parts of K; more than one: each with its own fp32 sums
  int items;                       // tiles times parts
  int a_mn, b_mn;                  // operands MN-major
  int a, b, e;                     // its first maps
};
struct GemmParams {
  Sub sub[3];
  int items, act, keep;            // keep: GATE writes G and U too
  int* status;
};
// Operands by source (K) or matrix (N), and what the epilogue moves: PRODUCTS: the outputs by matrix, or the sums [matrix][part][rows][cols];
// GATE: H, G, U;  DGATE: G, U (read), dG, dU, H
struct GemmMaps { CUtensorMap a[4], b[5], e[5]; };

struct Shared {
  uint64_t full[6], empty[6], acc_full[2], acc_empty[2], in_full[EPI_WARPS];
  uint32_t tmem_base;
  int abort_flag;
};
inline int chunks(long long k) { return (int)((k + TK - 1) / TK); }
__host__ __device__ constexpr size_t smem_bytes(int epi, int nt = TN) { return (size_t)ring_stages(epi) * stage_bytes(nt) + (size_t)EPI_WARPS * areas(epi) * AREA + sizeof(Shared) + 1024; }
static_assert(smem_bytes(PRODUCTS) <= 232448 && smem_bytes(GATE) <= 232448 && smem_bytes(DGATE) <= 232448, "227 KB a block");

// act(g) and, with SLOPE, its derivative.  The cubic inside gelu_tanh saturates long before |g| = 16.
__device__ __forceinline__ float exponential(float v) { return ex2(1.4426950408889634f * v); }
__device__ __forceinline__ float sigmoid(float v) { return rcp(1.f + exponential(-v)); }
template <int ACT, bool SLOPE>
__device__ __forceinline__ float activation(float g, float* slope) {
  if constexpr (ACT == FF_ACT_SILU) {
    const float s = sigmoid(g);
    if (SLOPE) *slope = s * (1.f + g * (1.f - s));
    return g * s;
  } else if constexpr (ACT == FF_ACT_GELU_TANH) {
    const float c = 1.5957691216057308f;         // 2 sqrt(2 / pi)
    const float t = g != g ? g : fminf(fmaxf(g, -16.f), 16.f), t2 = t * t;
    const float s = sigmoid(c * t * (1.f + 0.044715f * t2));
    if (SLOPE) *slope = s + t * s * (1.f - s) * c * (1.f + 0.134145f * t2);
    return g * s;
  } else {
    // 1 - Phi(|g|) = e^(-x^2) (a1 t + .. + a5 t^5) / 2, x = |g| / sqrt 2, t = 1 / (1 + 0.3275911 x), to 0.75e-7: Abramowitz and
    // Stegun, "Handbook of Mathematical Functions", 7.1.26.  Relative to 1 - Phi that is 5e-4 at |g| = 4, 1.6e-3 at 5 and 3.6e-3 at 6,
    // below half a step of bf16 (3.9e-3) where the result is above 1e-9 g.  Its exponential is the one of the derivative.  (With erfcf the launches
    // of dH and dWd took 276 us instead of 249: 16384 tokens, dim and hidden 2048.)
    const float x = 0.70710678118654752f * fabsf(g), t = rcp(fmaf(0.3275911f, x, 1.f)), e = exponential(-x * x);
    const float h = 0.5f * e * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    const float p = g < 0.f ? h : 1.f - h;
    if (SLOPE) *slope = p + fminf(fmaxf(g, -32.f), 32.f) * 0.3989422804014327f * e;
    return g * p;
  }
}
// body(constant) with the configuration's activation as a compile-time constant: chosen once for many elements, whose
// instructions then overlap (chosen for each of them, the launch of dH took 266 us instead of 221: 9999 tokens, dim 2048, hidden 5632)
template <int ACT> struct Act { static constexpr int value = ACT; };
template <class Body>
__device__ __forceinline__ void with_activation(int act, Body body) {
  if (act == FF_ACT_SILU) body(Act<FF_ACT_SILU>());
  else if (act == FF_ACT_GELU_TANH) body(Act<FF_ACT_GELU_TANH>());
  else body(Act<FF_ACT_GELU>());
}

template <int N>
__device__ __forceinline__ void pack(const float (&v)[N], uint32_t* w) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) w[i] = bf16_pair(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]));
}
// A lane's row of a staging area: pieces of 16 bytes in the order of the 128-byte swizzle.  `half` selects 32 of the 64 columns.
__device__ __forceinline__ void stage32(uint8_t* area, int lane, int half, const uint32_t* w) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *(uint4*)(area + lane * 128 + (((half * 4 + j) ^ (lane & 7)) * 16)) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
}
__device__ __forceinline__ void stage32(uint8_t* area, int lane, int half, const float (&v)[32]) {
  uint32_t w[16];
  pack(v, w);
  stage32(area, lane, half, w);
}
template <int N>
__device__ __forceinline__ float element(const uint4 (&v)[N], int i) {
  const uint32_t w = ((const uint32_t*)v)[i >> 1];
  return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
}

// Work item t: a tile and its part of K.  The tiles of up to eight rows of tiles follow one another column by column, so that
// what runs at the same time reads few rows of A and few columns of B (row by row, dWg and dWu of dim 2048, hidden 5632, 9999
// tokens read dG and dU from memory in each of five waves: 420 us in a row of calls, 372 column by column).
struct Item { int m, n, mat, part; };
__device__ __forceinline__ Item item_of(const Sub& P, int t) {
  const int cols = P.n_tiles * P.mats, tiles = P.m_tiles * cols;
  Item w;
  w.part = P.split > 1 ? t / tiles : 0;
  t -= w.part * tiles;
  const int band = t / (8 * cols), height = min(8, P.m_tiles - band * 8);
  const int r = t - band * 8 * cols, c = r / height;
  w.m = band * 8 + r - c * height;
  w.mat = P.mats > 1 && c >= P.n_tiles;
  w.n = c - w.mat * P.n_tiles;
  return w;
}
// The product of item t of the launch; t becomes the item of the product.
template <int EPI>
__device__ __forceinline__ const Sub& sub_of(const GemmParams& P, int& t) {
  const Sub* s = P.sub;
  if (EPI == PRODUCTS)
    for (; t >= s->items; ++s) t -= s->items;
  return *s;
}
// K chunks of a part
__device__ __forceinline__ void part_of_k(const Sub& P, int part, int& begin, int& end) {
  const int k = P.kchunks * P.sources, q = k / P.split, r = k - q * P.split;         // (the first r parts have one more)
  begin = part * q + min(part, r);
  end = begin + q + (part < r);
}

template <bool V> struct Const { static constexpr bool value = V; };
// A_MN, B_MN: the operands' majorness; of PRODUCTS each product says its own: both MN-major, B alone, or neither, the
// one case with two sources.
template <bool A_MN, bool B_MN, int EPI, int NT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
ffn_gemm_kernel(const __grid_constant__ GemmMaps maps, const GemmParams P) {
  constexpr int NSTAGE = ring_stages(EPI), AREAS = areas(EPI), STAGE = stage_bytes(NT);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  Shared& sh = *(Shared*)(smem + NSTAGE * STAGE + EPI_WARPS * AREAS * AREA);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (threadIdx.x < 14) tma_prefetch_desc(&maps.a[0] + threadIdx.x);
  if (threadIdx.x == 0) {
    for (int i = 0; i < NSTAGE; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.acc_full[i], 1); mbar_init(&sh.acc_empty[i], 2 * EPI_WARPS); }
    for (int i = 0; i < EPI_WARPS; ++i) mbar_init(&sh.in_full[i], 1);
    sh.abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) { tmem_alloc_pair(&sh.tmem_base, 2 * NT); tmem_relinquish_pair(); }
  tc_fence_before();
  __syncthreads();
  cluster_sync();                                               // the other CTA's barriers are there
  tc_fence_after();
  ff_pdl_wait();
  const uint32_t tm = sh.tmem_base;
  volatile int* abort_flag = &sh.abort_flag;

  if (warp == 0) {
    if (lane == 0) {
      unsigned n = 0;
      bool ok = true;
      for (int i = pair; i < P.items && ok; i += pairs) {
        int t = i;
        const Sub sub = sub_of<EPI>(P, t);                      // (a copy: read once an item, not once a chunk)
        const Item w = item_of(sub, t);
        const int m0 = w.m * TM + (int)rank * 128;
        const int n0 = EPI == GATE ? w.n * (NT / 2) : w.n * NT + (int)rank * (NT / 2);
        int k_begin, k_end;
        part_of_k(sub, w.part, k_begin, k_end);
        // (a loop for each majorness, here and at the products: with it as a variable the product with Wd took 15 % more)
        auto load = [&](auto a_mn, auto b_mn, const CUtensorMap* ma, const CUtensorMap* mb, int from, int to, int first) {
          for (int kc = from; kc < to && ok; ++kc, ++n) {
            const int slot = n % NSTAGE, k0 = (kc - first) * TK;
            if (n >= (unsigned)NSTAGE) ok = mbar_wait(&sh.empty[slot], ((n / NSTAGE) - 1) & 1, abort_flag);
            if (!ok) break;
            uint8_t* dst = smem + slot * STAGE;
            const uint32_t bar = map_shared(&sh.full[slot], 0);
            if (rank == 0) mbar_arrive_expect_tx(&sh.full[slot], 2 * STAGE);
            if constexpr (decltype(a_mn)::value) {
              tma_load_3d_pair(dst, ma, bar, m0, k0, 0);
              tma_load_3d_pair(dst + PIECE, ma, bar, m0 + 64, k0, 0);
            } else {
              tma_load_3d_pair(dst, ma, bar, k0, m0, 0);
            }
            if constexpr (decltype(b_mn)::value) {
              tma_load_3d_pair(dst + OPERAND, mb, bar, n0, k0, 0);
              if (NT == 256) tma_load_3d_pair(dst + OPERAND + PIECE, mb, bar, n0 + 64, k0, 0);
            } else {
              tma_load_3d_pair(dst + OPERAND, mb, bar, k0, n0, 0);
            }
          }
        };
        const CUtensorMap *ma = &maps.a[sub.a], *mb = &maps.b[EPI == GATE ? (int)rank : sub.b + w.mat];
        if constexpr (EPI != PRODUCTS) {
          load(Const<A_MN>(), Const<B_MN>(), ma, mb, k_begin, k_end, 0);
        } else if (sub.a_mn) {
          load(Const<true>(), Const<true>(), ma, mb, k_begin, k_end, 0);
        } else if (sub.b_mn) {
          load(Const<false>(), Const<true>(), ma, mb, k_begin, k_end, 0);
        } else {                                                // the one with two sources
          load(Const<false>(), Const<false>(), ma, mb, k_begin, min(k_end, sub.kchunks), 0);
          load(Const<false>(), Const<false>(), ma + 1, mb + 1, max(k_begin, sub.kchunks), k_end, sub.kchunks);
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      unsigned n = 0, nt = 0;
      bool ok = true;
      for (int i = pair; i < P.items && ok; i += pairs, ++nt) {
        const int ab = nt & 1;
        int t = i, k_begin, k_end;
        const Sub sub = sub_of<EPI>(P, t);                      // (a copy: read once an item, not once a chunk)
        part_of_k(sub, sub.split > 1 ? t / (sub.m_tiles * sub.n_tiles * sub.mats) : 0, k_begin, k_end);
        if (nt >= 2) ok = mbar_wait_warp(&sh.acc_empty[ab], ((nt >> 1) - 1) & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        auto multiply = [&](auto a_mn, auto b_mn) {
          constexpr bool AM = decltype(a_mn)::value, BM = decltype(b_mn)::value;
          constexpr uint32_t idesc = idesc_bf16_f32(TM, NT, AM, BM);
          constexpr uint64_t A_STEP = AM ? 128 : 2, B_STEP = BM ? 128 : 2;      // 16 K elements on, in units of 16 bytes
          const uint64_t a0 = smem_desc_sw128(smem_u32(smem), AM ? PIECE : 16, 1024);
          const uint64_t b0 = smem_desc_sw128(smem_u32(smem) + OPERAND, BM ? PIECE : 16, 1024);
          for (int kc = k_begin; kc < k_end && ok; ++kc, ++n) {
            const int slot = n % NSTAGE;
            ok = mbar_wait_warp(&sh.full[slot], (n / NSTAGE) & 1, abort_flag);
            if (!ok) break;
            tc_fence_after();
            const uint64_t at = (uint64_t)(slot * (STAGE >> 4));
#pragma unroll
            for (int ks = 0; ks < TK / 16; ++ks)
              umma_ss_pair(tm + ab * NT, a0 + at + ks * A_STEP, b0 + at + ks * B_STEP, idesc, ks > 0 ? 1u : (kc > k_begin ? 1u : 0u));
            umma_commit_pair(&sh.empty[slot]);
          }
        };
        if constexpr (EPI != PRODUCTS) multiply(Const<A_MN>(), Const<B_MN>());
        else if (sub.a_mn) multiply(Const<true>(), Const<true>());
        else if (sub.b_mn) multiply(Const<false>(), Const<true>());
        else multiply(Const<false>(), Const<false>());
        if (!ok) break;
        umma_commit_pair(&sh.acc_full[ab]);
      }
    }
  } else {
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
    uint8_t* area = smem + NSTAGE * STAGE + (warp - 2) * AREAS * AREA;
    uint64_t* in_full = &sh.in_full[warp - 2];
    unsigned nt = 0, loads = 0;
    bool ok = true;
    // The warp's rows of one output, 64 columns of them, from `values` by way of a staging area.
    auto put = [&](const CUtensorMap* map, uint8_t* to, int col, int row, auto values, auto read) {
      if (lane == 0) bulk_wait_read0();                         // (the area's last store has read it)
      __syncwarp();
#pragma unroll 1
      for (int q = 0; q < 2; ++q) {
        float v[32];
        values(q, v);
        if (q) read();
        stage32(to, lane, q, v);
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) { tma_store_3d(to, map, col, row, 0); bulk_commit(); }
    };
    for (int i = pair; i < P.items && ok; i += pairs, ++nt) {
      int t = i;
      const Sub sub = sub_of<EPI>(P, t);                      // (a copy: read once an item, not once a chunk)
      const Item w = item_of(sub, t);
      const int ab = nt & 1;
      const int row = w.m * TM + (int)rank * 128 + quarter * 32;
      const uint32_t acc = tm + lane_addr + ab * NT;
      // Columns of the warp.  Of a narrow tile's 64 hidden columns H is the first half's warps', G and U the second's.
      constexpr bool SHARED = EPI == GATE && NT == 128;
      constexpr int WIDTH = EPI == GATE ? 64 : NT / 2;
      const int at0 = SHARED ? 0 : half * WIDTH, c0 = SHARED ? w.n * WIDTH : w.n * (2 * WIDTH) + at0;
      const bool rows = row < sub.rows;
      auto get = [&](int col) {                                 // DGATE: G and U of 64 columns into the first two areas
        if (lane == 0) {
          bulk_wait_read0();
          mbar_arrive_expect_tx(in_full, 2 * AREA);
          tma_load_3d(area, &maps.e[0], in_full, col, row, 0);
          tma_load_3d(area + AREA, &maps.e[1], in_full, col, row, 0);
        }
      };
      if (EPI == DGATE && rows && c0 < sub.cols) {                // (on their way before the accumulator is complete)
        get(c0);
        if (WIDTH > 64 && lane == 0 && c0 + 64 < sub.cols) {
          tma_prefetch_3d(&maps.e[0], c0 + 64, row, 0);
          tma_prefetch_3d(&maps.e[1], c0 + 64, row, 0);
        }
      }
      ok = __all_sync(0xffffffffu, mbar_wait(&sh.acc_full[ab], (nt >> 1) & 1, abort_flag));
      if (!ok) break;
      tc_fence_after();
      auto release = [&] {                                      // the warp has read its part of the accumulator
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(map_shared(&sh.acc_empty[ab], 0));
      };
      const int parts = rows && !(SHARED && half && !P.keep) ? min(WIDTH, (sub.cols - c0 + 63) / 64 * 64) : 0;
      if (parts <= 0) release();
#pragma unroll 1
      for (int s = 0; s < parts; s += 64) {
        const int col = c0 + s;
        const uint32_t at = acc + at0 + s;
        const bool last = s + 64 >= parts;
        auto done = [&] { if (last) release(); };
        auto more = [] {};
        auto sums = [&](uint32_t from) {
          return [=](int q, float (&v)[32]) {
            uint32_t r[32];
            tmem_ld32(from + q * 32, r);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
          };
        };
        if (EPI == PRODUCTS && sub.split == 1) {
          put(&maps.e[sub.e + w.mat], area, col, row, sums(at), done);
        } else if (EPI == PRODUCTS) {
#pragma unroll 1
          for (int q = 0; q < 2; ++q) {                         // 32 columns of fp32 fill a row of the area
            uint32_t r[32];
            tmem_ld32(at + q * 32, r);
            tmem_wait_ld();
            if (q) done();
            if (lane == 0) bulk_wait_read0();
            __syncwarp();
            stage32(area, lane, 0, r);
            stage32(area, lane, 1, r + 16);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0 && col + q * 32 < sub.cols) { tma_store_3d(area, &maps.e[sub.e], col + q * 32, row, w.mat * sub.split + w.part); bulk_commit(); }
          }
        } else if (EPI == GATE) {
          if (P.keep && (!SHARED || half)) {                    // for the backward pass
            put(&maps.e[1], area, col, row, sums(at), more);
            if (SHARED) put(&maps.e[2], area, col, row, sums(at + NT / 2), done);
            else put(&maps.e[2], area, col, row, sums(at + NT / 2), more);
          }
          if (SHARED && half) break;
          put(&maps.e[0], area, col, row, [&](int q, float (&v)[32]) {
            uint32_t g[32], u[32];
            tmem_ld32(at + q * 32, g);
            tmem_ld32(at + NT / 2 + q * 32, u);
            tmem_wait_ld();
            with_activation(P.act, [&](auto act) {
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = activation<act.value, false>(__uint_as_float(g[i]), nullptr) * __uint_as_float(u[i]);
            });
          }, done);
        } else {
          if (s) get(col);
          ok = __all_sync(0xffffffffu, mbar_wait(in_full, loads++ & 1, abort_flag));
          if (!ok) break;
          // The gradients take the places of what they are made from, H that of dG once it has left.
          uint32_t hid[32];
#pragma unroll
          for (int q = 0; q < 4; ++q) {                         // 16 columns: two pieces of a row
            uint32_t d[16];
            tmem_ld16(at + q * 16, d);
            uint4* const p[2] = {(uint4*)(area + lane * 128 + (((2 * q) ^ (lane & 7)) * 16)), (uint4*)(area + lane * 128 + (((2 * q + 1) ^ (lane & 7)) * 16))};
            const uint4 g[2] = {*p[0], *p[1]}, u[2] = {p[0][AREA / 16], p[1][AREA / 16]};
            tmem_wait_ld();
            if (q == 3 && last) release();
            float dg[16], du[16], h[16];
            with_activation(P.act, [&](auto act) {
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float dh = __uint_as_float(d[i]), up = element(u, i);
                float slope;
                const float a = activation<act.value, true>(element(g, i), &slope);
                dg[i] = dh * up * slope; du[i] = dh * a; h[i] = a * up;
              }
            });
            uint32_t w0[8], w1[8];
            pack(dg, w0); pack(du, w1); pack(h, hid + 8 * q);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              *p[j] = make_uint4(w0[4 * j], w0[4 * j + 1], w0[4 * j + 2], w0[4 * j + 3]);
              p[j][AREA / 16] = make_uint4(w1[4 * j], w1[4 * j + 1], w1[4 * j + 2], w1[4 * j + 3]);
            }
          }
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            tma_store_3d(area, &maps.e[2], col, row, 0);
            bulk_commit();
            tma_store_3d(area + AREA, &maps.e[3], col, row, 0);
            bulk_commit();
            bulk_wait_read1();                                  // (the first of the two has read its area)
          }
          __syncwarp();
          stage32(area, lane, 0, hid);
          stage32(area, lane, 1, hid + 16);
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) { tma_store_3d(area, &maps.e[4], col, row, 0); bulk_commit(); }
        }
      }
    }
    if (lane == 0) bulk_wait0();
  }

  tc_fence_before();
  __syncthreads();
  if (sh.abort_flag) {
    if (threadIdx.x == 0) atomicExch(P.status, FF_ERR_TIMEOUT | 0xa00);   // low byte: status, next byte: which kernel
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000) { }
    __syncthreads();
  }
  cluster_sync();                                               // neither CTA leaves while the other still reads or signals it
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tm, 2 * NT);
  }
}

// The parts of K added up, in their order, and rounded.  A block has 2048 values of one output, a thread eight.
struct Joined { const float* sums; __nv_bfloat16* out; long long values; int split, first; };     // first: its first block
struct JoinParams { Joined j[4]; int count; };
__global__ void __launch_bounds__(256) ffn_join_kernel(const JoinParams P) {
  int n = 0;
  while (n + 1 < P.count && (int)blockIdx.x >= P.j[n + 1].first) ++n;
  const Joined& j = P.j[n];
  ff_pdl_wait();
  const long long i = ((long long)((int)blockIdx.x - j.first) * 256 + threadIdx.x) * 8;
  if (i >= j.values) return;
  const float* p = j.sums + i;
  float v[8] = {};
#pragma unroll 4
  for (int s = 0; s < j.split; ++s) {
    const float4 a = *(const float4*)(p + s * j.values), b = *(const float4*)(p + s * j.values + 4);
    v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
    v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
  }
  uint32_t w[4];
  pack(v, w);
  *(uint4*)(j.out + i) = make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- few tokens -----------------------------------------------------------------------------------------------------------
// With few tokens the products are as long as their weights take to arrive, and tiles of 256 tokens leave most of the device
// idle (one token, dim 2048: eight tiles for the product with Wd).  Here the weights are the A operand, read as they lie
// (MN-major): 128 features are the rows of the accumulator, and the tokens (16 .. 128 of them) its columns.  K is split over a
// cluster of up to eight CTAs, so that about every SM streams its own part of the weights; the partial sums meet in shared memory,
// where every CTA of the cluster adds up a part of the tile, in the order of the ranks: the same bits in every call.
//   GATE   128 features of Wg and the same of Wu beside each other, two accumulators
//   STORE  (the product with Wd) starts while the launch before it, of the same call, still runs: that one writes nothing of
//          Wd, and had itself waited for everything before it; so the first stages of weights are requested ahead of the wait
constexpr size_t FEW_SMEM = 193 * 1024;
constexpr int FEW_THREADS = 64 + 32 * EPI_WARPS;
struct FewParams {
  int tokens, cols, kchunks;       // tokens; features in all; K chunks
  int nt, stages, stage_bytes;     // tokens of a tile; ring
  int act;
  __nv_bfloat16* out[3];           // STORE: out;  GATE: H, G or NULL, U
  int* status;
};
struct FewShared {
  uint64_t full[8], empty[8], done;
  uint32_t tmem_base;
  int abort_flag;
};
__device__ __forceinline__ float4 load_cluster(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void add4(float (&v)[4], const float4& a) { v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; }
__device__ __forceinline__ void store4(__nv_bfloat16* dst, const float (&v)[4]) {
  *(uint2*)dst = make_uint2(bf16_pair(__float_as_uint(v[0]), __float_as_uint(v[1])), bf16_pair(__float_as_uint(v[2]), __float_as_uint(v[3])));
}

template <int EPI>
__global__ void __launch_bounds__(FEW_THREADS, 1)
ffn_few_kernel(const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1,
               const __grid_constant__ CUtensorMap map_x, const FewParams P) {
  constexpr int MATS = EPI == GATE ? 2 : 1;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  __shared__ FewShared sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_rank(), split = (int)cluster_size();
  const int f0 = (int)(blockIdx.x / split) * 128, t0 = (int)blockIdx.y * P.nt;
  const int k_begin = (int)((long long)P.kchunks * rank / split), k_end = (int)((long long)P.kchunks * (rank + 1) / split);
  const uint32_t columns = MATS * P.nt < 32 ? 32 : MATS * P.nt;

  if (threadIdx.x == 32) {
    tma_prefetch_desc(&map_w0); tma_prefetch_desc(&map_x);
    if (EPI == GATE) tma_prefetch_desc(&map_w1);
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < P.stages; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
    mbar_init(&sh.done, 1);
    sh.abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) { tmem_alloc(&sh.tmem_base, columns); tmem_relinquish(); }
  if (EPI == GATE) ff_pdl_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (EPI == PRODUCTS && warp != 0) ff_pdl_wait();                 // (warp 0: below)
  const uint32_t tm = sh.tmem_base;
  volatile int* abort_flag = &sh.abort_flag;

  if (warp == 0) {
    if (lane == 0) {
      auto weights = [&](int kc, int slot) {
        uint8_t* dst = smem + slot * P.stage_bytes;
        mbar_arrive_expect_tx(&sh.full[slot], P.stage_bytes);
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
          for (int c = 0; c < 2; ++c)
            tma_load_3d(dst + (2 * m + c) * PIECE, m ? &map_w1 : &map_w0, &sh.full[slot], f0 + 64 * c, kc * TK, 0);
      };
      int ahead = 0;
      if (EPI == PRODUCTS) {
        for (; ahead < P.stages && k_begin + ahead < k_end; ++ahead) weights(k_begin + ahead, ahead);
        ff_pdl_wait();
      }
      bool ok = true;
      int slot = 0;
      unsigned phase = 1;                                       // (a slot's first use waits for nothing)
      for (int kc = k_begin, n = 0; kc < k_end && ok; ++kc, ++n) {
        if (n >= P.stages) ok = mbar_wait(&sh.empty[slot], phase, abort_flag);
        if (!ok) break;
        if (n >= ahead) weights(kc, slot);
        tma_load_3d(smem + slot * P.stage_bytes + 2 * MATS * PIECE, &map_x, &sh.full[slot], kc * TK, t0, 0);
        if (++slot == P.stages) { slot = 0; phase ^= 1; }
      }
    }
  } else if (warp == 1) {
    const uint32_t idesc = idesc_bf16_f32(128, P.nt, true, false);
    const uint64_t a0 = smem_desc_sw128(smem_u32(smem), PIECE, 1024), b0 = smem_desc_sw128(smem_u32(smem) + 2 * MATS * PIECE, 16, 1024);
    bool ok = true;
    int slot = 0;
    unsigned phase = 0;
    for (int kc = k_begin; kc < k_end && ok; ++kc) {
      ok = mbar_wait_warp(&sh.full[slot], phase, abort_flag);
      if (!ok) break;
      tc_fence_after();
      const uint64_t at = (uint64_t)(slot * (P.stage_bytes >> 4));
#pragma unroll
      for (int ks = 0; ks < TK / 16; ++ks)
#pragma unroll
        for (int m = 0; m < MATS; ++m)
          umma_ss(tm + m * P.nt, a0 + at + (uint64_t)(m * (2 * PIECE >> 4) + ks * 128), b0 + at + (uint64_t)(ks * 2), idesc, ks > 0 ? 1u : (kc > k_begin ? 1u : 0u));
      umma_commit(&sh.empty[slot]);
      if (++slot == P.stages) { slot = 0; phase ^= 1; }
    }
    umma_commit(&sh.done);
  }

  // partial sums [MATS][token][128 features] over the ring, whose last stage the tensor core has read
  float* part = (float*)smem;
  const int live = min(P.nt, P.tokens - t0);
  if (warp >= 2) {
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    const bool ok = __all_sync(0xffffffffu, mbar_wait(&sh.done, 0, abort_flag));
    if (ok) {
      tc_fence_after();
#pragma unroll 1
      for (int m = 0; m < MATS; ++m)
#pragma unroll 1
        for (int c = 16 * half; c < live; c += 32) {
          uint32_t r[16];
          tmem_ld16(tm + ((uint32_t)(quarter * 32) << 16) + m * P.nt + c, r);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; ++i) part[(m * P.nt + c + i) * 128 + quarter * 32 + lane] = __uint_as_float(r[i]);
        }
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  if (!sh.abort_flag) {
    // a warp's share: 128 features of one token, four a lane; the CTAs of the cluster take the tokens in turns
    for (int i = (warp * split + rank) * 32 + lane; i < live * 32; i += split * FEW_THREADS) {
      const int token = i >> 5, fg = (i & 31) * 4;
      if (f0 + fg >= P.cols) continue;
      float g[4] = {}, u[4] = {};
      for (int r0 = 0; r0 < split; r0 += 4) {                   // four CTAs' values are on their way together
        float4 a[4][MATS];
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (r0 + r < split) {
            const uint32_t at = map_shared(part + token * 128 + fg, r0 + r);
#pragma unroll
            for (int m = 0; m < MATS; ++m) a[r][m] = load_cluster(at + (uint32_t)(m * P.nt * 512));
          }
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (r0 + r < split) {
            add4(g, a[r][0]);
            if constexpr (EPI == GATE) add4(u, a[r][1]);
          }
      }
      const size_t to = (size_t)(t0 + token) * P.cols + f0 + fg;
      if (EPI == GATE) {
        if (P.out[1]) { store4(P.out[1] + to, g); store4(P.out[2] + to, u); }
        with_activation(P.act, [&](auto act) {
#pragma unroll
          for (int j = 0; j < 4; ++j) g[j] = activation<act.value, false>(g[j], nullptr) * u[j];
        });
      }
      store4(P.out[0] + to, g);
    }
  } else {
    if (threadIdx.x == 0) atomicExch(P.status, FF_ERR_TIMEOUT | 0xb00);   // low byte: status, next byte: which kernel
    const long long start = clock64();
    while (clock64() - start < 2000000) { }
  }
  __syncthreads();
  cluster_sync();                                               // no CTA leaves while another reads its sums
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tm, columns);
  }
}

// [rows][cols] bf16 with a box of box_rows rows x 64 columns, 128-byte swizzle.
bool matrix_map(const ff_ffn* h, CUtensorMap* map, const void* base, long long rows, long long cols, int box_rows) {
  // (of the two extents one is dim or hidden: those two, the other extent and the box name the map)
  const int code = (int)(cols == h->cfg.dim ? 0 : 1) * 1024 + box_rows;
  return h->maps.get(map, base, code, (int)rows, [&] {
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, 1};
    cuuint64_t strides[2] = {(cuuint64_t)cols * 2, (cuuint64_t)rows * cols * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
    return ff_encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
  });
}

// fp32 sums [parts][rows][cols] with a box of 32 x 32.
bool sums_map(CUtensorMap* map, const void* base, long long rows, long long cols, int parts) {
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)parts};
  cuuint64_t strides[2] = {(cuuint64_t)cols * 4, (cuuint64_t)rows * cols * 4};
  cuuint32_t box[3] = {32, 32, 1};
  return ff_encode_map(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

// A matrix [rows][cols] as it lies in memory.  An operand's rows are one M or N index each (K-major) or one K index (MN-major).
struct Matrix { const void* p; long long rows, cols; };

// Parts of K for a product with `tiles` tiles of `k` chunks each and an output of `values` values: the number whose estimated time is
// least.  A pair takes 0.28 us for a chunk; with several parts, their sums are written and read in fp32 (4 TB/s) by a second
// launch (2.5 us), and at most two waves of pairs have one each, which bounds the workspace at 148 tiles.
int split_of(long long tiles, int k, double values, double* us = nullptr) {
  constexpr int pairs = FF_B200_SMS / 2;
  int best = 1;
  double least = 0;
  for (int s = 1; s <= 16 && s <= k && (s == 1 || tiles * s <= 2 * pairs); ++s) {
    const double t = 0.28 * (double)((tiles * s + pairs - 1) / pairs) * ((k + s - 1) / s) + (s > 1 ? 2.5 + values * 4 * 2 * s / 4e6 : 0);
    if (s == 1 || t < least) { best = s; least = t; }
  }
  if (us) *us = least;
  return best;
}
// The same for a product with an epilogue, whose K stays whole: tiles of 256 columns or narrow ones, of which there are twice as many.
// A chunk of a narrow tile takes 0.22 us (three quarters of the bytes for half the products), the epilogue of a tile, which overlaps the
// next tile's products, `epilogue` us of a wide one and of a narrow one.  Measured in captured rows of calls, wide / narrow, us: backward of
// 200 tokens, dim 1264, hidden 2464 36.6 / 31.4, of 4000 152 / 158 (estimated the other way round, dH 32 / 26), of 4000 tokens, dim 1024,
// hidden 2816 132 / 135; forward of 128 tokens, dim 512, hidden 1408 16.0 / 12.8, of 1000 tokens, dim 1024, hidden 2816 28.2 / 28.6.
// A forward that keeps G and U has a longer epilogue (10,500 cycles a wide tile, about 5.5 us) than the estimate knows of; its choice was the
// faster one all the same: 128 tokens, dim 512, hidden 1408 14.0 / 11.9, 4000 tokens, dim 768, hidden 2056 43.0 / 46.8, 16384 159 / 174,
// 2000 tokens, dim 2048, hidden 5632 106 / 124.
struct Tiling { bool narrow; double us; };
Tiling tiling_of(long long rows, int cols, int width, int k, const double (&epilogue)[2]) {
  constexpr int pairs = FF_B200_SMS / 2;
  auto time = [&](int w, double chunk, double epi) {
    const long long tiles = ((rows + TM - 1) / TM) * ((cols + w - 1) / w);
    return (double)((tiles + pairs - 1) / pairs) * (k * chunk > epi ? k * chunk : epi) + epi;
  };
  const double wide = time(width, 0.28, epilogue[0]), narrow = time(width / 2, 0.22, epilogue[1]);
  return {narrow < wide, narrow < wide ? narrow : wide};
}
constexpr double GATE_EPILOGUE[2] = {2, 1.8}, DGATE_EPILOGUE[2] = {8, 4};       // (of a narrow gated tile half the warps make H)
struct Product {
  long long rows;                  // extents of an output
  int cols, mats, k;               // matrices, K chunks in all
  long long tiles() const { return ((rows + TM - 1) / TM) * ((cols + TN - 1) / TN) * mats; }
  long long values() const { return rows * cols * mats; }
};
int split_of(const Product& p, double* us = nullptr) { return split_of(p.tiles(), p.k, (double)p.values(), us); }
size_t sums_bytes(const Product& p, int split) { return split > 1 ? ((size_t)p.values() * split * 4 + 255) / 256 * 256 : 0; }
// The same for several products in one launch, whose items go to the pairs as they come: K of each is cut into parts of at most one
// length, that of the least estimated time (the work evenly divided and half an item more, or the longest item).
void splits_of(const Product* p, int count, int* split) {
  constexpr int pairs = FF_B200_SMS / 2;
  int longest = 0;
  for (int i = 0; i < count; ++i) longest = p[i].k > longest ? p[i].k : longest;
  double least = 0;
  for (int s = 1; s <= 16 && s <= longest; ++s) {
    const int most = (longest + s - 1) / s;
    double work = 0, item = 0, moved = 0;
    long long tiles = 0;
    int cut[3];
    for (int i = 0; i < count; ++i) {
      cut[i] = (p[i].k + most - 1) / most;
      work += (double)p[i].tiles() * p[i].k;
      const double length = (p[i].k + cut[i] - 1) / cut[i];
      item = length > item ? length : item;
      if (cut[i] > 1) { tiles += p[i].tiles() * cut[i]; moved += (double)p[i].values() * 8 * cut[i]; }
    }
    if (tiles > 4 * pairs) continue;                             // (bounds the sums at 296 tiles)
    const double even = work / pairs + item / 2, us = 0.28 * (even > item ? even : item) + (tiles ? 2.5 + moved / 4e6 : 0);
    if (s == 1 || us < least) {
      least = us;
      for (int i = 0; i < count; ++i) split[i] = cut[i];
    }
  }
}

// (na, nb, ne: the maps there are; the others, which no product names, are copies)
template <int EPI, int NT>
cudaError_t launch_gemm(const ff_ffn* h, void (*kernel)(GemmMaps, GemmParams), GemmMaps& m, int na, int nb, int ne, GemmParams& P, cudaStream_t st) {
  for (int i = na; i < 4; ++i) m.a[i] = m.a[0];
  for (int i = nb; i < 5; ++i) m.b[i] = m.b[0];
  for (int i = ne; i < 5; ++i) m.e[i] = m.e[0];
  P.act = h->cfg.activation;
  P.status = h->status;
  const int pairs = h->sm_count / 2;
  return ff_launch(kernel, dim3(2 * (unsigned)(P.items < pairs ? P.items : pairs)), dim3(THREADS), smem_bytes(EPI, NT), st, m, P);
}
// GATE or DGATE: `e` are the matrices of the epilogue in the order of GemmMaps, all with the extents of the output.
template <bool A_MN, bool B_MN, int EPI, int NT>
cudaError_t gemm(const ff_ffn* h, const Matrix& a, const Matrix& b0, const Matrix& b1, long long rows, int cols, int k, std::initializer_list<const void*> e,
                 int keep, cudaStream_t st) {
  GemmMaps m = {};
  if (!matrix_map(h, &m.a[0], a.p, a.rows, a.cols, A_MN ? 64 : 128) || !matrix_map(h, &m.b[0], b0.p, b0.rows, b0.cols, B_MN ? 64 : NT / 2) ||
      !matrix_map(h, &m.b[1], b1.p, b1.rows, b1.cols, B_MN ? 64 : NT / 2))
    return cudaErrorInvalidValue;
  int n = 0;
  for (const void* p : e)
    if (!matrix_map(h, &m.e[n++], p, rows, cols, 32)) return cudaErrorInvalidValue;
  GemmParams P = {};
  Sub& s = P.sub[0];
  const int width = EPI == GATE ? NT / 2 : NT;
  s.rows = rows; s.cols = cols;
  s.m_tiles = (int)((rows + TM - 1) / TM);
  s.n_tiles = (cols + width - 1) / width;
  s.mats = s.sources = s.split = 1;
  s.kchunks = k;
  P.items = s.items = s.m_tiles * s.n_tiles;
  P.keep = keep;
  return launch_gemm<EPI, NT>(h, ffn_gemm_kernel<A_MN, B_MN, EPI, NT>, m, 1, 2, n, P, st);
}
// Up to three products without more to do, in one launch, and the join of those cut along K: out[i] = A[0] B[i], or with two sources
// out[0] = A[0] B[0] + A[1] B[1].
struct Wanted { Product p; int split, sources; bool a_mn, b_mn; Matrix a[2], b[2]; void* out[2]; };
cudaError_t products(const ff_ffn* h, const Wanted* w, int count, char* sums, cudaStream_t st) {
  GemmMaps m = {};
  GemmParams P = {};
  JoinParams J = {};
  int na = 0, nb = 0, ne = 0, order[3] = {0, 1, 2}, blocks = 0;
  for (int i = 1; i < count; ++i)                                // the longest items first
    for (int j = i; j && w[order[j]].p.k / w[order[j]].split > w[order[j - 1]].p.k / w[order[j - 1]].split; --j) {
      const int t = order[j]; order[j] = order[j - 1]; order[j - 1] = t;
    }
  for (int i = 0; i < count; ++i) {
    const Wanted& x = w[order[i]];
    Sub& s = P.sub[i];
    s.rows = x.p.rows; s.cols = x.p.cols; s.mats = x.p.mats;
    s.m_tiles = (int)((s.rows + TM - 1) / TM);
    s.n_tiles = (s.cols + TN - 1) / TN;
    s.sources = x.sources; s.kchunks = x.p.k / x.sources;
    s.split = x.split;
    s.items = s.m_tiles * s.n_tiles * s.mats * s.split;
    s.a_mn = x.a_mn; s.b_mn = x.b_mn;
    s.a = na; s.b = nb; s.e = ne;
    P.items += s.items;
    for (int j = 0; j < x.sources; ++j)
      if (!matrix_map(h, &m.a[na++], x.a[j].p, x.a[j].rows, x.a[j].cols, x.a_mn ? 64 : 128)) return cudaErrorInvalidValue;
    for (int j = 0; j < (x.sources > s.mats ? x.sources : s.mats); ++j)
      if (!matrix_map(h, &m.b[nb++], x.b[j].p, x.b[j].rows, x.b[j].cols, x.b_mn ? 64 : 128)) return cudaErrorInvalidValue;
    if (s.split == 1) {
      for (int j = 0; j < s.mats; ++j)
        if (!matrix_map(h, &m.e[ne++], x.out[j], s.rows, s.cols, 32)) return cudaErrorInvalidValue;
      continue;
    }
    if (!sums_map(&m.e[ne++], sums, s.rows, s.cols, s.mats * s.split)) return cudaErrorInvalidValue;
    const long long values = s.rows * s.cols;
    for (int j = 0; j < s.mats; ++j) {
      J.j[J.count++] = Joined{(const float*)sums + j * s.split * values, (__nv_bfloat16*)x.out[j], values, s.split, blocks};
      blocks += (int)((values + 2047) / 2048);
    }
    sums += sums_bytes(x.p, s.split);
  }
  const cudaError_t e = launch_gemm<PRODUCTS, TN>(h, ffn_gemm_kernel<false, false, PRODUCTS, TN>, m, na, nb, ne, P, st);
  return e != cudaSuccess || !J.count ? e : ff_launch(ffn_join_kernel, dim3((unsigned)blocks), dim3(256), 0, st, J);
}

// How the few-token kernel would run a product (tokens of a tile, CTAs of a cluster), and the estimated time of that: a chunk of
// K takes a CTA 0.35 us (0.5 with two matrices: more to load), the exchange of the partial sums 0.02 us for a token and matrix
// (what a CTA reads from others' shared memory, at 25 B/ns; 0.012 from its own), start and end 1 us.  Clusters of three and more do not fill all SMs.
struct FewShape { int nt, split, f_tiles, t_tiles; double us; };
int few_stages(int nt, int mats) {
  // Up to 64 tokens the rings leave room for a CTA of either product on an SM, so that the second one's weights are on their way
  // while the first one ends (one token, dim 2048, hidden 5632: four stages each 18.4 us, three and six 18.8; the rest of Wd asked
  // into L2 ahead of the wait as well: 20.1).
  return nt <= 64 ? (mats == 2 ? (nt <= 16 ? 4 : 3) : nt == 32 ? 5 : 4) : 192 * 1024 / (mats * OPERAND + nt * 128);
}
size_t few_smem(int nt, int mats) {
  const size_t ring = (size_t)few_stages(nt, mats) * (mats * OPERAND + nt * 128), sums = (size_t)mats * nt * 512;
  return (ring > sums ? ring : sums) + 1024;
}
FewShape few_shape(const ff_ffn* h, long long tokens, int features, int kchunks, int mats) {
  FewShape s;
  s.nt = tokens <= 16 ? 16 : tokens <= 32 ? 32 : tokens <= 64 ? 64 : 128;
  s.f_tiles = (features + 127) / 128;
  s.t_tiles = (int)((tokens + s.nt - 1) / s.nt);
  const long long tiles = (long long)s.f_tiles * s.t_tiles;
  s.us = 1e30;
  s.split = 1;
  if (s.t_tiles > 65535) return s;                              // (more than a grid has)
  for (int split = 1; split <= 8 && split <= kchunks; ++split) {
    const int room = h->room[mats - 1][s.nt == 128][split];
    if (room < split) continue;
    const double exchange = (split > 1 ? 0.02 : 0.012) * mats * (double)(tokens < s.nt ? tokens : s.nt);
    const double us = 1 + (double)((tiles * split + room - 1) / room) * (((kchunks + split - 1) / split) * (mats == 2 ? 0.5 : 0.35) + exchange);
    if (us < s.us) { s.split = split; s.us = us; }
  }
  return s;
}

template <int EPI>
cudaError_t few(const ff_ffn* h, const FewShape& s, const void* w0, const void* w1, const void* x, long long tokens, int features, int k,
                void* const (&out)[3], cudaStream_t st) {
  CUtensorMap m[3];
  if (!matrix_map(h, &m[0], w0, k, features, 64) || !matrix_map(h, &m[2], x, tokens, k, s.nt)) return cudaErrorInvalidValue;
  if (EPI != GATE) m[1] = m[0];
  else if (!matrix_map(h, &m[1], w1, k, features, 64)) return cudaErrorInvalidValue;
  FewParams P{};
  P.tokens = (int)tokens; P.cols = features; P.kchunks = chunks(k);
  P.nt = s.nt;
  const int mats = EPI == GATE ? 2 : 1;
  P.stage_bytes = mats * OPERAND + s.nt * 128;
  P.stages = few_stages(s.nt, mats);
  P.act = h->cfg.activation;
  for (int i = 0; i < 3; ++i) P.out[i] = (__nv_bfloat16*)out[i];
  P.status = h->status;
  return ff_launch_cluster(ffn_few_kernel<EPI>, dim3((unsigned)(s.f_tiles * s.split), (unsigned)s.t_tiles), dim3(FEW_THREADS), s.split,
                           few_smem(s.nt, mats), st, m[0], m[1], m[2], P);
}


ff_status_t fail(ff_ffn* h, ff_status_t code, const char* msg) {
  if (h) snprintf(h->err, sizeof h->err, "%s", msg);
  else ff_set_thread_error(msg);
  return code;
}
ff_status_t cuda_fail(ff_ffn* h, cudaError_t e) {
  char msg[256];
  snprintf(msg, sizeof msg, "CUDA error: %s", cudaGetErrorString(e));
  return fail(h, FF_ERR_CUDA, msg);
}
#define FFN_CUDA(h, call)                                  \
  do {                                                     \
    const cudaError_t e__ = (call);                        \
    if (e__ != cudaSuccess) return cuda_fail((h), e__);    \
  } while (0)

bool misaligned(std::initializer_list<const void*> ps) {
  uintptr_t all = 0;
  for (const void* p : ps) all |= (uintptr_t)p;
  return all & 15;
}
// A tensor of a call that a launch reads or writes; NULL: not given, or not read by then.
struct Span { const void* p; size_t bytes; };
bool meet(const Span& a, const Span& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return a.p && b.p && x < y + b.bytes && y < x + a.bytes;
}
// Does one of `written` overlap another of them or one of `read`?
bool overlap(std::initializer_list<Span> written, std::initializer_list<Span> read) {
  for (const Span* w = written.begin(); w != written.end(); ++w) {
    for (const Span* v = written.begin(); v != w; ++v)
      if (meet(*w, *v)) return true;
    for (const Span& r : read)
      if (meet(*w, r)) return true;
  }
  return false;
}
// More tokens than the kernels' indexes and tensor maps take
constexpr char MOST_TOKENS[] = "tokens must be at most 2^31 - 256, and tokens * hidden (or dim) at most 2^38";
bool too_many(const ff_ffn_config_t& c, int64_t tokens) {
  return tokens > 0x7fffff00 || tokens * (int64_t)(c.dim > c.hidden ? c.dim : c.hidden) > (1ll << 38);
}
ff_status_t check_call(ff_ffn* h, int64_t tokens, void* ws, size_t ws_bytes, int training, size_t* need) {
  if (tokens < 0) return fail(h, FF_ERR_INVALID_ARG, "tokens must not be negative");
  if (too_many(h->cfg, tokens)) return fail(h, FF_ERR_UNSUPPORTED, MOST_TOKENS);
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess || device != h->device) return fail(h, FF_ERR_INVALID_ARG, "the handle belongs to another device than the current one");
  *need = 0;
  ff_ffn_workspace_bytes(&h->cfg, tokens, training, need);
  if (*need && (!ws || ws_bytes < *need)) return fail(h, FF_ERR_WORKSPACE, "the workspace is missing or smaller than ff_ffn_workspace_bytes");
  if (*need && (((uintptr_t)ws) & 255)) return fail(h, FF_ERR_WORKSPACE, "the workspace must be 256-byte aligned");
  return FF_OK;
}
Product down_product(const ff_ffn_config_t& c, int64_t tokens) { return {tokens, c.dim, 1, chunks(c.hidden)}; }
// dX;  dWg and dWu;  dWd, with their parts, the same whichever of them a call wants
struct Gradients { Product p[3]; int split[3]; };
Gradients gradients_of(const ff_ffn_config_t& c, int64_t tokens) {
  Gradients g = {{{tokens, c.dim, 1, 2 * chunks(c.hidden)}, {c.dim, c.hidden, 2, chunks(tokens)}, {c.hidden, c.dim, 1, chunks(tokens)}}, {1, 1, 1}};
  splits_of(g.p, 3, g.split);
  return g;
}
size_t hidden_bytes(const ff_ffn_config_t& c, int64_t tokens) { return ((size_t)tokens * c.hidden * 2 + 255) / 256 * 256; }

}  // namespace

extern "C" ff_status_t ff_ffn_validate(const ff_ffn_config_t* c) {
  if (!c) return fail(nullptr, FF_ERR_INVALID_ARG, "cfg is NULL");
  if (c->dim < 1 || c->hidden < 1) return fail(nullptr, FF_ERR_INVALID_ARG, "dim and hidden must be positive");
  if (c->activation < FF_ACT_SILU || c->activation > FF_ACT_GELU) return fail(nullptr, FF_ERR_INVALID_ARG, "unknown activation");
  if (c->dim % 8 || c->hidden % 8 || c->dim > (1 << 20) || c->hidden > (1 << 20))
    return fail(nullptr, FF_ERR_UNSUPPORTED, "dim and hidden must be multiples of 8 (rows of 16-byte pieces), at most 2^20");
  return FF_OK;
}

extern "C" ff_status_t ff_ffn_workspace_bytes(const ff_ffn_config_t* c, int64_t tokens, int32_t training, size_t* bytes) {
  const ff_status_t s = ff_ffn_validate(c);
  if (s != FF_OK) return s;
  if (!bytes || tokens < 0) return fail(nullptr, FF_ERR_INVALID_ARG, "bytes is NULL or tokens negative");
  if (too_many(*c, tokens)) return fail(nullptr, FF_ERR_UNSUPPORTED, MOST_TOKENS);
  // H;  backward: dG, dU, H;  behind them the sums of products whose K is cut
  *bytes = (training ? 3 : 1) * hidden_bytes(*c, tokens);
  if (tokens > 0 && training) {
    const Gradients g = gradients_of(*c, tokens);
    for (int i = 0; i < 3; ++i) *bytes += sums_bytes(g.p[i], g.split[i]);
  } else if (tokens > 0) {
    const Product down = down_product(*c, tokens);
    *bytes += sums_bytes(down, split_of(down));
  }
  return FF_OK;
}

extern "C" ff_status_t ff_ffn_create(const ff_ffn_config_t* cfg, ff_ffn_t** out) {
  if (!out) return fail(nullptr, FF_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  const ff_status_t s = ff_ffn_validate(cfg);
  if (s != FF_OK) return s;
  ff_ffn* h = new (std::nothrow) ff_ffn();
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "out of host memory");
  h->cfg = *cfg;
  cudaError_t e = cudaGetDevice(&h->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->sm_count, cudaDevAttrMultiProcessorCount, h->device);
  const struct { const void* kernel; size_t smem; } kernels[] = {
      {(const void*)ffn_gemm_kernel<false, true, GATE, TN>, smem_bytes(GATE)}, {(const void*)ffn_gemm_kernel<false, true, GATE, 128>, smem_bytes(GATE, 128)},
      {(const void*)ffn_gemm_kernel<false, false, DGATE, TN>, smem_bytes(DGATE)}, {(const void*)ffn_gemm_kernel<false, false, DGATE, 128>, smem_bytes(DGATE, 128)},
      {(const void*)ffn_gemm_kernel<false, false, PRODUCTS, TN>, smem_bytes(PRODUCTS)}, {(const void*)ffn_few_kernel<GATE>, FEW_SMEM},
      {(const void*)ffn_few_kernel<PRODUCTS>, FEW_SMEM}};
  for (const auto& k : kernels)
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)k.smem);
  for (int mats = 1; mats <= 2; ++mats)
    for (int wide = 0; wide < 2; ++wide)
      for (int split = 1; split <= 8 && e == cudaSuccess; ++split) {
        int clusters = 0;
        const size_t smem = few_smem(wide ? 128 : 64, mats);
        e = mats == 2 ? ff_max_clusters(&clusters, ffn_few_kernel<GATE>, dim3(FEW_THREADS), split, smem)
                      : ff_max_clusters(&clusters, ffn_few_kernel<PRODUCTS>, dim3(FEW_THREADS), split, smem);
        // (asked for kernels that use tensor memory, the runtime counts one block an SM; two run where shared memory has room for them)
        h->room[mats - 1][wide][split] = clusters * split * (int)(233472 / (smem + 1024));
      }
  if (e == cudaSuccess) e = cudaMalloc((void**)&h->status, 256);
  // (cleared before the handle is out, on a stream of its own: the default stream may be busy, and others do not wait for it)
  cudaStream_t st = nullptr;
  if (e == cudaSuccess) e = cudaStreamCreateWithFlags(&st, cudaStreamNonBlocking);
  if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, 256, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (st) cudaStreamDestroy(st);
  if (e != cudaSuccess) {
    if (h->status) cudaFree(h->status);
    delete h;
    return cuda_fail(nullptr, e);
  }
  *out = h;
  return FF_OK;
}

extern "C" ff_status_t ff_ffn_destroy(ff_ffn_t* h) {
  if (h) {
    if (h->status) cudaFree(h->status);
    delete h;
  }
  return FF_OK;
}

extern "C" const char* ff_ffn_last_error(const ff_ffn_t* h) { return h ? h->err : ff_last_error(nullptr); }

extern "C" ff_status_t ff_ffn_device_status(ff_ffn_t* h, void* stream) {
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "the handle is NULL");
  int word = 0;
  cudaStream_t st = (cudaStream_t)stream;
  FFN_CUDA(h, cudaMemcpyAsync(&word, h->status, sizeof word, cudaMemcpyDeviceToHost, st));
  FFN_CUDA(h, cudaStreamSynchronize(st));
  if (!word) return FF_OK;
  FFN_CUDA(h, cudaMemsetAsync(h->status, 0, sizeof word, st));
  FFN_CUDA(h, cudaStreamSynchronize(st));
  return fail(h, word & 255, "a device-side wait expired");
}

extern "C" ff_status_t ff_ffn_forward(ff_ffn_t* h, int64_t tokens, const void* X, const void* Wg, const void* Wu, const void* Wd, void* gate,
                                      void* up, void* out, void* ws, size_t ws_bytes, void* stream) {
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "the handle is NULL");
  size_t need;
  ff_status_t s = check_call(h, tokens, ws, ws_bytes, 0, &need);
  if (s != FF_OK) return s;
  if (!gate != !up) return fail(h, FF_ERR_INVALID_ARG, "gate and up are kept together, or neither is");
  if (tokens == 0) return FF_OK;
  if (!X || !Wg || !Wu || !Wd || !out) return fail(h, FF_ERR_INVALID_ARG, "X, Wg, Wu, Wd or out is NULL");
  if (misaligned({X, Wg, Wu, Wd, gate, up, out})) return fail(h, FF_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  const int D = h->cfg.dim, F = h->cfg.hidden;
  // (out is written when X, Wg and Wu have been read)
  const size_t row = (size_t)tokens * D * 2, hidden = (size_t)tokens * F * 2, weight = (size_t)D * F * 2;
  if (overlap({{gate, hidden}, {up, hidden}, {ws, need}}, {{X, row}, {Wg, weight}, {Wu, weight}, {Wd, weight}, {out, row}}) || meet({out, row}, {Wd, weight}))
    return fail(h, FF_ERR_INVALID_ARG, "gate, up or the workspace overlaps another tensor, or out overlaps Wd");
  cudaStream_t st = (cudaStream_t)stream;
  const Matrix x{X, tokens, D}, hid{ws, tokens, F}, wg{Wg, D, F}, wu{Wu, D, F}, wd{Wd, F, D};
  // Either product runs on the kernel whose estimate is lower (2 us more for start and end of the larger one).  Measured in captured rows of
  // calls, dim 2048, hidden 5632, both products on the tiles that tiling_of gives / on the few-token kernel, us: 1 token 36.9 / 18.9,
  // 64 tokens 29.3 / 23.6, 128 30.0 / 26.9, 512 42.9 / 62.4; dim 1024, hidden 2816, product with Wd: 400 tokens 22.2 / 19.3, 768 24.2 / 23.6.
  const FewShape up_few = few_shape(h, tokens, F, chunks(D), 2), down_few = few_shape(h, tokens, D, chunks(F), 1);
  const Product down = down_product(h->cfg, tokens);
  double down_us;
  const int down_split = split_of(down, &down_us);
  down_us += 2;
  const Tiling up_tiling = tiling_of(tokens, F, 128, chunks(D), GATE_EPILOGUE);
  if (up_few.us < up_tiling.us) {
    FFN_CUDA(h, few<GATE>(h, up_few, Wg, Wu, X, tokens, F, D, {ws, gate, up}, st));
  } else {
    const auto run = up_tiling.narrow ? gemm<false, true, GATE, 128> : gemm<false, true, GATE, TN>;
    FFN_CUDA(h, run(h, x, wg, wu, tokens, F, chunks(D), {ws, gate ? gate : ws, up ? up : ws}, gate != nullptr, st));
  }
  if (down_few.us < down_us) {
    FFN_CUDA(h, few<PRODUCTS>(h, down_few, Wd, Wd, ws, tokens, D, F, {out, nullptr, nullptr}, st));
  } else {
    const Wanted w = {down, down_split, 1, false, true, {hid}, {wd}, {out}};
    FFN_CUDA(h, products(h, &w, 1, (char*)ws + hidden_bytes(h->cfg, tokens), st));
  }
  return FF_OK;
}

extern "C" ff_status_t ff_ffn_backward(ff_ffn_t* h, int64_t tokens, const void* X, const void* Wg, const void* Wu, const void* Wd, const void* gate,
                                       const void* up, const void* dout, void* dX, void* dWg, void* dWu, void* dWd, void* ws, size_t ws_bytes,
                                       void* stream) {
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "the handle is NULL");
  size_t need;
  ff_status_t s = check_call(h, tokens, ws, ws_bytes, 1, &need);
  if (s != FF_OK) return s;
  if (!dWg != !dWu) return fail(h, FF_ERR_INVALID_ARG, "dWg and dWu are made together, or neither is");
  if (misaligned({X, Wg, Wu, Wd, gate, up, dout, dX, dWg, dWu, dWd})) return fail(h, FF_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  const int D = h->cfg.dim, F = h->cfg.hidden;
  cudaStream_t st = (cudaStream_t)stream;
  if (tokens == 0) {               // sums over no tokens
    void* w[3] = {dWg, dWu, dWd};
    for (void* p : w)
      if (p) FFN_CUDA(h, cudaMemsetAsync(p, 0, (size_t)D * F * 2, st));
    return FF_OK;
  }
  if (!X || !Wg || !Wu || !Wd || !gate || !up || !dout) return fail(h, FF_ERR_INVALID_ARG, "X, Wg, Wu, Wd, gate, up or dout is NULL");
  if (!dX && !dWg && !dWd) return FF_OK;
  // (the launch that writes the gradients reads X for dWg and dWu, dout for dWd, Wg and Wu for dX; gate, up and Wd have been read by then)
  const size_t row = (size_t)tokens * D * 2, hidden = (size_t)tokens * F * 2, weight = (size_t)D * F * 2;
  const Span all{ws, need};
  if (overlap({{dX, row}, {dWg, weight}, {dWu, weight}, {dWd, weight}, all},
              {{dWg ? X : nullptr, row}, {dWd ? dout : nullptr, row}, {dX ? Wg : nullptr, weight}, {dX ? Wu : nullptr, weight}}) ||
      overlap({all}, {{X, row}, {Wg, weight}, {Wu, weight}, {Wd, weight}, {gate, hidden}, {up, hidden}, {dout, row}}))
    return fail(h, FF_ERR_INVALID_ARG, "a gradient overlaps another one or what it is made from, or the workspace overlaps a tensor");
  char* base = (char*)ws;
  void *dG = base, *dU = base + hidden_bytes(h->cfg, tokens), *H = base + 2 * hidden_bytes(h->cfg, tokens);
  const Matrix x{X, tokens, D}, g{dout, tokens, D}, wg{Wg, D, F}, wu{Wu, D, F}, wd{Wd, F, D};
  const Matrix dg{dG, tokens, F}, du{dU, tokens, F}, hid{H, tokens, F};
  const auto run = tiling_of(tokens, F, TN, chunks(D), DGATE_EPILOGUE).narrow ? gemm<false, false, DGATE, 128> : gemm<false, false, DGATE, TN>;
  FFN_CUDA(h, run(h, g, wd, wd, tokens, F, chunks(D), {gate, up, dG, dU, H}, 0, st));
  const Gradients made = gradients_of(h->cfg, tokens);
  Wanted w[3];
  int count = 0;
  if (dX) w[count++] = Wanted{made.p[0], made.split[0], 2, false, false, {dg, du}, {wg, wu}, {dX}};
  if (dWg) w[count++] = Wanted{made.p[1], made.split[1], 1, true, true, {x}, {dg, du}, {dWg, dWu}};
  if (dWd) w[count++] = Wanted{made.p[2], made.split[2], 1, true, true, {hid}, {g}, {dWd}};
  FFN_CUDA(h, products(h, w, count, base + 3 * hidden_bytes(h->cfg, tokens), st));
  return FF_OK;
}
