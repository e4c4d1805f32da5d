// Cross attention to an encoder's states: forward pass and the C entry points.
//
//   out = softmax_j(scale q k_j) v,   lse = ln sum_j e^(scale q k_j),   over the keys j that count
//
// One pass over the keys with the running maximum m and sum l of the softmax (Milakov and Gimelshein, "Online normalizer
// calculation for softmax", 2018), scores in units of log2.
//
// A CTA takes items (sample, key head, one or two neighbouring tiles of queries, part of the keys); the two tiles, "streams" A and
// B, share every tile of keys and values, and while the softmax of one works the tensor core runs the products of the other.
//   warp 0       TMA producer: the query tiles; tiles of 64 keys and of their values, each through a ring of its own
//   warps 1, 3   tcgen05.mma issuers of A and B: S_x = Q_x K^T (both from shared memory) into one of two places in turns, O_x += P_x V (P from
//                tensor memory), in the order QK[j+1], PV[j], but an item's last PV before the next item's first QK, since its softmax warps
//                wait for it (16K queries, 12 heads, 8192 keys 845 -> 788 us).  (One warp for both was the limit, and so were more commits
//                than the one for the scores: some 32 cycles an instruction, 150 a commit or wait.  What else waits for a product
//                within an item is told by the softmax warps, when they see scores that were asked for behind it.)  Warp 1 owns the tensor memory
//   warp 2       zeros in rows of V whose keys do not count, in tiles that may hold such rows
//   warps 4..11  softmax: a thread per query row; P goes back to tensor memory as bf16 over the scores, while the next tile's scores are
//                made in the other place.  O accumulates in tensor memory and is rescaled only when a row's maximum
//                grows by more than 2^8.  At the end O / l goes out through shared memory by TMA.
// With tiles of 128 keys there is room for one place of scores a stream: the next ones had to wait for the product with the last P, and
// 64K queries, 24 heads of 128, 512 keys took 578 us; P in shared memory freed that place, but the products then read more from shared memory
// than it gives (589 us).  Now 457 us (243 at the rate of a large matrix product) for some 20 ms of calls, captured or not, at 1.9 GHz; 525 in a row for
// seconds, when the board's power limit holds the clock at 1.7.  The issuers are the limit, whose products with M = 128, N = 64
// read more operand bytes a cycle than larger tiles, then the softmax (1070 cycles a tile of its own, 1024 of them the two streams' exponentials).
// Tensor memory (512 columns): S/P of A and of B, twice 64 each, O of A, O of B.  Every wait is bounded; when one runs out the CTA raises
// FF_ERR_TIMEOUT in the handle's status word, takes no more work and returns.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <initializer_list>
#include <new>

#include "ff_cross.cuh"

using namespace sm100;

namespace {

constexpr int TILE = CX_TILE;
constexpr int TILE_BYTES = TILE * 128 * 2, HALF_BYTES = TILE_BYTES / 2;
constexpr int THREADS = 128 + 2 * 128;
constexpr int KEYS = 64;       // of a tile
constexpr float LAZY_LOG2 = 8.0f;

struct CrossParams {
  CrossDims dm;
  int pair, pairs, splits;     // tiles of an item (1 or 2), items of a key head of a sample, parts of the keys
  CxDiv by_pairs, by_splits;
  int items;
  float* lse;                  // or NULL
  float *part, *part_lse;      // splits > 1: [part][batch][heads][tokens][d] O / l, and the sums' log2
};

template <int HD> constexpr int PLACES = HD == 64 ? 4 : 3;              // of the rings
struct Shared {
  uint64_t q_full[2], q_empty[2];                                       // per stream
  uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4];                // per place
  uint64_t v_raw[4];                                                    // in place of v_full for a tile that has to be cleaned first
  uint64_t s_full[2][2], p_full[2][2];                                  // per stream and place of its scores
  uint64_t pv_done[2], o_full[2], o_empty[2], staged[2], sent[2];       // per stream
  uint32_t tmem_base;
  int abort_flag;
};
constexpr size_t SMEM = 7 * TILE_BYTES + sizeof(Shared) + 1024;
// The place of a ring that a tile has, and the parity of its turn there.
template <int N> struct Place {
  unsigned at = 0, turn = 0;
  __device__ __forceinline__ void next() { if (++at == N) { at = 0; turn ^= 1; } }
  __device__ __forceinline__ unsigned back(unsigned n) const { return at >= n ? at - n : at + N - n; }
  __device__ __forceinline__ void skip(unsigned n) { n += at; at = n % N; turn ^= n / N & 1; }
};

struct Item { int b, g, part, tile, has_b, keys, j0, j1; };
__device__ __forceinline__ Item item_of(const CrossParams& P, int it) {
  Item x;
  const int rest = P.by_pairs(it);
  x.tile = (it - rest * P.pairs) * P.pair;
  x.has_b = P.pair == 2 && x.tile + 1 < P.dm.tiles;
  const int bg = P.by_splits(rest);
  x.part = rest - bg * P.splits;
  x.b = P.dm.by_G(bg);
  x.g = bg - x.b * P.dm.G;
  x.keys = cx_keys(P.dm, x.b);
  const int nk = (x.keys + KEYS - 1) / KEYS;
  x.j0 = cx_first(nk, x.part, P.splits, P.by_splits);
  x.j1 = cx_first(nk, x.part + 1, P.splits, P.by_splits);
  return x;
}

// The tiles of keys of a CTA's items, one after the other.
struct Steps {
  const CrossParams& P;
  int it, j;
  Item x;
  bool there;
  __device__ __forceinline__ Steps(const CrossParams& P_) : P(P_), it((int)blockIdx.x - (int)gridDim.x), there(true) { item(); }
  __device__ __forceinline__ void item() {                   // (items without keys have none)
    do {
      it += gridDim.x;
      if (it >= P.items) { there = false; return; }
      x = item_of(P, it);
    } while (x.j0 == x.j1);
    j = x.j0;
  }
  __device__ __forceinline__ void next() { if (++j == x.j1) item(); }
  __device__ __forceinline__ bool first() const { return j == x.j0; }
};

// The same with what the issuers need alone.
struct Cursor {
  int it, left, keys;          // item; tiles of it from here on; keys from the tile's first one on
  bool has_b, first, there;    // is it the item's first tile?
  __device__ __forceinline__ Cursor(const CrossParams& P) : it((int)blockIdx.x - (int)gridDim.x) { item(P); }
  __device__ __forceinline__ void item(const CrossParams& P) {
    do {
      it += gridDim.x;
      there = it < P.items;
      if (!there) return;
      const Item x = item_of(P, it);
      left = cx_uniform(x.j1 - x.j0); keys = cx_uniform(x.keys - x.j0 * KEYS); has_b = x.has_b;
    } while (left == 0);
    first = true;
  }
  __device__ __forceinline__ void next(const CrossParams& P) {
    keys -= KEYS; first = false;
    if (--left == 0) item(P);
  }
  __device__ __forceinline__ bool last() const { return left == 1; }
  __device__ __forceinline__ int sixteens() const { return keys >= KEYS ? KEYS / 16 : (keys + 15) / 16; }      // of the tile's keys
};

template <int HD>
__global__ void __launch_bounds__(THREADS, 1)
cross_forward_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                     const __grid_constant__ CUtensorMap map_o, const __grid_constant__ CrossParams P) {
  extern __shared__ uint8_t smem_raw[];
  constexpr int HALVES = HD / 64, BYTES = TILE * HD * 2, NP = PLACES<HD>, KV_BYTES = KEYS * HD * 2, KV_HALF = KEYS * 128;
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sQ = smem;                       // queries of streams A and B
  uint8_t* sO = sQ + 2 * BYTES;             // outputs of A and B
  uint8_t* sK = sO + 2 * BYTES;             // NP places
  uint8_t* sV = sK + NP * KV_BYTES;         // NP places
  Shared& sh = *(Shared*)(smem + 7 * TILE_BYTES);
  static_assert(4 * BYTES + 2 * NP * KV_BYTES <= 7 * TILE_BYTES, "");
  const CrossDims& D = P.dm;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NP; ++i) {
      mbar_init(&sh.k_full[i], 1); mbar_init(&sh.k_empty[i], 2);
      mbar_init(&sh.v_full[i], 1); mbar_init(&sh.v_empty[i], 2); mbar_init(&sh.v_raw[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], 1); mbar_init(&sh.q_empty[i], 1);
      for (int k = 0; k < 2; ++k) { mbar_init(&sh.s_full[i][k], 1); mbar_init(&sh.p_full[i][k], 128); }
      mbar_init(&sh.pv_done[i], 1); mbar_init(&sh.o_full[i], 1); mbar_init(&sh.o_empty[i], 128);
      mbar_init(&sh.staged[i], 128); mbar_init(&sh.sent[i], 1);
    }
    sh.abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&map_q); tma_prefetch_desc(&map_k); tma_prefetch_desc(&map_v); tma_prefetch_desc(&map_o);
  }
  if (warp == 1) { tmem_alloc(&sh.tmem_base, 512); tmem_relinquish(); }
  ff_pdl_join();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = sh.tmem_base;
  volatile int* abort_flag = &sh.abort_flag;

  if (warp < 4) {
    reg_dec<104>();
    if (warp == 0) {
      // ------------------------------------------------------------------ TMA producer
      if (lane == 0) {
        const int q_bytes = D.bn * D.bh * HD * 2;
        unsigned items[2] = {0, 0}, g = 0;
        Place<NP> kp, vp;
        bool ok = true;
        // the keys of tile gt, ahead of them the queries of its item where that begins
        auto load_keys = [&](const Steps& w, unsigned gt) {
          const Item& x = w.x;
          if (w.first())
            for (int sx = 0; sx <= x.has_b && ok; ++sx) {
              if (items[sx] >= 1) ok = mbar_wait(&sh.q_empty[sx], (items[sx] - 1) & 1, abort_flag);
              if (!ok) break;
              ++items[sx];
              int h0, n0;
              cx_place(D, x.g, x.tile + sx, h0, n0);
              mbar_arrive_expect_tx(&sh.q_full[sx], q_bytes);
              cx_load(sQ + sx * BYTES, HALF_BYTES, HALVES, &map_q, &sh.q_full[sx], n0, h0 * D.once[0][1], x.b * D.once[0][0]);
            }
          if (ok && gt >= NP) ok = mbar_wait(&sh.k_empty[kp.at], kp.turn ^ 1, abort_flag);
          if (!ok) return;
          mbar_arrive_expect_tx(&sh.k_full[kp.at], KV_BYTES);
          cx_load(sK + kp.at * KV_BYTES, KV_HALF, HALVES, &map_k, &sh.k_full[kp.at], w.j * KEYS, x.g * D.once[1][1], x.b * D.once[1][0]);
          kp.next();
        };
        Steps ahead(P);
        // the values of the tile behind it
        int j = 0, h = 0, b = 0;
        bool clean = false;
        auto load_values = [&] {
          if (g >= NP) ok = mbar_wait(&sh.v_empty[vp.at], vp.turn ^ 1, abort_flag);
          if (!ok) return;
          uint64_t* bar = clean ? &sh.v_raw[vp.at] : &sh.v_full[vp.at];
          mbar_arrive_expect_tx(bar, KV_BYTES);
          cx_load(sV + vp.at * KV_BYTES, KV_HALF, HALVES, &map_v, bar, j * KEYS, h, b);
          vp.next();
        };
        bool there = ahead.there;
        if (there) load_keys(ahead, 0);
        for (; there && ok; ++g) {
          j = ahead.j; h = ahead.x.g * D.once[2][1]; b = ahead.x.b * D.once[2][0];
          clean = cx_unclean<KEYS>(D, ahead.x.keys, j);
          ahead.next();
          there = ahead.there;
          // Values first where their place is free, else the next keys, whose place is free sooner.
          const bool first = g < NP || mbar_try_wait(&sh.v_empty[vp.at], vp.turn ^ 1);
          if (first) load_values();
          if (ok && there) load_keys(ahead, g + 1);
          if (ok && !first) load_values();
        }
      }
    } else if (warp == 1 || warp == 3) {
      // ------------------------------------------------------------------ MMA issuers, one for either stream
      const int sx = warp >> 1;
      const uint32_t idesc_qk = idesc_bf16_f32(TILE, 0, false, false);
      const uint32_t idesc_pv = idesc_bf16_f32(TILE, HD, false, true);
      unsigned asked = 0, done = 0;           // steps whose scores have been asked for, whose P has been consumed
      unsigned begun = 0, ended = 0;          // items whose scores have begun, whose outputs are complete
      bool ok = true;
      const uint64_t q_desc = smem_desc_sw128(smem_u32(sQ + sx * BYTES), 16, 1024), k_desc = smem_desc_sw128(smem_u32(sK), 16, 1024);
      const uint64_t v_desc = smem_desc_sw128(smem_u32(sV), KV_HALF, 1024);
      const uint32_t s_tm = tm + sx * 128, o_tm = s_tm + 256;
      Place<NP> kp, vp;
      auto mine = [&](const Cursor& w) { return sx == 0 || w.has_b; };
      // the scores of a tile (their place has been read: the P in it by the product two tiles before, issued by then)
      auto scores = [&](const Cursor& w) -> bool {
        if (!mbar_wait_warp(&sh.k_full[kp.at], kp.turn, abort_flag)) return false;
        if (mine(w)) {
          if (w.first && !mbar_wait_warp(&sh.q_full[sx], begun++ & 1, abort_flag)) return false;
          tc_fence_after();
          const uint32_t idesc = idesc_qk | (uint32_t)(w.sixteens() * 2) << 17;              // (N in eights)
          const uint64_t kd = k_desc + (uint64_t)(kp.at * (KV_BYTES >> 4));
          const int place = asked++ & 1;
#pragma unroll
          for (int k = 0; k < HALVES; ++k)
            umma_ss4(s_tm + place * 64, q_desc + (uint64_t)(k * (HALF_BYTES >> 4)), kd + (uint64_t)(k * (KV_HALF >> 4)), idesc, k > 0 ? 1u : 0u);
          umma_commit(&sh.s_full[sx][place]);
          if (w.last()) umma_commit(&sh.q_empty[sx]);
        } else if (lane == 0) {
          mbar_arrive(&sh.k_empty[kp.at]);
        }
        kp.next();
        return true;
      };
      auto product = [&](const Cursor& w) -> bool {
        if (!mbar_wait_warp(&sh.v_full[vp.at], vp.turn, abort_flag)) return false;
        if (mine(w)) {
          const int place = done & 1, steps = w.sixteens();
          if (!mbar_wait_warp(&sh.p_full[sx][place], done >> 1 & 1, abort_flag)) return false;
          if (w.first && ended >= 1 && !mbar_wait_warp(&sh.o_empty[sx], (ended - 1) & 1, abort_flag)) return false;
          tc_fence_after();
          const uint64_t vd = v_desc + (uint64_t)(vp.at * (KV_BYTES >> 4));
          const uint32_t p_tm = s_tm + place * 64, on = w.first ? 0u : 1u;
          if (steps == KEYS / 16) {
            umma_ts4(o_tm, p_tm, vd, idesc_pv, on);
          } else {
            for (int k = 0; k < steps; ++k) umma_ts(o_tm, p_tm + k * 8, vd + (uint64_t)(k * (2048 >> 4)), idesc_pv, k == 0 ? on : 1u);
          }
          ++done;
          if (w.left == 2) umma_commit(&sh.pv_done[sx]);
          if (w.last()) { umma_commit(&sh.o_full[sx]); umma_commit(&sh.v_empty[vp.at]); ++ended; }
        } else if (lane == 0) {
          mbar_arrive(&sh.v_empty[vp.at]);
        }
        vp.next();
        return true;
      };
      Cursor now(P);
      if (now.there) ok = scores(now);
      while (now.there && ok) {
        Cursor ahead = now;
        ahead.next(P);
        // The next tile's scores first, but those of another item behind this one's last product, for which the softmax warps wait.
        const bool early = ahead.there && !ahead.first;
        if (early) ok = scores(ahead);
        if (ok) ok = product(now);
        if (ok && ahead.there && !early) ok = scores(ahead);
        now = ahead;
      }
    } else if (warp == 2) {
      // ------------------------------------------------------------------ rows of V that do not count
      unsigned turns = 0;                                   // whether each place has been cleaned an odd number of times
      Place<NP> vp;
      bool ok = true;
      for (Steps w(P); w.there && ok; w.next(), vp.next()) {
        if (!cx_unclean<KEYS>(D, w.x.keys, w.j)) continue;
        const CxValid64 valid = cx_valid64(D, w.x.b, w.x.keys, w.j * KEYS, lane);
        ok = mbar_wait_warp(&sh.v_raw[vp.at], turns >> vp.at & 1, abort_flag);
        if (!ok) break;
        turns ^= 1u << vp.at;
        cx_clean(sV + vp.at * KV_BYTES, KV_HALF, HALVES, valid.w, lane);
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.v_full[vp.at]);
      }
    }
  } else {
    reg_inc<200>();
    // ------------------------------------------------------------------ softmax
    const int quarter = warp & 3;
    const int sx = (warp - 4) >> 2;
    const int row = quarter * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
    const uint32_t s_addr = tm + lane_addr + sx * 128;
    const uint32_t o_addr = tm + lane_addr + 256 + sx * 128;
    uint8_t* stage = sO + sx * BYTES;
    const float sl2 = D.sl2;
    unsigned n = 0, items = 0, ends = 0;      // tiles this stream has taken, items (with keys; with more than one tile of them) it has ended
    Place<NP> vp;                     // of the tile's keys and values
    unsigned staged = 0;              // items it has put on the stage
    bool ok = true;
    for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
      int b, keys, from;
      bool work;                                            // (rows that a tile does not have take no time)
      {
        const Item x = item_of(P, it);
        if (sx == 1 && !x.has_b) {
          vp.skip(x.j1 - x.j0);
          continue;
        }
        int h0, n0;
        cx_place(D, x.g, x.tile + sx, h0, n0);
        const int row_h = D.by_bn(row);
        work = __any_sync(0xffffffffu, row_h < D.bh && n0 + row - row_h * D.bn < D.N);
        b = x.b; from = x.j0 * KEYS; keys = x.keys < x.j1 * KEYS ? x.keys : x.j1 * KEYS;       // (of this part)
      }
      const bool some = from < keys;
      float m_ref = -INFINITY, mb = 0.f, l = 0.f;
      bool counts = false;                                  // has a key counted?
      for (int first = from; first < keys && ok; first += KEYS, ++n, vp.next()) {
        const bool full = !D.mask && first + KEYS <= keys;
        CxValid64 valid = {};
        if (!full) valid = cx_valid64(D, b, keys, first, lane);
        const uint32_t at = s_addr + (n & 1) * 64;
        ok = mbar_wait_warp(&sh.s_full[sx][n & 1], n >> 1 & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        if (row == 0) {                                     // what has been read by now: the keys, and the values two tiles back
          mbar_arrive(&sh.k_empty[vp.at]);
          if (first >= from + 2 * KEYS) mbar_arrive(&sh.v_empty[vp.back(2)]);
        }
        if (work) {
          uint32_t r[2][32];
          // scores into registers, those of keys that do not count as -infinity; their maximum
          tmem_ld32(at, r[0]);
          tmem_ld32(at + 32, r[1]);
          tmem_wait_ld();
          if (!full) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!(valid.w[i & 1] >> (c * 16 + (i >> 1)) & 1)) r[c][i] = 0xff800000u;
          }
          counts |= full || (valid.w[0] | valid.w[1]);
          float t4[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) t4[c] = fmaxf(__uint_as_float(r[c >> 1][(c & 1) * 16]), __uint_as_float(r[c >> 1][(c & 1) * 16 + 1]));
#pragma unroll
          for (int i = 2; i < 16; i += 2)
#pragma unroll
            for (int c = 0; c < 4; ++c) t4[c] = max3f(t4[c], __uint_as_float(r[c >> 1][(c & 1) * 16 + i]), __uint_as_float(r[c >> 1][(c & 1) * 16 + i + 1]));
          const float m_new = fmaxf(m_ref, fmaxf(max3f(t4[0], t4[1], t4[2]), t4[3]));
          const bool need = (m_new - m_ref) * sl2 > LAZY_LOG2;          // (no: NaN, where no key has counted yet)
          if (__any_sync(0xffffffffu, need)) {
            if (first > from) {
              // O is rescaled in place, behind the product of the tile before: it is done when the next scores are, which were asked for behind
              // it, or, at an item's last tile, when the issuer says so.
              if (!(first + KEYS < keys ? mbar_wait_warp(&sh.s_full[sx][~n & 1], (n + 1) >> 1 & 1, abort_flag)
                                        : mbar_wait_warp(&sh.pv_done[sx], ends & 1, abort_flag))) { ok = false; break; }
              tc_fence_after();
              const float alpha = need ? ex2((m_ref - m_new) * sl2) : 1.f;
#pragma unroll
              for (int c = 0; c < HD / 16; ++c) {
                uint32_t v[16];
                tmem_ld16(o_addr + c * 16, v);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * alpha);
                tmem_st16(o_addr + c * 16, v);
              }
              l *= alpha;
            }
            if (need) { m_ref = m_new; mb = m_new * sl2; }
          }
          // P = 2^(s scale log2(e) - m) as bf16 over the scores; the row's sum is of the unrounded ones.  (What the product takes: 1.3e-3 to 1.7e-3 of the
          // result, beside 1.7e-3 by the result's own rounding.  Two bf16 parts of P would be a second product, where the products are the limit.)
          float2 sum2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          const float2 sl22 = make_float2(sl2, sl2), nmb2 = make_float2(-mb, -mb);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t pk[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 arg = __ffma2_rn(make_float2(__uint_as_float(r[c][2 * i]), __uint_as_float(r[c][2 * i + 1])), sl22, nmb2);
              const float2 pp = make_float2(ex2(arg.x), ex2(arg.y));
              sum2[i & 1] = __fadd2_rn(sum2[i & 1], pp);
              pk[i] = bf16_pair(__float_as_uint(pp.x), __float_as_uint(pp.y));
            }
            tmem_st16(at + c * 16, pk);
          }
          l += (sum2[0].x + sum2[1].x) + (sum2[0].y + sum2[1].y);
          tmem_wait_st();
        }
        tc_fence_before();
        mbar_arrive(&sh.p_full[sx][n & 1]);
      }
      if (!ok) break;
      if (some) {
        ok = mbar_wait_warp(&sh.o_full[sx], items++ & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        if (keys - from > KEYS) {                           // (the last values: the issuer)
          if (row == 0) mbar_arrive(&sh.v_empty[vp.back(2)]);
          ++ends;
        }
      }
      // (worked out again: kept through the loop it would take registers from the scores)
      int again = it, h0, n0;
      asm volatile("" : "+r"(again));
      const Item x = item_of(P, again);
      cx_place(D, x.g, x.tile + sx, h0, n0);
      const int row_h = D.by_bn(row), row_n = row - row_h * D.bn;
      const bool here = row_h < D.bh && n0 + row_n < D.N;
      const float inv = 1.f / l;
      const long long at = ((long long)x.b * D.H + h0 + row_h) * D.N + n0 + row_n;
      const float lse2 = counts ? mb + log2f(l) : -INFINITY;
      if (P.splits > 1) {
        const long long pat = (long long)x.part * D.B * D.H * D.N + at;
        if (here) P.part_lse[pat] = lse2;
        if (some && work) {
          float* to = P.part + pat * D.d;
#pragma unroll 1
          for (int c = 0; c < HD / 32; ++c) {
            uint32_t r[32];
            tmem_ld32(o_addr + c * 32, r);
            tmem_wait_ld();
            if (here && counts) {
#pragma unroll
              for (int v4 = 0; v4 < 8; ++v4)
                if (c * 32 + v4 * 4 < D.d)
                  *(float4*)(to + c * 32 + v4 * 4) = make_float4(__uint_as_float(r[v4 * 4]) * inv, __uint_as_float(r[v4 * 4 + 1]) * inv,
                                                                 __uint_as_float(r[v4 * 4 + 2]) * inv, __uint_as_float(r[v4 * 4 + 3]) * inv);
            }
          }
        }
      } else {
        if (P.lse && here) P.lse[at] = lse2 * 0.69314718055994531f;
        if (staged >= 1) {                                  // the item before has left the stage
          if (row == 0) { bulk_wait_read0(); mbar_arrive(&sh.sent[sx]); }
          ok = mbar_wait_warp(&sh.sent[sx], (staged - 1) & 1, abort_flag);
          if (!ok) break;
        }
#pragma unroll
        for (int c = 0; c < HD / 32; ++c) {
          uint32_t r[32];
          if (some) {
            tmem_ld32(o_addr + c * 32, r);
            tmem_wait_ld();
          }
          if (!counts) {
#pragma unroll
            for (int i = 0; i < 32; ++i) r[i] = 0;
          }
          cx_stage(stage + (c / 2) * HALF_BYTES, row, c & 1, r, counts ? inv : 1.f);
        }
        fence_proxy_async();
        mbar_arrive(&sh.staged[sx]);
        if (quarter == 0) {
          ok = mbar_wait_warp(&sh.staged[sx], staged & 1, abort_flag);
          if (!ok) break;
          if (row == 0) {
            tma_store_4d(stage, &map_o, 0, n0, h0, x.b);
            if (HALVES > 1) tma_store_4d(stage + HALF_BYTES, &map_o, 64, n0, h0, x.b);
            bulk_commit();
          }
        }
        ++staged;
      }
      if (some) {
        tc_fence_before();
        mbar_arrive(&sh.o_empty[sx]);
      }
    }
    if (row == 0) bulk_wait0();
  }

  // ------------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (sh.abort_flag) {
    if (threadIdx.x == 0) atomicExch(D.status, FF_ERR_TIMEOUT | 0x100);
    // let copies that were already issued land before the shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000) { }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tm, 512);
  }
}

// Joins the parts of the keys: a row's outputs weighted by 2^(lse of the part - the largest of them).  A warp has a row.
struct JoinParams { const float *part, *lse; float* lse_out; long long rows; int parts, H, N, d; char* out; long long sb, sh, sn; };
__global__ void __launch_bounds__(256) cross_join_kernel(const __grid_constant__ JoinParams P) {
  ff_pdl_wait();
  const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (row >= P.rows) return;
  float m = -INFINITY;
  for (int s = 0; s < P.parts; ++s) m = fmaxf(m, P.lse[s * P.rows + row]);
  if (m == -INFINITY) m = 0.f;                              // (no key counts, or a NaN, which stays one)
  float total = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = 0; s < P.parts; ++s) {
    const float w = exp2f(P.lse[s * P.rows + row] - m);
    if (w == 0.f) continue;                                 // (parts without keys have written nothing)
    total += w;
    if (lane * 4 < P.d) {
      const float4 v = *(const float4*)(P.part + (s * P.rows + row) * P.d + lane * 4);
      o.x += w * v.x; o.y += w * v.y; o.z += w * v.z; o.w += w * v.w;
    }
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  const long long n = row % P.N, bh = row / P.N;
  if (lane * 4 < P.d) {
    char* to = P.out + bh / P.H * P.sb + bh % P.H * P.sh + n * P.sn + lane * 8;
    *(uint2*)to = make_uint2(bf16_pair(__float_as_uint(o.x * inv), __float_as_uint(o.y * inv)),
                             bf16_pair(__float_as_uint(o.z * inv), __float_as_uint(o.w * inv)));
  }
  if (P.lse_out && lane == 0) P.lse_out[row] = total == 0.f ? -INFINITY : (m + log2f(total)) * 0.69314718055994531f;
}

ff_status_t fail(ff_cross_attention* h, ff_status_t code, const char* msg) {
  if (h) snprintf(h->err, sizeof h->err, "%s", msg);
  else ff_set_thread_error(msg);
  return code;
}
ff_status_t cuda_fail(ff_cross_attention* h, cudaError_t e) {
  char msg[256];
  snprintf(msg, sizeof msg, "CUDA error: %s", cudaGetErrorString(e));
  return fail(h, FF_ERR_CUDA, msg);
}
#define CX_CUDA(h, call)                                   \
  do {                                                     \
    const cudaError_t e__ = (call);                        \
    if (e__ != cudaSuccess) return cuda_fail((h), e__);    \
  } while (0)

// How queries are laid out in tiles.
void shape_of(const ff_cross_attention_config_t& c, int64_t batch, int64_t queries, int64_t keys, CrossDims* D) {
  *D = CrossDims{};
  D->B = (int)batch; D->H = c.heads; D->G = c.kv_heads; D->group = c.heads / c.kv_heads;
  D->N = (int)queries; D->K = (int)keys; D->d = c.head_dim;
  D->bn = TILE; D->bh = 1;
  if (queries >= 1 && queries <= TILE / 2)
    for (int n = 2; n <= D->group && n * queries <= TILE; ++n)
      if (D->group % n == 0) { D->bn = (int)queries; D->bh = n; }
  D->n_tiles = (int)((queries + D->bn - 1) / D->bn);
  D->tiles = D->n_tiles * (D->group / D->bh);
  D->by_bn = cx_div(D->bn); D->by_n_tiles = cx_div(D->n_tiles); D->by_tiles = cx_div(D->tiles); D->by_G = cx_div(D->G);
  D->scale = c.scale > 0.f ? c.scale : (float)(1.0 / sqrt((double)c.head_dim));
  D->sl2 = (float)(D->scale * 1.4426950408889634);
}
// Items of the forward launch: one or two tiles, all keys or parts of them, by the estimated time.  A tile of keys takes a pair of query
// tiles 1.2 us and a single one 0.75, an item 2 us more; joining the parts takes 3 us and what they write and read.  With lengths, which the host does
// not know, two thirds of the keys are expected, unevenly over the items, so that more and shorter ones are better.
struct Forward { int pair, pairs, splits; double us; };
Forward forward_of(const CrossDims& D, bool lengths) {
  Forward best = {1, D.tiles, 1, 1e30};
  const long long nk = (D.K + KEYS - 1) / KEYS;
  for (int pair = 1; pair <= 2; ++pair) {
    const int pairs = (D.tiles + pair - 1) / pair;
    for (int splits = 1; splits <= 64 && splits <= (nk > 1 ? nk : 1); ++splits) {
      const double items = (double)D.B * D.G * pairs * splits;
      if (splits > 1 && items > 4 * FF_B200_SMS) break;
      const double even = items / FF_B200_SMS, waves = !lengths ? ceil(even) : even * 2 / 3 + 0.35 > 1 ? even * 2 / 3 + 0.35 : 1;
      const double us = waves * ((double)((nk + splits - 1) / splits) * (pair == 2 ? 1.2 : 0.75) + 2) +
                        (splits > 1 ? 3 + (double)splits * D.B * D.H * D.N * D.d * 8 / 4e6 : 0);
      if (us < best.us) best = {pair, pairs, splits, us};
    }
  }
  return best;
}
size_t part_bytes(const CrossDims& D, int splits) { return (size_t)splits * D.B * D.H * D.N * D.d * sizeof(float); }
size_t part_lse_bytes(const CrossDims& D, int splits) { return (size_t)splits * D.B * D.H * D.N * sizeof(float); }

// Sizes that the kernels' indexes (items, and a grid more) and tensor maps take
constexpr double MOST_TILES = 2147483648.0 - 1024;
constexpr char MOST[] = "queries and keys must be at most 2^31 - 256, the 128-row tiles of all heads' queries (and of keys) below 2^31 - 1024, all values below 2^42";
bool too_large(const ff_cross_attention_config_t& c, int64_t batch, int64_t queries, int64_t keys) {
  if (batch > 0x7fffffff || queries > 0x7fffff00 || keys > 0x7fffff00) return true;
  const double bh = (double)batch * c.heads;
  return bh >= MOST_TILES || bh * (double)((queries + TILE - 1) / TILE) >= MOST_TILES || bh * (double)((keys + TILE - 1) / TILE) >= MOST_TILES ||
         bh * (double)queries * c.head_dim >= 4398046511104.0;
}

ff_status_t check_heads(ff_cross_attention* h, const ff_heads_t* t, int heads, int64_t batch, int64_t tokens, bool written, bool shared) {
  if (!t || !t->data) return fail(h, FF_ERR_INVALID_ARG, "a tensor is NULL");
  if (t->heads != heads) return fail(h, FF_ERR_INVALID_ARG, "a tensor has another number of heads than the handle");
  if (t->stride_batch < 0 || t->stride_head < 0 || t->stride_token < 0) return fail(h, FF_ERR_INVALID_ARG, "strides must not be negative");
  const bool sb = batch > 1, sh = heads > 1, sn = tokens > 1;
  if (written && ((sb && !t->stride_batch) || (sh && !t->stride_head) || (sn && !t->stride_token)))
    return fail(h, FF_ERR_INVALID_ARG, "an output's stride is 0: rows would be written over one another");
  if ((sn && !t->stride_token) || (!shared && ((sb && !t->stride_batch) || (sh && !t->stride_head))))
    return fail(h, FF_ERR_UNSUPPORTED, "a stride is 0 (k and v may have such a batch or head stride)");
  if ((((uintptr_t)t->data) & 15) || (sb && (t->stride_batch & 7)) || (sh && (t->stride_head & 7)) || (sn && (t->stride_token & 7)))
    return fail(h, FF_ERR_UNSUPPORTED, "addresses and strides must be multiples of 16 bytes");
  if ((sb && t->stride_batch >= (1ll << 38)) || (sh && t->stride_head >= (1ll << 38)) || (sn && t->stride_token >= (1ll << 38)))
    return fail(h, FF_ERR_UNSUPPORTED, "strides must be below 2^38 elements");
  return FF_OK;
}
ff_status_t check_call(ff_cross_attention* h, int64_t batch, int64_t queries, int64_t keys, void* ws, size_t ws_bytes, int training) {
  if (batch < 0 || queries < 0 || keys < 0) return fail(h, FF_ERR_INVALID_ARG, "batch, queries and keys must not be negative");
  if (too_large(h->cfg, batch, queries, keys)) return fail(h, FF_ERR_UNSUPPORTED, MOST);
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess || device != h->device) return fail(h, FF_ERR_INVALID_ARG, "the handle belongs to another device than the current one");
  const int64_t sizes[4] = {batch, queries, keys, training};
  if (memcmp(sizes, h->sizes, sizeof sizes)) {               // (estimates that take a microsecond)
    ff_cross_attention_workspace_bytes(&h->cfg, batch, queries, keys, training, &h->need);
    memcpy(h->sizes, sizes, sizeof sizes);
  }
  const size_t need = h->need;
  if (need && (!ws || ws_bytes < need)) return fail(h, FF_ERR_WORKSPACE, "the workspace is missing or smaller than ff_cross_attention_workspace_bytes");
  if (need && (((uintptr_t)ws) & 255)) return fail(h, FF_ERR_WORKSPACE, "the workspace must be 256-byte aligned");
  return FF_OK;
}
void keys_of(CrossDims* D, const ff_cross_attention* h, const ff_heads_t* q, const ff_heads_t* k, const ff_heads_t* v, const int32_t* lengths, const uint8_t* mask) {
  const ff_heads_t* t[3] = {q, k, v};
  for (int i = 0; i < 3; ++i) { D->once[i][0] = t[i]->stride_batch != 0 || D->B == 1; D->once[i][1] = t[i]->stride_head != 0 || t[i]->heads == 1; }
  D->lengths = lengths; D->mask = mask; D->status = h->status;
}

}  // namespace

bool cx_map(CUtensorMap* map, const ff_heads_t* t, int64_t batch, int64_t tokens, int d, int rows, int heads) {
  // (a stride that no second element uses may be anything: the map gets one that it takes; rows shared by all: extent 1)
  const bool sb = batch > 1 && t->stride_batch, sh = t->heads > 1 && t->stride_head;
  const cuuint64_t row = ((cuuint64_t)d * 2 + 15) / 16 * 16;
  const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)tokens, sh ? (cuuint64_t)t->heads : 1, sb ? (cuuint64_t)batch : 1};
  const cuuint64_t strides[3] = {tokens > 1 ? (cuuint64_t)t->stride_token * 2 : row, sh ? (cuuint64_t)t->stride_head * 2 : row,
                                 sb ? (cuuint64_t)t->stride_batch * 2 : row};
  const cuuint32_t box[4] = {64, (cuuint32_t)rows, (cuuint32_t)heads, 1};
  return ff_encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, t->data, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

extern "C" ff_status_t ff_cross_attention_validate(const ff_cross_attention_config_t* c) {
  if (!c) return fail(nullptr, FF_ERR_INVALID_ARG, "cfg is NULL");
  if (c->head_dim < 1 || c->heads < 1 || c->kv_heads < 1) return fail(nullptr, FF_ERR_INVALID_ARG, "head_dim, heads and kv_heads must be positive");
  if (c->heads % c->kv_heads) return fail(nullptr, FF_ERR_INVALID_ARG, "heads must be a multiple of kv_heads");
  // (times log2(e), as the kernels count, it is finite too)
  if (!(c->scale >= 0.f && c->scale < 2.3e38f)) return fail(nullptr, FF_ERR_INVALID_ARG, "scale must be positive and below 2.3e38, or 0 for 1 / sqrt(head_dim)");
  if (c->head_dim % 8 || c->head_dim > 128) return fail(nullptr, FF_ERR_UNSUPPORTED, "head_dim must be a multiple of 8 and at most 128");
  if (c->heads > 65536) return fail(nullptr, FF_ERR_UNSUPPORTED, "at most 65536 heads are supported");
  return FF_OK;
}

extern "C" ff_status_t ff_cross_attention_workspace_bytes(const ff_cross_attention_config_t* c, int64_t batch, int64_t queries, int64_t keys,
                                                          int32_t training, size_t* bytes) {
  const ff_status_t s = ff_cross_attention_validate(c);
  if (s != FF_OK) return s;
  if (!bytes || batch < 0 || queries < 0 || keys < 0) return fail(nullptr, FF_ERR_INVALID_ARG, "bytes is NULL, or batch, queries or keys negative");
  if (too_large(*c, batch, queries, keys)) return fail(nullptr, FF_ERR_UNSUPPORTED, MOST);
  *bytes = 0;
  if (batch == 0 || (queries == 0 && !training)) return FF_OK;
  CrossDims D;
  shape_of(*c, batch, queries, keys, &D);
  if (training) {
    *bytes = cx_backward_bytes(D);
  } else {                                                   // (whichever kernel runs)
    const int a = forward_of(D, false).splits, b = forward_of(D, true).splits, most = a > b ? a : b;      // (whether there are lengths, the call says)
    if (most > 1) *bytes = part_bytes(D, most) + part_lse_bytes(D, most);
  }
  return FF_OK;
}

extern "C" ff_status_t ff_cross_attention_create(const ff_cross_attention_config_t* cfg, ff_cross_attention_t** out) {
  if (!out) return fail(nullptr, FF_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  const ff_status_t s = ff_cross_attention_validate(cfg);
  if (s != FF_OK) return s;
  ff_cross_attention* h = new (std::nothrow) ff_cross_attention();
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "out of host memory");
  h->cfg = *cfg;
  h->sizes[0] = -1;
  cudaError_t e = cudaGetDevice(&h->device);
  for (const void* kernel : {(const void*)cross_forward_kernel<128>, (const void*)cross_forward_kernel<64>})
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM);
  if (e == cudaSuccess) e = cx_few_init();
  if (e == cudaSuccess) e = cx_backward_init();
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

extern "C" ff_status_t ff_cross_attention_destroy(ff_cross_attention_t* h) {
  if (h) {
    if (h->status) cudaFree(h->status);
    delete h;
  }
  return FF_OK;
}

extern "C" const char* ff_cross_attention_last_error(const ff_cross_attention_t* h) { return h ? h->err : ff_last_error(nullptr); }

extern "C" ff_status_t ff_cross_attention_device_status(ff_cross_attention_t* h, void* stream) {
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "the handle is NULL");
  int word = 0;
  cudaStream_t st = (cudaStream_t)stream;
  CX_CUDA(h, cudaMemcpyAsync(&word, h->status, sizeof word, cudaMemcpyDeviceToHost, st));
  CX_CUDA(h, cudaStreamSynchronize(st));
  if (!word) return FF_OK;
  CX_CUDA(h, cudaMemsetAsync(h->status, 0, sizeof word, st));
  CX_CUDA(h, cudaStreamSynchronize(st));
  return fail(h, word & 255, "a device-side wait expired");
}

extern "C" ff_status_t ff_cross_attention_forward(ff_cross_attention_t* h, int64_t batch, int64_t queries, int64_t keys, const ff_heads_t* q,
                                                  const ff_heads_t* k, const ff_heads_t* v, const int32_t* lengths, const uint8_t* mask,
                                                  const ff_heads_t* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "the handle is NULL");
  ff_status_t s = check_call(h, batch, queries, keys, ws, ws_bytes, 0);
  if (s != FF_OK) return s;
  if (batch == 0 || queries == 0) return FF_OK;
  const ff_cross_attention_config_t& c = h->cfg;
  const ff_heads_t none = {h->status, 8, 8, 8, c.kv_heads};              // (no keys: no row is read)
  if (keys == 0) k = v = &none;
  s = check_heads(h, q, c.heads, batch, queries, false, false);
  if (s == FF_OK) s = check_heads(h, k, c.kv_heads, batch, keys, false, true);
  if (s == FF_OK) s = check_heads(h, v, c.kv_heads, batch, keys, false, true);
  if (s == FF_OK) s = check_heads(h, out, c.heads, batch, queries, true, false);
  if (s != FF_OK) return s;
  if ((((uintptr_t)lse) | ((uintptr_t)lengths)) & 3) return fail(h, FF_ERR_INVALID_ARG, "lse and lengths must be 4-byte aligned");
  // (out is written while other tiles still read the keys and values, and queries of other places)
  if (keys && (out->data == k->data || out->data == v->data)) return fail(h, FF_ERR_INVALID_ARG, "out lies over k or v");
  if (out->data == q->data && ((batch > 1 && out->stride_batch != q->stride_batch) || (c.heads > 1 && out->stride_head != q->stride_head) ||
                               (queries > 1 && out->stride_token != q->stride_token)))
    return fail(h, FF_ERR_INVALID_ARG, "out lies over q with other strides");
  cudaStream_t st = (cudaStream_t)stream;
  CrossParams P{};
  shape_of(c, batch, queries, keys, &P.dm);
  keys_of(&P.dm, h, q, k, v, lengths, mask);
  const Forward f = forward_of(P.dm, lengths != nullptr);
  // A few rows wait longer for a tile than that estimate says.  Few rows / tiles, us, one query: 1 head of 64, 16,000 keys 13 / 30, 64,000 46 / 39, 128,000
  // 88 / 50; 8 heads of 128, 16,000 keys 20 / 28, 64,000 62 / 63, 128,000 116 / 110; 32 on 8 of 128, 64,000 keys 62 / 83; 32 samples, 16 heads on 8 of 128,
  // 2000 keys 43 / 89 (with lengths from all of them to a quarter, where only the tiles' estimate counts fewer: 32 / 74).  Near the border the slower one
  // may be chosen: 4 heads of 128, 16,000 keys 27 in place of 19, 1 of 64, 32,000 keys 33 in place of 22.
  if (cx_few_us(P.dm) < 1.3 * f.us + 4) {
    CX_CUDA(h, cx_few_forward(P.dm, q, k, v, out, lse, st));
    return FF_OK;
  }
  P.pair = f.pair; P.pairs = f.pairs; P.splits = f.splits; P.by_pairs = cx_div(f.pairs); P.by_splits = cx_div(f.splits);
  const long long items = (long long)P.dm.B * P.dm.G * f.pairs * f.splits;
  P.items = (int)items;
  P.lse = lse;
  P.part = (float*)ws;
  P.part_lse = (float*)((char*)ws + part_bytes(P.dm, f.splits));
  CUtensorMap mq, mk, mv, mo;
  const int64_t kn = keys > 0 ? keys : 1;
  if (!cx_map(&mq, q, batch, queries, c.head_dim, P.dm.bn, P.dm.bh) || !cx_map(&mk, k, keys > 0 ? batch : 1, kn, c.head_dim, KEYS, 1) ||
      !cx_map(&mv, v, keys > 0 ? batch : 1, kn, c.head_dim, KEYS, 1) || !cx_map(&mo, out, batch, queries, c.head_dim, P.dm.bn, P.dm.bh))
    return fail(h, FF_ERR_CUDA, "could not encode the tensor maps");
  const dim3 grid((unsigned)(P.items < FF_B200_SMS ? P.items : FF_B200_SMS));
  const auto kernel = c.head_dim > 64 ? cross_forward_kernel<128> : cross_forward_kernel<64>;
  CX_CUDA(h, ff_launch(kernel, grid, dim3(THREADS), SMEM, st, mq, mk, mv, mo, P));
  if (f.splits > 1) {
    JoinParams J{P.part, P.part_lse, lse, (long long)batch * c.heads * queries, f.splits, c.heads, (int)queries, c.head_dim, (char*)out->data,
                 (long long)out->stride_batch * 2, (long long)out->stride_head * 2, (long long)out->stride_token * 2};
    CX_CUDA(h, ff_launch(cross_join_kernel, dim3((unsigned)((J.rows + 7) / 8)), dim3(256), 0, st, J));
  }
  return FF_OK;
}

extern "C" ff_status_t ff_cross_attention_backward(ff_cross_attention_t* h, int64_t batch, int64_t queries, int64_t keys, const ff_heads_t* q,
                                                   const ff_heads_t* k, const ff_heads_t* v, const int32_t* lengths, const uint8_t* mask,
                                                   const ff_heads_t* out, const float* lse, const ff_heads_t* dout, const ff_heads_t* dq,
                                                   const ff_heads_t* dk, const ff_heads_t* dv, void* ws, size_t ws_bytes, void* stream) {
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "the handle is NULL");
  ff_status_t s = check_call(h, batch, queries, keys, ws, ws_bytes, 1);
  if (s != FF_OK) return s;
  if (!dk != !dv) return fail(h, FF_ERR_INVALID_ARG, "dk and dv are made together, or neither is");
  if (batch == 0 || (!dq && !dk)) return FF_OK;
  const ff_cross_attention_config_t& c = h->cfg;
  const ff_heads_t none = {h->status, 8, 8, 8, c.kv_heads}, no_query = {h->status, 8, 8, 8, c.heads};   // (no rows: none is read)
  if (keys == 0) k = v = &none;
  if (queries == 0) q = out = dout = &no_query;
  if (!(queries == 0 || lse)) return fail(h, FF_ERR_INVALID_ARG, "lse is NULL");
  s = check_heads(h, q, c.heads, queries ? batch : 1, queries, false, false);
  if (s == FF_OK) s = check_heads(h, k, c.kv_heads, batch, keys, false, true);
  if (s == FF_OK) s = check_heads(h, v, c.kv_heads, batch, keys, false, true);
  if (s == FF_OK) s = check_heads(h, out, c.heads, queries ? batch : 1, queries, false, false);
  if (s == FF_OK) s = check_heads(h, dout, c.heads, queries ? batch : 1, queries, false, false);
  if (s == FF_OK && dq && queries) s = check_heads(h, dq, c.heads, batch, queries, true, false);
  if (s == FF_OK && dk && keys) s = check_heads(h, dk, c.kv_heads, batch, keys, true, false);
  if (s == FF_OK && dv && keys) s = check_heads(h, dv, c.kv_heads, batch, keys, true, false);
  if (s != FF_OK) return s;
  if ((((uintptr_t)lse) | ((uintptr_t)lengths)) & 3) return fail(h, FF_ERR_INVALID_ARG, "lse and lengths must be 4-byte aligned");
  // (dq is written while other tiles still read q, dout and out; dk and dv while others read k and v, and the other launch's inputs)
  const ff_heads_t *in[5] = {q, k, v, out, dout}, *made[3] = {queries ? dq : nullptr, keys ? dk : nullptr, keys ? dv : nullptr};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 5; ++j)
      if (made[i] && made[i]->data == in[j]->data) return fail(h, FF_ERR_INVALID_ARG, "a gradient lies over an input");
    for (int j = 0; j < i; ++j)
      if (made[i] && made[j] && made[i]->data == made[j]->data) return fail(h, FF_ERR_INVALID_ARG, "a gradient lies over another one");
  }
  CrossDims D;
  shape_of(c, batch, queries, keys, &D);
  keys_of(&D, h, q, k, v, lengths, mask);
  CX_CUDA(h, cx_backward(D, q, k, v, out, lse, dout, queries ? dq : nullptr, keys ? dk : nullptr, dv, ws, (cudaStream_t)stream));
  return FF_OK;
}
