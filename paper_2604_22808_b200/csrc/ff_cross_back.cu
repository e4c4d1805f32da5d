// Cross attention, backward pass.
//
//   P_ij = e^(scale q_i k_j - lse_i),  D_i = dout_i out_i,  dP = dout V^T,  dS = P (dP - D)
//   dq = scale dS K,   dk = scale dS^T Q,   dv = P^T dout        (dk, dv: sums over the queries of all heads of the group)
//
// Two launches, neither with atomics: one owns tiles of queries, walks over the keys and sums dq in tensor memory; the other
// owns tiles of keys, walks over the queries and sums dk and dv there.  Both make the scores again (7 products in place of the 5 that
// one launch would need), and in return every sum has one owner and one order.
//
// dq: a CTA takes a tile of queries (of a part of the keys, where tiles are few).
//   warp 0       TMA producer: Q, dout, out (with 128 channels into the stage), tiles of K (three places) and V (one, or two of 64 channels)
//   warp 1       tcgen05.mma issuer: S = Q K^T into two buffers in turns, dP = dout V^T
//   warp 2       zeros in rows of K whose keys do not count, in tiles that may hold such rows
//   warp 3       tcgen05.mma issuer: dQ += dS K (dS from tensor memory, K as an MN-major operand); sends dQ out of the stage
//   warps 4..11  a thread per query row and half of the keys: P, then dS as bf16 over the scores; D at the item's first tile, from dout
//                and out in shared memory.  (Warpgroups that took whole tiles in turns: 70 instead of 60 us for 16K queries, 6 heads of
//                128, 512 keys.)
//   tensor memory: S (twice), dP, dQ
//
// dk, dv: a CTA takes a tile of keys and a run of the query tiles of its group.
//   warp 0       TMA producer: K, V; tiles of Q and dout (two stages each)
//   warp 1       tcgen05.mma issuer: S^T = K Q^T, dP^T = V dout^T, dV += P^T dout, dK += dS^T Q, in the order dV[j], S[j+1], dK[j], dP[j+1]
//   warp 2       -lse and D of the tile's rows into shared memory
//   warps 4..11  a thread per key row and half of the queries: P^T and dS^T as bf16 over S^T and dP^T
//   tensor memory: S^T, dP^T, dV, dK
// A row of zeros where the key does not count keeps what stands in K and V there out of every sum.
// P and dS are rounded to bf16 where they enter a product, which takes no wider ones: 1.6e-3 to 1.8e-3 of dq, dk and dv, beside 1.7e-3 by their own
// rounding.  Two bf16 parts of each would be 10 products in place of 7, and the products are the limit.
#include "ff_cross.cuh"

using namespace sm100;

namespace {

constexpr int TILE = CX_TILE;
constexpr int TILE_BYTES = TILE * 128 * 2, HALF_BYTES = TILE_BYTES / 2;
constexpr int THREADS = 128 + 2 * 128;
constexpr float LOG2E = 1.4426950408889634f;

struct QueryParams {
  CrossDims dm;
  int splits, items;           // parts of the keys
  CxDiv by_splits;
  const float* lse;
  float* delta;                // [batch][heads][queries]: D, for the other launch
  float* part;                 // splits > 1: [part][batch][heads][tokens][d]
  char* dq; long long sb, sh, sn;   // and strides in bytes, for rows without keys
};
struct KeyParams {
  CrossDims dm;
  int key_tiles, chunks, items;  // parts of the query tiles
  CxDiv by_key_tiles, by_chunks;
  const float *lse, *delta;
  float *part_k, *part_v;      // chunks > 1: [part][batch][kv_heads][keys][d]
  char *dk, *dv;               // and strides in bytes, for tiles whose keys do not count
  long long k_sb, k_sh, k_sn, v_sb, v_sh, v_sn;
};

// ---- dq -------------------------------------------------------------------------------------------------------------------
struct QueryShared {
  uint64_t q_full[2], q_empty[2], o_full, d_full, staged, stage_free;
  uint64_t k_full[3], k_empty[3], k_raw[3], v_full[2], v_empty[2];
  float d[2][TILE];                                          // sums of either half of the channels
  uint64_t s_full[2], ds_full[2], dp_full, dp_empty, dq_full;
  uint32_t tmem_base;
  int abort_flag;
};
constexpr size_t QUERY_SMEM = 7 * TILE_BYTES + sizeof(QueryShared) + 1024;

struct QueryItem { int b, g, part, tile, keys, j0, j1; };
__device__ __forceinline__ QueryItem query_item(const QueryParams& P, int it) {
  QueryItem x;
  const int rest = P.dm.by_tiles(it);
  x.tile = it - rest * P.dm.tiles;
  const int bg = P.by_splits(rest);
  x.part = rest - bg * P.splits;
  x.b = P.dm.by_G(bg);
  x.g = bg - x.b * P.dm.G;
  x.keys = cx_keys(P.dm, x.b);
  const int nk = (x.keys + TILE - 1) / TILE;
  x.j0 = cx_first(nk, x.part, P.splits, P.by_splits);
  x.j1 = cx_first(nk, x.part + 1, P.splits, P.by_splits);
  return x;
}

template <int HD>
__global__ void __launch_bounds__(THREADS, 1)
cross_dq_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_dout, const __grid_constant__ CUtensorMap map_dq,
                const __grid_constant__ QueryParams P) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  constexpr int BYTES = TILE * HD * 2, NQ = HD == 64 ? 2 : 1;         // places of queries (with dout) and of values
  uint8_t *sQ = smem, *sG = sQ + NQ * BYTES, *sK = sG + NQ * BYTES, *sV = sK + 3 * BYTES, *stage = sV + NQ * BYTES;
  uint8_t* sO = HD == 64 ? stage + BYTES : stage;            // (128 channels leave no room beside the stage)
  static_assert((3 * NQ + 4) * BYTES + (HD == 64 ? BYTES : 0) <= 7 * TILE_BYTES, "");
  QueryShared& sh = *(QueryShared*)(smem + 7 * TILE_BYTES);
  const CrossDims& D = P.dm;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int HALVES = HD / 64;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.q_full[i], 1); mbar_init(&sh.q_empty[i], 1 + 8); mbar_init(&sh.v_full[i], 1); mbar_init(&sh.v_empty[i], 1); }
    mbar_init(&sh.o_full, 1);
    mbar_init(&sh.d_full, 256); mbar_init(&sh.staged, 256); mbar_init(&sh.stage_free, 1);
    for (int i = 0; i < 3; ++i) { mbar_init(&sh.k_full[i], 1); mbar_init(&sh.k_empty[i], 1); mbar_init(&sh.k_raw[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.s_full[i], 1); mbar_init(&sh.ds_full[i], 256); }
    mbar_init(&sh.dp_full, 1); mbar_init(&sh.dp_empty, 256); mbar_init(&sh.dq_full, 1);
    sh.abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&map_q); tma_prefetch_desc(&map_k); tma_prefetch_desc(&map_v);
    tma_prefetch_desc(&map_out); tma_prefetch_desc(&map_dout); tma_prefetch_desc(&map_dq);
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
        unsigned iter = 0, g = 0;
        bool ok = true;
        auto load_keys = [&](const QueryItem& x, int j) {
          const int st = g % 3;
          if (g >= 3) ok = mbar_wait(&sh.k_empty[st], (g / 3 - 1) & 1, abort_flag);
          if (!ok) return;
          uint64_t* full = cx_unclean<TILE>(D, x.keys, j) ? &sh.k_raw[st] : &sh.k_full[st];
          mbar_arrive_expect_tx(full, BYTES);
          cx_load(sK + st * BYTES, HALF_BYTES, HALVES, &map_k, full, j * TILE, x.g * D.once[1][1], x.b * D.once[1][0]);
        };
        auto load_values = [&](const QueryItem& x, int j) {
          const int vp = g % NQ;
          if (g >= NQ) ok = mbar_wait(&sh.v_empty[vp], (g / NQ - 1) & 1, abort_flag);
          if (!ok) return;
          mbar_arrive_expect_tx(&sh.v_full[vp], BYTES);
          cx_load(sV + vp * BYTES, HALF_BYTES, HALVES, &map_v, &sh.v_full[vp], j * TILE, x.g * D.once[2][1], x.b * D.once[2][0]);
          ++g;
        };
        for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
          const QueryItem x = query_item(P, it);
          if (x.j0 == x.j1) continue;
          int h0, n0;
          cx_place(D, x.g, x.tile, h0, n0);
          load_keys(x, x.j0);                                // (their place is free before that of the queries)
          const int qb = iter % NQ;
          if (ok && iter >= NQ) ok = mbar_wait(&sh.q_empty[qb], (iter / NQ - 1) & 1, abort_flag);
          if (!ok) break;
          mbar_arrive_expect_tx(&sh.q_full[qb], 2 * q_bytes);
          cx_load(sQ + qb * BYTES, HALF_BYTES, HALVES, &map_q, &sh.q_full[qb], n0, h0 * D.once[0][1], x.b * D.once[0][0]);
          cx_load(sG + qb * BYTES, HALF_BYTES, HALVES, &map_dout, &sh.q_full[qb], n0, h0, x.b);
          load_values(x, x.j0);
          if (it + (int)gridDim.x < P.items) {               // what the next item reads first, from memory into L2
            const QueryItem y = query_item(P, it + gridDim.x);
            int h1, n1;
            cx_place(D, y.g, y.tile, h1, n1);
            cx_prefetch(HALVES, &map_q, n1, h1 * D.once[0][1], y.b * D.once[0][0]);
            cx_prefetch(HALVES, &map_dout, n1, h1, y.b);
            cx_prefetch(HALVES, &map_out, n1, h1, y.b);
          }
          // (behind the first keys and values: their place may be the stage, and still be on its way out)
          if (ok && iter >= 1) ok = mbar_wait(HD == 64 ? &sh.d_full : &sh.stage_free, (iter - 1) & 1, abort_flag);
          if (!ok) break;
          mbar_arrive_expect_tx(&sh.o_full, q_bytes);
          cx_load(sO, HALF_BYTES, HALVES, &map_out, &sh.o_full, n0, h0, x.b);
          for (int j = x.j0 + 1; j < x.j1 && ok; ++j) {
            load_keys(x, j);
            if (ok) load_values(x, j);
          }
          ++iter;
        }
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------------ MMA issuer
      const int sixteens = (D.d + 15) / 16;                  // of the channels: the products leave out what is zero behind them
      const uint32_t idesc_s = idesc_bf16_f32(TILE, TILE, false, false);
      const uint64_t q_desc = smem_desc_sw128(smem_u32(sQ), 16, 1024), g_desc = smem_desc_sw128(smem_u32(sG), 16, 1024);
      const uint64_t k_desc = smem_desc_sw128(smem_u32(sK), 16, 1024), v_desc = smem_desc_sw128(smem_u32(sV), 16, 1024);
      unsigned iter = 0, g = 0;
      bool ok = true;
      auto score = [&](uint32_t d_tm, uint64_t a, uint64_t b) {
#pragma unroll
        for (int k = 0; k < HALVES; ++k) umma_ss_up_to_4(d_tm, a + (uint64_t)(k * (HALF_BYTES >> 4)), b + (uint64_t)(k * (HALF_BYTES >> 4)), idesc_s, k > 0 ? 1u : 0u, sixteens - k * 4);
      };
      // (the buffer's dS has been read when the keys of two tiles before are free; their place was filled, so that turn has ended)
      auto issue_s = [&](unsigned gt) -> bool {
        if (!mbar_wait_warp(&sh.k_full[gt % 3], (gt / 3) & 1, abort_flag)) return false;
        if (gt >= 2 && !mbar_wait_warp(&sh.k_empty[(gt - 2) % 3], ((gt - 2) / 3) & 1, abort_flag)) return false;
        tc_fence_after();
        score(tm + (gt & 1) * 128, q_desc + (uint64_t)(iter % NQ * (BYTES >> 4)), k_desc + (uint64_t)((gt % 3) * (BYTES >> 4)));
        umma_commit(&sh.s_full[gt & 1]);
        return true;
      };
      auto issue_dp = [&](unsigned gt, bool last) -> bool {
        if (!mbar_wait_warp(&sh.v_full[gt % NQ], (gt / NQ) & 1, abort_flag)) return false;
        if (gt >= 1 && !mbar_wait_warp(&sh.dp_empty, (gt - 1) & 1, abort_flag)) return false;
        tc_fence_after();
        score(tm + 256, g_desc + (uint64_t)(iter % NQ * (BYTES >> 4)), v_desc + (uint64_t)(gt % NQ * (BYTES >> 4)));
        umma_commit(&sh.dp_full);
        umma_commit(&sh.v_empty[gt % NQ]);
        if (last) umma_commit(&sh.q_empty[iter % NQ]);
        return true;
      };
      for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
        const QueryItem x = query_item(P, it);
        const int nk = cx_uniform(x.j1 - x.j0);
        if (nk == 0) continue;
        ok = mbar_wait_warp(&sh.q_full[iter % NQ], (iter / NQ) & 1, abort_flag);
        for (int i = 0; i < nk && ok; ++i) ok = issue_s(g + i) && issue_dp(g + i, i + 1 == nk);
        g += nk;
        ++iter;
      }
    } else if (warp == 3) {
      // ------------------------------------------------------------------ dQ += dS K
      const uint32_t idesc_q = idesc_bf16_f32(TILE, (D.d + 15) / 16 * 16, false, true);
      const uint64_t km_desc = smem_desc_sw128(smem_u32(sK), HALF_BYTES, 1024);
      unsigned iter = 0, g = 0;
      bool ok = true;
      for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
        const QueryItem x = query_item(P, it);
        const int nk = cx_uniform(x.j1 - x.j0);
        if (nk == 0) continue;
        for (int i = 0; i < nk && ok; ++i, ++g) {
          ok = mbar_wait_warp(&sh.ds_full[g & 1], (g >> 1) & 1, abort_flag);
          if (!ok) break;
          tc_fence_after();
          const uint64_t kd = km_desc + (uint64_t)((g % 3) * (BYTES >> 4));
          umma_ts4(tm + 384, tm + (g & 1) * 128, kd, idesc_q, i == 0 ? 0u : 1u);
          umma_ts4(tm + 384, tm + (g & 1) * 128 + 64, kd + (uint64_t)(4 * (2048 >> 4)), idesc_q, 1u);    // (dS of either half of the keys)
          umma_commit(&sh.k_empty[g % 3]);
        }
        if (!ok) break;
        umma_commit(&sh.dq_full);
        // dQ has been read and lies in the stage: out with it, which takes less time than the next item's first dS
        ok = mbar_wait_warp(&sh.staged, iter & 1, abort_flag);
        if (ok && lane == 0) {
          if (P.splits == 1) {
            int h0, n0;
            cx_place(D, x.g, x.tile, h0, n0);
            tma_store_4d(stage, &map_dq, 0, n0, h0, x.b);
            if (HALVES > 1) tma_store_4d(stage + HALF_BYTES, &map_dq, 64, n0, h0, x.b);
            bulk_commit();
            bulk_wait_read0();
          }
          mbar_arrive(&sh.stage_free);
        }
        __syncwarp();
        ++iter;
      }
      if (lane == 0) bulk_wait0();
    } else if (warp == 2) {
      // ------------------------------------------------------------------ rows of K that do not count
      unsigned g = 0, raw[3] = {0, 0, 0};
      bool ok = true;
      for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
        const QueryItem x = query_item(P, it);
        for (int j = x.j0; j < x.j1 && ok; ++j, ++g) {
          if (!cx_unclean<TILE>(D, x.keys, j)) continue;
          const int st = g % 3;
          const CxValid valid = cx_valid(D, x.b, x.keys, j, lane);
          const unsigned n = st == 0 ? raw[0]++ : st == 1 ? raw[1]++ : raw[2]++;
          ok = mbar_wait_warp(&sh.k_raw[st], n & 1, abort_flag);
          if (!ok) break;
          cx_clean(sK + st * BYTES, HALF_BYTES, HALVES, valid.w, lane);
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.k_full[st]);
        }
      }
    }
  } else {
    reg_inc<200>();
    // ------------------------------------------------------------------ P and dS
    const int quarter = warp & 3;
    const int wg = (warp - 4) >> 2;
    const int row = quarter * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
    const uint32_t s_addr = tm + lane_addr + wg * 64, dp_addr = s_addr + 256, dq_addr = tm + lane_addr + 384;
    const int rows = D.bn * D.bh;
    const int row_h = D.by_bn(row), row_n = row - row_h * D.bn;
    unsigned iter = 0, g = 0;
    bool ok = true;
    auto nlse2_of = [&](int it) {                            // (rows that are not there: P = 0)
      if (it >= P.items) return 0.f;
      const QueryItem x = query_item(P, it);
      int h0, n0;
      cx_place(D, x.g, x.tile, h0, n0);
      return row < rows && n0 + row_n < D.N ? -P.lse[((long long)x.b * D.H + h0 + row_h) * D.N + n0 + row_n] * LOG2E : -INFINITY;
    };
    float next = nlse2_of(blockIdx.x);
    for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
      const QueryItem x = query_item(P, it);
      int h0, n0;
      cx_place(D, x.g, x.tile, h0, n0);
      const float nlse2 = next;
      const bool here = row < rows && n0 + row_n < D.N;
      const long long at = ((long long)x.b * D.H + h0 + row_h) * D.N + n0 + row_n;
      const int c0 = wg * (HD / 2);                          // at the end each warpgroup has half of the columns
      float* part = P.splits > 1 ? P.part + ((long long)x.part * D.B * D.H * D.N + at) * D.d : nullptr;
      if (x.j0 == x.j1) {                                    // no keys: zeros
        if (here)
          for (int c = c0; c < c0 + HD / 2 && c < D.d; c += 8) {
            if (part) {
              *(float4*)(part + c) = make_float4(0.f, 0.f, 0.f, 0.f);
              *(float4*)(part + c + 4) = make_float4(0.f, 0.f, 0.f, 0.f);
            } else {
              *(uint4*)(P.dq + x.b * P.sb + (h0 + row_h) * P.sh + (long long)(n0 + row_n) * P.sn + c * 2) = make_uint4(0, 0, 0, 0);
            }
          }
        next = nlse2_of(it + gridDim.x);
        continue;
      }
      float delta = 0.f;
      for (int j = x.j0; j < x.j1 && ok; ++j, ++g) {
        const bool full = !D.mask && (j + 1) * TILE <= x.keys;
        CxValid valid = {};
        if (!full) valid = cx_valid(D, x.b, x.keys, j, lane);
        const uint32_t at_s = s_addr + (g & 1) * 128;
        ok = mbar_wait_warp(&sh.s_full[g & 1], (g >> 1) & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        uint32_t p[2][32];
        tmem_ld32(at_s, p[0]);
        tmem_ld32(at_s + 32, p[1]);
        tmem_wait_ld();
        const float2 sl22 = make_float2(D.sl2, D.sl2), nl2 = make_float2(nlse2, nlse2);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 arg = __ffma2_rn(make_float2(__uint_as_float(p[c][2 * i]), __uint_as_float(p[c][2 * i + 1])), sl22, nl2);
            p[c][2 * i] = __float_as_uint(ex2(arg.x));
            p[c][2 * i + 1] = __float_as_uint(ex2(arg.y));
          }
        if (j == x.j0) {                                     // D = dout out of this row, half of the channels each
          ok = mbar_wait_warp(&sh.q_full[iter % NQ], (iter / NQ) & 1, abort_flag) && mbar_wait_warp(&sh.o_full, iter & 1, abort_flag);
          if (!ok) break;
          const uint8_t* g_row = sG + iter % NQ * BYTES + (HALVES > 1 ? wg * HALF_BYTES : 0) + row * 128;
          const uint8_t* o_row = sO + (HALVES > 1 ? wg * HALF_BYTES : 0) + row * 128;
          float2 d2 = make_float2(0.f, 0.f);
#pragma unroll
          for (int c = 0; c < 4 * HALVES; ++c) {
            const int off = ((HALVES > 1 ? c : wg * 4 + c) ^ (row & 7)) * 16;
            const uint4 a = *(const uint4*)(g_row + off), b = *(const uint4*)(o_row + off);
            const uint32_t av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
              d2 = __ffma2_rn(make_float2(__uint_as_float(av[i] << 16), __uint_as_float(av[i] & 0xffff0000u)),
                              make_float2(__uint_as_float(bv[i] << 16), __uint_as_float(bv[i] & 0xffff0000u)), d2);
          }
          sh.d[wg][row] = d2.x + d2.y;
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.q_empty[iter % NQ]);
          mbar_arrive(&sh.d_full);                           // (and out in the stage has been read by all)
          ok = mbar_wait_warp(&sh.d_full, iter & 1, abort_flag);
          if (!ok) break;
          delta = sh.d[0][row] + sh.d[1][row];
          if (wg == 0 && x.j0 == 0 && here) P.delta[at] = delta;
        }
        ok = mbar_wait_warp(&sh.dp_full, g & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        const float2 nd2 = make_float2(-delta, -delta);
        uint32_t r[2][32];
        tmem_ld32(dp_addr, r[0]);
        tmem_ld32(dp_addr + 32, r[1]);
        tmem_wait_ld();
        tc_fence_before();
        mbar_arrive(&sh.dp_empty);
        uint32_t pk[2][16];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 v = __fmul2_rn(make_float2(__uint_as_float(p[c][2 * i]), __uint_as_float(p[c][2 * i + 1])),
                                        __fadd2_rn(make_float2(__uint_as_float(r[c][2 * i]), __uint_as_float(r[c][2 * i + 1])), nd2));
            pk[c][i] = bf16_pair(__float_as_uint(v.x), __float_as_uint(v.y));
          }
        if (!full) {                                         // zeros, whatever stands in K and V there
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int bit = wg * 16 + c * 8 + (i >> 1);
              if (!(valid.w[(2 * i) & 3] >> bit & 1)) pk[c][i] &= 0xffff0000u;
              if (!(valid.w[(2 * i + 1) & 3] >> bit & 1)) pk[c][i] &= 0xffffu;
            }
        }
        tmem_st16(at_s, pk[0]);
        tmem_st16(at_s + 16, pk[1]);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&sh.ds_full[g & 1]);
      }
      if (!ok) break;
      next = nlse2_of(it + gridDim.x);
      ok = (HD == 128 || iter == 0 || mbar_wait_warp(&sh.stage_free, (iter - 1) & 1, abort_flag)) && mbar_wait_warp(&sh.dq_full, iter & 1, abort_flag);
      if (!ok) break;
      tc_fence_after();
      ++iter;
      for (int c = c0; c < c0 + HD / 2; c += 32) {
        uint32_t r[32];
        tmem_ld32(dq_addr + c, r);
        tmem_wait_ld();
        if (!part) {
          cx_stage(stage + (c / 64) * HALF_BYTES, row, (c % 64) / 32, r, D.scale);
        } else if (here) {
#pragma unroll
          for (int v = 0; v < 8; ++v)
            if (c + v * 4 < D.d)
              *(float4*)(part + c + v * 4) = make_float4(__uint_as_float(r[v * 4]) * D.scale, __uint_as_float(r[v * 4 + 1]) * D.scale,
                                                         __uint_as_float(r[v * 4 + 2]) * D.scale, __uint_as_float(r[v * 4 + 3]) * D.scale);
        }
      }
      tc_fence_before();
      fence_proxy_async();
      mbar_arrive(&sh.staged);
    }
  }

  // ------------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (sh.abort_flag) {
    if (threadIdx.x == 0) atomicExch(D.status, FF_ERR_TIMEOUT | 0x200);
    const long long t0 = clock64();                           // (copies that were already issued land first)
    while (clock64() - t0 < 2000000) { }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tm, 512);
  }
}

// ---- dk, dv ---------------------------------------------------------------------------------------------------------------
struct KeyShared {
  uint64_t kv_full, kv_empty, q_full[2], q_empty[2], g_full[2], g_empty[2], row_full[2], row_empty[2];
  uint64_t s_full, dp_full, p_full[2], ds_full[2], sum_full, sum_empty, staged[2];
  uint32_t tmem_base;
  int abort_flag;
  alignas(16) float nlse2[2][TILE];     // (read four at a time)
  alignas(16) float ndelta[2][TILE];
};
constexpr size_t KEY_SMEM = 6 * TILE_BYTES + sizeof(KeyShared) + 1024;

struct KeyItem { int b, g, chunk, j, keys, t0, t1; };
__device__ __forceinline__ KeyItem key_item(const KeyParams& P, int it) {
  KeyItem x;
  const int rest = P.by_key_tiles(it);
  x.j = it - rest * P.key_tiles;
  const int bg = P.by_chunks(rest);
  x.chunk = rest - bg * P.chunks;
  x.b = P.dm.by_G(bg);
  x.g = bg - x.b * P.dm.G;
  x.keys = cx_keys(P.dm, x.b);
  x.t0 = cx_first(P.dm.tiles, x.chunk, P.chunks, P.by_chunks);
  x.t1 = cx_first(P.dm.tiles, x.chunk + 1, P.chunks, P.by_chunks);
  if (x.j * TILE >= x.keys) x.t1 = x.t0;                     // no key of the tile counts
  return x;
}

template <int HD>
__global__ void __launch_bounds__(THREADS, 1)
cross_dkv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const __grid_constant__ CUtensorMap map_dout, const __grid_constant__ CUtensorMap map_dk, const __grid_constant__ CUtensorMap map_dv,
                 const __grid_constant__ KeyParams P) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *sK = smem, *sV = smem + TILE_BYTES, *sQ = smem + 2 * TILE_BYTES, *sG = smem + 4 * TILE_BYTES;   // Q, dout: two stages
  KeyShared& sh = *(KeyShared*)(smem + 6 * TILE_BYTES);
  const CrossDims& D = P.dm;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int HALVES = HD / 64;
  const int rows = D.bn * D.bh;

  if (threadIdx.x == 0) {
    mbar_init(&sh.kv_full, 1); mbar_init(&sh.kv_empty, 2);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], 1); mbar_init(&sh.q_empty[i], 1); mbar_init(&sh.g_full[i], 1); mbar_init(&sh.g_empty[i], 1);
      mbar_init(&sh.row_full[i], 32); mbar_init(&sh.row_empty[i], 8);
      mbar_init(&sh.p_full[i], 128); mbar_init(&sh.ds_full[i], 128); mbar_init(&sh.staged[i], 128);
    }
    mbar_init(&sh.s_full, 1); mbar_init(&sh.dp_full, 1); mbar_init(&sh.sum_full, 1); mbar_init(&sh.sum_empty, 256);
    sh.abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&map_q); tma_prefetch_desc(&map_k); tma_prefetch_desc(&map_v);
    tma_prefetch_desc(&map_dout); tma_prefetch_desc(&map_dk); tma_prefetch_desc(&map_dv);
  }
  // Rows that no copy reaches (tiles of few queries) meet probabilities of zero in the products: they have to be numbers.
  if (rows < TILE) {
    for (int i = threadIdx.x; i < 4 * TILE_BYTES / 16; i += THREADS)
      if ((i * 16) % HALF_BYTES / 128 >= rows) ((uint4*)sQ)[i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async();
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
        unsigned iter = 0, g = 0;
        bool ok = true;
        for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
          const KeyItem x = key_item(P, it);
          if (x.t0 == x.t1) continue;
          if (iter >= 1) ok = mbar_wait(&sh.kv_empty, (iter - 1) & 1, abort_flag);
          if (!ok) break;
          ++iter;
          mbar_arrive_expect_tx(&sh.kv_full, 2 * TILE * HD * 2);
          cx_load(sK, HALF_BYTES, HALVES, &map_k, &sh.kv_full, x.j * TILE, x.g * D.once[1][1], x.b * D.once[1][0]);
          cx_load(sV, HALF_BYTES, HALVES, &map_v, &sh.kv_full, x.j * TILE, x.g * D.once[2][1], x.b * D.once[2][0]);
          for (int t = x.t0; t < x.t1; ++t, ++g) {
            const int st = g & 1;
            int h0, n0;
            cx_place(D, x.g, t, h0, n0);
            if (g >= 2) ok = mbar_wait(&sh.q_empty[st], ((g >> 1) - 1) & 1, abort_flag);
            if (!ok) break;
            mbar_arrive_expect_tx(&sh.q_full[st], rows * HD * 2);
            cx_load(sQ + st * TILE_BYTES, HALF_BYTES, HALVES, &map_q, &sh.q_full[st], n0, h0 * D.once[0][1], x.b * D.once[0][0]);
            if (g >= 2) ok = mbar_wait(&sh.g_empty[st], ((g >> 1) - 1) & 1, abort_flag);
            if (!ok) break;
            mbar_arrive_expect_tx(&sh.g_full[st], rows * HD * 2);
            cx_load(sG + st * TILE_BYTES, HALF_BYTES, HALVES, &map_dout, &sh.g_full[st], n0, h0, x.b);
          }
        }
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------------ MMA issuer
      const int sixteens = (D.d + 15) / 16;                  // of the channels: the products leave out what is zero behind them
      const uint32_t idesc_s = idesc_bf16_f32(TILE, TILE, false, false);
      const uint32_t idesc_d = idesc_bf16_f32(TILE, sixteens * 16, false, true);
      const uint64_t k_desc = smem_desc_sw128(smem_u32(sK), 16, 1024), v_desc = smem_desc_sw128(smem_u32(sV), 16, 1024);
      const uint64_t q_desc = smem_desc_sw128(smem_u32(sQ), 16, 1024), g_desc = smem_desc_sw128(smem_u32(sG), 16, 1024);
      const uint64_t qm_desc = smem_desc_sw128(smem_u32(sQ), HALF_BYTES, 1024), gm_desc = smem_desc_sw128(smem_u32(sG), HALF_BYTES, 1024);
      unsigned iter = 0, g = 0;
      bool ok = true;
      auto score = [&](uint32_t d_tm, uint64_t a, uint64_t b) {
#pragma unroll
        for (int k = 0; k < HALVES; ++k) umma_ss_up_to_4(d_tm, a + (uint64_t)(k * (HALF_BYTES >> 4)), b + (uint64_t)(k * (HALF_BYTES >> 4)), idesc_s, k > 0 ? 1u : 0u, sixteens - k * 4);
      };
      auto issue_s = [&](unsigned gt) -> bool {              // (P^T in its place has been read by dV, issued before)
        const int st = gt & 1;
        if (!mbar_wait_warp(&sh.q_full[st], (gt >> 1) & 1, abort_flag)) return false;
        tc_fence_after();
        score(tm, k_desc, q_desc + (uint64_t)(st * (TILE_BYTES >> 4)));
        umma_commit(&sh.s_full);
        return true;
      };
      auto issue_dp = [&](unsigned gt) -> bool {
        const int st = gt & 1;
        if (!mbar_wait_warp(&sh.g_full[st], (gt >> 1) & 1, abort_flag)) return false;
        tc_fence_after();
        score(tm + 128, v_desc, g_desc + (uint64_t)(st * (TILE_BYTES >> 4)));
        umma_commit(&sh.dp_full);
        return true;
      };
      // D += A^T-tile times rows of the stage; either warpgroup's half of A (queries 0 .. 63 and 64 .. 127) lies in its own 64 columns
      auto issue_sum = [&](uint32_t d_tm, uint32_t a_tm, uint64_t b, uint64_t* half, unsigned parity, bool first) -> bool {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (!mbar_wait_warp(&half[h], parity, abort_flag)) return false;
          tc_fence_after();
          umma_ts4(d_tm, a_tm + h * 64, b + (uint64_t)(h * 4 * (2048 >> 4)), idesc_d, h == 0 && first ? 0u : 1u);
        }
        return true;
      };
      for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
        const KeyItem x = key_item(P, it);
        const int nt = cx_uniform(x.t1 - x.t0);
        if (nt == 0) continue;
        ok = mbar_wait_warp(&sh.kv_full, iter & 1, abort_flag) && issue_s(g) && issue_dp(g);
        if (ok && iter >= 1) ok = mbar_wait_warp(&sh.sum_empty, (iter - 1) & 1, abort_flag);
        for (int i = 0; i < nt && ok; ++i) {
          const unsigned gt = g + i;
          const int st = gt & 1;
          ok = issue_sum(tm + 256, tm, gm_desc + (uint64_t)(st * (TILE_BYTES >> 4)), sh.p_full, gt & 1, i == 0);
          if (!ok) break;
          if (i + 1 < nt) ok = issue_s(gt + 1);
          if (ok) ok = issue_sum(tm + 384, tm + 128, qm_desc + (uint64_t)(st * (TILE_BYTES >> 4)), sh.ds_full, gt & 1, i == 0);
          if (!ok) break;
          umma_commit(&sh.q_empty[st]);
          umma_commit(&sh.g_empty[st]);
          if (i + 1 < nt) ok = issue_dp(gt + 1);
        }
        if (ok) umma_commit(&sh.sum_full);
        g += nt;
        ++iter;
      }
    } else if (warp == 2) {
      // ------------------------------------------------------------------ -lse log2(e) and -D of the tile's rows
      unsigned g = 0;
      bool ok = true;
      for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
        const KeyItem x = key_item(P, it);
        for (int t = x.t0; t < x.t1 && ok; ++t, ++g) {
          const int st = g & 1;
          int h0, n0;
          cx_place(D, x.g, t, h0, n0);
          float l[4], d[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = lane + 32 * i, rh = D.by_bn(row), rn = row - rh * D.bn;
            const bool here = row < rows && n0 + rn < D.N;
            const long long at = ((long long)x.b * D.H + h0 + rh) * D.N + n0 + rn;
            l[i] = here ? -P.lse[at] * LOG2E : -INFINITY;    // (rows that are not there: P = 0)
            d[i] = here ? -P.delta[at] : 0.f;
          }
          if (g >= 2) ok = mbar_wait_warp(&sh.row_empty[st], ((g >> 1) - 1) & 1, abort_flag);
          if (!ok) break;
#pragma unroll
          for (int i = 0; i < 4; ++i) { sh.nlse2[st][lane + 32 * i] = l[i]; sh.ndelta[st][lane + 32 * i] = d[i]; }
          mbar_arrive(&sh.row_full[st]);
        }
      }
    }
  } else {
    reg_inc<200>();
    // ------------------------------------------------------------------ P^T and dS^T
    const int quarter = warp & 3;
    const int wg = (warp - 4) >> 2;
    const int row = quarter * 32 + lane;                     // the key
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
    const uint32_t s_addr = tm + lane_addr + wg * 64, dp_addr = s_addr + 128, sum_addr = tm + lane_addr + 256 + wg * 128;
    uint8_t* stage = wg ? sK : sV;                           // (free at the item's end) where dV, dK go
    const float factor = wg ? D.scale : 1.f;
    unsigned iter = 0, g = 0;
    bool ok = true;
    for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
      const KeyItem x = key_item(P, it);
      const int key = x.j * TILE + row;
      const bool here = key < D.K;
      const bool counts = key < x.keys && (!D.mask || __ldg(D.mask + (long long)x.b * D.K + key) != 0);
      const bool empty = x.t0 == x.t1, all = __all_sync(0xffffffffu, counts);
      for (int t = x.t0; t < x.t1 && ok; ++t, ++g) {
        const int st = g & 1;
        const float4 *nlse = (const float4*)(sh.nlse2[st] + wg * 64), *nd = (const float4*)(sh.ndelta[st] + wg * 64);
        ok = mbar_wait_warp(&sh.row_full[st], (g >> 1) & 1, abort_flag) && mbar_wait_warp(&sh.s_full, g & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        uint32_t p[2][32];
        tmem_ld32(s_addr, p[0]);
        tmem_ld32(s_addr + 32, p[1]);
        tmem_wait_ld();
        const float2 sl22 = make_float2(D.sl2, D.sl2);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 n4 = nlse[c * 8 + i];
            const float2 a = __ffma2_rn(make_float2(__uint_as_float(p[c][4 * i]), __uint_as_float(p[c][4 * i + 1])), sl22, make_float2(n4.x, n4.y));
            const float2 b = __ffma2_rn(make_float2(__uint_as_float(p[c][4 * i + 2]), __uint_as_float(p[c][4 * i + 3])), sl22, make_float2(n4.z, n4.w));
            p[c][4 * i] = __float_as_uint(ex2(a.x)); p[c][4 * i + 1] = __float_as_uint(ex2(a.y));
            p[c][4 * i + 2] = __float_as_uint(ex2(b.x)); p[c][4 * i + 3] = __float_as_uint(ex2(b.y));
          }
          if (!all)                                          // (rows of zeros, whatever stands in K)
#pragma unroll
            for (int i = 0; i < 32; ++i) p[c][i] = counts ? p[c][i] : 0u;
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) pk[i] = bf16_pair(p[c][2 * i], p[c][2 * i + 1]);
          tmem_st16(s_addr + c * 16, pk);
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&sh.p_full[wg]);
        ok = mbar_wait_warp(&sh.dp_full, g & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        uint32_t r[2][32];
        tmem_ld32(dp_addr, r[0]);
        tmem_ld32(dp_addr + 32, r[1]);
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 n4 = nd[c * 8 + i];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float2 v = __fmul2_rn(make_float2(__uint_as_float(p[c][4 * i + 2 * e]), __uint_as_float(p[c][4 * i + 2 * e + 1])),
                                          __fadd2_rn(make_float2(__uint_as_float(r[c][4 * i + 2 * e]), __uint_as_float(r[c][4 * i + 2 * e + 1])),
                                                     e ? make_float2(n4.z, n4.w) : make_float2(n4.x, n4.y)));
              pk[2 * i + e] = bf16_pair(__float_as_uint(v.x), __float_as_uint(v.y));
            }
          }
          if (!all)                                          // (... and in V)
#pragma unroll
            for (int i = 0; i < 16; ++i) pk[i] = counts ? pk[i] : 0u;
          tmem_st16(dp_addr + c * 16, pk);
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&sh.ds_full[wg]);
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.row_empty[st]);
      }
      if (!ok) break;
      if (!empty) {
        ok = mbar_wait_warp(&sh.sum_full, iter & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        ++iter;
      }
      if (P.chunks > 1 || empty) {
        float* part = P.chunks > 1 ? (wg ? P.part_k : P.part_v) + (((long long)x.chunk * D.B * D.G + (long long)x.b * D.G + x.g) * D.K + key) * D.d : nullptr;
        char* out = wg ? P.dk + x.b * P.k_sb + x.g * P.k_sh + (long long)key * P.k_sn : P.dv + x.b * P.v_sb + x.g * P.v_sh + (long long)key * P.v_sn;
        for (int c = 0; c < HD; c += 32) {
          uint32_t r[32];
          if (!empty) {
            tmem_ld32(sum_addr + c, r);
            tmem_wait_ld();
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) r[i] = 0;
          }
          if (here && part) {
#pragma unroll
            for (int v = 0; v < 8; ++v)
              if (c + v * 4 < D.d)
                *(float4*)(part + c + v * 4) = make_float4(__uint_as_float(r[v * 4]) * factor, __uint_as_float(r[v * 4 + 1]) * factor,
                                                           __uint_as_float(r[v * 4 + 2]) * factor, __uint_as_float(r[v * 4 + 3]) * factor);
          } else if (here) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
              if (c + v * 8 < D.d) *(uint4*)(out + (c + v * 8) * 2) = make_uint4(0, 0, 0, 0);
          }
        }
        if (!empty && row == 0) mbar_arrive(&sh.kv_empty);
      } else {
        for (int c = 0; c < HD; c += 32) {
          uint32_t r[32];
          tmem_ld32(sum_addr + c, r);
          tmem_wait_ld();
          cx_stage(stage + (c / 64) * HALF_BYTES, row, (c % 64) / 32, r, factor);
        }
        fence_proxy_async();
        mbar_arrive(&sh.staged[wg]);
        if (quarter == 0) ok = mbar_wait_warp(&sh.staged[wg], (iter - 1) & 1, abort_flag);
        if (!ok) break;
        if (row == 0) {
          const CUtensorMap* map = wg ? &map_dk : &map_dv;
          tma_store_4d(stage, map, 0, x.j * TILE, x.g, x.b);
          if (HALVES > 1) tma_store_4d(stage + HALF_BYTES, map, 64, x.j * TILE, x.g, x.b);
          bulk_commit();
          bulk_wait_read0();
          mbar_arrive(&sh.kv_empty);
        }
      }
      if (!empty) {
        tc_fence_before();
        mbar_arrive(&sh.sum_empty);
      }
    }
    if (row == 0) bulk_wait0();
  }

  // ------------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (sh.abort_flag) {
    if (threadIdx.x == 0) atomicExch(D.status, FF_ERR_TIMEOUT | 0x300);
    const long long t0 = clock64();                           // (copies that were already issued land first)
    while (clock64() - t0 < 2000000) { }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tm, 512);
  }
}

// ---- the small launches ---------------------------------------------------------------------------------------------------
struct Rows { char* p; long long sb, sh, sn; };              // strides in bytes
Rows rows_of(const ff_heads_t* t) { return Rows{(char*)t->data, (long long)t->stride_batch * 2, (long long)t->stride_head * 2, (long long)t->stride_token * 2}; }
__device__ __forceinline__ char* row_at(const Rows& r, long long row, int heads, int tokens) {
  const long long n = row % tokens, bh = row / tokens;
  return r.p + bh / heads * r.sb + bh % heads * r.sh + n * r.sn;
}

// Sums of parts [part][rows][d], in their order.  A warp has a row.
struct SumParams { const float* part[2]; Rows out[2]; long long rows; int parts, heads, tokens, d; };
__global__ void __launch_bounds__(256) cross_sum_kernel(const __grid_constant__ SumParams P) {
  ff_pdl_wait();
  const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int c = (threadIdx.x & 31) * 4;
  if (row >= P.rows || c >= P.d) return;
  const float* from = P.part[blockIdx.y] + row * P.d + c;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int i = 0; i < P.parts; ++i) {
    const float4 v = *(const float4*)(from + (long long)i * P.rows * P.d);
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  *(uint2*)(row_at(P.out[blockIdx.y], row, P.heads, P.tokens) + c * 2) =
      make_uint2(bf16_pair(__float_as_uint(s.x), __float_as_uint(s.y)), bf16_pair(__float_as_uint(s.z), __float_as_uint(s.w)));
}

// D alone, for calls that want no dq.  A warp has a row.
struct DeltaParams { Rows out, dout; float* delta; long long rows; int heads, tokens, d; };
__global__ void __launch_bounds__(256) cross_delta_kernel(const __grid_constant__ DeltaParams P) {
  ff_pdl_wait();
  const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (row >= P.rows) return;
  float d = 0.f;
  if (lane * 4 < P.d) {
    const uint2 a = *(const uint2*)(row_at(P.out, row, P.heads, P.tokens) + lane * 8), b = *(const uint2*)(row_at(P.dout, row, P.heads, P.tokens) + lane * 8);
    d = __uint_as_float(a.x << 16) * __uint_as_float(b.x << 16) + __uint_as_float(a.x & 0xffff0000u) * __uint_as_float(b.x & 0xffff0000u) +
        __uint_as_float(a.y << 16) * __uint_as_float(b.y << 16) + __uint_as_float(a.y & 0xffff0000u) * __uint_as_float(b.y & 0xffff0000u);
  }
#pragma unroll
  for (int m = 16; m; m >>= 1) d += __shfl_xor_sync(0xffffffffu, d, m);
  if (lane == 0) P.delta[row] = d;
}

// Parts by the estimated time: `items` of `steps` steps of 1.6 us, 3 us more for an item, joining the parts 3 us and what they write and read.
int parts_of(long long items, long long steps, double values) {
  int best = 1;
  double least = 1e30;
  for (int parts = 1; parts <= 64 && parts <= (steps > 1 ? steps : 1); ++parts) {
    if (parts > 1 && (double)items * parts > 8.0 * FF_B200_SMS) break;
    const double waves = (double)((items * parts + FF_B200_SMS - 1) / FF_B200_SMS);
    const double us = waves * ((double)((steps + parts - 1) / parts) * 1.6 + 3) + (parts > 1 ? 3 + parts * values * 8 / 4e6 : 0);
    if (us < least) { least = us; best = parts; }
  }
  return best;
}
struct Sizes { int key_tiles, splits, chunks; size_t delta, dq, dkv; };
size_t align256(size_t n) { return (n + 255) / 256 * 256; }
Sizes sizes_of(const CrossDims& D) {
  Sizes z;
  z.key_tiles = (D.K + TILE - 1) / TILE;
  const double qv = (double)D.B * D.H * D.N * D.d, kv = (double)D.B * D.G * D.K * D.d;
  z.splits = parts_of((long long)D.B * D.G * D.tiles, z.key_tiles, qv);
  z.chunks = parts_of((long long)D.B * D.G * z.key_tiles, D.tiles, 2 * kv);
  z.delta = align256((size_t)D.B * D.H * D.N * sizeof(float));
  z.dq = z.splits > 1 ? align256((size_t)z.splits * D.B * D.H * D.N * D.d * sizeof(float)) : 0;
  z.dkv = z.chunks > 1 ? align256((size_t)z.chunks * D.B * D.G * D.K * D.d * sizeof(float)) : 0;
  return z;
}

}  // namespace

cudaError_t cx_backward_init() {
  cudaError_t e = cudaFuncSetAttribute(cross_dq_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)QUERY_SMEM);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(cross_dq_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)QUERY_SMEM);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(cross_dkv_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)KEY_SMEM);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(cross_dkv_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)KEY_SMEM);
  return e;
}

size_t cx_backward_bytes(const CrossDims& D) {
  const Sizes z = sizes_of(D);
  return z.delta + z.dq + 2 * z.dkv;
}

// (the tensors have been checked; D.N or D.K may be 0: the rows there would be are then not read)
cudaError_t cx_backward(const CrossDims& D, const ff_heads_t* q, const ff_heads_t* k, const ff_heads_t* v, const ff_heads_t* out, const float* lse,
                        const ff_heads_t* dout, const ff_heads_t* dq, const ff_heads_t* dk, const ff_heads_t* dv, void* ws, cudaStream_t st) {
  const Sizes z = sizes_of(D);
  float* delta = (float*)ws;
  float *part_q = (float*)((char*)ws + z.delta), *part_k = (float*)((char*)ws + z.delta + z.dq), *part_v = (float*)((char*)ws + z.delta + z.dq + z.dkv);
  const int64_t kb = D.K > 0 ? D.B : 1, kn = D.K > 0 ? D.K : 1, qb = D.N > 0 ? D.B : 1, qn = D.N > 0 ? D.N : 1;
  CUtensorMap mq, mk, mv, mo, mg, mdq, mdk, mdv;
  if (!cx_map(&mq, q, qb, qn, D.d, D.bn, D.bh) || !cx_map(&mk, k, kb, kn, D.d, TILE, 1) || !cx_map(&mv, v, kb, kn, D.d, TILE, 1) ||
      !cx_map(&mo, out, qb, qn, D.d, D.bn, D.bh) || !cx_map(&mg, dout, qb, qn, D.d, D.bn, D.bh))
    return cudaErrorInvalidValue;
  cudaError_t e = cudaSuccess;
  if (dq) {
    if (!cx_map(&mdq, dq, D.B, D.N, D.d, D.bn, D.bh)) return cudaErrorInvalidValue;
    QueryParams P{};
    P.dm = D; P.splits = z.splits; P.by_splits = cx_div(z.splits);
    P.items = D.B * D.G * D.tiles * z.splits;
    P.lse = lse; P.delta = delta; P.part = part_q;
    const Rows r = rows_of(dq);
    P.dq = r.p; P.sb = r.sb; P.sh = r.sh; P.sn = r.sn;
    const dim3 grid((unsigned)(P.items < FF_B200_SMS ? P.items : FF_B200_SMS));
    e = D.d > 64 ? ff_launch(cross_dq_kernel<128>, grid, dim3(THREADS), QUERY_SMEM, st, mq, mk, mv, mo, mg, mdq, P)
                 : ff_launch(cross_dq_kernel<64>, grid, dim3(THREADS), QUERY_SMEM, st, mq, mk, mv, mo, mg, mdq, P);
    if (e == cudaSuccess && z.splits > 1) {
      const SumParams S{{part_q, part_q}, {r, r}, (long long)D.B * D.H * D.N, z.splits, D.H, D.N, D.d};
      e = ff_launch(cross_sum_kernel, dim3((unsigned)((S.rows + 7) / 8)), dim3(256), 0, st, S);
    }
  } else if (D.N > 0) {
    const DeltaParams P{rows_of(out), rows_of(dout), delta, (long long)D.B * D.H * D.N, D.H, D.N, D.d};
    e = ff_launch(cross_delta_kernel, dim3((unsigned)((P.rows + 7) / 8)), dim3(256), 0, st, P);
  }
  if (e != cudaSuccess || !dk || D.K == 0) return e;
  if (!cx_map(&mdk, dk, D.B, D.K, D.d, TILE, 1) || !cx_map(&mdv, dv, D.B, D.K, D.d, TILE, 1)) return cudaErrorInvalidValue;
  KeyParams P{};
  P.dm = D; P.key_tiles = z.key_tiles; P.chunks = z.chunks; P.by_key_tiles = cx_div(z.key_tiles); P.by_chunks = cx_div(z.chunks);
  P.items = D.B * D.G * z.key_tiles * z.chunks;
  P.lse = lse; P.delta = delta; P.part_k = part_k; P.part_v = part_v;
  const Rows rk = rows_of(dk), rv = rows_of(dv);
  P.dk = rk.p; P.k_sb = rk.sb; P.k_sh = rk.sh; P.k_sn = rk.sn;
  P.dv = rv.p; P.v_sb = rv.sb; P.v_sh = rv.sh; P.v_sn = rv.sn;
  const dim3 grid((unsigned)(P.items < FF_B200_SMS ? P.items : FF_B200_SMS));
  e = D.d > 64 ? ff_launch(cross_dkv_kernel<128>, grid, dim3(THREADS), KEY_SMEM, st, mq, mk, mv, mg, mdk, mdv, P)
               : ff_launch(cross_dkv_kernel<64>, grid, dim3(THREADS), KEY_SMEM, st, mq, mk, mv, mg, mdk, mdv, P);
  if (e == cudaSuccess && z.chunks > 1) {
    const SumParams S{{part_k, part_v}, {rk, rv}, (long long)D.B * D.G * D.K, z.chunks, D.G, D.K, D.d};
    e = ff_launch(cross_sum_kernel, dim3((unsigned)((S.rows + 7) / 8), 2), dim3(256), 0, st, S);
  }
  return e;
}
