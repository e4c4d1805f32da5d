// Cross attention to an encoder's states: forward pass and the C entry points.
//
//   out = softmax_j(scale q k_j) v,   lse = ln sum_j e^(scale q k_j),   over the keys j that count
//
// One pass over the keys with the running maximum m and sum l of the softmax (Milakov and Gimelshein, "Online normalizer
// calculation for softmax", 2018), scores in units of log2.
//
// A CTA takes items (sample, key head, one or two neighbouring tiles of queries, part of the keys); the two tiles, "streams" A and
// B, share every tile of keys and values, and while the softmax of one works the tensor core runs the products of the other.
//   warp 0       TMA producer: the query tiles, tiles of keys and values (two stages each)
//   warp 1       tcgen05.mma issuer: S_x = Q_x K^T (both from shared memory), O_x += P_x V (P from tensor memory), in the order
//                PV_A[j], QK_A[j+1], PV_B[j], QK_B[j+1]; owns the tensor memory
//   warp 2       zeros in rows of V whose keys do not count, in tiles that may hold such rows
//   warps 4..11  softmax: a thread per query row; P goes back to tensor memory as bf16 over the scores; O accumulates in tensor memory
//                and is rescaled only when a row's maximum grows by more than 2^8.  At the end O / l goes out through
//                shared memory by TMA.
// Tensor memory (512 columns): S/P of A, S/P of B, O of A, O of B.  Every wait is bounded; when one runs out the CTA raises
// FF_ERR_TIMEOUT in the handle's status word, takes no more work and returns.
#include <math.h>
#include <stdio.h>

#include <initializer_list>
#include <new>

#include "ff_cross.cuh"

using namespace sm100;

namespace {

constexpr int TILE = CX_TILE;
constexpr int TILE_BYTES = TILE * 128 * 2, HALF_BYTES = TILE_BYTES / 2;
constexpr int THREADS = 128 + 2 * 128;
constexpr float LAZY_LOG2 = 8.0f;

struct CrossParams {
  CrossDims dm;
  int pair, pairs, splits;     // tiles of an item (1 or 2), items of a key head of a sample, parts of the keys
  int items;
  float* lse;                  // or NULL
  float *part, *part_lse;      // splits > 1: [part][batch][heads][tokens][d] O / l, and the sums' log2
};

struct Shared {
  uint64_t q_full, q_empty, k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t v_raw[2];           // in place of v_full for a tile that has to be cleaned first
  uint64_t s_full[2], p_half[2], p_full[2], o_full[2], o_empty[2];      // per stream
  uint32_t tmem_base;
  int abort_flag;
};
constexpr size_t SMEM = 7 * TILE_BYTES + sizeof(Shared) + 1024;

struct Item { int b, g, part, tile, has_b, keys, j0, j1; };
__device__ __forceinline__ Item item_of(const CrossParams& P, int it) {
  Item x;
  int rest = it / P.pairs;
  x.tile = (it - rest * P.pairs) * P.pair;
  x.has_b = P.pair == 2 && x.tile + 1 < P.dm.tiles;
  const int bg = rest / P.splits;
  x.part = rest - bg * P.splits;
  x.b = bg / P.dm.G;
  x.g = bg - x.b * P.dm.G;
  x.keys = cx_keys(P.dm, x.b);
  const long long nk = (x.keys + TILE - 1) / TILE;
  x.j0 = (int)(nk * x.part / P.splits);
  x.j1 = (int)(nk * (x.part + 1) / P.splits);
  return x;
}

template <int HD>
__global__ void __launch_bounds__(THREADS, 1)
cross_forward_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                     const __grid_constant__ CUtensorMap map_o, const __grid_constant__ CrossParams P) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sQ = smem;                       // streams A and B
  uint8_t* sK = smem + 2 * TILE_BYTES;      // two stages
  uint8_t* sV = smem + 4 * TILE_BYTES;      // two stages
  uint8_t* sO = smem + 6 * TILE_BYTES;      // half a tile for either stream's output
  Shared& sh = *(Shared*)(smem + 7 * TILE_BYTES);
  const CrossDims& D = P.dm;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int HALVES = HD / 64;

  if (threadIdx.x == 0) {
    mbar_init(&sh.q_full, 1); mbar_init(&sh.q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.k_full[i], 1); mbar_init(&sh.k_empty[i], 1);
      mbar_init(&sh.v_full[i], 1); mbar_init(&sh.v_empty[i], 1); mbar_init(&sh.v_raw[i], 1);
      mbar_init(&sh.s_full[i], 1); mbar_init(&sh.p_half[i], 128); mbar_init(&sh.p_full[i], 128);
      mbar_init(&sh.o_full[i], 1); mbar_init(&sh.o_empty[i], 128);
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
        unsigned iter = 0, g = 0;
        bool ok = true;
        for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
          const Item x = item_of(P, it);
          if (x.j0 == x.j1) continue;
          if (iter >= 1) ok = mbar_wait(&sh.q_empty, (iter - 1) & 1, abort_flag);
          if (!ok) break;
          mbar_arrive_expect_tx(&sh.q_full, x.has_b ? 2 * q_bytes : q_bytes);
          for (int sx = 0; sx <= x.has_b; ++sx) {
            int h0, n0;
            cx_place(D, x.g, x.tile + sx, h0, n0);
            cx_load(sQ + sx * TILE_BYTES, HALF_BYTES, HALVES, &map_q, &sh.q_full, n0, h0 * D.once[0][1], x.b * D.once[0][0]);
          }
          ++iter;
          for (int j = x.j0; j < x.j1; ++j, ++g) {
            const int st = g & 1;
            if (g >= 2) ok = mbar_wait(&sh.k_empty[st], ((g >> 1) - 1) & 1, abort_flag);
            if (!ok) break;
            mbar_arrive_expect_tx(&sh.k_full[st], TILE * HD * 2);
            cx_load(sK + st * TILE_BYTES, HALF_BYTES, HALVES, &map_k, &sh.k_full[st], j * TILE, x.g * D.once[1][1], x.b * D.once[1][0]);
            if (g >= 2) ok = mbar_wait(&sh.v_empty[st], ((g >> 1) - 1) & 1, abort_flag);
            if (!ok) break;
            uint64_t* full = cx_unclean(D, x.keys, j) ? &sh.v_raw[st] : &sh.v_full[st];
            mbar_arrive_expect_tx(full, TILE * HD * 2);
            cx_load(sV + st * TILE_BYTES, HALF_BYTES, HALVES, &map_v, full, j * TILE, x.g * D.once[2][1], x.b * D.once[2][0]);
          }
        }
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------------ MMA issuer
      const uint32_t idesc_qk = idesc_bf16_f32(TILE, TILE, false, false);
      const uint32_t idesc_pv = idesc_bf16_f32(TILE, HD, false, true);
      unsigned iter = 0, g = 0;
      unsigned cp[2] = {0, 0};          // P phases consumed per stream
      unsigned ce[2] = {0, 0};          // items seen per stream (for the hand-back of O)
      bool ok = true;
      const uint64_t q_desc = smem_desc_sw128(smem_u32(sQ), 16, 1024), k_desc = smem_desc_sw128(smem_u32(sK), 16, 1024);
      const uint64_t v_desc = smem_desc_sw128(smem_u32(sV), HALF_BYTES, 1024);
      auto issue_qk = [&](int sx, unsigned gt, bool last, bool release_q) {
        const int st = gt & 1;
        const uint64_t qd = q_desc + (uint64_t)(sx * (TILE_BYTES >> 4)), kd = k_desc + (uint64_t)(st * (TILE_BYTES >> 4));
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          const uint64_t off = (uint64_t)(((k >> 2) * HALF_BYTES + (k & 3) * 32) >> 4);
          umma_ss(tm + sx * 128, qd + off, kd + off, idesc_qk, k > 0 ? 1u : 0u);
        }
        umma_commit(&sh.s_full[sx]);
        if (last) umma_commit(&sh.k_empty[st]);
        if (release_q) umma_commit(&sh.q_empty);
      };
      auto issue_pv = [&](int sx, unsigned gt, bool first, bool last, bool last_of_item) -> bool {
        const int st = gt & 1;
        if (!mbar_wait_warp(&sh.p_half[sx], cp[sx] & 1, abort_flag)) return false;
        if (first && ce[sx] >= 1 && !mbar_wait_warp(&sh.o_empty[sx], (ce[sx] - 1) & 1, abort_flag)) return false;
        tc_fence_after();
        const uint64_t vd = v_desc + (uint64_t)(st * (TILE_BYTES >> 4));
        const uint32_t p_tm = tm + sx * 128, d_tm = p_tm + 256;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (k == 4) {
            if (!mbar_wait_warp(&sh.p_full[sx], cp[sx] & 1, abort_flag)) return false;
            ++cp[sx];
            tc_fence_after();
          }
          umma_ts(d_tm, p_tm + k * 8, vd + (uint64_t)(k * (2048 >> 4)), idesc_pv, k == 0 && first ? 0u : 1u);
        }
        if (last_of_item) umma_commit(&sh.o_full[sx]);
        if (last) umma_commit(&sh.v_empty[st]);
        return true;
      };
      for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
        const Item x = item_of(P, it);
        if (x.j0 == x.j1) continue;
        ok = mbar_wait_warp(&sh.q_full, iter & 1, abort_flag) && mbar_wait_warp(&sh.k_full[g & 1], (g >> 1) & 1, abort_flag);
        if (!ok) break;
        ++iter;
        tc_fence_after();
        const int nk = x.j1 - x.j0;
        issue_qk(0, g, !x.has_b, nk == 1 && !x.has_b);
        if (x.has_b) issue_qk(1, g, true, nk == 1);
        for (int i = 0; i < nk && ok; ++i) {
          const unsigned gt = g + i;
          const bool more = i + 1 < nk;
          ok = mbar_wait_warp(&sh.v_full[gt & 1], (gt >> 1) & 1, abort_flag);
          for (int sx = 0; sx <= x.has_b && ok; ++sx) {
            const bool last = sx == x.has_b;
            ok = issue_pv(sx, gt, i == 0, last, !more);
            if (!ok || !more) continue;
            if (sx == 0) {
              ok = mbar_wait_warp(&sh.k_full[(gt + 1) & 1], ((gt + 1) >> 1) & 1, abort_flag);
              if (!ok) break;
              tc_fence_after();
            }
            issue_qk(sx, gt + 1, last, last && i + 2 == nk);
          }
        }
        g += nk;
        ce[0] += 1;
        if (x.has_b) ce[1] += 1;
      }
    } else if (warp == 2) {
      // ------------------------------------------------------------------ rows of V that do not count
      unsigned g = 0, raw[2] = {0, 0};                      // tiles; those cleaned, per stage
      bool ok = true;
      for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
        const Item x = item_of(P, it);
        for (int j = x.j0; j < x.j1 && ok; ++j, ++g) {
          if (!cx_unclean(D, x.keys, j)) continue;
          const int st = g & 1;
          const CxValid valid = cx_valid(D, x.b, x.keys, j, lane);
          ok = mbar_wait_warp(&sh.v_raw[st], raw[st]++ & 1, abort_flag);
          if (!ok) break;
          cx_clean(sV + st * TILE_BYTES, HALF_BYTES, HALVES, valid, lane);
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.v_full[st]);
        }
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
    uint8_t* stage = sO + sx * HALF_BYTES;
    const float sl2 = D.sl2;
    const int rows = D.bn * D.bh;
    const int row_h = row / D.bn, row_n = row - row_h * D.bn;
    unsigned cs = 0;                  // tiles of keys this stream has processed (phases of s_full / p_full)
    unsigned co = 0;                  // phases of o_full consumed: one per item with keys
    bool ok = true, staged = false;
    for (int it = blockIdx.x; it < P.items && ok; it += gridDim.x) {
      const Item x = item_of(P, it);
      if (sx == 1 && !x.has_b) continue;
      int h0, n0;
      cx_place(D, x.g, x.tile + sx, h0, n0);
      const bool here = row < rows && n0 + row_n < D.N;
      const bool work = __any_sync(0xffffffffu, here);      // (rows that a tile does not have take no time)
      float m_ref = -INFINITY, mb = 0.f, l = 0.f;
      bool counts = false;                                  // has a key counted?
      for (int j = x.j0; j < x.j1 && ok; ++j) {
        const bool full = !D.mask && (j + 1) * TILE <= x.keys;
        CxValid valid = {};
        if (!full) valid = cx_valid(D, x.b, x.keys, j, lane);
        ok = mbar_wait_warp(&sh.s_full[sx], cs & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        if (work) {
          uint32_t r[4][32];
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + c * 32, r[c]);
          tmem_wait_ld();
          if (!full) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!(valid.w[i & 3] >> (c * 8 + (i >> 2)) & 1)) r[c][i] = 0xff800000u;
          }
          counts |= full || (valid.w[0] | valid.w[1] | valid.w[2] | valid.w[3]);
          float t4[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) t4[c] = fmaxf(__uint_as_float(r[c][0]), __uint_as_float(r[c][1]));
#pragma unroll
          for (int i = 2; i < 32; i += 2)
#pragma unroll
            for (int c = 0; c < 4; ++c) t4[c] = max3f(t4[c], __uint_as_float(r[c][i]), __uint_as_float(r[c][i + 1]));
          const float m_new = fmaxf(m_ref, fmaxf(max3f(t4[0], t4[1], t4[2]), t4[3]));
          const bool need = (m_new - m_ref) * sl2 > LAZY_LOG2;          // (no: NaN, where no key has counted yet)
          // The previous PV of this stream has completed: the scores of this tile, which s_full announces, were issued
          // behind it by the same warp.  So O may be rescaled in place.
          if (j > x.j0 && __any_sync(0xffffffffu, need)) {
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
            tmem_wait_st();
            l *= alpha;
          }
          if (need) { m_ref = m_new; mb = m_new * sl2; }
          // P = 2^(s scale log2(e) - m) as bf16 over the scores; the row's sum is of the unrounded ones
          float2 sum2 = make_float2(0.f, 0.f);
          const float2 sl22 = make_float2(sl2, sl2), nmb2 = make_float2(-mb, -mb);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t pk[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 arg = __ffma2_rn(make_float2(__uint_as_float(r[c][2 * i]), __uint_as_float(r[c][2 * i + 1])), sl22, nmb2);
              const float2 pp = make_float2(ex2(arg.x), ex2(arg.y));
              sum2 = __fadd2_rn(sum2, pp);
              const __nv_bfloat162 v = __floats2bfloat162_rn(pp.x, pp.y);
              pk[i] = *(const uint32_t*)&v;
            }
            tmem_st16(s_addr + c * 16, pk);
            if (c & 1) {                                    // 64 keys are there
              tmem_wait_st();
              tc_fence_before();
              mbar_arrive(c == 1 ? &sh.p_half[sx] : &sh.p_full[sx]);
            }
          }
          l += sum2.x + sum2.y;
        } else {
          tc_fence_before();
          mbar_arrive(&sh.p_half[sx]);
          mbar_arrive(&sh.p_full[sx]);
        }
        ++cs;
      }
      if (!ok) break;
      if (x.j0 < x.j1) {
        ok = mbar_wait_warp(&sh.o_full[sx], co & 1, abort_flag);
        ++co;
        if (!ok) break;
        tc_fence_after();
      }
      const float inv = 1.f / l;
      const long long at = ((long long)x.b * D.H + h0 + row_h) * D.N + n0 + row_n;
      const float lse2 = counts ? mb + log2f(l) : -INFINITY;
      if (P.splits > 1) {
        const long long pat = (long long)x.part * D.B * D.H * D.N + at;
        if (here) P.part_lse[pat] = lse2;
        if (x.j0 < x.j1) {
          float* to = P.part + pat * D.d;
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
#pragma unroll 1
        for (int half = 0; half < HALVES; ++half) {
          if (staged) {                                     // the store before has read the stage
            if (row == 0) bulk_wait_read0();
            bar_sync(1 + sx, 128);
          }
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t r[32];
            if (x.j0 < x.j1) {
              tmem_ld32(o_addr + half * 64 + c * 32, r);
              tmem_wait_ld();
            }
            if (!counts) {
#pragma unroll
              for (int i = 0; i < 32; ++i) r[i] = 0;
            }
            cx_stage(stage, row, c, r, counts ? inv : 1.f);
          }
          fence_proxy_async();
          bar_sync(1 + sx, 128);
          if (row == 0) {
            tma_store_4d(stage, &map_o, half * 64, n0, h0, x.b);
            bulk_commit();
          }
          staged = true;
        }
      }
      if (x.j0 < x.j1) {
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
  D->scale = c.scale > 0.f ? c.scale : (float)(1.0 / sqrt((double)c.head_dim));
  D->sl2 = (float)(D->scale * 1.4426950408889634);
}
// Items of the forward launch: one or two tiles, all keys or parts of them, by the estimated time.  A tile of keys takes a pair of query
// tiles 1.6 us and a single one 1.0, an item 2 us more; joining the parts takes 3 us and what they write and read.
struct Forward { int pair, pairs, splits; };
Forward forward_of(const CrossDims& D) {
  Forward best = {1, D.tiles, 1};
  double least = 1e30;
  const long long nk = (D.K + TILE - 1) / TILE;
  for (int pair = 1; pair <= 2; ++pair) {
    const int pairs = (D.tiles + pair - 1) / pair;
    for (int splits = 1; splits <= 64 && splits <= (nk > 1 ? nk : 1); ++splits) {
      const double items = (double)D.B * D.G * pairs * splits;
      if (splits > 1 && items > 2 * FF_B200_SMS) break;
      const double waves = ceil(items / FF_B200_SMS);
      const double us = waves * ((double)((nk + splits - 1) / splits) * (pair == 2 ? 1.6 : 1.0) + 2) +
                        (splits > 1 ? 3 + (double)splits * D.B * D.H * D.N * D.d * 8 / 4e6 : 0);
      if (us < least) { least = us; best = {pair, pairs, splits}; }
    }
  }
  return best;
}
size_t part_bytes(const CrossDims& D, int splits) { return (size_t)splits * D.B * D.H * D.N * D.d * sizeof(float); }
size_t part_lse_bytes(const CrossDims& D, int splits) { return (size_t)splits * D.B * D.H * D.N * sizeof(float); }

// Sizes that the kernels' indexes and tensor maps take
constexpr char MOST[] = "queries and keys must be at most 2^31 - 256, batch * heads and their tiles of queries (and of keys) below 2^31, all values below 2^42";
bool too_large(const ff_cross_attention_config_t& c, int64_t batch, int64_t queries, int64_t keys) {
  if (batch > 0x7fffffff || queries > 0x7fffff00 || keys > 0x7fffff00) return true;
  const double bh = (double)batch * c.heads;
  return bh >= 2147483648.0 || bh * (double)((queries + TILE - 1) / TILE) >= 2147483648.0 || bh * (double)((keys + TILE - 1) / TILE) >= 2147483648.0 ||
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
  size_t need = 0;
  ff_cross_attention_workspace_bytes(&h->cfg, batch, queries, keys, training, &need);
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
  if (!(c->scale >= 0.f && c->scale < 3.0e38f)) return fail(nullptr, FF_ERR_INVALID_ARG, "scale must be positive and finite, or 0 for 1 / sqrt(head_dim)");
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
  } else {
    const Forward f = forward_of(D);
    if (f.splits > 1) *bytes = part_bytes(D, f.splits) + part_lse_bytes(D, f.splits);
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
  cudaError_t e = cudaGetDevice(&h->device);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(cross_forward_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(cross_forward_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM);
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
  cudaStream_t st = (cudaStream_t)stream;
  CrossParams P{};
  shape_of(c, batch, queries, keys, &P.dm);
  keys_of(&P.dm, h, q, k, v, lengths, mask);
  const Forward f = forward_of(P.dm);
  P.pair = f.pair; P.pairs = f.pairs; P.splits = f.splits;
  const long long items = (long long)P.dm.B * P.dm.G * f.pairs * f.splits;
  if (items >= 0x7fffffff - FF_B200_SMS) return fail(h, FF_ERR_UNSUPPORTED, MOST);
  P.items = (int)items;
  P.lse = lse;
  P.part = (float*)ws;
  P.part_lse = (float*)((char*)ws + part_bytes(P.dm, f.splits));
  CUtensorMap mq, mk, mv, mo;
  const int64_t kn = keys > 0 ? keys : 1;
  if (!cx_map(&mq, q, batch, queries, c.head_dim, P.dm.bn, P.dm.bh) || !cx_map(&mk, k, keys > 0 ? batch : 1, kn, c.head_dim, TILE, 1) ||
      !cx_map(&mv, v, keys > 0 ? batch : 1, kn, c.head_dim, TILE, 1) || !cx_map(&mo, out, batch, queries, c.head_dim, P.dm.bn, P.dm.bh))
    return fail(h, FF_ERR_CUDA, "could not encode the tensor maps");
  const dim3 grid((unsigned)(P.items < FF_B200_SMS ? P.items : FF_B200_SMS));
  CX_CUDA(h, c.head_dim > 64 ? ff_launch(cross_forward_kernel<128>, grid, dim3(THREADS), SMEM, st, mq, mk, mv, mo, P)
                             : ff_launch(cross_forward_kernel<64>, grid, dim3(THREADS), SMEM, st, mq, mk, mv, mo, P));
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
