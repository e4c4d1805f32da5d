// The gated feed-forward block, forward and backward, bf16 with fp32 accumulation:
//   G = X Wg, U = X Wu, H = act(G) * U, out = H Wd                                      X [M][D], Wg, Wu [D][F], Wd [F][D]
//   dH = dout Wd^T, dG = dH U act'(G), dU = dH act(G), dX = dG Wg^T + dU Wu^T,
//   dWg = X^T dG, dWu = X^T dU, dWd = H^T dout
//
// Every product is one launch of one kernel: a persistent GEMM on CTA pairs (tcgen05, cta_group::2) with tiles of 256 x 256
// (128 rows of A and 128 columns of B in either CTA's shared memory), K in chunks of 64, a ring of six stages filled by TMA, and
// two accumulators of 256 tensor-memory columns, so that the epilogue of a tile overlaps the main loop of the next.  Operands
// are read as they lie in memory, K-major or MN-major, so nothing is transposed: the products differ in majorness and epilogue.
//   gate and up   one tile is 128 columns of G (the even CTA's half of B) beside the same 128 columns of U (the odd CTA's), so
//                 that both values of an element lie in one lane of tensor memory and H leaves without G and U reaching memory
//   dH            its epilogue reads G and U and writes dG, dU and H (needed for dWd; made again rather than kept)
//   dX            K runs over the columns of dG, then those of dU
//   dWg, dWu      one launch, the matrices side by side along N; K runs over the tokens
// H, dG and dU are rounded to bf16 between the products: they are operands of the next one.
//
//   warp 0      TMA producer          warp 1      tcgen05.mma issuer of the pair (even CTA), owns the tensor memory
//   warps 2..9  epilogue: a thread owns one row of the tile and half its columns
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
  int* status;             // device status word (plan-like: raised by an expired wait)
  char err[512];
};

namespace {

constexpr int TM = 256, TN = 256, TK = 64;
constexpr int PIECE = 64 * 128;                  // 64 rows of 128 bytes
constexpr int OPERAND = 2 * PIECE;               // one CTA's 128 rows (or columns) of a K chunk
constexpr int STAGE = 2 * OPERAND;
constexpr int NSTAGE = 6;
constexpr int EPI_WARPS = 8;
constexpr int THREADS = 64 + 32 * EPI_WARPS;

enum { STORE = 0, GATE = 1, DGATE = 2 };         // epilogues

struct GemmParams {
  long long rows;                  // output rows
  int cols;                        // output columns of one matrix
  int m_tiles, n_tiles, mats;      // tiles; matrices side by side
  int kchunks, sources;            // K chunks of one source, sources one after the other
  int act;
  __nv_bfloat16* out[3];           // STORE: one per matrix;  GATE: H, G or NULL, U;  DGATE: dG, dU, H
  const __nv_bfloat16* gate;       // DGATE
  const __nv_bfloat16* up;
  int* status;
};

struct Shared {
  uint64_t full[NSTAGE], empty[NSTAGE], acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int abort_flag;
};
constexpr size_t SMEM = (size_t)NSTAGE * STAGE + sizeof(Shared) + 1024;

// act(g) and, with SLOPE, its derivative.  The cubic inside gelu_tanh saturates long before |g| = 16.
__device__ __forceinline__ float sigmoid(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }
template <bool SLOPE>
__device__ __forceinline__ float activation(int act, float g, float* slope) {
  if (act == FF_ACT_SILU) {
    const float s = sigmoid(g);
    if (SLOPE) *slope = s * (1.f + g * (1.f - s));
    return g * s;
  }
  if (act == FF_ACT_GELU_TANH) {
    const float c = 1.5957691216057308f;         // 2 sqrt(2 / pi)
    const float t = fminf(fmaxf(g, -16.f), 16.f), t2 = t * t;
    const float s = sigmoid(c * t * (1.f + 0.044715f * t2));
    if (SLOPE) *slope = s + t * s * (1.f - s) * c * (1.f + 0.134145f * t2);
    return g * s;
  }
  const float p = 0.5f * erfcf(-0.70710678118654752f * g);
  if (SLOPE) {
    const float t = fminf(fmaxf(g, -32.f), 32.f);
    *slope = p + t * 0.3989422804014327f * __expf(-0.5f * t * t);
  }
  return g * p;
}

__device__ __forceinline__ void store32(__nv_bfloat16* dst, const float (&v)[32], int left) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j * 8 < left) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = bf16_pair(__float_as_uint(v[j * 8 + 2 * i]), __float_as_uint(v[j * 8 + 2 * i + 1]));
      *(uint4*)(dst + j * 8) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
__device__ __forceinline__ void load32(const __nv_bfloat16* src, uint4 (&v)[4], int left) {
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = j * 8 < left ? __ldcs((const uint4*)(src + j * 8)) : make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ float element(const uint4 (&v)[4], int i) {
  const uint32_t w = ((const uint32_t*)v)[i >> 1];
  return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
}

template <bool A_MN, bool B_MN, int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
ffn_gemm_kernel(const __grid_constant__ CUtensorMap map_a0, const __grid_constant__ CUtensorMap map_a1,
                const __grid_constant__ CUtensorMap map_b0, const __grid_constant__ CUtensorMap map_b1, const GemmParams P) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  Shared& sh = *(Shared*)(smem + NSTAGE * STAGE);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int per_row = P.n_tiles * P.mats;                       // tiles of a row of tiles
  const long long tiles = (long long)P.m_tiles * per_row;
  const int kchunks = P.kchunks * P.sources;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NSTAGE; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.acc_full[i], 1); mbar_init(&sh.acc_empty[i], 2 * EPI_WARPS); }
    sh.abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) { tmem_alloc_pair(&sh.tmem_base, 512); tmem_relinquish_pair(); }
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
      for (long long t = pair; t < tiles && ok; t += pairs) {
        const int mt = (int)(t / per_row), j = (int)(t % per_row), mat = j / P.n_tiles, nt = j % P.n_tiles;
        const int m0 = mt * TM + (int)rank * 128;
        const int n0 = EPI == GATE ? nt * 128 : nt * TN + (int)rank * 128;
        for (int kc = 0; kc < kchunks && ok; ++kc, ++n) {
          const int slot = n % NSTAGE;
          if (n >= (unsigned)NSTAGE) ok = mbar_wait(&sh.empty[slot], ((n / NSTAGE) - 1) & 1, abort_flag);
          if (!ok) break;
          const int second = kc >= P.kchunks, k0 = (kc - (second ? P.kchunks : 0)) * TK;
          const CUtensorMap* ma = second ? &map_a1 : &map_a0;
          const CUtensorMap* mb = (EPI == GATE ? (int)rank : second | mat) ? &map_b1 : &map_b0;
          uint8_t* dst = smem + slot * STAGE;
          const uint32_t bar = map_shared(&sh.full[slot], 0);
          if (rank == 0) mbar_arrive_expect_tx(&sh.full[slot], 2 * STAGE);
          if (A_MN) {
            tma_load_3d_pair(dst, ma, bar, m0, k0, 0);
            tma_load_3d_pair(dst + PIECE, ma, bar, m0 + 64, k0, 0);
          } else {
            tma_load_3d_pair(dst, ma, bar, k0, m0, 0);
          }
          if (B_MN) {
            tma_load_3d_pair(dst + OPERAND, mb, bar, n0, k0, 0);
            tma_load_3d_pair(dst + OPERAND + PIECE, mb, bar, n0 + 64, k0, 0);
          } else {
            tma_load_3d_pair(dst + OPERAND, mb, bar, k0, n0, 0);
          }
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t idesc = idesc_bf16_f32(TM, TN, A_MN, B_MN);
      const uint64_t a0 = smem_desc_sw128(smem_u32(smem), A_MN ? PIECE : 16, 1024);
      const uint64_t b0 = smem_desc_sw128(smem_u32(smem) + OPERAND, B_MN ? PIECE : 16, 1024);
      constexpr uint64_t A_STEP = A_MN ? 128 : 2, B_STEP = B_MN ? 128 : 2;      // 16 K elements on, in units of 16 bytes
      unsigned n = 0, nt = 0;
      bool ok = true;
      for (long long t = pair; t < tiles && ok; t += pairs, ++nt) {
        const int ab = nt & 1;
        if (nt >= 2) ok = mbar_wait_warp(&sh.acc_empty[ab], ((nt >> 1) - 1) & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        for (int kc = 0; kc < kchunks && ok; ++kc, ++n) {
          const int slot = n % NSTAGE;
          ok = mbar_wait_warp(&sh.full[slot], (n / NSTAGE) & 1, abort_flag);
          if (!ok) break;
          tc_fence_after();
          const uint64_t at = (uint64_t)(slot * (STAGE >> 4));
#pragma unroll
          for (int ks = 0; ks < TK / 16; ++ks)
            umma_ss_pair(tm + ab * TN, a0 + at + ks * A_STEP, b0 + at + ks * B_STEP, idesc, ks > 0 ? 1u : (kc > 0 ? 1u : 0u));
          umma_commit_pair(&sh.empty[slot]);
        }
        umma_commit_pair(&sh.acc_full[ab]);
      }
    }
  } else {
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
    unsigned nt = 0;
    bool ok = true;
    for (long long t = pair; t < tiles && ok; t += pairs, ++nt) {
      const int ab = nt & 1;
      const int j = (int)(t % per_row), mat = j / P.n_tiles;
      const long long row = (t / per_row) * TM + rank * 128 + quarter * 32 + lane;
      const bool live = row < P.rows;
      const size_t line = (size_t)row * P.cols;
      const uint32_t acc = tm + lane_addr + ab * TN;
      constexpr int WIDTH = EPI == GATE ? 64 : 128;             // columns of the warp
      const int c0 = (j % P.n_tiles) * (2 * WIDTH) + half * WIDTH;
      uint4 g[4], u[4];
      if (EPI == DGATE) {                                       // (on their way before the accumulator is complete)
        load32(P.gate + line + c0, g, live ? P.cols - c0 : 0);
        load32(P.up + line + c0, u, live ? P.cols - c0 : 0);
      }
      ok = __all_sync(0xffffffffu, mbar_wait(&sh.acc_full[ab], (nt >> 1) & 1, abort_flag));
      if (!ok) break;
      tc_fence_after();
#pragma unroll 1
      for (int q = 0; q < WIDTH / 32; ++q) {
        const int col = c0 + q * 32, left = live ? P.cols - col : 0;
        uint32_t r[32];
        tmem_ld32(acc + half * WIDTH + q * 32, r);
        float v[32];
        if (EPI == STORE) {
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
          store32((mat ? P.out[1] : P.out[0]) + line + col, v, left);
        } else if (EPI == GATE) {
          uint32_t s[32];
          tmem_ld32(acc + 128 + half * WIDTH + q * 32, s);
          tmem_wait_ld();
          if (P.out[1]) {                                       // kept for the backward pass
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
            store32(P.out[1] + line + col, v, left);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(s[i]);
            store32(P.out[2] + line + col, v, left);
          }
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = activation<false>(P.act, __uint_as_float(r[i]), nullptr) * __uint_as_float(s[i]);
          store32(P.out[0] + line + col, v, left);
        } else {
          uint4 g2[4], u2[4];
          const bool more = q + 1 < WIDTH / 32;
          load32(P.gate + line + col + 32, g2, more ? left - 32 : 0);
          load32(P.up + line + col + 32, u2, more ? left - 32 : 0);
          tmem_wait_ld();
          float dg[32], h[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float d = __uint_as_float(r[i]), up = element(u, i);
            float slope;
            const float a = activation<true>(P.act, element(g, i), &slope);
            dg[i] = d * up * slope; v[i] = d * a; h[i] = a * up;
          }
          store32(P.out[0] + line + col, dg, left);
          store32(P.out[1] + line + col, v, left);
          store32(P.out[2] + line + col, h, left);
#pragma unroll
          for (int i = 0; i < 4; ++i) { g[i] = g2[i]; u[i] = u2[i]; }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_shared(&sh.acc_empty[ab], 0));
    }
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
    tmem_dealloc_pair(tm, 512);
  }
}

// [rows][cols] bf16 with a box of box_rows rows x 64 columns, 128-byte swizzle.
bool matrix_map(CUtensorMap* map, const void* base, long long rows, long long cols, int box_rows) {
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, 1};
  cuuint64_t strides[2] = {(cuuint64_t)cols * 2, (cuuint64_t)rows * cols * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
  return ff_encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B,
                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

// The matrix of an operand: [rows][cols] as it lies in memory.  K-major: a row is one M or N index; MN-major: one K index.
struct Operand { const void* p; long long rows, cols; };

template <bool A_MN, bool B_MN, int EPI>
cudaError_t gemm(const ff_ffn* h, const Operand (&a)[2], const Operand (&b)[2], GemmParams P, cudaStream_t st) {
  CUtensorMap m[4];
  for (int i = 0; i < 2; ++i)
    if (!matrix_map(&m[i], a[i].p, a[i].rows, a[i].cols, A_MN ? 64 : 128) || !matrix_map(&m[2 + i], b[i].p, b[i].rows, b[i].cols, B_MN ? 64 : 128))
      return cudaErrorInvalidValue;
  const int width = EPI == GATE ? 128 : TN;
  P.m_tiles = (int)((P.rows + TM - 1) / TM);
  P.n_tiles = (P.cols + width - 1) / width;
  P.act = h->cfg.activation;
  P.status = h->status;
  const long long tiles = (long long)P.m_tiles * P.n_tiles * P.mats;
  const int pairs = h->sm_count / 2;
  return ff_launch(ffn_gemm_kernel<A_MN, B_MN, EPI>, dim3(2 * (unsigned)(tiles < pairs ? tiles : pairs)), dim3(THREADS), SMEM, st, m[0], m[1], m[2], m[3], P);
}
inline int chunks(long long k) { return (int)((k + TK - 1) / TK); }

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
ff_status_t check_call(ff_ffn* h, int64_t tokens, void* ws, size_t ws_bytes, int training) {
  if (tokens < 0) return fail(h, FF_ERR_INVALID_ARG, "tokens must not be negative");
  if (tokens > 0x7fffff00) return fail(h, FF_ERR_UNSUPPORTED, "tokens must be below 2^31 - 256");
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess || device != h->device) return fail(h, FF_ERR_INVALID_ARG, "the handle belongs to another device than the current one");
  size_t need = 0;
  ff_ffn_workspace_bytes(&h->cfg, tokens, training, &need);
  if (need && (!ws || ws_bytes < need)) return fail(h, FF_ERR_WORKSPACE, "the workspace is missing or smaller than ff_ffn_workspace_bytes");
  if (need && (((uintptr_t)ws) & 255)) return fail(h, FF_ERR_WORKSPACE, "the workspace must be 256-byte aligned");
  return FF_OK;
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
  *bytes = (training ? 3 : 1) * hidden_bytes(*c, tokens);      // H;  backward: dG, dU, H
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
  const void* kernels[] = {(const void*)ffn_gemm_kernel<false, true, GATE>, (const void*)ffn_gemm_kernel<false, true, STORE>,
                           (const void*)ffn_gemm_kernel<false, false, DGATE>, (const void*)ffn_gemm_kernel<false, false, STORE>,
                           (const void*)ffn_gemm_kernel<true, true, STORE>};
  for (const void* k : kernels)
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM);
  if (e == cudaSuccess) e = cudaMalloc((void**)&h->status, 256);
  if (e == cudaSuccess) e = cudaMemset(h->status, 0, 256);
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
  ff_status_t s = check_call(h, tokens, ws, ws_bytes, 0);
  if (s != FF_OK) return s;
  if (!gate != !up) return fail(h, FF_ERR_INVALID_ARG, "gate and up are kept together, or neither is");
  if (tokens == 0) return FF_OK;
  if (!X || !Wg || !Wu || !Wd || !out) return fail(h, FF_ERR_INVALID_ARG, "X, Wg, Wu, Wd or out is NULL");
  if (misaligned({X, Wg, Wu, Wd, gate, up, out})) return fail(h, FF_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  const int D = h->cfg.dim, F = h->cfg.hidden;
  cudaStream_t st = (cudaStream_t)stream;
  GemmParams P{};
  P.rows = tokens; P.mats = 1; P.sources = 1;
  P.cols = F; P.kchunks = chunks(D);
  P.out[0] = (__nv_bfloat16*)ws; P.out[1] = (__nv_bfloat16*)gate; P.out[2] = (__nv_bfloat16*)up;
  const Operand x{X, tokens, D}, hid{ws, tokens, F}, wd{Wd, F, D};
  FFN_CUDA(h, (gemm<false, true, GATE>(h, {x, x}, {Operand{Wg, D, F}, Operand{Wu, D, F}}, P, st)));
  P.cols = D; P.kchunks = chunks(F);
  P.out[0] = (__nv_bfloat16*)out;
  FFN_CUDA(h, (gemm<false, true, STORE>(h, {hid, hid}, {wd, wd}, P, st)));
  return FF_OK;
}

extern "C" ff_status_t ff_ffn_backward(ff_ffn_t* h, int64_t tokens, const void* X, const void* Wg, const void* Wu, const void* Wd, const void* gate,
                                       const void* up, const void* dout, void* dX, void* dWg, void* dWu, void* dWd, void* ws, size_t ws_bytes,
                                       void* stream) {
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "the handle is NULL");
  ff_status_t s = check_call(h, tokens, ws, ws_bytes, 1);
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
  char* base = (char*)ws;
  void *dG = base, *dU = base + hidden_bytes(h->cfg, tokens), *H = base + 2 * hidden_bytes(h->cfg, tokens);
  const Operand x{X, tokens, D}, g{dout, tokens, D}, wd{Wd, F, D}, dg{dG, tokens, F}, du{dU, tokens, F}, hid{H, tokens, F};
  GemmParams P{};
  P.mats = 1; P.sources = 1;
  P.rows = tokens; P.cols = F; P.kchunks = chunks(D);
  P.gate = (const __nv_bfloat16*)gate; P.up = (const __nv_bfloat16*)up;
  P.out[0] = (__nv_bfloat16*)dG; P.out[1] = (__nv_bfloat16*)dU; P.out[2] = (__nv_bfloat16*)H;
  FFN_CUDA(h, (gemm<false, false, DGATE>(h, {g, g}, {wd, wd}, P, st)));
  if (dX) {
    P.cols = D; P.kchunks = chunks(F); P.sources = 2;
    P.out[0] = (__nv_bfloat16*)dX;
    FFN_CUDA(h, (gemm<false, false, STORE>(h, {dg, du}, {Operand{Wg, D, F}, Operand{Wu, D, F}}, P, st)));
  }
  P.sources = 1; P.kchunks = chunks(tokens);
  if (dWg) {
    P.rows = D; P.cols = F; P.mats = 2;
    P.out[0] = (__nv_bfloat16*)dWg; P.out[1] = (__nv_bfloat16*)dWu;
    FFN_CUDA(h, (gemm<true, true, STORE>(h, {x, x}, {dg, du}, P, st)));
  }
  if (dWd) {
    P.rows = F; P.cols = D; P.mats = 1;
    P.out[0] = (__nv_bfloat16*)dWd;
    FFN_CUDA(h, (gemm<true, true, STORE>(h, {hid, hid}, {g, g}, P, st)));
  }
  return FF_OK;
}
