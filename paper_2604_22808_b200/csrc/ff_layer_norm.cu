// Layer norm of rows of dim values, forward and backward, with weights and bias of the model or of each sample.
//
//   forward    c = x - mean,  r = 1 / sqrt(mean(c^2) + eps),  n = c r,  y = n w + b      (w = 1 + weight with unit_offset)
//   backward   g = dy w;  dx = r (g - mean(g) - n mean(g n));  dweight = sum over rows of dy n;  dbias = sum over rows of dy
//
// One pass over the rows: a row is read once, stays in registers, and is written once, so memory bounds it: 2 (backward 3) tensors.
// The mean is subtracted before the squares are summed (the values are in registers, a second sum costs no memory traffic), so
// rows whose mean is far from zero lose nothing.
//
// Forward, up to 2048 bf16 or 1024 fp32 values: a warp has a row (at most 64 values a thread) and the sums are shuffles alone.
// Longer rows, and all rows of the backward pass, where a thread also keeps the weights and both gradients' sums of its channels,
// go to a block with 16 values a thread.
#include <stdio.h>

#include <new>

#include "ff_chunks.cuh"
#include "ff_internal.h"

struct ff_layer_norm {
  ff_layer_norm_config_t cfg;
  char err[512];
};

namespace {

constexpr int VALUES = 16;                        // values of a row that a thread of a block has
constexpr int MAX_DIM = 8192, MAX_THREADS = MAX_DIM / VALUES;
constexpr int ROW_WARPS = 4;                      // rows at a time in a block whose warps have a row each

struct RowsView { char* p; long long sb, st; };   // strides in bytes
struct NormParams {
  RowsView x, y, g;                 // input, output (backward: dx, or p NULL), gradient of the forward pass's output
  const float *w, *bias;            // or NULL
  long long w_stride;               // dim: weights of each sample; 0: of the model
  float plus;                       // added to the weight
  float *dw, *db;                   // backward: where a block's sums go (or NULL) ...
  long long part_stride;            // ... and how far those of the blocks are apart
  unsigned tokens, segment, parts;  // tokens of a sample; rows whose gradients are summed together, blocks that do it
  FFFastDiv by_tokens;
  int rows, d, pieces;
  float inv_d, eps;
};

__device__ __forceinline__ unsigned divide(unsigned n, const FFFastDiv& f) { return (unsigned)(((unsigned long long)__umulhi(n, f.m) + n) >> f.s); }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int m = 16; m; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}
// Sum over the threads that have a row: the warp, or the block, whose warps' sums meet in one of several places in turns.
template <bool WARP>
__device__ __forceinline__ float row_sum(float v, float* place) {
  v = warp_sum(v);
  if constexpr (WARP) return v;
  const int warps = blockDim.x >> 5;
  if ((threadIdx.x & 31) == 0) place[threadIdx.x >> 5] = v;
  __syncthreads();
  const int lane = threadIdx.x & 31;
  return warp_sum(lane < warps ? place[lane] : 0.f);
}

// A thread's pieces of a row: piece `first + i * step`.
template <class T, int CH, int PER>
struct Row {
  static constexpr int N = pairs_of(CH);
  using C = Chunk<T, CH>;
  static __device__ __forceinline__ void load(C (&raw)[PER], const char* row, int first, int step, int pieces) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const C none{};
      raw[i] = first + i * step < pieces ? *(const C*)(row + (long long)(first + i * step) * sizeof(C)) : none;
    }
  }
  static __device__ __forceinline__ void store(char* row, const F2 (&v)[PER][N], int first, int step, int pieces) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (first + i * step < pieces) *(C*)(row + (long long)(first + i * step) * sizeof(C)) = pack<T, CH>(v[i]);
  }
  static __device__ __forceinline__ float sum(const F2 (&v)[PER][N]) {
    F2 s = two(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int c = 0; c < N; ++c) s = __fadd2_rn(s, v[i][c]);
    return low(s) + high(s);
  }
  static __device__ __forceinline__ float dot(const F2 (&u)[PER][N], const F2 (&v)[PER][N]) {
    F2 s = two(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int c = 0; c < N; ++c) s = fma(u[i][c], v[i][c], s);
    return low(s) + high(s);
  }
  // Values minus `m`, and zeros where the row has none.
  static __device__ __forceinline__ void centre(F2 (&v)[PER][N], float m, int first, int step, int pieces) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool have = first + i * step < pieces;
#pragma unroll
      for (int c = 0; c < N; ++c) v[i][c] = have ? two(low(v[i][c]) - m, CH > 1 ? high(v[i][c]) - m : 0.f) : two(0.f, 0.f);
    }
  }
  // raw -> n = (x - mean) r; the result is r.  Rows whose squares (or sum) leave fp32 are taken again, scaled by 2^-80, and eps by its
  // square (which is far below their variance).  The sums meet in places 0 and 1, 2 and 3.
  template <bool WARP>
  static __device__ __forceinline__ float normalise(const C (&raw)[PER], F2 (&n)[PER][N], const NormParams& P, int first, int step, float (*place)[32]) {
#pragma unroll
    for (int i = 0; i < PER; ++i) unpack<T, CH>(raw[i], n[i]);
    centre(n, row_sum<WARP>(sum(n), place[0]) * P.inv_d, first, step, P.pieces);
    const float var = row_sum<WARP>(dot(n, n), place[1]) * P.inv_d;
    float r = rsqrtf(var + P.eps), scale = r;
    if (!(var < 3.0e38f)) {
      const float down = 8.2718061255302767e-25f;              // 2^-80
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        unpack<T, CH>(raw[i], n[i]);
#pragma unroll
        for (int c = 0; c < N; ++c) n[i][c] = mul(n[i][c], two(down, down));
      }
      centre(n, row_sum<WARP>(sum(n), place[2]) * P.inv_d, first, step, P.pieces);
      scale = rsqrtf(row_sum<WARP>(dot(n, n), place[3]) * P.inv_d + P.eps * down * down);
      r = scale * down;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int c = 0; c < N; ++c) n[i][c] = mul(n[i][c], two(scale, scale));
    return r;
  }
  // Neighbouring weights of a piece as they multiply, or ones.
  static __device__ __forceinline__ F2 weight(const NormParams& P, const float* w, int piece, int c) {
    if (!w || piece >= P.pieces) return two(1.f, 1.f);
    return two(w[piece * CH + 2 * c] + P.plus, CH > 1 ? w[piece * CH + 2 * c + 1] + P.plus : 0.f);
  }
};

__device__ __forceinline__ const char* row_at(const RowsView& v, unsigned b, unsigned n) { return v.p + (long long)b * v.sb + (long long)n * v.st; }

// Forward.  The next row is on its way while this one is summed.
template <class T, int CH, int PER, bool WARP>
__global__ void __launch_bounds__(WARP ? ROW_WARPS * 32 : MAX_THREADS) norm_forward_kernel(const __grid_constant__ NormParams P) {
  using R = Row<T, CH, PER>;
  constexpr int N = R::N;
  __shared__ float place[WARP ? 1 : 4][32];
  const int first = WARP ? threadIdx.x & 31 : threadIdx.x, step = WARP ? 32 : blockDim.x;
  const int teams = WARP ? gridDim.x * ROW_WARPS : gridDim.x;
  int row = WARP ? blockIdx.x * ROW_WARPS + (threadIdx.x >> 5) : blockIdx.x;
  ff_pdl_wait();
  if (row >= P.rows) return;
  typename R::C raw[PER];
  unsigned b = divide(row, P.by_tokens), n = row - b * P.tokens;
  R::load(raw, row_at(P.x, b, n), first, step, P.pieces);
#pragma unroll 1
  while (true) {
    F2 v[PER][N];
    R::template normalise<WARP>(raw, v, P, first, step, place);
    char* to = (char*)row_at(P.y, b, n);
    const float *w = P.w ? P.w + b * P.w_stride : nullptr, *bias = P.bias ? P.bias + b * P.w_stride : nullptr;
    row += teams;
    const bool more = row < P.rows;
    if (more) {
      b = divide(row, P.by_tokens), n = row - b * P.tokens;
      R::load(raw, row_at(P.x, b, n), first, step, P.pieces);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int piece = first + i * step;
      if (piece >= P.pieces) break;
#pragma unroll
      for (int c = 0; c < N; ++c) {
        const F2 add = bias ? two(bias[piece * CH + 2 * c], CH > 1 ? bias[piece * CH + 2 * c + 1] : 0.f) : two(0.f, 0.f);
        v[i][c] = fma(v[i][c], R::weight(P, w, piece, c), add);
      }
    }
    R::store(to, v, first, step, P.pieces);
    if (!more) break;
  }
}

// Backward: a block has a row at a time; block s * parts + i takes every parts-th row of segment s.
template <class T, int CH, int PER>
__global__ void __launch_bounds__(MAX_THREADS) norm_backward_kernel(const __grid_constant__ NormParams P) {
  using R = Row<T, CH, PER>;
  constexpr int N = R::N;
  __shared__ float place[6][32];
  const int first = threadIdx.x, step = blockDim.x;
  const unsigned segment = blockIdx.x / P.parts, part = blockIdx.x - segment * P.parts;
  ff_pdl_wait();
  F2 w[PER][N], dw[PER][N], db[PER][N];
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int c = 0; c < N; ++c) {
      w[i][c] = R::weight(P, P.w ? P.w + segment * P.w_stride : nullptr, first + i * step, c);
      dw[i][c] = db[i][c] = two(0.f, 0.f);
    }
  typename R::C x[PER], g[PER];
  unsigned at = part, b, n;
  auto ask = [&] {
    const unsigned row = segment * P.segment + at;
    b = divide(row, P.by_tokens), n = row - b * P.tokens;
    R::load(x, row_at(P.x, b, n), first, step, P.pieces);
    R::load(g, row_at(P.g, b, n), first, step, P.pieces);
  };
  if (at < P.segment) ask();
#pragma unroll 1
  while (at < P.segment) {
    F2 v[PER][N], dy[PER][N];
    const float r = R::template normalise<false>(x, v, P, first, step, place);
    char* to = P.y.p ? (char*)row_at(P.y, b, n) : nullptr;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      unpack<T, CH>(g[i], dy[i]);
#pragma unroll
      for (int c = 0; c < N; ++c) {
        dw[i][c] = fma(dy[i][c], v[i][c], dw[i][c]);
        db[i][c] = __fadd2_rn(db[i][c], dy[i][c]);
        dy[i][c] = mul(dy[i][c], w[i][c]);                     // g
      }
    }
    at += P.parts;
    if (at < P.segment) ask();
    const float m = row_sum<false>(R::sum(dy), place[4]) * P.inv_d, k = row_sum<false>(R::dot(dy, v), place[5]) * P.inv_d;
    if (to) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int c = 0; c < N; ++c)
          dy[i][c] = mul(fma(v[i][c], two(-k, -k), two(low(dy[i][c]) - m, high(dy[i][c]) - m)), two(r, r));
      R::store(to, dy, first, step, P.pieces);
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int piece = first + i * step;
    if (piece >= P.pieces) break;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const long long to = blockIdx.x * P.part_stride + piece * CH + c;
      if (P.dw) P.dw[to] = c & 1 ? high(dw[i][c / 2]) : low(dw[i][c / 2]);
      if (P.db) P.db[to] = c & 1 ? high(db[i][c / 2]) : low(db[i][c / 2]);
    }
  }
}

// The blocks' sums of a segment, joined in a fixed order: block (32 columns, weight or bias, segment).
__global__ void __launch_bounds__(1024) norm_join_kernel(const float* partial, int parts, int d, int columns, float* dw, float* db) {
  __shared__ float sum[32][33];
  ff_pdl_wait();
  const unsigned segment = blockIdx.x / columns;
  const int c = (blockIdx.x - segment * columns) * 32 + (threadIdx.x & 31), ty = threadIdx.x >> 5;
  float* out = blockIdx.y ? db : dw;
  if (!out) return;
  const float* p = partial + ((long long)segment * parts * 2 + blockIdx.y) * d + c;
  float s = 0.f;
  if (c < d)
#pragma unroll 4
    for (int i = ty; i < parts; i += 32) s += p[(long long)i * 2 * d];
  sum[ty][threadIdx.x & 31] = s;
  __syncthreads();
  if (ty == 0 && c < d) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sum[i][threadIdx.x];
    out[(long long)segment * d + c] = s;
  }
}

ff_status_t fail(ff_layer_norm* h, ff_status_t code, const char* msg) {
  if (h) snprintf(h->err, sizeof h->err, "%s", msg);
  else ff_set_thread_error(msg);
  return code;
}
ff_status_t cuda_fail(ff_layer_norm* h, cudaError_t e) {
  char msg[256];
  snprintf(msg, sizeof msg, "CUDA error: %s", cudaGetErrorString(e));
  return fail(h, FF_ERR_CUDA, msg);
}

// What a call's tensors have to fulfil; the bits of their addresses and strides decide the piece.
ff_status_t check_rows(ff_layer_norm* h, const ff_rows_t* v, int64_t batch, int64_t tokens, bool written, int e, uint64_t* bits) {
  if (!v || !v->data) return fail(h, FF_ERR_INVALID_ARG, "a tensor is NULL");
  if (v->stride_batch < 0 || v->stride_token < 0) return fail(h, FF_ERR_INVALID_ARG, "strides must not be negative");
  if (written && ((batch > 1 && v->stride_batch == 0) || (tokens > 1 && v->stride_token == 0)))
    return fail(h, FF_ERR_INVALID_ARG, "an output's stride is 0: rows would be written over one another");
  if ((uintptr_t)v->data % e) return fail(h, FF_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  *bits |= (uint64_t)(uintptr_t)v->data;
  if (batch > 1) *bits |= (uint64_t)v->stride_batch * e;
  if (tokens > 1) *bits |= (uint64_t)v->stride_token * e;
  return FF_OK;
}
RowsView view(const ff_rows_t* v, int e) { return RowsView{(char*)v->data, (long long)v->stride_batch * e, (long long)v->stride_token * e}; }

// Values of a piece that dim and the tensors' alignment allow.
int piece_of(int d, int e, uint64_t bits) {
  for (int ch = 16 / e; ch > 1; ch = ch == 8 ? 2 : ch >> 1)
    if (d % ch == 0 && bits % ((uint64_t)ch * e) == 0 && (ch == 16 / e || e == 2)) return ch;
  return 1;
}
int block_threads(int pieces, int per) { return ((pieces + per - 1) / per + 31) / 32 * 32; }

// Blocks whose sums are joined: enough for every SM, and no more than rows.
constexpr int PART_BLOCKS = 4 * FF_B200_SMS;
struct Parts { unsigned segments, rows, parts; };
Parts parts_of(int64_t batch, int64_t tokens, int per_sample) {
  Parts p;
  p.segments = per_sample ? (unsigned)batch : 1;
  p.rows = (unsigned)(per_sample ? tokens : batch * tokens);
  p.parts = PART_BLOCKS / (p.segments ? p.segments : 1);
  if (p.parts > p.rows) p.parts = p.rows;
  if (p.parts < 1) p.parts = 1;
  return p;
}

template <class T, int CH, int PER, bool WARP>
cudaError_t forward(NormParams& P, cudaStream_t st) {
  // Blocks of one wave take the rows in turns.
  const int threads = WARP ? ROW_WARPS * 32 : block_threads(P.pieces, PER);
  const long long blocks = WARP ? (P.rows + ROW_WARPS - 1) / ROW_WARPS : P.rows, wave = (long long)FF_B200_SMS * (2048 / threads);
  return ff_launch(norm_forward_kernel<T, CH, PER, WARP>, dim3((unsigned)(blocks < 4 * wave ? blocks : 4 * wave)), dim3(threads), 0, st, P);
}
template <class T, int CH, int PER>
cudaError_t backward(NormParams& P, unsigned blocks, cudaStream_t st) {
  return ff_launch(norm_backward_kernel<T, CH, PER>, dim3(blocks), dim3(block_threads(P.pieces, PER)), 0, st, P);
}
template <class T, int CH>
cudaError_t forward_of(NormParams& P, cudaStream_t st) {
  if constexpr (CH * sizeof(T) == 16) {
    if (P.pieces <= 32) return forward<T, CH, 1, true>(P, st);
    if (P.pieces <= 64) return forward<T, CH, 2, true>(P, st);
    if (P.pieces <= 128) return forward<T, CH, 4, true>(P, st);
    if (P.pieces <= 256) return forward<T, CH, 8, true>(P, st);
  }
  return forward<T, CH, VALUES / CH, false>(P, st);
}

ff_status_t check_call(ff_layer_norm* h, int64_t batch, int64_t tokens, std::initializer_list<const float*> weights) {
  if (batch < 0 || tokens < 0) return fail(h, FF_ERR_INVALID_ARG, "batch and tokens must not be negative");
  if (batch > 0x7fffffff || tokens > 0x7fffffff || batch * tokens > 0x7fffffff) return fail(h, FF_ERR_UNSUPPORTED, "batch * tokens must be below 2^31");
  for (const float* w : weights)
    if (((uintptr_t)w) & 3) return fail(h, FF_ERR_INVALID_ARG, "weights, biases and their gradients must be 4-byte aligned");
  return FF_OK;
}
NormParams common(const ff_layer_norm* h, int64_t batch, int64_t tokens, const float* weight, int per_sample, int ch) {
  NormParams P{};
  P.w = weight;
  P.w_stride = per_sample ? h->cfg.dim : 0;
  P.plus = h->cfg.unit_offset ? 1.f : 0.f;
  P.tokens = (unsigned)tokens;
  P.by_tokens = ff_fast_div((unsigned)tokens);
  P.rows = (int)(batch * tokens);
  P.d = h->cfg.dim;
  P.pieces = P.d / ch;
  P.inv_d = 1.f / (float)P.d;
  P.eps = h->cfg.eps;
  return P;
}

}  // namespace

extern "C" ff_status_t ff_layer_norm_create(const ff_layer_norm_config_t* cfg, ff_layer_norm_t** out) {
  if (!cfg || !out) return fail(nullptr, FF_ERR_INVALID_ARG, "cfg or out is NULL");
  *out = nullptr;
  if (cfg->dtype != FF_BF16 && cfg->dtype != FF_FP32) return fail(nullptr, FF_ERR_INVALID_ARG, "dtype must be FF_BF16 or FF_FP32");
  if (cfg->dim < 1) return fail(nullptr, FF_ERR_INVALID_ARG, "dim must be positive");
  if (cfg->dim > MAX_DIM) return fail(nullptr, FF_ERR_UNSUPPORTED, "dim must be at most 8192");
  if (!(cfg->eps > 0.f && cfg->eps < 3.0e38f)) return fail(nullptr, FF_ERR_INVALID_ARG, "eps must be positive and finite");
  ff_layer_norm* h = new (std::nothrow) ff_layer_norm();
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "out of host memory");
  h->cfg = *cfg;
  *out = h;
  return FF_OK;
}

extern "C" ff_status_t ff_layer_norm_destroy(ff_layer_norm_t* h) {
  delete h;
  return FF_OK;
}

extern "C" const char* ff_layer_norm_last_error(const ff_layer_norm_t* h) { return h ? h->err : ff_last_error(nullptr); }

extern "C" ff_status_t ff_layer_norm_forward(const ff_layer_norm_t* handle, int64_t batch, int64_t tokens, const ff_rows_t* x, const float* weight,
                                             const float* bias, int32_t per_sample, const ff_rows_t* y, void* stream) {
  ff_layer_norm* h = const_cast<ff_layer_norm*>(handle);
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "the handle is NULL");
  ff_status_t s = check_call(h, batch, tokens, {weight, bias});
  if (s != FF_OK) return s;
  if (batch * tokens == 0) return FF_OK;
  const int e = h->cfg.dtype == FF_FP32 ? 4 : 2;
  uint64_t bits = 0;
  s = check_rows(h, x, batch, tokens, false, e, &bits);
  if (s == FF_OK) s = check_rows(h, y, batch, tokens, true, e, &bits);
  if (s != FF_OK) return s;
  const int ch = piece_of(h->cfg.dim, e, bits);
  NormParams P = common(h, batch, tokens, weight, per_sample, ch);
  P.x = view(x, e); P.y = view(y, e);
  P.bias = bias;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t err = e == 4 ? (ch == 4 ? forward_of<float, 4>(P, st) : forward_of<float, 1>(P, st))
                                 : ch == 8 ? forward_of<__nv_bfloat16, 8>(P, st) : ch == 2 ? forward_of<__nv_bfloat16, 2>(P, st) : forward_of<__nv_bfloat16, 1>(P, st);
  return err == cudaSuccess ? FF_OK : cuda_fail(h, err);
}

extern "C" ff_status_t ff_layer_norm_workspace_bytes(const ff_layer_norm_t* handle, int64_t batch, int64_t tokens, int32_t per_sample, size_t* bytes) {
  ff_layer_norm* h = const_cast<ff_layer_norm*>(handle);
  if (!h || !bytes) return fail(h, FF_ERR_INVALID_ARG, "handle or bytes is NULL");
  const ff_status_t s = check_call(h, batch, tokens, {});
  if (s != FF_OK) return s;
  const Parts p = parts_of(batch, tokens, per_sample);
  *bytes = batch * tokens == 0 || p.parts == 1 ? 0 : (size_t)p.segments * p.parts * 2 * h->cfg.dim * sizeof(float);
  return FF_OK;
}

extern "C" ff_status_t ff_layer_norm_backward(const ff_layer_norm_t* handle, int64_t batch, int64_t tokens, const ff_rows_t* x, const float* weight,
                                              int32_t per_sample, const ff_rows_t* dy, const ff_rows_t* dx, float* dweight, float* dbias,
                                              void* ws, size_t ws_bytes, void* stream) {
  ff_layer_norm* h = const_cast<ff_layer_norm*>(handle);
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "the handle is NULL");
  ff_status_t s = check_call(h, batch, tokens, {weight, dweight, dbias});
  if (s != FF_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  const int d = h->cfg.dim;
  if (batch * tokens == 0) {                 // sums over no rows
    const size_t n = (size_t)(per_sample ? batch : 1) * d * sizeof(float);
    cudaError_t err = cudaSuccess;
    if (dweight && n) err = cudaMemsetAsync(dweight, 0, n, st);
    if (err == cudaSuccess && dbias && n) err = cudaMemsetAsync(dbias, 0, n, st);
    return err == cudaSuccess ? FF_OK : cuda_fail(h, err);
  }
  const int e = h->cfg.dtype == FF_FP32 ? 4 : 2;
  uint64_t bits = 0;
  s = check_rows(h, x, batch, tokens, false, e, &bits);
  if (s == FF_OK) s = check_rows(h, dy, batch, tokens, false, e, &bits);
  if (s == FF_OK && dx) s = check_rows(h, dx, batch, tokens, true, e, &bits);
  if (s != FF_OK) return s;
  size_t need = 0;
  ff_layer_norm_workspace_bytes(handle, batch, tokens, per_sample, &need);
  if (need && (!ws || ws_bytes < need)) return fail(h, FF_ERR_WORKSPACE, "the workspace is missing or smaller than ff_layer_norm_workspace_bytes");
  if (need && (((uintptr_t)ws) & 15)) return fail(h, FF_ERR_WORKSPACE, "the workspace must be 16-byte aligned");
  if (!dx && !dweight && !dbias) return FF_OK;
  const int ch = piece_of(d, e, bits);
  const Parts parts = parts_of(batch, tokens, per_sample);
  NormParams P = common(h, batch, tokens, weight, per_sample, ch);
  P.x = view(x, e); P.g = view(dy, e);
  if (dx) P.y = view(dx, e);
  P.segment = parts.rows;
  P.parts = parts.parts;
  if (parts.parts == 1) {
    P.dw = dweight; P.db = dbias;
    P.part_stride = d;
  } else {
    P.dw = dweight ? (float*)ws : nullptr;
    P.db = dbias ? (float*)ws + d : nullptr;
    P.part_stride = 2 * d;
  }
  const unsigned blocks = parts.segments * parts.parts;
  cudaError_t err = e == 4 ? (ch == 4 ? backward<float, 4, VALUES / 4>(P, blocks, st) : backward<float, 1, VALUES>(P, blocks, st))
                           : ch == 8 ? backward<__nv_bfloat16, 8, VALUES / 8>(P, blocks, st)
                           : ch == 2 ? backward<__nv_bfloat16, 2, VALUES / 2>(P, blocks, st) : backward<__nv_bfloat16, 1, VALUES>(P, blocks, st);
  if (err == cudaSuccess && parts.parts > 1 && (dweight || dbias)) {
    const int columns = (d + 31) / 32;
    err = ff_launch(norm_join_kernel, dim3(parts.segments * columns, 2), dim3(1024), 0, st, (const float*)ws, (int)parts.parts, d, columns, dweight, dbias);
  }
  return err == cudaSuccess ? FF_OK : cuda_fail(h, err);
}
