// Cross attention: what the forward and backward launches share.
//
// Work is laid out by tiles of 128 query rows.  The heads of a group (those that read one key head) read the same keys, so a
// tile's rows may be of any of them: with at least 65 query tokens a tile is 128 tokens of one head, with fewer as many whole heads
// of the group as fit.  A tile of keys is 128 keys of one key head.
#pragma once
#include "ff_internal.h"
#include "ff_sm100.cuh"

struct ff_cross_attention {
  ff_cross_attention_config_t cfg;
  int device;
  float scale;
  int* status;                 // device
  int64_t sizes[4];            // batch, queries, keys and training of the last call, and the workspace that it takes
  size_t need;
  char err[512];
};

constexpr int CX_TILE = 128;

// x / d for 0 <= x < 2^31 as a product (Granlund and Montgomery 1994): with 2^s >= d > 2^(s-1) and m = (2^(31+s) + e) / d, 0 < e <= d, the product
// x m / 2^(31+s) is above x / d by less than 1 / d.  A kernel's roles each find their items' places by four or five divisions one after the other:
// 1200 cycles for each item as plain divisions.
struct CxDiv {
  unsigned m;
  int shift;
#if defined(__CUDACC__)
  __device__ __forceinline__ int operator()(int x) const { return (int)((unsigned long long)(unsigned)x * m >> shift); }
#endif
};
inline CxDiv cx_div(int d) {
  int s = 0;
  while (s < 31 && (1ll << s) < d) ++s;
  return CxDiv{d > 0 ? (unsigned)((1ull << (31 + s)) / (unsigned)d + 1) : 0u, 31 + s};
}

struct CrossDims {
  int B, H, G, group;          // samples, heads, key heads, heads of a key head
  int N, K, d;                 // query tokens, keys, channels
  int bn, bh;                  // tokens and heads of a tile of queries
  int n_tiles, tiles;          // tiles along the tokens, tiles of a key head of a sample
  int once[3][2];              // q, k, v: coordinate factors (0: the same rows for all) of batch and head
  CxDiv by_bn, by_n_tiles, by_tiles, by_G;
  const int* lengths;
  const uint8_t* mask;
  float scale, sl2;            // scale; scale * log2(e)
  int* status;
};

#if defined(__CUDACC__)
// Keys of sample b that may count, and tiles of them.
__device__ __forceinline__ int cx_keys(const CrossDims& D, int b) {
  if (!D.lengths) return D.K;
  const int n = __ldg(D.lengths + b);
  return n < 0 ? 0 : n < D.K ? n : D.K;
}
// The first of n steps that part `part` of `parts` has: n part / parts.
__device__ __forceinline__ int cx_first(int n, int part, int parts, const CxDiv& by_parts) {
  const int each = by_parts(n);
  return each * part + by_parts((n - each * parts) * part);
}
// A value that all lanes have, from the first of them: so the compiler knows that they do, and keeps what follows from it (loops over tiles,
// operands of the tensor core's instructions) in registers of the warp.  Otherwise each operand is moved there for each instruction.
__device__ __forceinline__ int cx_uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
// Does tile j of a sample with `keys` keys hold rows that do not count, yet have been loaded?
template <int KEYS>
__device__ __forceinline__ bool cx_unclean(const CrossDims& D, int keys, int j) {
  return D.mask || (keys < D.K && (j + 1) * KEYS > keys);
}
// The keys of a tile that count, as the bits of four words: bit l of word k is key 4 l + k.  All 32 lanes.
struct CxValid { uint32_t w[4]; };
__device__ __forceinline__ CxValid cx_valid(const CrossDims& D, int b, int keys, int j, int lane) {
  CxValid v;
  const long long at = (long long)b * D.K;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int key = j * CX_TILE + 4 * lane + k;
    const bool on = key < keys && (!D.mask || __ldg(D.mask + at + key) != 0);
    v.w[k] = __ballot_sync(0xffffffffu, on);
  }
  return v;
}
// Of 64 keys from `first` on, those that count: bit l of word k is key first + 2 l + k.  All 32 lanes.
struct CxValid64 { uint32_t w[2]; };
__device__ __forceinline__ CxValid64 cx_valid64(const CrossDims& D, int b, int keys, int first, int lane) {
  CxValid64 v;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int key = first + 2 * lane + k;
    v.w[k] = __ballot_sync(0xffffffffu, key < keys && (!D.mask || __ldg(D.mask + (long long)b * D.K + key) != 0));
  }
  return v;
}
// First head and token of tile t of key head g.
__device__ __forceinline__ void cx_place(const CrossDims& D, int g, int t, int& h0, int& n0) {
  const int pack = D.by_n_tiles(t);
  h0 = g * D.group + pack * D.bh;
  n0 = (t - pack * D.n_tiles) * D.bn;
}
// Loads a tile of rows (halves of 64 channels, `bytes` apart in shared memory); the caller has announced its bytes.
__device__ __forceinline__ void cx_load(uint8_t* dst, int bytes, int halves, const CUtensorMap* map, uint64_t* bar, int n, int h, int b) {
  sm100::tma_load_4d(dst, map, bar, 0, n, h, b);
  if (halves > 1) sm100::tma_load_4d(dst + bytes, map, bar, 64, n, h, b);
}
// The same tile on its way into L2.
__device__ __forceinline__ void cx_prefetch(int halves, const CUtensorMap* map, int n, int h, int b) {
  sm100::tma_prefetch_4d(map, 0, n, h, b);
  if (halves > 1) sm100::tma_prefetch_4d(map, 64, n, h, b);
}
// Zeros in the rows of a tile in shared memory (rows of 128 bytes, halves `bytes` apart) whose keys do not count: in the product they
// meet probabilities of zero, and zero times what may stand there need not be zero.  W words of valid bits: bit l of word k is row
// W l + k.  All 32 lanes.
template <int W>
__device__ __forceinline__ void cx_clean(uint8_t* tile, int bytes, int halves, const uint32_t (&valid)[W], int lane) {
  const int sub = lane >> 3;                                 // four rows at a time, eight lanes of 16 bytes each
  uint32_t mine = valid[0];
#pragma unroll
  for (int k = 1; k < W; ++k)
    if (sub % W == k) mine = valid[k];
  uint8_t* to = tile + lane * 16;
#pragma unroll 8
  for (int i = 0; i < 8 * W; ++i)                            // rows 4 i + sub
    if (!(mine >> (i * 4 / W + sub / W) & 1))
      for (int h = 0; h < halves; ++h) *(uint4*)(to + h * bytes + i * 512) = make_uint4(0, 0, 0, 0);
  sm100::fence_proxy_async();
}
// Puts 32 consecutive fp32 values of a row (columns 32 c .. of the 64 of a swizzled half in shared memory) there as bf16.
__device__ __forceinline__ void cx_stage(uint8_t* half, int row, int c, const uint32_t (&r)[32], float factor) {
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = sm100::bf16_pair(__float_as_uint(__uint_as_float(r[v * 8 + 2 * i]) * factor), __float_as_uint(__uint_as_float(r[v * 8 + 2 * i + 1]) * factor));
    *(uint4*)(half + row * 128 + (((c * 4 + v) ^ (row & 7)) * 16)) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
#endif

// A map over the rows of head rows: [batch][heads][tokens][head_dim] with boxes of 64 channels, `rows` tokens and `heads` heads.
bool cx_map(CUtensorMap* map, const ff_heads_t* t, int64_t batch, int64_t tokens, int d, int rows, int heads);
// At most eight query rows for a key head: a kernel of its own, and what it is expected to take (never where it cannot).
cudaError_t cx_few_init();
double cx_few_us(const CrossDims& D);
cudaError_t cx_few_forward(const CrossDims& D, const ff_heads_t* q, const ff_heads_t* k, const ff_heads_t* v, const ff_heads_t* out, float* lse, cudaStream_t st);
cudaError_t cx_backward_init();
cudaError_t cx_backward(const CrossDims& D, const ff_heads_t* q, const ff_heads_t* k, const ff_heads_t* v, const ff_heads_t* out, const float* lse,
                        const ff_heads_t* dout, const ff_heads_t* dq, const ff_heads_t* dk, const ff_heads_t* dv, void* ws, cudaStream_t st);
size_t cx_backward_bytes(const CrossDims& D);
