// Cross attention of few queries a key head (a decoder's tokens, one after the other): forward pass.
//
//   out = softmax_j(scale q k_j) v,   lse = ln sum_j e^(scale q k_j),   over the keys j that count
//
// With at most eight query rows for a key head, every key and value is read once for a few products: memory is the bound, and a tile of 128 rows
// would be nearly empty.  A cluster of up to eight CTAs has a key head of a sample, each CTA a part of its keys, and each warp batches of 16 keys in
// turns, through a ring of its own in shared memory; keys that do not count are not read and are zeros.  The products are the warp's own small
// ones, with the keys (then the channels) as their 16 rows and the query rows as their 8 columns:
//   S^T = K Q^T, running maximum and sum of a column, P^T = 2^(S^T - m) as bf16 (one transposition within the warp), O^T += V^T P^T
// so a column's maximum is where its sums are.  (With fp32 products in the lanes, a key's row over 16 of them, the instructions were the bound: 8 samples,
// 4096 keys, 32 heads on 8 of 128 took 30 us.)  The warps' sums are joined in shared memory and the CTAs' over the cluster's, always in the same order.
#include "ff_cross.cuh"
#include "ff_chunks.cuh"

using namespace sm100;

namespace {

constexpr int WARPS = 4;
constexpr int BATCH = 16;                                    // keys of a warp's step
constexpr int ROWS = 8;                                      // query rows of a key head, at most
// Bytes of a warp's ring (three batches), CTAs of an SM: 128 KB of keys and values on their way to it.  (Two batches of 128 channels and three CTAs:
// the same for many CTAs, but 162 in place of 94 us for 100000 keys of 8 heads, on 64 CTAs.)
template <int HD> constexpr int RING = 3 * 2 * BATCH * HD * 2;
template <int HD> constexpr int BLOCKS = HD == 64 ? 4 : 2;
constexpr float LN2 = 0.69314718055994531f;

struct FewRows { const char* p; long long sb, sh, sn; };     // strides in bytes
struct FewParams {
  int G, group, N, K, d, parts, rows;                        // CTAs of a cluster; query rows of a key head
  const int* lengths;
  const uint8_t* mask;
  float sl2;
  FewRows q, k, v;
  char* out; long long o_sb, o_sh, o_sn;
  float* lse;                                                // or NULL
};

// What a CTA's warps, and then its cluster's CTAs, join: a row's maximum and sum, and sums of values relative to that maximum.
template <int HD> struct alignas(16) Sums { float acc[ROWS][HD]; float m[ROWS], l[ROWS]; };

// 8 x 8 tiles of bf16 from rows in shared memory (a lane gives the address of a row), as they are or transposed
__device__ __forceinline__ void tiles4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void tiles4_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t r) {
  uint32_t t;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(t) : "r"(r));
  return t;
}
// d (16 x 8, fp32) += a (16 x 16) b (16 x 8)
__device__ __forceinline__ void product(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int HD>
__global__ void __launch_bounds__(WARPS * 32, BLOCKS<HD>)
cross_few_kernel(const __grid_constant__ FewParams P) {
  constexpr int CHUNKS = HD / 8, AT_ONCE = 32 / CHUNKS;      // 16-byte chunks of a row; rows that a warp copies at once
  constexpr int STEPS = HD / 16;
  constexpr int HALF = BATCH * HD * 2, STAGES = 3;      // bytes of a batch's keys (its values lie behind them)
  extern __shared__ __align__(128) uint8_t few_smem[];
  __shared__ Sums<HD> total;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int bg = blockIdx.x / P.parts, part = blockIdx.x - bg * P.parts;
  const int b = bg / P.G, g = bg - b * P.G;

  ff_pdl_wait();
  int keys = P.K;
  if (P.lengths) { const int n = __ldg(P.lengths + b); keys = n < 0 ? 0 : n < keys ? n : keys; }
  const int each = keys / P.parts, rest = keys - each * P.parts;
  const int k0 = each * part + (part < rest ? part : rest), k1 = k0 + each + (part < rest ? 1 : 0);

  // Q^T: row lane / 4 of the queries, its channels in pairs
  uint32_t q[STEPS][2];
  {
    const int r = lane >> 2, h = r / P.N;
    const char* row = P.q.p + b * P.q.sb + (long long)(g * P.group + h) * P.q.sh + (long long)(r - h * P.N) * P.q.sn;
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int c = s * 16 + i * 8 + (lane & 3) * 2;
        q[s][i] = r < P.rows && c < P.d ? *(const uint32_t*)(row + c * 2) : 0u;
      }
  }

  // ---- the ring: rows of HD channels, the chunks of row r at places ^ (r & 7)
  uint8_t* ring = few_smem + warp * RING<HD>;
  const int cc = lane % CHUNKS, cr = lane / CHUNKS;
  const char *kp = P.k.p + b * P.k.sb + g * P.k.sh + cc * 16, *vp = P.v.p + b * P.v.sb + g * P.v.sh + cc * 16;
  const uint8_t* mp = P.mask ? P.mask + (long long)b * P.K : nullptr;
  const bool mine = cc * 8 < P.d;
  auto counting = [&](int batch) {                           // a bit for each of its keys
    const int key = batch + (lane & 15);
    return __ballot_sync(0xffffffffu, key < k1 && (!mp || __ldg(mp + key) != 0)) & 0xffffu;
  };
  auto copy = [&](int batch, int stage, unsigned bits) {
    uint8_t* to = ring + stage * 2 * HALF;
#pragma unroll
    for (int i = 0; i < BATCH / AT_ONCE; ++i) {
      const int r = i * AT_ONCE + cr;
      const bool on = (bits >> r & 1) && mine;
      const long long key = on ? batch + r : 0;
      uint8_t* at = to + r * HD * 2 + ((cc ^ (r & 7)) * 16);
      copy_async<16>(at, kp + key * P.k.sn, on);
      copy_async<16>(at + HALF, vp + key * P.v.sn, on);
    }
  };

  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};    // of query rows 2 (lane % 4) and the next; of the sums, this lane's keys
  float acc[STEPS][4];                                       // O^T: channels lane / 4 and 8 more, these rows
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[s][i] = 0.f;

  constexpr int STEP = WARPS * BATCH;
  unsigned on_way[STAGES], any = 0;                          // bits of the batches in the ring, the oldest first; of all so far
  int ahead = k0 + warp * BATCH;
  unsigned bits = counting(ahead);
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) {
    copy(ahead, s, bits);
    copy_commit();
    on_way[s] = bits;
    ahead += STEP;
    bits = counting(ahead);
  }
  const uint32_t ring_at = smem_u32(ring);
  int stage = 0;
  for (int batch = k0 + warp * BATCH; batch < k1; batch += STEP) {
    copy_wait<STAGES - 2>();
    __syncwarp();                                            // (all lanes' pieces are there, and all have read the batch before)
    copy(ahead, stage == 0 ? STAGES - 1 : stage - 1, bits);  // (in its place)
    copy_commit();
    on_way[STAGES - 1] = bits;
    ahead += STEP;
    bits = counting(ahead);                                  // (asked for a batch ahead of its use)
    const unsigned now = on_way[0];
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) on_way[s] = on_way[s + 1];
    any |= now;
    const uint32_t keys_at = ring_at + stage * 2 * HALF, values_at = keys_at + HALF;
    float s[2][4] = {};                                      // two chains
    const int row = lane & 15, sw = row & 7, hi = lane >> 4;
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      uint32_t a[4];
      tiles4(a, keys_at + row * HD * 2 + (((2 * t + hi) ^ sw) * 16));
      product(s[t & 1], a, q[t][0], q[t][1]);
    }
    float sc[4];                                             // keys lane / 4 (0, 1) and 8 more (2, 3), rows of m[0] and m[1]
#pragma unroll
    for (int i = 0; i < 4; ++i) sc[i] = now >> ((lane >> 2) + (i >> 1) * 8) & 1 ? (s[0][i] + s[1][i]) * P.sl2 : -INFINITY;
    float most[2] = {fmaxf(sc[0], sc[2]), fmaxf(sc[1], sc[3])};
    if (__any_sync(0xffffffffu, most[0] > m[0] || most[1] > m[1])) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) most[i] = fmaxf(most[i], __shfl_xor_sync(0xffffffffu, most[i], x));
        const float to = fmaxf(m[i], most[i]), factor = to == -INFINITY ? 1.f : ex2(m[i] - to);
        m[i] = to;
        l[i] *= factor;
#pragma unroll
        for (int t = 0; t < STEPS; ++t) { acc[t][i] *= factor; acc[t][2 + i] *= factor; }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float ref = m[i & 1];
      sc[i] = ex2(sc[i] - (ref == -INFINITY ? 0.f : ref));
      l[i & 1] += sc[i];
    }
    // (bf16 is what the product takes, the sum is of the unrounded: see the tiles' kernel)
    const uint32_t p0 = transposed(bf16_pair(__float_as_uint(sc[0]), __float_as_uint(sc[1])));
    const uint32_t p1 = transposed(bf16_pair(__float_as_uint(sc[2]), __float_as_uint(sc[3])));
    // V^T: rows of eight keys and channels, transposed; channels 0 .. 7 and 8 .. 15 of the first eight keys, then of the others
    const int vrow = (lane & 7) + (lane >> 4) * 8, vhi = lane >> 3 & 1;
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      uint32_t a[4];
      tiles4_trans(a, values_at + vrow * HD * 2 + (((2 * t + vhi) ^ (vrow & 7)) * 16));
      product(acc[t], a, p0, p1);
    }
    stage = stage + 1 == STAGES ? 0 : stage + 1;
  }
  copy_wait<0>();

  // ---- join: the lanes' keys
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
  __syncthreads();                                           // (the rings are free)
  Sums<HD>* sums = (Sums<HD>*)few_smem;
#pragma unroll
  for (int t = 0; t < STEPS; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[warp].acc[(lane & 3) * 2 + (i & 1)][t * 16 + (lane >> 2) + (i >> 1) * 8] = acc[t][i];
  if (lane < 4)
#pragma unroll
    for (int i = 0; i < 2; ++i) { sums[warp].m[lane * 2 + i] = m[i]; sums[warp].l[lane * 2 + i] = any ? l[i] : -1.f; }   // (a sum below zero: no key counted)
  __syncthreads();
  // ---- the CTA's warps
  auto weigh = [&](const float (&ms)[8], const float (&ls)[8], int n, float (&w)[8], float& top, float& sum) {
    top = -INFINITY; sum = -1.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) top = fmaxf(top, ms[i]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = 0.f;
      if (i < n && ls[i] != -1.f) {
        w[i] = ex2(ms[i] - ref);
        sum = (sum == -1.f ? 0.f : sum) + ls[i] * w[i];
      }
    }
  };
  for (int e = threadIdx.x; e < ROWS * HD / 4; e += WARPS * 32) {
    const int r = e / (HD / 4), at = e % (HD / 4) * 4;
    float ms[8], ls[8], w[8], top, sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) { ms[i] = i < WARPS ? sums[i % WARPS].m[r] : 0.f; ls[i] = i < WARPS ? sums[i % WARPS].l[r] : 0.f; }
    weigh(ms, ls, WARPS, w, top, sum);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < WARPS; ++i)
      if (ls[i] != -1.f) {
        const float4 a = *(const float4*)&sums[i].acc[r][at];
        o.x += a.x * w[i]; o.y += a.y * w[i]; o.z += a.z * w[i]; o.w += a.w * w[i];
      }
    *(float4*)&total.acc[r][at] = o;
    if (at == 0) { total.m[r] = top; total.l[r] = sum; }
  }
  // ---- the cluster's CTAs: each has a share of the values
  if (P.parts > 1) cluster_sync();
  else __syncthreads();
  for (int e = threadIdx.x * P.parts + part; e < P.rows * (P.d / 8); e += WARPS * 32 * P.parts) {
    const int r = e / (P.d / 8), at = (e - r * (P.d / 8)) * 8;
    float ms[8], ls[8], w[8], top, sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      ms[i] = ls[i] = -1.f;
      if (i < P.parts) {
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(ms[i]) : "r"(map_shared(&total.m[r], i)) : "memory");
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(ls[i]) : "r"(map_shared(&total.l[r], i)) : "memory");
      }
    }
    weigh(ms, ls, P.parts, w, top, sum);
    const bool some = sum != -1.f;
    const float inv = some ? 1.f / sum : 0.f;
    float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < P.parts && ls[i] != -1.f) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float4 a;
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(a.x), "=f"(a.y), "=f"(a.z), "=f"(a.w) : "r"(map_shared(&total.acc[r][at + 4 * j], i)) : "memory");
          o[4 * j] += a.x * w[i]; o[4 * j + 1] += a.y * w[i]; o[4 * j + 2] += a.z * w[i]; o[4 * j + 3] += a.w * w[i];
        }
      }
    const int h = r / P.N, n = r - h * P.N;
    uint32_t pk[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) pk[i] = bf16_pair(__float_as_uint(o[2 * i] * inv), __float_as_uint(o[2 * i + 1] * inv));
    *(uint4*)(P.out + b * P.o_sb + (long long)(g * P.group + h) * P.o_sh + n * P.o_sn + at * 2) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
    if (P.lse && at == 0) P.lse[((long long)b * P.G * P.group + g * P.group + h) * P.N + n] = some ? (top + log2f(sum)) * LN2 : -INFINITY;
  }
  if (P.parts > 1) cluster_sync();                           // (the others may still read here)
}

}  // namespace

cudaError_t cx_few_init() {
  const cudaError_t e = cudaFuncSetAttribute(cross_few_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, WARPS * RING<64>);
  return e != cudaSuccess ? e : cudaFuncSetAttribute(cross_few_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, WARPS * RING<128>);
}

// Parts of the keys: the fewest keys for the SM that has most of them, where starting and joining takes as long as some 64 keys.
static int parts_of(const CrossDims& D, long long* waves) {
  const long long room = (D.d > 64 ? BLOCKS<128> : BLOCKS<64>) * FF_B200_SMS;
  long long best = 1, least = 0;
  for (int parts = 1; parts <= 8 && (parts == 1 || parts * 64ll <= D.K); ++parts) {
    const long long turns = ((long long)D.B * D.G * parts + room - 1) / room, cost = turns * ((D.K + parts - 1) / parts + 64);
    if (parts == 1 || cost < least) { least = cost; best = parts; *waves = turns; }
  }
  return (int)best;
}
// Estimated time (us): a CTA takes 70 bytes of keys and values a ns, all of them 6000.
double cx_few_us(const CrossDims& D) {
  if ((long long)D.group * D.N > ROWS || D.K > 1 << 30) return 1e30;
  long long waves = 1;
  const int parts = parts_of(D, &waves);
  const double row = D.d > 64 ? 512 : 256, cta = (double)waves * ((D.K + parts - 1) / parts) * row / 70e3, all = (double)D.B * D.G * D.K * row / 6e6;
  return 4 + (cta > all ? cta : all);
}

cudaError_t cx_few_forward(const CrossDims& D, const ff_heads_t* q, const ff_heads_t* k, const ff_heads_t* v, const ff_heads_t* out, float* lse, cudaStream_t st) {
  auto rows_of = [](const ff_heads_t* t) {
    return FewRows{(const char*)t->data, (long long)t->stride_batch * 2, (long long)t->stride_head * 2, (long long)t->stride_token * 2};
  };
  FewParams P{};
  P.G = D.G; P.group = D.group; P.N = D.N; P.K = D.K; P.d = D.d;
  long long waves = 1;
  P.parts = parts_of(D, &waves);
  P.rows = D.group * D.N;
  P.lengths = D.lengths; P.mask = D.mask; P.sl2 = D.sl2;
  P.q = rows_of(q); P.k = rows_of(k); P.v = rows_of(v);
  const FewRows o = rows_of(out);
  P.out = (char*)out->data; P.o_sb = o.sb; P.o_sh = o.sh; P.o_sn = o.sn;
  P.lse = lse;
  const auto kernel = D.d > 64 ? cross_few_kernel<128> : cross_few_kernel<64>;
  return ff_launch_cluster(kernel, dim3((unsigned)(D.B * D.G * P.parts)), dim3(WARPS * 32), P.parts, WARPS * (D.d > 64 ? RING<128> : RING<64>), st, P);
}
