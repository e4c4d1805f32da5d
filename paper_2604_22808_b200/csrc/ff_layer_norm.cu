// Layer norm of rows of dim values, forward and backward, with weights and bias of the model or of each sample.
//
//   forward    c = x - mean,  r = 1 / sqrt(mean(c^2) + eps),  n = c r,  y = n w + b      (w = 1 + weight with unit_offset)
//   backward   g = dy w;  dx = r (g - mean(g) - n mean(g n));  dweight = sum over rows of dy n;  dbias = sum over rows of dy
//
// One pass over the rows: a row is read once, stays in registers, and is written once, so memory bounds it: 2 (backward 3) tensors.
// The mean is subtracted before the squares are summed (the values are in registers, a second sum costs no memory traffic).  A mean of
// fp32 values is off by 2^-24 of itself for every addition in a chain, 32 at most.  Rows whose mean is above 16 deviations, where that
// would count, are centred again (centre_again), so that n is off by less than 2^-14 however far from zero a row lies.
//
// A team of threads, a warp or a block, takes rows in turns, every thread the same channels of each (32 at most), so that weights, bias and,
// backward, the gradients' sums of those channels stay in its registers; the next rows are on their way while these are summed.
#include <float.h>
#include <stdio.h>

#include <initializer_list>
#include <new>
#include <type_traits>

#include "ff_chunks.cuh"
#include "ff_internal.h"

struct ff_layer_norm {
  ff_layer_norm_config_t cfg;
  char err[512];
};

namespace {

// Values of a row that a thread has (in pieces of one value 8, where more of them have to be on their way, or 16; forward in pieces of two 16: 20000 x
// 1154 bf16 42 us instead of 48, 9999 x 6002 72 instead of 98, backward 45 and 175 instead of 41 and 143).  With 32 instead of 16 the
// shuffles, barriers and addresses of a row are shared by twice the values: 16384 x 1024 bf16 backward 24 us instead of 30, 32768 x 5120
// forward 114 instead of 148 (65536 x 2048 forward: 100, with 16 and two rows at a time 89).  Weights and both sums then leave room for
// one block of eight warps on an SM backward; three blocks of four, which spill, took 36 to 60 us for the former.
constexpr int VALUES = 32;
constexpr int MAX_DIM = 8192, MAX_THREADS = 512;
constexpr int BLOCK_WARPS = 8;                    // warps of a block, unless a team has more
constexpr int EIGHTS_WARPS = 16;                  // warps on an SM, backward, of the kernel whose threads have 8 values that come one by one
// Forward, warps on an SM by the registers of their kernels: 64 with up to 8 values a thread (80 where they come one by one), 96 with 16, else 128.
// (16 for all: 11000 x 1155 fp32 33.5 us instead of 25.6, 20000 x 1155 bf16 54 instead of 36.5.)
template <int CH, int PER> constexpr int FORWARD_WARPS = CH * PER <= (CH > 1 ? 8 : 4) ? 32 : CH * PER <= (CH > 1 ? 16 : 8) ? (CH > 1 ? 20 : 24) : 16;
template <class T> constexpr int STAGES = sizeof(T) == 4 ? 3 : 4;   // rows of a team on their way or being read

struct RowsView { char* p; long long sb, st; };   // strides in bytes
struct NormParams {
  RowsView x, y, g;                 // input, output (backward: dx, or p NULL), gradient of the forward pass's output
  const float *w, *bias;            // or NULL
  long long w_stride;               // dim: weights of each sample; 0: of the model
  float plus;                       // added to the weight
  float *dw, *db;                   // backward: where a block's sums go (or NULL) ...
  long long part_stride;            // ... and how far those of the blocks are apart
  int even;                         // the rows of a segment lie at one distance
  unsigned tokens, segment, parts;  // tokens of a sample; rows whose gradients are summed together, blocks that do it
  FFFastDiv by_tokens;
  int rows, d, pieces, team_warps;
  float inv_d, least, eps;          // 1 / d, d / 256
};

__device__ __forceinline__ unsigned divide(unsigned n, const FFFastDiv& f) { return (unsigned)(((unsigned long long)__umulhi(n, f.m) + n) >> f.s); }
// A team: `warps` neighbouring warps of a block, which holds several.
struct Team { int warps, index, teams, thread, threads; };
template <bool WARP>
__device__ __forceinline__ Team team_of(const NormParams& P) {
  Team t;
  t.warps = WARP ? 1 : P.team_warps;
  const int warp = threadIdx.x >> 5;
  t.teams = (blockDim.x >> 5) / t.warps;
  t.index = warp / t.warps;
  t.threads = t.warps * 32;
  t.thread = threadIdx.x - t.index * t.threads;
  return t;
}
// Sums over a team, whose warps' sums meet in a place of their own: four at a time are read (one after the other they took
// longer than the rest of the row).
template <int WARPS> using Place = float[BLOCK_WARPS][WARPS];  // [team][warp]
template <bool WARP, int K, int PLACE>
__device__ __forceinline__ void team_sum(const Team& t, float (&v)[K], float (*place)[BLOCK_WARPS][PLACE]) {
  static_assert(K <= 4, "");
  const int lane = threadIdx.x & 31;
  // With several sums a lane gives away half of them at the first exchanges and goes on with the others.
  float mine = v[0];
  int which = 0;
  if constexpr (K > 2) {
    const bool h = lane & 16, g = lane & 8;
    const float v3 = K > 3 ? v[K - 1] : 0.f;
    const float k0 = (h ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, h ? v[0] : v[2], 16), k1 = (h ? v3 : v[1]) + __shfl_xor_sync(0xffffffffu, h ? v[1] : v3, 16);
    mine = (g ? k1 : k0) + __shfl_xor_sync(0xffffffffu, g ? k0 : k1, 8);
    which = (lane >> 3) & 3;
  } else if constexpr (K == 2) {
    const bool h = lane & 16;
    mine = (h ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, h ? v[0] : v[1], 16);
    which = lane >> 4;
  }
#pragma unroll
  for (int m = K > 2 ? 4 : K == 2 ? 8 : 16; m; m >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, m);
  if constexpr (WARP) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = K == 1 ? mine : __shfl_sync(0xffffffffu, mine, K == 2 ? 16 * k : 8 * k);
  } else {
    if ((lane & (K > 2 ? 7 : K == 2 ? 15 : 31)) == 0 && which < K) place[which][t.index][t.thread >> 5] = mine;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + t.index), "r"(t.threads) : "memory");
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float4 s = *(const float4*)place[k][t.index];
#pragma unroll
      for (int w = 4; w < PLACE; w += 4)
        if (w < t.warps) {
          const float4 u = *(const float4*)(place[k][t.index] + w);
          s.x += u.x; s.y += u.y; s.z += u.z; s.w += u.w;
        }
      v[k] = (s.x + s.y) + (s.z + s.w);
    }
  }
}
// (the places of warps that a team does not have)
template <bool WARP, int K, int PLACE>
__device__ __forceinline__ void clear(float (&place)[K][BLOCK_WARPS][PLACE]) {
  if constexpr (!WARP) {
    for (int i = threadIdx.x; i < K * BLOCK_WARPS * PLACE; i += blockDim.x) (&place[0][0][0])[i] = 0.f;
    __syncthreads();
  }
}

// A thread's pieces of a row, every `threads`-th of the team: their first channels, and whether the row has them.
// FULL: it has them all.
template <int CH, int PER, bool FULL>
struct Mine {
  int at[PER];
  bool on[PER];
  __device__ __forceinline__ Mine(const Team& t, int pieces) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int piece = t.thread + i * t.threads;
      on[i] = piece < pieces;
      at[i] = FULL || on[i] ? piece * CH : 0;
    }
  }
  __device__ __forceinline__ bool have(int i) const { return FULL || on[i]; }
};
template <class T, int CH, int PER, bool FULL>
struct Row {
  static constexpr int N = pairs_of(CH);
  using C = Chunk<T, CH>;
  // Pairs of a piece's neighbouring values; of two pieces' single ones (each beside a zero they took 40 registers and a third of the instructions
  // more: 9999 x 3001 fp32 backward 173 us instead of 98).
  static constexpr int GROUPS = CH > 1 ? PER : PER / 2;
  static_assert(CH > 1 || PER % 2 == 0, "");
  using V = F2[GROUPS][N];
  using M = Mine<CH, PER, FULL>;
  static __device__ __forceinline__ void put(V& v, int i, const C& piece) {
    if constexpr (CH > 1) {
      unpack<T, CH>(piece, v[i]);
    } else {
      F2 one[1];
      unpack<T, 1>(piece, one);
      v[i / 2][0] = i & 1 ? two(low(v[i / 2][0]), low(one[0])) : two(low(one[0]), 0.f);
    }
  }
  static __device__ __forceinline__ float value(const V& v, int i, int c) {
    if constexpr (CH > 1) return c & 1 ? high(v[i][c / 2]) : low(v[i][c / 2]);
    else return i & 1 ? high(v[i / 2][0]) : low(v[i / 2][0]);
  }
  static __device__ __forceinline__ void load(V& v, const char* row, const M& m) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const C none{};
      put(v, i, m.have(i) ? *(const C*)(row + m.at[i] * sizeof(T)) : none);
    }
  }
  static __device__ __forceinline__ void store(char* row, const V& v, const M& m) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (m.have(i)) {
        if constexpr (CH > 1) {
          *(C*)(row + m.at[i] * sizeof(T)) = pack<T, CH>(v[i]);
        } else {
          const F2 one[1] = {two(value(v, i, 0), 0.f)};
          *(C*)(row + m.at[i] * sizeof(T)) = pack<T, 1>(one);
        }
      }
  }
  static __device__ __forceinline__ float sum(const V& v) {
    F2 s = two(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int c = 0; c < N; ++c) s = __fadd2_rn(s, v[i][c]);
    return low(s) + high(s);
  }
  static __device__ __forceinline__ float dot(const V& u, const V& v) {
    F2 s = two(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int c = 0; c < N; ++c) s = fma(u[i][c], v[i][c], s);
    return low(s) + high(s);
  }
  static __device__ __forceinline__ void times(V& v, float f) {
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int c = 0; c < N; ++c) v[i][c] = mul(v[i][c], two(f, f));
  }
  // Values minus `m`, and zeros where the row has none.
  static __device__ __forceinline__ void centre(V& v, float mean, const M& m) {
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      if constexpr (CH > 1) {
        const float mine = m.have(i) ? -mean : 0.f;
#pragma unroll
        for (int c = 0; c < N; ++c) v[i][c] = __fadd2_rn(v[i][c], two(mine, mine));
      } else {
        v[i][0] = __fadd2_rn(v[i][0], two(m.have(2 * i) ? -mean : 0.f, m.have(2 * i + 1) ? -mean : 0.f));
      }
    }
  }
  // Neighbouring weights of a piece, `plus` more, or `none` where there are none.
  static __device__ __forceinline__ void weights(V& w, const float* from, float plus, float none, const M& m) {
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int c = 0; c < N; ++c) {
        if constexpr (CH > 1) w[i][c] = from && m.have(i) ? two(from[m.at[i] + 2 * c] + plus, from[m.at[i] + 2 * c + 1] + plus) : two(none, none);
        else w[i][c] = two(from && m.have(2 * i) ? from[m.at[2 * i]] + plus : none, from && m.have(2 * i + 1) ? from[m.at[2 * i + 1]] + plus : none);
      }
  }
};
// A team's rows on their way: every thread copies its own pieces of them into places of its own in shared memory, STAGES - 1 sets of rows
// ahead.  (Pieces of two bytes cannot be copied that way: one set ahead, in registers.)
template <class T, int CH, int PER, bool FULL, int SET>
struct Ring {
  using R = Row<T, CH, PER, FULL>;
  using C = typename R::C;
  static constexpr bool SHARED = sizeof(C) >= 4;
  unsigned char* places;                                       // [stage][row of the set][piece][thread of the block]
  int stage, stage_bytes;
  C raw[SHARED ? 1 : SET][SHARED ? 1 : PER];
  __device__ __forceinline__ Ring(void* shared) : places((unsigned char*)shared + threadIdx.x * sizeof(C)), stage(0), stage_bytes(SET * PER * (int)sizeof(C) * (int)blockDim.x) {}
  __device__ __forceinline__ C* place(int s, int row, int piece) const { return (C*)(places + s * stage_bytes + (row * PER + piece) * (int)sizeof(C) * (int)blockDim.x); }
  // Row `k` of the set that goes into stage `to` (the row is there or not).
  __device__ __forceinline__ void ask(int to, int k, const char* row, bool there, const typename R::M& m) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const char* from = row + m.at[i] * sizeof(T);
      if constexpr (SHARED) {
        copy_async<sizeof(C)>(place(to, k, i), from, there && m.have(i));
      } else {
        const C none{};
        raw[k][i] = there && m.have(i) ? *(const C*)from : none;
      }
    }
  }
  __device__ __forceinline__ void asked() { if constexpr (SHARED) copy_commit(); }
  __device__ __forceinline__ void arrived() { if constexpr (SHARED) copy_wait<STAGES<T> - 2>(); }
  __device__ __forceinline__ void take(int k, typename R::V& v) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if constexpr (SHARED) R::put(v, i, *place(stage, k, i));
      else R::put(v, i, raw[k][i]);
    }
  }
  // The stage that has just been read is asked for again, and the next one follows.
  __device__ __forceinline__ int next() {
    const int was = stage;
    stage = stage + 1 == STAGES<T> ? 0 : stage + 1;
    return was;
  }
};
template <class T, int CH, int PER, int SET>
constexpr size_t ring_bytes(int threads) { return sizeof(T) * CH >= 4 ? (size_t)STAGES<T> * SET * PER * sizeof(T) * CH * threads : 0; }
constexpr float DOWN = 8.2718061255302767e-25f;                // 2^-80, for rows whose squares (or sum) leave fp32 ...
constexpr float MOST = 3.0e38f;                                // ... when they are beyond this
// Squares beyond fp32, or below `least`: a mean of more than 16 deviations, whose rounding, and that of its sum, count among them.
__device__ __forceinline__ bool far_from_centred(float squares, float least) { return !(squares < MOST && squares >= least); }
template <class T> __device__ __forceinline__ float value_at(const char* row, int c) {
  if constexpr (sizeof(T) == 4) return ((const float*)row)[c];
  else return __uint_as_float((unsigned)((const unsigned short*)row)[c] << 16);
}

// Row `at` of a segment, and the team's way from one to the next.  (Rows that follow one another at one distance, of a sample or of a whole
// contiguous batch, need no division.)
__device__ __forceinline__ char* row_at(const RowsView& v, const NormParams& P, unsigned segment, unsigned at) {
  if (P.even) return v.p + (long long)segment * v.sb + (long long)at * v.st;
  const unsigned b = divide(at, P.by_tokens), n = at - b * P.tokens;          // (then there is one segment)
  return v.p + (long long)b * v.sb + (long long)n * v.st;
}
struct Way {
  char* p;
  long long step;
  __device__ __forceinline__ Way(const RowsView& v, const NormParams& P, unsigned segment, unsigned at, unsigned stride)
      : p(row_at(v, P, segment, at)), step((long long)stride * v.st) {}
  __device__ __forceinline__ void to(const RowsView& v, const NormParams& P, unsigned at) {
    if (P.even) p += step;
    else p = row_at(v, P, 0, at);
  }
};

// A row that one mean does not centre (far_from_centred), once more from memory, `factor` times it where its squares leave fp32.  The mean of what the
// mean left is taken away too, and that of what this left.  Where all values are the same, the mean is the first of them: minus it they are
// zeros, or NaN, and eps counts as it is.
// A call of its own, piece by piece, so that such rows, which are rare, take no registers from the others: in its place it cost 20000 x 1154 bf16 forward 47 us
// in place of 45, 9999 x 3001 fp32 backward 103 in place of 99.  (A tensor of such rows alone takes two to three times as long: 65536 x 2048 bf16 283 us.)
// AT_ONCE pieces at a time: one, but four backward where rows of several warps come value by value, whose kernel then spills nothing (8000 x 2051 bf16
// 73 us in place of 93).
struct Centre { float factor, mean[3], squares; };
template <class T, int CH, int AT_ONCE, bool WARP, int PLACE>
__device__ __noinline__ Centre centre_again(const char* row, float factor, const NormParams& P, const Team& team, float (*place)[BLOCK_WARPS][PLACE]) {
  auto each = [&](auto&& use) {
#pragma unroll(AT_ONCE)
    for (int piece = team.thread; piece < P.pieces; piece += team.threads) {
      F2 v[pairs_of(CH)];
      unpack<T, CH>(*(const Chunk<T, CH>*)(row + piece * (int)sizeof(Chunk<T, CH>)), v);
#pragma unroll
      for (int c = 0; c < CH; ++c) use(c & 1 ? high(v[c / 2]) : low(v[c / 2]));
    }
  };
  const float first = value_at<T>(row, 0);
  float s[2] = {0.f, 0.f};
  each([&](float x) { s[0] = fmaf(x, factor, s[0]); s[1] += x != first ? 1.f : 0.f; });
  team_sum<WARP>(team, s, place);
  if (s[1] == 0.f) return Centre{1.f, {first, 0.f, 0.f}, first - first};
  Centre to = {factor, {s[0] * P.inv_d, 0.f, 0.f}, 0.f};
#pragma unroll 1
  for (int again = 1; again < 3; ++again) {
    s[0] = s[1] = 0.f;
    each([&](float x) {
      const float c = fmaf(x, factor, -to.mean[0]) - to.mean[1];
      s[0] += c;
      s[1] = fmaf(c, c, s[1]);
    });
    team_sum<WARP>(team, s, place + 2 * again);
    const float left = s[0] * P.inv_d;
    (again == 1 ? to.mean[1] : to.mean[2]) = left;
    to.squares = fmaf(-left, s[0], s[1]);
  }
  return to;
}
// The same, and the row's values minus all of these.
template <class R, class T, int CH, int AT_ONCE, bool WARP, int PLACE>
__device__ __forceinline__ Centre centre_again(typename R::V& v, float squares, const char* row, const NormParams& P, const Team& team, const typename R::M& mine,
                                               float (*place)[BLOCK_WARPS][PLACE]) {
  const Centre to = centre_again<T, CH, AT_ONCE, WARP>(row, squares < MOST ? 1.f : DOWN, P, team, place);
  R::load(v, row, mine);
  R::times(v, to.factor);
#pragma unroll
  for (int i = 0; i < 3; ++i) R::centre(v, to.mean[i], mine);
  return to;
}

// Forward: the teams of blocks s * parts .. (s + 1) * parts - 1 take the rows of segment s in turns.
template <class T, int CH, int PER, bool FULL, bool WARP, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == BLOCK_WARPS * 32 ? FORWARD_WARPS<CH, PER> / BLOCK_WARPS : 1) norm_forward_kernel(const __grid_constant__ NormParams P) {
  using R = Row<T, CH, PER, FULL>;
  constexpr int N = R::N;
  __shared__ __align__(16) Place<THREADS / 32> place[8];
  extern __shared__ __align__(16) unsigned char shared[];
  const Team team = team_of<WARP>(P);
  const typename R::M mine(team, P.pieces);
  const unsigned segment = blockIdx.x / P.parts, part = blockIdx.x - segment * P.parts;
  const unsigned stride = P.parts * team.teams;
  unsigned at = part * team.teams + team.index;
  clear<WARP>(place);
  ff_pdl_wait();
  Ring<T, CH, PER, FULL, 1> ring(shared);
  unsigned asked = at;
  Way from(P.x, P, segment, at, stride), to(P.y, P, segment, at, stride);
  auto ask = [&](int stage) {
    ring.ask(stage, 0, from.p, asked < P.segment, mine);
    ring.asked();
    asked += stride;
    if (asked < P.segment) from.to(P.x, P, asked);
  };
#pragma unroll
  for (int i = 0; i < (ring.SHARED ? STAGES<T> - 1 : 1); ++i) ask(i);
  typename R::V w, b;
  R::weights(w, P.w ? P.w + segment * P.w_stride : nullptr, P.plus, 1.f, mine);
  R::weights(b, P.bias ? P.bias + segment * P.w_stride : nullptr, 0.f, 0.f, mine);
#pragma unroll 1
  while (at < P.segment) {
    typename R::V v;
    ring.arrived();
    ring.take(0, v);
    float s[1] = {R::sum(v)};
    ask((ring.next() + STAGES<T> - 1) % STAGES<T>);
    team_sum<WARP>(team, s, place);
    const float mean = s[0] * P.inv_d, least = mean * mean * P.least;
    R::centre(v, mean, mine);
    s[0] = R::dot(v, v);
    team_sum<WARP>(team, s, place + 1);
    float f = 1.f;
    if (__builtin_expect(far_from_centred(s[0], least), 0)) {  // (the same in the whole team)
      const Centre to = centre_again<R, T, CH, 1, WARP>(v, s[0], row_at(P.x, P, segment, at), P, team, mine, place + 2);
      s[0] = to.squares;
      f = to.factor;
    }
    const float r = rsqrtf(fmaf(s[0], P.inv_d, P.eps * f * f));        // (a row that was scaled down: eps is far below its variance)
#pragma unroll
    for (int i = 0; i < R::GROUPS; ++i)
#pragma unroll
      for (int c = 0; c < N; ++c) v[i][c] = fma(mul(v[i][c], two(r, r)), w[i][c], b[i][c]);
    R::store(to.p, v, mine);
    at += stride;
    if (at < P.segment) to.to(P.y, P, at);
  }
}

// Backward: the teams' rows as in the forward pass, one at a time.  The sums of dweight and dbias of a block's teams are joined and go to its
// place among the parts.
template <class T, int CH, int PER, bool FULL, bool WARP, int THREADS>
__global__ void __launch_bounds__(CH == 1 && PER == 8 && !WARP ? EIGHTS_WARPS * 32 : THREADS, 1) norm_backward_kernel(const __grid_constant__ NormParams P) {
  using R = Row<T, CH, PER, FULL>;
  constexpr int N = R::N;
  __shared__ __align__(16) Place<THREADS / 32> place[10];
  extern __shared__ __align__(16) unsigned char shared[];
  float* joined = (float*)shared;                              // at the end: [teams][d]
  const Team team = team_of<WARP>(P);
  const typename R::M mine(team, P.pieces);
  const unsigned segment = blockIdx.x / P.parts, part = blockIdx.x - segment * P.parts;
  const unsigned stride = P.parts * team.teams;
  unsigned at = part * team.teams + team.index;
  clear<WARP>(place);
  ff_pdl_wait();
  Ring<T, CH, PER, FULL, 2> ring(shared);                            // (a row of x, one of dy)
  unsigned asked = at;
  Way x(P.x, P, segment, at, stride), g(P.g, P, segment, at, stride), to(P.y, P, segment, at, stride);
  auto ask = [&](int stage) {
    ring.ask(stage, 0, x.p, asked < P.segment, mine);
    ring.ask(stage, 1, g.p, asked < P.segment, mine);
    ring.asked();
    asked += stride;
    if (asked < P.segment) { x.to(P.x, P, asked); g.to(P.g, P, asked); }
  };
#pragma unroll
  for (int i = 0; i < (ring.SHARED ? STAGES<T> - 1 : 1); ++i) ask(i);
  typename R::V w, dw, db;
  R::weights(w, P.w ? P.w + segment * P.w_stride : nullptr, P.plus, 1.f, mine);
#pragma unroll
  for (int i = 0; i < R::GROUPS; ++i)
#pragma unroll
    for (int c = 0; c < N; ++c) dw[i][c] = db[i][c] = two(0.f, 0.f);
#pragma unroll 1
  while (at < P.segment) {
    typename R::V v, dy;
    ring.arrived();
    ring.take(0, v);
    ring.take(1, dy);
    ask((ring.next() + STAGES<T> - 1) % STAGES<T>);
    float m[1] = {R::sum(v)};
    team_sum<WARP>(team, m, place);
    const float mean = m[0] * P.inv_d, least = mean * mean * P.least;
    R::centre(v, mean, mine);
    // sums of c^2, of g = dy w and of g c
    auto sums = [&](float (&s)[3]) {
      s[0] = R::dot(v, v);
      F2 u = two(0.f, 0.f), t = u;
#pragma unroll
      for (int i = 0; i < R::GROUPS; ++i)
#pragma unroll
        for (int c = 0; c < N; ++c) {
          const F2 gw = mul(dy[i][c], w[i][c]);
          u = __fadd2_rn(u, gw);
          t = fma(gw, v[i][c], t);
        }
      s[1] = low(u) + high(u);
      s[2] = low(t) + high(t);
      team_sum<WARP>(team, s, place + 1);
    };
    float s[3], f = 1.f;
    sums(s);
    if (__builtin_expect(far_from_centred(s[0], least), 0)) {  // (as in the forward pass)
      f = centre_again<R, T, CH, CH == 1 && !WARP ? 4 : 1, WARP>(v, s[0], row_at(P.x, P, segment, at), P, team, mine, place + 4).factor;
      sums(s);
    }
    const float scale = rsqrtf(fmaf(s[0], P.inv_d, P.eps * f * f)), r = scale * f;
    const float mean_g = -s[1] * P.inv_d, mean_gn = -s[2] * scale * P.inv_d;
#pragma unroll
    for (int i = 0; i < R::GROUPS; ++i)
#pragma unroll
      for (int c = 0; c < N; ++c) {
        const F2 n = mul(v[i][c], two(scale, scale));
        dw[i][c] = fma(dy[i][c], n, dw[i][c]);
        db[i][c] = __fadd2_rn(db[i][c], dy[i][c]);
        dy[i][c] = mul(fma(n, two(mean_gn, mean_gn), fma(dy[i][c], w[i][c], two(mean_g, mean_g))), two(r, r));
      }
    if (P.y.p) R::store(to.p, dy, mine);
    at += stride;
    if (at < P.segment) to.to(P.y, P, at);
  }
  if constexpr (ring.SHARED) copy_wait<0>();
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* out = which ? P.db : P.dw;
    if (!out) continue;
    out += blockIdx.x * P.part_stride;
    const typename R::V& v = which ? db : dw;
    __syncthreads();                                           // (the other one has been read)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (mine.have(i))
#pragma unroll
        for (int c = 0; c < CH; ++c) joined[team.index * P.d + mine.at[i] + c] = R::value(v, i, c);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < P.d; c += blockDim.x) {
      float s = 0.f;
      for (int k = 0; k < team.teams; ++k) s += joined[k * P.d + c];
      out[c] = s;
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
// Do the rows of a batch follow one another at one distance?  (With one token a sample at that of the samples, which is then the tokens'.)
bool even(RowsView* v, int64_t batch, int64_t tokens) {
  if (tokens == 1) v->st = v->sb;
  return batch == 1 || tokens == 1 || v->sb == tokens * v->st;
}

// Values of a piece that dim and the tensors' alignment allow.
int piece_of(int d, int e, uint64_t bits) {
  for (int ch = 16 / e; ch > 1; ch = ch == 8 ? 2 : ch >> 1)
    if (d % ch == 0 && bits % ((uint64_t)ch * e) == 0 && (ch == 16 / e || e == 2)) return ch;
  return 1;
}
// A block: teams of as many warps as a row takes, BLOCK_WARPS warps in all unless a team has more, or there are few rows: then every SM
// gets some of them (8 rows of 2048: 4.6 us in two blocks, 2.9 in eight).
struct Block { int team_warps, teams, threads; };
Block block_of(int pieces, int per, long long rows) {
  Block b;
  b.team_warps = (pieces + per * 32 - 1) / (per * 32);
  b.teams = b.team_warps < BLOCK_WARPS ? BLOCK_WARPS / b.team_warps : 1;
  const long long fair = (rows + FF_B200_SMS - 1) / FF_B200_SMS;
  if (b.teams > fair) b.teams = (int)(fair < 1 ? 1 : fair);
  b.threads = b.teams * b.team_warps * 32;
  return b;
}
// The rows whose gradients are summed together (the model's, or each sample's) and the blocks they are divided between: one wave of
// them, and at most one for every `each` rows.
struct Parts { unsigned segments, rows, parts; };
Parts parts_of(int64_t batch, int64_t tokens, int per_sample, int blocks, long long each) {
  Parts p;
  p.segments = per_sample ? (unsigned)batch : 1;
  p.rows = (unsigned)(per_sample ? tokens : batch * tokens);
  const long long most = ((long long)p.rows + each - 1) / each, wave = (long long)FF_B200_SMS * blocks / (p.segments ? p.segments : 1);
  p.parts = (unsigned)(wave < most ? wave : most);
  if (p.parts < 1) p.parts = 1;
  return p;
}

// More than the default limit of shared memory, with every call that needs it (a handle serves any device), and always as much as the longest
// row takes, so that calls of several threads do not lower each other's.
constexpr int MOST_SMEM = STAGES<float> * 2 * MAX_DIM * (int)sizeof(float);
cudaError_t allow(void (*kernel)(NormParams), size_t smem) {
  return smem <= 40 * 1024 ? cudaSuccess : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST_SMEM);
}

template <class T, int CH, int PER, bool WARP, int THREADS>
cudaError_t forward(NormParams& P, int64_t batch, int64_t tokens, int per_sample, cudaStream_t st) {
  const Block b = block_of(P.pieces, PER, P.rows);
  const Parts p = parts_of(batch, tokens, per_sample, FORWARD_WARPS<CH, PER> * 32 / b.threads, b.teams);
  P.segment = p.rows; P.parts = p.parts; P.team_warps = b.team_warps;
  const size_t smem = ring_bytes<T, CH, PER, 1>(b.threads);
  const bool full = P.pieces == PER * 32 * b.team_warps;
  const auto kernel = full && CH > 1 ? norm_forward_kernel<T, CH, PER, (CH > 1), WARP, THREADS> : norm_forward_kernel<T, CH, PER, false, WARP, THREADS>;
  const cudaError_t e = allow(kernel, smem);
  return e != cudaSuccess ? e : ff_launch(kernel, dim3(p.segments * p.parts), dim3(b.threads), smem, st, P);
}
template <class T, int CH, int PER, bool WARP, int THREADS>
cudaError_t backward(NormParams& P, unsigned blocks, cudaStream_t st) {
  const Block b = block_of(P.pieces, PER, P.rows);
  P.team_warps = b.team_warps;
  const size_t ring = ring_bytes<T, CH, PER, 2>(b.threads), joined = (size_t)b.teams * P.d * sizeof(float), smem = ring > joined ? ring : joined;
  const bool full = P.pieces == PER * 32 * b.team_warps;
  const auto kernel = full && CH > 1 ? norm_backward_kernel<T, CH, PER, (CH > 1), WARP, THREADS> : norm_backward_kernel<T, CH, PER, false, WARP, THREADS>;
  const cudaError_t e = allow(kernel, smem);
  return e != cudaSuccess ? e : ff_launch(kernel, dim3(blocks), dim3(b.threads), smem, st, P);
}
// The team and the pieces of a thread: a warp where it has room for the row, with as few pieces a thread as do, else several warps.  (Rows above 4096
// values that come one by one, 16 of a thread: 512 threads leave it 128 registers, and backward 300 bytes go to memory with bf16, whose next
// row waits in registers, 60 with fp32: 8000 x 4101 334 and 143 us.)
template <class T, int CH, bool FORWARD, class Run>
cudaError_t with_team(int pieces, Run run) {
  using std::integral_constant;
  constexpr int MOST = CH == 1 || (CH == 2 && FORWARD) ? 8 : VALUES / CH;
  using True = integral_constant<bool, true>;
  using False = integral_constant<bool, false>;
  using Small = integral_constant<int, BLOCK_WARPS * 32>;
  using Large = integral_constant<int, MOST == 8 && CH <= 2 ? MAX_THREADS : MAX_DIM / VALUES>;
  if constexpr (MOST >= 4) if (pieces <= 32 * (MOST / 4)) return run(integral_constant<int, MOST / 4>(), True(), Small());
  if (pieces <= 32 * (MOST / 2)) return run(integral_constant<int, MOST / 2>(), True(), Small());
  if (pieces <= 32 * MOST) return run(integral_constant<int, MOST>(), True(), Small());
  if (pieces <= 32 * BLOCK_WARPS * MOST) return run(integral_constant<int, MOST>(), False(), Small());
  if constexpr (CH == 1 && MOST < 16) if (pieces > MAX_THREADS * MOST) return run(integral_constant<int, 16>(), False(), Large());
  return run(integral_constant<int, MOST>(), False(), Large());
}
template <class Run>
cudaError_t with_piece(int e, int ch, Run run) {
  if (e == 4) return ch == 4 ? run(float(), std::integral_constant<int, 4>()) : run(float(), std::integral_constant<int, 1>());
  return ch == 8 ? run(__nv_bfloat16(), std::integral_constant<int, 8>())
                 : ch == 2 ? run(__nv_bfloat16(), std::integral_constant<int, 2>()) : run(__nv_bfloat16(), std::integral_constant<int, 1>());
}

// Backward: the same blocks whatever the tensors' alignment, so that the workspace does not depend on it.  Kernels of rows of up to 256 values have
// 100 to 130 registers, and two blocks on an SM: 30000 x 128 bf16 13.9 us instead of 16.4.  Longer ones that come one by one, 8 of a thread, are held to
// 128, so that 16 warps fit, and get as many blocks: 9999 x 1155 bf16 36.5 us instead of 73 with one block of a team of five.  (With room for a block
// more than there are, blocks come three to an SM and two to another: 9999 x 1155 fp32 53 us with ten warps instead of 41.)
Parts backward_parts(const ff_layer_norm_config_t& c, int64_t batch, int64_t tokens, int per_sample) {
  const bool single = c.dim % (c.dtype == FF_FP32 ? 4 : 2) != 0, light = c.dim <= 256;
  const bool eights = single && !light && c.dim <= 8 * 32 * BLOCK_WARPS;
  const Block b = block_of(c.dim, eights ? 8 : VALUES, batch * tokens);
  const int blocks = light ? 2 : eights ? EIGHTS_WARPS * 32 / b.threads : 1;
  return parts_of(batch, tokens, per_sample, blocks > 1 ? blocks : 1, b.teams);
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
  P.least = (float)P.d / 256.f;
  P.eps = h->cfg.eps;
  P.even = 1;                                // (each sample's rows are)
  return P;
}

// Does an output lie over an input in other places than the input's own rows?
bool misplaced(const ff_rows_t* y, const ff_rows_t* x, int64_t batch, int64_t tokens) {
  return y->data == x->data && ((batch > 1 && y->stride_batch != x->stride_batch) || (tokens > 1 && y->stride_token != x->stride_token));
}

}  // namespace

extern "C" ff_status_t ff_layer_norm_create(const ff_layer_norm_config_t* cfg, ff_layer_norm_t** out) {
  if (!cfg || !out) return fail(nullptr, FF_ERR_INVALID_ARG, "cfg or out is NULL");
  *out = nullptr;
  if (cfg->dtype != FF_BF16 && cfg->dtype != FF_FP32) return fail(nullptr, FF_ERR_INVALID_ARG, "dtype must be FF_BF16 or FF_FP32");
  if (cfg->dim < 1) return fail(nullptr, FF_ERR_INVALID_ARG, "dim must be positive");
  if (cfg->dim > MAX_DIM) return fail(nullptr, FF_ERR_UNSUPPORTED, "dim must be at most 8192");
  // (below FLT_MIN eps, and the squares that it is added to, have lost digits)
  if (!(cfg->eps >= FLT_MIN && cfg->eps < 3.0e38f)) return fail(nullptr, FF_ERR_INVALID_ARG, "eps must be at least 2^-126, and finite");
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
  if (misplaced(y, x, batch, tokens)) return fail(h, FF_ERR_INVALID_ARG, "y lies over x with other strides");
  const int ch = piece_of(h->cfg.dim, e, bits);
  NormParams P = common(h, batch, tokens, weight, per_sample, ch);
  P.x = view(x, e); P.y = view(y, e);
  if (!per_sample) P.even = even(&P.x, batch, tokens) & even(&P.y, batch, tokens);
  P.bias = bias;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t err = with_piece(e, ch, [&](auto t, auto piece) {
    using T = decltype(t);
    constexpr int CH = decltype(piece)::value;
    return with_team<T, CH, true>(P.pieces, [&](auto per, auto warp, auto threads) {
      return forward<T, CH, decltype(per)::value, decltype(warp)::value, decltype(threads)::value>(P, batch, tokens, per_sample, st);
    });
  });
  return err == cudaSuccess ? FF_OK : cuda_fail(h, err);
}

extern "C" ff_status_t ff_layer_norm_workspace_bytes(const ff_layer_norm_t* handle, int64_t batch, int64_t tokens, int32_t per_sample, size_t* bytes) {
  ff_layer_norm* h = const_cast<ff_layer_norm*>(handle);
  if (!h || !bytes) return fail(h, FF_ERR_INVALID_ARG, "handle or bytes is NULL");
  const ff_status_t s = check_call(h, batch, tokens, {});
  if (s != FF_OK) return s;
  const Parts p = backward_parts(h->cfg, batch, tokens, per_sample);
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
  if (dx && (misplaced(dx, x, batch, tokens) || misplaced(dx, dy, batch, tokens)))
    return fail(h, FF_ERR_INVALID_ARG, "dx lies over x or dy with other strides");
  size_t need = 0;
  ff_layer_norm_workspace_bytes(handle, batch, tokens, per_sample, &need);
  if (need && (!ws || ws_bytes < need)) return fail(h, FF_ERR_WORKSPACE, "the workspace is missing or smaller than ff_layer_norm_workspace_bytes");
  if (need && (((uintptr_t)ws) & 15)) return fail(h, FF_ERR_WORKSPACE, "the workspace must be 16-byte aligned");
  if ((dweight && (dweight == dbias || dweight == weight)) || (dbias && dbias == weight))
    return fail(h, FF_ERR_INVALID_ARG, "a gradient lies over another one or over the weight");
  if (!dx && !dweight && !dbias) return FF_OK;
  const int ch = piece_of(d, e, bits);
  const Parts parts = backward_parts(h->cfg, batch, tokens, per_sample);
  NormParams P = common(h, batch, tokens, weight, per_sample, ch);
  P.x = view(x, e); P.g = view(dy, e);
  if (dx) P.y = view(dx, e);
  if (!per_sample) P.even = even(&P.x, batch, tokens) & even(&P.g, batch, tokens) & (!dx || even(&P.y, batch, tokens));
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
  cudaError_t err = with_piece(e, ch, [&](auto t, auto piece) {
    using T = decltype(t);
    constexpr int CH = decltype(piece)::value;
    return with_team<T, CH, false>(P.pieces, [&](auto per, auto warp, auto threads) {
      return backward<T, CH, decltype(per)::value, decltype(warp)::value, decltype(threads)::value>(P, blocks, st);
    });
  });
  if (err == cudaSuccess && parts.parts > 1 && (dweight || dbias)) {
    const int columns = (d + 31) / 32;
    err = ff_launch(norm_join_kernel, dim3(parts.segments * columns, 2), dim3(1024), 0, st, (const float*)ws, (int)parts.parts, d, columns, dweight, dbias);
  }
  return err == cudaSuccess ? FF_OK : cuda_fail(h, err);
}
