// Queries and keys between the projections and the attention: rotary positions, and the norm of every head row with the
// rotation in the same pass, forward and backward.
//
//   rotation   (a, b) of pair p -> m (a cos t - b sin t, a sin t + b cos t),   t = position * theta_p
//   norm       z = x r w,  r = 1 / sqrt(mean(x^2) + eps) over the row's head_dim channels,  y = rotation of z
//   backward   dz = the rotation's transpose of dy;  n = x r;  g = dz w;  dx = r (g - n mean(g n));  dw = sum over rows of dz n
//
// All of it is one pass over the rows: a row of head_dim channels is read once, stays in registers in fp32 and is written
// once, so the bound is memory: 2 (backward 3) tensors.  What could exceed that are the angles, one sine and cosine per
// token and pair; they do not depend on the head, so a thread that owns the same pairs of one token computes them once and
// keeps them in registers while it walks over the heads.
//
// Angles: theta_p / 2 pi is kept as a 64-bit fraction of a turn, cut off.  position * fraction modulo 2^64 is then the angle modulo a
// whole turn, less than 2^-33 turns off for any 32-bit position, and its high word, cut off again, less than 1.5 x 2^-32.  The word gives
// the quadrant and a remainder of at most an eighth of a turn (as a float another 2^-28 turns off at most), whose sine and cosine are
// short Taylor polynomials (two values an instruction: the pair of them), and no floating-point product of a far position ever has to be
// reduced.
//
// Threads: a row is cut in chunks of CH channels (16 bytes where strides, rot_dim and head_dim allow, else 8, 4 or 2), and a
// thread owns two chunks of it so that both channels of a pair are its own: no exchange between threads for the rotation.
//   half layout          chunk j of the first half of the turned channels and chunk j of the second; the channels that are not
//                        turned follow in the same manner, so that neighbouring lanes have neighbouring chunks (two chunks of
//                        a lane side by side, every lane half a sector: 11000 tokens, 12 + 4 fp32 heads of 80, 28 us instead of 25)
//   interleaved layout   chunk j of the first half of the row and chunk j of the second: pairs lie inside a chunk
// A row takes L = 2^k lanes (8 for 128 bf16 channels), a warp 32 / L tokens at a time.
#include <math.h>
#include <stdio.h>

#include <new>

#include "ff_chunks.cuh"
#include "ff_internal.h"

struct ff_rotary {
  ff_rotary_config_t cfg;
  int pairs;                       // rot_dim / 2
  int axis_end[2];                 // pairs below the first turn with axis t, below the second with h, then w
  int axes;                        // position components of a token: 1 or 3
  double theta[128];               // radians per position
  unsigned long long phase[128];   // the same as a 64-bit fraction of a turn
  float magnitude;
  char err[512];
};

namespace {

enum { ROTATE = 0, NORM = 1, NORM_BACKWARD = 2 };
constexpr int H_THREADS = 256, H_WARPS = H_THREADS / 32;
constexpr int FORWARD_WAVES = 8;                  // waves of blocks that a large forward launch is cut in
constexpr int FORWARD_BLOCKS = 2;                 // blocks of a forward launch on an SM
constexpr int PARTIAL_ROWS = 2 * FF_B200_SMS;     // rows of partial weight gradients at most: one wave of two blocks per SM

struct HeadsView { char* p; long long sb, sh, st; };   // strides in bytes

struct HeadsParams {
  HeadsView x[2], y[2], g[2];      // q and k: input, output, (backward) the gradient of the forward pass's output
  const float* w[2];               // norm weights or NULL
  float* partial;                  // backward: [blocks of q, then of k][head_dim]
  const int* positions;
  long long pos_stride;            // elements between the samples' positions
  int rows;                        // batch * tokens
  FFFastDiv tokens, gw, gh;        // tokens per sample; the grid's W and H
  int heads[2], groups;            // heads of q and k; groups of tokens
  int nblocks0;                    // backward: blocks that belong to q
  int d, rot, np, lanes_log2;      // channels, turned channels, chunk pairs of a row, log2 of the lanes of a row
  int axis_end0, axis_end1, axes;
  int inverse;
  float magnitude, eps;
  unsigned long long phase[128];
};

// What turns two chunks a, b of a row.  Half layout: a' = a p + b q, b' = a r + b t;  interleaved: every pair (x, y) of a goes to
// (x, x) p + (y, y) q, those of b to (x, x) r + (y, y) t.  Chunks that are not turned are left alone: what stands beside them does not
// touch them, infinite or not.
template <int CH> struct Turn { F2 p[pairs_of(CH)], q[pairs_of(CH)], r[pairs_of(CH)], t[pairs_of(CH)]; };

template <int CH, bool INTER>
__device__ __forceinline__ void turn(F2 (&a)[pairs_of(CH)], F2 (&b)[pairs_of(CH)], const Turn<CH>& k, bool turned_a, bool turned_b) {
  constexpr int N = pairs_of(CH);
  if constexpr (INTER) {
    if (turned_a) {
#pragma unroll
      for (int i = 0; i < N; ++i) a[i] = fma(two(low(a[i]), low(a[i])), k.p[i], mul(two(high(a[i]), high(a[i])), k.q[i]));
    }
    if (turned_b) {
#pragma unroll
      for (int i = 0; i < N; ++i) b[i] = fma(two(low(b[i]), low(b[i])), k.r[i], mul(two(high(b[i]), high(b[i])), k.t[i]));
    }
  } else if (turned_a) {            // (both chunks of a half-layout pair are turned or neither is)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const F2 x = a[i];
      a[i] = fma(x, k.p[i], mul(b[i], k.q[i]));
      b[i] = fma(x, k.r[i], mul(b[i], k.t[i]));
    }
  }
}

template <int N, int PER>
__device__ __forceinline__ float dot(const F2 (&x)[PER][N], const F2 (&y)[PER][N], const F2 (&u)[PER][N], const F2 (&v)[PER][N]) {
  F2 s = two(0.f, 0.f), t = s;
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int c = 0; c < N; ++c) { s = fma(x[i][c], y[i][c], s); t = fma(u[i][c], v[i][c], t); }
  return (low(s) + high(s)) + (low(t) + high(t));
}
__device__ __forceinline__ float row_sum(float v, int lanes) {
  for (int m = 1; m < lanes; m <<= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}
// 1 / sqrt(mean of squares + eps) of a row whose values the lanes of a group hold.  Rows whose squares leave fp32 are summed
// again scaled by 2^-70, and eps by its square (an eps that vanishes by that is far below their mean).
template <int N, int PER>
__device__ __forceinline__ float row_rms(const F2 (&a)[PER][N], const F2 (&b)[PER][N], int lanes, float inv_d, float eps) {
  const float ss = row_sum(dot<N, PER>(a, a, b, b), lanes);
  const bool big = !(ss < 3.0e38f);
  if (!__any_sync(0xffffffffu, big)) return rsqrtf(ss * inv_d + eps);
  const float down = 8.4703294725430034e-22f;   // 2^-70
  F2 sa[PER][N], sb[PER][N];
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int c = 0; c < N; ++c) { sa[i][c] = mul(a[i][c], two(down, down)); sb[i][c] = mul(b[i][c], two(down, down)); }
  const float sc = row_sum(dot<N, PER>(sa, sa, sb, sb), lanes);
  return big ? rsqrtf(fmaf(sc, inv_d, eps * down * down)) * down : rsqrtf(ss * inv_d + eps);
}

// The chunks that lane `lig` of a row has: channels, whether there are any, whether they are turned.
template <int CH, int PER, bool INTER>
struct Own {
  int oa[PER], ob[PER];
  bool have[PER], ta[PER], tb[PER];
  __device__ __forceinline__ Own(const HeadsParams& P, int lig, int lanes) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int j = lig + i * lanes;
      have[i] = j < P.np;
      if (INTER) {
        oa[i] = j * CH; ob[i] = (j + P.np) * CH;
        ta[i] = have[i] && oa[i] < P.rot; tb[i] = have[i] && ob[i] < P.rot;
      } else {
        const int turned = P.rot / (2 * CH);
        ta[i] = tb[i] = have[i] && j < turned;
        oa[i] = j < turned ? j * CH : P.rot + (j - turned) * CH;
        ob[i] = j < turned ? P.rot / 2 + j * CH : oa[i] + (P.d - P.rot) / 2;
      }
    }
  }
  // Two neighbouring weights of a chunk, or ones.
  __device__ __forceinline__ F2 weights(const float* w, int i, int at, int c) const {
    if (!w || !have[i]) return two(1.f, 1.f);
    return two(w[at + 2 * c], CH > 1 ? w[at + 2 * c + 1] : 1.f);
  }
};

// Sine and cosine of an angle in 2^-32 turns.  |x| <= pi / 4: the first terms left out are x^11 / 11! < 2e-9 and x^12 / 12! < 2e-10.
__device__ __forceinline__ void sine_and_cosine(unsigned turns, float& sine, float& cosine) {
  const unsigned quadrant = (turns + 0x20000000u) >> 30;
  const float x = (float)(int)(turns - (quadrant << 30)) * 1.4629180792671596e-9f;          // 2 pi / 2^32
  const F2 x2 = two(x * x, x * x);
  F2 v = two(2.7557319224e-6f, fmaf(x * x, -2.7557319224e-7f, 2.4801587302e-5f));             // sin(x) / x: 1/9!;  cos(x): 1/8!, -1/10!
  v = fma(x2, v, two(-1.9841269841e-4f, -1.3888888889e-3f));
  v = fma(x2, v, two(8.3333333333e-3f, 4.1666666667e-2f));
  v = fma(x2, v, two(-1.6666666667e-1f, -0.5f));
  v = fma(x2, v, two(1.f, 1.f));
  const float s = x * low(v), c = high(v);
  sine = __uint_as_float(__float_as_uint(quadrant & 1 ? c : s) ^ ((quadrant & 2) << 30));
  cosine = __uint_as_float(__float_as_uint(quadrant & 1 ? s : c) ^ (((quadrant + 1) & 2) << 30));
}

// The rotation of token n of sample b for a lane's chunks.
template <int CH, int PER, bool INTER>
__device__ __forceinline__ void turn_of_token(const HeadsParams& P, const Own<CH, PER, INTER>& own, unsigned b, unsigned n, Turn<CH> (&k)[PER]) {
  int pos[3];
  if (P.positions) {
    const int* at = P.positions + b * P.pos_stride + (long long)n * P.axes;
    pos[0] = at[0];
    pos[1] = P.axes == 3 ? at[1] : 0;
    pos[2] = P.axes == 3 ? at[2] : 0;
  } else if (P.axes == 3) {
    const unsigned line = ff_div(n, P.gw), plane = ff_div(line, P.gh);
    pos[0] = (int)plane; pos[1] = (int)(line - plane * P.gh.d); pos[2] = (int)(n - line * P.gw.d);
  } else {
    pos[0] = (int)n; pos[1] = pos[2] = 0;
  }
  auto angle = [&](int p, float& c, float& s) {               // times the magnitude
    const int at = p < P.axis_end0 ? pos[0] : (p < P.axis_end1 ? pos[1] : pos[2]);
    sine_and_cosine((unsigned)(((unsigned long long)(long long)at * P.phase[p]) >> 32), s, c);
    c *= P.magnitude;
    s *= P.inverse ? -P.magnitude : P.magnitude;
  };
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int c = 0; c < pairs_of(CH); ++c) {
      k[i].p[c] = k[i].q[c] = k[i].r[c] = k[i].t[c] = two(0.f, 0.f);
      float c0, s0, c1 = 0.f, s1 = 0.f;
      if constexpr (INTER) {
        if (own.ta[i]) {
          angle(own.oa[i] / 2 + c, c0, s0);
          k[i].p[c] = two(c0, s0); k[i].q[c] = two(-s0, c0);
        }
        if (own.tb[i]) {
          angle(own.ob[i] / 2 + c, c1, s1);
          k[i].r[c] = two(c1, s1); k[i].t[c] = two(-s1, c1);
        }
      } else if (own.ta[i]) {
        angle(own.oa[i] + 2 * c, c0, s0);
        if (CH > 1) angle(own.oa[i] + 2 * c + 1, c1, s1);
        k[i].p[c] = k[i].t[c] = two(c0, c1);
        k[i].q[c] = two(-s0, -s1); k[i].r[c] = two(s0, s1);
      }
    }
}

// The positions of a token that will be turned soon, on their way into L1.
__device__ __forceinline__ void prefetch_position(const HeadsParams& P, unsigned b, unsigned n) {
  if (P.positions) asm volatile("prefetch.global.L1 [%0];" ::"l"(P.positions + b * P.pos_stride + (long long)n * P.axes) : "memory");
}

// The lane's token of a group; false: behind the last row (it then reads that one once more and writes nothing).
__device__ __forceinline__ bool token_of(const HeadsParams& P, int group, int warp, int lane, unsigned& b, unsigned& n) {
  const long long row = ((long long)group * H_WARPS + warp) * (32 >> P.lanes_log2) + (lane >> P.lanes_log2);
  const unsigned r = (unsigned)min(row, (long long)P.rows - 1);
  b = ff_div(r, P.tokens); n = r - b * P.tokens.d;
  return row < P.rows;
}

// A block's way through the units (group of 8 x 32 / lanes tokens, head or two): a run of them, those of a group following one another, all
// blocks' runs equally long.  (Whole groups in turns over all blocks and shares of what is left measured no better.)
struct Walk {
  int group, head, heads, count;
  __device__ __forceinline__ Walk(int groups, int heads_, int blocks, int block) : heads(heads_) {
    const long long units = (long long)groups * heads, first = units * block / blocks;
    count = (int)(units * (block + 1) / blocks - first);
    group = (int)(first / heads); head = (int)(first - (long long)group * heads);
  }
  __device__ __forceinline__ bool next() {                    // to the next unit; true: another group
    if (++head < heads) return false;
    head = 0; ++group;
    return true;
  }
};

// Forward.  A unit is two heads of q, or of k behind them: the rotation of a thread's pairs of one token stays in
// its registers for all heads.  The rows on their way wait in shared memory, each thread's pieces in places of its own, two units ahead,
// from one group into the next.  (Rows of two-byte pieces, which cannot be copied that way, are loaded when they are needed.)
// Bound by memory: 64K tokens, 16 + 16 heads of 64 turned in 82 us = 6.5 TB/s, 24 + 24 heads of 128 normed in 258 = 6.2 TB/s.  (Loaded
// into registers, four heads at a time, by blocks of 32 tokens and up to 24 heads: 87 and 262, but 16.7 us instead of 6.6 for 6855 tokens of
// 4 + 2 heads of 128, where such blocks are few or each compute the angles again.)
template <class T, int CH, int PER, bool INTER, int MODE>
__global__ void __launch_bounds__(H_THREADS, FORWARD_BLOCKS) heads_kernel(const __grid_constant__ HeadsParams P) {
  constexpr int N = pairs_of(CH), U = 2;
  using C = Chunk<T, CH>;
  constexpr bool RING = sizeof(C) >= 4;
  constexpr int STAGES = RING ? 3 : 1;
  __shared__ __align__(16) C ring_store[STAGES * U * 2 * PER * H_THREADS];       // [stage][head][a, b][piece][thread]
  C* ring = ring_store + threadIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lanes = 1 << P.lanes_log2;
  const int in_q = (P.heads[0] + U - 1) / U, in_k = (P.heads[1] + U - 1) / U;
  const float inv_d = 1.f / (float)P.d;
  const Own<CH, PER, INTER> own(P, lane & (lanes - 1), lanes);
  ff_pdl_wait();

  Walk now(P.groups, in_q + in_k, gridDim.x, blockIdx.x), ahead = now;           // what is computed, what is requested next
  const int count = now.count;
  int asked = 0;
  unsigned nb, nn;
  const char* xp;
  auto go_to = [&](bool other) {                              // to the rows of `ahead`, of another group or not
    if (other) { token_of(P, ahead.group, warp, lane, nb, nn); prefetch_position(P, nb, nn); }
    const int t = ahead.head >= in_q;
    xp = P.x[t].p + nb * P.x[t].sb + nn * P.x[t].st + (long long)(ahead.head - (t ? in_q : 0)) * U * P.x[t].sh;
  };
  go_to(true);
  auto advance = [&] {
    const bool other = ahead.next();
    if (other || ahead.head == in_q) go_to(other);
    else xp += U * P.x[ahead.head > in_q].sh;
  };
  auto heads_of = [&](const Walk& w) {                        // of the unit's heads, those there are
    const int t = w.head >= in_q;
    return min(U, P.heads[t] - (w.head - (t ? in_q : 0)) * U);
  };
  auto ask = [&](int stage) {
    if (asked < count) {
      C* to = ring + stage * U * 2 * PER * H_THREADS;
      const int there = heads_of(ahead);
      const long long sh = P.x[ahead.head >= in_q].sh;
#pragma unroll
      for (int h = 0; h < U; ++h)
        if (h < there)
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            copy_async<sizeof(C)>(to + (h * 2 * PER + i) * H_THREADS, xp + h * sh + own.oa[i] * sizeof(T), own.have[i]);
            copy_async<sizeof(C)>(to + (h * 2 * PER + PER + i) * H_THREADS, xp + h * sh + own.ob[i] * sizeof(T), own.have[i]);
          }
      if (++asked < count) advance();
    }
    copy_commit();
  };
  if constexpr (RING) {
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) ask(s);
  }

  int stage = 0;
  bool live = false, other = true;
  Turn<CH> k[PER];
  F2 wa[PER][N], wb[PER][N];
  char* yp = nullptr;
  unsigned b, n;
#pragma unroll 1
  for (int u = 0; u < count; ++u) {
    const int t = now.head >= in_q, there = heads_of(now);
    if (other) {                                              // another group: its tokens' rotation
      live = token_of(P, now.group, warp, lane, b, n);
      turn_of_token<CH, PER, INTER>(P, own, b, n, k);
    }
    if (other || now.head == in_q) {
      yp = P.y[t].p + b * P.y[t].sb + n * P.y[t].st + (long long)(now.head - (t ? in_q : 0)) * U * P.y[t].sh;
      if constexpr (MODE == NORM) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
          for (int c = 0; c < N; ++c) { wa[i][c] = own.weights(P.w[t], i, own.oa[i], c); wb[i][c] = own.weights(P.w[t], i, own.ob[i], c); }
      }
    }
    C xa[U][PER], xb[U][PER];
    if constexpr (RING) {
      ask(stage == 0 ? STAGES - 1 : stage - 1);               // (the stage read last)
      copy_wait<STAGES - 1>();
      const C* from = ring + stage * U * 2 * PER * H_THREADS;
#pragma unroll
      for (int h = 0; h < U; ++h)
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          xa[h][i] = from[(h * 2 * PER + i) * H_THREADS];
          xb[h][i] = from[(h * 2 * PER + PER + i) * H_THREADS];
        }
      if (++stage == STAGES) stage = 0;
    } else {
#pragma unroll
      for (int h = 0; h < U; ++h)
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const char* from = xp + h * P.x[t].sh;
          xa[h][i] = own.have[i] && h < there ? *(const C*)(from + own.oa[i] * sizeof(T)) : C{};
          xb[h][i] = own.have[i] && h < there ? *(const C*)(from + own.ob[i] * sizeof(T)) : C{};
        }
      if (u + 1 < count) advance();
    }
#pragma unroll
    for (int h = 0; h < U; ++h) {
      if (h && h >= there) break;                             // (the whole block)
      F2 a[PER][N], c[PER][N];                                // the two chunks
#pragma unroll
      for (int i = 0; i < PER; ++i) { unpack<T, CH>(xa[h][i], a[i]); unpack<T, CH>(xb[h][i], c[i]); }
      if constexpr (MODE == NORM) {
        const float r = row_rms<N, PER>(a, c, lanes, inv_d, P.eps);
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
          for (int j = 0; j < N; ++j) { a[i][j] = mul(mul(a[i][j], two(r, r)), wa[i][j]); c[i][j] = mul(mul(c[i][j], two(r, r)), wb[i][j]); }
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) turn<CH, INTER>(a[i], c[i], k[i], own.ta[i], own.tb[i]);
      if (live) {
        char* to = yp + h * P.y[t].sh;
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (own.have[i]) {
            *(C*)(to + own.oa[i] * sizeof(T)) = pack<T, CH>(a[i]);
            *(C*)(to + own.ob[i] * sizeof(T)) = pack<T, CH>(c[i]);
          }
      }
    }
    yp += U * P.y[t].sh;
    other = now.next();
  }
}

// Backward.  One wave of blocks, divided between q and k by their heads.  Weights, their gradients and the rotation fill the registers, so the rows on their way wait
// in shared memory, each thread's pieces in places of its own: two units ahead, from one group into the next.  (Rows of two-byte pieces,
// which cannot be copied that way, are loaded when they are needed.)  Instructions and memory together bound it: 2 x 8191 tokens, 32 + 8 heads
// of 128, 89 us = 5.7 TB/s at 60 % of the issue slots; with the rows of two heads at a time in registers 105.
template <class T, int CH, int PER, bool INTER>
__global__ void __launch_bounds__(H_THREADS, 2) heads_backward_kernel(const __grid_constant__ HeadsParams P) {
  constexpr int N = pairs_of(CH);
  constexpr bool RING = sizeof(T) * CH >= 4;
  constexpr int STAGES = 3;
  using C = Chunk<T, CH>;
  constexpr int RING_BYTES = RING ? STAGES * 4 * PER * H_THREADS * (int)sizeof(C) : 0, SUM_BYTES = H_WARPS * 256 * 4;
  __shared__ __align__(16) unsigned char smem[RING_BYTES > SUM_BYTES ? RING_BYTES : SUM_BYTES];
  C* ring = (C*)smem + threadIdx.x;                           // [stage][x a, x b, g a, g b][piece][thread]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lanes = 1 << P.lanes_log2;
  const int t = blockIdx.x >= (unsigned)P.nblocks0;           // 0: q, 1: k
  const int heads = P.heads[t];
  Walk now(P.groups, heads, t ? (int)gridDim.x - P.nblocks0 : P.nblocks0, (int)blockIdx.x - (t ? P.nblocks0 : 0)), ahead = now;
  const int count = now.count;                                // (`now`: what is computed, `ahead`: what is requested next)
  const float inv_d = 1.f / (float)P.d;
  const Own<CH, PER, INTER> own(P, lane & (lanes - 1), lanes);
  ff_pdl_wait();
  F2 wa[PER][N], wb[PER][N], da[PER][N], db[PER][N];          // weights, the thread's share of dw
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int c = 0; c < N; ++c) {
      wa[i][c] = own.weights(P.w[t], i, own.oa[i], c);
      wb[i][c] = own.weights(P.w[t], i, own.ob[i], c);
      da[i][c] = db[i][c] = two(0.f, 0.f);
    }

  int asked = 0;
  const char *xp, *gp;
  auto go_to = [&] {
    unsigned b, n;
    token_of(P, ahead.group, warp, lane, b, n);
    prefetch_position(P, b, n);
    xp = P.x[t].p + b * P.x[t].sb + n * P.x[t].st + ahead.head * P.x[t].sh;
    gp = P.g[t].p + b * P.g[t].sb + n * P.g[t].st + ahead.head * P.g[t].sh;
  };
  go_to();
  auto advance = [&] {
    if (ahead.next()) go_to();
    else { xp += P.x[t].sh; gp += P.g[t].sh; }
  };
  auto ask = [&](int stage) {
    if (asked < count) {
      C* to = ring + stage * 4 * PER * H_THREADS;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        copy_async<sizeof(C)>(to + (0 * PER + i) * H_THREADS, xp + own.oa[i] * sizeof(T), own.have[i]);
        copy_async<sizeof(C)>(to + (1 * PER + i) * H_THREADS, xp + own.ob[i] * sizeof(T), own.have[i]);
        copy_async<sizeof(C)>(to + (2 * PER + i) * H_THREADS, gp + own.oa[i] * sizeof(T), own.have[i]);
        copy_async<sizeof(C)>(to + (3 * PER + i) * H_THREADS, gp + own.ob[i] * sizeof(T), own.have[i]);
      }
      if (++asked < count) advance();
    }
    copy_commit();
  };
  if constexpr (RING) {
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) ask(s);
  }

  int stage = 0;
  bool other = true, live = false;
  Turn<CH> k[PER];
  char* yp = nullptr;
#pragma unroll 1
  for (int u = 0; u < count; ++u) {
    if (other) {                                              // another group: its tokens' rotation
      unsigned b, n;
      live = token_of(P, now.group, warp, lane, b, n);
      turn_of_token<CH, PER, INTER>(P, own, b, n, k);
      yp = P.y[t].p + b * P.y[t].sb + n * P.y[t].st + now.head * P.y[t].sh;
    }
    F2 a[PER][N], c[PER][N], g0[PER][N], g1[PER][N];
    if constexpr (RING) {
      ask(stage == 0 ? STAGES - 1 : stage - 1);               // (the stage read last)
      copy_wait<STAGES - 1>();
      const C* from = ring + stage * 4 * PER * H_THREADS;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        unpack<T, CH>(from[(0 * PER + i) * H_THREADS], a[i]); unpack<T, CH>(from[(1 * PER + i) * H_THREADS], c[i]);
        unpack<T, CH>(from[(2 * PER + i) * H_THREADS], g0[i]); unpack<T, CH>(from[(3 * PER + i) * H_THREADS], g1[i]);
      }
      if (++stage == STAGES) stage = 0;
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const C none{};
        unpack<T, CH>(own.have[i] ? *(const C*)(xp + own.oa[i] * sizeof(T)) : none, a[i]);
        unpack<T, CH>(own.have[i] ? *(const C*)(xp + own.ob[i] * sizeof(T)) : none, c[i]);
        unpack<T, CH>(own.have[i] ? *(const C*)(gp + own.oa[i] * sizeof(T)) : none, g0[i]);
        unpack<T, CH>(own.have[i] ? *(const C*)(gp + own.ob[i] * sizeof(T)) : none, g1[i]);
      }
    }
    const float r = row_rms<N, PER>(a, c, lanes, inv_d, P.eps);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      turn<CH, INTER>(g0[i], g1[i], k[i], own.ta[i], own.tb[i]);                          // dz
#pragma unroll
      for (int j = 0; j < N; ++j) {
        a[i][j] = mul(a[i][j], two(r, r)); c[i][j] = mul(c[i][j], two(r, r));                    // n
        if (live) { da[i][j] = fma(g0[i][j], a[i][j], da[i][j]); db[i][j] = fma(g1[i][j], c[i][j], db[i][j]); }
        g0[i][j] = mul(g0[i][j], wa[i][j]); g1[i][j] = mul(g1[i][j], wb[i][j]);                  // g
      }
    }
    const float m = -row_sum(dot<N, PER>(g0, a, g1, c), lanes) * inv_d;
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        a[i][j] = mul(fma(a[i][j], two(m, m), g0[i][j]), two(r, r));
        c[i][j] = mul(fma(c[i][j], two(m, m), g1[i][j]), two(r, r));
      }
    if (live) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (own.have[i]) {
          *(C*)(yp + own.oa[i] * sizeof(T)) = pack<T, CH>(a[i]);
          *(C*)(yp + own.ob[i] * sizeof(T)) = pack<T, CH>(c[i]);
        }
    }
    yp += P.y[t].sh;
    other = now.next();
    if constexpr (!RING) { if (u + 1 < count) advance(); }
  }

  // the block's rows of dw: lanes that own the same channels, then the warps, in a fixed order
  if constexpr (RING) { copy_wait<0>(); __syncthreads(); }
  float (*sum)[256] = (float (*)[256])smem;
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float va = c & 1 ? high(da[i][c / 2]) : low(da[i][c / 2]), vb = c & 1 ? high(db[i][c / 2]) : low(db[i][c / 2]);
      for (int m = lanes; m < 32; m <<= 1) {
        va += __shfl_xor_sync(0xffffffffu, va, m);
        vb += __shfl_xor_sync(0xffffffffu, vb, m);
      }
      if (lane < lanes && own.have[i]) { sum[warp][own.oa[i] + c] = va; sum[warp][own.ob[i] + c] = vb; }
    }
  __syncthreads();
  for (int c = threadIdx.x; c < P.d; c += H_THREADS) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < H_WARPS; ++w) s += sum[w][c];
    P.partial[(long long)blockIdx.x * P.d + c] = s;
  }
}

// dw[t][c] = sum of the partial rows of q (t = 0) or k, in a fixed order (no rows: zeros).  One block: 32 columns of one of them.
__global__ void __launch_bounds__(1024) weight_gradient_kernel(const float* partial, int rows_q, int rows_k, int d, float* dwq, float* dwk) {
  __shared__ float sum[32][33];
  ff_pdl_wait();
  const int t = blockIdx.y, c = blockIdx.x * 32 + (threadIdx.x & 31), ty = threadIdx.x >> 5;
  const float* p = partial + (t ? (long long)rows_q * d : 0);
  const int rows = t ? rows_k : rows_q;
  float s = 0.f;
  constexpr int EACH = (PARTIAL_ROWS + 31) / 32;              // (all on their way together)
  float v[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) v[i] = c < d && ty + 32 * i < rows ? p[(long long)(ty + 32 * i) * d + c] : 0.f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) s += v[i];
  sum[ty][threadIdx.x & 31] = s;
  __syncthreads();
  if (ty == 0) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sum[i][threadIdx.x];
    float* out = t ? dwk : dwq;
    if (c < d && out) out[c] = s;
  }
}

ff_status_t fail(ff_rotary* h, ff_status_t code, const char* msg) {
  if (h) snprintf(h->err, sizeof h->err, "%s", msg);
  else ff_set_thread_error(msg);
  return code;
}
ff_status_t cuda_fail(ff_rotary* h, cudaError_t e) {
  char msg[256];
  snprintf(msg, sizeof msg, "CUDA error: %s", cudaGetErrorString(e));
  return fail(h, FF_ERR_CUDA, msg);
}

// What a call's tensors have to fulfil; the greatest common divisor of their strides and addresses decides the chunk.
struct Call {
  ff_rotary* h;
  int64_t batch, tokens;
  int e;                            // bytes of an element
  uint64_t bits;                    // all addresses and strides in bytes, or-ed
};
ff_status_t check_view(Call& c, const ff_heads_t* v, int heads, bool written) {
  if (!v || !v->data) return fail(c.h, FF_ERR_INVALID_ARG, "a tensor is NULL");
  if (v->heads != heads) return fail(c.h, FF_ERR_INVALID_ARG, "tensors of one kind must have the same number of heads");
  if (written && ((c.batch > 1 && v->stride_batch == 0) || (c.tokens > 1 && v->stride_token == 0) || (heads > 1 && v->stride_head == 0)))
    return fail(c.h, FF_ERR_INVALID_ARG, "an output's stride is 0: rows would be written over one another");
  if (v->stride_batch < 0 || v->stride_head < 0 || v->stride_token < 0) return fail(c.h, FF_ERR_INVALID_ARG, "strides must not be negative");
  // (strides that no second element uses do not count)
  c.bits |= (uint64_t)(uintptr_t)v->data;
  if (c.batch > 1) c.bits |= (uint64_t)v->stride_batch * c.e;
  if (c.tokens > 1) c.bits |= (uint64_t)v->stride_token * c.e;
  if (heads > 1) c.bits |= (uint64_t)v->stride_head * c.e;
  if ((uintptr_t)v->data % c.e) return fail(c.h, FF_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  return FF_OK;
}
HeadsView view(const ff_heads_t* v, int e) {
  return HeadsView{(char*)v->data, (long long)v->stride_batch * e, (long long)v->stride_head * e, (long long)v->stride_token * e};
}

template <class T, int CH, int PER, int MODE>
cudaError_t launch_layout(bool inter, dim3 grid, cudaStream_t st, const HeadsParams& P) {
  if constexpr (MODE == NORM_BACKWARD) {
    if constexpr (CH > 1)
      if (inter) return ff_launch(heads_backward_kernel<T, CH, PER, true>, grid, dim3(H_THREADS), 0, st, P);
    return ff_launch(heads_backward_kernel<T, CH, PER, false>, grid, dim3(H_THREADS), 0, st, P);
  } else {
    if constexpr (CH > 1)
      if (inter) return ff_launch(heads_kernel<T, CH, PER, true, MODE>, grid, dim3(H_THREADS), 0, st, P);
    return ff_launch(heads_kernel<T, CH, PER, false, MODE>, grid, dim3(H_THREADS), 0, st, P);
  }
}
template <class T, int MODE>
cudaError_t launch_chunk(int ch, bool inter, dim3 grid, cudaStream_t st, const HeadsParams& P) {
  if constexpr (sizeof(T) == 2)
    if (ch == 8) return launch_layout<T, 8, 1, MODE>(inter, grid, st, P);
  if (ch == 4) return launch_layout<T, 4, 1, MODE>(inter, grid, st, P);
  if (ch == 2) return launch_layout<T, 2, 2, MODE>(inter, grid, st, P);
  return launch_layout<T, 1, 4, MODE>(inter, grid, st, P);
}

// Common to the three entry points.  `mode` NORM_BACKWARD: g = gradients of the forward outputs, y = dq / dk.
ff_status_t run(const ff_rotary_t* handle, int mode, int64_t batch, int64_t tokens, const int32_t* positions, int64_t position_stride,
                const ff_heads_t* const x[2], const ff_heads_t* const y[2], const ff_heads_t* const g[2], const float* const w[2], float eps,
                int inverse, float* dwq, float* dwk, void* ws, size_t ws_bytes, void* stream) {
  ff_rotary* h = const_cast<ff_rotary*>(handle);
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "the rotary handle is NULL");
  const ff_rotary_config_t& c = h->cfg;
  if (batch < 0 || tokens < 0) return fail(h, FF_ERR_INVALID_ARG, "batch and tokens must not be negative");
  if (!x[0] || !y[0]) return fail(h, FF_ERR_INVALID_ARG, "q is NULL");
  if (!x[1] != !y[1]) return fail(h, FF_ERR_INVALID_ARG, "k comes with its output, or neither does");
  if (mode != ROTATE && !(eps > 0.f && eps < 3.0e38f)) return fail(h, FF_ERR_INVALID_ARG, "eps must be positive and finite");
  if (batch > 0x7fffffff || tokens > 0x7fffffff || batch * tokens > 0x7fffffff) return fail(h, FF_ERR_UNSUPPORTED, "batch * tokens must be below 2^31");
  if (!positions && h->axes == 3) {
    const int64_t cells = (int64_t)c.grid[0] * c.grid[1] * c.grid[2];
    if (cells == 0) return fail(h, FF_ERR_INVALID_ARG, "without a grid the positions along its axes have to be given");
    if (cells != tokens) return fail(h, FF_ERR_INVALID_ARG, "without positions the tokens are the grid's cells: T * H * W of them");
  }
  if (positions && (((uintptr_t)positions) & 3)) return fail(h, FF_ERR_INVALID_ARG, "positions must be 4-byte aligned");
  if ((((uintptr_t)w[0]) | ((uintptr_t)w[1]) | ((uintptr_t)dwq) | ((uintptr_t)dwk)) & 3)
    return fail(h, FF_ERR_INVALID_ARG, "norm weights and their gradients must be 4-byte aligned");
  if (positions && position_stride < 0) return fail(h, FF_ERR_INVALID_ARG, "the positions' stride must not be negative");
  HeadsParams P{};
  Call call{h, batch, tokens, c.dtype == FF_FP32 ? 4 : 2, 0};
  const int kinds = x[1] ? 2 : 1;
  for (int t = 0; t < kinds; ++t) {
    if (x[t]->heads < 1) return fail(h, FF_ERR_INVALID_ARG, "a tensor has no heads");
    if (x[t]->heads > 65536) return fail(h, FF_ERR_UNSUPPORTED, "at most 65536 heads are supported");
    P.heads[t] = x[t]->heads;
    if (batch * tokens == 0) continue;
    ff_status_t s = check_view(call, x[t], x[t]->heads, false);
    if (s == FF_OK) s = check_view(call, y[t], x[t]->heads, true);
    if (s == FF_OK && mode == NORM_BACKWARD) s = g[t] ? check_view(call, g[t], x[t]->heads, false) : fail(h, FF_ERR_INVALID_ARG, "a gradient is NULL");
    if (s != FF_OK) return s;
    P.x[t] = view(x[t], call.e);
    P.y[t] = view(y[t], call.e);
    if (mode == NORM_BACKWARD) P.g[t] = view(g[t], call.e);
  }
  const bool want_dw = mode == NORM_BACKWARD && (dwq || dwk);
  size_t need = 0;
  if (mode == NORM_BACKWARD) {
    ff_qk_norm_workspace_bytes(handle, &need);
    if (!ws || ws_bytes < need) return fail(h, FF_ERR_WORKSPACE, "the workspace is missing or smaller than ff_qk_norm_workspace_bytes");
    if (((uintptr_t)ws) & 15) return fail(h, FF_ERR_WORKSPACE, "the workspace must be 16-byte aligned");
  }
  cudaStream_t st = (cudaStream_t)stream;
  if (batch * tokens == 0) {        // nothing to turn; sums over no rows are zero
    cudaError_t e = cudaSuccess;
    if (mode == NORM_BACKWARD && dwq) e = cudaMemsetAsync(dwq, 0, sizeof(float) * c.head_dim, st);
    if (e == cudaSuccess && mode == NORM_BACKWARD && dwk) e = cudaMemsetAsync(dwk, 0, sizeof(float) * c.head_dim, st);
    return e == cudaSuccess ? FF_OK : cuda_fail(h, e);
  }

  // the widest chunk that alignment and the channels' division allow
  const int half = c.rot_dim / 2, d = c.head_dim;
  const bool inter = c.layout == FF_ROTARY_INTERLEAVED;
  int ch = c.dtype == FF_FP32 ? 4 : 8;
  for (; ch > 1; ch >>= 1) {
    const bool fits = inter ? (c.rot_dim % ch == 0 && d % (2 * ch) == 0) : (half % ch == 0 && (d - c.rot_dim) % (2 * ch) == 0);
    if (fits && call.bits % ((uint64_t)ch * call.e) == 0) break;
  }
  if (inter && ch < 2) return fail(h, FF_ERR_UNSUPPORTED, "interleaved pairs need tensors aligned to two elements");
  P.np = d / (2 * ch);
  int lg = 0;
  while ((1 << lg) < P.np && lg < 5) ++lg;
  P.lanes_log2 = lg;
  P.rows = (int)(batch * tokens);
  P.tokens = ff_fast_div((unsigned)tokens);
  P.gw = ff_fast_div(c.grid[2] > 0 ? c.grid[2] : 1);
  P.gh = ff_fast_div(c.grid[1] > 0 ? c.grid[1] : 1);
  P.positions = positions; P.pos_stride = position_stride;
  P.d = d; P.rot = c.rot_dim;
  P.axis_end0 = h->axis_end[0]; P.axis_end1 = h->axis_end[1]; P.axes = h->axes;
  P.inverse = inverse; P.magnitude = h->magnitude; P.eps = eps;
  P.w[0] = w[0]; P.w[1] = w[1];
  memcpy(P.phase, h->phase, sizeof P.phase);

  const long long per_block = (long long)H_WARPS * (32 >> lg);
  P.groups = (int)((P.rows + per_block - 1) / per_block);
  dim3 grid;
  if (mode == NORM_BACKWARD) {
    const long long units0 = (long long)P.groups * P.heads[0], units1 = (long long)P.groups * P.heads[1];
    long long n0 = (units0 * PARTIAL_ROWS + (units0 + units1) / 2) / (units0 + units1);
    if (kinds == 2) n0 = n0 < 1 ? 1 : n0 >= PARTIAL_ROWS ? PARTIAL_ROWS - 1 : n0;
    long long n1 = kinds == 2 ? PARTIAL_ROWS - n0 : 0;
    if (n0 > units0) n0 = units0;
    if (n1 > units1) n1 = units1;
    P.nblocks0 = (int)n0;
    grid = dim3((unsigned)(n0 + n1));
  } else {
    const long long units = (long long)P.groups * ((P.heads[0] + 1) / 2 + (P.heads[1] + 1) / 2);
    // Runs of 16 units where there are eight waves of blocks of that many, shorter ones down to 8 units where there are not, and one wave
    // of equal runs where those would be fewer.  The SMs are not served by memory equally fast, so one wave of equal runs waits for the
    // last (64K tokens, 24 + 24 heads of 128 normed: 297 us in one wave, 258 in runs of 16; 16 + 16 heads of 64 turned: 95 and 82); a run has
    // to pay for its first token's angles and first loads (18228 tokens, 8 + 8 heads of 80 turned: 19.8 us in runs of 8, 23 of 4, 30 of 2).
    const long long wave = FORWARD_BLOCKS * FF_B200_SMS;
    long long each = units / (FORWARD_WAVES * wave);
    each = each < 8 ? 8 : each > 16 ? 16 : each;
    const long long blocks = units < wave ? units : units / each > wave ? units / each : wave;
    grid = dim3((unsigned)blocks);
  }
  P.partial = (float*)ws;
  cudaError_t e;
  if (mode == ROTATE) e = call.e == 4 ? launch_chunk<float, ROTATE>(ch, inter, grid, st, P) : launch_chunk<__nv_bfloat16, ROTATE>(ch, inter, grid, st, P);
  else if (mode == NORM) e = call.e == 4 ? launch_chunk<float, NORM>(ch, inter, grid, st, P) : launch_chunk<__nv_bfloat16, NORM>(ch, inter, grid, st, P);
  else e = call.e == 4 ? launch_chunk<float, NORM_BACKWARD>(ch, inter, grid, st, P) : launch_chunk<__nv_bfloat16, NORM_BACKWARD>(ch, inter, grid, st, P);
  if (e == cudaSuccess && want_dw)
    e = ff_launch(weight_gradient_kernel, dim3((d + 31) / 32, dwk ? 2 : 1), dim3(1024), 0, st, (const float*)P.partial, P.nblocks0,
                  (int)grid.x - P.nblocks0, d, dwq, dwk);
  return e == cudaSuccess ? FF_OK : cuda_fail(h, e);
}

}  // namespace

const ff_rotary_config_t* ffk_rotary_config(const ff_rotary_t* rotary) { return &rotary->cfg; }

extern "C" ff_status_t ff_rotary_create(const ff_rotary_config_t* cfg, ff_rotary_t** out) {
  if (!cfg || !out) return fail(nullptr, FF_ERR_INVALID_ARG, "cfg or out is NULL");
  *out = nullptr;
  const ff_rotary_config_t& c = *cfg;
  if (c.dtype != FF_BF16 && c.dtype != FF_FP32) return fail(nullptr, FF_ERR_INVALID_ARG, "dtype must be FF_BF16 or FF_FP32");
  if (c.layout != FF_ROTARY_HALF && c.layout != FF_ROTARY_INTERLEAVED) return fail(nullptr, FF_ERR_INVALID_ARG, "layout must be FF_ROTARY_HALF or FF_ROTARY_INTERLEAVED");
  if (c.scaling < FF_ROTARY_SCALE_NONE || c.scaling > FF_ROTARY_SCALE_BY_PARTS) return fail(nullptr, FF_ERR_INVALID_ARG, "unknown scaling");
  if (c.head_dim < 1 || c.rot_dim < 2 || (c.rot_dim & 1) || c.rot_dim > c.head_dim)
    return fail(nullptr, FF_ERR_INVALID_ARG, "rot_dim must be even and between 2 and head_dim");
  if (c.head_dim % 8 != 0 || c.head_dim > 256) return fail(nullptr, FF_ERR_UNSUPPORTED, "head_dim must be a multiple of 8 and <= 256");
  if (!(c.base >= 1.0) || !(c.base < 1e300)) return fail(nullptr, FF_ERR_INVALID_ARG, "base must be finite and at least 1");
  if (c.scaling != FF_ROTARY_SCALE_NONE && (!(c.factor >= 1.0) || !(c.factor <= 1e9))) return fail(nullptr, FF_ERR_INVALID_ARG, "the scaling factor must be between 1 and 1e9");
  if (c.scaling == FF_ROTARY_SCALE_BY_PARTS && c.original_length < 1) return fail(nullptr, FF_ERR_INVALID_ARG, "scaling by parts needs the original length");
  const int32_t* a = c.axis_pairs;
  const bool axes = a[0] || a[1] || a[2];
  if (a[0] < 0 || a[1] < 0 || a[2] < 0 || (axes && (int64_t)a[0] + a[1] + a[2] != c.rot_dim / 2))
    return fail(nullptr, FF_ERR_INVALID_ARG, "the pairs of the axes must add up to rot_dim / 2");
  const int32_t* n = c.grid;
  if (n[0] < 0 || n[1] < 0 || n[2] < 0 || ((n[0] || n[1] || n[2]) && !(n[0] && n[1] && n[2])))
    return fail(nullptr, FF_ERR_INVALID_ARG, "a grid has three positive axis lengths");
  if (n[0] && !axes) return fail(nullptr, FF_ERR_INVALID_ARG, "a grid needs the pairs of its axes");
  if ((double)n[0] * n[1] * n[2] > 2147483647.0) return fail(nullptr, FF_ERR_UNSUPPORTED, "a grid has fewer than 2^31 cells");
  ff_rotary* h = new (std::nothrow) ff_rotary();
  if (!h) return fail(nullptr, FF_ERR_INVALID_ARG, "out of host memory");
  h->cfg = c;
  h->pairs = c.rot_dim / 2;
  h->axes = axes ? 3 : 1;
  const int count[3] = {axes ? a[0] : h->pairs, axes ? a[1] : 0, axes ? a[2] : 0};
  h->axis_end[0] = count[0];
  h->axis_end[1] = count[0] + count[1];
  const long double tau = 6.283185307179586476925286766559005768L, s = c.scaling == FF_ROTARY_SCALE_NONE ? 1.0L : (long double)c.factor;
  for (int axis = 0, p = 0; axis < 3; ++axis)
    for (int i = 0; i < count[axis]; ++i, ++p) {
      const int P = count[axis];
      long double base = c.base;
      if (c.scaling == FF_ROTARY_SCALE_NTK && P > 1) base *= powl(s, (long double)P / (P - 1));
      long double th = powl(base, -(long double)i / P);
      if (c.scaling == FF_ROTARY_SCALE_LINEAR) th /= s;
      if (c.scaling == FF_ROTARY_SCALE_BY_PARTS) {
        long double keep = (c.original_length * th / tau - 1.0L) / 31.0L;
        keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
        th *= keep + (1 - keep) / s;
      }
      h->theta[p] = (double)th;
      h->phase[p] = (unsigned long long)ldexpl(th / tau, 64);      // theta <= 1: below 0.16 of a turn
    }
  h->magnitude = c.scaling == FF_ROTARY_SCALE_BY_PARTS ? (float)(0.1L * logl(s) + 1.0L) : 1.0f;
  *out = h;
  return FF_OK;
}

extern "C" ff_status_t ff_rotary_destroy(ff_rotary_t* h) {
  delete h;
  return FF_OK;
}

extern "C" const char* ff_rotary_last_error(const ff_rotary_t* h) { return h ? h->err : ff_last_error(nullptr); }

extern "C" ff_status_t ff_rotary_frequencies(const ff_rotary_t* h, double* theta, double* magnitude) {
  if (!h || !theta || !magnitude) return fail(const_cast<ff_rotary*>(h), FF_ERR_INVALID_ARG, "handle, theta or magnitude is NULL");
  for (int p = 0; p < h->pairs; ++p) theta[p] = h->theta[p];
  *magnitude = h->magnitude;
  return FF_OK;
}

extern "C" ff_status_t ff_qk_norm_workspace_bytes(const ff_rotary_t* h, size_t* bytes) {
  if (!h || !bytes) return fail(const_cast<ff_rotary*>(h), FF_ERR_INVALID_ARG, "handle or bytes is NULL");
  *bytes = (size_t)PARTIAL_ROWS * h->cfg.head_dim * sizeof(float);
  return FF_OK;
}

extern "C" ff_status_t ff_rotary_apply(const ff_rotary_t* h, int64_t batch, int64_t tokens, const int32_t* positions, int64_t position_stride,
                                       const ff_heads_t* q, const ff_heads_t* k, int32_t inverse, const ff_heads_t* q_out,
                                       const ff_heads_t* k_out, void* stream) {
  const ff_heads_t *x[2] = {q, k}, *y[2] = {q_out, k_out}, *g[2] = {};
  const float* w[2] = {};
  return run(h, ROTATE, batch, tokens, positions, position_stride, x, y, g, w, 0.f, inverse != 0, nullptr, nullptr, nullptr, 0, stream);
}

extern "C" ff_status_t ff_qk_norm(const ff_rotary_t* h, int64_t batch, int64_t tokens, const int32_t* positions, int64_t position_stride,
                                  const ff_heads_t* q, const ff_heads_t* k, const float* wq, const float* wk, float eps,
                                  const ff_heads_t* q_out, const ff_heads_t* k_out, void* stream) {
  const ff_heads_t *x[2] = {q, k}, *y[2] = {q_out, k_out}, *g[2] = {};
  const float* w[2] = {wq, wk};
  return run(h, NORM, batch, tokens, positions, position_stride, x, y, g, w, eps, 0, nullptr, nullptr, nullptr, 0, stream);
}

extern "C" ff_status_t ff_qk_norm_backward(const ff_rotary_t* h, int64_t batch, int64_t tokens, const int32_t* positions, int64_t position_stride,
                                           const ff_heads_t* q, const ff_heads_t* k, const float* wq, const float* wk, float eps,
                                           const ff_heads_t* dq_out, const ff_heads_t* dk_out, const ff_heads_t* dq, const ff_heads_t* dk,
                                           float* dwq, float* dwk, void* workspace, size_t workspace_bytes, void* stream) {
  const ff_heads_t *x[2] = {q, k}, *y[2] = {dq, dk}, *g[2] = {dq_out, dk_out};
  const float* w[2] = {wq, wk};
  return run(h, NORM_BACKWARD, batch, tokens, positions, position_stride, x, y, g, w, eps, 1, dwq, dwk, workspace, workspace_bytes, stream);
}
