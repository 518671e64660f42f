// Rows of the vocabulary matrix for tokens, and the gradient of that lookup:
//   y[i] = scale * W[t_i],           dW[v] = scale * sum over i with t_i = v of g[i]  (+ dW[v]),
// where a token outside [0, V) (the -1 of padded targets and of beams without a candidate) is a row of zeros
// and gives no gradient.  In 8 bits a row of W is s_v * q[v].
//
// The gradient is made without atomics on values: the positions are sorted by token, positions of one token in
// ascending order, and the sums run over the sorted positions, so repeated calls agree bit for bit.
//   k_sort_tokens  a CTA for each of about 148 ranges of the vocabulary reads all tokens (they are in L2) and
//                  lays its own out in order: no CTA needs another's result, so one launch sorts.  Meanwhile
//                  other CTAs of that launch fill dW with zeros, whatever the tokens are.
//   k_embed_grad   a thread sums eight columns over a window of sorted positions.  A token whose positions pass the
//                  end of a window leaves a partial sum for each window, and the last of its threads adds these up in
//                  order (in two steps where they are many).
//   k_embed_grad_few  few tokens: all of it in one launch.  A CTA fills its rows with zeros, finds its own among all
//                  tokens meanwhile and writes their sums behind the zeros.
// Both directions are bound by HBM where they are large (32,768 tokens of 151,936 x 2,560 bf16: 48.5 us, 6.2 TB/s; the
// gradient of as many into 151,936 x 1,024: 69 us, 5.4 TB/s), by their launches where they are small (64 tokens: 1.8 us; 1,999 into
// 5,003 x 510: 12 us, two launches and the chain from a token to its last partial sum).
#include "../../include/prunedctc.h"
#include "pctc_internal.h"
#include "vec8.cuh"

#include <atomic>
#include <cmath>

namespace pctc {
namespace {

constexpr int EMBED_THREADS = 128;
// Groups of n values a thread.  Twice as many and twice the threads a block, which stores them a longer while after the loads: 32,768 tokens
// of 2,560 bf16 49.3 -> 51.5 us, of 1,020 27.5 -> 49.7, of 1,023 78 -> 111; half as many: 51, 36, 137.
constexpr int embed_each(int n) { return n == 8 ? 2 : 3; }

struct EmbedArgs {
  const int* tokens;
  const void* W;
  const float* row_scales;                       // 8-bit matrix: [V], else null
  void* out;
  long long M, V, D, ld_w, ld_out;
  unsigned per_row;                              // groups of N values a row
  float scale;
};

// N: as many values as every row is cut into evenly and aligned for.  (Eight unaligned ones a thread, put together from words
// and odd halves, spread a warp's accesses over eight times the lines: 13,195 x 141 fp32 7.1 -> 12.7 us.)
template <typename W, typename T, int N>
__global__ void __launch_bounds__(EMBED_THREADS) k_embed(const EmbedArgs a) {
  constexpr int EACH = embed_each(N);
  const long long g0 = (long long)blockIdx.x * (EMBED_THREADS * EACH) + threadIdx.x;
  // the row of the first group by division, those of the others by what they are further on
  long long row = g0 / a.per_row;
  unsigned col = (unsigned)(g0 - row * a.per_row);
  long long rows[EACH];
  unsigned cols[EACH];
  int token[EACH];
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    rows[k] = row;
    cols[k] = col;
    token[k] = row < a.M ? a.tokens[row] : -1;
    col += EMBED_THREADS;
    if (col >= a.per_row) { row += col / a.per_row; col %= a.per_row; }
  }
  VecN<W, N> v[EACH];
  float f[EACH];
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    if ((unsigned long long)(long long)token[k] >= (unsigned long long)a.V) token[k] = -1;
    f[k] = a.scale;
    if (token[k] < 0) continue;
    v[k].load((const W*)a.W + token[k] * a.ld_w + cols[k] * (long long)N);
    if (a.row_scales) f[k] *= a.row_scales[token[k]];
  }
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    if (rows[k] >= a.M) continue;
    float x[N] = {};
    if (token[k] >= 0)
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = v[k].value(j) * f[k];
    VecN<T, N>::store((T*)a.out + rows[k] * a.ld_out + cols[k] * (long long)N, x);
  }
}

// ---------------------------------------------------------------------------------------------
// Gradient
// ---------------------------------------------------------------------------------------------
constexpr int SORT_THREADS = 512;
constexpr int SORT_WARPS = SORT_THREADS / 32;
static_assert(SORT_WARPS % 8 == 0, "the counters of eight warps at a time");
constexpr int SORT_BUCKETS = 148;                // ranges of the vocabulary: one CTA on every SM of a B200
constexpr int SORT_MAX_WIDTH = 2048;             // tokens of a range: a counter for each and every warp, 128 KB
constexpr int SORT_AHEAD = 4;                    // groups of four tokens that a thread loads before it looks at the first
constexpr int SORT_KEEP = 256;                   // tokens of its range that a warp keeps; one with more reads its run again
                                                 // (three blocks an SM: with two 70,000 x 512 takes 23.8 us for 22.0)
constexpr int SORT_RUN_BITS = 21;                // a kept token: 11 bits of token, 21 of position in the warp's run

// Zeros into a matrix, in pieces of about ZERO_BYTES: of rows, or of the bytes of a matrix without gaps.
constexpr int ZERO_BYTES = 32768;
struct ZeroArgs {
  char* p;
  long long rows, ld, width;                     // bytes
  long long piece;                               // rows a piece
  long long pieces;
};
__device__ __forceinline__ void zero_row(char* row, long long n, int lane, int lanes) {
  const long long head = min((long long)((16 - ((size_t)row & 15)) & 15), n) / 2, vecs = (n - 2 * head) / 16;
  for (long long i = lane; i < head; i += lanes) reinterpret_cast<short*>(row)[i] = 0;
  uint4* body = reinterpret_cast<uint4*>(row + 2 * head);
#pragma unroll 4
  for (long long i = lane; i < vecs; i += lanes) body[i] = make_uint4(0u, 0u, 0u, 0u);
  for (long long i = head + vecs * 8 + lane; i < n / 2; i += lanes) reinterpret_cast<short*>(row)[i] = 0;
}
template <int THREADS>
__device__ __forceinline__ void zero_piece(const ZeroArgs& a, long long piece) {
  const long long r0 = piece * a.piece, r1 = min(r0 + a.piece, a.rows);
  if (a.width == a.ld) {
    zero_row(a.p + r0 * a.ld, (r1 - r0) * a.ld, threadIdx.x, THREADS);
  } else {
    for (long long r = r0 + (threadIdx.x >> 5); r < r1; r += THREADS / 32) zero_row(a.p + r * a.ld, a.width, threadIdx.x & 31, 32);
  }
}

struct SortArgs {
  const int* tokens;
  int M;
  long long V;
  int width;                                     // tokens of a range
  int2* sorted;                                  // [M] (position, token) by token, then position; (0, -1) behind them
  int* first;                                    // [V + 1] where a token's positions begin
  int* clear;                                    // counters of k_embed_grad, zeroed here
  long long n_clear;
  unsigned buckets;                              // blocks that sort; the others fill dW with zeros
  ZeroArgs zero;
};

// Tokens p .. p + 3 of a run that ends at p1 (p is a multiple of 4); -1 behind the end.
__device__ __forceinline__ int4 four_tokens(const int* tokens, bool aligned, int p, int p1) {
  if (aligned && p + 4 <= p1) return *reinterpret_cast<const int4*>(tokens + p);
  return make_int4(p < p1 ? tokens[p] : -1, p + 1 < p1 ? tokens[p + 1] : -1, p + 2 < p1 ? tokens[p + 2] : -1,
                   p + 3 < p1 ? tokens[p + 3] : -1);
}

__global__ void __launch_bounds__(SORT_THREADS, 3) k_sort_tokens(const SortArgs a) {
  extern __shared__ int count[];                 // [SORT_WARPS][width]: counts, then where each warp's next one goes
  __shared__ unsigned kept[SORT_WARPS][SORT_KEEP];
  __shared__ int below_sum[SORT_WARPS], scan_sum[SORT_WARPS], count_end;
  launch_next();
  if (blockIdx.x >= a.buckets) {
    zero_piece<SORT_THREADS>(a.zero, blockIdx.x - a.buckets);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned lo = blockIdx.x * (unsigned)a.width, width = (unsigned)min((long long)a.width, a.V - lo);
  for (long long i = (long long)blockIdx.x * SORT_THREADS + threadIdx.x; i < a.n_clear; i += (long long)a.buckets * SORT_THREADS)
    a.clear[i] = 0;
  for (int i = threadIdx.x; i < SORT_WARPS * a.width; i += SORT_THREADS) count[i] = 0;
  __syncthreads();

  // a warp takes a run of positions, so that warps, steps, lanes and a lane's four in order are positions in order
  const int run = (int)(((long long)a.M + SORT_WARPS * 128 - 1) / (SORT_WARPS * 128)) * 128;
  const int p0 = (int)min((long long)warp * run, (long long)a.M), p1 = (int)min((long long)p0 + run, (long long)a.M);
  const bool aligned = ((size_t)a.tokens & 15) == 0;
  const unsigned lower = (1u << lane) - 1;
  int* mine = count + warp * a.width;
  int below = 0, n = 0;
  // 128 tokens a step, SORT_AHEAD steps loaded at once; f(v, first position of the lane) for those with a token of the range
  const auto for_all = [&](auto f) {
    for (int p = p0 + lane * 4; p - lane * 4 < p1; p += 128 * SORT_AHEAD) {
      int4 t[SORT_AHEAD];
#pragma unroll
      for (int k = 0; k < SORT_AHEAD; ++k) t[k] = four_tokens(a.tokens, aligned, p + k * 128, p1);
#pragma unroll
      for (int k = 0; k < SORT_AHEAD; ++k) f(t[k], p + k * 128);
    }
  };
  // keeps those of the four that are in the range, in order, behind the n that are there; counts them
  const auto keep = [&](const unsigned (&v)[4], unsigned position, bool count_them) {
    int before = n;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned hits = __ballot_sync(0xffffffffu, v[j] < width);
      before += __popc(hits & lower);
      n += __popc(hits);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (v[j] < width) {
        if (count_them) atomicAdd(&mine[v[j]], 1);
        if (before < SORT_KEEP) kept[warp][before] = (v[j] << SORT_RUN_BITS) | (position + j);
        ++before;
      }
  };
  for_all([&](const int4& t, int p) {
    const unsigned v[4] = {(unsigned)t.x - lo, (unsigned)t.y - lo, (unsigned)t.z - lo, (unsigned)t.w - lo};
    below += ((unsigned)t.x < lo) + ((unsigned)t.y < lo) + ((unsigned)t.z < lo) + ((unsigned)t.w < lo);   // none below 0
    if (!__any_sync(0xffffffffu, v[0] < width || v[1] < width || v[2] < width || v[3] < width)) return;
    keep(v, (unsigned)(p - p0), true);
  });
  below = __reduce_add_sync(0xffffffffu, below);
  if (lane == 0) below_sum[warp] = below;
  __syncthreads();

  // counts -> where each warp's first position of each token goes
  const unsigned per = (width + SORT_THREADS - 1) / SORT_THREADS, k0 = threadIdx.x * per;
  int sum = 0;
  for (unsigned k = k0; k < k0 + per && k < width; ++k)
#pragma unroll
    for (int w = 0; w < SORT_WARPS; ++w) sum += count[w * a.width + k];
  int scan = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, scan, d);
    if (lane >= d) scan += up;
  }
  if (lane == 31) scan_sum[warp] = scan;
  __syncthreads();
  int at = scan - sum;
#pragma unroll
  for (int w = 0; w < SORT_WARPS; ++w) at += below_sum[w] + (w < warp ? scan_sum[w] : 0);
  for (unsigned k = k0; k < k0 + per && k < width; ++k) {
    a.first[lo + k] = at;
#pragma unroll
    for (int w0 = 0; w0 < SORT_WARPS; w0 += 8) {
      int c[8];
#pragma unroll
      for (int w = 0; w < 8; ++w) c[w] = count[(w0 + w) * a.width + k];
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        count[(w0 + w) * a.width + k] = at;
        at += c[w];
      }
    }
  }
  if (k0 < width && k0 + per >= width) {
    count_end = at;
    if (lo + (long long)width == a.V) a.first[a.V] = at;
  }
  __syncthreads();
  if (lo + (long long)width == a.V)              // positions without a token
    for (int i = count_end + threadIdx.x; i < a.M; i += SORT_THREADS) a.sorted[i] = make_int2(0, -1);

  // the kept ones, 32 at a time: equal ones by lane
  const auto place = [&](int from) {
    __syncwarp();
    for (int i = lane; i - lane < n; i += 32) {
      const bool there = i < n;
      const unsigned x = there ? kept[warp][i] : 0u;
      const int key = (int)(x >> SORT_RUN_BITS);
      const unsigned hits = __ballot_sync(0xffffffffu, there);
      if (there) {
        const unsigned equal = __match_any_sync(hits, key);
        const int rank = __popc(equal & lower), to = mine[key] + rank;
        __syncwarp(hits);
        if (rank == 0) mine[key] = to + __popc(equal);
        a.sorted[to] = make_int2(from + (int)(x & ((1u << SORT_RUN_BITS) - 1)), (int)lo + key);
      }
      __syncwarp();
    }
    n = 0;
  };
  if (n <= SORT_KEEP && run <= 1 << SORT_RUN_BITS) {
    place(p0);
    return;
  }
  // more than are kept: once more over the run, in portions that fit
  n = 0;
  int from = p0;
  for_all([&](const int4& t, int p) {
    const unsigned v[4] = {(unsigned)t.x - lo, (unsigned)t.y - lo, (unsigned)t.z - lo, (unsigned)t.w - lo};
    if (!__any_sync(0xffffffffu, v[0] < width || v[1] < width || v[2] < width || v[3] < width)) return;
    const int first = p - lane * 4;
    if (n > SORT_KEEP - 128 || first - from > (1 << SORT_RUN_BITS) - 128) place(from);
    if (n == 0) from = first;
    keep(v, (unsigned)(p - from), false);
  });
  place(from);
}

struct GradArgs {
  const void* g;
  void* dW;
  const int2* sorted;
  const int* first;
  float* part;                                   // [windows][2][per_row * N]
  int* arrived;                                  // [windows][2][per_row]
  long long ld_g, ld_w, M;
  long long windows;
  unsigned per_row;                              // groups of N values a row
  int window;                                    // sorted positions a thread takes
  float scale;
};

template <bool ADD, typename T, int N>
__device__ __forceinline__ void write_row(T* p, const float (&sum)[N], float scale) {
  float x[N];
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = sum[j] * scale;
  if (ADD) {
    VecN<T, N> old;
    old.load(p);
    old.add_to(x);
  }
  VecN<T, N>::store(p, x);
}

constexpr int GRAD_THREADS = 256;
constexpr int GRAD_AHEAD = 8;                    // rows that a thread loads before it adds the first; windows are a multiple of it
constexpr int GRAD_MOST = 64;                    // sorted positions of a window, at most (32: 70 -> 74 us)
constexpr int GRAD_JOIN = 32;                    // windows whose parts one thread adds up, of a token of more than twice as many (65,536
                                                 // tokens of 500, as frequent as in text, D = 64: 96 -> 39 us)
constexpr int GRAD_STAGED = 2048;                // sorted positions of a block's windows, at most
constexpr int GRAD_PER_SM = 2;                   // blocks that run on an SM at a time: three spill registers (72 -> 74 us)
constexpr int GRAD_WAVE = 148 * GRAD_PER_SM * GRAD_THREADS;

// N: as many values as 16 bytes of g hold where all is aligned for that, else 2 or 1.
template <bool ADD, typename G, typename T, int N>
__global__ void __launch_bounds__(GRAD_THREADS, N >= 4 ? GRAD_PER_SM : 4) k_embed_grad(const GradArgs a) {
  __shared__ int2 staged[GRAD_STAGED + 2];       // the block's sorted positions, with one before and one behind
  const long long id0 = (long long)blockIdx.x * GRAD_THREADS, block_w = id0 / a.per_row;
  const unsigned id = (unsigned)(id0 - block_w * a.per_row) + threadIdx.x, nth = id / a.per_row, c = id - nth * a.per_row;
  const long long from = block_w * a.window, w = block_w + nth;
  const int count = (int)min((long long)((unsigned)(id0 - block_w * a.per_row) + GRAD_THREADS - 1) / a.per_row + 1, a.windows - block_w) * a.window;
  wait_for_previous();
  for (int i = threadIdx.x; i < count + 2; i += GRAD_THREADS) {
    const long long at = from + i - 1;
    staged[i] = at >= 0 && at < a.M ? a.sorted[at] : make_int2(0, -1);
  }
  __syncthreads();
  if (w >= a.windows) return;
  const int2* mine = staged + 1 + nth * a.window;
  const int v0 = mine[0].y;                      // -1: nothing but positions without a token from here on
  if (v0 < 0) return;
  const G* g = (const G*)a.g + (long long)c * N;
  T* dW = (T*)a.dW + (long long)c * N;
  // a token whose positions pass an end of the window leaves a part of its sum; what the end of its sum will need is
  // loaded ahead
  const int last = mine[a.window - 1].y;
  const bool head = v0 == mine[-1].y, tail = last >= 0 && last == mine[a.window].y;
  int2 head_range, tail_range;
  if (head) head_range = make_int2(a.first[v0], a.first[v0 + 1]);
  if (tail) tail_range = make_int2(a.first[last], a.first[last + 1]);

  float sum[N] = {}, head_sum[N];
  int v = v0;
  bool aside = head;                             // the sum that runs goes to head_sum
  for (int s = 0; s < a.window; s += GRAD_AHEAD) {
    VecN<G, N> x[GRAD_AHEAD];
#pragma unroll
    for (int k = 0; k < GRAD_AHEAD; ++k)
      if (mine[s + k].y >= 0) x[k].load(g + mine[s + k].x * a.ld_g);
#pragma unroll
    for (int k = 0; k < GRAD_AHEAD; ++k) {
      const int key = mine[s + k].y;
      if (key < 0) break;
      if (key != v) {
        if (aside) {
#pragma unroll
          for (int j = 0; j < N; ++j) head_sum[j] = sum[j];
        } else {
          write_row<ADD>(dW + v * a.ld_w, sum, a.scale);
        }
        aside = false;
        v = key;
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] = 0.f;
      }
      x[k].add_to(sum);
    }
  }
  if (!aside && !tail) write_row<ADD>(dW + v * a.ld_w, sum, a.scale);
  if (!head && !tail) return;

  // parts: those of a window's first token at 0, those of a token that begins in it at `width`
  const long long width = (long long)a.per_row * N;
  float* part = a.part + w * 2 * width + (long long)c * N;
  if (head) {
    if (aside) VecN<float, N>::store(part, sum); else VecN<float, N>::store(part, head_sum);
  }
  if (tail && !aside) VecN<float, N>::store(part + width, sum);
  // Whoever comes last adds up the parts of a token, in the order of the windows.  Those of a token of more than 2 GRAD_JOIN windows
  // are added up by GRAD_JOIN of them (from every multiple of it on), and these sums by the last of these.  A part's place and
  // counter are those of its first window.
  __threadfence();
  constexpr int JOIN_AHEAD = N == 8 ? 4 : 8;     // parts loaded at once
  float* parts = a.part + (long long)c * N;
#pragma unroll 1
  for (int e = 0; e < 2; ++e) {
    if (e == 0 ? !head : !tail || aside) continue;
    const int2 range = e == 0 ? head_range : tail_range;
    const int w0 = range.x / a.window, w1 = (range.y - 1) / a.window, start = (int)w & -GRAD_JOIN;
    const bool all_at_once = w1 - w0 < 2 * GRAD_JOIN;
    const int u0 = all_at_once || start < w0 ? w0 : start, u1 = all_at_once || start + GRAD_JOIN > w1 ? w1 : start + GRAD_JOIN - 1;
    const auto place = [&](int u) { return (long long)(u * 2 + (u == w0 ? 1 : 0)); };
    if (u1 > u0) {
      if (atomicAdd(&a.arrived[place(u0) * a.per_row + c], 1) % (4 * GRAD_JOIN) != u1 - u0) continue;
      __threadfence();
    }
    // first the parts of windows u0 .. u1, then the sums at w0 and at every multiple of GRAD_JOIN behind it
    int first = u0, base = u0, step = 1, n = u1 - u0 + 1;
    bool whole = u0 == w0 && u1 == w1;
#pragma unroll 1
    while (true) {
      float all[N] = {};
#pragma unroll 1
      for (int i = 0; i < n; i += JOIN_AHEAD) {
        VecN<float, N> q[JOIN_AHEAD];
#pragma unroll
        for (int k = 0; k < JOIN_AHEAD; ++k)
          if (i + k < n) q[k].load_l2(parts + place(i + k == 0 ? first : base + (i + k) * step) * width);
#pragma unroll
        for (int k = 0; k < JOIN_AHEAD; ++k)
          if (i + k < n) q[k].add_to(all);
      }
      if (whole) {
        write_row<ADD>(dW + (e == 0 ? v0 : last) * a.ld_w, all, a.scale);
        break;
      }
      VecN<float, N>::store(parts + place(u0) * width, all);
      __threadfence();
      base = w0 & -GRAD_JOIN;
      n = (w1 - base) / GRAD_JOIN + 1;
      if (atomicAdd(&a.arrived[place(w0) * a.per_row + c], 4 * GRAD_JOIN) / (4 * GRAD_JOIN) != n - 1) break;
      __threadfence();
      first = w0;
      step = GRAD_JOIN;
      whole = true;
    }
  }
}

// Up to GRAD_FEW tokens (1 to 256 into 5,003 x 510 fp32: 4.3 to 6.4 us, by sorting 5.4 to 9.9).  Block (x, y) takes every
// gridDim.x-th piece of rows from piece x on, and columns y * GRAD_SLICE ..
constexpr int GRAD_FEW = GRAD_THREADS;           // a token a thread
constexpr int GRAD_SLICE = 1024;                 // columns of a block

struct FewArgs {
  const int* tokens;
  const void* g;
  void* dW;
  long long ld_g, ld_w, V, D;
  int M;
  int accumulate;
  float scale;
  ZeroArgs zero;                                 // the pieces (and, if the block has all columns, where the zeros go)
};

template <typename G, typename T, int N>
__global__ void __launch_bounds__(GRAD_THREADS) k_embed_grad_few(const FewArgs a) {
  __shared__ int found[GRAD_FEW], row_of[GRAD_FEW + 1], position[GRAD_FEW], begin[GRAD_FEW];
  __shared__ int warp_count[GRAD_THREADS / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long c0 = (long long)blockIdx.y * GRAD_SLICE;
  const int cols = (int)min((long long)GRAD_SLICE, a.D - c0);
  const int token = threadIdx.x < a.M ? a.tokens[threadIdx.x] : -1;
  if (!a.accumulate) {                           // before any token is known: the stores go out while the first load is on its way
    ZeroArgs z = a.zero;
    z.p += c0 * sizeof(T);
    if (gridDim.y > 1) z.width = cols * (long long)sizeof(T);
    for (long long piece = blockIdx.x; piece < z.pieces; piece += gridDim.x) zero_piece<GRAD_THREADS>(z, piece);
  }
  const bool hit = token >= 0 && token < a.V && (token / a.zero.piece) % gridDim.x == blockIdx.x;
  // the block's tokens, in order of their positions
  const auto compact = [&](bool yes, int& n) {   // the place of a thread that says yes, and how many do
    const unsigned all = __ballot_sync(0xffffffffu, yes);
    __syncthreads();
    if (lane == 0) warp_count[warp] = __popc(all);
    __syncthreads();
    int at = __popc(all & ((1u << lane) - 1));
    n = 0;
#pragma unroll
    for (int w = 0; w < GRAD_THREADS / 32; ++w) {
      if (w < warp) at += warp_count[w];
      n += warp_count[w];
    }
    return at;
  };
  int n, rows;
  const int at = compact(hit, n);
  if (n == 0) return;
  if (hit) found[at] = token;
  __syncthreads();
  if (hit) {                                     // by row, then position
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += found[j] < token || (found[j] == token && j < at);
    row_of[rank] = token;
    position[rank] = threadIdx.x;
  }
  if (threadIdx.x == 0) row_of[n] = -1;
  __syncthreads();
  const bool first = (int)threadIdx.x < n && (threadIdx.x == 0 || row_of[threadIdx.x - 1] != row_of[threadIdx.x]);
  const int nth = compact(first, rows);
  if (first) begin[nth] = threadIdx.x;
  __syncthreads();                               // the zeros of the block's rows come before their sums, too

  const int per_row = cols / N;
  for (int i = threadIdx.x; i < rows * per_row; i += GRAD_THREADS) {
    const int r = i / per_row, c = (i - r * per_row) * N, s = begin[r], row = row_of[s];
    const int end = r + 1 < rows ? begin[r + 1] : n;
    float sum[N] = {};
    for (int e = s; e < end; e += GRAD_AHEAD) {
      VecN<G, N> x[GRAD_AHEAD];
#pragma unroll
      for (int k = 0; k < GRAD_AHEAD; ++k)
        if (e + k < end) x[k].load((const G*)a.g + position[e + k] * a.ld_g + c0 + c);
#pragma unroll
      for (int k = 0; k < GRAD_AHEAD; ++k)
        if (e + k < end) x[k].add_to(sum);
    }
    T* to = (T*)a.dW + row * a.ld_w + c0 + c;
    if (a.accumulate) write_row<true>(to, sum, a.scale); else write_row<false>(to, sum, a.scale);
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
constexpr size_t EMBED_ALIGN = 256;
size_t up(size_t b) { return (b + EMBED_ALIGN - 1) / EMBED_ALIGN * EMBED_ALIGN; }

struct GradPlan {
  int window;
  long long windows;
  size_t sorted, first, part, arrived, total;
};
// The window: as many threads as run at a time, and no more partial sums than that takes.
GradPlan grad_plan(const pctc_embed_t* p) {
  GradPlan g;
  const long long groups = (p->D + 7) / 8, rows = (p->M * groups + GRAD_WAVE - 1) / GRAD_WAVE;
  // a block's windows fit its staging, with as few as one group a row
  const long long fit = GRAD_STAGED / (GRAD_THREADS / groups + 2) / 8 * 8, most = fit < 8 ? 8 : fit < GRAD_MOST ? fit : GRAD_MOST;
  const int window = (int)(rows < 8 ? 8 : rows > most ? most : (rows + 7) / 8 * 8);
  g.window = window;
  g.windows = (p->M + window - 1) / window;
  size_t o = 0;
  const auto take = [&](size_t bytes) { const size_t r = o; o += up(bytes); return r; };
  g.sorted = take((size_t)p->M * 8);
  g.first = take(((size_t)p->V + 1) * 4);
  g.arrived = take((size_t)g.windows * 2 * p->D * 4);   // a counter a group of values, or a value
  g.part = take((size_t)g.windows * 2 * p->D * 4);
  g.total = o;
  return g;
}

pctc_status_t check_embed(const pctc_embed_t* p) {
  if (!p || p->M < 0 || p->V < 1 || p->D < 1 || !std::isfinite(p->scale)) return PCTC_ERR_INVALID_ARG;
  if (p->ld_w < p->D || p->ld_x < p->D) return PCTC_ERR_INVALID_ARG;
  // (the sort's steps of positions run past M by up to 128 * SORT_AHEAD * 2)
  if (p->M > 0x7fffffffLL - 4096 || p->V > 0x7fffffffLL - 1 || p->D > (1 << 24)) return PCTC_ERR_UNSUPPORTED;
  if (p->ld_w > MAX_ELEMENTS / p->V || p->ld_x > MAX_ELEMENTS / (p->M + 1)) return PCTC_ERR_UNSUPPORTED;
  return PCTC_OK;
}
size_t size_of(int dtype) { return dtype == PCTC_BF16 ? 2 : dtype == PCTC_FP32 ? 4 : 1; }
// Whether rows of D values can be cut into groups of n that are aligned for their accesses.
bool fits(int n, long long D, const void* p, long long ld, size_t size) {
  const size_t bytes = n * size < 16 ? n * size : 16;
  return D % n == 0 && (size_t)p % bytes == 0 && ld * size % bytes == 0;
}

template <typename W, typename T, int N>
cudaError_t embed_launch(EmbedArgs a, cudaStream_t stream) {
  a.per_row = (unsigned)(a.D / N);
  constexpr int per = EMBED_THREADS * embed_each(N);
  const long long blocks = (a.M * a.per_row + per - 1) / per;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
  k_embed<W, T, N><<<(unsigned)blocks, EMBED_THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}
template <typename W, typename T>
cudaError_t embed_launch(const EmbedArgs& a, cudaStream_t stream) {
  const auto can = [&](int n) { return fits(n, a.D, a.W, a.ld_w, sizeof(W)) && fits(n, a.D, a.out, a.ld_out, sizeof(T)); };
  return can(8)   ? embed_launch<W, T, 8>(a, stream)
         : can(4) ? embed_launch<W, T, 4>(a, stream)
         : can(2) ? embed_launch<W, T, 2>(a, stream)
                  : embed_launch<W, T, 1>(a, stream);
}
template <typename W>
cudaError_t embed_launch(const EmbedArgs& a, int out, cudaStream_t stream) {
  return out == PCTC_BF16 ? embed_launch<W, __nv_bfloat16>(a, stream) : embed_launch<W, float>(a, stream);
}

ZeroArgs zero_args(void* dW, long long V, long long D, long long ld, size_t size, long long least_pieces) {
  ZeroArgs z;
  z.p = (char*)dW;
  z.rows = V;
  z.ld = ld * (long long)size;
  z.width = D * (long long)size;
  const long long fit = ZERO_BYTES / z.width, spread = V / least_pieces;   // rows: that fill a piece, that leave enough pieces
  z.piece = fit < spread ? fit : spread;
  if (z.piece < 1) z.piece = 1;
  z.pieces = (V + z.piece - 1) / z.piece;
  return z;
}

// The widest groups of g's values that every row of both matrices is cut into evenly and aligned for.
int group_of(const void* g, long long ld_g, size_t gs, const void* dW, long long ld_w, size_t ws, long long D) {
  const auto can = [&](int n) { return fits(n, D, g, ld_g, gs) && fits(n, D, dW, ld_w, ws); };
  return can(16 / (int)gs) ? 16 / (int)gs : can(2) ? 2 : 1;
}

template <typename G, typename T, int N>
cudaError_t grad_launch(GradArgs a, long long D, bool add, cudaStream_t stream) {
  a.per_row = (unsigned)(D / N);
  const long long blocks = (a.windows * a.per_row + GRAD_THREADS - 1) / GRAD_THREADS;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
  return launch_behind(add ? k_embed_grad<true, G, T, N> : k_embed_grad<false, G, T, N>, (unsigned)blocks, GRAD_THREADS, 0, stream, a);
}
template <typename G, typename T>
cudaError_t grad_launch(const GradArgs& a, long long D, int group, bool add, cudaStream_t stream) {
  return group == 1 ? grad_launch<G, T, 1>(a, D, add, stream) : group == 2 ? grad_launch<G, T, 2>(a, D, add, stream)
                    : grad_launch<G, T, 16 / (int)sizeof(G)>(a, D, add, stream);
}

// A block for 48 KB of dW, at least 8 an SM and at most 32: every one of them goes over all tokens, and few blocks leave the
// memory idle at the end (148 * 8, 16 and 32 blocks: 10 MB 4.7, 6.6 and 11 us, 116 MB 18.4, 17.6 and 17.7, 622 MB 93, 89 and 88).
constexpr long long FEW_BYTES = 49152, FEW_LEAST = 148 * 8, FEW_MOST = 148 * 32;
template <typename G, typename T>
cudaError_t few_launch(FewArgs a, int group, cudaStream_t stream) {
  const long long pieces = a.accumulate ? 0 : a.V * a.D * (long long)sizeof(T) / FEW_BYTES;
  const long long blocks = pieces < FEW_LEAST ? FEW_LEAST : pieces > FEW_MOST ? FEW_MOST : pieces;
  const long long slices = (a.D + GRAD_SLICE - 1) / GRAD_SLICE, most = (blocks + slices - 1) / slices;
  a.zero = zero_args(a.dW, a.V, a.D, a.ld_w, sizeof(T), most);
  const dim3 grid((unsigned)(a.zero.pieces < most ? a.zero.pieces : most), (unsigned)slices);
  if (group == 1) k_embed_grad_few<G, T, 1><<<grid, GRAD_THREADS, 0, stream>>>(a);
  else if (group == 2) k_embed_grad_few<G, T, 2><<<grid, GRAD_THREADS, 0, stream>>>(a);
  else k_embed_grad_few<G, T, 16 / (int)sizeof(G)><<<grid, GRAD_THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}

pctc_status_t status_of(cudaError_t e) {
  return e == cudaSuccess ? PCTC_OK : e == cudaErrorInvalidValue ? PCTC_ERR_UNSUPPORTED : PCTC_ERR_CUDA;
}

}  // namespace
}  // namespace pctc

using namespace pctc;

extern "C" {

pctc_status_t pctc_embed(const pctc_embed_t* p, const int32_t* tokens, const void* W, const float* row_scales, void* out,
                         void* stream_v) {
  const pctc_status_t st = check_embed(p);
  if (st != PCTC_OK) return st;
  if (p->dtype_w != PCTC_BF16 && p->dtype_w != PCTC_FP32 && p->dtype_w != PCTC_INT8) return PCTC_ERR_UNSUPPORTED;
  if (p->dtype_x != PCTC_BF16 && p->dtype_x != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
  if ((p->dtype_w == PCTC_INT8) != (row_scales != nullptr)) return PCTC_ERR_INVALID_ARG;
  if (p->M == 0) return PCTC_OK;
  const size_t ws = size_of(p->dtype_w), xs = size_of(p->dtype_x);
  if (!tokens || !W || !out || ((size_t)tokens & 3) || ((size_t)row_scales & 3) || ((size_t)W & (ws - 1)) || ((size_t)out & (xs - 1)))
    return PCTC_ERR_INVALID_ARG;
  const Rows to{out, p->M, p->ld_x, p->D, xs};
  if (to.overlaps(Rows{W, p->V, p->ld_w, p->D, ws}) || to.overlaps(Rows{tokens, 1, p->M, p->M, 4}) ||
      to.overlaps(Rows{row_scales, 1, p->V, p->V, 4}))
    return PCTC_ERR_INVALID_ARG;
  EmbedArgs a = {};
  a.tokens = tokens;
  a.W = W;
  a.row_scales = row_scales;
  a.out = out;
  a.M = p->M; a.V = p->V; a.D = p->D;
  a.ld_w = p->ld_w;
  a.ld_out = p->ld_x;
  a.scale = p->scale;
  cudaStream_t stream = (cudaStream_t)stream_v;
  return status_of(p->dtype_w == PCTC_BF16   ? embed_launch<__nv_bfloat16>(a, p->dtype_x, stream)
                   : p->dtype_w == PCTC_FP32 ? embed_launch<float>(a, p->dtype_x, stream)
                                             : embed_launch<signed char>(a, p->dtype_x, stream));
}

pctc_status_t pctc_embed_grad_workspace_bytes(const pctc_embed_t* p, size_t* bytes_out) {
  if (!bytes_out) return PCTC_ERR_INVALID_ARG;
  const pctc_status_t st = check_embed(p);
  if (st != PCTC_OK) return st;
  *bytes_out = grad_plan(p).total;
  return PCTC_OK;
}

pctc_status_t pctc_embed_grad(const pctc_embed_t* p, const int32_t* tokens, const void* grad, void* dW, void* workspace,
                              size_t workspace_bytes, void* stream_v) {
  const pctc_status_t st = check_embed(p);
  if (st != PCTC_OK) return st;
  for (const int32_t t : {p->dtype_w, p->dtype_x})
    if (t != PCTC_BF16 && t != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
  if (p->M == 0 && p->accumulate) return PCTC_OK;
  const size_t ws = size_of(p->dtype_w), xs = size_of(p->dtype_x);
  if (!dW || ((size_t)dW & (ws - 1)) || !workspace || ((size_t)workspace & (EMBED_ALIGN - 1))) return PCTC_ERR_INVALID_ARG;
  if (p->M > 0 && (!tokens || !grad || ((size_t)tokens & 3) || ((size_t)grad & (xs - 1)))) return PCTC_ERR_INVALID_ARG;
  const GradPlan g = grad_plan(p);
  if (workspace_bytes < g.total) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  const Rows to{dW, p->V, p->ld_w, p->D, ws}, own{workspace, 1, (long long)g.total, (long long)g.total, 1},
      from{grad, p->M, p->ld_x, p->D, xs}, ids{tokens, 1, p->M, p->M, 4};
  if (to.overlaps(from) || to.overlaps(ids) || to.overlaps(own) || own.overlaps(from) || own.overlaps(ids)) return PCTC_ERR_INVALID_ARG;

  cudaStream_t stream = (cudaStream_t)stream_v;
  char* w = (char*)workspace;
  const int group = group_of(grad, p->ld_x, xs, dW, p->ld_w, ws, p->D);
  cudaError_t e;
  if (p->M <= GRAD_FEW) {
    const FewArgs a{tokens, grad, dW, p->ld_x, p->ld_w, p->V, p->D, (int)p->M, p->accumulate, p->scale, {}};
    if (p->dtype_x == PCTC_BF16)
      e = p->dtype_w == PCTC_BF16 ? few_launch<__nv_bfloat16, __nv_bfloat16>(a, group, stream) : few_launch<__nv_bfloat16, float>(a, group, stream);
    else
      e = p->dtype_w == PCTC_BF16 ? few_launch<float, __nv_bfloat16>(a, group, stream) : few_launch<float, float>(a, group, stream);
    return status_of(e);
  }
  const long long width = (p->V + SORT_BUCKETS - 1) / SORT_BUCKETS;
  SortArgs s = {};
  s.tokens = tokens;
  s.M = (int)p->M;
  s.V = p->V;
  s.width = (int)(width < SORT_MAX_WIDTH ? width : SORT_MAX_WIDTH);
  s.sorted = (int2*)(w + g.sorted);
  s.first = (int*)(w + g.first);
  s.clear = (int*)(w + g.arrived);
  s.n_clear = g.windows * 2 * (p->D / group);
  const int smem = SORT_WARPS * s.width * 4;
  static std::atomic<bool> configured[MAX_DEVICES];
  const int dev = current_device();
  if (!configured[dev].load(std::memory_order_acquire)) {
    e = cudaFuncSetAttribute(k_sort_tokens, cudaFuncAttributeMaxDynamicSharedMemorySize, SORT_WARPS * SORT_MAX_WIDTH * 4);
    if (e != cudaSuccess) return PCTC_ERR_CUDA;
    configured[dev].store(true, std::memory_order_release);
  }
  s.buckets = (unsigned)((p->V + s.width - 1) / s.width);
  if (!p->accumulate) s.zero = zero_args(dW, p->V, p->D, p->ld_w, ws, 1);
  const long long blocks = s.buckets + s.zero.pieces;
  if (blocks > 0x7fffffffLL) return PCTC_ERR_UNSUPPORTED;
  k_sort_tokens<<<(unsigned)blocks, SORT_THREADS, smem, stream>>>(s);
  e = cudaGetLastError();
  if (e != cudaSuccess) return PCTC_ERR_CUDA;

  GradArgs a = {};
  a.g = grad;
  a.dW = dW;
  a.sorted = s.sorted;
  a.first = s.first;
  a.part = (float*)(w + g.part);
  a.arrived = s.clear;
  a.ld_g = p->ld_x;
  a.ld_w = p->ld_w;
  a.M = p->M;
  a.windows = g.windows;
  a.window = g.window;
  a.scale = p->scale;
  if (p->dtype_x == PCTC_BF16)
    e = p->dtype_w == PCTC_BF16 ? grad_launch<__nv_bfloat16, __nv_bfloat16>(a, p->D, group, p->accumulate != 0, stream)
                                : grad_launch<__nv_bfloat16, float>(a, p->D, group, p->accumulate != 0, stream);
  else
    e = p->dtype_w == PCTC_BF16 ? grad_launch<float, __nv_bfloat16>(a, p->D, group, p->accumulate != 0, stream)
                                : grad_launch<float, float>(a, p->D, group, p->accumulate != 0, stream);
  return status_of(e);
}

}  // extern "C"
