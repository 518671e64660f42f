// CTC prefix beam search over the k best classes of every frame.
//
// A slot holds a prefix x (a label sequence) with pb, the probability of all alignments of the frames so far
// that collapse to x and end in blank, and pn, of those that end in x's last label.  One frame with class
// probabilities p (classes not among its k count as impossible):
//   total = pb + pn
//   stay:       pb' = total * p[blank],   pn' = pn * p[last(x)]
//   grow by c:  pn'(x c) = (c == last(x) ? pb : total) * p[c]      for c != blank
// where a grown prefix that another slot already holds is added to that slot's pn' and is no candidate of
// its own.  The `beams` candidates with the largest pb' + pn' go on; equal ones in the order stays by
// slot, then r * k + j of the grown ones.
//
// The arithmetic is linear in the probabilities, in 64 bits: two products and at most two sums a value and
// frame, no logarithms in the chain of frames.  p is exp(logprob - the frame's largest logprob), so the best
// class has p = 1, rounded to 24 significant bits: that is what the fp32 input carries, and it makes every
// later operation an IEEE product or sum of the same bits whoever computes exp (candidates that tie by
// symmetry then tie everywhere).  Classes under exp(-700) of the frame's best count as absent.  Every 16
// frames all values are scaled by a power of two; what falls under 2^-1022 of the best is dropped.
#include "../../include/prunedctc.h"
#include "pctc_internal.h"

#include <math_constants.h>

namespace pctc {
namespace {

constexpr int PFX_MAX_BEAMS = 32, PFX_MAX_K = 32;
constexpr int PFX_RESCALE = 16;                   // frames between rescalings: values move by at most 3^16
constexpr int PFX_TILE = 32;                      // frames whose probabilities are staged at a time
constexpr int PFX_THREADS = 128;
constexpr int PFX_SLICE = 1024;                   // utterances whose lengths one launch takes as a parameter

struct Slots {
  double pb[PFX_MAX_BEAMS], pn[PFX_MAX_BEAMS];
  unsigned long long hash[PFX_MAX_BEAMS];         // of the prefix
  unsigned long long up[PFX_MAX_BEAMS];           // of the prefix without its last label
  int last[PFX_MAX_BEAMS], size[PFX_MAX_BEAMS], node[PFX_MAX_BEAMS];
};
struct PrefixState {                              // one utterance, between calls
  unsigned magic;
  int beams, max_frames, frames, flags, power;
  double shift;                                   // log scale: shift + power * ln 2
  Slots s;
};
constexpr unsigned PFX_MAGIC = 0x70667831u;
constexpr size_t PFX_STATE_BYTES = (sizeof(PrefixState) + 255) / 256 * 256;

struct Lengths { int n[PFX_SLICE]; };

__host__ __device__ inline size_t nodes_per_utt(int beams, int max_frames) { return 1 + (size_t)beams * max_frames; }

// Hash of the prefix x c from that of x.  Two prefixes of one size are taken for equal when their 64-bit
// hashes are (the finaliser of SplitMix64, Steele et al. 2014, over a sum of the parts): a false match among
// the at most 32 x 32 pairs of a frame has probability 2^-54, 1e-11 over a million frames.
__device__ __forceinline__ unsigned long long grow_hash(unsigned long long h, int c) {
  unsigned long long z = h + 0x9e3779b97f4a7c15ull * (unsigned long long)(c + 1);
  z = (z ^ (z >> 30)) * 0xbf58476d1ce4e5b9ull;
  z = (z ^ (z >> 27)) * 0x94d049bb133111ebull;
  return z ^ (z >> 31);
}

__device__ __forceinline__ double round24(double p) {
  const long long b = __double_as_longlong(p) + (1ll << 28);
  return __longlong_as_double(b & ~((1ll << 29) - 1));
}

struct Tile {                                     // staged frames
  double p[PFX_TILE][PFX_MAX_K];
  int cls[PFX_TILE][PFX_MAX_K];                   // -2: no class (absent, impossible, second of its kind)
  double blank[PFX_TILE];
  double shift[PFX_TILE];
};

// One warp a frame, one lane a class.
__device__ void stage_frame(Tile& t, int f, const int* cls, const float* lp, int k, int blank, int* flags) {
  const int lane = threadIdx.x & 31;
  const int c = lane < k ? cls[lane] : -1;
  const float v = lane < k ? lp[lane] : -CUDART_INF_F;
  const bool bad = c >= 0 && (isnan(v) || v == CUDART_INF_F);
  bool ok = c >= 0 && isfinite(v);
  const unsigned same = __match_any_sync(0xffffffffu, ok ? c : -1 - lane);
  ok = ok && (same & ((1u << lane) - 1)) == 0;    // a class given twice counts where it stands first
  float top = ok ? v : -CUDART_INF_F;
#pragma unroll
  for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (top == -CUDART_INF_F) top = 0.f;
  const double z = (double)v - (double)top;
  ok = ok && z >= -700.0;
  const double p = ok ? round24(exp(z)) : 0.0;
  const unsigned isb = __ballot_sync(0xffffffffu, ok && c == blank);
  const double pbl = __shfl_sync(0xffffffffu, p, isb ? __ffs(isb) - 1 : 0);
  if (lane < k) {
    t.p[f][lane] = p;
    t.cls[f][lane] = ok ? c : -2;
  }
  if (lane == 0) {
    t.blank[f] = isb ? pbl : 0.0;
    t.shift[f] = (double)top;
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(flags, PCTC_UTT_NONFINITE);
}

__global__ void __launch_bounds__(PFX_THREADS) k_prefix_advance(
    const int* __restrict__ classes, const float* __restrict__ logprobs, const __grid_constant__ Lengths len, int n0,
    int T, int k, int B, int blank, int max_frames, int fresh, char* __restrict__ states, int2* __restrict__ nodes) {
  __shared__ Tile tile;
  __shared__ Slots buf[2];
  __shared__ double key[PFX_MAX_BEAMS * (PFX_MAX_K + 1)];
  __shared__ double new_b[PFX_MAX_BEAMS], new_n[PFX_MAX_BEAMS];
  __shared__ unsigned taken[PFX_MAX_BEAMS];
  __shared__ int flags;
  const int n = n0 + blockIdx.x, tid = threadIdx.x, warp = tid >> 5;
  const int Tn = len.n[blockIdx.x];
  PrefixState* st = (PrefixState*)(states + (size_t)n * PFX_STATE_BYTES);
  int2* my_nodes = nodes + (size_t)n * nodes_per_utt(B, max_frames);
  int frames0 = 0, power = 0;
  double shift = 0.0;
  if (fresh) {
    if (tid < B) {
      buf[0].pb[tid] = tid == 0 ? 1.0 : 0.0;
      buf[0].pn[tid] = 0.0;
      buf[0].hash[tid] = buf[0].up[tid] = 0;
      buf[0].last[tid] = -1;
      buf[0].size[tid] = buf[0].node[tid] = 0;
    }
    if (tid == 0) { flags = 0; my_nodes[0] = make_int2(-1, -1); }
  } else {
    // a state that was not started with these sizes, or has no room for the frames, takes nothing
    if (st->magic != PFX_MAGIC || st->beams != B || st->max_frames != max_frames || st->frames < 0 ||
        st->frames > max_frames - Tn) {
      if (tid == 0) atomicOr(&st->flags, PCTC_UTT_STATE_FULL);
      return;
    }
    frames0 = st->frames;
    power = st->power;
    shift = st->shift;
    for (int i = tid; i < (int)(sizeof(Slots) / 4); i += PFX_THREADS) ((int*)&buf[0])[i] = ((const int*)&st->s)[i];
    if (tid == 0) flags = st->flags;
  }
  __syncthreads();
  const int nc = B * (k + 1);
  int cur = 0;
  for (int t0 = 0; t0 < Tn; t0 += PFX_TILE) {
    const int nf = Tn - t0 < PFX_TILE ? Tn - t0 : PFX_TILE;
    for (int f = warp; f < nf; f += PFX_THREADS / 32) {
      const size_t at = ((size_t)n * T + t0 + f) * k;
      stage_frame(tile, f, classes + at, logprobs + at, k, blank, &flags);
    }
    __syncthreads();
    for (int f = 0; f < nf; ++f) {
      Slots& a = buf[cur];
      Slots& b = buf[cur ^ 1];
      const int frame = frames0 + t0 + f;
      if (tid < B) taken[tid] = 0;
      __syncthreads();
      if (tid < B) {
        const int last = a.last[tid];
        const double total = __dadd_rn(a.pb[tid], a.pn[tid]);
        int jl = -1;
        for (int j = 0; j < k; ++j)
          if (tile.cls[f][j] == last) jl = j;
        const double pl = jl >= 0 ? tile.p[f][jl] : 0.0;
        const double sb = __dmul_rn(total, tile.blank[f]);
        double sn = __dmul_rn(a.pn[tid], pl);
        if (jl >= 0 && total > 0.0) {
          for (int r = 0; r < B; ++r) {
            const double rt = __dadd_rn(a.pb[r], a.pn[r]);
            if (rt > 0.0 && a.hash[r] == a.up[tid] && a.size[r] + 1 == a.size[tid]) {
              sn = __dadd_rn(sn, __dmul_rn(a.last[r] == last ? a.pb[r] : rt, pl));
              atomicOr(&taken[r], 1u << jl);
              break;
            }
          }
        }
        new_b[tid] = sb;
        new_n[tid] = sn;
        key[tid] = __dadd_rn(sb, sn);
        b.pb[tid] = b.pn[tid] = 0.0;
        b.hash[tid] = b.up[tid] = 0;
        b.last[tid] = -1;
        b.size[tid] = b.node[tid] = 0;
      }
      __syncthreads();
      for (int i = tid; i < B * k; i += PFX_THREADS) {
        const int r = i / k, j = i % k, c = tile.cls[f][j];
        double v = 0.0;
        if (c >= 0 && c != blank && !((taken[r] >> j) & 1))
          v = __dmul_rn(c == a.last[r] ? a.pb[r] : __dadd_rn(a.pb[r], a.pn[r]), tile.p[f][j]);
        key[B + i] = v;
      }
      __syncthreads();
      for (int i = tid; i < nc; i += PFX_THREADS) {
        const double v = key[i];
        if (!(v > 0.0)) continue;
        int rank = 0;
        for (int m = 0; m < nc; ++m) rank += key[m] > v || (key[m] == v && m < i);
        if (rank >= B) continue;
        if (i < B) {
          b.pb[rank] = new_b[i];
          b.pn[rank] = new_n[i];
          b.hash[rank] = a.hash[i];
          b.up[rank] = a.up[i];
          b.last[rank] = a.last[i];
          b.size[rank] = a.size[i];
          b.node[rank] = a.node[i];
        } else {
          const int r = (i - B) / k, c = tile.cls[f][(i - B) % k];
          const int node = 1 + frame * B + rank;
          b.pb[rank] = 0.0;
          b.pn[rank] = v;
          b.hash[rank] = grow_hash(a.hash[r], c);
          b.up[rank] = a.hash[r];
          b.last[rank] = c;
          b.size[rank] = a.size[r] + 1;
          b.node[rank] = node;
          my_nodes[node] = make_int2(a.node[r], c);
        }
      }
      __syncthreads();
      if (frame % PFX_RESCALE == PFX_RESCALE - 1) {
        const double top = __dadd_rn(b.pb[0], b.pn[0]);
        const int e = top > 0.0 ? (int)((__double_as_longlong(top) >> 52) & 0x7ff) - 1022 : 0;
        const double s = __longlong_as_double((long long)(1023 - e) << 52);
        power += e;
        __syncthreads();
        if (tid < B) {
          b.pb[tid] = __dmul_rn(b.pb[tid], s);
          b.pn[tid] = __dmul_rn(b.pn[tid], s);
        }
        __syncthreads();
      }
      shift += tile.shift[f];
      cur ^= 1;
    }
    __syncthreads();
  }
  for (int i = tid; i < (int)(sizeof(Slots) / 4); i += PFX_THREADS) ((int*)&st->s)[i] = ((const int*)&buf[cur])[i];
  if (tid == 0) {
    st->magic = PFX_MAGIC;
    st->beams = B;
    st->max_frames = max_frames;
    st->frames = frames0 + Tn;
    st->power = power;
    st->shift = shift;
    st->flags = flags;
  }
}

// The hypotheses of a state: every slot's labels from its chain of nodes, last label first.
__global__ void __launch_bounds__(PFX_THREADS) k_prefix_read(
    const char* __restrict__ states, const int2* __restrict__ nodes, int B, int max_frames, int stride,
    int* __restrict__ tokens, int* __restrict__ sizes, float* __restrict__ scores, int* __restrict__ flags) {
  const int n = blockIdx.x, tid = threadIdx.x;
  const PrefixState* st = (const PrefixState*)(states + (size_t)n * PFX_STATE_BYTES);
  const int2* my_nodes = nodes + (size_t)n * nodes_per_utt(B, max_frames);
  const bool valid = st->magic == PFX_MAGIC && st->beams == B && st->max_frames == max_frames;
  for (int b = 0; b < B; ++b) {
    const bool live = valid && st->s.pb[b] + st->s.pn[b] > 0.0;
    const int size = live ? st->s.size[b] : 0;
    for (int i = size + tid; i < stride; i += PFX_THREADS) tokens[((size_t)n * B + b) * stride + i] = -1;
  }
  if (tid < B) {
    const double total = valid ? st->s.pb[tid] + st->s.pn[tid] : 0.0;
    const int size = total > 0.0 ? st->s.size[tid] : 0;
    int node = total > 0.0 ? st->s.node[tid] : 0;
    int* out = tokens + ((size_t)n * B + tid) * stride;
    for (int i = size - 1; i >= 0 && node > 0 && node < (int)nodes_per_utt(B, max_frames); --i) {
      const int2 v = my_nodes[node];
      if (i < stride) out[i] = v.y;
      if (v.x >= node) break;                     // nodes are made after their parents
      node = v.x;
    }
    sizes[n * B + tid] = size;
    scores[n * B + tid] = total > 0.0 ? (float)(log(total) + st->power * 0.693147180559945309417 + st->shift)
                                      : -CUDART_INF_F;
  }
  if (tid == 0 && flags) {
    bool any = false;
    for (int b = 0; b < B && valid; ++b) any = any || st->s.pb[b] + st->s.pn[b] > 0.0;
    flags[n] = valid ? st->flags | (any ? 0 : PCTC_UTT_INFEASIBLE) : PCTC_UTT_STATE_FULL;
  }
}

pctc_status_t check(const pctc_prefix_t* p) {
  if (!p) return PCTC_ERR_INVALID_ARG;
  if (p->N <= 0 || p->T <= 0 || p->k <= 0 || p->beams <= 0 || p->max_frames <= 0 || p->blank_id < 0)
    return PCTC_ERR_INVALID_ARG;
  if (p->k > PFX_MAX_K || p->beams > PFX_MAX_BEAMS) return PCTC_ERR_UNSUPPORTED;
  if ((long long)p->max_frames * p->beams >= 0x7fffffffLL) return PCTC_ERR_UNSUPPORTED;
  return PCTC_OK;
}
size_t state_bytes(const pctc_prefix_t* p) {
  return p->N * (PFX_STATE_BYTES + nodes_per_utt(p->beams, p->max_frames) * sizeof(int2));
}

}  // namespace
}  // namespace pctc

using namespace pctc;

extern "C" {

pctc_status_t pctc_prefix_state_bytes(const pctc_prefix_t* p, size_t* bytes_out) {
  const pctc_status_t st = check(p);
  if (st != PCTC_OK) return st;
  if (!bytes_out) return PCTC_ERR_INVALID_ARG;
  *bytes_out = state_bytes(p);
  return PCTC_OK;
}

pctc_status_t pctc_prefix_advance(const pctc_prefix_t* p, const int32_t* classes, const float* logprobs,
                                  const int32_t* lengths, int32_t fresh, void* state, size_t bytes, void* stream_v) {
  const pctc_status_t st = check(p);
  if (st != PCTC_OK) return st;
  if (!classes || !logprobs || !lengths || !state || ((size_t)state & 255) || (fresh & ~1)) return PCTC_ERR_INVALID_ARG;
  if (((size_t)classes & 3) || ((size_t)logprobs & 3)) return PCTC_ERR_INVALID_ARG;
  for (int n = 0; n < p->N; ++n)
    if (lengths[n] < 0 || lengths[n] > p->T || lengths[n] > p->max_frames) return PCTC_ERR_INVALID_ARG;
  if (bytes < state_bytes(p)) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  int2* nodes = (int2*)((char*)state + (size_t)p->N * PFX_STATE_BYTES);
  for (int n0 = 0; n0 < p->N; n0 += PFX_SLICE) {
    Lengths len;
    const int m = p->N - n0 < PFX_SLICE ? p->N - n0 : PFX_SLICE;
    for (int i = 0; i < m; ++i) len.n[i] = lengths[n0 + i];
    k_prefix_advance<<<m, PFX_THREADS, 0, (cudaStream_t)stream_v>>>(classes, logprobs, len, n0, p->T, p->k, p->beams,
                                                                    p->blank_id, p->max_frames, fresh, (char*)state, nodes);
    if (cudaGetLastError() != cudaSuccess) return PCTC_ERR_CUDA;
  }
  return PCTC_OK;
}

pctc_status_t pctc_prefix_read(const pctc_prefix_t* p, const void* state, size_t bytes, int32_t* tokens,
                               int32_t token_stride, int32_t* token_lengths, float* scores, int32_t* utt_flags,
                               void* stream_v) {
  const pctc_status_t st = check(p);
  if (st != PCTC_OK) return st;
  if (!state || ((size_t)state & 255) || !tokens || token_stride <= 0 || !token_lengths || !scores)
    return PCTC_ERR_INVALID_ARG;
  if (bytes < state_bytes(p)) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  const int2* nodes = (const int2*)((const char*)state + (size_t)p->N * PFX_STATE_BYTES);
  k_prefix_read<<<p->N, PFX_THREADS, 0, (cudaStream_t)stream_v>>>((const char*)state, nodes, p->beams, p->max_frames,
                                                                  token_stride, tokens, token_lengths, scores, utt_flags);
  return cudaGetLastError() == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
}

}  // extern "C"
