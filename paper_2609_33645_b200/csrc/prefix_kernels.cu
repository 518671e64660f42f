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
constexpr int PFX_LAST_WINDOW = 2560;             // nodes of a window where the search itself reads its hypotheses out
constexpr int PFX_SLICE = 1024;                   // utterances whose lengths one launch takes as a parameter

struct Slots {
  double pb[PFX_MAX_BEAMS], pn[PFX_MAX_BEAMS];
  unsigned long long hash[PFX_MAX_BEAMS];         // of the prefix
  unsigned long long up[PFX_MAX_BEAMS];           // of the prefix without its last label
  int last[PFX_MAX_BEAMS], size[PFX_MAX_BEAMS], node[PFX_MAX_BEAMS];
  int par[PFX_MAX_BEAMS];                         // slot of the prefix without its last label, or -1
};
struct PrefixState {                              // one utterance, between calls
  unsigned magic;
  int utts, beams, max_frames, frames, flags, power;
  double shift;                                   // log scale: shift + power * ln 2
  Slots s;
};
constexpr unsigned PFX_MAGIC = 0x70667832u;
constexpr size_t PFX_STATE_BYTES = (sizeof(PrefixState) + 255) / 256 * 256;

struct Lengths { int n[PFX_SLICE]; };

// Whether the state that begins at `states` was started for these sizes.  The first utterance's tells: where the
// others lie does not depend on the sizes, but what lies there does.
__device__ __forceinline__ bool started_for(const char* states, int N, int B, int max_frames) {
  const PrefixState* first = (const PrefixState*)states;
  return first->magic == PFX_MAGIC && first->utts == N && first->beams == B && first->max_frames == max_frames;
}

__host__ __device__ inline size_t nodes_per_utt(int beams, int max_frames) { return 1 + (size_t)beams * max_frames; }

// Hash of the prefix x c from that of x: two 32-bit halves, each a bijection of the half for a given label (additions,
// exclusive ors, shifts and odd factors from the square roots of 2, 3, 5 and 7), short because the search waits for it.
// Prefixes of different hashes are different; those of equal ones are compared label by label (same_prefix): pairs that
// differ can be solved for, and among the two-label prefixes over 2^18 labels there is one.
__device__ __forceinline__ unsigned long long grow_hash(unsigned long long h, int c) {
  unsigned lo = ((unsigned)h + (unsigned)c + 1u) * 0x6a09e667u, hi = ((unsigned)(h >> 32) ^ ((unsigned)c + 1u)) * 0xbb67ae85u;
  lo = (lo ^ (lo >> 15)) * 0x3c6ef373u;
  hi = (hi ^ (hi >> 13)) * 0xa54ff53bu;
  return (unsigned long long)hi << 32 | lo;
}

// Whether two nodes stand for the same labels.  Their chains mostly meet after a step or two: a prefix that comes back
// is grown from the node that it was grown from before.
__device__ __forceinline__ bool same_prefix(const int2* nodes, int x, int y) {
  while (x != y) {
    if (x <= 0 || y <= 0) return false;           // one of them is the empty prefix
    const int2 u = nodes[x], v = nodes[y];
    if (u.y != v.y || u.x >= x || v.x >= y) return false;      // nodes are made after their parents
    x = u.x;
    y = v.x;
  }
  return true;
}

__device__ __forceinline__ double round24(double p) {
  const long long b = __double_as_longlong(p) + (1ll << 28);
  return __longlong_as_double(b & ~((1ll << 29) - 1));
}

// Where hypotheses go.
struct Hypotheses {
  int* tokens;                                    // [N, B, stride]; null: nowhere
  int* sizes;
  float* scores;
  int* flags;                                     // or null
  int stride;
};
template <int WINDOW>
struct ReadShared {
  int2 window[WINDOW];
  int newest, oldest, size[PFX_MAX_BEAMS];
};

// The hypotheses of a state: every slot's labels from its chain of nodes, last label first.  A chain is
// as long as the hypothesis, and a node read from L2 a step would cost 0.3 us; nodes are numbered by frame, so the
// table is taken through shared memory in windows from the last frame to the first, and all chains of an
// utterance walk through a window before the next one is fetched.  Called by all threads of a CTA.
template <int THREADS, int WINDOW>
__device__ void read_out(ReadShared<WINDOW>& sh, bool valid, const PrefixState* st, const int2* my_nodes, int n, int B,
                         int max_frames, const Hypotheses& h) {
  const int tid = threadIdx.x;
  const int most = (int)nodes_per_utt(B, max_frames);
  if (tid == 0) sh.newest = 0;
  __syncthreads();
  int at = 0, node = 0;
  int* out = nullptr;
  bool live = false;
  if (tid < B) {
    const double total = valid ? st->s.pb[tid] + st->s.pn[tid] : 0.0;
    live = total > 0.0;
    at = live ? st->s.size[tid] : 0;
    node = live ? st->s.node[tid] : 0;
    if (node < 0 || node >= most) node = 0;
    out = h.tokens + ((size_t)n * B + tid) * h.stride;
    sh.size[tid] = at;
    h.sizes[n * B + tid] = at;
    h.scores[n * B + tid] = live ? (float)(log(total) + st->power * 0.693147180559945309417 + st->shift) : -CUDART_INF_F;
    atomicMax(&sh.newest, node);
  }
  const bool any = __syncthreads_or(live);
  if (tid == 0 && h.flags) h.flags[n] = valid ? st->flags | (any ? 0 : PCTC_UTT_INFEASIBLE) : PCTC_UTT_STATE_FULL;
  for (int b = 0; b < B; ++b)
    for (int i = sh.size[b] + tid; i < h.stride; i += THREADS) h.tokens[((size_t)n * B + b) * h.stride + i] = -1;
  for (int hi = sh.newest + 1; hi > 1;) {         // nodes [lo, hi); node 0 is the empty prefix
    const int lo = max(1, hi - WINDOW);
    for (int i = tid; i < hi - lo; i += THREADS) sh.window[i] = my_nodes[lo + i];
    if (tid == 0) sh.oldest = 0;
    __syncthreads();
    if (tid < B) {
      while (node >= lo && at > 0) {
        const int2 v = sh.window[node - lo];
        if (--at < h.stride) out[at] = v.y;
        node = v.x >= 0 && v.x < node ? v.x : 0;  // nodes are made after their parents
      }
      atomicMax(&sh.oldest, at > 0 ? node : 0);   // the newest node that is still to be read
    }
    __syncthreads();
    hi = min(lo, sh.oldest + 1);
    __syncthreads();
  }
}

// Frames staged for the search: KM >= k classes a frame.  The blank stands in `blank` only; what does not count
// (absent, impossible, the second of its kind, behind k) has class -2 and probability 0.
template <int KM>
struct Tile {
  __align__(16) double p[PFX_TILE][KM];
  __align__(16) int cls[PFX_TILE][KM];
  double blank[PFX_TILE];
  double shift[PFX_TILE];
};

// Stages frames f0, f0 + step, ... of a tile: KM lanes a frame.
template <int KM>
__device__ __forceinline__ void stage(Tile<KM>& t, int nf, int warp, int warps, const int* cls, const float* lp, int k,
                                      int blank, int* flags) {
  constexpr int PER = 32 / KM;
  const int lane = threadIdx.x & 31, j = lane % KM, sub = lane / KM;
  for (int f0 = warp * PER; f0 < nf; f0 += warps * PER) {
    const int f = f0 + sub;
    const bool in = f < nf && j < k;
    const int c = in ? cls[(size_t)f * k + j] : -1;
    const float v = in ? lp[(size_t)f * k + j] : -CUDART_INF_F;
    const bool bad = c >= 0 && (isnan(v) || v == CUDART_INF_F);
    bool ok = c >= 0 && isfinite(v);
    const int mine = ok ? c : -1 - lane;
    bool again = false;                           // a class given twice counts where it stands first
#pragma unroll
    for (int d = 1; d < KM; ++d) {
      const int o = __shfl_up_sync(0xffffffffu, mine, d, KM);
      again = again || (j >= d && o == mine);
    }
    ok = ok && !again;
    float top = ok ? v : -CUDART_INF_F;
#pragma unroll
    for (int o = KM / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o, KM));
    if (top == -CUDART_INF_F) top = 0.f;
    const double z = (double)v - (double)top;
    ok = ok && z >= -700.0;
    const double p = ok ? round24(exp(z)) : 0.0;
    const bool is_blank = ok && c == blank;
    if (f < nf) {
      t.p[f][j] = is_blank ? 0.0 : p;
      t.cls[f][j] = ok && !is_blank ? c : -2;
    }
    double pbl = is_blank ? p : 0.0;
#pragma unroll
    for (int o = KM / 2; o; o >>= 1) pbl = fmax(pbl, __shfl_xor_sync(0xffffffffu, pbl, o, KM));
    if (f < nf && j == 0) {
      t.blank[f] = pbl;
      t.shift[f] = (double)top;
    }
    if (bad) atomicOr(flags, PCTC_UTT_NONFINITE);
  }
}

// Order of non-negative doubles up to ties: the upper word, at least 1 for what is not zero.
__device__ __forceinline__ unsigned coarse(double x) {
  const unsigned h = (unsigned)__double2hiint(x);
  return h == 0 && x > 0.0 ? 1u : h;
}

// A lane's share of a frame: classes first, first + 1, ... (first a multiple of KP), and the blank.
template <int KP>
struct Share {
  double p[KP], blank;
  int cls[KP];
  template <int KM>
  __device__ __forceinline__ void load(const Tile<KM>& t, int f, int first) {
    if constexpr (KP % 4 == 0) {
#pragma unroll
      for (int q = 0; q < KP; q += 4) {
        const int4 c = *(const int4*)&t.cls[f][first + q];
        cls[q] = c.x; cls[q + 1] = c.y; cls[q + 2] = c.z; cls[q + 3] = c.w;
      }
    } else {
#pragma unroll
      for (int q = 0; q < KP; ++q) cls[q] = t.cls[f][first + q];
    }
#pragma unroll
    for (int q = 0; q < KP; q += 2) {
      const double2 d = *(const double2*)&t.p[f][first + q];
      p[q] = d.x; p[q + 1] = d.y;
    }
    blank = t.blank[f];
  }
};

template <int KM, int BM>
struct Search {                                   // what lanes hand each other within a frame
  // coarse keys: BM stays, then (at first) every slot's best extension, then the extensions that are ranked; 16 of padding
  __align__(16) unsigned key[BM + (KM > 1 ? KM : 1) * BM + 16];
  double value[KM * BM];                          // of the extensions that are ranked ...
  int2 from[KM * BM];                             // ... and 32 + slot * 32 + class number, and the class
  double stay[BM];
  double slot_value[32];                          // by new slot
  int2 slot_from[32];
  unsigned taken[32];
  __align__(16) unsigned grown[BM];               // lower words of the hashes of prefixes that have just been grown, else 0
};

// One CTA an utterance: warp 0 searches while the other warps stage the next frames.  The search is a chain of
// dependent frames, so what counts is its latency: a slot lives in registers of a lane, lanes talk by shuffles and a
// few words of shared memory, and the only barrier is one per 32 frames.  BM >= B slots; with fewer than 32 every
// slot is held by 32 / BM lanes alike, which share its classes.
// Candidates are ranked by counting, in two steps: the B-th largest of the stays and every slot's best extension
// bounds the result from below, and only what reaches the bound is ranked.  Both compare upper words (coarse());
// where two of those tie, the ranks are taken again with all bits and the order of equals.  In most frames of
// speech the blank or the last label takes nearly all, no extension reaches even the worst stay, the stays
// keep their order, and neither step is needed.
// Measured on confusable posteriors, of which a third of the frames are such: 0.65 us a frame at beam 4 and 0.95 us at
// beam 16, k = 8 (8 utterances of up to 1500 frames: 1.42 ms; a CTA of 128 threads with three barriers a frame that
// ranks all candidates: 7.6 ms).  A frame is about 330 dependent instructions at 5 cycles each; shuffles, votes, reductions
// and shared-memory loads take 25 to 45 cycles each.  Taking the B winners one after the other by warp-wide maxima, in
// place of bound and ranks, measured the same at beam 4 and 30% slower at beam 16.
template <int KM, int BM>
__global__ void __launch_bounds__(PFX_THREADS, 1) k_prefix_advance(
    const int* __restrict__ classes, const float* __restrict__ logprobs, const __grid_constant__ Lengths len, int n0,
    int N, int T, int k, int B, int blank, int max_frames, int fresh, char* states, int2* nodes, const Hypotheses out) {
  constexpr unsigned ALL = 0xffffffffu;
  constexpr int REP = 32 / BM, KP = KM / REP;     // lanes a slot, classes a lane
  constexpr unsigned SLOTS = BM == 32 ? ALL : (1u << BM) - 1;
  __shared__ Tile<KM> tiles[2];
  __shared__ Search<KM, BM> sh;
  __shared__ int flags;
  const int n = n0 + blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int slot = lane % BM, part = lane / BM;
  const int Tn = len.n[blockIdx.x];
  PrefixState* st = (PrefixState*)(states + (size_t)n * PFX_STATE_BYTES);
  int2* my_nodes = nodes + (size_t)n * nodes_per_utt(B, max_frames);
  if (!fresh) {
    // a state that was not started with these sizes, or has no room for the frames, takes nothing
    const PrefixState* first = (const PrefixState*)states;
    const bool fits = started_for(states, N, B, max_frames) && st->frames >= 0 && st->frames <= max_frames - Tn;
    if (!fits) {
      // (of a state for fewer utterances there may be something else in this place)
      if (tid == 0 && first->magic == PFX_MAGIC && n < first->utts) atomicOr(&st->flags, PCTC_UTT_STATE_FULL);
      return;
    }
  }
  int frames0 = 0, power = 0;
  double shift = 0.0;
  double pb = 0.0, pn = 0.0;
  unsigned long long hash = 0, up = 0;
  int last = -1, size = 0, node = 0, par = -1;    // par: the slot that holds the prefix without its last label
  if (warp == 0) {
    if (fresh) {
      if (slot == 0) pb = 1.0;
      if (lane == 0) my_nodes[0] = make_int2(-1, -1);
    } else {
      frames0 = st->frames;
      power = st->power;
      shift = st->shift;
      if (slot < B) {
        pb = st->s.pb[slot]; pn = st->s.pn[slot];
        hash = st->s.hash[slot]; up = st->s.up[slot];
        last = st->s.last[slot]; size = st->s.size[slot]; node = st->s.node[slot];
        par = st->s.par[slot];
        // indexes of a state that something else has written to stay in range
        if (node < 0 || node >= (int)nodes_per_utt(B, max_frames)) node = 0;
        if (par < -1 || par >= B) par = -1;
      }
    }
    sh.taken[lane] = 0;
  }
  if (tid == 0) flags = fresh ? 0 : st->flags;
  __syncthreads();
  const int* cls_n = classes + (size_t)n * T * k;
  const float* lp_n = logprobs + (size_t)n * T * k;
  stage<KM>(tiles[0], min(Tn, PFX_TILE), warp, PFX_THREADS / 32, cls_n, lp_n, k, blank, &flags);
  __syncthreads();

  for (int t0 = 0; t0 < Tn; t0 += PFX_TILE) {
    Tile<KM>& tile = tiles[(t0 / PFX_TILE) & 1];
    const int nf = min(Tn - t0, PFX_TILE);
    if (warp > 0) {
      const int t1 = t0 + PFX_TILE;
      if (t1 < Tn)
        stage<KM>(tiles[(t1 / PFX_TILE) & 1], min(Tn - t1, PFX_TILE), warp - 1, PFX_THREADS / 32 - 1,
                  cls_n + (size_t)t1 * k, lp_n + (size_t)t1 * k, k, blank, &flags);
    } else {
      // the next frame's share is on its way while a frame is searched (where the registers allow)
      constexpr bool PREFETCH = KP <= 8;
      Share<KP> now;
      if (PREFETCH) now.load(tile, 0, part * KP);
      for (int f = 0; f < nf; ++f) {
        const int frame = frames0 + t0 + f;
        if (!PREFETCH) now.load(tile, f, part * KP);
        const Share<KP> in = now;
        if (PREFETCH && f + 1 < nf) now.load(tile, f + 1, part * KP);
        // ---- this lane's candidates: its slot's stay, and the slot grown by its share of the classes ----
        const double total = __dadd_rn(pb, pn);
        double v[KP];
        int jl = -1;
        double pl = 0.0;                          // probability of this prefix's last label
#pragma unroll
        for (int q = 0; q < KP; ++q) {
          const bool same = in.cls[q] == last;
          if (same) { jl = part * KP + q; pl = in.p[q]; }
          v[q] = __dmul_rn(same ? pb : total, in.p[q]);
        }
#pragma unroll
        for (int o = BM; o < 32; o *= 2) {
          const int oj = __shfl_xor_sync(ALL, jl, o);
          const double op = __shfl_xor_sync(ALL, pl, o);
          if (oj > jl) { jl = oj; pl = op; }
        }
        const double sb = __dmul_rn(total, in.blank);
        double sn = __dmul_rn(pn, pl);
        const bool child = par >= 0 && jl >= 0 && total > 0.0;
        if (__any_sync(ALL, child)) {             // slot par grown by `last` is this slot's prefix
          const int r = child ? par : lane;
          const int rl = __shfl_sync(ALL, last, r);
          const double rb = __shfl_sync(ALL, pb, r), rt = __shfl_sync(ALL, total, r);
          if (child) {
            sn = __dadd_rn(sn, __dmul_rn(rl == last ? rb : rt, pl));
            atomicOr(&sh.taken[par], 1u << jl);
          }
          __syncwarp();
          const unsigned gone = sh.taken[slot] >> (part * KP);
          __syncwarp();
          sh.taken[lane] = 0;
          __syncwarp();
#pragma unroll
          for (int q = 0; q < KP; ++q)
            if (gone >> q & 1) v[q] = 0.0;
        }
        const double stay = __dadd_rn(sb, sn);
        shift += tile.shift[f];

        unsigned best = 0;
#pragma unroll
        for (int q = 0; q < KP; ++q) best = max(best, coarse(v[q]));
        const unsigned sk = coarse(stay);
        const unsigned worst = __reduce_min_sync(ALL, slot < B ? sk : ALL);
        const bool grows = __any_sync(ALL, best >= worst && best > 0);
        const double ahead = __shfl_up_sync(ALL, stay, 1, BM);
        if (!grows && worst > 0 && __all_sync(ALL, slot == 0 || slot >= B || ahead >= stay)) {
          pb = sb;                                // all stay, in their order
          pn = sn;
        } else {
          // ---- the bound, and the extensions that reach it ----
          int ne = 0;
          if (part == 0) sh.key[slot] = sk;
          if (grows) {
#pragma unroll
            for (int o = BM; o < 32; o *= 2) best = max(best, __shfl_xor_sync(ALL, best, o));
            if (part == REP - 1) sh.key[BM + slot] = best;
            __syncwarp();
            unsigned least;
            if (BM < 32) {
              const unsigned mine = lane < BM ? sk : best;
              int a0 = 0, a1 = 0, a2 = 0, a3 = 0;
#pragma unroll
              for (int i = 0; i < BM / 2; ++i) {
                const uint4 o = ((const uint4*)sh.key)[i];
                a0 += o.x > mine; a1 += o.y > mine; a2 += o.z > mine; a3 += o.w > mine;
              }
              const int above = a0 + a1 + a2 + a3;
              least = __reduce_min_sync(ALL, above < B ? mine : ALL);
            } else {
              int a0 = 0, a1 = 0;
#pragma unroll
              for (int i = 0; i < BM / 2; ++i) {
                const uint4 o = ((const uint4*)sh.key)[i];
                a0 += (o.x > sk) + (o.y > sk) + (o.z > sk) + (o.w > sk);
                a1 += (o.x > best) + (o.y > best) + (o.z > best) + (o.w > best);
              }
              least = __reduce_min_sync(ALL, min(a0 < B ? sk : ALL, a1 < B ? best : ALL));
            }
            least = max(least, 1u);
            int mine = 0;
#pragma unroll
            for (int q = 0; q < KP; ++q) mine += coarse(v[q]) >= least;
            int at = 0;                           // places before this lane's: a scan over the bits of the counts
#pragma unroll
            for (int bit = 1; bit <= KP; bit *= 2) {
              const unsigned m = __ballot_sync(ALL, mine & bit);
              at += bit * __popc(m & ((1u << lane) - 1));
              ne += bit * __popc(m);
            }
            __syncwarp();
#pragma unroll
            for (int q = 0; q < KP; ++q) {
              if (coarse(v[q]) >= least) {
                const int j = part * KP + q;
                sh.key[BM + at] = coarse(v[q]);
                sh.value[at] = v[q];
                sh.from[at] = make_int2(32 + slot * 32 + j, in.cls[q]);
                ++at;
              }
            }
          }
          const int all = BM + ne;
          if (lane < 16) sh.key[all + lane] = 0;
          __syncwarp();

          // ---- ranks among the stays and those extensions; the first B are the new slots ----
          int place = -1;                         // of this lane's stay (lanes below BM)
          int count = 0, sum = 0;
          for (int x0 = 0; x0 < all; x0 += 32) {
            const int x = x0 + lane;
            const unsigned mine = x < all ? sh.key[x] : 0;
            const int e = max(x - BM, 0);
            const bool ext = x >= BM && x < all;
            const double val = ext ? sh.value[e] : 0.0;
            const int2 src = ext ? sh.from[e] : make_int2(lane, 0);
            int r0 = 0, r1 = 0, r2 = 0, r3 = 0;
            for (int y = 0; y < all; y += 16) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint4 o = *(const uint4*)&sh.key[y + 4 * i];
                r0 += o.x > mine; r1 += o.y > mine; r2 += o.z > mine; r3 += o.w > mine;
              }
            }
            const int rank = r0 + r1 + r2 + r3;
            if (mine > 0 && rank < B) {
              sh.slot_value[rank] = val;
              sh.slot_from[rank] = src;
              if (x < BM) place = rank;
            }
            count += __popc(__ballot_sync(ALL, mine > 0));
            sum += __reduce_add_sync(ALL, mine > 0 ? (unsigned)rank : 0u);
          }
          if (sum != count * (count - 1) / 2) {   // ties of upper words: all bits, and the order of equals
            if (part == 0) sh.stay[slot] = stay;
            place = -1;
            __syncwarp();
            for (int x = lane; x < all; x += 32) {
              const double val = x < BM ? sh.stay[x] : sh.value[x - BM];
              const int2 src = x < BM ? make_int2(x, 0) : sh.from[x - BM];
              if (!(val > 0.0)) continue;
              int rank = 0;
              for (int y = 0; y < all; ++y) {
                const double o = y < BM ? sh.stay[y] : sh.value[y - BM];
                rank += o > val || (o == val && (y < BM ? y : sh.from[y - BM].x) < src.x);
              }
              if (rank < B) {
                sh.slot_value[rank] = val;
                sh.slot_from[rank] = src;
                if (x < BM) place = rank;
              }
            }
          }
          __syncwarp();

          // ---- the new slots ----
          const bool live = slot < min(count, B);
          const double value = sh.slot_value[slot];
          const int2 src = live ? sh.slot_from[slot] : make_int2(lane, 0);
          const bool grown = src.x >= 32;
          const int r = grown ? (src.x - 32) >> 5 : src.x;
          const int moved = __shfl_sync(ALL, place, max(par, 0));        // where this slot's parent goes
          const int stay_par = par >= 0 ? moved : -1;
          const int grown_par = __shfl_sync(ALL, place, r);
          par = __shfl_sync(ALL, stay_par, r);
          const double rb = __shfl_sync(ALL, sb, r), rn = __shfl_sync(ALL, sn, r);
          const unsigned long long rh = __shfl_sync(ALL, hash, r), ru = __shfl_sync(ALL, up, r);
          last = __shfl_sync(ALL, last, r);
          size = __shfl_sync(ALL, size, r);
          node = __shfl_sync(ALL, node, r);
          pb = rb;
          pn = rn;
          hash = rh;
          up = ru;
          if (grown) {
            const int parent = node;
            pb = 0.0;
            pn = value;
            hash = grow_hash(rh, src.y);
            up = rh;
            last = src.y;
            size += 1;
            node = 1 + frame * B + slot;
            par = grown_par;
            if (part == 0) my_nodes[node] = make_int2(parent, src.y);
          }
          if (!live) {
            pb = pn = 0.0;
            hash = up = 0;
            last = par = -1;
            size = node = 0;
          }
          // a prefix that had left the beam and is back is the parent of slots that stayed
          const bool orphan = live && par < 0 && size > 0 && !grown;
          const unsigned grew = __ballot_sync(ALL, grown) & SLOTS;
          if (__any_sync(ALL, orphan) && grew) {
            if (part == 0) sh.grown[slot] = grown ? (unsigned)hash : 0u;
            __syncwarp();
            const unsigned low = (unsigned)up;
            int e = -1;
#pragma unroll
            for (int i = 0; i < BM; i += 4) {
              const uint4 h = *(const uint4*)&sh.grown[i];
              if (h.x == low) e = i;
              if (h.y == low) e = i + 1;
              if (h.z == low) e = i + 2;
              if (h.w == low) e = i + 3;
            }
            if (__any_sync(ALL, orphan && e >= 0)) {      // all bits and all labels, one new prefix after the other
              unsigned fresh_slots = grew;
              while (fresh_slots) {
                e = __ffs(fresh_slots) - 1;
                fresh_slots &= fresh_slots - 1;
                const unsigned long long h = __shfl_sync(ALL, hash, e);
                const int come = __shfl_sync(ALL, node, e);
                if (orphan && h == up && same_prefix(my_nodes, my_nodes[node].x, come)) par = e;
              }
            }
          }
        }
        if (frame % PFX_RESCALE == PFX_RESCALE - 1) {
          const double top = __shfl_sync(ALL, __dadd_rn(pb, pn), 0);
          const int e = top > 0.0 ? (int)((unsigned)__double2hiint(top) >> 20 & 0x7ff) - 1022 : 0;
          const double s = __longlong_as_double((long long)(1023 - e) << 52);
          power += e;
          pb = __dmul_rn(pb, s);
          pn = __dmul_rn(pn, s);
        }
      }
    }
    __syncthreads();
  }
  if (warp == 0) {
    if (lane < B) {
      st->s.pb[lane] = pb; st->s.pn[lane] = pn;
      st->s.hash[lane] = hash; st->s.up[lane] = up;
      st->s.last[lane] = last; st->s.size[lane] = size; st->s.node[lane] = node;
      st->s.par[lane] = par;
    }
    if (lane == 0) {
      st->magic = PFX_MAGIC;
      st->utts = N;
      st->beams = B;
      st->max_frames = max_frames;
      st->frames = frames0 + Tn;
      st->power = power;
      st->shift = shift;
      st->flags = flags;
    }
  }
  if constexpr (KM == 8) {                        // whole utterances: the hypotheses, in the same launch
    if (out.tokens) {
      __shared__ ReadShared<PFX_LAST_WINDOW> rd;
      __syncthreads();
      read_out<PFX_THREADS>(rd, true, st, my_nodes, n, B, max_frames, out);
    }
  }
}

constexpr int PFX_READ_THREADS = 256, PFX_READ_WINDOW = 5120;
__global__ void __launch_bounds__(PFX_READ_THREADS) k_prefix_read(const char* __restrict__ states,
                                                                  const int2* __restrict__ nodes, int B, int max_frames,
                                                                  const Hypotheses out) {
  __shared__ ReadShared<PFX_READ_WINDOW> sh;
  const int n = blockIdx.x;
  read_out<PFX_READ_THREADS>(sh, started_for(states, gridDim.x, B, max_frames), (const PrefixState*)(states + (size_t)n * PFX_STATE_BYTES),
                             nodes + (size_t)n * nodes_per_utt(B, max_frames), n, B, max_frames, out);
}

pctc_status_t check(const pctc_prefix_t* p) {
  if (!p) return PCTC_ERR_INVALID_ARG;
  if (p->N <= 0 || p->T <= 0 || p->k <= 0 || p->beams <= 0 || p->max_frames <= 0 || p->blank_id < 0)
    return PCTC_ERR_INVALID_ARG;
  if (p->k > PFX_MAX_K || p->beams > PFX_MAX_BEAMS) return PCTC_ERR_UNSUPPORTED;
  if ((long long)p->max_frames * p->beams >= 0x7fffffffLL) return PCTC_ERR_UNSUPPORTED;
  if ((long long)p->N * p->beams > 0x7fffffffLL) return PCTC_ERR_UNSUPPORTED;      // places of hypotheses are 32 bits
  return PCTC_OK;
}
size_t state_bytes(const pctc_prefix_t* p) {
  return p->N * (PFX_STATE_BYTES + nodes_per_utt(p->beams, p->max_frames) * sizeof(int2));
}

bool bad_outputs(const Hypotheses& h) {
  return !h.tokens || h.stride <= 0 || !h.sizes || !h.scores ||
         (((size_t)h.tokens | (size_t)h.sizes | (size_t)h.scores | (size_t)h.flags) & 3);
}

// Whether something that the call writes overlaps something else that it takes.  Null: not part of the call.
bool overlaps(const pctc_prefix_t* p, const void* classes, const void* logprobs, const void* state, bool advances,
              const Hypotheses& h) {
  Span s[7];
  size_t n = 0;
  auto add = [&](const void* at, size_t bytes, bool write) {
    if (at) s[n++] = Span{(size_t)at, (size_t)at + bytes, write};
  };
  const size_t frames = 4 * (size_t)p->N * p->T * p->k, slots = 4 * (size_t)p->N * p->beams;
  add(classes, frames, false);
  add(logprobs, frames, false);
  add(state, state_bytes(p), advances);
  add(h.tokens, slots * h.stride, true);
  add(h.sizes, slots, true);
  add(h.scores, slots, true);
  add(h.flags, 4 * (size_t)p->N, true);
  return spans_conflict(s, n);
}

// out: what the call returns, if it does; read: in the same launch.
pctc_status_t advance(const pctc_prefix_t* p, const int32_t* classes, const float* logprobs, const int32_t* lengths,
                      int32_t fresh, void* state, size_t bytes, const Hypotheses& out, bool read, void* stream) {
  const pctc_status_t st = check(p);
  if (st != PCTC_OK) return st;
  if (!classes || !logprobs || !lengths || !state || ((size_t)state & 255) || (fresh & ~1)) return PCTC_ERR_INVALID_ARG;
  if (((size_t)classes & 3) || ((size_t)logprobs & 3)) return PCTC_ERR_INVALID_ARG;
  for (int n = 0; n < p->N; ++n)
    if (lengths[n] < 0 || lengths[n] > p->T || lengths[n] > p->max_frames) return PCTC_ERR_INVALID_ARG;
  if (bytes < state_bytes(p)) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  if (overlaps(p, classes, logprobs, state, true, out)) return PCTC_ERR_INVALID_ARG;
  int2* nodes = (int2*)((char*)state + (size_t)p->N * PFX_STATE_BYTES);
  for (int n0 = 0; n0 < p->N; n0 += PFX_SLICE) {
    Lengths len;
    const int m = p->N - n0 < PFX_SLICE ? p->N - n0 : PFX_SLICE;
    for (int i = 0; i < m; ++i) len.n[i] = lengths[n0 + i];
    auto kern = p->k <= 8 ? (p->beams <= 8 ? k_prefix_advance<8, 8> : p->beams <= 16 ? k_prefix_advance<8, 16> : k_prefix_advance<8, 32>)
                          : (p->beams <= 8 ? k_prefix_advance<32, 8> : p->beams <= 16 ? k_prefix_advance<32, 16> : k_prefix_advance<32, 32>);
    kern<<<m, PFX_THREADS, 0, (cudaStream_t)stream>>>(classes, logprobs, len, n0, p->N, p->T, p->k, p->beams, p->blank_id,
                                                      p->max_frames, fresh, (char*)state, nodes, read ? out : Hypotheses{});
    if (cudaGetLastError() != cudaSuccess) return PCTC_ERR_CUDA;
  }
  return PCTC_OK;
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
                                  const int32_t* lengths, int32_t fresh, void* state, size_t bytes, void* stream) {
  return advance(p, classes, logprobs, lengths, fresh, state, bytes, Hypotheses{}, false, stream);
}

pctc_status_t pctc_prefix_read(const pctc_prefix_t* p, const void* state, size_t bytes, int32_t* tokens,
                               int32_t token_stride, int32_t* token_lengths, float* scores, int32_t* utt_flags,
                               void* stream_v) {
  const pctc_status_t st = check(p);
  if (st != PCTC_OK) return st;
  const Hypotheses out{tokens, token_lengths, scores, utt_flags, token_stride};
  if (!state || ((size_t)state & 255) || bad_outputs(out)) return PCTC_ERR_INVALID_ARG;
  if (bytes < state_bytes(p)) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  if (overlaps(p, nullptr, nullptr, state, false, out)) return PCTC_ERR_INVALID_ARG;
  const int2* nodes = (const int2*)((const char*)state + (size_t)p->N * PFX_STATE_BYTES);
  k_prefix_read<<<p->N, PFX_READ_THREADS, 0, (cudaStream_t)stream_v>>>(
      (const char*)state, nodes, p->beams, p->max_frames, out);
  return cudaGetLastError() == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
}

pctc_status_t pctc_prefix_decode(const pctc_prefix_t* p, const int32_t* classes, const float* logprobs,
                                 const int32_t* lengths, void* state, size_t bytes, int32_t* tokens, int32_t token_stride,
                                 int32_t* token_lengths, float* scores, int32_t* utt_flags, void* stream) {
  const Hypotheses out{tokens, token_lengths, scores, utt_flags, token_stride};
  if (bad_outputs(out)) return PCTC_ERR_INVALID_ARG;
  const bool one = p && p->k <= 8;
  const pctc_status_t st = advance(p, classes, logprobs, lengths, 1, state, bytes, out, one, stream);
  if (st != PCTC_OK || one) return st;
  return pctc_prefix_read(p, state, bytes, tokens, token_stride, token_lengths, scores, utt_flags, stream);
}

}  // extern "C"
