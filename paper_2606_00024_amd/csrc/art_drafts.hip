// What surrounds attention in a decode step that verifies drafts: a tree's masks
// and positions (art_tree_layout), the choice of the drafts that are kept
// (art_verify_drafts), and their keys and values moved up to the context's end
// (art_keep_accepted).
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include "art.h"
#include "art_internal.h"
#include "art_rows.h"

namespace art {
namespace {

// ---- a tree's masks and positions ------------------------------------------------

struct LayoutParams {
  int32_t batch, rows, per_seq, words;
  const int32_t* offsets;
  const int32_t* positions;   // contexts, or NULL
  const int32_t* parents;
  uint64_t* mask;
  int32_t* out;
};

// The rows of sequence b within 0 .. rows.
template <class Params>
__device__ __forceinline__ int2 rows_of(const Params& P, int b) {
  int first = P.offsets ? P.offsets[b] : b * P.per_seq, end = P.offsets ? P.offsets[b + 1] : first + P.per_seq;
  first = min(max(first, 0), P.rows);
  end = min(max(end, first), P.rows);
  return make_int2(first, end);
}

// A workgroup to a sequence: its parents in LDS, and every thread walks up from a
// node for one word of its mask.  (A chain of 64 nodes 6 us; 1024 nodes with 16 words:
// trees 44 to 66 us, a chain 2.0 ms, as every word walks the whole path.)
__global__ void __launch_bounds__(kThreads) layout_kernel(const LayoutParams P) {
  __shared__ int s_parent[ART_MAX_NODES];
  const int b = blockIdx.x;
  const int2 span = rows_of(P, b);
  const int n = span.y - span.x, context = P.positions ? P.positions[b] : 0;
  if (n == 0 || n > ART_MAX_NODES || context < 0) return;
  if (P.out && context > INT32_MAX - (n - 1)) return;   // a chain's positions would not be held by 32 bits
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int p = P.parents[span.x + i];
    s_parent[i] = p >= 0 && p < i ? p : -1;
  }
  __syncthreads();
  for (int at = threadIdx.x; at < n * P.words; at += kThreads) {
    const int i = at / P.words, word = at - i * P.words;
    uint64_t bits = 0;
    int depth = -1;
    for (int j = i; j >= 0; j = s_parent[j]) {
      if (j >> 6 == word) bits |= 1ull << (j & 63);
      ++depth;
    }
    P.mask[(int64_t)(span.x + i) * P.words + word] = bits;
    if (word == 0 && P.out) P.out[span.x + i] = context + depth;
  }
}

// ---- verification --------------------------------------------------------------------
//
// With q, the weights after j rejections at a node are max(p - a_j q, 0) / F_j:
// subtracting q from them, clipping at 0 and dividing by the sum again gives the
// same form with a_{j+1} = a_j + F_j, so two numbers are all that a walk carries.
// Only the sums over the vocabulary are work.  A walk needs them one after the
// other, and a chain needs one: at its end.  The first launch walks to the first
// sum that it needs, in every workgroup of a sequence alike (nothing but gathered
// probabilities), and each of them adds up one slice of the vocabulary.  The
// second, one workgroup to a sequence, goes on with that sum in hand and draws the
// token.  A walk's further sums are that workgroup's own: a sampled tree needs one after
// each rejection that leaves siblings and one at the end, a chain and given drafts the
// last alone.  No workgroup ever waits for another.  32 chains of 8 drafts
// against 128000 tokens: 12 and 5.7 us, of which the 33 MB that are read need 6; the rest
// is the chain of dependent loads (offsets, nodes, their probabilities, the rows).  Three
// children of a node, 128000 tokens in fp32, one sequence: 10 us with the first accepted,
// 71 with two or three rejected; 8 sequences 11 and 73, 128 of them 30 and 135.

constexpr int kMaxSlices = 64;
constexpr int kSumThreads = 256;
constexpr int kDrawThreads = 1024;

// Where a walk stands.  It is the same in every lane of the wavefront.
struct Walk {
  double a, f;                 // with q: a and F; without: f is what is left of 1
  int now, count, next;        // the current node, nodes accepted, the first one not tried
  int done;                    // the next token is drawn from the current weights
  int tried;                   // (without q) the current node's children have been rejected
};

struct VerifyParams {
  int32_t batch, rows, per_seq, vocab, max_path, slices;
  int64_t ts, ds;              // row strides in elements
  const void* target;
  const void* draft;
  const int32_t* tokens;
  const int32_t* parents;
  const int32_t* offsets;
  const float* uniforms;
  const float* last;
  int32_t* accepted;
  int32_t* counts;
  int32_t* next;
  double* sums;                // [batch][slices]
  Walk* walks;                 // [batch]: after the first launch
};

template <int DT>
__device__ __forceinline__ float load(const void* p, int64_t i) {
  if constexpr (DT == ART_ROWS_F32) return static_cast<const float*>(p)[i];
  else if constexpr (DT == ART_ROWS_F16) return (float)static_cast<const _Float16*>(p)[i];
  else return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
}

struct Nodes {
  double p[ART_MAX_NODES];     // the target's and the draft's probability of the
  double q[ART_MAX_NODES];     // node's token after its parent
  float u[ART_MAX_NODES];
  int parent[ART_MAX_NODES];   // -1: no child of any node
  int token[ART_MAX_NODES];
};

template <int THREADS>
__device__ __forceinline__ void load_tree(const VerifyParams& P, int first, int n, int* parents, int* tokens) {
  for (int i = threadIdx.x; i < n; i += THREADS) {
    int parent = P.parents[first + i];
    const int x = P.tokens[first + i];
    if (i == 0 || parent < 0 || parent >= i || x < 0 || x >= P.vocab) parent = -1;
    parents[i] = parent;
    tokens[i] = x;
  }
}
template <int DT, int THREADS>
__device__ __forceinline__ void load_nodes(const VerifyParams& P, int first, int n, Nodes& s) {
  load_tree<THREADS>(P, first, n, s.parent, s.token);
  for (int i = threadIdx.x; i < n; i += THREADS) {   // (each thread those that it has just loaded)
    const int parent = s.parent[i], x = s.token[i];
    s.u[i] = P.uniforms[first + i];
    s.p[i] = s.q[i] = 0.0;
    if (parent >= 0) {
      s.p[i] = load<DT>(P.target, (first + parent) * P.ts + x);
      if (P.draft) s.q[i] = load<DT>(P.draft, (first + parent) * P.ds + x);
    }
  }
  __syncthreads();
}

// The first child of `now` from node `from` on, or -1.
__device__ __forceinline__ int next_child(const Nodes& s, int n, int lane, int from, int now) {
  for (int base = from & ~63; base < n; base += 64) {
    const int i = base + lane;
    const uint64_t m = __ballot(i >= from && i < n && s.parent[min(i, n - 1)] == now);
    if (m) return base + __ffsll((unsigned long long)m) - 1;
  }
  return -1;
}
// Whether the token of child c is that of an earlier child of `now` (all of them
// have been rejected).
__device__ __forceinline__ bool again(const Nodes& s, int c, int lane, int now) {
  const int x = s.token[c];
  for (int base = 0; base < c; base += 64) {
    const int i = min(base + lane, c);
    if (__any(i < c && s.parent[i] == now && s.token[i] == x)) return true;
  }
  return false;
}

// Goes on until a sum is needed: of the weights with the new a, after a rejection
// that leaves other children, or of those to draw from (done).
__device__ __forceinline__ void walk_on(const VerifyParams& P, const Nodes& s, int n, int lane, int32_t* path, Walk& w) {
  if (w.done) return;
  while (w.count < P.max_path) {
    const int c = next_child(s, n, lane, w.next, w.now);
    if (c < 0) {
      w.tried = 1;
      break;
    }
    w.next = c + 1;
    const double u = s.u[c];
    bool ok;
    if (P.draft) {
      const double qx = s.q[c], left = s.p[c] - w.a * qx;
      ok = u * qx * w.f < (left > 0.0 ? left : 0.0);
      if (!ok) {
        w.a += w.f;
        if (next_child(s, n, lane, w.next, w.now) >= 0) return;   // F is asked for
        break;
      }
    } else {
      const double px = again(s, c, lane, w.now) ? 0.0 : s.p[c];
      ok = u * w.f < px;
      if (!ok) {
        w.f -= px;
        if (!(w.f > 0.0)) w.f = 0.0;
      }
    }
    if (ok) {
      if (path && lane == 0) path[w.count] = c;
      ++w.count;
      w.now = c;
      w.a = 0.0;
      w.f = 1.0;
    }
  }
  w.done = 1;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// Sums of lanes 0 .. lane.
__device__ __forceinline__ double scan(double x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// What a weight is made of: the current node's rows, a, and the tokens left out
// (its children, where they were tried and rejected without q).
struct Weights {
  const void* p;
  const void* q;
  double a;
  const int* out;
  int n_out;
};
template <int DT>
__device__ __forceinline__ Weights weights_of(const VerifyParams& P, const Walk& w, int first, const int* out, int n_out) {
  constexpr int size = DT == ART_ROWS_F32 ? 4 : 2;
  return Weights{static_cast<const char*>(P.target) + (first + w.now) * P.ts * size,
                 static_cast<const char*>(P.draft) + (w.a > 0.0 ? (first + w.now) * P.ds * size : 0), w.a, out, w.tried ? n_out : 0};
}
// The children of `now` among the nodes: their tokens into `out` (one wavefront).
__device__ __forceinline__ int left_out(const int* parent, const int* token, int n, int lane, int now, int* out) {
  int count = 0;
  for (int base = now + 1; base < n; base += 64) {
    const int i = base + lane;
    const bool mine = i < n && parent[min(i, n - 1)] == now;
    const uint64_t m = __ballot(mine);
    if (mine) out[count + __popcll(m & ((1ull << lane) - 1))] = token[i];
    count += __popcll(m);
  }
  return count;
}

// Sixteen bytes of a row (at any place that its type may lie at).
template <int DT>
constexpr int kSpan = DT == ART_ROWS_F32 ? 4 : 8;
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
template <int DT>
__device__ __forceinline__ u32x4 load16(const void* p, int v) {
  return *reinterpret_cast<const u32x4_any*>(static_cast<const char*>(p) + (int64_t)v * (16 / kSpan<DT>));
}
// The weights of tokens v .. v + span - 1, those from `end` on 0.
template <int DT>
__device__ __forceinline__ void weigh(const Weights& w, int v, int end, double (&x)[kSpan<DT>]) {
  constexpr int N = kSpan<DT>;
  if (v + N <= end) {
    const u32x4 p = load16<DT>(w.p, v);
    u32x4 q{0u, 0u, 0u, 0u};
    if (w.a > 0.0) q = load16<DT>(w.q, v);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double y = (double)value<DT>(p, i) - w.a * (double)value<DT>(q, i);
      x[i] = w.a > 0.0 && !(y > 0.0) ? 0.0 : y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = 0.0;
      if (v + i < end) {
        x[i] = load<DT>(w.p, v + i);
        if (w.a > 0.0) {
          const double y = x[i] - w.a * (double)load<DT>(w.q, v + i);
          x[i] = y > 0.0 ? y : 0.0;
        }
      }
    }
  }
  for (int j = 0; j < w.n_out; ++j) {
    const int d = w.out[j] - v;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (d == i) x[i] = 0.0;
  }
}
// A thread's share of the sum over a range: tokens range.x + span (thread + threads i).
template <int DT>
__device__ __forceinline__ double sum_of(const Weights& w, int2 range, int thread, int threads) {
  constexpr int N = kSpan<DT>;
  double sum = 0.0;
#pragma unroll 4
  for (int v = range.x + N * thread; v < range.y; v += N * threads) {
    double x[N];
    weigh<DT>(w, v, range.y, x);
#pragma unroll
    for (int i = 0; i < N; ++i) sum += x[i];
  }
  return sum;
}

// Slice i of the vocabulary.
__device__ __forceinline__ int2 slice_of(const VerifyParams& P, int i) {
  const int each = ((P.vocab + P.slices - 1) / P.slices + 7) & ~7;
  return make_int2(min(i * each, P.vocab), min((i + 1) * each, P.vocab));
}

template <int DT>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const VerifyParams P) {
  __shared__ Nodes s;
  __shared__ int s_out[ART_MAX_NODES], s_n_out;
  __shared__ double s_part[kSumThreads / 64];
  const int b = blockIdx.x / P.slices, slice = blockIdx.x - b * P.slices;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int2 span = rows_of(P, b);
  const int n = span.y - span.x;
  if (n == 0 || n > ART_MAX_NODES) return;
  load_nodes<DT, kSumThreads>(P, span.x, n, s);
  // (every wavefront walks; the first one of the first slice writes what is accepted)
  int32_t* const path = slice == 0 && wave == 0 ? P.accepted + (int64_t)b * P.max_path : nullptr;
  if (path && lane == 0) path[0] = 0;
  Walk w{0.0, 1.0, 0, 1, 1, 0, 0};
  walk_on(P, s, n, lane, path, w);
  if (path && lane == 0) P.walks[b] = w;
  if (wave == 0) {
    const int count = !P.draft && w.tried ? left_out(s.parent, s.token, n, lane, w.now, s_out) : 0;
    if (lane == 0) s_n_out = count;
  }
  __syncthreads();
  const Weights at = weights_of<DT>(P, w, span.x, s_out, s_n_out);
  const double sum = wave_sum(sum_of<DT>(at, slice_of(P, slice), threadIdx.x, kSumThreads));
  if (lane == 0) s_part[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double total = 0.0;
    for (int i = 0; i < kSumThreads / 64; ++i) total += s_part[i];
    P.sums[blockIdx.x] = total;
  }
}

template <int DT>
__global__ void __launch_bounds__(kDrawThreads) draw_kernel(const VerifyParams P) {
  constexpr int kWavesHere = kDrawThreads / 64, N = kSpan<DT>;
  __shared__ Nodes s;
  __shared__ int s_out[ART_MAX_NODES], s_n_out, s_found, s_positive;
  __shared__ double s_sums[kMaxSlices], s_part[kWavesHere];
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int2 span = rows_of(P, b);
  const int n = span.y - span.x;
  int32_t* const path = P.accepted + (int64_t)b * P.max_path;
  if (n == 0 || n > ART_MAX_NODES) {
    for (int i = threadIdx.x; i < P.max_path; i += kDrawThreads) path[i] = -1;
    if (threadIdx.x == 0) {
      P.counts[b] = 0;
      P.next[b] = -1;
    }
    return;
  }
  Walk w = P.walks[b];
  const double u = P.last[b];
  // lane i has the sum of slice i
  double mine = lane < P.slices ? P.sums[(int64_t)b * P.slices + lane] : 0.0;
  if (!w.done) load_nodes<DT, kDrawThreads>(P, span.x, n, s);
  else if (!P.draft && w.tried) load_tree<kDrawThreads>(P, span.x, n, s.parent, s.token);
  Weights at;
  double upto, total;
  for (bool first = true;; first = false) {
    at = weights_of<DT>(P, w, span.x, s_out, 0);
    if (!P.draft && w.tried) {     // (the last weights only: nodes that are not done have q)
      __syncthreads();
      if (wave == 0) {
        const int count = left_out(s.parent, s.token, n, lane, w.now, s_out);
        if (lane == 0) s_n_out = count;
      }
      __syncthreads();
      at.n_out = s_n_out;
    }
    if (!first) {
      // a sum of this workgroup's own: a slice to a wavefront
      __syncthreads();
      for (int i = wave; i < P.slices; i += kWavesHere) {
        const double sum = wave_sum(sum_of<DT>(at, slice_of(P, i), lane, 64));
        if (lane == 0) s_sums[i] = sum;
      }
      __syncthreads();
      mine = lane < P.slices ? s_sums[lane] : 0.0;
    }
    upto = scan(mine, lane);
    total = __shfl(upto, 63);
    if (!w.done) {
      w.f = total;
      walk_on(P, s, n, lane, wave == 0 ? path : nullptr, w);
    } else if (!(total > 0.0) && (w.a > 0.0 || at.n_out > 0)) {
      // nothing is left: from p itself (the walk is over: it changes nothing more)
      w.a = 0.0;
      w.tried = 0;
    } else {
      break;
    }
  }
  // the slice that the draw falls into, or the last of positive weight
  const double want = u * total;
  const uint64_t passed = __ballot(mine > 0.0 && upto > want), some = __ballot(mine > 0.0);
  int token = 0;
  if (some) {
    const int chosen = passed ? __ffsll((unsigned long long)passed) - 1 : 63 - __clzll((long long)some);
    double before = __shfl(upto - mine, chosen);
    // a span to every thread, 1024 spans at a time: the first token whose running sum
    // passes, or the last positive one
    const int2 range = slice_of(P, chosen);
    if (threadIdx.x == 0) {
      s_found = P.vocab;
      s_positive = -1;
    }
    for (int v0 = range.x; v0 < range.y; v0 += N * kDrawThreads) {
      const int v = v0 + N * threadIdx.x;
      double x[N], own = 0.0;
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = 0.0;
      if (v < range.y) weigh<DT>(at, v, range.y, x);
#pragma unroll
      for (int i = 0; i < N; ++i) own += x[i];
      const double sum = scan(own, lane);
      __syncthreads();     // (the parts of the spans before have been read)
      if (lane == 63) s_part[wave] = sum;
      __syncthreads();
      const double part = lane < kWavesHere ? s_part[lane] : 0.0, parts = scan(part, lane);
      double at_here = before + __shfl(parts - part, wave) + (sum - own);
      before += __shfl(parts, 63);
      int found = P.vocab, positive = -1;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        at_here += x[i];
        if (x[i] > 0.0) {
          positive = v + i;
          if (at_here > want && found == P.vocab) found = v + i;
        }
      }
      // (tokens grow with the lanes: one lane of each wavefront speaks)
      const uint64_t f = __ballot(found < P.vocab), g = __ballot(positive >= 0);
      if (f && lane == __ffsll((unsigned long long)f) - 1) atomicMin(&s_found, found);
      if (g && lane == 63 - __clzll((long long)g)) atomicMax(&s_positive, positive);
      __syncthreads();
      if (s_found < P.vocab) break;
    }
    __syncthreads();
    token = s_found < P.vocab ? s_found : max(s_positive, 0);
  }
  if (threadIdx.x == 0) {
    P.next[b] = token;
    P.counts[b] = w.count;
  }
  for (int i = w.count + threadIdx.x; i < P.max_path; i += kDrawThreads) path[i] = -1;
}

// ---- the accepted nodes' keys and values ------------------------------------------------

struct KeepParams {
  int32_t max_path, heads;
  int32_t page_shift, num_pages, max_pages;
  const int32_t* accepted;
  const int32_t* counts;
  const int32_t* positions;
  const int32_t* table;
  uint16_t* pool[2];
  int64_t sp[2], sh[2], st[2];
};

// A thread owns 16 bytes of a head's key or value in every slot of a sequence.
// Nodes move down (node accepted[j] >= j) in increasing order, so that a thread
// which moves them in order never reads what it has written.
__global__ void __launch_bounds__(kThreads) keep_kernel(const KeepParams P) {
  constexpr int kPieces = kHeadDim / 8, kAhead = 4;
  const int b = blockIdx.x, n = P.counts[b], context = P.positions[b];
  if (n <= 0 || n > P.max_path || context < 0) return;
  const int32_t* const nodes = P.accepted + (int64_t)b * P.max_path;
  const int64_t cap = (int64_t)P.max_pages << P.page_shift;
  bool fine = true;
  for (int j = threadIdx.x; j < n; j += kThreads)
    fine &= nodes[j] >= j && (j == 0 || nodes[j] > nodes[j - 1]) && (int64_t)context + nodes[j] < cap;
  if (!__syncthreads_and(fine)) return;
  const int at = blockIdx.y * kThreads + threadIdx.x, piece = at % kPieces, head = at / kPieces % P.heads;
  const int side = at / kPieces / P.heads;
  if (side > 1) return;
  uint16_t* const pool = P.pool[side] + head * P.sh[side] + 8 * piece;
  const int slots = 1 << P.page_shift;
  // (tokens in 64 bits: a context near 2^31 and a node's number pass it)
  auto where = [&](int64_t token) -> uint16_t* {
    const int page = P.table[(int64_t)b * P.max_pages + (token >> P.page_shift)];
    if (page < 0 || page >= P.num_pages) return nullptr;
    return pool + page * P.sp[side] + (token & (slots - 1)) * P.st[side];
  };
  for (int j0 = 0; j0 < n; j0 += kAhead) {
    u32x4 x[kAhead];
    uint16_t* to[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int j = j0 + i;
      to[i] = nullptr;
      if (j >= n || nodes[j] == j) continue;
      const uint16_t* from = where((int64_t)context + nodes[j]);
      if (!from) continue;
      to[i] = where((int64_t)context + j);
      x[i] = *reinterpret_cast<const u32x4*>(from);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (to[i]) *reinterpret_cast<u32x4*>(to[i]) = x[i];
  }
}

int log2_of(int64_t v) {
  int s = 0;
  while ((int64_t(1) << s) < v) ++s;
  return s;
}

art_status check_verify(const art_verify_opts* o) {
  if (!o || o->batch < 0 || o->rows < 0 || o->vocab <= 0 || o->max_path <= 0 || o->dtype < ART_ROWS_BF16 ||
      o->dtype > ART_ROWS_F32 || o->target_stride < o->vocab)
    return ART_ERR_INVALID_ARG;
  if (o->vocab >= (1 << 24) || o->rows >= (1 << 24) || o->batch >= (1 << 18) || o->target_stride >= (int64_t(1) << 38) ||
      o->draft_stride >= (int64_t(1) << 38))
    return ART_ERR_UNSUPPORTED;
  return ART_OK;
}

// Slices of the vocabulary: about four workgroups a CU, of 2048 tokens at least.
int slices_of(const art_verify_opts* o) {
  int n = o->batch > 0 ? 1024 / o->batch : 1;
  const int most = (o->vocab + 2047) / 2048;
  n = n < most ? n : most;
  return n < 1 ? 1 : n > kMaxSlices ? kMaxSlices : n;
}

template <int DT>
void launch_verify(const VerifyParams& p, hipStream_t stream) {
  hipLaunchKernelGGL(sum_kernel<DT>, dim3((unsigned)(p.batch * p.slices)), dim3(kSumThreads), 0, stream, p);
  hipLaunchKernelGGL(draw_kernel<DT>, dim3((unsigned)p.batch), dim3(kDrawThreads), 0, stream, p);
}

}  // namespace
}  // namespace art

extern "C" {

art_status art_tree_layout(int32_t batch, int32_t rows, const int32_t* parents, const int32_t* row_offsets,
                           const int32_t* context_lens, int32_t mask_words, uint64_t* mask, int32_t* positions,
                           hipStream_t stream) {
  using namespace art;
  if (batch < 0 || rows < 0 || mask_words < 1) return ART_ERR_INVALID_ARG;
  if (!row_offsets && batch > 0 && rows % batch) return ART_ERR_INVALID_ARG;
  if (mask_words > 16 || batch >= (1 << 24)) return ART_ERR_UNSUPPORTED;   // a launch has less than 2^32 threads
  if (!row_offsets && batch > 0 && rows / batch > ART_MAX_NODES) return ART_ERR_UNSUPPORTED;
  if (batch == 0 || rows == 0) return ART_OK;
  if (!parents || !mask || (positions && !context_lens) || (uintptr_t)mask % 8) return ART_ERR_INVALID_ARG;
  LayoutParams p;
  memset(&p, 0, sizeof p);
  p.batch = batch;
  p.rows = rows;
  p.per_seq = rows / batch;
  p.words = mask_words;
  p.offsets = row_offsets;
  p.positions = context_lens;
  p.parents = parents;
  p.mask = mask;
  p.out = positions;
  hipLaunchKernelGGL(layout_kernel, dim3((unsigned)batch), dim3(kThreads), 0, stream, p);
  return hipGetLastError() == hipSuccess ? ART_OK : ART_ERR_HIP;
}

size_t art_verify_workspace_bytes(const art_verify_opts* opts, int32_t* status) {
  const art_status st = art::check_verify(opts);
  if (status) *status = st;
  if (st != ART_OK) return 0;
  const size_t bytes = (sizeof(double) * art::slices_of(opts) + sizeof(art::Walk)) * opts->batch;
  return bytes < 256 ? 256 : bytes;
}

art_status art_verify_drafts(const art_verify_opts* opts, const void* target, const void* draft, const int32_t* tokens,
                             const int32_t* parents, const int32_t* row_offsets, const float* uniforms,
                             const float* last_uniforms, int32_t* accepted, int32_t* counts, int32_t* next_tokens,
                             void* workspace, size_t workspace_bytes, hipStream_t stream) {
  using namespace art;
  int32_t status = 0;
  const size_t need = art_verify_workspace_bytes(opts, &status);
  if (status != ART_OK) return (art_status)status;
  if (draft && opts->draft_stride < opts->vocab) return ART_ERR_INVALID_ARG;
  if (!row_offsets && opts->batch > 0 && opts->rows % opts->batch) return ART_ERR_INVALID_ARG;
  if (!row_offsets && opts->batch > 0 && opts->rows / opts->batch > ART_MAX_NODES) return ART_ERR_UNSUPPORTED;
  if (opts->batch == 0) return ART_OK;
  if (!accepted || !counts || !next_tokens || !last_uniforms ||
      (opts->rows > 0 && (!target || !tokens || !parents || !uniforms)))
    return ART_ERR_INVALID_ARG;
  const uintptr_t size = opts->dtype == ART_ROWS_F32 ? 4 : 2;
  if ((uintptr_t)target % size || (uintptr_t)draft % size || (uintptr_t)workspace % 8) return ART_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < need) return ART_ERR_WORKSPACE_TOO_SMALL;
  VerifyParams p;
  memset(&p, 0, sizeof p);
  p.batch = opts->batch;
  p.rows = opts->rows;
  p.per_seq = opts->rows / opts->batch;
  p.vocab = opts->vocab;
  p.max_path = opts->max_path;
  p.slices = slices_of(opts);
  p.ts = opts->target_stride;
  p.ds = opts->draft_stride;
  p.target = target;
  p.draft = draft;
  p.tokens = tokens;
  p.parents = parents;
  p.offsets = row_offsets;
  p.uniforms = uniforms;
  p.last = last_uniforms;
  p.accepted = accepted;
  p.counts = counts;
  p.next = next_tokens;
  p.sums = static_cast<double*>(workspace);
  p.walks = reinterpret_cast<Walk*>(p.sums + (int64_t)p.batch * p.slices);
  if (opts->dtype == ART_ROWS_BF16) launch_verify<ART_ROWS_BF16>(p, stream);
  else if (opts->dtype == ART_ROWS_F16) launch_verify<ART_ROWS_F16>(p, stream);
  else launch_verify<ART_ROWS_F32>(p, stream);
  return hipGetLastError() == hipSuccess ? ART_OK : ART_ERR_HIP;
}

art_status art_keep_accepted(const art_decode_shape* shape, int32_t max_path, const int32_t* accepted,
                             const int32_t* counts, const int32_t* context_lens, const int32_t* page_table,
                             void* k_cache, void* v_cache, hipStream_t stream) {
  using namespace art;
  const art_status st = check_cache(shape);
  if (st != ART_OK) return st;
  if (max_path <= 0) return ART_ERR_INVALID_ARG;
  const int64_t slabs = ((int64_t)shape->num_kv_heads * 2 * (kHeadDim / 8) + kThreads - 1) / kThreads;
  if (shape->batch >= (1 << 20) || slabs > 65535 || slabs * shape->batch >= (1 << 24)) return ART_ERR_UNSUPPORTED;
  if (shape->batch == 0) return ART_OK;
  if (!accepted || !counts || !context_lens || !page_table || !k_cache || !v_cache) return ART_ERR_INVALID_ARG;
  if (((uintptr_t)k_cache | (uintptr_t)v_cache) % 16) return ART_ERR_UNSUPPORTED;
  KeepParams p;
  memset(&p, 0, sizeof p);
  p.max_path = max_path;
  p.heads = shape->num_kv_heads;
  p.page_shift = log2_of(shape->page_size);
  p.num_pages = shape->num_pages;
  p.max_pages = shape->max_pages_per_seq;
  p.accepted = accepted;
  p.counts = counts;
  p.positions = context_lens;
  p.table = page_table;
  p.pool[0] = static_cast<uint16_t*>(k_cache);
  p.pool[1] = static_cast<uint16_t*>(v_cache);
  p.sp[0] = shape->k_stride_page;
  p.sh[0] = shape->k_stride_head;
  p.st[0] = shape->k_stride_token;
  p.sp[1] = shape->v_stride_page;
  p.sh[1] = shape->v_stride_head;
  p.st[1] = shape->v_stride_token;
  hipLaunchKernelGGL(keep_kernel, dim3((unsigned)shape->batch, (unsigned)slabs), dim3(kThreads), 0, stream, p);
  return hipGetLastError() == hipSuccess ? ART_OK : ART_ERR_HIP;
}

}  // extern "C"
