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
// node for one word of its mask.
__global__ void __launch_bounds__(kThreads) layout_kernel(const LayoutParams P) {
  __shared__ int s_parent[ART_MAX_NODES];
  const int b = blockIdx.x;
  const int2 span = rows_of(P, b);
  const int n = span.y - span.x, context = P.positions ? P.positions[b] : 0;
  if (n == 0 || n > ART_MAX_NODES || context < 0) return;
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
// second walks again with that sum in hand, in one workgroup to a sequence, and
// draws the token; the rare further sums (siblings rejected one after another) are
// its own.  No workgroup ever waits for another.

constexpr int kMaxSlices = 64;
constexpr int kSumThreads = 256;
constexpr int kDrawThreads = 1024;

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

template <int DT, int THREADS>
__device__ __forceinline__ void load_nodes(const VerifyParams& P, int first, int n, Nodes& s) {
  for (int i = threadIdx.x; i < n; i += THREADS) {
    int parent = P.parents[first + i];
    const int x = P.tokens[first + i];
    if (i == 0 || parent < 0 || parent >= i || x < 0 || x >= P.vocab) parent = -1;
    s.parent[i] = parent;
    s.token[i] = x;
    s.u[i] = P.uniforms[first + i];
    s.p[i] = s.q[i] = 0.0;
    if (parent >= 0) {
      s.p[i] = load<DT>(P.target, (first + parent) * P.ts + x);
      if (P.draft) s.q[i] = load<DT>(P.draft, (first + parent) * P.ds + x);
    }
  }
  __syncthreads();
  if (P.draft) return;
  // the token of an earlier sibling has been rejected when a node is tried
  for (int i = threadIdx.x; i < n; i += THREADS) {
    bool again = false;
    for (int j = 1; j < i; ++j) again |= s.parent[j] == s.parent[i] && s.token[j] == s.token[i];
    if (again) s.p[i] = 0.0;
  }
  __syncthreads();
}

// Where a walk stands.  It is the same in every lane of the wavefront.
struct Walk {
  int now, count, next;        // the current node, nodes accepted, the first one not tried
  double a, f;                 // with q: a and F; without: f is what is left of 1
  bool done;                   // the next token is drawn from the current weights
  bool tried;                  // (without q) the current node's children have been rejected
};

// Goes on until a sum is needed: of the weights with the new a, after a
// rejection, or of those to draw from (done).
__device__ __forceinline__ void walk_on(const VerifyParams& P, const Nodes& s, int n, int lane, int32_t* path, Walk& w) {
  if (w.done) return;
  while (w.count < P.max_path) {
    int c = -1;
    for (int base = w.next & ~63; base < n && c < 0; base += 64) {
      const int i = base + lane;
      const uint64_t m = __ballot(i >= w.next && i < n && s.parent[min(i, n - 1)] == w.now);
      if (m) c = base + __ffsll((unsigned long long)m) - 1;
    }
    if (c < 0) {
      w.tried = true;
      break;
    }
    w.next = c + 1;
    const double px = s.p[c], u = s.u[c];
    if (P.draft) {
      const double qx = s.q[c], left = px - w.a * qx;
      if (u * qx * w.f < (left > 0.0 ? left : 0.0)) {
        if (path && lane == 0) path[w.count] = c;
        ++w.count;
        w.now = c;
        w.a = 0.0;
        w.f = 1.0;
      } else {
        w.a += w.f;
        return;   // F is asked for
      }
    } else if (u * w.f < px) {
      if (path && lane == 0) path[w.count] = c;
      ++w.count;
      w.now = c;
      w.f = 1.0;
    } else {
      w.f -= px;
      if (!(w.f > 0.0)) w.f = 0.0;
    }
  }
  w.done = true;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// What a weight is made of: row `now`, a, and the tokens left out (the children
// of `now`, where they were tried and rejected without q).
struct Weights {
  int64_t p, q;                // element indices of the rows
  double a;
  int skip_parent;             // -1: no token is left out
  int n;                       // nodes
};

template <int DT>
__device__ __forceinline__ double weight(const VerifyParams& P, const Nodes& s, const Weights& w, int v) {
  const double p = load<DT>(P.target, w.p + v);
  if (w.a > 0.0) {
    const double x = p - w.a * (double)load<DT>(P.draft, w.q + v);
    return x > 0.0 ? x : 0.0;
  }
  if (w.skip_parent >= 0)
    for (int i = w.skip_parent + 1; i < w.n; ++i)
      if (s.parent[i] == w.skip_parent && s.token[i] == v) return 0.0;
  return p;
}

__device__ __forceinline__ Weights weights_of(const VerifyParams& P, const Walk& w, int first, int n) {
  return Weights{(first + w.now) * P.ts, (first + w.now) * P.ds, w.a, !P.draft && w.tried ? w.now : -1, n};
}

// Slice i of the vocabulary.
__device__ __forceinline__ int2 slice_of(const VerifyParams& P, int i) {
  const int each = (P.vocab + P.slices - 1) / P.slices;
  return make_int2(min(i * each, P.vocab), min((i + 1) * each, P.vocab));
}

template <int DT>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const VerifyParams P) {
  __shared__ Nodes s;
  __shared__ double s_part[kSumThreads / 64];
  const int b = blockIdx.x / P.slices, slice = blockIdx.x - b * P.slices;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int2 span = rows_of(P, b);
  const int n = span.y - span.x;
  if (n == 0 || n > ART_MAX_NODES) return;
  load_nodes<DT, kSumThreads>(P, span.x, n, s);
  Walk w{0, 1, 1, 0.0, 1.0, false, false};
  walk_on(P, s, n, lane, nullptr, w);
  const Weights at = weights_of(P, w, span.x, n);
  const int2 range = slice_of(P, slice);
  double sum = 0.0;
  for (int v = range.x + threadIdx.x; v < range.y; v += kSumThreads) sum += weight<DT>(P, s, at, v);
  sum = wave_sum(sum);
  if (lane == 0) s_part[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double total = 0.0;
    for (int i = 0; i < kSumThreads / 64; ++i) total += s_part[i];
    P.sums[blockIdx.x] = total;
  }
}

// Sums of the kDrawThreads / 64 equal parts of a range, one to a wavefront.
template <int DT>
__device__ __forceinline__ void part_sums(const VerifyParams& P, const Nodes& s, const Weights& at, int2 range, double* parts) {
  constexpr int kParts = kDrawThreads / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int each = (range.y - range.x + kParts - 1) / kParts;
  const int end = min(range.x + (wave + 1) * each, range.y);
  double sum = 0.0;
  for (int v = range.x + wave * each + lane; v < end; v += 64) sum += weight<DT>(P, s, at, v);
  sum = wave_sum(sum);
  __syncthreads();
  if (lane == 0) parts[wave] = sum;
  __syncthreads();
}

template <int DT>
__global__ void __launch_bounds__(kDrawThreads) draw_kernel(const VerifyParams P) {
  constexpr int kParts = kDrawThreads / 64;
  __shared__ Nodes s;
  __shared__ double s_sums[kMaxSlices];
  __shared__ double s_part[kParts];
  const int b = blockIdx.x, lane = threadIdx.x & 63;
  const int2 span = rows_of(P, b);
  const int n = span.y - span.x;
  int32_t* const path = P.accepted + (int64_t)b * P.max_path;
  const bool none = n == 0 || n > ART_MAX_NODES;
  if (none) {
    for (int i = threadIdx.x; i < P.max_path; i += kDrawThreads) path[i] = -1;
    if (threadIdx.x == 0) {
      P.counts[b] = 0;
      P.next[b] = -1;
    }
    return;
  }
  load_nodes<DT, kDrawThreads>(P, span.x, n, s);
  // (every wavefront walks, the first one writes what is accepted)
  if (threadIdx.x == 0) path[0] = 0;
  int32_t* const mine = threadIdx.x < 64 ? path : nullptr;
  Walk w{0, 1, 1, 0.0, 1.0, false, false};
  const double u = P.last[b];
  int2 range{0, 0};
  Weights at;
  // the sums of the slices, from the first launch or, later ones, made here
  for (int k = 0;; ++k) {
    walk_on(P, s, n, lane, mine, w);
    at = weights_of(P, w, span.x, n);
    if (k == 0) {
      if (threadIdx.x < P.slices) s_sums[threadIdx.x] = P.sums[(int64_t)b * P.slices + threadIdx.x];
      __syncthreads();
    } else {
      for (int i = 0; i < P.slices; ++i) {
        part_sums<DT>(P, s, at, slice_of(P, i), s_part);
        if (threadIdx.x == 0) {
          double total = 0.0;
          for (int j = 0; j < kParts; ++j) total += s_part[j];
          s_sums[i] = total;
        }
      }
      __syncthreads();
    }
    double total = 0.0;
    for (int i = 0; i < P.slices; ++i) total += s_sums[i];
    __syncthreads();
    if (!w.done) {
      w.f = total;
      continue;
    }
    if (!(total > 0.0) && (w.a > 0.0 || at.skip_parent >= 0)) {
      // nothing is left: from p itself (the walk is over: it changes nothing more)
      w.a = 0.0;
      w.tried = false;
      continue;
    }
    // the slice that the draw falls into, or the last of positive weight
    const double want = u * total;
    double before = 0.0, run = 0.0;
    int chosen = -1;
    for (int i = 0; i < P.slices; ++i) {
      const double x = s_sums[i];
      if (x > 0.0) {
        before = run;
        chosen = i;
        if (run + x > want) break;
      }
      run += x;
    }
    if (chosen < 0) {
      if (threadIdx.x == 0) P.next[b] = 0;
      break;
    }
    range = slice_of(P, chosen);
    // narrowed to one part after the other, to 64 tokens at most
    while (range.y - range.x > 64) {
      part_sums<DT>(P, s, at, range, s_part);
      const int each = (range.y - range.x + kParts - 1) / kParts;
      run = before;
      int part = -1;
      for (int i = 0; i < kParts; ++i) {
        const double x = s_part[i];
        if (x > 0.0) {
          before = run;
          part = i;
          if (run + x > want) break;
        }
        run += x;
      }
      part = max(part, 0);
      range = make_int2(range.x + part * each, min(range.x + (part + 1) * each, range.y));
    }
    if (threadIdx.x < 64) {
      const int v = range.x + lane;
      const double x = v < range.y ? weight<DT>(P, s, at, v) : 0.0;
      double sum = x;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(sum, o);
        if (lane >= o) sum += y;
      }
      const uint64_t over = __ballot(x > 0.0 && before + sum > want), some = __ballot(x > 0.0);
      int token = range.x;
      if (over) token += __ffsll((unsigned long long)over) - 1;
      else if (some) token += 63 - __clzll((long long)some);
      if (lane == 0) P.next[b] = min(token, P.vocab - 1);
    }
    break;
  }
  if (threadIdx.x == 0) P.counts[b] = w.count;
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
  auto where = [&](int token) -> uint16_t* {
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
      const uint16_t* from = where(context + nodes[j]);
      if (!from) continue;
      to[i] = where(context + j);
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

// Slices of the vocabulary: about two workgroups a CU, of 2048 tokens at least.
int slices_of(const art_verify_opts* o) {
  int n = o->batch > 0 ? 512 / o->batch : 1;
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
  const size_t bytes = sizeof(double) * opts->batch * art::slices_of(opts);
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
