// Rotary positions: rows of queries and keys turned by the angles of their
// positions, in place, into other rows (art_rope_rows) or, keys and values,
// into the slots of a paged bf16 cache (art_rope_append).
//
// A wavefront works on the heads of one row.  Its lane i computes the cosine and
// sine of pair i once for all of them:
//   t = position * freqs[i] / pi, less twice its nearest whole turn, in fp64,
//   (cos, sin)(pi t) in fp32, times the factor,
// and leaves them in LDS, from where every lane takes the eight pairs of its own
// 16 dims.  Memory bounds it: ragged prompts of 66K tokens, 32 + 8 + 8 heads, take 254
// us, 5.2 TB/s read and written (a copy of 4 GiB runs at 5.0); one token 2.8 us.  64K
// rows of 32 heads, 128 dims rotated: 199 us in bf16 or fp16 (5.4 TB/s), 402 to 479 in
// fp32 (4.5 to 5.3), 305 from fp32 to bf16.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "art.h"
#include "art_internal.h"
#include "art_rows.h"

namespace art {
namespace {

constexpr int kUnits = kHeadDim / 16;        // lanes of a head: 16 dims each
constexpr int kHeadsAStep = 64 / kUnits;     // heads that a wavefront has at a time

struct Rows {
  char* p;                  // (read or written)
  int64_t row, head;        // strides in bytes
  int32_t heads;
};

struct RopeParams {
  int32_t batch, rows, per_seq;
  int32_t page_shift, num_pages, max_pages;
  int32_t heads;                 // of q, k and v together
  int32_t parts;                 // wavefronts that share a row's heads
  int32_t rot, interleaved;
  float scale;
  const int32_t* offsets;
  const int32_t* positions;      // of the sequences: the tokens that each holds (append)
  const int32_t* row_positions;
  const int32_t* table;
  const double* freqs;
  Rows q, q_out, k, v;           // k.heads == 0: no cache
  uint16_t* k_cache;
  uint16_t* v_cache;
  int64_t ksp, ksh, kst, vsp, vsh, vst;   // of the pools, in elements
};

// Sixteen consecutive or twice eight values of a row.
template <int DT>
struct Half {
  u32x4 w[DT == ART_ROWS_F32 ? 2 : 1];
};
template <int DT>
__device__ __forceinline__ Half<DT> load8(const char* p, int dim) {
  Half<DT> h;
  const char* at = p + dim * (DT == ART_ROWS_F32 ? 4 : 2);
  h.w[0] = *reinterpret_cast<const u32x4*>(at);
  if constexpr (DT == ART_ROWS_F32) h.w[1] = *reinterpret_cast<const u32x4*>(at + 16);
  return h;
}
template <int DT>
__device__ __forceinline__ float at8(const Half<DT>& h, int i) {
  if constexpr (DT == ART_ROWS_F32) return value<DT>(h.w[i >> 2], i & 3);
  else return value<DT>(h.w[0], i);
}
template <int DT>
__device__ __forceinline__ void store8(char* p, int dim, const float (&x)[8]) {
  char* at = p + dim * (DT == ART_ROWS_F32 ? 4 : 2);
  if constexpr (DT == ART_ROWS_F32) {
    const float a[4] = {x[0], x[1], x[2], x[3]}, b[4] = {x[4], x[5], x[6], x[7]};
    *reinterpret_cast<u32x4*>(at) = packed<DT, 4>(a);
    *reinterpret_cast<u32x4*>(at + 16) = packed<DT, 4>(b);
  } else {
    *reinterpret_cast<u32x4*>(at) = packed<DT, 8>(x);
  }
}
template <int DT>
__device__ __forceinline__ float load1(const char* p, int dim) {
  if constexpr (DT == ART_ROWS_F32) return reinterpret_cast<const float*>(p)[dim];
  else if constexpr (DT == ART_ROWS_F16) return (float)reinterpret_cast<const _Float16*>(p)[dim];
  else return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[dim] << 16);
}

// DT, OT: types of the rows and of what is written.  EVEN: rot is a multiple of
// 16, so that a lane's 16 dims are eight whole pairs (or none).
template <int DT, int OT, bool EVEN>
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeParams P) {
  __shared__ float2 s_turn[kWaves][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t job = (int64_t)blockIdx.x * kWaves + wave;
  const int row = (int)(job / P.parts), part = (int)(job - (int64_t)row * P.parts);
  if (row >= P.rows) return;

  // where the row lies, and its position
  int page = -1, slot = 0;
  double position = 0.0;
  if (P.k.heads || !P.row_positions) {
    const SpanTable table = span_table(P, lane);
    const Span s = span_of(P, table, row, lane);
    const int64_t cap = (int64_t)P.max_pages << P.page_shift;
    if (s.b >= P.batch || row < s.first || row >= s.end || s.pos < 0 || s.pos + (s.end - s.first) > cap) return;
    const int64_t token = s.pos + (row - s.first);
    page = page_of(P, s.b, token);
    slot = (int)(token & ((1 << P.page_shift) - 1));
    position = (double)(uint32_t)token;   // (a context near 2^31 and its rows pass that, but no 2^32)
  }
  if (P.row_positions) position = P.row_positions[row];

  const int half = P.rot >> 1;
  float c = 1.f, sn = 0.f;
  if (lane < half) {
    // half turns: 1 / pi in fp64 costs 2^-53 of them.  What is left after the nearest
    // whole turn goes to the functions as fp32, and what that leaves of it (2^-25) in
    // by the first order.
    double t = position * (P.freqs[lane] * 0.3183098861837907);
    t -= 2.0 * rint(0.5 * t);
    const float near = (float)t, rest = (float)((t - near) * 3.141592653589793);
    float s0, c0;
    sincospif(near, &s0, &c0);
    c = fmaf(-rest, s0, c0) * P.scale;
    sn = fmaf(rest, c0, s0) * P.scale;
  }
  s_turn[wave][lane] = make_float2(c, sn);
  __builtin_amdgcn_wave_barrier();

  const int unit = lane & (kUnits - 1);
  // the first dims of the lane's two halves, and the first of its pairs; the
  // units behind the rotated dims copy theirs
  int d0 = 16 * unit, d1 = d0 + 8;
  bool turns = d0 < P.rot;
  float2 turn[EVEN ? 8 : 1];
  if constexpr (EVEN) {
    if (turns && !P.interleaved) {
      d0 = 8 * unit;
      d1 = d0 + half;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) turn[i] = s_turn[wave][turns ? 8 * unit + i : 0];
  }

  for (int h0 = part * kHeadsAStep; h0 < P.heads; h0 += P.parts * kHeadsAStep) {
    int h = h0 + lane / kUnits;
    if (h >= P.heads) continue;
    const char* from;
    char* to;
    bool rotate = turns;
    if (h < P.q.heads) {
      from = P.q.p + row * P.q.row + h * P.q.head;
      to = P.q_out.p + row * P.q_out.row + h * P.q_out.head;
    } else {
      h -= P.q.heads;
      if (page < 0) continue;
      if (h < P.k.heads) {
        from = P.k.p + row * P.k.row + h * P.k.head;
        to = reinterpret_cast<char*>(P.k_cache + (page * P.ksp + h * P.ksh + slot * P.kst));
      } else {
        h -= P.k.heads;
        from = P.v.p + row * P.v.row + h * P.v.head;
        to = reinterpret_cast<char*>(P.v_cache + (page * P.vsp + h * P.vsh + slot * P.vst));
        rotate = false;
      }
    }
    float x[8], y[8];
    if constexpr (EVEN) {
      const Half<DT> a = load8<DT>(from, d0), b = load8<DT>(from, d1);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = at8<DT>(a, i);
        y[i] = at8<DT>(b, i);
      }
      if (rotate) {
        if (P.interleaved) {
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const float2 s = turn[i / 2], t = turn[4 + i / 2];
            const float x0 = x[i], x1 = x[i + 1], y0 = y[i], y1 = y[i + 1];
            x[i] = fmaf(x0, s.x, -(x1 * s.y));
            x[i + 1] = fmaf(x1, s.x, x0 * s.y);
            y[i] = fmaf(y0, t.x, -(y1 * t.y));
            y[i + 1] = fmaf(y1, t.x, y0 * t.y);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float x0 = x[i], y0 = y[i];
            x[i] = fmaf(x0, turn[i].x, -(y0 * turn[i].y));
            y[i] = fmaf(y0, turn[i].x, x0 * turn[i].y);
          }
        }
      }
    } else {
      // any even rot: dim by dim, each with its partner (all loads of a head come
      // before its stores: its eight lanes are of one wavefront).  Loads of one value
      // bound it: the 64K rows above take 0.71 ms with 20 dims rotated, 0.96 to 1.06 with
      // 126.
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int d = d0 + i;
        float v = load1<DT>(from, d);
        const bool on = d < P.rot && h0 + lane / kUnits < P.q.heads + P.k.heads;
        if (on) {
          const int pair = P.interleaved ? d >> 1 : d < half ? d : d - half;
          const bool second = P.interleaved ? d & 1 : d >= half;
          const int other = P.interleaved ? d ^ 1 : second ? d - half : d + half;
          const float w = load1<DT>(from, other);
          const float2 s = s_turn[wave][pair];
          v = second ? fmaf(v, s.x, w * s.y) : fmaf(v, s.x, -(w * s.y));
        }
        if (i < 8) x[i] = v;
        else y[i - 8] = v;
      }
      __builtin_amdgcn_wave_barrier();
    }
    store8<OT>(to, d0, x);
    store8<OT>(to, d1, y);
  }
}

int log2_of(int64_t v) {
  int s = 0;
  while ((int64_t(1) << s) < v) ++s;
  return s;
}

int64_t size_of(int dtype) { return dtype == ART_ROWS_F32 ? 4 : 2; }

art_status check_rope(const art_rope* r) {
  if (!r) return ART_OK;
  if ((r->layout != ART_ROPE_HALF && r->layout != ART_ROPE_INTERLEAVED) || r->rot_dim < 0 || r->rot_dim > kHeadDim ||
      r->rot_dim % 2 || !isfinite(r->scale))
    return ART_ERR_INVALID_ARG;
  return ART_OK;
}

art_status check_rows(const art_rows* r) {
  if (!r || r->dtype < ART_ROWS_BF16 || r->dtype > ART_ROWS_F32 || r->heads <= 0 || r->stride_row < 0 || r->stride_head < 0)
    return ART_ERR_INVALID_ARG;
  const int64_t size = size_of(r->dtype);
  // heads of q, k and v together, and a step past them, are counted in 32 bits
  if (r->heads >= (1 << 28)) return ART_ERR_UNSUPPORTED;
  // (each by itself: a product could leave 64 bits)
  if (r->stride_row >= (1 << 28) || r->stride_row * size >= (1 << 28) || r->stride_head >= (int64_t(1) << 40) ||
      r->stride_row * size % 16 || r->stride_head * size % 16)
    return ART_ERR_UNSUPPORTED;
  return ART_OK;
}

Rows rows_of(const art_rows* r, const void* p) {
  return Rows{(char*)p, r->stride_row * size_of(r->dtype), r->stride_head * size_of(r->dtype), r->heads};
}

template <int DT, int OT>
void launch(const RopeParams& p, unsigned grid, hipStream_t stream) {
  if (p.rot % 16 == 0) hipLaunchKernelGGL((rope_kernel<DT, OT, true>), dim3(grid), dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL((rope_kernel<DT, OT, false>), dim3(grid), dim3(kThreads), 0, stream, p);
}
template <int DT>
void launch(const RopeParams& p, int out, unsigned grid, hipStream_t stream) {
  if (out == ART_ROWS_BF16) launch<DT, ART_ROWS_BF16>(p, grid, stream);
  else if (out == ART_ROWS_F16) launch<DT, ART_ROWS_F16>(p, grid, stream);
  else launch<DT, ART_ROWS_F32>(p, grid, stream);
}

art_status launch_rope(RopeParams& p, int dtype, int out, hipStream_t stream) {
  // a wavefront to a row, or to every step of its heads where the rows are few: the
  // chip holds 8192 wavefronts
  const int64_t steps = (p.heads + kHeadsAStep - 1) / kHeadsAStep;
  p.parts = (int32_t)steps;
  while (p.parts > 1 && (int64_t)p.rows * p.parts > 8192) p.parts = (p.parts + 1) / 2;
  const int64_t grid = ((int64_t)p.rows * p.parts + kWaves - 1) / kWaves;
  if (grid >= (1 << 24)) return ART_ERR_UNSUPPORTED;   // a launch has less than 2^32 threads
  if (dtype == ART_ROWS_BF16) launch<ART_ROWS_BF16>(p, out, (unsigned)grid, stream);
  else if (dtype == ART_ROWS_F16) launch<ART_ROWS_F16>(p, out, (unsigned)grid, stream);
  else launch<ART_ROWS_F32>(p, out, (unsigned)grid, stream);
  return hipGetLastError() == hipSuccess ? ART_OK : ART_ERR_HIP;
}

}  // namespace

// The page and stride fields of a shape that a call on a bf16 cache reads.
art_status check_cache(const art_decode_shape* s) {
  if (!s) return ART_ERR_INVALID_ARG;
  if (s->batch < 0 || s->num_kv_heads <= 0 || s->head_dim <= 0 || s->page_size <= 0 || s->num_pages <= 0 ||
      s->max_pages_per_seq <= 0 || s->k_stride_page < 0 || s->k_stride_head < 0 || s->k_stride_token < 0 ||
      s->v_stride_page < 0 || s->v_stride_head < 0 || s->v_stride_token < 0)
    return ART_ERR_INVALID_ARG;
  if (s->head_dim != kHeadDim || s->page_size < 16 || (s->page_size & (s->page_size - 1))) return ART_ERR_UNSUPPORTED;
  if ((s->k_stride_page | s->k_stride_head | s->k_stride_token | s->v_stride_page | s->v_stride_head |
       s->v_stride_token) % 8)
    return ART_ERR_UNSUPPORTED;
  return ART_OK;
}

}  // namespace art

extern "C" {

art_status art_rope_rows(const art_rope* rope, int32_t rows, const art_rows* x_rows, const void* x,
                         const art_rows* out_rows, void* out, const int32_t* positions, const double* freqs,
                         hipStream_t stream) {
  using namespace art;
  if (!rope || rows < 0) return ART_ERR_INVALID_ARG;
  art_status st = check_rope(rope);
  if (st == ART_OK) st = check_rows(x_rows);
  if (st == ART_OK) st = check_rows(out_rows);
  if (st != ART_OK) return st;
  if (x_rows->heads != out_rows->heads) return ART_ERR_INVALID_ARG;
  if (rows >= (1 << 24)) return ART_ERR_UNSUPPORTED;
  if (rows == 0) return ART_OK;
  if (!x || !out || !positions || (rope->rot_dim && !freqs) || (uintptr_t)freqs % 8) return ART_ERR_INVALID_ARG;
  if (((uintptr_t)x | (uintptr_t)out) % 16) return ART_ERR_UNSUPPORTED;
  RopeParams p;
  memset(&p, 0, sizeof p);
  p.rows = rows;
  p.heads = x_rows->heads;
  p.rot = rope->rot_dim;
  p.interleaved = rope->layout == ART_ROPE_INTERLEAVED;
  p.scale = rope->scale;
  p.row_positions = positions;
  p.freqs = freqs;
  p.q = rows_of(x_rows, x);
  p.q_out = rows_of(out_rows, out);
  return launch_rope(p, x_rows->dtype, out_rows->dtype, stream);
}

art_status art_rope_append(const art_decode_shape* shape, const art_rope* rope, int32_t rows, const art_rows* q_rows,
                           const void* q, const art_rows* q_out_rows, void* q_out, const art_rows* k_rows,
                           const void* k, const art_rows* v_rows, const void* v, const int32_t* row_offsets,
                           const int32_t* context_lens, const int32_t* row_positions, const double* freqs,
                           const int32_t* page_table, void* k_cache, void* v_cache, hipStream_t stream) {
  using namespace art;
  art_status st = check_cache(shape);
  if (st == ART_OK && rows < 0) st = ART_ERR_INVALID_ARG;
  if (st == ART_OK) st = check_rope(rope);
  if (st == ART_OK) st = check_rows(k_rows);
  if (st == ART_OK) st = check_rows(v_rows);
  if (st == ART_OK && q) st = check_rows(q_rows);
  if (st == ART_OK && q) st = check_rows(q_out_rows);
  if (st != ART_OK) return st;
  if (k_rows->heads != shape->num_kv_heads || v_rows->heads != shape->num_kv_heads || v_rows->dtype != k_rows->dtype)
    return ART_ERR_INVALID_ARG;
  if (q && (q_rows->heads != shape->num_q_heads || q_out_rows->heads != q_rows->heads || q_rows->dtype != k_rows->dtype))
    return ART_ERR_INVALID_ARG;
  if (!row_offsets && shape->batch > 0 && rows % shape->batch) return ART_ERR_INVALID_ARG;
  if (rows >= (1 << 24)) return ART_ERR_UNSUPPORTED;
  if (q && q_out_rows->dtype != ART_ROWS_BF16) return ART_ERR_UNSUPPORTED;   // what attention over the cache reads
  if (shape->batch == 0 || rows == 0) return ART_OK;
  if (!k || !v || !context_lens || !page_table || !k_cache || !v_cache || (q && !q_out) ||
      (rope && rope->rot_dim && !freqs) || (uintptr_t)freqs % 8)
    return ART_ERR_INVALID_ARG;
  if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)q | (uintptr_t)q_out | (uintptr_t)k_cache | (uintptr_t)v_cache) % 16)
    return ART_ERR_UNSUPPORTED;
  RopeParams p;
  memset(&p, 0, sizeof p);
  p.batch = shape->batch;
  p.rows = rows;
  p.per_seq = rows / shape->batch;
  p.page_shift = log2_of(shape->page_size);
  p.num_pages = shape->num_pages;
  p.max_pages = shape->max_pages_per_seq;
  p.rot = rope ? rope->rot_dim : 0;
  p.interleaved = rope && rope->layout == ART_ROPE_INTERLEAVED;
  p.scale = rope ? rope->scale : 1.f;
  p.offsets = row_offsets;
  p.positions = context_lens;
  p.row_positions = row_positions;
  p.table = page_table;
  p.freqs = freqs;
  if (q) {
    p.q = rows_of(q_rows, q);
    p.q_out = rows_of(q_out_rows, q_out);
  }
  p.k = rows_of(k_rows, k);
  p.v = rows_of(v_rows, v);
  p.heads = p.q.heads + p.k.heads + p.v.heads;
  p.k_cache = static_cast<uint16_t*>(k_cache);
  p.v_cache = static_cast<uint16_t*>(v_cache);
  p.ksp = shape->k_stride_page;
  p.ksh = shape->k_stride_head;
  p.kst = shape->k_stride_token;
  p.vsp = shape->v_stride_page;
  p.vsh = shape->v_stride_head;
  p.vst = shape->v_stride_token;
  return launch_rope(p, k_rows->dtype, ART_ROWS_BF16, stream);
}

}  // extern "C"
