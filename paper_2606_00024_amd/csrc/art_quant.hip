// The 8-bit cache's writer and reader: rows of K and V in 16 or 32 bits are
// quantised into paged pools of codes with a scale for every run of slots
// (art_quant_append), and stored tokens come back as rows (art_quant_read).
//
// Both take rows packed over the sequences of a batch.  A wavefront finds the
// sequence of its first row by counting the row offsets at or below it (64 a
// step), so no launch is needed to turn offsets into a plan, and a batch may
// mix long and short (or no) spans.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include "art.h"
#include "art_internal.h"

namespace art {
namespace {

constexpr int kMaxRun = 256;      // slots that share a scale, at most (append)
constexpr int kLowestExp = -120;  // exponent of the smallest scale

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// K or V of a call.
struct Side {
  char* rows;               // read by append, written by read
  int64_t row, head;        // strides of the rows, in bytes
  uint8_t* codes;
  int64_t sp, sh, st;       // page, head and token strides of the pool
  float* scale;
  int64_t scp, sch;         // page and head strides of the scales
};

struct QuantParams {
  int32_t batch, heads, rows, per_seq;   // per_seq: rows of every sequence without offsets
  int32_t page_shift, run_shift, num_pages, max_pages;
  int32_t window;                        // append: rows whose runs one wavefront starts
  const int32_t* offsets;
  const int32_t* positions;
  const int32_t* table;
  Side side[2];
};

// Where a row belongs: sequence b holds rows [first, end) from token `pos` on.
// b == batch: no sequence.
struct Span {
  int b, first, end;
  int64_t pos;
};

__device__ __forceinline__ Span span_of(const QuantParams& P, int row, int lane) {
  Span s;
  if (!P.offsets) {
    s.b = P.per_seq > 0 ? row / P.per_seq : P.batch;
    s.first = s.b * P.per_seq;
    s.end = s.first + P.per_seq;
  } else {
    // the number of sequences that end at or before the row
    s.b = 0;
    for (int i = 0; i < P.batch; i += 64)
      s.b += __popcll(__ballot(i + lane < P.batch && P.offsets[i + lane + 1] <= row));
    s.first = s.end = row;
    if (s.b < P.batch) {
      s.first = P.offsets[s.b];
      s.end = min(P.offsets[s.b + 1], P.rows);
    }
  }
  s.b = __builtin_amdgcn_readfirstlane(s.b);
  s.first = __builtin_amdgcn_readfirstlane(s.first);
  s.end = __builtin_amdgcn_readfirstlane(s.end);
  s.pos = s.b < P.batch && P.positions ? P.positions[s.b] : 0;
  return s;
}

// Physical page of token t of sequence b, or -1 (a token past the table's
// end or a page id out of range: nothing is read or written there).
__device__ __forceinline__ int page_of(const QuantParams& P, int b, int64_t t) {
  if (t < 0 || (t >> P.page_shift) >= P.max_pages) return -1;
  const int pg = P.table[(int64_t)b * P.max_pages + (t >> P.page_shift)];
  return pg >= 0 && pg < P.num_pages ? pg : -1;
}

// Eight values of a row, and the reverse.
template <int DT>
__device__ __forceinline__ void load8(const char* p, float (&x)[8]) {
  if constexpr (DT == ART_ROWS_F32) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
  } else {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == ART_ROWS_BF16) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        const uint32_t u = w[i];   // (a cast of the element itself takes element 0)
        const f16x2 h = __builtin_bit_cast(f16x2, u);
        x[2 * i] = (float)h[0];
        x[2 * i + 1] = (float)h[1];
      }
    }
  }
}
template <int DT>
__device__ __forceinline__ void store8(char* p, const float (&x)[8]) {
  if constexpr (DT == ART_ROWS_F32) {
    reinterpret_cast<f32x4*>(p)[0] = f32x4{x[0], x[1], x[2], x[3]};
    reinterpret_cast<f32x4*>(p)[1] = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 y{x[2 * i], x[2 * i + 1]};
      w[i] = DT == ART_ROWS_BF16 ? __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2))
                                 : __builtin_bit_cast(uint32_t, __builtin_convertvector(y, f16x2));
    }
    *reinterpret_cast<u32x4*>(p) = w;
  }
}

// Four codes in a word, and the reverse.  Rounding is to the nearest code,
// ties to even; |x| beyond the largest code (infinities only) is clamped.
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, float* x) {
  if constexpr (FMT == ART_QUANT_E4M3) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
  } else {
    x[0] = (float)(int8_t)w;
    x[1] = (float)(int8_t)(w >> 8);
    x[2] = (float)(int8_t)(w >> 16);
    x[3] = (float)(int8_t)(w >> 24);
  }
}
template <int FMT>
__device__ __forceinline__ uint32_t encode4(const float* x) {
  float y[4];
  if constexpr (FMT == ART_QUANT_E4M3) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = x[i] != x[i] ? x[i] : fminf(fmaxf(x[i], -448.f), 448.f);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  } else {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = x[i] != x[i] ? 0.f : fminf(fmaxf(x[i], -127.f), 127.f);
      w |= ((uint32_t)(int)rintf(y[i]) & 0xffu) << (8 * i);
    }
    return w;
  }
}

// Bits of the scale that a largest magnitude (its bits) needs: the smallest
// power of two 2^e, e >= -120, with a <= M 2^e.  M is 448 = 1.75 * 2^8 or
// 127 = 1.984375 * 2^6, so e is a's exponent less M's, and one more where a's
// significand is above M's: exact, with no logarithm.
template <int FMT>
__device__ __forceinline__ uint32_t needed_scale(uint32_t a) {
  constexpr int kExp = FMT == ART_QUANT_E4M3 ? 8 : 6;
  constexpr uint32_t kFrac = FMT == ART_QUANT_E4M3 ? 0x600000u : 0x7e0000u;
  int e = (int)(a >> 23) - 127 - kExp + ((a & 0x7fffffu) > kFrac ? 1 : 0);
  e = e < kLowestExp ? kLowestExp : e;
  return (uint32_t)(e + 127) << 23;
}

// Append.  One wavefront quantises one run of slots of one head's K or V: 16
// lanes hold a row (8 values each), four rows at a time.  The first pass over
// the new rows takes their largest magnitude, the second rounds them.  A run
// that a sequence has begun before keeps its scale unless it has to grow;
// only then are its old codes read and rounded anew.
template <int FMT, int DT>
__device__ void append_run(const QuantParams& P, const Side& S, int head, int b, int64_t t, int row, int n, int old,
                           int lane) {
  constexpr int kSize = DT == ART_ROWS_F32 ? 4 : 2;
  const int pg = page_of(P, b, t);
  if (pg < 0) return;
  const int slot = (int)(t & ((1 << P.page_shift) - 1));
  float* sp = S.scale + pg * S.scp + head * S.sch + (slot >> P.run_shift);
  const int r4 = lane >> 4, c = lane & 15;
  const char* src = S.rows + (int64_t)row * S.row + head * S.head + c * (8 * kSize);
  uint8_t* dst = S.codes + pg * S.sp + head * S.sh + c * 8;
  const float old_scale = old > 0 ? *sp : 0.f;

  uint32_t a = 0;
  for (int i = r4; i < n; i += 4) {
    float x[8];
    load8<DT>(src + i * S.row, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t u = __float_as_uint(x[j]) & 0x7fffffffu;
      a = max(a, u < 0x7f800000u ? u : 0u);
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o));
  const float need = __uint_as_float(needed_scale<FMT>(a));
  const float scale = old > 0 ? fmaxf(need, old_scale) : need;
  const float inv = 1.0f / scale;

  if (old > 0 && scale != old_scale) {
    const float ratio = old_scale * inv;
    for (int i = r4; i < old; i += 4) {
      u32x2* p = reinterpret_cast<u32x2*>(dst + (int64_t)(slot - old + i) * S.st);
      u32x2 w = *p;
      float x[8];
      decode4<FMT>(w[0], x);
      decode4<FMT>(w[1], x + 4);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= ratio;
      *p = u32x2{encode4<FMT>(x), encode4<FMT>(x + 4)};
    }
  }
  for (int i = r4; i < n; i += 4) {
    float x[8];
    load8<DT>(src + i * S.row, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= inv;
    *reinterpret_cast<u32x2*>(dst + (int64_t)(slot + i) * S.st) = u32x2{encode4<FMT>(x), encode4<FMT>(x + 4)};
  }
  if (lane == 0 && (old == 0 || scale != old_scale)) *sp = scale;
}

// A wavefront takes the runs whose first new row lies in its window of rows.
template <int FMT, int DT>
__global__ void __launch_bounds__(kThreads) append_kernel(const QuantParams P) {
  const int lane = threadIdx.x & 63;
  const int u = blockIdx.y * kWaves + (threadIdx.x >> 6);
  if (u >= 2 * P.heads) return;
  const Side& S = P.side[u & 1];
  const int head = u >> 1;
  const int run = 1 << P.run_shift;
  const int64_t cap = (int64_t)P.max_pages << P.page_shift;
  int row = blockIdx.x * P.window;
  const int stop = min(row + P.window, P.rows);
  while (row < stop) {
    const Span s = span_of(P, row, lane);
    if (s.b >= P.batch) return;                                    // rows behind the last sequence
    if (s.first > row || s.end <= row) { ++row; continue; }        // before the first one (or no offsets)
    const int64_t t = s.pos + ((int64_t)row - s.first);
    if (s.pos < 0 || t >= cap) { row = s.end; continue; }
    const int in = (int)(t & (run - 1));
    const int left = min(run - in, s.end - row);                   // rows to the run's or the span's end
    if (row == s.first || in == 0) append_run<FMT, DT>(P, S, head, s.b, t, row, left, row == s.first ? in : 0, lane);
    row += left;
  }
}

// Read.  A wavefront brings back eight rows of one head's K or V, eight lanes
// and 16 codes a lane to a row.
template <int FMT, int DT>
__global__ void __launch_bounds__(kThreads) read_kernel(const QuantParams P) {
  constexpr int kSize = DT == ART_ROWS_F32 ? 4 : 2;
  const int lane = threadIdx.x & 63;
  const int u = blockIdx.y * kWaves + (threadIdx.x >> 6);
  if (u >= 2 * P.heads) return;
  const Side& S = P.side[u & 1];
  const int head = u >> 1, c = lane & 7;
  const int row = blockIdx.x * 8 + (lane >> 3);
  Span s = span_of(P, blockIdx.x * 8, lane);
  // lanes whose row lies behind the span go on to their own
  while (P.offsets && s.b < P.batch && row >= s.end) {
    ++s.b;
    if (s.b < P.batch) {
      s.first = P.offsets[s.b];
      s.end = max(s.end, min(P.offsets[s.b + 1], P.rows));
      s.pos = P.positions ? P.positions[s.b] : 0;
    }
  }
  if (!P.offsets && P.per_seq > 0) {
    s.b = row / P.per_seq;
    s.first = s.b * P.per_seq;
    s.pos = s.b < P.batch && P.positions ? P.positions[s.b] : 0;
  }
  if (row >= P.rows || s.b >= P.batch || s.pos < 0 || s.first < 0 || row < s.first) return;
  const int64_t t = s.pos + ((int64_t)row - s.first);
  const int pg = page_of(P, s.b, t);
  if (pg < 0) return;
  const int slot = (int)(t & ((1 << P.page_shift) - 1));
  const float scale = S.scale[pg * S.scp + head * S.sch + (slot >> P.run_shift)];
  const u32x4 w = *reinterpret_cast<const u32x4*>(S.codes + pg * S.sp + head * S.sh + slot * S.st + c * 16);
  char* dst = S.rows + (int64_t)row * S.row + head * S.head + c * (16 * kSize);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float x[8];
    decode4<FMT>(w[2 * h], x);
    decode4<FMT>(w[2 * h + 1], x + 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= scale;
    store8<DT>(dst + h * 8 * kSize, x);
  }
}

int log2_of(int64_t v) {
  int s = 0;
  while ((int64_t(1) << s) < v) ++s;
  return s;
}
bool pow2(int64_t v) { return v > 0 && (v & (v - 1)) == 0; }

}  // namespace

art_status check_quant(const art_decode_shape* s, const art_quant_cache* c) {
  if (!s || !c) return ART_ERR_INVALID_ARG;
  if (s->batch < 0 || s->num_kv_heads <= 0 || s->head_dim <= 0 || s->page_size <= 0 || s->num_pages <= 0 ||
      s->max_pages_per_seq <= 0 || s->k_stride_page < 0 || s->k_stride_head < 0 || s->k_stride_token < 0 ||
      s->v_stride_page < 0 || s->v_stride_head < 0 || s->v_stride_token < 0)
    return ART_ERR_INVALID_ARG;
  if ((c->format != ART_QUANT_E4M3 && c->format != ART_QUANT_INT8) || c->scale_tokens <= 0 ||
      c->k_scale_stride_page < 0 || c->k_scale_stride_head < 0 || c->v_scale_stride_page < 0 ||
      c->v_scale_stride_head < 0)
    return ART_ERR_INVALID_ARG;
  if (s->head_dim != kHeadDim || !pow2(s->page_size) || s->page_size < 16) return ART_ERR_UNSUPPORTED;
  if (!pow2(c->scale_tokens) || c->scale_tokens < 16 || c->scale_tokens > s->page_size) return ART_ERR_UNSUPPORTED;
  if ((s->k_stride_page | s->k_stride_head | s->k_stride_token | s->v_stride_page | s->v_stride_head |
       s->v_stride_token) % 16 ||
      s->k_stride_token >= (1 << 24) || s->v_stride_token >= (1 << 24))
    return ART_ERR_UNSUPPORTED;
  return ART_OK;
}

namespace {

// Host checks of a call, and its kernel parameters.
art_status check_rows(const art_decode_shape* s, const art_quant_cache* c, const art_quant_rows* r, const void* k_rows,
                      const void* v_rows, const int32_t* offsets, const int32_t* positions, const int32_t* table,
                      const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                      bool append, QuantParams* p) {
  const art_status st = check_quant(s, c);
  if (st != ART_OK) return st;
  if (!r || r->rows < 0 || r->rows_dtype < ART_ROWS_BF16 || r->rows_dtype > ART_ROWS_F32 || r->k_stride_row < 0 ||
      r->k_stride_head < 0 || r->v_stride_row < 0 || r->v_stride_head < 0)
    return ART_ERR_INVALID_ARG;
  if (append && c->scale_tokens > kMaxRun) return ART_ERR_UNSUPPORTED;
  if (!offsets && s->batch > 0 && r->rows % s->batch) return ART_ERR_INVALID_ARG;
  const int64_t size = r->rows_dtype == ART_ROWS_F32 ? 4 : 2;
  if ((r->k_stride_row | r->k_stride_head | r->v_stride_row | r->v_stride_head) * size % 16) return ART_ERR_UNSUPPORTED;
  // the grid's dimensions: threads along the first (at most 2^32) and
  // workgroups along the second
  if (r->rows >= (1 << 24) || s->num_kv_heads > 65536) return ART_ERR_UNSUPPORTED;
  if (s->batch == 0 || r->rows == 0) return ART_OK;
  if (!k_rows || !v_rows || !table || !k_cache || !v_cache || !k_scale || !v_scale) return ART_ERR_INVALID_ARG;
  if (((uintptr_t)k_scale | (uintptr_t)v_scale) % 4) return ART_ERR_INVALID_ARG;
  if (((uintptr_t)k_rows | (uintptr_t)v_rows | (uintptr_t)k_cache | (uintptr_t)v_cache) % 16) return ART_ERR_UNSUPPORTED;
  memset(p, 0, sizeof *p);
  p->batch = s->batch;
  p->heads = s->num_kv_heads;
  p->rows = r->rows;
  p->per_seq = r->rows / s->batch;
  p->page_shift = log2_of(s->page_size);
  p->run_shift = log2_of(c->scale_tokens);
  p->num_pages = s->num_pages;
  p->max_pages = s->max_pages_per_seq;
  p->offsets = offsets;
  p->positions = positions;
  p->table = table;
  p->side[0] = Side{(char*)k_rows, r->k_stride_row * size, r->k_stride_head * size, (uint8_t*)k_cache,
                    s->k_stride_page, s->k_stride_head, s->k_stride_token, (float*)k_scale,
                    c->k_scale_stride_page, c->k_scale_stride_head};
  p->side[1] = Side{(char*)v_rows, r->v_stride_row * size, r->v_stride_head * size, (uint8_t*)v_cache,
                    s->v_stride_page, s->v_stride_head, s->v_stride_token, (float*)v_scale,
                    c->v_scale_stride_page, c->v_scale_stride_head};
  return ART_OK;
}

template <int FMT>
void launch_append(const QuantParams& p, int dtype, dim3 grid, hipStream_t stream) {
  auto k = dtype == ART_ROWS_BF16  ? append_kernel<FMT, ART_ROWS_BF16>
           : dtype == ART_ROWS_F16 ? append_kernel<FMT, ART_ROWS_F16>
                                   : append_kernel<FMT, ART_ROWS_F32>;
  hipLaunchKernelGGL(k, grid, dim3(kThreads), 0, stream, p);
}
template <int FMT>
void launch_read(const QuantParams& p, int dtype, dim3 grid, hipStream_t stream) {
  auto k = dtype == ART_ROWS_BF16  ? read_kernel<FMT, ART_ROWS_BF16>
           : dtype == ART_ROWS_F16 ? read_kernel<FMT, ART_ROWS_F16>
                                   : read_kernel<FMT, ART_ROWS_F32>;
  hipLaunchKernelGGL(k, grid, dim3(kThreads), 0, stream, p);
}

}  // namespace
}  // namespace art

extern "C" {

art_status art_quant_append(const art_decode_shape* shape, const art_quant_cache* cache, const art_quant_rows* rows,
                            const void* k_rows, const void* v_rows, const int32_t* row_offsets,
                            const int32_t* positions, const int32_t* page_table, void* k_cache, void* v_cache,
                            float* k_scale, float* v_scale, hipStream_t stream) {
  using namespace art;
  QuantParams p;
  const art_status st = check_rows(shape, cache, rows, k_rows, v_rows, row_offsets, positions, page_table, k_cache,
                                   v_cache, k_scale, v_scale, true, &p);
  if (st != ART_OK || shape->batch == 0 || rows->rows == 0) return st;
  // as many rows to a window as a sequence has on average (a power of two of
  // at most a run): a window then starts about one run
  int window = 1;
  while (window < cache->scale_tokens && window * 2 <= p.per_seq) window *= 2;
  p.window = window;
  const dim3 grid((unsigned)((p.rows + window - 1) / window), (unsigned)((2 * p.heads + kWaves - 1) / kWaves));
  if (cache->format == ART_QUANT_E4M3)
    launch_append<ART_QUANT_E4M3>(p, rows->rows_dtype, grid, stream);
  else
    launch_append<ART_QUANT_INT8>(p, rows->rows_dtype, grid, stream);
  return hipGetLastError() == hipSuccess ? ART_OK : ART_ERR_HIP;
}

art_status art_quant_read(const art_decode_shape* shape, const art_quant_cache* cache, const art_quant_rows* rows,
                          const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                          const int32_t* row_offsets, const int32_t* positions, const int32_t* page_table,
                          void* k_rows, void* v_rows, hipStream_t stream) {
  using namespace art;
  QuantParams p;
  const art_status st = check_rows(shape, cache, rows, k_rows, v_rows, row_offsets, positions, page_table, k_cache,
                                   v_cache, k_scale, v_scale, false, &p);
  if (st != ART_OK || shape->batch == 0 || rows->rows == 0) return st;
  const dim3 grid((unsigned)((p.rows + 7) / 8), (unsigned)((2 * p.heads + kWaves - 1) / kWaves));
  if (cache->format == ART_QUANT_E4M3)
    launch_read<ART_QUANT_E4M3>(p, rows->rows_dtype, grid, stream);
  else
    launch_read<ART_QUANT_INT8>(p, rows->rows_dtype, grid, stream);
  return hipGetLastError() == hipSuccess ? ART_OK : ART_ERR_HIP;
}

}  // extern "C"
