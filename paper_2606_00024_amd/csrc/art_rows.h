// Rows packed over the sequences of a batch, shared by the kernels that read
// or write them: a row's sequence and place, pages, and 16-byte pieces of rows.
// Params is a call's parameter structure; the fields used are batch, rows,
// per_seq, offsets and positions, and for pages page_shift, num_pages, max_pages
// and table.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "art.h"

namespace art {

// Host checks of a bf16 cache's page and stride fields (art_rope.hip).
art_status check_cache(const art_decode_shape* shape);

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Where a row belongs: sequence b holds rows [first, end) from token `pos` on.
// b == batch: no sequence.
struct Span {
  int b, first, end;
  int64_t pos;
};

// The offsets and positions of up to 64 sequences, lane i those of sequence i,
// read once and together (a row's span then costs no further round trip).
struct SpanTable {
  int begin, end, pos;
};
template <class Params>
__device__ __forceinline__ SpanTable span_table(const Params& P, int lane) {
  SpanTable t{0, 0, 0};
  if (P.offsets && P.batch <= 64 && lane < P.batch) {
    t.begin = P.offsets[lane];
    t.end = P.offsets[lane + 1];
    t.pos = P.positions ? P.positions[lane] : 0;
  }
  return t;
}

template <class Params>
__device__ __forceinline__ Span span_of(const Params& P, const SpanTable& t, int row, int lane) {
  Span s;
  if (P.offsets && P.batch <= 64) {
    // the number of sequences that end at or before the row
    s.b = __popcll(__ballot(lane < P.batch && t.end <= row));
    const int at = min(s.b, 63);
    s.first = __builtin_amdgcn_readlane(t.begin, at);
    s.end = min(__builtin_amdgcn_readlane(t.end, at), P.rows);
    s.pos = __builtin_amdgcn_readlane(t.pos, at);
    if (s.b >= P.batch) s.first = s.end = row;
    return s;
  }
  if (!P.offsets) {
    s.b = P.per_seq > 0 ? row / P.per_seq : P.batch;
    s.first = s.b * P.per_seq;
    s.end = s.first + P.per_seq;
  } else {
    // 64 places a step: each narrows the range to one 64th
    int n = P.batch;
    s.b = 0;
    while (n > 64) {
      const int each = (n + 63) / 64, at = (lane + 1) * each;   // sequences s.b + at - each .. s.b + at - 1
      const int c = __popcll(__ballot(at <= n && P.offsets[s.b + at] <= row)) * each;
      s.b += c;
      n = min(each, n - c);
    }
    s.b += __popcll(__ballot(lane < n && P.offsets[s.b + lane + 1] <= row));
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
template <class Params>
__device__ __forceinline__ int page_of(const Params& P, int b, int64_t t) {
  if (t < 0 || (t >> P.page_shift) >= P.max_pages) return -1;
  const int pg = P.table[(int64_t)b * P.max_pages + (t >> P.page_shift)];
  return pg >= 0 && pg < P.num_pages ? pg : -1;
}

// Sixteen bytes of a row: 8 values, or 4.
template <int DT>
constexpr int kValues = DT == ART_ROWS_F32 ? 4 : 8;
template <int DT>
__device__ __forceinline__ float value(const u32x4& w, int i) {
  if constexpr (DT == ART_ROWS_F32) {
    const uint32_t u = w[i];
    return __uint_as_float(u);
  } else {
    const uint32_t u = w[i >> 1];   // (a cast of the element itself takes element 0)
    if constexpr (DT == ART_ROWS_BF16) {
      return __uint_as_float(i & 1 ? u & 0xffff0000u : u << 16);
    } else {
      const f16x2 h = __builtin_bit_cast(f16x2, u);
      return (float)h[i & 1];
    }
  }
}
// N values (16 bytes of the rows' type).
template <int DT, int N>
__device__ __forceinline__ u32x4 packed(const float (&x)[N]) {
  u32x4 w;
  if constexpr (DT == ART_ROWS_F32) {
    static_assert(N == 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
  } else {
    static_assert(N == 8);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 y{x[2 * i], x[2 * i + 1]};
      w[i] = DT == ART_ROWS_BF16 ? __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2))
                                 : __builtin_bit_cast(uint32_t, __builtin_convertvector(y, f16x2));
    }
  }
  return w;
}

}  // namespace
}  // namespace art
