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

// The offsets and positions of up to 64 sequences, lane i those of sequence i,
// read once and together (a row's span then costs no further round trip).
struct SpanTable {
  int begin, end, pos;
};
__device__ __forceinline__ SpanTable span_table(const QuantParams& P, int lane) {
  SpanTable t{0, 0, 0};
  if (P.offsets && P.batch <= 64 && lane < P.batch) {
    t.begin = P.offsets[lane];
    t.end = P.offsets[lane + 1];
    t.pos = P.positions ? P.positions[lane] : 0;
  }
  return t;
}

__device__ __forceinline__ Span span_of(const QuantParams& P, const SpanTable& t, int row, int lane) {
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
__device__ __forceinline__ int page_of(const QuantParams& P, int b, int64_t t) {
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
// The largest magnitude, as bits of the rows' type without their sign: two
// 16-bit values at a time where the rows have them.  Bits of kNotFinite and
// above are infinities and NaN.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <int DT>
constexpr uint32_t kNotFinite = DT == ART_ROWS_F32 ? 0x7f800000u : DT == ART_ROWS_BF16 ? 0x7f80u : 0x7c00u;
template <int DT>
__device__ __forceinline__ uint32_t max_bits(uint32_t a, const u32x4& r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == ART_ROWS_F32) {
      a = max(a, r[i] & 0x7fffffffu);
    } else {
      const uint32_t w = r[i] & 0x7fff7fffu;
      a = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, w)));
    }
  }
  return a;
}
template <int DT>
__device__ __forceinline__ uint32_t as_f32_bits(uint32_t a) {
  if constexpr (DT == ART_ROWS_F32) return a;
  else if constexpr (DT == ART_ROWS_BF16) return a << 16;
  else return __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)a));
}
// ... of the finite values only, in fp32 bits
template <int DT>
__device__ __forceinline__ uint32_t max_finite_bits(uint32_t a, const u32x4& r) {
#pragma unroll
  for (int i = 0; i < kValues<DT>; ++i) {
    const uint32_t u = __float_as_uint(value<DT>(r, i)) & 0x7fffffffu;
    a = max(a, u < 0x7f800000u ? u : 0u);
  }
  return a;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t a) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o));
  return a;
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

// Four codes in a word, and the reverse.  Rounding is to the nearest code,
// ties to even.  WILD: the values may lie beyond the largest code or be NaN.
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
template <int FMT, bool WILD>
__device__ __forceinline__ uint32_t encode4(const float* x) {
  float y[4];
  if constexpr (FMT == ART_QUANT_E4M3) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = !WILD || x[i] != x[i] ? x[i] : fminf(fmaxf(x[i], -448.f), 448.f);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  } else {
    // |y| <= 127: adding 1.5 * 2^23 rounds to the nearest integer, ties to
    // even, whose two's complement then is the sum's low byte
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = !WILD ? x[i] : x[i] != x[i] ? 0.f : fminf(fmaxf(x[i], -127.f), 127.f);
      u[i] = __float_as_uint(__fadd_rn(y[i], 12582912.f));
    }
    const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u);
    return lo | hi << 16;
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

// Runs whose scale is no power of two (a cache that another writer began): the
// quotients and products are not exact in fp32, and rounding them there first
// could turn a value next to the midpoint of two codes into the midpoint.
// 64 bits hold them well enough (the quotient of two fp32 values that is not a
// midpoint lies 2^-29 of itself away from it, or more), and fp32 values rounded
// to odd (the neighbour with a set last bit, where the value is inexact) still
// tell which side of a midpoint they lie on.
__device__ __forceinline__ float odd_f32(double x) {
  const float f = (float)x;
  if ((double)f == x || x != x) return f;
  uint32_t u = __float_as_uint(f);
  if (fabs((double)f) > fabs(x)) --u;   // towards zero
  return __uint_as_float(u | 1u);
}
// x / s, inv = 1 / s rounded: one Newton step makes exact quotients exact.
__device__ __forceinline__ float quotient(float x, double s, double inv) {
  const double q = (double)x * inv, r = __builtin_fma(-q, s, (double)x);
  return odd_f32(fabs(r) > 0.0 ? __builtin_fma(r, inv, q) : q);   // (infinite x, or -0: q)
}
__device__ __forceinline__ bool power_of_two(float s) { return (__float_as_uint(s) & 0x7fffffu) == 0; }

// Append.  One wavefront quantises one run of slots of one head's K or V: 16
// bytes of a row to a lane, four rows a step (two of 32-bit values), and 64
// rows stay in registers (of fp32 rows, 128 registers, 4 to 6 in scratch) between
// the pass that takes their largest magnitude and the one that rounds them.  Longer runs have a workgroup each, whose
// wavefronts take the steps in turn and join their maxima in LDS.  A run that a
// sequence has begun before keeps its scale unless it has to grow; only then
// are its old codes read and rounded anew.
//
// The bound is HBM: rows read once and codes written once.  54K rows of 8
// heads, K and V: 68 us in bf16 (4.9 TB/s; 88 with loads that go through the
// caches), and 48K rows of fp32 93 us (5.3 TB/s; 184 with 32 rows in
// registers).  48K bf16 rows in runs of 256: 55 us (one wavefront a run: 137).
// Appends of a few rows a sequence are bound by the chain of lookups (offsets,
// position, page, rows) and want many wavefronts: with 4 steps in registers
// instead of 16, 4096 sequences of one token take 51 us instead of 80, and 8 of
// one 3.0 instead of 3.9; a long run among them has its rows read twice.
template <int DT>
struct Step {
  static constexpr int SLAB = DT == ART_ROWS_F32 ? 32 : 16;   // steps in registers, of long spans
  static constexpr int SHORT = 4;                             // ... of short ones
  static constexpr int LANES = kHeadDim / kValues<DT>;   // lanes of a row
  static constexpr int ROWS = 64 / LANES;                // rows of a step
};

template <int FMT, int DT, bool WILD>
__device__ __forceinline__ void store_codes(uint8_t* p, const u32x4& r, float inv) {
  float x[kValues<DT>];
#pragma unroll
  for (int i = 0; i < kValues<DT>; ++i) x[i] = value<DT>(r, i) * inv;
  if constexpr (kValues<DT> == 8)
    *reinterpret_cast<u32x2*>(p) = u32x2{encode4<FMT, WILD>(x), encode4<FMT, WILD>(x + 4)};
  else
    *reinterpret_cast<uint32_t*>(p) = encode4<FMT, WILD>(x);
}
template <int FMT, int DT>
__device__ __forceinline__ void store_quotients(uint8_t* p, const u32x4& r, double scale, double inv) {
  float x[kValues<DT>];
#pragma unroll
  for (int i = 0; i < kValues<DT>; ++i) x[i] = quotient(value<DT>(r, i), scale, inv);
#pragma unroll
  for (int q = 0; q < kValues<DT> / 4; ++q) reinterpret_cast<uint32_t*>(p)[q] = encode4<FMT, true>(x + 4 * q);
}

// What a team's wavefronts (4 of a run longer than one holds, or 1) tell each
// other of a run: their largest magnitudes, and the run's scale so far.
struct Team {
  uint32_t top[2][kWaves];
  float scale[2];
};

// The run's new rows are n from token t on, row `row` the first of them;
// `old` slots of the run were written before.  Uniform over a team, which takes
// the steps in turn; `turn` counts the team's exchanges (two buffers, as the
// next one may begin while a wavefront still reads the last).
template <int FMT, int DT, int kSlab, int TEAM>
__device__ void append_run(const QuantParams& P, const Side& S, int head, int b, int64_t t, int row, int n, int old,
                           int lane, int wave, Team* team, int& turn) {
  constexpr int ROWS = Step<DT>::ROWS, LANES = Step<DT>::LANES, EACH = ROWS * TEAM;
  // uniform bases and 32-bit lane offsets; the rows are on their way before
  // the page is known (they need none)
  const int r0 = lane / LANES, c = lane % LANES, mine = wave * ROWS;
  const char* src = S.rows + ((int64_t)row + mine) * S.row + head * S.head;
  const uint32_t from = (uint32_t)(r0 * (int)S.row) + c * 16, to = (uint32_t)(r0 * (int)S.st) + c * kValues<DT>;
  n -= mine;   // rows from this wavefront's first one on
  auto load = [&](int i) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + (int64_t)i * S.row + from)); };  // row i + r0
  const int page = page_of(P, b, t);
  u32x4 raw[kSlab];
  const bool held = n + mine <= kSlab * EACH;
  if (held) {
#pragma unroll
    for (int k = 0; k < kSlab; ++k) {
      raw[k] = u32x4{0u, 0u, 0u, 0u};
      if (EACH * k + r0 < n) raw[k] = load(EACH * k);
    }
  }
  const int pg = __builtin_amdgcn_readfirstlane(page);
  if (pg < 0) return;
  const int slot = (int)(t & ((1 << P.page_shift) - 1));
  float* sp = S.scale + pg * S.scp + head * S.sch + (slot >> P.run_shift);
  uint8_t* pool = S.codes + pg * S.sp + head * S.sh + slot * S.st;
  auto at = [&](int i) { return pool + ((int64_t)i + mine) * S.st + to; };
  // one wavefront of a team reads the scale, and writes it only after all know it
  float old_scale = old > 0 && wave == 0 ? *sp : 0.f;
  auto joined = [&](uint32_t a) {
    a = wave_max(a);
    if constexpr (TEAM > 1) {
      const int e = turn++ & 1;
      if (lane == 0) {
        team->top[e][wave] = a;
        if (wave == 0) team->scale[e] = old_scale;
      }
      __syncthreads();
      old_scale = team->scale[e];
#pragma unroll
      for (int i = 0; i < TEAM; ++i) a = max(a, team->top[e][i]);
      a = __builtin_amdgcn_readfirstlane(a);
    }
    return a;
  };

  // the run's scale from its new rows' largest finite magnitude (fp32 bits);
  // old codes follow it where it grows (to a power of two)
  auto settle = [&](uint32_t top) {
    const float need = __uint_as_float(needed_scale<FMT>(top));
    const float scale = old > 0 ? fmaxf(need, old_scale) : need;
    if (old > 0 && scale != old_scale) {
      const double ratio = (double)old_scale / (double)scale;
      for (int i = wave * 8 + (lane >> 3); i < old; i += 8 * TEAM) {
        u32x4* p = reinterpret_cast<u32x4*>(pool + (int64_t)(i - old) * S.st + (lane & 7) * 16);
        u32x4 w = *p;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x[4];
          decode4<FMT>(w[q], x);
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = odd_f32((double)x[j] * ratio);
          w[q] = encode4<FMT, true>(x);
        }
        *p = w;
      }
    }
    if (wave == 0 && lane == 0 && (old == 0 || scale != old_scale)) *sp = scale;
    return scale;
  };
  float scale = 0.f;
  if (held) {
    uint32_t a = 0;
#pragma unroll
    for (int k = 0; k < kSlab; ++k) a = max_bits<DT>(a, raw[k]);
    if constexpr (DT != ART_ROWS_F32) a = max(a & 0xffffu, a >> 16);
    a = joined(a);
    if (a < kNotFinite<DT>) {
      scale = settle(as_f32_bits<DT>(a));
      if (power_of_two(scale)) {
        const float inv = 1.0f / scale;
#pragma unroll
        for (int k = 0; k < kSlab; ++k) {
          if (EACH * k + r0 < n) store_codes<FMT, DT, false>(at(EACH * k), raw[k], inv);
        }
        return;
      }
    }
  }
  // more rows than the registers hold, infinities or NaN among them, or a kept
  // scale that is no power of two: the largest finite magnitude, then codes with
  // clamps, from the rows once more
  if (scale == 0.f) {
    uint32_t a = 0;
#pragma unroll 4
    for (int i = 0; i < n; i += EACH)
      if (i + r0 < n) a = max_finite_bits<DT>(a, load(i));
    scale = settle(joined(a));
  }
  if (power_of_two(scale)) {
    const float inv = 1.0f / scale;
#pragma unroll 4
    for (int i = 0; i < n; i += EACH)
      if (i + r0 < n) store_codes<FMT, DT, true>(at(i), load(i), inv);
  } else {
    const double inv = 1.0 / (double)scale;
#pragma unroll 1
    for (int i = 0; i < n; i += EACH)
      if (i + r0 < n) store_quotients<FMT, DT>(at(i), load(i), (double)scale, inv);
  }
}

// A wavefront, or a team, takes the runs whose first new row lies in its window
// of rows.
template <int FMT, int DT, int SLAB, int TEAM>
__global__ void __launch_bounds__(kThreads, SLAB == Step<DT>::SHORT ? 6 : 3) append_kernel(const QuantParams P) {
  static_assert(TEAM == 1 || (TEAM == kWaves && SLAB * Step<DT>::ROWS * TEAM >= kMaxRun));
  __shared__ Team team;
  constexpr int kSlices = kWaves / TEAM;   // heads of K or V in a workgroup
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t slices = (uint32_t)(2 * P.heads + kSlices - 1) / kSlices, part = blockIdx.x / slices;
  const int u = (blockIdx.x - part * slices) * kSlices + (TEAM > 1 ? 0 : wave);
  if (u >= 2 * P.heads) return;
  const Side& S = P.side[u >= P.heads ? 1 : 0];
  const int head = u >= P.heads ? u - P.heads : u;
  const int run = 1 << P.run_shift;
  const int64_t cap = (int64_t)P.max_pages << P.page_shift;
  int row = part * P.window, turn = 0;
  const int stop = min(row + P.window, P.rows);
  const SpanTable table = span_table(P, lane);
  Span s{0, 0, 0, 0};
  while (row < stop) {
    if (row >= s.end) s = span_of(P, table, row, lane);
    if (s.b >= P.batch) return;                                    // rows behind the last sequence
    if (s.first > row || s.end <= row) { ++row; continue; }        // before the first one (or no offsets)
    const int64_t t = s.pos + ((int64_t)row - s.first);
    if (s.pos < 0 || t >= cap) { row = s.end; continue; }
    const int in = (int)(t & (run - 1));
    const int left = min(run - in, s.end - row);                   // rows to the run's or the span's end
    if (row == s.first || in == 0)
      append_run<FMT, DT, SLAB, TEAM>(P, S, head, s.b, t, row, left, row == s.first ? in : 0, lane, TEAM > 1 ? wave : 0,
                                      &team, turn);
    row += left;
  }
}

// Read.  A wavefront brings back 8 steps of 4 rows (of 2 rows of 32-bit values)
// of one head's K or V: the page lookups of all of them, then their scales and
// codes, are in flight together.  A lane takes the codes that one 16-byte
// store holds the values of, so that a store instruction writes whole rows: 54K
// rows of 8 heads to fp32 take 101 us and 103K rows to bf16 121 (with 16 codes a
// lane 182 and 132, when this form took 106 and 126).  The wavefronts of a workgroup take
// neighbouring heads, whose parts of a row lie side by side, and neighbouring
// workgroups the rest of the row: all of a row moves at about the same time
// and meets every memory channel (with the heads far apart in the launch, fp32
// 121 us where this form took 107, and the append 110 where it took 88).
template <int DT>
struct ReadCfg {
  static constexpr int CODES = kValues<DT>;        // codes of a lane
  static constexpr int LANES = kHeadDim / CODES;   // lanes of a row
  static constexpr int ROWS = 64 / LANES;          // rows of a step
  static constexpr int STEPS = 8;                  // steps of a long read
};

template <int FMT, int DT, int STEPS>
__global__ void __launch_bounds__(kThreads) read_kernel(const QuantParams P) {
  using C = ReadCfg<DT>;
  const int lane = threadIdx.x & 63;
  const uint32_t slices = (uint32_t)(2 * P.heads + kWaves - 1) / kWaves, part = blockIdx.x / slices;
  const int u = (blockIdx.x - part * slices) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (u >= 2 * P.heads) return;
  const Side& S = P.side[u >= P.heads ? 1 : 0];
  const int head = u >= P.heads ? u - P.heads : u, c = lane % C::LANES;
  const int row0 = part * (C::ROWS * STEPS), in_step = lane / C::LANES;
  const SpanTable table = span_table(P, lane);
  Span s = span_of(P, table, row0, lane);
  int b[STEPS];
  int64_t t[STEPS];
  const int stop = min(row0 + C::ROWS * STEPS, P.rows);
  if (s.first <= row0 && stop <= s.end && s.pos >= 0) {   // all rows are one sequence's
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const int row = row0 + C::ROWS * k + in_step;
      b[k] = s.b;
      t[k] = row < stop ? s.pos + ((int64_t)row - s.first) : -1;
    }
  } else {
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      // the spans that the step's rows belong to, one after the other
      const int first = row0 + C::ROWS * k, last = min(first + C::ROWS, P.rows), row = first + in_step;
      b[k] = 0;
      t[k] = -1;
      for (int r = first; r < last;) {
        if (r >= s.end) s = span_of(P, table, r, lane);
        if (s.b >= P.batch) break;                                             // rows behind the last sequence
        if (s.first > r || s.end <= r) { r = max(r + 1, s.first); continue; }  // before the first one (or no offsets)
        if (row >= r && row < s.end && s.pos >= 0) {
          b[k] = s.b;
          t[k] = s.pos + ((int64_t)row - s.first);
        }
        r = s.end;
      }
      if (row >= last) t[k] = -1;
    }
  }
  int pg[STEPS], slot[STEPS];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    pg[k] = page_of(P, b[k], t[k]);
    slot[k] = (int)(t[k] & ((1 << P.page_shift) - 1));
  }
  float scale[STEPS];
  uint32_t w[STEPS][C::CODES / 4];
#pragma unroll
  for (int k = 0; k < STEPS; ++k)
    if (pg[k] >= 0) {
      scale[k] = S.scale[pg[k] * S.scp + head * S.sch + (slot[k] >> P.run_shift)];
      const uint8_t* src = S.codes + pg[k] * S.sp + head * S.sh + slot[k] * S.st + c * C::CODES;
      if constexpr (C::CODES == 8) {
        const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(src));
        w[k][0] = x[0];
        w[k][1] = x[1];
      } else {
        w[k][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(src));
      }
    }
#pragma unroll
  for (int k = 0; k < STEPS; ++k)
    if (pg[k] >= 0) {
      float x[C::CODES];
#pragma unroll
      for (int q = 0; q < C::CODES / 4; ++q) decode4<FMT>(w[k][q], x + 4 * q);
#pragma unroll
      for (int j = 0; j < C::CODES; ++j) x[j] *= scale[k];
      char* dst = S.rows + (int64_t)(row0 + C::ROWS * k + in_step) * S.row + head * S.head + c * 16;
      *reinterpret_cast<u32x4*>(dst) = packed<DT, C::CODES>(x);
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
  if ((r->k_stride_row | r->k_stride_head | r->v_stride_row | r->v_stride_head) * size % 16 ||
      r->k_stride_row * size >= (1 << 28) || r->v_stride_row * size >= (1 << 28))
    return ART_ERR_UNSUPPORTED;
  // a launch has less than 2^32 threads: 256 for every row and four slices
  if (r->rows >= (1 << 24) || (int64_t)r->rows * ((2 * (int64_t)s->num_kv_heads + kWaves - 1) / kWaves) >= (1 << 24))
    return ART_ERR_UNSUPPORTED;
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

template <int FMT, int DT>
void launch_append(const QuantParams& p, hipStream_t stream) {
  constexpr int kShort = Step<DT>::SHORT, kSlab = Step<DT>::SLAB;
  // few rows a sequence: few of them in registers, which leaves room for twice
  // the wavefronts; runs longer than a wavefront holds: a workgroup for each
  const bool brief = p.window <= 4, team = !brief && (1 << p.run_shift) > kSlab * Step<DT>::ROWS;
  auto k = brief  ? append_kernel<FMT, DT, kShort, 1>
           : team ? append_kernel<FMT, DT, kSlab, kWaves>
                  : append_kernel<FMT, DT, kSlab, 1>;
  const int64_t slices = team ? 2 * (int64_t)p.heads : (2 * (int64_t)p.heads + kWaves - 1) / kWaves;
  const dim3 grid((unsigned)(((int64_t)p.rows + p.window - 1) / p.window * slices));
  hipLaunchKernelGGL(k, grid, dim3(kThreads), 0, stream, p);
}
template <int FMT>
void launch_append(const QuantParams& p, int dtype, hipStream_t stream) {
  if (dtype == ART_ROWS_BF16) launch_append<FMT, ART_ROWS_BF16>(p, stream);
  else if (dtype == ART_ROWS_F16) launch_append<FMT, ART_ROWS_F16>(p, stream);
  else launch_append<FMT, ART_ROWS_F32>(p, stream);
}
template <int FMT, int DT>
void launch_read(const QuantParams& p, hipStream_t stream) {
  using C = ReadCfg<DT>;
  // several steps a wavefront where that still leaves the chip 16 wavefronts a
  // CU, one otherwise (522 rows of 4 heads in 32 bits: 4.6 us with one step)
  const int64_t slices = (int64_t)2 * p.heads, rows = C::ROWS * C::STEPS;
  const bool many = (p.rows + rows - 1) / rows * slices >= 16 * 256;
  const int64_t each = many ? rows : C::ROWS;
  const dim3 grid((unsigned)((p.rows + each - 1) / each * ((slices + kWaves - 1) / kWaves)));
  auto k = many ? read_kernel<FMT, DT, C::STEPS> : read_kernel<FMT, DT, 1>;
  hipLaunchKernelGGL(k, grid, dim3(kThreads), 0, stream, p);
}
template <int FMT>
void launch_read(const QuantParams& p, int dtype, hipStream_t stream) {
  if (dtype == ART_ROWS_BF16) launch_read<FMT, ART_ROWS_BF16>(p, stream);
  else if (dtype == ART_ROWS_F16) launch_read<FMT, ART_ROWS_F16>(p, stream);
  else launch_read<FMT, ART_ROWS_F32>(p, stream);
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
  if (cache->format == ART_QUANT_E4M3)
    launch_append<ART_QUANT_E4M3>(p, rows->rows_dtype, stream);
  else
    launch_append<ART_QUANT_INT8>(p, rows->rows_dtype, stream);
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
  if (cache->format == ART_QUANT_E4M3)
    launch_read<ART_QUANT_E4M3>(p, rows->rows_dtype, stream);
  else
    launch_read<ART_QUANT_INT8>(p, rows->rows_dtype, stream);
  return hipGetLastError() == hipSuccess ? ART_OK : ART_ERR_HIP;
}

}  // extern "C"
