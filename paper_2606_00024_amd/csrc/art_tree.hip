// Attention of drafted tokens over a paged bf16 cache (art_tree_attention).
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(c q.k_j - m),  c = scale log2 e
//
// over the tokens j that a row sees: the context, and of its sequence's nodes
// those in its mask (or the earlier ones and itself).
//
// The rows of a sequence's nodes that share a KV head lie together: a row tile is
// as many whole nodes as fit kRows rows.  Row tiles of all sequences and heads are
// the units of work; a unit has a tile of 64 or 128 tokens after the other to go
// through.  The tiles of all units, LEAD places for each unit's set-up in front
// of them, form one line, and every workgroup takes an equal, contiguous part of
// it, however ragged the batch is.  A unit that lies in one workgroup is written
// there; of the others each workgroup leaves a record (o, m, l) in the workspace
// and a second, small launch joins them in the order of the line.
//
// Scores are computed transposed, S^T = K Q^T, by 32x32x16 matrix instructions: a
// lane then holds 16 tokens' scores of one row, so that maximum and sum need no
// other lane but its partner 32 further, and the probabilities are, as they lie,
// the B operand of O^T = V^T P^T.
//
// Up to 64 rows of a sequence share a KV head's keys (eight nodes of eight heads):
// the memory is the bound, and a tile is loaded into LDS while the one before is in
// work.  8 x 32K tokens, 32/8 heads, 16 nodes each: 200 us, 5.4 TB/s of 6.1 that a
// plain read reaches; 32 ragged sequences of 8K to 64K, 64/8 heads, 8 nodes: 759 us,
// 5.8 TB/s.  From 128 rows on the matrix cores are: 4096 prompt tokens each behind
// 16K, 32/8 heads, run at 1.05 PFLOP/s, where a large matrix product runs at 1.62.
// There a wavefront's matrix and vector instructions are interleaved by hand (the
// scores' products with the exponentials of the tile before), two wavefronts to a
// SIMD: in a loop of such instructions alone, one matrix instruction of 16 ns with five
// multiply-adds and two exponentials takes 21.  Rows by 64 to a wavefront, which
// halves what LDS gives, had one wavefront to a SIMD and ran at 0.94 PFLOP/s.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "art.h"
#include "art_internal.h"
#include "art_rows.h"
#include "art_wave.h"

namespace art {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short v4i16 __attribute__((ext_vector_type(4)));

constexpr int kD = kHeadDim;
constexpr int kMaxWorkers = 512;   // two workgroups for each of 256 CUs

// RB: blocks of 32 rows of a row tile
template <int RB>
struct Tree {
  static constexpr int kRows = 32 * RB;
  static constexpr int TS = kWaves / RB;            // wavefronts that share a block's tokens
  // Wide row tiles, which the matrix cores bound: the next tile's scores are in work
  // with one's probabilities, so it has to be there before that one has been used up
  static constexpr bool WIDE = RB == kWaves;
  static constexpr int TK = RB == 1 ? 128 : WIDE ? 32 : 64;  // tokens of a tile
  static_assert(TK == 32 * TS);                     // a piece of 32 tokens to a wavefront
  // Places on the line of a unit's set-up and end (16 sequences of up to 2K tokens and
  // 16 nodes 35 us, without them 48), and of a workgroup, at least (one of 4K tokens, 4
  // heads to each of 2 KV heads 15 us, with four times as many 24).
  static constexpr int LEAD = RB == 1 ? 2 : 4;
  static constexpr int LEAST = RB == 1 ? 1 : 2;
  static constexpr int OWN = TK / kWaves;           // tokens of a tile that a wavefront loads
  static constexpr int LOADS = OWN / 4;             // its load instructions for K (and for V)
  static constexpr int BUFS = WIDE ? 4 : 2;         // tiles in LDS
  static constexpr int PITCH = kD + 4;              // floats of a row of a wavefront's record
  static constexpr int TILE_BYTES = 2 * TK * kD * 2;
  static constexpr int REC_BYTES = kWaves * 32 * PITCH * 4;
  static constexpr int LDS = BUFS * TILE_BYTES > REC_BYTES ? BUFS * TILE_BYTES : REC_BYTES;
};

struct TreeParams {
  int32_t batch, rows, per_seq;
  int32_t q_heads, kv_heads, group;
  int32_t nodes;               // of a row tile
  int32_t words;               // of a mask row; 0: chains
  int32_t page_shift, num_pages, max_pages;
  int32_t slots;               // entries of `units`
  int32_t by_unit;             // entries are units (else workgroups)
  int64_t most_units;          // that rows of distinct sequences can make
  int32_t out_bf16, negate;    // negate: a negative scale
  float scale_log2, scale_rest;  // its magnitude: rounded down to fp32, and what that leaves
  int64_t qs_row, qs_head;
  int64_t ks_page, ks_head, ks_tok, vs_page, vs_head, vs_tok;
  const int32_t* offsets;
  const int32_t* context;
  const int32_t* table;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const uint64_t* mask;
  void* out;
  float* lse;
  int4* units;                 // what the second launch has to join
  float* records;              // two for every workgroup
};

// The parameters are read where they are used, through the scalar cache; fresh()
// keeps the compiler from holding all of them in registers meanwhile.
typedef const __attribute__((address_space(4))) TreeParams TP;
__device__ __forceinline__ TP* fresh(TP* p) {
  __asm__ __volatile__("" : "+s"(p));
  return p;
}

// A sequence: its first row, nodes, context and row tiles.
struct Seq {
  int first, n, context, tiles;
};
__device__ __forceinline__ Seq seq_of(TP& P, int b) {
  int first = P.offsets ? P.offsets[b] : b * P.per_seq, end = P.offsets ? P.offsets[b + 1] : first + P.per_seq;
  first = min(max(first, 0), P.rows);
  end = min(max(end, first), P.rows);
  Seq s{first, end - first, P.context[b], 0};
  if (s.context < 0 || (int64_t)s.context + s.n > (int64_t)P.max_pages << P.page_shift) s.n = 0;
  s.tiles = (s.n + P.nodes - 1) / P.nodes;
  return s;
}

// The first kSeqs sequences, kept in LDS by the workgroup that has looked them all up.
constexpr int kSeqs = 256;
__device__ __forceinline__ Seq seq_of(TP& P, const int4* known, int b) {
  if (b >= kSeqs) return seq_of(P, b);
  const int4 s = known[b];
  return Seq{s.x, s.y, s.z, s.w};
}

// Tokens that row tile i goes through.
__device__ __forceinline__ int tokens_of(TP& P, const Seq& s, int i) {
  return s.context + (P.words ? s.n : (int)min((int64_t)s.n, (int64_t)(i + 1) * P.nodes));
}
// sum of floor((a i + b) / m) over i = 0 .. n - 1, by the steps of Euclid's
// algorithm (a, m <= 128, n < 2^24)
__device__ __forceinline__ int64_t floor_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b) {
  int64_t sum = 0;
  while (n > 0) {
    sum += (int64_t)n * (n - 1) / 2 * (a / m) + (int64_t)n * (b / m);
    a %= m;
    b %= m;
    const uint32_t y = a * n + b;
    if (y < m) break;
    n = y / m;
    b = y % m;
    const uint32_t t = m;
    m = a;
    a = t;
  }
  return sum;
}
// Places of a head's first `k` row tiles on the line.
template <int RB>
__device__ __forceinline__ int64_t places(TP& P, const Seq& s, int k) {
  constexpr int TK = Tree<RB>::TK, kLead = Tree<RB>::LEAD;
  if (k == 0) return 0;                            // (a sequence of no nodes has no tiles)
  const int64_t all = (s.context + s.n + TK - 1) / TK;
  if (P.words || s.tiles == 1) return k * (kLead + all);
  // all but the last row tile end a whole number of nodes further each
  const int64_t sum = floor_sum(min(k, s.tiles - 1), TK, P.nodes, s.context + P.nodes + TK - 1);
  return (int64_t)k * kLead + sum + (k == s.tiles ? all : 0);
}

// Sums of lanes 0 .. lane: within rows of 16 lanes, then over them.
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t add_lanes(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, false);
  return x + (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t scan(int64_t x) {
  x = add_lanes<0x111, 0xf>(x);   // row_shr:1, 2, 4, 8
  x = add_lanes<0x112, 0xf>(x);
  x = add_lanes<0x114, 0xf>(x);
  x = add_lanes<0x118, 0xf>(x);
  x = add_lanes<0x142, 0xa>(x);   // row_bcast:15 into rows 1 and 3
  return add_lanes<0x143, 0xc>(x);  // row_bcast:31 into rows 2 and 3
}
// a / b for 0 <= a < 2^52, 0 < b: the quotient in fp64, rounded to nearest, reaches no
// whole number that the exact one does not (which is at least 1 / b from it).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) { return (int64_t)((double)a / (double)b); }

__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A token's 16-byte piece in LDS: piece j of K lies at place j ^ (r & 15) of row r, so
// that the sixteen rows whose pieces are read in one cycle fall on distinct banks, and
// of V at j ^ 4 (r & 3), as the transposing reads of a cycle take four pieces of each
// of four rows.  (Half of the swizzle, r & 7 and 2 (r & 3), had half of LDS's cycles
// spent on conflicts.)
__device__ __forceinline__ int k_off(int r, int piece) { return r * kD + ((piece ^ (r & 15)) << 3); }
__device__ __forceinline__ int v_off(int r, int piece) { return r * kD + ((piece ^ (4 * (r & 3))) << 3); }

// Waits until at most N of the wavefront's loads are on their way.
template <int N>
__device__ __forceinline__ void wait_loads() {
  __asm__ __volatile__("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4 | 15 << 8);
  __asm__ __volatile__("" ::: "memory");
}
// (the wavefront's own reads of LDS have then ended: what they read may be overwritten)
__device__ __forceinline__ void end_reads() {
  __asm__ __volatile__("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
  __asm__ __volatile__("" ::: "memory");
}
__device__ __forceinline__ void barrier() {
  end_reads();
  __builtin_amdgcn_s_barrier();
  __asm__ __volatile__("" ::: "memory");
}
// 16 bytes for every lane straight into LDS, lane after lane from `to` on: `base`
// uniform, `offset` the lane's.  In assembly, as the compiler would have every later
// read of LDS wait for all loads on their way; wait_loads says when they are there.
// (It has no output register, so nothing can be taken for loaded too early; m0 is an
// operand, set by the compiler, which so knows what it holds.)
__device__ __forceinline__ void load_lds(const uint8_t* base, uint32_t offset, uint8_t* to) {
  const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)to);
  __asm__ __volatile__("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "{m0}"(at), "v"(offset), "s"(base) : "memory");
}
// ... of a lane's own address
__device__ __forceinline__ void load_lds(const uint8_t* from, uint8_t* to) {
  const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)to);
  __asm__ __volatile__("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "{m0}"(at), "v"(from) : "memory");
}

// Which of nodes j0 .. j0 + 31 row node i sees (bit k: node j0 + k; nodes below 0
// are context).  `word0`: the mask's first word.
__device__ __forceinline__ uint32_t sees(TP& P, const uint64_t* mask, uint64_t word0, int i, int n, int j0) {
  if (j0 <= -32) return 0xffffffffu;
  uint64_t v;
  int count;                     // of the 32 that may be seen
  if (!P.words) {
    v = ~0ull;
    count = i + 1 - j0;
  } else {
    count = n - j0;
    if (j0 < 0) {
      v = word0 << -j0 | ((1ull << -j0) - 1);
    } else {
      const int w = j0 >> 6, sh = j0 & 63;
      v = (w == 0 ? word0 : w < P.words ? mask[w] : 0) >> sh;
      if (sh > 32 && w + 1 < P.words) v |= mask[w + 1] << (64 - sh);
    }
  }
  if (count <= 0) return 0;
  return (uint32_t)v & (count >= 32 ? 0xffffffffu : (1u << count) - 1);
}

__device__ __forceinline__ float ln_of(float m, float l) { return (m + __log2f(l)) * 0.69314718055994531f; }
__device__ __forceinline__ float factor(float m, float top) {
  return m == kNegInf ? 0.f : fast_exp2(fmaxf(m - top, -126.f));
}

__device__ __forceinline__ void write4(TP& P, int64_t row, int d, const f32x4& x) {
  if (P.out_bf16) {
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(P.out) + row * kD + d) =
        u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(P.out) + row * kD + d) = x;
  }
}
__device__ __forceinline__ f32x4 over(const f32x4& o, float l) {
  const float inv = l == 0.f ? 0.f : 1.f / l;     // (l is 0 where nothing is seen)
  return f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
}

// PARTS: bf16 parts that a probability is multiplied in: three (24 bits) for fp32
// outputs.  For bf16 outputs two (16 bits, so that the output's own rounding is all that
// shows: 1.67e-3 of the output in the relative 2-norm, 1.88e-3 with one) in row tiles of
// up to 64 rows, where memory is the bound (8 x 32K tokens, 16 nodes: 204 us, 202 with
// one and 208 with three); one (8 bits, as the output has itself) in those of 128 rows,
// which the matrix cores bound (4096 prompt tokens each behind 16K: 2.16 ms, 3.14 with
// two and 4.32 with three).
template <int RB, int PARTS>
__global__ void __launch_bounds__(kThreads, RB == 1 ? 1 : 2) tree_kernel(const TreeParams) {
  TP* const args = (TP*)__builtin_amdgcn_kernarg_segment_ptr();
  TP& P = *args;
  using C = Tree<RB>;
  __shared__ __align__(16) uint8_t lds[C::LDS];
  __shared__ float s_m[kWaves][32], s_l[kWaves][32];
  __shared__ int64_t s_scan[2][kWaves], s_base;
  __shared__ int s_seq, s_units;
  __shared__ int4 s_known[kSeqs];
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, lo = lane & 31, half = lane >> 5;

  // ---- this workgroup's part of the line ----
  // thread tid has sequences b0 .. b1 - 1: `own` places and `mine` units, behind
  // `before` and `earlier`
  const int per = (P.batch + kThreads - 1) / kThreads;
  const int b0 = min(tid * per, P.batch), b1 = min(b0 + per, P.batch);
  int64_t own = 0, mine = 0;
  for (int b = b0; b < b1; ++b) {
    const Seq s = seq_of(P, b);
    if (b < kSeqs) s_known[b] = int4{s.first, s.n, s.context, s.tiles};
    own += P.kv_heads * places<RB>(P, s, s.tiles);
    mine += (int64_t)P.kv_heads * s.tiles;
  }
  int64_t before = scan(own), earlier = scan(mine);
  if (lane == 63) {
    s_scan[0][wave] = before;
    s_scan[1][wave] = earlier;
  }
  __syncthreads();
  int64_t line = 0, n_units = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) {
      before += s_scan[0][w];
      earlier += s_scan[1][w];
    }
    line += s_scan[0][w];
    n_units += s_scan[1][w];
  }
  before -= own;
  earlier -= mine;
  // Offsets that decrease can claim rows for many sequences: more units than there are
  // entries, and a line longer than its arithmetic holds.  Nothing is done for them.
  if (n_units > P.most_units) line = n_units = 0;
  line = uniform(line);
  const int64_t workers = min((int64_t)gridDim.x, max(line / C::LEAST, (int64_t)1));
  // Workgroups go to the eight XCDs in turn: each XCD gets one stretch of the line, so
  // that row tiles of the same keys meet in its L2.
  const int64_t me = gridDim.x % 8 ? blockIdx.x : blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
  // entries that no unit (or working workgroup) fills
  if (tid == 0) {
    if (!P.by_unit) {
      P.units[me] = int4{0, 0, 0, 0};
    } else {
      for (int64_t i = n_units + me; i < P.slots; i += gridDim.x) P.units[i] = int4{0, 0, 0, 0};
    }
  }
  if (me >= workers) return;
  const int64_t begin = uniform(quotient(me * line, workers)), end = uniform(quotient((me + 1) * line, workers));
  if (begin >= end) return;
  if (before <= begin && begin < before + own) {
    int b = b0;
    for (;; ++b) {
      const Seq s = seq_of(P, s_known, b);
      const int64_t n = P.kv_heads * places<RB>(P, s, s.tiles);
      if (begin < before + n) break;
      before += n;
      earlier += (int64_t)P.kv_heads * s.tiles;
    }
    s_seq = b;
    s_base = before;
    s_units = (int)earlier;
  }
  __syncthreads();
  int b = uniform(s_seq);
  int64_t base = uniform(s_base), unit0 = uniform(s_units);

  float* const s_rec = reinterpret_cast<float*>(lds);
  const int rb = wave / C::TS, ts = wave % C::TS;

  // Loading.  A wavefront loads tokens OWN wave .. of a tile, four rows an
  // instruction; lane l fetches the piece of row l / 16 that belongs at place l % 16.
  // (Its offset within the four rows: K's places depend on which of four the
  // instruction is.)
  const int k_row = wave * C::OWN % 16;
  uint32_t k_lane[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    k_lane[i] = (uint32_t)(lane >> 4) * (uint32_t)P.ks_tok * 2 + 16 * ((lane & 15) ^ (k_row + (lane >> 4) + 4 * i));
  const uint32_t v_lane = (uint32_t)(lane >> 4) * (uint32_t)P.vs_tok * 2 + 16 * ((lane & 15) ^ (4 * (lane >> 4)));

  // Reading.  K: lane l takes pieces 2 i + l / 32 of row l % 32 of a piece.  V^T, dims
  // 32 d + lane % 32: element e of K-step i is token 16 i + 8 (e / 4) + 4 half + e % 4.
  // Of the 16 lanes of a group lane 4 k + h points at elements 4 h .. 4 h + 3 of the
  // group's 16 dims in row k, and lane j receives dim j of the four rows.
  uint32_t k_read[8], v_read[4];
#pragma unroll
  for (int i = 0; i < 8; ++i) k_read[i] = 2 * k_off(lo, 2 * i + half);
#pragma unroll
  for (int d = 0; d < 4; ++d)
    v_read[d] = 2 * v_off(4 * half + ((lane & 15) >> 2), 4 * d + 2 * (lane >> 4 & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);

  // Where a part of the line begins inside a unit and goes on behind it, that rest of
  // a unit comes last: workgroups of wide row tiles then begin whole units together,
  // and go through the same keys at the same time, in the L2 of their XCD.
  const int first_b = b;
  const int64_t first_base = base, first_unit0 = unit0;
  bool put_off = false, rest = false;
  int64_t x = begin;
  while (x < end || put_off) {
    if (x >= end) {
      x = begin;
      b = first_b;
      base = first_base;
      unit0 = first_unit0;
      put_off = false;
      rest = true;
    }
    // ---- the segment at x: sequence, head, row tile, tiles ----
    TP& P = *fresh(args);
    Seq s = seq_of(P, s_known, b);
    int64_t each = places<RB>(P, s, s.tiles);          // of a head
    while (x >= base + each * P.kv_heads) {
      base += each * P.kv_heads;
      unit0 += (int64_t)P.kv_heads * s.tiles;
      s = seq_of(P, s_known, ++b);
      each = places<RB>(P, s, s.tiles);
    }
    s.first = uniform(s.first);
    s.n = uniform(s.n);
    s.context = uniform(s.context);
    s.tiles = uniform(s.tiles);
    const int kvh = uniform((int)quotient(x - base, each));
    const int64_t at = x - base - kvh * each;
    int rt = 0, rt_end = s.tiles;                      // the last row tile whose places begin at or before
    while (rt_end - rt > 1) {
      const int mid = (rt + rt_end) / 2;
      if (places<RB>(P, s, mid) <= at) rt = mid;
      else rt_end = mid;
    }
    rt = uniform(rt);
    const int64_t start = base + kvh * each + uniform(places<RB>(P, s, rt));
    const int seen = uniform(tokens_of(P, s, rt)), all = (seen + C::TK - 1) / C::TK;
    const int64_t next = min(end, start + C::LEAD + all);
    const int t0 = uniform(max((int)(x - start) - C::LEAD, 0)), t1 = uniform((int)(next - start) - C::LEAD);
    if (C::WIDE && !rest && x == begin && start < begin && next < end) {
      put_off = true;
      x = next;
      continue;
    }
    x = rest ? end : next;
    if (t1 <= t0) continue;                            // only places before its tiles
    const bool begins = t0 == 0, whole = begins && t1 == all;
    const int64_t last = quotient((start + C::LEAD + all) * workers - 1, line);   // who holds its last place

    const int node0 = rt * P.nodes, M = min(P.nodes, s.n - node0) * P.group;
    bf16x8 qf[8];
    const int row = 32 * rb + lo, head = kvh * P.group + row % P.group;
    const int node = node0 + row / P.group;
    const uint64_t* const mask = P.words && row < M ? P.mask + (int64_t)(s.first + node) * P.words : P.mask;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      u32x4 w{0u, 0u, 0u, 0u};
      if (row < M) {
        w = *reinterpret_cast<const u32x4*>(P.q + (s.first + node) * P.qs_row + head * P.qs_head + 16 * i + 8 * half);
        if (P.negate) w = w ^ 0x80008000u;
      }
      qf[i] = __builtin_bit_cast(bf16x8, w);
    }
    const uint64_t mask0 = P.words ? mask[0] : 0;
    f32x16 acc[4];
    float m, l;

    // Pages: lane i has that of the wavefront's 16-token group i from tile `paged` on,
    // and of 64 more, asked for that much ahead.
    constexpr int kRows = C::OWN < 16 ? C::OWN : 16;              // of one page
    constexpr int kGroups = C::OWN / kRows, kAhead = 64 / kGroups;  // tiles that 64 lanes serve
    auto pages_from = [&](int t) __attribute__((always_inline)) {
      TP& P = *fresh(args);
      const int tok = min((t + lane / kGroups) * C::TK + wave * C::OWN + kRows * (lane % kGroups), seen - 1);
      const int page = P.table[(int64_t)b * P.max_pages + (tok >> P.page_shift)];
      return min(max(page, 0), P.num_pages - 1);
    };
    int paged = t0, pages = pages_from(t0), more_pages = t0 + kAhead < t1 ? pages_from(t0 + kAhead) : 0;
    const int pages0 = pages, more_pages0 = more_pages;
    const uint8_t* const k_head = reinterpret_cast<const uint8_t*>(P.k + kvh * P.ks_head);
    const uint8_t* const v_head = reinterpret_cast<const uint8_t*>(P.v + kvh * P.vs_head);
    const int64_t k_page = P.ks_page * 2, v_page = P.vs_page * 2;
    const uint32_t k_tok = (uint32_t)P.ks_tok * 2, v_tok = (uint32_t)P.vs_tok * 2, slots = (1u << P.page_shift) - 1;
    // kRows rows, all of them before the end
    auto load_rows = [&](int first, int page, uint8_t* to_k) __attribute__((always_inline)) {
      const uint8_t* const k16 = k_head + page * k_page + (uint64_t)(first & slots) * k_tok;
      const uint8_t* const v16 = v_head + page * v_page + (uint64_t)(first & slots) * v_tok;
#pragma unroll
      for (int i = 0; i < kRows / 4; ++i) {
        load_lds(k16 + (uint64_t)(4 * i * k_tok), k_lane[i], to_k + 4 * i * kD * 2);
        load_lds(v16 + (uint64_t)(4 * i * v_tok), v_lane, to_k + C::TK * kD * 2 + 4 * i * kD * 2);
      }
    };
    auto next_pages = [&]() __attribute__((always_inline)) {
      paged += kAhead;
      pages = more_pages;
      more_pages = paged + kAhead < t1 ? pages_from(paged + kAhead) : 0;
    };
    auto load_tile = [&](int t, int buf) __attribute__((always_inline)) {
      uint8_t* const to = lds + buf * C::TILE_BYTES + wave * C::OWN * kD * 2;
      if (t >= paged + kAhead) next_pages();
      const int tok0 = t * C::TK + wave * C::OWN;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        const int first = tok0 + kRows * g;
        const int page = __builtin_amdgcn_readlane(pages, (t - paged) * kGroups + g);
        uint8_t* const to_k = to + kRows * g * kD * 2;
        uint8_t* const to_v = to_k + C::TK * kD * 2;
        if (first + kRows <= seen) {
          load_rows(first, page, to_k);
        } else {
          // tokens past the end are redirected to the last one
          const uint8_t* const k = k_head + page * k_page;
          const uint8_t* const v = v_head + page * v_page;
#pragma unroll
          for (int i = 0; i < kRows / 4; ++i) {
            const uint32_t slot = min(first + 4 * i + (lane >> 4), seen - 1) & slots;
            load_lds(k + (uint64_t)slot * k_tok + 16 * ((lane & 15) ^ (k_row + (lane >> 4) + 4 * i)), to_k + 4 * i * kD * 2);
            load_lds(v + (uint64_t)slot * v_tok + 16 * ((lane & 15) ^ (4 * (lane >> 4))), to_v + 4 * i * kD * 2);
          }
        }
      }
    };
    const int place = 32 * ts;     // the piece's first token of the tile
    // Tokens that every row of the tile sees; only behind them are rows told apart.
    const int open = P.words ? s.context : s.context + node0 + 1;
    auto is_tail = [&](int t) { return (t + 1) * C::TK > open; };

    // Infinities and NaN among the values: a row that does not see them must not get
    // them, but 0 times them is no 0 (and a probability's lower parts may be 0).  Sums
    // that are not finite are therefore made again, with care: such values are added to
    // the rows that see them, those with a score above -inf, and leave the tile before
    // its products.  (8 x 32K tokens, 16 nodes: 204 us, 348 with one such value in each
    // sequence and 654 with one in every page of 64 tokens.)
    auto wild = [&](int buf) __attribute__((always_inline)) {
      const uint8_t* const tile = lds + buf * C::TILE_BYTES + C::TK * kD * 2;
      bool found = false;
      int at = tid;
      __asm__ __volatile__("" : "+v"(at));   // (addresses made here, not held throughout)
      __syncthreads();     // (a wavefront may have waited for its own tokens only)
      for (int i = at; i < C::TK * kD / 8; i += kThreads) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(tile + 16 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) found |= (w[j] & 0x7f80u) == 0x7f80u || (w[j] & 0x7f800000u) == 0x7f800000u;
      }
      return __syncthreads_or(found) != 0;
    };
    auto clean = [&](int buf) __attribute__((always_inline)) {
      uint8_t* const tile = lds + buf * C::TILE_BYTES + C::TK * kD * 2;
      __syncthreads();     // (the wavefronts have added what is there)
      for (int i = tid; i < C::TK * kD / 8; i += kThreads) {
        u32x4 w = *reinterpret_cast<const u32x4*>(tile + 16 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if ((w[j] & 0x7f80u) == 0x7f80u) w[j] &= 0xffff0000u;
          if ((w[j] & 0x7f800000u) == 0x7f800000u) w[j] &= 0xffffu;
        }
        *reinterpret_cast<u32x4*>(tile + 16 * i) = w;
      }
      __syncthreads();
    };

    // The A operands: K-step i of a piece's keys; K-step i and dims 32 d .. of V^T.
    auto key_part = [&](int at, int i) __attribute__((always_inline)) {
      return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(lds + k_read[i] + at));
    };
    auto value_part = [&](int at, int i, int d) __attribute__((always_inline)) {
      v4i16 w[2];
#pragma unroll
      for (int e = 0; e < 2; ++e)
        w[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) v4i16*)(lds + v_read[d] + at + C::TK * kD * 2 + (16 * i + 8 * e) * kD * 2));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // Scores of a piece: st[r] is token 8 (r / 4) + 4 half + r % 4 of it.  (`at`: its
    // place in LDS, in bytes; where that is a constant, it goes into the reads.)
    auto scores = [&](int at, f32x16& st) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) st[r] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bf16x8 a = key_part(at, i);
        st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[i], st, 0, 0, 0);
      }
    };
    auto hide = [&](int t, f32x16& st) __attribute__((always_inline)) {
      TP& P = *fresh(args);
      const uint32_t bits = sees(P, mask, mask0, node, s.n, t * C::TK + place - s.context) >> (4 * half);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!(bits >> (8 * (r >> 2) + (r & 3)) & 1u)) st[r] = kNegInf;
    };
    // The reference m moves only where a score passes it by more than 2^8 (and at the
    // first score): sums keep their relative precision either way.
    const float scale = P.scale_log2, scale_rest = P.scale_rest;
    auto tops = [&](const f32x16& st, float& top) __attribute__((always_inline)) {
      top = st[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(top, st[r]);
      top *= scale;
    };
    auto refer = [&](float top) __attribute__((always_inline)) {
      if (__any(top > m + 8.f)) {
        float a, c;
        swap_rows32(top, a, c);
        const float mn = fmaxf(m, fmaxf(a, c));
        // (never 0: infinite sums stay so; the first reference finds no others)
        const float f = m == kNegInf ? 1.f : fast_exp2(fmaxf(m - mn, -126.f));
        m = mn;
        l *= f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[d][r] *= f;
      }
    };
    auto weights = [&](f32x16& st, bf16x8 (&p)[PARTS][2]) __attribute__((always_inline)) {
      const float ref = m == kNegInf ? 0.f : m;
      // (a tile's sum first: many small probabilities, added one by one to the large sum
      // that a few high scores have made, would round away)
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        // (where fp32 is kept, the scale's own rounding would move large scores by more
        // than their own does)
        const float x = PARTS > 1 ? fmaf(st[r], scale_rest, -ref) : -ref;
        st[r] = fast_exp2(fmaf(st[r], scale, x));
        sum += st[r];
      }
      l += sum;
#pragma unroll
      for (int k = 0; k < PARTS; ++k) {
        uint32_t w[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          w[r] = pack_bf16(st[2 * r], st[2 * r + 1]);
          if (k + 1 < PARTS) {
            st[2 * r] -= bf_lo(w[r]);
            st[2 * r + 1] -= bf_hi(w[r]);
          }
        }
        p[k][0] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
        p[k][1] = __builtin_bit_cast(bf16x8, u32x4{w[4], w[5], w[6], w[7]});
      }
    };
    auto products = [&](int at, const bf16x8 (&p)[PARTS][2]) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
        const bf16x8 a = value_part(at, i, d);
#pragma unroll
        for (int j = 0; j < PARTS; ++j)
          acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p[j][i], acc[d], 0, 0, 0);
      }
    };

    // A piece's values that are not finite, to the rows that see them.  (The reference is
    // above -inf where there is one, so no later factor is 0.)
    auto add_wild = [&](int at, const f32x16& st) __attribute__((always_inline)) {
      uint32_t bits = 0;   // the piece's tokens that the lane's row sees
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!(st[r] * scale == kNegInf)) bits |= 1u << (8 * (r >> 2) + 4 * half + (r & 3));
      const auto both = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
      bits = both[0] | both[1];
#pragma unroll 1
      for (int tok = 0; tok < 32; ++tok) {
        // (two values to a lane: most tokens have none)
        const uint32_t mine = *reinterpret_cast<const uint32_t*>(lds + at + C::TK * kD * 2 + tok * kD * 2 + 4 * lane);
        if (!__any((mine & 0x7f80u) == 0x7f80u || (mine & 0x7f800000u) == 0x7f800000u)) continue;
        const bool seen_here = bits >> tok & 1u;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const uint8_t* const from = lds + at + C::TK * kD * 2 + 2 * v_off(tok, 4 * d) + 8 * half;
#pragma unroll
          for (int e = 0; e < 4; ++e) {      // (16-byte pieces 4 d .. 4 d + 3 of a row lie in order)
            const u32x2 w = *reinterpret_cast<const u32x2*>(from + 16 * e);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float y = j & 1 ? bf_hi(w[j >> 1]) : bf_lo(w[j >> 1]);
              if (seen_here && !(fabsf(y) < __builtin_inff())) acc[d][4 * e + j] += y;
            }
            __builtin_amdgcn_sched_barrier(0);   // (few registers are left)
          }
        }
      }
    };
    auto weigh = [&](int at, f32x16& st) __attribute__((always_inline)) {
      bf16x8 p[PARTS][2];
      weights(st, p);
      products(at, p);
    };

    bool careful = false;
#pragma unroll 1
    for (;; careful = true) {
      m = kNegInf;
      l = 0.f;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
      __syncthreads();     // the segment before has left LDS
      if constexpr (C::WIDE) {
        // Four tiles in LDS: one whose probabilities are in work, the next with its
        // scores, and two on their way.
        const int first_tail = max(min(open / C::TK, t1), t0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t0 + i < t1) load_tile(t0 + i, i);
        wait_loads<0>();
        barrier();
        int t = t0;
        if (!careful && t + 8 < first_tail) {
          f32x16 st;
          float top;
          bf16x8 k_part[8];
          scores(0, st);
          tops(st, top);
#pragma unroll
          for (int i = 0; i < 8; ++i) k_part[i] = key_part(C::TILE_BYTES, i);
          // One tile, in buffer B, and the next one's scores, whose keys are in registers;
          // then that buffer is free for the tile four further, and the keys two further
          // are there.  (All of it is before the tail: every row of a tile exists.)  No
          // branch but the reference's.
          auto step = [&](auto B, int t) __attribute__((always_inline)) {
            constexpr int kB = decltype(B)::value, kHere = kB * C::TILE_BYTES;
            constexpr int kNext = (kB + 1) % 4 * C::TILE_BYTES, kAfter = (kB + 2) % 4 * C::TILE_BYTES;
            uint8_t* const free_place = lds + kHere + wave * C::OWN * kD * 2;
            f32x16 next_st;
            refer(top);
            const int at = t + 4 - paged, here = __builtin_amdgcn_readlane(pages, at & 63);
            const int ahead = __builtin_amdgcn_readlane(more_pages, at & 63), page = at < kAhead ? here : ahead;
            const int first = (t + 4) * C::TK + wave * C::OWN;
            if constexpr (PARTS > 1) {
              scores(kNext, next_st);
              weigh(kHere, st);
              wait_loads<2 * C::LOADS>();
              barrier();
              load_rows(first, page, free_place);
              tops(next_st, top);
            } else {
              // In this order: two probabilities and a piece of V behind every matrix
              // instruction of the scores, maxima, keys and loads behind those of the
              // products.  V is in registers by then, so the barrier comes between.
              bf16x8 v_part[8];
              uint32_t w[8];
              const uint8_t *k16 = nullptr, *v16 = nullptr;
              const float ref = m == kNegInf ? 0.f : m;
              float sum = 0.f;
#pragma unroll
              for (int r = 0; r < 16; ++r) next_st[r] = 0.f;
              __builtin_amdgcn_s_setprio(1);
              __builtin_amdgcn_sched_barrier(0);
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                if (i == 1) k16 = k_head + page * k_page;
                if (i == 2) v16 = v_head + page * v_page;
                if (i == 3) k16 += (uint64_t)(first & slots) * k_tok;
                if (i == 4) v16 += (uint64_t)(first & slots) * v_tok;
                next_st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_part[i], qf[i], next_st, 0, 0, 0);
                v_part[i] = value_part(kHere, i >> 2, i & 3);
                const float x = fast_exp2(fmaf(st[2 * i], scale, -ref));
                const float y = fast_exp2(fmaf(st[2 * i + 1], scale, -ref));
                sum += x;
                sum += y;
                w[i] = pack_bf16(x, y);
                __builtin_amdgcn_sched_barrier(0);
              }
              l += sum;
              wait_loads<2 * C::LOADS>();
              barrier();
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const uint32_t* const u = w + (i >> 2) * 4;
                acc[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    v_part[i], __builtin_bit_cast(bf16x8, u32x4{u[0], u[1], u[2], u[3]}), acc[i & 3], 0, 0, 0);
                if (i == 0) top = next_st[0];
                top = fmaxf(fmaxf(top, next_st[2 * i]), next_st[2 * i + 1]);
                if (i == 7) top *= scale;
                if (i < 4) {
                  k_part[2 * i] = key_part(kAfter, 2 * i);
                  k_part[2 * i + 1] = key_part(kAfter, 2 * i + 1);
                } else if (i - 4 < kRows / 4) {
                  load_lds(k16 + (uint64_t)(4 * (i - 4) * k_tok), k_lane[i - 4], free_place + 4 * (i - 4) * kD * 2);
                  load_lds(v16 + (uint64_t)(4 * (i - 4) * v_tok), v_lane, free_place + C::TK * kD * 2 + 4 * (i - 4) * kD * 2);
                }
                __builtin_amdgcn_sched_barrier(0);
              }
              __builtin_amdgcn_s_setprio(0);
            }
            st = next_st;
          };
#pragma unroll 1
          for (; t + 8 < first_tail; t += 4) {
            if (t + 4 >= paged + kAhead) next_pages();
            step(std::integral_constant<int, 0>{}, t);
            step(std::integral_constant<int, 1>{}, t + 1);
            step(std::integral_constant<int, 2>{}, t + 2);
            step(std::integral_constant<int, 3>{}, t + 3);
          }
        }
        // (behind the steps: the tile of the pending scores again, from its keys)
#pragma unroll 1
        for (; t < t1; ++t) {
          const int buf = (t - t0) & 3;
          const bool tail = t >= first_tail;
          f32x16 st;
          scores(buf * C::TILE_BYTES, st);
          if (tail) hide(t, st);
          float top;
          tops(st, top);
          refer(top);
          if (careful && wild(buf)) {
            add_wild(buf * C::TILE_BYTES, st);
            clean(buf);
          }
          weigh(buf * C::TILE_BYTES, st);
          if (t + 1 < t1) {
            // the next tile is there, and this one has been used up
            if (t + 3 < t1) wait_loads<4 * C::LOADS>();
            else wait_loads<0>();
            barrier();
            if (t + 4 < t1) load_tile(t + 4, buf);
          }
        }
      } else {
        load_tile(t0, t0 & 1);
#pragma unroll 1
        for (int t = t0; t < t1; ++t) {
          if constexpr (C::TS == kWaves) {
            // a wavefront works on the tokens that it loads itself: no other's are waited for
            end_reads();
            if (t + 1 < t1) {
              load_tile(t + 1, (t + 1) & 1);
              wait_loads<2 * C::LOADS>();
            } else {
              wait_loads<0>();
            }
          } else {
            wait_loads<0>();
            barrier();       // the tile is there, and the one before it has been read
            if (t + 1 < t1) load_tile(t + 1, (t + 1) & 1);
          }
          const int at = (t & 1) * C::TILE_BYTES + place * kD * 2;
          f32x16 st;
          scores(at, st);
          if (is_tail(t)) hide(t, st);
          float top;
          tops(st, top);
          refer(top);
          if (careful && wild(t & 1)) {
            add_wild(at, st);
            clean(t & 1);
          }
          weigh(at, st);
        }
      }
      float all_finite = 0.f;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) all_finite = fmaf(acc[d][r], 0.f, all_finite);
      // (the tiles have been read, too)
      if (!__syncthreads_or(!(all_finite == 0.f)) || careful) break;
      paged = t0;
      pages = pages0;
      more_pages = more_pages0;
    }

    // ---- the wavefronts' records, joined ----
    TP& W = *fresh(args);
    float* const to = W.records + (2 * me + (begins ? 1 : 0)) * (C::kRows * (kD + 2));
    const int64_t row0 = (int64_t)(s.first + node0) * W.q_heads + kvh * W.group;
    float l0, l1;
    swap_rows32(l, l0, l1);
    float* const rec = s_rec + wave * 32 * C::PITCH;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4*>(rec + lo * C::PITCH + 32 * d + 8 * e + 4 * half) =
            f32x4{acc[d][4 * e], acc[d][4 * e + 1], acc[d][4 * e + 2], acc[d][4 * e + 3]};
    if (half == 0) {
      s_m[wave][lo] = m;
      s_l[wave][lo] = l0 + l1;
    }
    __syncthreads();
    for (int i = tid; i < M * (kD / 4); i += kThreads) {
      const int r = i / (kD / 4), d = i % (kD / 4) * 4, w0 = r / 32 * C::TS, rr = r % 32;
      float top = kNegInf;
#pragma unroll
      for (int w = 0; w < C::TS; ++w) top = fmaxf(top, s_m[w0 + w][rr]);
      f32x4 sum{0.f, 0.f, 0.f, 0.f};
      float mass = 0.f;
#pragma unroll
      for (int w = 0; w < C::TS; ++w) {
        const float f = factor(s_m[w0 + w][rr], top);
        const f32x4 y = *reinterpret_cast<const f32x4*>(s_rec + (w0 + w) * 32 * C::PITCH + rr * C::PITCH + d);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = fmaf(y[j], f, sum[j]);
        mass = fmaf(s_l[w0 + w][rr], f, mass);
      }
      if (whole) {
        const int64_t at_row = row0 + (int64_t)(r / W.group) * W.q_heads + r % W.group;
        write4(W, at_row, d, over(sum, mass));
        if (d == 0) W.lse[at_row] = mass == 0.f ? kNegInf : ln_of(top, mass);
      } else {
        *reinterpret_cast<f32x4*>(to + r * kD + d) = sum;
        if (d == 0) {
          to[C::kRows * kD + r] = top;
          to[C::kRows * kD + C::kRows + r] = mass;
        }
      }
    }
    // what the second launch joins
    if (begins && tid == 0 && (W.by_unit || !whole))
      W.units[W.by_unit ? unit0 + (int64_t)kvh * s.tiles + rt : me] =
          whole ? int4{0, 0, 0, 0} : int4{s.first + node0, kvh << 10 | M, (int)me, (int)last};
  }
}

// The second launch: rows of units that lie in several workgroups.  ROWS rows to a
// workgroup, 32 lanes to a record of one.
template <int RB, int ROWS>
__global__ void __launch_bounds__(kThreads) tree_join_kernel(const TreeParams) {
  TP& P = *(TP*)__builtin_amdgcn_kernarg_segment_ptr();
  using C = Tree<RB>;
  constexpr int kGroups = kThreads / 32;
  __shared__ f32x4 s_o[kGroups][32];
  __shared__ float s_l[kGroups];
  const int per = C::kRows / ROWS;
  const int entry = blockIdx.x / per, r0 = (blockIdx.x - entry * per) * ROWS;
  const int4 u = P.units[entry];
  const int M = u.y & 1023, kvh = u.y >> 10, first = u.z, n = u.w - u.z + 1;
  if (r0 >= M) return;
  const int group = threadIdx.x / 32, lane = threadIdx.x & 31;
  auto record = [&](int i) {
    return P.records + (2 * (int64_t)(first + i) + (i == 0 ? 1 : 0)) * (C::kRows * (kD + 2));
  };
  const int r = ROWS == 1 ? r0 : r0 + group;
  const bool live = r < M;
  float top = kNegInf;
  for (int i = lane; live && i < n; i += 32) top = fmaxf(top, record(i)[C::kRows * kD + r]);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  f32x4 sum{0.f, 0.f, 0.f, 0.f};
  float mass = 0.f;
#pragma unroll 4
  for (int i = ROWS == 1 ? group : 0; live && i < n; i += ROWS == 1 ? kGroups : 1) {
    const float* p = record(i);
    const float f = factor(p[C::kRows * kD + r], top);
    const f32x4 y = *reinterpret_cast<const f32x4*>(p + r * kD + 4 * lane);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = fmaf(y[j], f, sum[j]);
    mass = fmaf(p[C::kRows * kD + C::kRows + r], f, mass);
  }
  if constexpr (ROWS == 1) {
    s_o[group][lane] = sum;
    if (lane == 0) s_l[group] = mass;
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int g = 1; g < kGroups; ++g) {
      sum = sum + s_o[g][lane];
      mass += s_l[g];
    }
  }
  if (!live) return;
  const int64_t row = (int64_t)(u.x + r / P.group) * P.q_heads + kvh * P.group + r % P.group;
  write4(P, row, 4 * lane, over(sum, mass));
  if (lane == 0) P.lse[row] = mass == 0.f ? kNegInf : ln_of(top, mass);
}

// ---- the host side ---------------------------------------------------------------

struct TreePlan {
  int rb, nodes, workers, slots;
  int64_t units;
  size_t records_off, total;
};

int rows_of(int rb) { return 32 * rb; }

art_status plan_tree(const art_decode_shape* s, const art_tree_opts* o, TreePlan* p) {
  const art_status st = check_cache(s);
  if (st != ART_OK) return st;
  if (!o || o->rows < 0 || o->mask_words < 0 || !isfinite(o->softmax_scale) ||
      (o->out_dtype != ART_OUT_F32 && o->out_dtype != ART_OUT_BF16) || o->q_stride_row < 0 || o->q_stride_head < 0 ||
      s->num_q_heads <= 0 || s->num_q_heads % s->num_kv_heads)
    return ART_ERR_INVALID_ARG;
  const int g = s->num_q_heads / s->num_kv_heads;
  const int64_t cap = (int64_t)s->max_pages_per_seq * s->page_size;
  if (g > 128 || s->num_kv_heads >= (1 << 20) || o->rows >= (1 << 24) || s->batch >= (1 << 20) || cap >= (1ll << 31) - (1 << 16) ||
      (o->q_stride_row | o->q_stride_head) % 8 || s->k_stride_token >= (1 << 27) || s->v_stride_token >= (1 << 27))
    return ART_ERR_UNSUPPORTED;
  // A row tile that holds a sequence's rows, on average.  32 rows at most: tiles of 128
  // tokens, each wavefront for itself, one workgroup to a CU, read fastest (8 x 32K
  // tokens, 32/8 heads, one node each: 190 us, 195 by tiles of 64 rows; one of 128K,
  // one KV head, 30 and 38), but where units are many or all of them short, two
  // workgroups to a CU end sooner (200 sequences of 50 to 150 tokens 44 us and 58; one of
  // 4K tokens, 8 KV heads, 19 and 21).  Tiles of 64 rows serve 48 and 64 rows in 203 and
  // 201 us where 128 rows take 228 both times, and 96 and 128 rows in 286 and 291 where
  // those take 231 and 235.  (A table 32 times as wide as
  // the sequences need slows none of these batches, long or short, by more than 1 %.)
  const int64_t rows = s->batch > 0 ? ((int64_t)o->rows + s->batch - 1) / s->batch * g : 0;
  const int64_t groups = (int64_t)s->batch * s->num_kv_heads;
  const bool few = rows <= 32 && g <= 32 && groups <= kMaxWorkers && groups * ((cap + 127) / 128) >= kMaxWorkers;
  p->rb = few ? 1 : rows <= 64 && g <= 64 ? 2 : 4;
  p->nodes = rows_of(p->rb) / g;
  const int tk = p->rb == 1 ? 128 : p->rb == 2 ? 64 : 32;
  const int64_t most = p->rb == 1 ? kMaxWorkers / 2 : kMaxWorkers;   // one or two to a CU
  const int64_t units = (int64_t)s->num_kv_heads * (o->rows / p->nodes + s->batch);   // at most
  // places on the line, by 512 workgroups, are counted in 52 bits
  if (units >= (int64_t(1) << 40) / ((cap + tk - 1) / tk + 4)) return ART_ERR_UNSUPPORTED;
  const int64_t tiles = units < most ? units * ((cap + tk - 1) / tk) : units;
  p->workers = (int)(tiles < most ? (tiles < 1 ? 1 : tiles) : most);
  p->units = units;
  p->slots = (int)(units < p->workers ? units : p->workers);
  if (p->slots < 1) p->slots = 1;
  p->records_off = ((size_t)p->slots * sizeof(int4) + 255) / 256 * 256;
  p->total = p->records_off + (size_t)2 * p->workers * rows_of(p->rb) * (kD + 2) * 4;
  return ART_OK;
}

template <int RB, int PARTS>
void launch(const TreePlan& plan, const TreeParams& p, hipStream_t stream) {
  hipLaunchKernelGGL((tree_kernel<RB, PARTS>), dim3((unsigned)plan.workers), dim3(kThreads), 0, stream, p);
  // a row to a workgroup where a unit may have a record in each of many workgroups
  // (one sequence of 128K tokens, one KV head: 30 us, 59 with eight), else eight (45 of
  // 400 to 1000 tokens: 37 us, 39 with one; 200 of 50 to 150 44 and 50)
  if (plan.workers > 32 * plan.slots)
    hipLaunchKernelGGL((tree_join_kernel<RB, 1>), dim3((unsigned)(plan.slots * rows_of(RB))), dim3(kThreads), 0, stream, p);
  else
    hipLaunchKernelGGL((tree_join_kernel<RB, 8>), dim3((unsigned)(plan.slots * (rows_of(RB) / 8))), dim3(kThreads), 0, stream, p);
}
template <int RB>
void launch(const TreePlan& plan, const TreeParams& p, hipStream_t stream) {
  if (p.out_bf16) launch<RB, RB == 4 ? 1 : 2>(plan, p, stream);
  else launch<RB, 3>(plan, p, stream);
}

}  // namespace
}  // namespace art

extern "C" {

size_t art_tree_workspace_bytes(const art_decode_shape* shape, const art_tree_opts* opts, int32_t* status) {
  art::TreePlan plan;
  const art_status st = art::plan_tree(shape, opts, &plan);
  if (status) *status = st;
  return st == ART_OK ? plan.total : 0;
}

art_status art_tree_attention(const art_decode_shape* shape, const art_tree_opts* opts, const void* q,
                              const void* k_cache, const void* v_cache, const int32_t* page_table,
                              const int32_t* context_lens, const int32_t* row_offsets, const uint64_t* mask, void* out,
                              float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  using namespace art;
  TreePlan plan;
  const art_status st = plan_tree(shape, opts, &plan);
  if (st != ART_OK) return st;
  if (!row_offsets && shape->batch > 0 && opts->rows % shape->batch) return ART_ERR_INVALID_ARG;
  if (shape->batch == 0 || opts->rows == 0) return ART_OK;
  if (!q || !k_cache || !v_cache || !page_table || !context_lens || !out || !lse || (opts->mask_words > 0) != (mask != nullptr) ||
      (uintptr_t)mask % 8 || (uintptr_t)workspace % 16)
    return ART_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)out) % 16) return ART_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < plan.total) return ART_ERR_WORKSPACE_TOO_SMALL;
  TreeParams p;
  memset(&p, 0, sizeof p);
  p.batch = shape->batch;
  p.rows = opts->rows;
  p.per_seq = opts->rows / shape->batch;
  p.q_heads = shape->num_q_heads;
  p.kv_heads = shape->num_kv_heads;
  p.group = shape->num_q_heads / shape->num_kv_heads;
  p.nodes = plan.nodes;
  p.words = opts->mask_words;
  while ((1 << p.page_shift) < shape->page_size) ++p.page_shift;
  p.num_pages = shape->num_pages;
  p.max_pages = shape->max_pages_per_seq;
  p.slots = plan.slots;
  p.by_unit = plan.slots < plan.workers;
  p.most_units = plan.units;
  p.out_bf16 = opts->out_dtype == ART_OUT_BF16;
  p.negate = opts->softmax_scale < 0.f;
  // (a scale of 0 weighs all tokens alike; hidden scores of -inf times 0 would not be -inf)
  const double scale_log2 = fabs((double)opts->softmax_scale) * 1.4426950408889634;
  // (both above 0: a hidden score of -inf stays one under either)
  p.scale_log2 = (float)scale_log2;
  if (p.scale_log2 > scale_log2) p.scale_log2 = nextafterf(p.scale_log2, 0.f);
  p.scale_rest = (float)(scale_log2 - p.scale_log2);
  if (p.scale_log2 < 1e-37f) p.scale_log2 = 1e-37f;
  if (p.scale_rest < 1e-37f) p.scale_rest = 1e-37f;
  p.qs_row = opts->q_stride_row;
  p.qs_head = opts->q_stride_head;
  p.ks_page = shape->k_stride_page;
  p.ks_head = shape->k_stride_head;
  p.ks_tok = shape->k_stride_token;
  p.vs_page = shape->v_stride_page;
  p.vs_head = shape->v_stride_head;
  p.vs_tok = shape->v_stride_token;
  p.offsets = row_offsets;
  p.context = context_lens;
  p.table = page_table;
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k_cache);
  p.v = static_cast<const uint16_t*>(v_cache);
  p.mask = mask;
  p.out = out;
  p.lse = lse;
  p.units = static_cast<int4*>(workspace);
  p.records = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.records_off);
  if (plan.rb == 1) launch<1>(plan, p, stream);
  else if (plan.rb == 2) launch<2>(plan, p, stream);
  else launch<4>(plan, p, stream);
  return hipGetLastError() == hipSuccess ? ART_OK : ART_ERR_HIP;
}

}  // extern "C"
