// Full attention (no stability test) over a cache held in 8 bits.
//
// Without the test nothing has to be decided block by block, so the work is cut
// for the memory system alone.  The 64-token tiles of all (sequence, KV head)
// groups form one line, and every workgroup takes an equal, contiguous part of
// it, however ragged the batch is; the part of a group in a workgroup's range
// is a segment.  (Short batches are cut by groups, many groups by wavefronts
// instead, see cut_of.)  The four wavefronts of a workgroup take a segment's
// tiles in turn, each with its own running maximum, mass and output sums in
// registers, and join at its end through LDS.  A group that lies in one
// workgroup is written out there; of the others each segment leaves a record
// (m, L, o) in the workspace and a second, small launch joins them.
//
//   s_j = scale * (ks_j (q . ck_j)),  p_j = 2^(s_j log2 e - m),
//   out = sum_j p_j vs_j cv_j / sum_j p_j
//
// with one scale for every 16 tokens, at least (see art_wave.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "art_internal.h"
#include "art_wave.h"

namespace art {
namespace {

constexpr int kD = kHeadDim;

template <int G>
struct Full {
  static constexpr int REP = G > 8 ? 1 : G > 4 ? 2 : 4;  // copies of the heads over the 16 score columns
  static constexpr int COLS = 16 / REP;
  static constexpr int NS = 4 / REP;                     // 16-token groups of a tile that a lane works on
  static constexpr int NP = G > 8 ? 3 : G > 4 ? 2 : 1;   // P operands of a K-step
  static constexpr int ND = G > 8 ? 8 : G > 4 ? 4 : 2;   // dims a lane holds in the end
  static constexpr int REC = G * kD + 2 * G;             // floats of a record: o, m, L
  // a wavefront's LDS: V's codes (8 KiB) and P's parts (up to 24 rows of 128
  // bytes); its record at a segment's end takes their place
  static constexpr int PARTS = G > 8 ? 0 : 24 * 128;
  static constexpr int WAVE_BYTES = 8192 + PARTS > REC * 4 ? 8192 + PARTS : REC * 4;
};

// The line of tiles.  A unit is what shares a length: a sequence (all its KV
// heads), or with a list per head one group.
__device__ __forceinline__ int seq_len(Params& P, int b) {
  const int64_t cap = (int64_t)P.max_pages << P.page_shift;
  const int L = P.seq_lens[b];
  return L < 0 ? 0 : (int)min((int64_t)L, cap);
}
__device__ __forceinline__ bool per_group_units(Params& P) { return P.block_list && P.list_per_head; }
__device__ __forceinline__ int unit_count(Params& P) {
  return per_group_units(P) ? P.batch * P.num_kv_heads : P.batch;
}
// blocks of a unit's traversal
__device__ __forceinline__ int unit_blocks(Params& P, int u, int L) {
  if (L == 0) return 0;
  if (!P.block_list) return (L + P.block_size - 1) / P.block_size;
  const int T = P.block_list_len[u];
  return T < 0 ? 0 : min(T, P.max_list);
}
__device__ __forceinline__ int unit_tiles(Params& P, int u) {
  const int L = seq_len(P, per_group_units(P) ? u / P.num_kv_heads : u);
  return P.block_list ? unit_blocks(P, u, L) * P.tiles_per_block : (L + kTile - 1) / kTile;
}
__device__ __forceinline__ int unit_heads(Params& P) { return per_group_units(P) ? 1 : P.num_kv_heads; }

// How the tiles are cut for `most` workgroups.  Up to as many groups:
//   kLine   the line in equal ranges, one to a workgroup
//   kParts  every group in parts of `part` tiles, of which there are no more
//           than `most`: for few groups, where a range would hold 16 tiles or
//           fewer (16 ragged sequences of up to 2K tokens 26.5 -> 19.3 us), and
//           whole groups where the longest is not much longer than a range (45
//           sequences of 376 to 1056 tokens, 8 heads: 36 -> 32.5 us)
// More groups (MANY): a workgroup would join its wavefronts at the end of every
// few tiles, so each wavefront works for itself.
//   kWaveLine  the line in equal ranges, one to a wavefront (256 sequences of
//              200 to 2000 tokens, 8 heads: 137 us by kLine, 123 so; of one
//              query head a group 131, 109)
//   kEach      every group to one wavefront: where the rounds of groups, each as
//              long as the longest one, end before the line's ranges with their
//              segments (4096 sequences of 100 tokens, 8 heads: 783 us by kLine,
//              310 by kWaveLine, 288 so)
// A segment's set-up and end take a wavefront about as long as 3 tiles (a
// workgroup, 8), so every group has kLead places for that on the line, before
// its tiles: a range of many short groups is then no longer than others (60
// sequences of 100 to 3000 tokens, 8 heads: 78 us without them and 53 with).
enum CutKind { kLine, kParts, kWaveLine, kEach };
struct Cut {
  CutKind kind;
  int64_t workers;   // ranges of the line
  int part;
};
template <bool MANY>
constexpr int kLead = MANY ? 3 : 8;
template <bool MANY>
__device__ __forceinline__ Cut cut_of(Params& P, int64_t total, int longest, int64_t most) {
  const int64_t groups = (int64_t)P.batch * P.num_kv_heads;
  if constexpr (MANY) {
    const int64_t waves = most * kWaves;
    if ((groups + waves - 1) / waves * (2 + longest) <= (total + 3 * groups) / waves + 3) return Cut{kEach, waves, 0};
    // (two records for each of its ranges, in the area of two for every chunk)
    return Cut{kWaveLine, max((int64_t)1, min(min(waves, groups * P.max_chunks), total)), 0};
  }
  const Cut line{kLine, max((int64_t)1, min(most, (total + kWaves - 1) / kWaves)), 0};
  if (2 * groups <= most) {
    if (total > 16 * most) return line;
    const int64_t room = most - groups;
    return Cut{kParts, most, max((int)((total + room - 1) / room), kWaves)};
  }
  if (longest <= (total + 8 * groups) / most + 6) return Cut{kParts, most, max(longest, 1)};
  return line;
}
__device__ __forceinline__ int parts_of(int tiles, int part) { return (tiles + part - 1) / part; }

__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor((long long)x, o);
  return x;
}

// ---- a tile's operands -------------------------------------------------------
// K: for 16-token group n, lane (lo, g) holds token 16n + lo, bytes 64j + 16g
// .. +15 (the query is read in the same order of the dims).  V: lane 8r + c
// holds token 8i + r, dims 16c .. 16c + 15.  Tokens past the sequence's end
// are redirected to its last one.  Every code is read once: past the caches (8 x
// 32K tokens 104 us with plain loads and 98 without, the ragged batch of 8K to
// 64K 397 and 381, 512K tokens 200 and 188).
struct Tile {
  u32x4 k[4][2];
  u32x4 v[8];
};
struct TileAt {
  int tok0;
  int pg[4];
};

__device__ __forceinline__ const uint8_t* rows_at(const uint16_t* pool, int64_t sp, int64_t sh, int64_t st, int pg,
                                                  int kvh, int slot) {
  return reinterpret_cast<const uint8_t*>(pool) + (int64_t)pg * sp + (int64_t)kvh * sh + (int64_t)slot * st;
}
__device__ __forceinline__ void load_k(Params& P, int kvh, int L, const TileAt& at, int lane, Tile& t) {
  const int lo = lane & 15, g = lane >> 4, mask = (1 << P.page_shift) - 1;
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const int t0 = min(at.tok0 + 16 * n, L - 1);
    const uint8_t* b = rows_at(P.k, P.ks_page, P.ks_head, P.ks_tok, at.pg[n], kvh, t0 & mask);
    const uint32_t o = __umul24(min(lo, L - 1 - t0), (uint32_t)P.ks_tok) + 16u * g;
#pragma unroll
    for (int j = 0; j < 2; ++j) t.k[n][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(b + (o + 64u * j)));
  }
}
__device__ __forceinline__ void load_v(Params& P, int kvh, int L, const TileAt& at, int lane, Tile& t) {
  const int mask = (1 << P.page_shift) - 1;
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const int t0 = min(at.tok0 + 16 * n, L - 1);
    const uint8_t* b = rows_at(P.v, P.vs_page, P.vs_head, P.vs_tok, at.pg[n], kvh, t0 & mask);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t o = __umul24(min(8 * j + (lane >> 3), L - 1 - t0), (uint32_t)P.vs_tok) + 16u * (lane & 7);
      t.v[2 * n + j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(b + o));
    }
  }
}

// What a wavefront reads ahead for 16 of its tiles: lane 4m + n holds the page
// and the scales of group n of tile m.
struct Ahead {
  int tok0, page;
  float ks, vs;
};

struct Segment {
  int b, kvh, L, T;      // T: blocks of the traversal
  int t0, n;             // its tiles of the group: t0 .. t0 + n - 1
  int off, step;         // of which this wavefront takes off, off + step, ...
  const int32_t* list;
};

// tiles of this wavefront
__device__ __forceinline__ int mine_of(const Segment& s) {
  return s.n > s.off ? (s.n - s.off + s.step - 1) / s.step : 0;
}

__device__ __forceinline__ void ahead_pages(Params& P, const Segment& s, int first, int n_mine,
                                            int lane, Ahead& a) {
  const int m = first + (lane >> 2);
  a.tok0 = 0;
  a.page = 0;
  if (m < n_mine) {
    const int tile = s.t0 + s.off + s.step * m;
    if (s.list) {
      const int i = tile / P.tiles_per_block, nblk = (s.L + P.block_size - 1) / P.block_size;
      int blk = s.list[i];
      blk = blk < 0 ? 0 : (blk >= nblk ? nblk - 1 : blk);
      a.tok0 = blk * P.block_size + (tile - i * P.tiles_per_block) * kTile;
    } else {
      a.tok0 = tile * kTile;
    }
    const int tok = min(a.tok0 + 16 * (lane & 3), s.L - 1);
    int pg = P.page_table[(int64_t)s.b * P.max_pages + (tok >> P.page_shift)];
    pg = pg < 0 ? 0 : pg;
    a.page = pg >= P.num_pages ? P.num_pages - 1 : pg;
  }
}
__device__ __forceinline__ void ahead_scales(Params& P, const Segment& s, int lane, Ahead& a) {
  const int tok = min(a.tok0 + 16 * (lane & 3), s.L - 1);
  const int run = (tok & ((1 << P.page_shift) - 1)) >> P.scale_shift;
  a.ks = P.k_scale[(int64_t)a.page * P.ksc_page + (int64_t)s.kvh * P.ksc_head + run];
  a.vs = P.v_scale[(int64_t)a.page * P.vsc_page + (int64_t)s.kvh * P.vsc_head + run];
}
__device__ __forceinline__ TileAt tile_at(const Ahead& a, int m) {
  TileAt t;
  t.tok0 = __builtin_amdgcn_readlane(a.tok0, 4 * m);
#pragma unroll
  for (int n = 0; n < 4; ++n) t.pg[n] = __builtin_amdgcn_readlane(a.page, 4 * m + n);
  return t;
}

// A wavefront's running state: the output sums in the accumulators of the
// P.V products (row 4g + r of A, dim 16d + lo), the maximum of the lane's
// head (base 2) and the lane's share of its mass.  The maximum is a reference
// that is moved only where a score passes it by more than 2^8 (and by the
// first score): the sums keep their relative precision either way, and a tile
// needs no reduction over the lanes, only a vote.  (Large values of V: by any
// score, see walk_tiles.)
struct State {
  f32x4 acc[8];
  float m, l;
};

template <int G, int FMT>
__device__ __forceinline__ void walk_tiles(Params& P, const Segment& s, int lane,
                                           const bf16x8 (&qa)[4], const Ahead (&first_sets)[2], uint8_t* stage,
                                           uint16_t* parts, State& st) {
  using C = Full<G>;
  constexpr int REP = C::REP, COLS = C::COLS, NS = C::NS, NP = C::NP;
  const int lo = lane & 15, g = lane >> 4, u = lo / COLS;
  const int n_mine = mine_of(s);
  if (n_mine == 0) return;
  // Pages are fetched two sets of 16 tiles ahead and scales one, before the
  // loads of a set's first tile: no wait for them then holds up for the tiles
  // in flight behind them.
  Ahead cur = first_sets[0], nxt = first_sets[1], far;
  ahead_scales(P, s, lane, cur);
  TileAt at = tile_at(cur, 0);
  Tile t;
  load_k(P, s.kvh, s.L, at, lane, t);
  load_v(P, s.kvh, s.L, at, lane, t);

#pragma unroll 1
  for (int first = 0; first < n_mine; first += 16) {
    const int n_set = min(16, n_mine - first);
    const TileAt over = tile_at(nxt, 0);
    ahead_scales(P, s, lane, nxt);
    ahead_pages(P, s, first + 32, n_mine, lane, far);
    // Where V is so large that 2^8 times a value of it, over the 2^29 tokens that
    // a traversal can have, could leave fp32's range (448 * 2^80 < 2^89), the
    // reference follows the maximum: no probability passes 1 and the sums have
    // the room of plain ones.
    const bool large = first + (lane >> 2) < n_mine && fabsf(cur.vs) >= 0x1p80f;
    const float slack = __any(large) ? 0.f : 8.f;
#pragma unroll 1
    for (int m = 0; m < n_set; ++m) {
      const int tok0 = at.tok0;
      // (behind the last tile one row of it over and over: the tile once more was
      // 6 % of the traffic of 8 x 32K tokens, and 24 sequences of 2K to 6K took 51
      // us, not 47)
      if (m + 1 < n_set) at = tile_at(cur, m + 1);
      else if (first + 16 < n_mine) at = over;
      else at.tok0 = s.L - 1;
      float ks[4], vs[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        ks[n] = read_lane(cur.ks, 4 * m + n);
        vs[n] = read_lane(cur.vs, 4 * m + n);
      }

      // scores, transposed: St[n][r] is token 16n + 4g + r, head lo mod COLS
      f32x4 St[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        St[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          St[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8, codes_bf16<FMT>(t.k[n][k >> 1], k & 1)), qa[k], St[n], 0, 0, 0);
      }
      // K's registers are free: the next tile's K is on its way while this one
      // goes through the softmax and P.V
      load_k(P, s.kvh, s.L, at, lane, t);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *reinterpret_cast<u32x4*>(stage + code_stage_off(8 * j + (lane >> 3), lane & 7)) = t.v[j];
      load_v(P, s.kvh, s.L, at, lane, t);
      __builtin_amdgcn_sched_barrier(0);

      float sc[NS][4];
      float top = kNegInf;
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        const float c = own_scale<REP>(ks[0], ks[1], ks[2], ks[3], j, u) * P.scale_log2;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float x = St[REP * j][r];
          if constexpr (REP == 2) {
            x = u ? St[2 * j + 1][r] : x;
          } else if constexpr (REP == 4) {
            const float y = (u & 1) ? St[1][r] : x, z = (u & 1) ? St[3][r] : St[2][r];
            x = (u & 2) ? z : y;
          }
          sc[j][r] = x * c;
        }
      }
      if (tok0 + kTile > s.L) {
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (tok0 + 16 * (REP * j + u) + 4 * g + r >= s.L) sc[j][r] = kNegInf;
      }
#pragma unroll
      for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, sc[j][r]);
      if (__any(top > st.m + slack)) {
        if constexpr (REP >= 2) top = fmaxf(top, dpp_f<kRowRor8>(top));
        if constexpr (REP == 4) top = fmaxf(top, dpp_f<kRowRor4>(top));
        const float mn = fmaxf(st.m, rows_max(top));
        const float a = st.m == kNegInf ? 0.f : fast_exp2(st.m - mn);
        st.m = mn;
        st.l *= a;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // the factor of row 4g + r's head
          float f = read_lane(a, r);
          if constexpr (COLS >= 8) f = (g & 1) ? read_lane(a, 4 + r) : f;
          if constexpr (COLS == 16) f = g == 2 ? read_lane(a, 8 + r) : g == 3 ? read_lane(a, 12 + r) : f;
#pragma unroll
          for (int d = 0; d < 8; ++d) st.acc[d][r] *= f;
        }
      }
      const float ref = st.m == kNegInf ? 0.f : st.m;
#pragma unroll
      for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          sc[j][r] = fast_exp2(sc[j][r] - ref);
          st.l += sc[j][r];
        }

      // P times V's scales, in three bf16 parts (24 significant bits); the
      // parts' rows of A are laid out as in the decode kernel: up to four heads
      // have all of them in one operand, eight in two
      uint32_t own[NS][3][2];
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        const float c = own_scale<REP>(vs[0], vs[1], vs[2], vs[3], j, u);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float a0 = sc[j][2 * e] * c, a1 = sc[j][2 * e + 1] * c;
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            const uint32_t w = pack_bf16(a0, a1);
            own[j][k][e] = w;
            a0 = a0 - bf_lo(w);
            a1 = a1 - bf_hi(w);
            if (G <= 8 && k == 1) {
              a0 = 0.5f * a0;
              a1 = 0.5f * a1;
            }
          }
        }
      }
      bf16x8 a[2][NP];
      if constexpr (G > 8) {
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
          for (int c = 0; c < 2; ++c)
            a[c][k] = __builtin_bit_cast(
                bf16x8, u32x4{own[2 * c][k][0], own[2 * c][k][1], own[2 * c + 1][k][0], own[2 * c + 1][k][1]});
      } else {
        const int h = lo & (COLS - 1);
#pragma unroll
        for (int k = 0; k < (G > 4 ? 3 : 4); ++k)
#pragma unroll
          for (int j = 0; j < NS; ++j)
            *reinterpret_cast<u32x2*>(parts + (COLS * k + h) * 64 + g * 16 + 4 * (REP * j + u)) =
                u32x2{own[j][k < 3 ? k : 2][0], own[j][k < 3 ? k : 2][1]};
        wave_lds_order();
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          a[c][0] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(parts + lo * 64 + g * 16 + 8 * c));
          if constexpr (NP == 2)
            a[c][1] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(parts + (16 + h) * 64 + g * 16 + 8 * c));
        }
      }
      wave_lds_order();

      // P.V: element e of lane (lo, g) of K-step c is token 16(2c + e/4) + 4g +
      // e%4, dim 16d + lo
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int k = lo >> 1, row = 16 * (2 * c + (k >> 2)) + 4 * g + (k & 3);
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          const bf16x8 b = codes_tr<FMT>(stage, row, d, lo);
#pragma unroll
          for (int j = 0; j < NP; ++j)
            st.acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[c][j], b, st.acc[d], 0, 0, 0);
        }
      }
      wave_lds_order();   // these reads come before the next tile's writes
    }
    cur = nxt;
    nxt = far;
  }
}

// The wavefront's record into LDS: o (sums relative to m), m, L.
template <int G>
__device__ __forceinline__ void leave_record(State& st, float* rec, int lane) {
  using C = Full<G>;
  constexpr int ND = C::ND;
  const int lo = lane & 15, g = lane >> 4;
  float l = st.l;
  if constexpr (C::REP >= 2) l = l + dpp_f<kRowRor8>(l);
  if constexpr (C::REP == 4) l = l + dpp_f<kRowRor4>(l);
  l = rows_sum(l);
  // the parts' rows are added by swapping halves (then rows) of accumulators
  f32x4 sum[ND];
  if constexpr (G > 8) {
#pragma unroll
    for (int d = 0; d < ND; ++d) sum[d] = st.acc[d];
  } else {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_int(st.acc[d][r]), __float_as_int(st.acc[d + 4][r]), false, false);
        st.acc[d][r] = __int_as_float(x[0]) + __int_as_float(x[1]);
      }
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (G > 4) {
          sum[d][r] = st.acc[d][r];
        } else {
          const auto x = __builtin_amdgcn_permlane16_swap(__float_as_int(st.acc[d][r]), __float_as_int(st.acc[d + 2][r]), false, false);
          sum[d][r] = __int_as_float(x[0]) + __int_as_float(x[1]);
        }
      }
  }
  const int h0 = G > 8 ? 4 * g : G > 4 ? 4 * (g & 1) : 0;
  float* const to = rec + h0 * kD + 16 * (G > 8 ? 0 : G > 4 ? 4 * (g >> 1) : 2 * g) + lo;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (r < G) {
#pragma unroll
      for (int d = 0; d < ND; ++d) to[r * kD + 16 * d] = sum[d][r];
    }
  if (g == 0 && lo < G) {
    rec[G * kD + lo] = st.m;
    rec[G * kD + G + lo] = l;
  }
}

__device__ __forceinline__ void write_out(Params& P, int64_t i, float x) {
  if (P.out_bf16) static_cast<uint16_t*>(P.out)[i] = (uint16_t)f32_to_bf16_bits(x);
  else static_cast<float*>(P.out)[i] = x;
}
__device__ __forceinline__ float ln_of(float m, float L) { return (m + __log2f(L)) * 0.69314718055994531f; }

// What a record of maximum m (base 2) counts for beside the largest one, `top`.
__device__ __forceinline__ float factor(float m, float top) { return m == kNegInf ? 0.f : fast_exp2(m - top); }

// What the first launch tells the second of a group that holds tiles: the
// workgroups that hold it (one: it is written) and how it was cut.  (In the
// workspace's flag words; bits 24 and up stay far below any call's tag there.)
__device__ __forceinline__ uint64_t split_word(int64_t first, int64_t last, bool in_parts) {
  return (uint64_t)last << 24 | (in_parts ? 1ull << 23 : 0ull) | (uint64_t)first;
}

template <int G, int FMT, bool MANY>
__global__ void __launch_bounds__(kThreads, 2) full_kernel(const KernelParams, const int most) {
  Params* const args = (Params*)__builtin_amdgcn_kernarg_segment_ptr();
  Params& P = *args;
  using C = Full<G>;
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ int64_t s_wave[2][kWaves];
  __shared__ int64_t s_base[kWaves];
  __shared__ int s_unit[kWaves], s_longest[kWaves];
  // (the wavefront's number in a scalar register: everything that follows from
  // it, page addresses above all, then stays there too)
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int units = unit_count(P), heads = unit_heads(P);

  // the tiles of all units, and the most that a group has
  int64_t total = 0;
  int longest = 0;
  for (int u = tid; u < units; u += kThreads) {
    const int n = unit_tiles(P, u);
    total += n;
    longest = max(longest, n);
  }
  total = wave_sum(total);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) longest = max(longest, __shfl_xor(longest, o));
  if (lane == 0) {
    s_wave[0][wave] = total;
    s_longest[wave] = longest;
  }
  __syncthreads();
  total = longest = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    total += s_wave[0][w];
    longest = max(longest, s_longest[w]);
  }
  const Cut cut = cut_of<MANY>(P, uniform(total * heads), __builtin_amdgcn_readfirstlane(longest), most);

  float* const rec = reinterpret_cast<float*>(lds + wave * C::WAVE_BYTES);
  uint8_t* const stage = lds + wave * C::WAVE_BYTES;
  uint16_t* const parts = reinterpret_cast<uint16_t*>(stage + 8192);
  // what a segment begins with: its group's query and its first pages.  They
  // are asked for while the segment before is joined and written.
  bf16x8 qa[4];
  Ahead sets[2];
  auto ask = [&](const Segment& s) {
    Params& P = *fresh(args);
    ahead_pages(P, s, 0, mine_of(s), lane, sets[0]);
    ahead_pages(P, s, 16, mine_of(s), lane, sets[1]);
    const int head = (lane & 15) & (C::COLS - 1);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      u32x4 w{0u, 0u, 0u, 0u};
      if (head < G)
        w = *reinterpret_cast<const u32x4*>(P.q + ((int64_t)s.b * P.num_q_heads + s.kvh * G + head) * kD +
                                            64 * (k >> 1) + 16 * (lane >> 4) + 8 * (k & 1));
      qa[k] = __builtin_bit_cast(bf16x8, w);
    }
  };
  State st;
  auto clear = [&]() {
    st.m = kNegInf;
    st.l = 0.f;
#pragma unroll
    for (int d = 0; d < 8; ++d) st.acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  };

  // A scan of the units' weights (places on the line, or parts): thread tid has
  // units u0 .. u1 - 1, `own` places behind the first `before`; returns the line.
  const int per = (units + kThreads - 1) / kThreads;
  const int u0 = tid * per, u1 = min(units, u0 + per);
  auto scan = [&](auto weight, int64_t& own, int64_t& before) {
    own = 0;
    for (int u = u0; u < u1; ++u) own += weight(u);
    before = own;   // inclusive scan over the wavefront, then the workgroup
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t x = __shfl_up((long long)before, o);
      if (lane >= o) before += x;
    }
    if (lane == 63) s_wave[1][wave] = before;
    __syncthreads();
    int64_t line = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) before += s_wave[1][w];
      line += s_wave[1][w];
    }
    before -= own;
    return uniform(line);
  };
  // (one thread) the unit that holds place `at`
  auto find = [&](auto weight, int64_t at, int64_t own, int64_t before, int i) {
    if (before <= at && at < before + own) {
      int u = u0;
      int64_t base = before;
      for (int64_t n; base + (n = weight(u)) <= at; ++u) base += n;
      s_unit[i] = u;
      s_base[i] = base;
    }
  };

  if constexpr (MANY) {
    const int64_t me = (int64_t)blockIdx.x * kWaves + wave, workers = cut.workers;
    const bool each_one = cut.kind == kEach;
    int64_t line = 0, x = 0, end = 0, base = 0;
    int u = 0;
    auto places = [&](int tiles) { return tiles == 0 ? 0 : kLead<true> + tiles; };
    if (!each_one) {
      auto weight = [&](int u) { return (int64_t)heads * places(unit_tiles(P, u)); };
      int64_t own, before;
      line = scan(weight, own, before);
#pragma unroll 1
      for (int i = 0; i < kWaves; ++i) {
        const int64_t w = (int64_t)blockIdx.x * kWaves + i;
        if (w < workers) find(weight, uniform(w * line / workers), own, before, i);
      }
      __syncthreads();
      if (me >= workers) return;
      x = uniform(me * line / workers);
      end = uniform((me + 1) * line / workers);
      if (x >= end) return;
      u = __builtin_amdgcn_readfirstlane(s_unit[wave]);
      base = uniform(s_base[wave]);
    }
    // A segment: of the line, its group's places begin at `start`; of kEach, a
    // group that holds tiles (the second launch writes empty ones).
    const int groups = P.batch * P.num_kv_heads;
    int64_t start = 0;
    int tiles = 0, group = (int)me;
    auto next_segment = [&](Segment& s) {
      s.off = 0;
      s.step = 1;
      while (each_one ? group < groups : x < end) {
        Params& P = *fresh(args);
        int v = u;   // its unit
        if (each_one) {
          s.b = group / P.num_kv_heads;
          s.kvh = group - s.b * P.num_kv_heads;
          v = per_group_units(P) ? group : s.b;
          s.n = tiles = __builtin_amdgcn_readfirstlane(unit_tiles(P, v));
          s.t0 = 0;
          group += most * kWaves;
        } else {
          tiles = __builtin_amdgcn_readfirstlane(unit_tiles(P, u));
          while (x >= base + (int64_t)places(tiles) * heads) {
            base += (int64_t)places(tiles) * heads;
            tiles = __builtin_amdgcn_readfirstlane(unit_tiles(P, ++u));
          }
          const int h = __builtin_amdgcn_readfirstlane((int)((x - base) / places(tiles)));
          start = base + (int64_t)h * places(tiles);
          const int64_t next = min(end, start + places(tiles));
          s.t0 = max((int)(x - start) - kLead<true>, 0);
          s.n = (int)(next - start) - kLead<true> - s.t0;
          x = next;
          v = u;
          s.b = per_group_units(P) ? u / P.num_kv_heads : u;
          s.kvh = per_group_units(P) ? u % P.num_kv_heads : h;
        }
        if (s.n <= 0) continue;
        s.L = __builtin_amdgcn_readfirstlane(seq_len(P, s.b));
        s.list = P.block_list ? P.block_list + (int64_t)v * P.max_list : nullptr;
        return true;
      }
      return false;
    };
    Segment s;
    bool more = next_segment(s);
    if (more) ask(s);
    while (more) {
      clear();
      walk_tiles<G, FMT>(*fresh(args), s, lane, qa, sets, stage, parts, st);
      const int b = s.b, kvh = s.kvh;
      const bool whole = s.n == tiles, begins = s.t0 == 0;
      const int64_t behind = start + kLead<true> + tiles;   // the place behind its last tile's
      more = next_segment(s);
      if (more) ask(s);
      leave_record<G>(st, rec, lane);
      wave_lds_sync();
      Params& W = *fresh(args);
      if (whole) {
        const int64_t row0 = (int64_t)b * W.num_q_heads + kvh * G;
        for (int i = lane; i < G * kD; i += 64) write_out(W, row0 * kD + i, rec[i] / rec[G * kD + G + i / kD]);
        if (lane < G) W.lse[row0 + lane] = ln_of(rec[G * kD + lane], rec[G * kD + G + lane]);
      } else {
        // (a group that began in an earlier range: this one's first place, one
        // that began here and goes on: its second)
        float* const to = W.records + (2 * me + (begins ? 1 : 0)) * W.record_floats;
        for (int i = lane; i < C::REC; i += 64) to[i] = rec[i];
      }
      // who holds it: up to the last w with w line / workers <= its last tile's place
      if (begins && lane == 0)
        W.flags[(int64_t)b * W.num_kv_heads + kvh] = split_word(me, whole ? me : (behind * workers - 1) / line, false);
      wave_lds_sync();   // the record is read before the next segment's tiles
    }
    return;
  }

  // this workgroup's part of the line, and the unit where it begins
  const bool in_parts = cut.kind == kParts;
  auto weight = [&](int u) {
    const int n = unit_tiles(P, u);
    return (int64_t)heads * (n == 0 ? 0 : in_parts ? parts_of(n, cut.part) : n + kLead<false>);
  };
  int64_t own, before;
  const int64_t line = scan(weight, own, before);   // places on the line, or parts
  const int64_t workers = in_parts ? line : cut.workers, me = blockIdx.x;
  if (me >= workers) return;
  const int64_t begin = in_parts ? me : uniform(me * line / workers);
  const int64_t end = in_parts ? me + 1 : uniform((me + 1) * line / workers);
  if (begin >= end) return;
  find(weight, begin, own, before, 0);
  __syncthreads();
  int u = __builtin_amdgcn_readfirstlane(s_unit[0]);
  int64_t base = uniform(s_base[0]);

  // A segment and where it lies: its group's places on the line (or its parts)
  // begin at `start` and are `each` of them.
  int64_t x = begin, start = 0;
  int tiles = 0, each = 0;
  auto next_segment = [&](Segment& s) {
    while (x < end) {
      Params& P = *fresh(args);
      tiles = __builtin_amdgcn_readfirstlane(unit_tiles(P, u));
      while (!in_parts && (tiles == 0 || x >= base + (int64_t)(tiles + kLead<false>) * heads)) {
        base += tiles == 0 ? 0 : (int64_t)(tiles + kLead<false>) * heads;
        tiles = __builtin_amdgcn_readfirstlane(unit_tiles(P, ++u));
      }
      each = in_parts ? parts_of(tiles, cut.part) : tiles + kLead<false>;
      const int h = __builtin_amdgcn_readfirstlane((int)((x - base) / each));
      start = base + (int64_t)h * each;
      const int64_t next = min(end, start + each);
      s.t0 = in_parts ? (int)(x - start) * cut.part : max((int)(x - start) - kLead<false>, 0);
      s.n = in_parts ? min(cut.part, tiles - s.t0) : (int)(next - start) - kLead<false> - s.t0;
      x = next;
      if (s.n <= 0) continue;   // only the places before its tiles
      s.b = per_group_units(P) ? u / P.num_kv_heads : u;
      s.kvh = per_group_units(P) ? u % P.num_kv_heads : h;
      s.L = __builtin_amdgcn_readfirstlane(seq_len(P, s.b));
      s.off = wave;
      s.step = kWaves;
      s.list = P.block_list ? P.block_list + (int64_t)u * P.max_list : nullptr;
      return true;
    }
    return false;
  };
  Segment s;
  bool more = next_segment(s);
  if (more) ask(s);
  while (more) {
    clear();
    walk_tiles<G, FMT>(*fresh(args), s, lane, qa, sets, stage, parts, st);
    const int b = s.b, kvh = s.kvh;
    const bool whole = s.n == tiles, begins = s.t0 == 0;
    // who holds the group: the last w with w line / workers <= its last place
    const int64_t last = in_parts ? me + each - 1 : ((start + each) * workers - 1) / line;
    more = !in_parts && next_segment(s);
    if (more) ask(s);
    leave_record<G>(st, rec, lane);
    __syncthreads();

    // the wavefronts' records joined: thread tid takes values tid, tid + 256 ..
    Params& W = *fresh(args);
    // (of the line) a group that began in an earlier workgroup leaves its record in
    // this one's first place, one that began here and goes on in its second
    float* const to = W.records + (in_parts ? me : 2 * me + (begins ? 1 : 0)) * W.record_floats;
    if (begins && tid == 0) W.flags[(int64_t)b * W.num_kv_heads + kvh] = split_word(me, last, in_parts);
    const int64_t row0 = (int64_t)b * W.num_q_heads + kvh * G;
#pragma unroll 1
    for (int i = tid; i < G * kD; i += kThreads) {
      const int h2 = i / kD;
      float m[kWaves], top = kNegInf;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        m[w] = reinterpret_cast<const float*>(lds + w * C::WAVE_BYTES)[G * kD + h2];
        top = fmaxf(top, m[w]);
      }
      float o = 0.f, L = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float* r = reinterpret_cast<const float*>(lds + w * C::WAVE_BYTES);
        const float f = factor(m[w], top);
        o += r[i] * f;
        L += r[G * kD + G + h2] * f;
      }
      if (whole) {
        write_out(W, row0 * kD + i, o / L);
        if (i % kD == 0) W.lse[row0 + h2] = ln_of(top, L);
      } else {
        to[i] = o;
        if (i % kD == 0) {
          to[G * kD + h2] = top;
          to[G * kD + G + h2] = L;
        }
      }
    }
    if (more) __syncthreads();   // the records are read before the next segment's tiles
  }
}

// The second launch: `each` query heads to a workgroup.  Groups in several
// workgroups are joined from their records, in the order of the line; empty
// ones are written; every group's stop_block is its number of blocks.
template <int G>
__global__ void __launch_bounds__(kThreads) join_kernel(const KernelParams, const int each) {
  Params& P = *(Params*)__builtin_amdgcn_kernarg_segment_ptr();
  __shared__ float s_o[kThreads], s_l[kThreads];
  const int tid = threadIdx.x, lane = tid & 63, d = tid & (kD - 1);
  const int64_t items = (int64_t)P.batch * P.num_kv_heads * G;
  for (int64_t it = (int64_t)blockIdx.x * each; it < min(items, ((int64_t)blockIdx.x + 1) * each); ++it) {
    const int gidx = (int)(it / G), hq = (int)(it - (int64_t)gidx * G);
    const int b = gidx / P.num_kv_heads, kvh = gidx - b * P.num_kv_heads;
    const int unit = per_group_units(P) ? gidx : b;
    const uint64_t split = P.flags[gidx];
    const int64_t row = (int64_t)b * P.num_q_heads + kvh * G + hq;
    const int blocks = unit_blocks(P, unit, seq_len(P, b));
    if (hq == 0 && tid == 0) P.stop_block[gidx] = blocks;
    if (blocks == 0) {
      if (tid < kD) write_out(P, row * kD + tid, 0.f);
      if (tid == 0) P.lse[row] = kNegInf;
      continue;
    }
    const int first = (int)(split & 0x7fffffu), last = (int)(split >> 24), n = last - first + 1;
    const bool in_parts = (split >> 23) & 1u;
    if (n == 1) continue;   // written by its workgroup
    // (of a line, the group's first record is in its workgroup's second place)
    auto record = [&](int i) {
      return P.records + (int64_t)(in_parts ? first + i : 2 * (first + i) + (i == 0 ? 1 : 0)) * P.record_floats;
    };
    float top = kNegInf;
    for (int i = lane; i < n; i += 64) top = fmaxf(top, record(i)[G * kD + hq]);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    float o = 0.f, l = 0.f;
#pragma unroll 4
    for (int i = tid / kD; i < n; i += kThreads / kD) {
      const float* r = record(i);
      const float f = factor(r[G * kD + hq], top);
      o += r[hq * kD + d] * f;
      l += r[G * kD + G + hq] * f;
    }
    s_o[tid] = o;
    s_l[tid] = l;
    __syncthreads();
    if (tid < kD) {
      const float os = s_o[tid] + s_o[tid + kD], ls = s_l[tid] + s_l[tid + kD];
      write_out(P, row * kD + tid, os / ls);
      if (tid == 0) P.lse[row] = ln_of(top, ls);
    }
    __syncthreads();   // read before the next one's
  }
}

// Workgroups of full_kernel that the current device holds at once (asked of
// the runtime once per device: the two queries cost about a microsecond).
template <int G, int FMT>
hipError_t resident(int* n) {
  constexpr int kDevices = 64;
  static std::atomic<int> known[kDevices];
  int dev = 0, cus = 0, per_cu = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  *n = dev < kDevices ? known[dev].load(std::memory_order_relaxed) : 0;
  if (*n > 0) return hipSuccess;
  e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e == hipSuccess)
    e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, full_kernel<G, FMT, false>, kThreads,
                                                     (size_t)kWaves * Full<G>::WAVE_BYTES);
  *n = cus * max(per_cu, 1);
  if (e == hipSuccess && dev < kDevices) known[dev].store(*n, std::memory_order_relaxed);
  return e;
}

template <int G, int FMT>
int launch(const Plan& plan, const KernelParams& params, hipStream_t stream) {
  const size_t bytes = (size_t)kWaves * Full<G>::WAVE_BYTES;
  int held = 0;
  hipError_t e = resident<G, FMT>(&held);
  if (e != hipSuccess) return (int)e;
  // as many workgroups as the chip holds, two records for each in the plan's
  // area, and no more than the longest sequences could use
  const int64_t cap = (int64_t)params.max_pages << params.page_shift;
  const int64_t tiles = (int64_t)plan.n_groups * max((cap + kTile - 1) / kTile, (int64_t)params.max_list * params.tiles_per_block);
  const int64_t most = min(min((int64_t)held, (int64_t)plan.n_groups * plan.max_chunks),
                           (tiles + kWaves - 1) / kWaves + plan.n_groups);
  const dim3 grid((unsigned)most), block(kThreads);
  if (plan.n_groups > most) hipLaunchKernelGGL((full_kernel<G, FMT, true>), grid, block, bytes, stream, params, (int)most);
  else hipLaunchKernelGGL((full_kernel<G, FMT, false>), grid, block, bytes, stream, params, (int)most);
  e = hipGetLastError();
  if (e != hipSuccess) return (int)e;
  // one head to a workgroup, and of many, most of them written already, up to 16
  // (a launch has less than 2^32 threads)
  const int64_t items = (int64_t)plan.n_groups * G;
  const int each = (int)max(min(max(items >> 12, (int64_t)1), (int64_t)16), items >> 22);
  hipLaunchKernelGGL(join_kernel<G>, dim3((unsigned)((items + each - 1) / each)), dim3(kThreads), 0, stream, params, each);
  return (int)hipGetLastError();
}

template <int FMT>
int launch_group(const Plan& plan, const KernelParams& params, hipStream_t stream) {
  switch (plan.group) {
    case 1: return launch<1, FMT>(plan, params, stream);
    case 2: return launch<2, FMT>(plan, params, stream);
    case 4: return launch<4, FMT>(plan, params, stream);
    case 8: return launch<8, FMT>(plan, params, stream);
    case 16: return launch<16, FMT>(plan, params, stream);
    default: return (int)hipErrorInvalidValue;
  }
}

}  // namespace

int launch_quant_full(const Plan& plan, const KernelParams& params, int format, hipStream_t stream) {
  return format == ART_QUANT_E4M3 ? launch_group<ART_QUANT_E4M3>(plan, params, stream)
                                  : launch_group<ART_QUANT_INT8>(plan, params, stream);
}

}  // namespace art
