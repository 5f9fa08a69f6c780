// Attention of a batch of sequences to a prefix that all of them share and to the pages of their own:
//   o = sum_j e^(scale q.k_j) v_j / sum_j e^(scale q.k_j),   j over prefix ++ own rows (causal: up to the token's own)
//
// Rows.  The query heads that share a key head and the tokens of a sequence are rows of one matrix: row r of sequence b and
// key head h is token offsets[b] + r / group, query head h * group + r % group.  A tile is R of these rows.
//
// The line.  The work of a launch is one line: for every key head, every sequence, every tile of its rows, the keys
// that the tile attends to, prefix first.  It is cut into equal shares, one per workgroup, wherever the cuts fall
// (in the tile at the next unit of keys); lengths are read on the device, so a captured call follows the sequences as
// they grow.  A workgroup finds the start of its share by a scan over the sequences, and walks.  What a share holds of a tile
// is a piece; a piece that is not its whole tile leaves its maximum, sum and un-normalised product in the workspace, and
// combine_kernel adds the pieces of every row up, in the order of the keys: results are run-to-run identical.
//
// Prefix, computed once.  Where sequences have few rows each, the line has two parts: the prefix against tiles that are cut
// from the rows of all sequences together, so that its keys are read once per tile of the whole batch and not per
// sequence, and behind it every sequence's own keys; combine_kernel joins the two.  Where a sequence fills tiles by
// itself, or prefix and batch are small, that would save nothing: there its tiles run over prefix and own keys in one go (choose()).
//
// A wave.  S^T = K Q^T with v_mfma_f32_16x16x32_bf16 (A = 16 keys x 32 channels, B = 32 channels x 16 rows): a lane has
// one row's scores of 4 of 16 keys, so that statistics are sums in a lane and two exchanges.  The weights go from the
// accumulators straight into the B operand of O^T += V^T P^T, which fixes the order of keys in an operand (lane group
// g: 4 g + 0..3 and 16 + 4 g + 0..3); V^T in that order are two transposing LDS reads of the row-major rows.  The
// waves of a workgroup take a share's units in turn and meet at the end of the piece.
//
// Softmax.  m is a running shift, not the maximum: it follows when a score is more than 2^kSlack above it, which
// after the first unit is rare, and a comparison per score pays for it.
//
// Rounding.  Scores, shifts, sums and products are held in fp32.  Weights are rounded to bf16 once, as the matrix instruction takes them: half a step of
// each, 2^-8 at most, which random errors leave at 0.0023 of the output, root mean square, with the output's own rounding; fp32
// weights would leave 0.0017, for twice the products with V.  Tiles of few rows add up the weights in front of that rounding.  Tiles of 256 rows
// add them up behind it, two in an instruction (v_dot2_f32_bf16) where unrounded ones take an addition each: what a weight is off then enters sum and
// product alike, sum p (v - o) instead of sum p v.
//
// Measured, and what bounds it.  Tiles of few rows: memory, 64 streams of 100 to 5496 rows behind 28 700 shared keys, 16 heads, 160 us, 5.3 TB/s of
// what has to be read (a sum over 2 GiB reaches 6.16); one token to 5516 keys, 16 heads, is a chain of latencies, 10.7 us for 3.9 us of reading.
// The same from a cache in 4 bits: 64 streams of 100 to 21 984 rows, 32 heads on 8, 86 us, 4.5 TB/s of the 375 MB that come (32 of a
// unit's 116 vector instructions turn codes into values).  Tiles of 256 rows from it: 551 to 574 us where the same rows in 16 bits take 592, 4 x 1374 tokens to 5516 shared
// and up to 27 480 own keys, 16 heads.
// Tiles of 256 rows: vector issue and power, 4 frames of 1374 tokens behind 28 650 shared keys, 16 heads, 0.90 to 0.95 PFLOP/s in the loop (a bf16
// product of 8192^3 reaches 1.20).
#include <algorithm>
#include <type_traits>

#include "attention_common.hpp"
#include "dev_common.hpp"
#include "kernels.hpp"
#include "mx4.hpp"

namespace httm {

namespace {

// What a kernel is made for: the cache's rows in 16 bits; the same, with the logarithms of the sums (which cost others registers that they do not
// have: 2.8 % of the time of tiles of 256 rows); rows in 4 bits, with or without them, behind a prefix or alone
enum { ROWS, ROWS_AND_SUMS, MX4_ROWS, MX4_ALONE };

constexpr int kUnit = 32;                       // keys
constexpr int kUnitBytes = kUnit * kRowBytes;
constexpr float kSlack = 10.f;
constexpr float kLowest = -3.402823466e38f;     // a finite shift for sums without a key

// Where the pieces of a row of q are, as rows of the workspace: the first in `first`, the i-th in base + i * stride
struct RowPieces {
  int32_t first, base, stride, n;   // n = 0: the row is written already
};

// A part of the line
struct Part {
  int32_t stacked;        // one sequence that has the tokens of all of them
  int32_t with_prefix, with_own;
  int32_t max_slots;
  RowPieces* rows;        // [n_tokens * H_q]
  float2* slot_ml;        // [max_slots][R] shift (log2 units) and sum
  float* slot_o;          // [max_slots][R][64]
};
struct LineArgs {
  CachedAttnArgs c;
  int32_t H_q;
  uint32_t group_magic;   // ceil(2^32 / group), for more than 1
  int32_t finish;         // (one part) whole tiles are written to o; else every piece is left in its slot
  int32_t min_length;     // positions that a share has at least
  Part part[2];
};

// over the four lane groups that share a row
__device__ __forceinline__ float groups_max(float x) {
  LanePair p = swap16(x);
  p = swap32(fmaxf(p.a, p.b));
  return fmaxf(p.a, p.b);
}
__device__ __forceinline__ float groups_sum(float x) {
  LanePair p = swap16(x);
  p = swap32(p.a + p.b);
  return p.a + p.b;
}
// (the IEEE 754-2019 maximum: fmaxf() would quiet every operand with an instruction of its own first)
__device__ __forceinline__ float max8(const f32x4& a, const f32x4& b) {
  auto max3 = [](float x, float y, float z) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, y), z); };
  return max3(max3(a[0], a[1], a[2]), max3(a[3], b[0], b[1]), __builtin_elementwise_maximum(b[2], b[3]));
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32) | (uint32_t)uniform((int)x));
}

// floor(x / y) for 0 <= x, 0 < y, both below 2^52: the compiler's 64-bit division takes some 200 instructions, in front of
// everything else that a workgroup does
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
  int64_t q = (int64_t)((double)x / (double)y);
  const int64_t r = x - q * y;
  q += r < 0 ? -1 : (r >= y ? 1 : 0);
  return uniform64(q);
}

// A sequence as the line sees it.  Positions on the line are units of kUnit keys, or single keys where tiles are large (FINE).  A
// tile is as long as the keys that its last row sees, behind its front; with `causal` and FINE those grow by `grow` from tile to
// tile (rounded down, the last tile apart: lengths on the line only share out the work).
struct Seq {
  int first, n;    // tokens
  int len;         // own keys
  int tiles;       // of R rows
  int last;        // length of the last tile
  int base, grow;  // of tile j before the last: base + grow * (j + 1)
  __device__ __forceinline__ int64_t before(int j) const { return (int64_t)j * base + (int64_t)grow * j * (j + 1) / 2; }
  __device__ __forceinline__ int length(int j) const { return j == tiles - 1 ? last : base + grow * (j + 1); }
  __device__ __forceinline__ int64_t total() const { return tiles ? before(tiles - 1) + last : 0; }
  // the tile that has position x of the sequence
  __device__ __forceinline__ int tile_at(int64_t x) const {
    if (tiles == 1) return 0;
    int64_t j;
    if (grow == 0) {
      j = quotient(x, base);
    } else {
      const double b = 2.0 * base + grow;
      j = (int64_t)((sqrt(b * b + 8.0 * grow * (double)x) - b) / (2.0 * grow));
    }
    int t = uniform((int)std::clamp<int64_t>(j, 0, tiles - 1));
    while (t > 0 && before(t) > x) --t;
    while (t + 1 < tiles && before(t + 1) <= x) ++t;
    return t;
  }
};
// What a tile costs besides its keys - rows in, statistics and product joined and out - in positions: its front.  Fronts of 128 / 256 / 512
// keys for few rows: a token each of 256 streams 89.8 / 93.6 / 107 us, of 64 short ones 20.6 / 22.0 / 24.6.
template <bool FINE>
constexpr int kTileFront = FINE ? 256 : 128 / kUnit;

template <int R, bool CAUSAL, bool FINE>
__device__ __forceinline__ void measure(const LineArgs& a, const Part& part, Seq& s) {
  const int P = part.with_prefix ? (int)a.c.P : 0;
  s.tiles = (s.n * a.c.group + R - 1) / R;
  s.last = kTileFront<FINE> + (FINE ? P + s.len : (P + kUnit - 1) / kUnit + (s.len + kUnit - 1) / kUnit);
  const bool grows = FINE && CAUSAL && part.with_own;
  s.grow = !grows ? 0 : a.c.group < R ? R / a.c.group : 1;
  s.base = !grows ? s.last : std::max(s.last - s.n, kTileFront<FINE>);
}
// 64 sequences from `base` on, one per lane; those behind the last have no tokens
template <int R, bool CAUSAL, bool FINE>
__device__ __forceinline__ Seq load_window(const LineArgs& a, const Part& part, int base, int lane) {
  const CachedAttnArgs& c = a.c;
  const int n_seq = part.stacked ? 1 : c.cache.n_seqs, b = base + lane, T = (int)c.n_tokens;
  Seq s = {};
  if (b < n_seq) {
    const int o0 = c.offsets[b], o1 = c.offsets[part.stacked ? c.cache.n_seqs : b + 1];
    const int len = part.with_own ? c.seq_lens[b] : 0;
    s.first = std::clamp(o0, 0, T);
    s.n = std::clamp(o1, s.first, T) - s.first;
    s.len = std::clamp(len, 0, c.cache.table_stride << c.cache.page_shift);
  }
  measure<R, CAUSAL, FINE>(a, part, s);
  return s;
}
template <int R, bool CAUSAL, bool FINE>
__device__ __forceinline__ Seq of_lane(const LineArgs& a, const Part& part, const Seq& window, int l) {
  Seq s;
  s.first = __builtin_amdgcn_readlane(window.first, l);
  s.n = __builtin_amdgcn_readlane(window.n, l);
  s.len = __builtin_amdgcn_readlane(window.len, l);
  measure<R, CAUSAL, FINE>(a, part, s);
  return s;
}

// A part of the line in all, for a key head
struct Extent {
  int64_t length;
  int tiles;
};
template <int R, bool CAUSAL, bool FINE>
__device__ __forceinline__ Extent extent(const LineArgs& a, const Part& part, int lane, Seq& window) {
  const int n_seq = part.stacked ? 1 : a.c.cache.n_seqs;
  window = load_window<R, CAUSAL, FINE>(a, part, 0, lane);
  int64_t sum = window.total();
  int tiles = window.tiles;
  for (int i = 64; i < n_seq; i += 64) {
    const Seq s = load_window<R, CAUSAL, FINE>(a, part, i, lane);
    sum += s.total();
    tiles += s.tiles;
  }
  for (int i = 1; i < n_seq && i < 64; i <<= 1) {
    sum += __shfl_xor(sum, i);
    tiles += __shfl_xor(tiles, i);
  }
  return {uniform64(sum), uniform(tiles)};
}

// A workgroup's share: positions [at, end) of the line
struct Share {
  int id;
  int64_t at, end;
  int64_t length, longer;    // of a share; the first `longer` shares have one more
  // the share that has position x of the line
  __device__ __forceinline__ int of(int64_t x) const {
    const int64_t split = longer * (length + 1);
    return (int)(x < split ? quotient(x, length + 1) : longer + quotient(x - split, length));
  }
};
__device__ __forceinline__ bool find_share(const LineArgs& a, int64_t total, Share& s) {
  if (total == 0) return false;
  const int shares = (int)std::clamp<int64_t>(quotient(total, a.min_length), 1, gridDim.x);
  // workgroups go to the 8 XCDs in turn: shares next to each other, which read the same keys, go to one of them
  const int per_xcd = (shares + 7) / 8;
  s.id = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per_xcd || s.id >= shares) return false;
  s.length = quotient(total, shares);
  s.longer = total - s.length * shares;
  s.at = s.id * s.length + std::min<int64_t>(s.id, s.longer);
  s.end = s.at + s.length + (s.id < s.longer ? 1 : 0);
  return true;
}
// (A cut that falls in a tile's front is one in front of the tile: see cut_piece().)

// Where a walk along a part is
struct Place {
  int h, b, tile;
  int tile_id;      // of (h, b, tile) in the part
  int at;           // position in the tile
  int base;         // first sequence of the window
};
// x: position in the part
template <int R, bool CAUSAL, bool FINE>
__device__ __forceinline__ bool find_place(const LineArgs& a, const Part& part, const Extent& ex, int64_t x, int lane, Place& p, Seq& window) {
  const int n_seq = part.stacked ? 1 : a.c.cache.n_seqs;
  const int lanes = n_seq < 64 ? n_seq : 64;
  p.h = (int)quotient(x, ex.length);
  int64_t rest = x - p.h * ex.length;
  int before = 0;
  for (p.base = 0;; p.base += 64) {
    if (p.base > 0 || n_seq > 64) window = load_window<R, CAUSAL, FINE>(a, part, p.base, lane);
    int64_t scan = window.total();
    int tscan = window.tiles;
    for (int d = 1; d < lanes; d <<= 1) {
      const int64_t v = __shfl_up(scan, d);
      const int tv = __shfl_up(tscan, d);
      scan += lane >= d ? v : 0;
      tscan += lane >= d ? tv : 0;
    }
    const uint64_t in = __ballot(lane < lanes && rest < scan);
    if (in == 0) {
      if (p.base + 64 >= n_seq) return false;
      rest -= uniform64(__shfl(scan, 63));
      before += uniform(__shfl(tscan, 63));
      continue;
    }
    const int l = __builtin_ctzll(in);
    const Seq s = of_lane<R, CAUSAL, FINE>(a, part, window, l);
    rest -= uniform64(__shfl(scan, l)) - s.total();
    p.b = p.base + l;
    p.tile = s.tile_at(rest);
    p.at = (int)(rest - s.before(p.tile));
    p.tile_id = p.h * ex.tiles + before + uniform(__shfl(tscan, l)) - s.tiles + p.tile;
    return true;
  }
}
// On to the start of the next tile; false behind the last
template <int R, bool CAUSAL, bool FINE>
__device__ __forceinline__ bool next_tile(const LineArgs& a, const Part& part, Place& p, Seq& window, Seq& s, int lane) {
  p.at = 0;
  ++p.tile_id;
  if (++p.tile < s.tiles) return true;
  p.tile = 0;
  do {
    if (++p.b == (part.stacked ? 1 : a.c.cache.n_seqs)) {
      p.b = 0;
      if (++p.h == a.c.cache.H_kv) return false;
    }
    if (p.b < p.base || p.b >= p.base + 64) {
      p.base = p.b;
      window = load_window<R, CAUSAL, FINE>(a, part, p.b, lane);
    }
    s = of_lane<R, CAUSAL, FINE>(a, part, window, p.b - p.base);
  } while (s.tiles == 0);
  return true;
}

// A row of a tile as q and o have it
struct Row {
  int token, head;
};
// r / group by a product with 2^32 / group: exact for what rows there can be, 2^20 tokens of 64 heads (the compiler's division by
// a variable takes 25 instructions)
__device__ __forceinline__ int token_of(const LineArgs& a, int r) {
  return a.c.group == 1 ? r : (int)__umulhi((uint32_t)r, a.group_magic);
}
__device__ __forceinline__ Row row_of(const LineArgs& a, const Place& p, const Seq& s, int r) {
  const int i = token_of(a, r);
  return {s.first + i, p.h * a.c.group + (r - i * a.c.group)};
}
__device__ __forceinline__ const char* q_row(const LineArgs& a, const Row& r) {
  return a.c.q.data + (r.token * a.c.q.token_stride + r.head * a.c.q.head_stride) * 2;
}
// Own keys that row r sees
template <bool CAUSAL>
__device__ __forceinline__ int seen_by(const LineArgs& a, const Seq& s, int r) {
  return CAUSAL ? std::clamp(s.len - s.n + token_of(a, r) + 1, 0, s.len) : s.len;
}

// What a share has of a tile: positions [at, to) of it, units [u0, u1) of keys; nothing if it ends in the tile's front
struct Piece {
  int to, u0, u1;
  bool starts, ends;
};
template <int UNIT, bool FINE>
__device__ __forceinline__ bool cut_piece(Piece& c, const Place& p, const Seq& s, int P, int64_t left, int most) {
  constexpr int F = kTileFront<FINE>;
  const int length = s.length(p.tile), prefix_units = (P + UNIT - 1) / UNIT;
  c.to = (int)std::min<int64_t>(length, p.at + left);
  c.starts = p.at <= F;
  c.ends = c.to == length;
  const int units = prefix_units + (most + UNIT - 1) / UNIT;
  auto unit_at = [&](int x) {
    x -= F;
    return std::min(units, !FINE ? x : x <= P ? (x + UNIT - 1) / UNIT : prefix_units + (x - P + UNIT - 1) / UNIT);
  };
  c.u0 = c.starts ? 0 : unit_at(p.at);
  c.u1 = c.ends ? units : unit_at(c.to);
  return c.ends || c.to > F;
}

// Where a piece goes: to o, or to a slot
struct Target {
  bool finish;
  int slot;
};
// The piece that starts a tile says where the others are; `first`: the share's first one, `tile`: where the tile starts on the line.
// By all threads.
template <int R>
__device__ __forceinline__ Target place_piece(const LineArgs& a, const Part& part, const Share& share, const Place& p, const Seq& s,
                                              const Piece& c, bool first, int64_t tile) {
  Target t = {a.finish && c.starts && c.ends, 0};
  if (!t.finish) t.slot = a.finish ? 2 * share.id + (first ? 0 : 1) : share.id + p.tile_id;
  if (c.starts) {
    const int r0 = p.tile * R, n_rows = s.n * a.c.group;
    RowPieces rp = {0, 0, 0, 0};
    if (!t.finish) {
      rp.n = share.of(tile + s.length(p.tile) - 1) - share.id + 1;
      rp.first = t.slot * R;
      rp.base = (a.finish ? 2 * share.id : t.slot) * R;
      rp.stride = a.finish ? 2 * R : R;
    }
    for (int i = threadIdx.x; i < R; i += 256)
      if (r0 + i < n_rows) {
        const Row r = row_of(a, p, s, r0 + i);
        part.rows[(int64_t)r.token * a.H_q + r.head] = {rp.first + i, rp.base + i, rp.stride, rp.n};
      }
  }
  return t;
}
// The logarithm of a row's sum of l 2^m; of none, minus infinity
__device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}
// Four channels of row r of the tile; l: the row's sum
template <int R>
__device__ __forceinline__ void put(const LineArgs& a, const Part& part, const Place& p, const Seq& s, const Target& t, int r, int channel,
                                    const f32x4& o, float l) {
  if (p.tile * R + r >= s.n * a.c.group) return;
  if (t.finish) {
    const float f = l == 0.f ? 0.f : 1.f / l;
    const Row row = row_of(a, p, s, p.tile * R + r);
    *(u32x2*)((char*)a.c.o + (((int64_t)row.token * a.H_q + row.head) * kDHead + channel) * 2) =
        u32x2{pack_bf16x2(o[0] * f, o[1] * f), pack_bf16x2(o[2] * f, o[3] * f)};
  } else if ((uint32_t)t.slot < (uint32_t)part.max_slots) {
    *(f32x4*)(part.slot_o + ((int64_t)t.slot * R + r) * kDHead + channel) = o;
  }
}
template <int R, bool LSE>
__device__ __forceinline__ void put_sums(const LineArgs& a, const Part& part, const Place& p, const Seq& s, const Target& t, int r, float m,
                                         float l) {
  if constexpr (LSE)
    if (t.finish && a.c.lse && p.tile * R + r < s.n * a.c.group) {
      const Row row = row_of(a, p, s, p.tile * R + r);
      a.c.lse[(int64_t)row.token * a.H_q + row.head] = log_sum(m, l);
    }
  if (!t.finish && (uint32_t)t.slot < (uint32_t)part.max_slots && p.tile * R + r < s.n * a.c.group) part.slot_ml[(int64_t)t.slot * R + r] = float2{m, l};
}

// V^T operands: 16 channels x 32 keys in the order of the weights (see the top)
__device__ __forceinline__ void load_v_operands(bf16x8 (&av)[4], const bf16_t* sv, int l16, int grp) {
  const int krow = 4 * grp + (l16 >> 2);
  const int sw = v_swizzle(krow);
#pragma unroll
  for (int ct = 0; ct < 4; ++ct) {
    const bf16_t* at = sv + krow * kDHead + ((2 * ct + ((l16 & 3) >> 1)) ^ sw) * 8 + 4 * (l16 & 1);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 16 * kDHead));
    av[ct] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
}

template <int NQ>
struct WaveState {
  bf16x8 qf[NQ][2];     // Q^T, 32 channels each
  f32x4 o[4][NQ];       // O^T, 16 channels each
  float m[NQ], l[NQ];   // shift in log2 units, sum over the lane's keys
};

// One unit of keys on its way to a wave.  Next to a cache in 4 bits a lane has 16 channels in a piece, of K and of V, of one row of
// either half of 16: 16 * grp + 0..7 and + 8..15.  (Which 32 channels an operand of K Q^T has does not matter, as long as Q is taken alike.)
struct UnitData {
  u32x4 k[4];       // [key half * 2 + channel half]: the A operands
  u32x4 v[4];       // 8 rows each; with 4 bits as k
};
// A unit of keys in 4 bits: the codes of 16 channels of K and of V of a row of either half, and the block's two exponents
struct MxUnit {
  u32x2 k[2], v[2];
  uint32_t exponents[2];
};
__device__ __forceinline__ void expand(UnitData& d, const MxUnit& x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float ku = mx4_key_unit(x.exponents[i]), vu = mx4_value_unit(x.exponents[i]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      d.k[2 * i + e] = mx4_values(x.k[i][e], ku);
      d.v[2 * i + e] = mx4_values(x.v[i][e], vu);
    }
  }
}

// Rows of K or V: 16 from `at` on, of which the first `n` are there; the others are read as zeros, wherever they would be
__device__ __forceinline__ __amdgpu_buffer_rsrc_t half_rows(const char* at, int n) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)at, 0, n * kRowBytes, kRawBufferWord3);
}
// The same of `row_bytes` each, where the compiler does not see that all lanes ask for the same rows: it would load for one lane after the other
// and wait for each
__device__ __forceinline__ __amdgpu_buffer_rsrc_t uniform_rows(const char* at, int n, int row_bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)uniform64((int64_t)at), 0, uniform(n * row_bytes), kRawBufferWord3);
}
__device__ __forceinline__ u32x4 load_row(__amdgpu_buffer_rsrc_t rows, int offset) {
  return __builtin_amdgcn_raw_buffer_load_b128(rows, offset, 0, 0);
}

// Whether some value of a lane's V rows is an infinity or NaN
__device__ __forceinline__ bool not_finite(const u32x4 (&v)[4]) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) bad |= (v[i][e] & 0x7F80u) == 0x7F80u || (v[i][e] & 0x7F800000u) == 0x7F800000u;
  return bad;
}
// Weights times V where a row must not see a key whose V is not finite: 0 * inf would reach it.  Key by key, each
// added where it is seen.
template <int NQ>
__device__ __forceinline__ void add_seen(f32x4 (&o)[4][NQ], const bf16x8 (&av)[4], const bf16x8 (&p)[NQ], const int (&limit)[NQ], int row0,
                                         int lane) {
  const int grp = lane >> 4;
#pragma unroll 1
  for (int j = 0; j < kUnit; ++j) {
    const int e = (j & 3) + (j >> 4) * 4;
    const bool here = grp == ((j & 15) >> 2);
    u32x4 keep;
#pragma unroll
    for (int w = 0; w < 4; ++w) keep[w] = here && w == (e >> 1) ? ((e & 1) ? 0xFFFF0000u : 0xFFFFu) : 0u;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
      const bf16x8 one = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, av[ct]) & keep);
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
        const f32x4 d = mfma16(one, p[qt], f32x4{0.f, 0.f, 0.f, 0.f});
        o[ct][qt] += row0 + j < limit[qt] ? d : f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
  }
}

// Scores, statistics and product of a unit.  row0: its first key; end: keys from there on are masked in all rows (causal
// own keys: in some); ok: bit per half of 16 keys, whether it has a page; limit_of(qt): own keys that the lane's row sees.
template <int NQ, bool CAUSAL, int KIND, typename Limit>
__device__ __forceinline__ void unit_step(WaveState<NQ>& w, const UnitData& d, bf16_t* sv, float c, int row0, int end, int ok, bool own,
                                          int lane, Limit limit_of) {
  constexpr bool MX4 = KIND == MX4_ROWS || KIND == MX4_ALONE;
  const int l16 = lane & 15, grp = lane >> 4;
  const bool masked = ok != 3 || row0 + kUnit > end;
  const bool wild = CAUSAL && masked && own && __ballot(not_finite(d.v)) != 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = MX4 ? 16 * (i >> 1) + l16 : 8 * i + (lane >> 3), chunk = MX4 ? 2 * grp + (i & 1) : lane & 7;
    *(u32x4*)(sv + r * kDHead + (chunk ^ v_swizzle(r)) * 8) = d.v[i];
  }
  f32x4 s[2][NQ];
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      s[kt][qt] = mfma16(__builtin_bit_cast(bf16x8, d.k[kt * 2]), w.qf[qt][0], f32x4{0.f, 0.f, 0.f, 0.f});
      s[kt][qt] = mfma16(__builtin_bit_cast(bf16x8, d.k[kt * 2 + 1]), w.qf[qt][1], s[kt][qt]);
    }
  if (masked) {
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      const int limit = (CAUSAL && own ? limit_of(qt) : end) - row0 - 4 * grp;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (16 * kt + r >= limit || !((ok >> kt) & 1)) s[kt][qt][r] = -__builtin_inff();
    }
  }
  float top[NQ];
  bool above = false;
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    top[qt] = max8(s[0][qt], s[1][qt]);
    above = above || fmaf(top[qt], c, -w.m[qt]) > kSlack;
  }
  if (__ballot(above)) {
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      const float m = fmaxf(w.m[qt], groups_max(top[qt]) * c);
      const float f = __builtin_amdgcn_exp2f(w.m[qt] - m);
      w.m[qt] = m;
      w.l[qt] *= f;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) w.o[ct][qt] *= f;
    }
  }
  bf16x8 p[NQ];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    float x[8], sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][qt][e & 3], c, -w.m[qt]));
      sum += x[e];
    }
    w.l[qt] += sum;
    p[qt] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])});
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  bf16x8 av[4];
  load_v_operands(av, sv, l16, grp);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (CAUSAL && __builtin_expect(wild, 0)) {
    int limit[NQ];
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) limit[qt] = limit_of(qt);
    add_seen<NQ>(w.o, av, p, limit, row0, lane);
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) av[ct] = bf16x8{};
  }
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) w.o[ct][qt] = mfma16(av[ct], p[qt], w.o[ct][qt]);
}

// A share's way along a part of the line: four waves take the units of a piece in turn.  [x, end): positions in the part, `line`:
// where it starts on the line.
constexpr int kWaves = 4;
template <int NQ, bool CAUSAL, int KIND>
__device__ __forceinline__ void walk(const LineArgs& a, const Part& part, const Share& share, const Extent& ex, int64_t line, int64_t x,
                                     int64_t end, Seq window, char* s_mem, float2* s_ml) {
  constexpr bool MX4 = KIND == MX4_ROWS || KIND == MX4_ALONE;
  constexpr int R = 16 * NQ, KS = kWaves;
  constexpr int DEPTH = 1;     // units of a wave on their way besides the one in work
  const CachedAttnArgs& c = a.c;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int l16 = lane & 15, grp = lane >> 4;
  bf16_t* sv = (bf16_t*)(s_mem + wave * kUnitBytes);
  Place p;
  if (!find_place<R, CAUSAL, false>(a, part, ex, x, lane, p, window)) return;
  Seq s = of_lane<R, CAUSAL, false>(a, part, window, p.b - p.base);
  const int P = KIND != MX4_ALONE && part.with_prefix ? (int)c.P : 0, prefix_units = (P + kUnit - 1) / kUnit;
  const int k_offset = l16 * kRowBytes + grp * (MX4 ? 32 : 16), v_offset = MX4 ? k_offset : lane * 16;
  bool first = true;

  while (true) {
    const int n_rows = s.n * c.group, r0 = p.tile * R;
    const int least = uniform(seen_by<CAUSAL>(a, s, r0)), most = uniform(seen_by<CAUSAL>(a, s, std::min(r0 + R, n_rows) - 1));
    Piece piece;
    if (!cut_piece<kUnit, false>(piece, p, s, P, end - x, most)) return;
    const int stop = piece.u1;
    // (constant memory: scalar loads, which are waited for apart from those of the keys)
    const auto* table = (const __attribute__((address_space(4))) int32_t*)(c.cache.table + (int64_t)p.b * c.cache.table_stride);

    // Pages of a unit's two halves, asked for well before its rows; a prefix needs none
    struct Pages {
      int page[2];
    };
    auto look_up = [&](int unit) {
      Pages g = {{0, 0}};
      if (unit >= prefix_units) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int index = ((unit - prefix_units) * kUnit + 16 * i) >> c.cache.page_shift;
          g.page[i] = index < c.cache.table_stride ? table[index] : -1;
        }
      }
      return g;
    };
    // Requests a unit's rows; returns its ok bits
    auto fetch = [&](int unit, const Pages& g, UnitData& d) {
      int ok = 3;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const char *k, *v;
        int n;
        if (unit < prefix_units) {
          const int row = unit * kUnit + 16 * i;
          const int64_t at = (p.h * c.P + row) * kRowBytes;
          k = c.k_prefix + at;
          v = c.v_prefix + at;
          n = (int)c.P - row;
        } else {
          const int row = (unit - prefix_units) * kUnit + 16 * i;
          const bool there = g.page[i] >= 0 && g.page[i] < c.cache.n_pages;
          const int64_t page = there ? g.page[i] : 0;
          const int64_t at = (((page * c.cache.H_kv + p.h) << c.cache.page_shift) + (row & ((1 << c.cache.page_shift) - 1))) * kRowBytes;
          k = c.cache.k_pages + at;
          v = c.cache.v_pages + at;
          n = there ? s.len - row : 0;
          ok &= there ? 3 : ~(1 << i);
        }
        n = std::clamp(n, 0, 16);
        const __amdgpu_buffer_rsrc_t kr = MX4 ? uniform_rows(k, n, kRowBytes) : half_rows(k, n), vr = MX4 ? uniform_rows(v, n, kRowBytes) : half_rows(v, n);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) d.k[2 * i + ks] = load_row(kr, k_offset + ks * (MX4 ? 16 : 64));
#pragma unroll
        for (int e = 0; e < 2; ++e) d.v[2 * i + e] = load_row(vr, v_offset + e * (MX4 ? 16 : 1024));
      }
      return ok;
    };

    WaveState<NQ> w;
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      const int r = std::min(r0 + 16 * qt + l16, n_rows - 1);
      const char* q = q_row(a, row_of(a, p, s, r));
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) w.qf[qt][ks] = *(const bf16x8*)(q + (MX4 ? 2 * grp + ks : ks * 4 + grp) * 16);
      w.m[qt] = kLowest;
      w.l[qt] = 0.f;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) w.o[ct][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    auto limit_of = [&](int qt) { return seen_by<CAUSAL>(a, s, std::min(r0 + 16 * qt + l16, n_rows - 1)); };
    // DEPTH units are on their way, the pages of the next one are asked for.  (The data moves through registers: two copies
    // of the step in the loop need more scalar registers than there are.)
    int unit = piece.u0 + wave;
    const int stop_rows = MX4 ? std::min(stop, prefix_units) : stop;      // of the units in 16 bits
    UnitData d[DEPTH + 1];
    int ok[DEPTH + 1];
    Pages g = look_up(unit);
    if constexpr (KIND != MX4_ALONE) {
#pragma unroll
      for (int i = 0; i < DEPTH; ++i) {
        if (unit + i * KS < stop_rows) ok[i] = fetch(unit + i * KS, g, d[i]);
        g = look_up(unit + (i + 1) * KS);
      }
#pragma unroll 1
      for (; unit < stop_rows; unit += KS) {
        if (unit + DEPTH * KS < stop_rows) ok[DEPTH] = fetch(unit + DEPTH * KS, g, d[DEPTH]);
        g = look_up(unit + (DEPTH + 1) * KS);
        const bool own = unit >= prefix_units;
        unit_step<NQ, CAUSAL, KIND>(w, d[0], sv, c.scale_log2, (own ? unit - prefix_units : unit) * kUnit, own ? least : P, ok[0], own, lane, limit_of);
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
          d[i] = d[i + 1];
          ok[i] = ok[i + 1];
        }
      }
    }
    if constexpr (MX4) {
      // Own keys in 4 bits: a unit's codes are turned into values, and those of a later one requested in their place.  (64 streams: 104 us with one unit ahead
      // and loads that wait for each other, 86 with three.  Next to a prefix's loop there are no registers for more than one.)
      constexpr int AHEAD = KIND == MX4_ALONE && NQ == 1 ? 3 : 1;
      MxUnit raw[AHEAD];
      int ok_raw[AHEAD];
      auto request = [&](int u, const Pages& p2, MxUnit& r, int& ok) {
        const int row = (u - prefix_units) * kUnit;
        ok = 3;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bool there = p2.page[i] >= 0 && p2.page[i] < c.cache.n_pages;
          const int64_t page = there ? p2.page[i] : 0;
          const int64_t at = ((page * c.cache.H_kv + p.h) << c.cache.page_shift) + ((row + 16 * i) & ((1 << c.cache.page_shift) - 1));
          const int n = there ? std::clamp(s.len - row - 16 * i, 0, 16) : 0;
          ok &= there ? 3 : ~(1 << i);
          const int in = l16 * kMxRowBytes + grp * 8;
          r.k[i] = __builtin_amdgcn_raw_buffer_load_b64(uniform_rows(c.cache.k_pages + at * kMxRowBytes, n, kMxRowBytes), in, 0, 0);
          r.v[i] = __builtin_amdgcn_raw_buffer_load_b64(uniform_rows(c.cache.v_pages + at * kMxRowBytes, n, kMxRowBytes), in, 0, 0);
          r.exponents[i] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(
              uniform_rows((const char*)c.scales + at * kMxScaleBytes, n, kMxScaleBytes), l16 * kMxScaleBytes + 2 * (grp >> 1), 0, 0);
        }
      };
      if constexpr (KIND != MX4_ALONE) g = look_up(unit);
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (unit + i * KS < stop) request(unit + i * KS, g, raw[i], ok_raw[i]);
        g = look_up(unit + (i + 1) * KS);
      }
#pragma unroll 1
      while (unit < stop) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          if (unit >= stop) break;
          UnitData now;
          expand(now, raw[i]);
          const int ok_now = ok_raw[i];
          if (unit + AHEAD * KS < stop) request(unit + AHEAD * KS, g, raw[i], ok_raw[i]);
          g = look_up(unit + (AHEAD + 1) * KS);
          unit_step<NQ, CAUSAL, KIND>(w, now, sv, c.scale_log2, (unit - prefix_units) * kUnit, least, ok_now, true, lane, limit_of);
          unit += KS;
        }
      }
    }

    // ---- the piece's end ---------------------------------------------------------------------------------
    const Target to = place_piece<R>(a, part, share, p, s, piece, first, line + x - p.at);
    // The waves meet, 16 rows at a time: each leaves its sums and products where its V rows were (chunk c of row r at c ^ r, which
    // spreads the rows over the banks), and 16 lanes join a row's.
    f32x4* so = (f32x4*)s_mem;      // [KS][16][16 chunks]
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      if (qt) __syncthreads();
      const float l = groups_sum(w.l[qt]);
      if (grp == 0) s_ml[wave * 16 + l16] = float2{w.m[qt], l};
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) so[(wave * 16 + l16) * 16 + ((4 * ct + grp) ^ l16)] = w.o[ct][qt];
      __syncthreads();
      const int row = threadIdx.x >> 4, chunk = threadIdx.x & 15;
      float2 ml[KS];
      float top = kLowest, sum = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        ml[k] = s_ml[k * 16 + row];
        top = fmaxf(top, ml[k].x);
      }
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const float f = __builtin_amdgcn_exp2f(ml[k].x - top);
        sum += ml[k].y * f;
        o += so[(k * 16 + row) * 16 + (chunk ^ row)] * f;
      }
      if (chunk == 0) put_sums<R, KIND != ROWS>(a, part, p, s, to, 16 * qt + row, top, sum);
      put<R>(a, part, p, s, to, 16 * qt + row, 4 * chunk, o, sum);
    }
    __syncthreads();

    x += piece.to - p.at;
    if (x >= end || !next_tile<R, CAUSAL, false>(a, part, p, window, s, lane)) return;
    first = false;
  }
}

// NA query tiles of 16 rows for the first part of the line, the prefix against all sequences' rows, or 0: there is none;
// NB for the second.
constexpr int waves_per_simd(int nq) { return nq == 1 ? 3 : 2; }
template <int NA, int NB, bool CAUSAL, int KIND>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(waves_per_simd(NA > NB ? NA : NB), waves_per_simd(NA > NB ? NA : NB)))) void
attention_cached_kernel(const LineArgs a) {
  __shared__ __attribute__((aligned(16))) char s_mem[kWaves * kUnitBytes];
  __shared__ float2 s_ml[kWaves * 16];
  const int lane = threadIdx.x & 63;
  Seq window_a = {}, window_b;
  Extent ea = {0, 0};
  if constexpr (NA > 0) ea = extent<16 * NA, false, false>(a, a.part[0], lane, window_a);
  const Extent eb = extent<16 * NB, CAUSAL, false>(a, a.part[1], lane, window_b);
  const int64_t total_a = ea.length * a.c.cache.H_kv, total_b = eb.length * a.c.cache.H_kv;
  Share share;
  if (!find_share(a, total_a + total_b, share)) return;
  if constexpr (NA > 0)
    if (share.at < total_a) {
      walk<NA, false, ROWS>(a, a.part[0], share, ea, 0, share.at, std::min(share.end, total_a), window_a, s_mem, s_ml);
    }
  if (share.end > total_a)
    walk<NB, CAUSAL, KIND>(a, a.part[1], share, eb, total_a, std::max(share.at, total_a) - total_a, share.end - total_a, window_b, s_mem, s_ml);
}

// ---- many rows -------------------------------------------------------------------------------------------------
//
// Tiles of 256 rows, 64 for each of four waves, which share the keys: units of 64 go through registers into LDS, two of
// them there at a time.  Bound by the matrix cores and, close behind, by the vector instructions of the softmax, so a wave's
// step of 32 keys has the products of the step before and of the step behind in one block with the weights of its
// own, which depend on neither: the order of issue mixes them.  (V therefore runs a unit behind K.)  Whether a shift has to
// follow is looked at before the block, on scores that the step before has left.

enum { MIXED_UNITS, PREFIX_UNITS, OWN_UNITS };
constexpr int kWideUnit = 64;
constexpr int kWideWaves = 4;
constexpr int kWideQ = 4;
constexpr int kWideRows = 16 * kWideQ * kWideWaves;

// The state of a wave of 64 rows
struct WideState {
  bf16x8 qf[kWideQ][2];     // Q^T, 32 channels each
  f32x4 o[4][kWideQ];       // O^T, 16 channels each
  f32x4 cur[2][kWideQ];     // scores of the step in work
  bf16x8 p[kWideQ];         // weights of the step before
  float l[kWideQ];          // sums over the lane's keys
  float m[kWideQ];          // minus the shift, in log2 units
};
// The shift follows the scores of the step in work, and all that is relative to it.  It is a whole number (of log2 units), so that the factor is a
// power of two and the weights that wait for their product, up to 2^kSlack, keep the rounding they have.
__device__ __forceinline__ void raise_shift(WideState& w, const float (&top)[kWideQ], float c) {
#pragma unroll
  for (int qt = 0; qt < kWideQ; ++qt) {
    const float m = fminf(w.m[qt], floorf(-(groups_max(top[qt]) * c)));
    // (2^-1024 is 0: the first shift comes from kLowest)
    const float f = ldexpf(1.f, (int)fmaxf(m - w.m[qt], -1024.f));
    w.m[qt] = m;
    w.l[qt] *= f;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) w.o[ct][qt] *= f;
    u32x4 x = __builtin_bit_cast(u32x4, w.p[qt]);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = pack_bf16x2(bf16_lo(x[e]) * f, bf16_hi(x[e]) * f);
    w.p[qt] = __builtin_bit_cast(bf16x8, x);
  }
}

template <bool CAUSAL, int KIND>
__global__ __launch_bounds__(64 * kWideWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void attention_cached_wide_kernel(const LineArgs a) {
  constexpr bool MX4 = KIND == MX4_ROWS || KIND == MX4_ALONE;
  constexpr int NQ = kWideQ, R = kWideRows, UNIT = kWideUnit;
  // K of two units, V of two.  All that reads or writes them goes by offsets that change sides once a unit.
  constexpr int kSide = UNIT * kRowBytes, kHalf = kSide / 2;
  __shared__ __attribute__((aligned(4 * kSide))) char s_mem[4 * kSide];
  const CachedAttnArgs& c = a.c;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int l16 = lane & 15, grp = lane >> 4;
  const Part& part = a.part[0];
  Seq window;
  const Extent ex = extent<R, CAUSAL, true>(a, part, lane, window);
  Share share;
  if (!find_share(a, ex.length * c.cache.H_kv, share)) return;
  Place p;
  if (!find_place<R, CAUSAL, true>(a, part, ex, share.at, lane, p, window)) return;
  Seq s = of_lane<R, CAUSAL, true>(a, part, window, p.b - p.base);
  const int P = KIND != MX4_ALONE && part.with_prefix ? (int)c.P : 0, prefix_units = (P + UNIT - 1) / UNIT;
  int64_t x = share.at;
  bool first = true;
  // lanes' offsets: K operands (channel halves), V operands (channel quarters), the rows that a wave brings (K, V)
  int k_at[2], v_at[4], to_k, to_v;
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) k_at[ks] = l16 * kRowBytes + ((ks * 4 + grp) ^ k_swizzle(l16)) * 16;
  {
    const int row = 4 * grp + (l16 >> 2);
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) v_at[ct] = 2 * kSide + row * kRowBytes + ((2 * ct + ((l16 & 3) >> 1)) ^ v_swizzle(row)) * 16 + 8 * (l16 & 1);
    // and the row 8 further, whose place among the chunks is the same one; with 4 bits the chunk beside it (of 16 channels in a lane)
    const int in = 16 * wave + (MX4 ? lane >> 2 : lane >> 3), chunk = MX4 ? 2 * (lane & 3) : lane & 7;
    to_k = in * kRowBytes + (chunk ^ k_swizzle(in)) * 16;
    to_v = 2 * kSide + in * kRowBytes + (chunk ^ v_swizzle(in)) * 16;
  }
  auto change_sides = [&] {
#pragma unroll
    for (int i = 0; i < 2; ++i) k_at[i] ^= kSide;
#pragma unroll
    for (int i = 0; i < 4; ++i) v_at[i] ^= kSide;
    to_k ^= kSide;
    to_v ^= kSide;
  };
  auto barrier = [] {      // LDS only: rows on their way from memory stay so
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  while (true) {
    const int n_rows = s.n * c.group, r0 = p.tile * R, wr0 = r0 + wave * 16 * NQ;
    const auto* table = (const __attribute__((address_space(4))) int32_t*)(c.cache.table + (int64_t)p.b * c.cache.table_stride);
    const bool active = uniform(wr0 < n_rows) != 0;
    const int least = uniform(seen_by<CAUSAL>(a, s, std::min(wr0, n_rows - 1)));
    const int most = uniform(seen_by<CAUSAL>(a, s, std::min(r0 + R, n_rows) - 1));
    Piece piece;
    if (!cut_piece<UNIT, true>(piece, p, s, P, share.end - x, most)) return;
    const int u0 = piece.u0, stop = piece.u1;

    WideState w;
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      const char* q = q_row(a, row_of(a, p, s, std::min(wr0 + 16 * qt + l16, n_rows - 1)));
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) w.qf[qt][ks] = *(const bf16x8*)(q + (ks * 4 + grp) * 16);
      w.m[qt] = -kLowest;
      w.l[qt] = 0.f;
      w.p[qt] = bf16x8{};
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) w.o[ct][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    auto page_of = [&](int unit, int quarter) {
      const int index = ((unit - prefix_units) * UNIT + 16 * quarter) >> c.cache.page_shift;
      return index < c.cache.table_stride ? table[index] : -1;
    };
    auto there = [&](int page) { return page >= 0 && page < (int)c.cache.n_pages; };
    auto load_k = [&](bf16x8 (&ak)[4], int half) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) ak[kt * 2 + ks] = *(const bf16x8*)(s_mem + k_at[ks] + half + kt * 16 * kRowBytes);
    };
    auto score = [&](const bf16x8 (&ak)[4], int qt) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) w.cur[kt][qt] = mfma16(ak[kt * 2], w.qf[qt][0], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) w.cur[kt][qt] = mfma16(ak[kt * 2 + 1], w.qf[qt][1], w.cur[kt][qt]);
    };
    const bf16x2 ones = __builtin_bit_cast(bf16x2, local(0x3F803F80u));   // (a literal is not taken as two bf16 halves)
    auto limit_of = [&](int qt) { return seen_by<CAUSAL>(a, s, std::min(wr0 + 16 * qt + l16, n_rows - 1)); };
    // V operands for the weights of the step before.  Where a row must not see one of its keys, whose V is not finite: key by
    // key, and zeros are left
    int old_row0 = -1;      // the first key of the step before, if some rows do not see all of it
    auto load_v = [&](bf16x8 (&av)[4], int half) {
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) {
        const char* at = s_mem + v_at[ct] + half;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 16 * kRowBytes));
        av[ct] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
      if (CAUSAL && __builtin_expect(old_row0 >= 0, 0)) {
        bool bad = false;
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t x = __builtin_bit_cast(u32x4, av[ct])[e];
            bad |= (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
          }
        if (__ballot(bad)) {
          int limit[NQ];
#pragma unroll
          for (int qt = 0; qt < NQ; ++qt) limit[qt] = limit_of(qt);
          add_seen<NQ>(w.o, av, w.p, limit, old_row0, lane);
#pragma unroll
          for (int ct = 0; ct < 4; ++ct) av[ct] = bf16x8{};
        }
      }
    };
    // A step of 32 keys from row0 on.  half: where the K rows of the step behind it and the V rows of the step before are in their
    // sides; end, ok, own as in unit_step()
    auto step = [&](int half, int row0, int end, uint32_t ok, bool own) __attribute__((always_inline)) {
      bf16x8 ak[4], av[4];
      load_v(av, half);
      const bool partial = row0 + 32 > end;
      if (__builtin_expect(partial || ok != 3, 0)) {
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) {
          const int limit = (CAUSAL && own ? limit_of(qt) : end) - row0 - 4 * grp;
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (16 * kt + r >= limit || !((ok >> kt) & 1)) w.cur[kt][qt][r] = -__builtin_inff();
        }
      }
      if (CAUSAL) old_row0 = partial && own ? row0 : -1;
      float top[NQ], over[NQ];
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
        top[qt] = max8(w.cur[0][qt], w.cur[1][qt]);
        over[qt] = fmaf(top[qt], c.scale_log2, w.m[qt]);
      }
      // (not "above": a row whose scores are no numbers makes the maximum none, and must not hide the lane's three others)
      if (__ballot(!(max8(f32x4{over[0], over[1], over[2], over[3]}, f32x4{over[0], over[0], over[0], over[0]}) <= kSlack))) raise_shift(w, top, c.scale_log2);
      load_k(ak, half);
      __builtin_amdgcn_sched_barrier(0);
      // (a wave inside this block goes first: the other one of its SIMD fills what it leaves.  16 heads x 8192 tokens x 16384 keys 620 -> 578 us)
      __builtin_amdgcn_s_setprio(1);
      // query tile qt: its weights next to its product with V and the scores of the tile before
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) w.o[ct][qt] = mfma16(av[ct], w.p[qt], w.o[ct][qt]);
        u32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x4& y = w.cur[e >> 1][qt];
          const float x0 = __builtin_amdgcn_exp2f(fmaf(y[2 * (e & 1)], c.scale_log2, w.m[qt]));
          const float x1 = __builtin_amdgcn_exp2f(fmaf(y[2 * (e & 1) + 1], c.scale_log2, w.m[qt]));
          uint32_t pair = pack_bf16x2(x0, x1);
          asm("" : "+v"(pair));     // (else the compiler takes the same element of x for all four sums: seen in its assembly)
          x[e] = pair;
          w.l[qt] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), ones, w.l[qt], false);
        }
        if (qt > 0) score(ak, qt - 1);
        // order of issue: a product, then an exp2 or two, then others
        if (qt > 0) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        w.p[qt] = __builtin_bit_cast(bf16x8, x);
      }
      score(ak, NQ - 1);
      __builtin_amdgcn_s_setprio(0);
    };

    // The units [u0, stop) of a piece.  OWN: all of them prefix or all own keys, known to the compiler (rows in 4 bits: one loop for each of the two, without a
    // choice between two kinds of loads in it: 662 -> 574 us, 4 x 1374 rows to 5516 shared keys in 16 bits and up to 27480 own ones in 4, 16 heads), or by the unit
    bool holes = false;
    auto run_units = [&](auto own_units, const int u0, const int stop) __attribute__((always_inline)) {
      constexpr int OWN = decltype(own_units)::value;
      auto is_own = [&](int unit) { return OWN == OWN_UNITS || (OWN == MIXED_UNITS && unit >= prefix_units); };
      // A wave brings the unit's rows 16 * wave .. + 15, of K and, a unit later, of V
      struct RowsAt {
        int64_t offset;     // from k_prefix or k_pages, and from v_prefix or v_pages, in bytes; of rows in 4 bits in rows
        int n;
        bool own;
      };
      auto rows_at = [&](int unit) {
        RowsAt r = {0, 0, is_own(unit)};
        const int row = (r.own ? unit - prefix_units : unit) * UNIT + 16 * wave;
        if (unit >= stop) {
        } else if (!r.own) {
          r.offset = (p.h * c.P + row) * kRowBytes;
          r.n = std::clamp((int)c.P - row, 0, 16);
        } else {
          const int page = page_of(unit, wave);
          r.n = there(page) ? std::clamp(s.len - row, 0, 16) : 0;
          r.offset = ((((int64_t)(r.n ? page : 0) * c.cache.H_kv + p.h) << c.cache.page_shift) + (row & ((1 << c.cache.page_shift) - 1))) *
                     (MX4 ? 1 : kRowBytes);
        }
        return r;
      };
      u32x4 in_k[2], in_v[2];
      bool k_own = false, v_own = false;      // what they hold is codes (MX4): two words, and in the second of them an exponent as a unit
      auto request = [&](u32x4 (&in)[2], const RowsAt& r, const char* prefix, const char* pages, int exponent) {
        if (MX4 && r.own) {
          const u32x2 codes = __builtin_amdgcn_raw_buffer_load_b64(uniform_rows(pages + r.offset * kMxRowBytes, r.n, kMxRowBytes), lane * 8, 0, 0);
          in[0][0] = codes[0];
          in[0][1] = codes[1];
          in[1][0] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(uniform_rows((const char*)c.scales + r.offset * kMxScaleBytes, r.n, kMxScaleBytes),
                                                                  (lane >> 2) * kMxScaleBytes + (lane & 2) + exponent, 0, 0);
          return;
        }
        const char* at = (r.own ? pages : prefix) + r.offset;
        const __amdgpu_buffer_rsrc_t rows = MX4 ? uniform_rows(at, r.n, kRowBytes) : half_rows(at, r.n);
#pragma unroll
        for (int i = 0; i < 2; ++i) in[i] = load_row(rows, MX4 ? lane * 32 + i * 16 : lane * 16 + i * 1024);
      };
      auto request_k = [&](u32x4 (&in)[2], const RowsAt& r) { request(in, r, c.k_prefix, c.cache.k_pages, 0); };
      auto request_v = [&](u32x4 (&in)[2], const RowsAt& r) { request(in, r, c.v_prefix, c.cache.v_pages, 1); };
      auto expanded = [&](u32x4 (&in)[2], bool own) {
        if (MX4 && own) {
          const float unit = __uint_as_float(in[1][0] << 23);
          const uint32_t c0 = in[0][0], c1 = in[0][1];
          in[0] = mx4_values(c0, unit);
          in[1] = mx4_values(c1, unit);
        }
      };
      auto store_k = [&](int to, u32x4 (&in)[2], bool own) {
        expanded(in, own);
        *(u32x4*)(s_mem + to) = in[0];
        if constexpr (MX4)
          *(u32x4*)(s_mem + (to ^ 16)) = in[1];
        else
          *(u32x4*)(s_mem + (to ^ 64) + 8 * kRowBytes) = in[1];      // (k_swizzle() of the row 8 further: 4 more)
      };
      auto store_v = [&](int to, u32x4 (&in)[2], bool own) {
        expanded(in, own);
        *(u32x4*)(s_mem + to) = in[0];
        *(u32x4*)(s_mem + (MX4 ? to ^ 16 : to + 8 * kRowBytes)) = in[1];
      };
      // 4 bits for a unit, whether its quarters have pages: looked at only where some entry of the tile's is none
      auto ok_of = [&](int unit) {
        uint32_t ok = 15;
        if (holes && is_own(unit)) {
#pragma unroll
          for (int i = 0; i < 4; ++i) ok &= there(page_of(unit, i)) ? 15u : ~(1u << i);
        }
        return ok;
      };
      // K units u0 and u0 + 1 and V unit u0 are there before the first step; zeros for the V unit in front of it
      RowsAt v_next = rows_at(u0), k_next = rows_at(u0 + 1);
      {
        u32x4 k1[2];
        request_k(in_k, v_next);
        request_v(in_v, v_next);
        request_k(k1, k_next);
        store_k(to_k, in_k, v_next.own);
        store_k(to_k ^ kSide, k1, k_next.own);
        store_v(to_v ^ kSide, in_v, v_next.own);
        *(u32x4*)(s_mem + (v_at[0] & ~(kSide - 1)) + kHalf + threadIdx.x * 16) = u32x4{0, 0, 0, 0};
      }
      v_next = k_next;
      k_next = rows_at(u0 + 2);
      request_k(in_k, k_next);
      request_v(in_v, v_next);
      k_own = k_next.own;
      v_own = v_next.own;
      bool hole = false;
      if (OWN != PREFIX_UNITS)
        for (int i = lane; i < (most + (1 << c.cache.page_shift) - 1) >> c.cache.page_shift; i += 64) hole |= !there(table[i]);
      holes = __ballot(hole) != 0;
      barrier();
      if (active) {
        bf16x8 ak[4];
        load_k(ak, 0);
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) score(ak, qt);
      }
      for (int unit = u0; unit < stop; ++unit) {
        const bool own = is_own(unit);
        const int row0 = (own ? unit - prefix_units : unit) * UNIT, end = own ? least : P;
        const uint32_t ok = ok_of(unit);
        if (active) step(kHalf, row0, end, ok & 3, own);
        barrier();      // K of this unit and V of the one before have been read by everybody
        store_k(to_k, in_k, k_own);
        store_v(to_v, in_v, v_own);
        v_next = k_next;
        k_next = rows_at(unit + 3);
        request_k(in_k, k_next);
        request_v(in_v, v_next);
        k_own = k_next.own;
        v_own = v_next.own;
        change_sides();
        if (active) step(0, row0 + 32, end, ok >> 2, own);
      }
      if (active) {
        bf16x8 av[4];
        load_v(av, kHalf);
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
          for (int ct = 0; ct < 4; ++ct) w.o[ct][qt] = mfma16(av[ct], w.p[qt], w.o[ct][qt]);
      }
    };
    if constexpr (KIND == MX4_ROWS) {
      const int split = std::clamp(prefix_units, u0, std::max(u0, stop));
      if (u0 < split) run_units(std::integral_constant<int, PREFIX_UNITS>(), u0, split);
      if (u0 < split && split < stop) {
        old_row0 = -1;
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) w.p[qt] = bf16x8{};      // (they have been multiplied)
        barrier();      // everybody is done with the buffers
      }
      if (split < stop) run_units(std::integral_constant<int, OWN_UNITS>(), split, stop);
    } else {
      if (u0 < stop) run_units(std::integral_constant<int, KIND == MX4_ALONE ? OWN_UNITS : MIXED_UNITS>(), u0, stop);
    }

    const Target to = place_piece<R>(a, part, share, p, s, piece, first, x - p.at);
    // Out through the LDS, 32 rows of a wave at a time (chunk c of row r at c ^ r % 16): a loop that is 30 instructions long and writes whole
    // rows.  Straight from the registers it is a thousand, each run once and fetched first, and took 3 us a piece.
    barrier();      // everybody is done with the keys
    f32x4* so = (f32x4*)(s_mem + wave * kSide);
#pragma unroll
    for (int pair = 0; pair < NQ / 2; ++pair) {
      float l[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int qt = 2 * pair + i;
        l[i] = groups_sum(w.l[qt]);
        if (grp == 0) put_sums<R, KIND != ROWS>(a, part, p, s, to, wave * 16 * NQ + 16 * qt + l16, -w.m[qt], l[i]);
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) so[(16 * i + l16) * 16 + ((4 * ct + grp) ^ l16)] = w.o[ct][qt];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 2
      for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + grp;      // (16 lanes a row; its sum is in lane r % 16 of either half)
        const float sum = __shfl(i < 4 ? l[0] : l[1], r & 15);
        put<R>(a, part, p, s, to, wave * 16 * NQ + 32 * pair + r, 4 * l16, so[r * 16 + (l16 ^ (r & 15))], sum);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }

    x += piece.to - p.at;
    if (x >= share.end || !next_tile<R, CAUSAL, true>(a, part, p, window, s, lane)) return;
    first = false;
    barrier();      // the buffers are free
  }
}

// ---- joining the pieces --------------------------------------------------------------------------------------

struct PartPieces {
  const RowPieces* rows;
  const float2* ml;
  const float* o;
  int32_t max_rows;
};
struct CombineArgs {
  PartPieces part[2];     // in the order of the keys
  int32_t n_parts;
  int32_t n_seqs;
  int32_t H_q;
  int64_t n_tokens;
  const int32_t* offsets;
  void* o;
  float* lse;
};

// 16 lanes have a piece's 64 channels; GP groups of them take a row's pieces in turn.
template <int GP>
__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a) {
  __shared__ f32x4 s_o[GP > 1 ? 256 : 1];
  __shared__ float2 s_ml[GP > 1 ? 16 : 1];
  constexpr int kAtOnce = 4;     // pieces on their way to a group
  const int group = threadIdx.x >> 4, l16 = threadIdx.x & 15, turn = group % GP;
  const int64_t row = (int64_t)blockIdx.x * (16 / GP) + group / GP;
  const int64_t t = row / a.H_q;
  const bool real = t < a.n_tokens && t >= a.offsets[0] && t < a.offsets[a.n_seqs];
  float m = kLowest, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  int pieces = 0;
  for (int i = 0; real && i < a.n_parts; ++i) {
    const PartPieces& part = a.part[i];
    const RowPieces rp = part.rows[row];
    pieces += rp.n;
    for (int k0 = turn; k0 < rp.n; k0 += GP * kAtOnce) {
      float2 ml[kAtOnce];
      f32x4 x[kAtOnce];
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) {
        const int k = std::min(k0 + e * GP, rp.n - 1);
        const int64_t at = k == 0 ? rp.first : rp.base + (int64_t)k * rp.stride;
        const int64_t in = std::clamp<int64_t>(at, 0, part.max_rows - 1);
        ml[e] = part.ml[in];
        x[e] = *(const f32x4*)(part.o + in * kDHead + 4 * l16);
        if (k0 + e * GP >= rp.n || in != at) ml[e] = float2{kLowest, 0.f}, x[e] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) {
        const float top = fmaxf(m, ml[e].x);
        const float f = __builtin_amdgcn_exp2f(m - top), g = __builtin_amdgcn_exp2f(ml[e].x - top);
        m = top;
        l = l * f + ml[e].y * g;
        o = o * f + x[e] * g;
      }
    }
  }
  if constexpr (GP > 1) {
    if (l16 == 0) s_ml[group] = float2{m, l};
    s_o[threadIdx.x] = o;
    __syncthreads();
    if (turn != 0) return;
    float top = m;
#pragma unroll
    for (int i = 1; i < GP; ++i) top = fmaxf(top, s_ml[group + i].x);
    m = top;
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < GP; ++i) {
      const float f = __builtin_amdgcn_exp2f(s_ml[group + i].x - top);
      l += s_ml[group + i].y * f;
      o += s_o[threadIdx.x + i * 16] * f;
    }
  }
  if (pieces == 0) return;
  if (a.lse && l16 == 0) a.lse[row] = log_sum(m, l);
  const float f = l == 0.f ? 0.f : 1.f / l;
  *(u32x2*)((char*)a.o + (row * kDHead + 4 * l16) * 2) = u32x2{pack_bf16x2(o[0] * f, o[1] * f), pack_bf16x2(o[2] * f, o[3] * f)};
}

// ---- what runs -----------------------------------------------------------------------------------------------

// Tiles of the line's parts: query tiles of 16 rows in the kernel of few rows, 0: tiles of 256 rows in a launch of their own
struct Choice {
  int tiles[2];             // of the part with the prefix against all rows (stacked), and of the sequences' part
  bool stacked;             // there is a first part; else the second one has the prefix too
  int shares[2];
  int64_t slots[2];
  int rows[2];              // of a tile
  int64_t row_pieces;       // bytes of the RowPieces of a part
};

// Own rows in 4 bits behind a prefix that is taken with the rows of all sequences: from so many on (of all sequences and key heads, by the room in the page table, which
// is what the host knows of lengths) the prefix has a launch of its own, in tiles of 256 rows, and the own keys one of three waves a SIMD instead of
// two.  In one launch / apart, us, 32 heads on 8, prefixes of 3000 and 20 000: 64 sequences with room for 0.56 M 33.1 / 34.7 and 49.9 / 49.0, 1.6 M 47.8 / 41.1 and
// 62.8 / 56.1, 11.3 M 172.9 / 114.3 and 209.1 / 134.1; 24 x 4 tokens 0.29 M 29.2 / 37.3 and 54.8 / 55.8, 0.95 M 38.6 / 42.8 and 61.8 / 62.0, 3.7 M 83.5 / 66.2 and
// 107.8 / 83.8; 40 sequences 1.3 M 41.6 / 38.0 and 55.4 / 51.9.  (Tables half full, or full.)  Less full: 64 sequences, 11.3 M, at a tenth 54.8 / 44.1 and 70.2 / 58.2, at a
// hundredth 26.9 / 30.5 and 45.1 / 45.7; 24 x 4 tokens, 4.2 M, at a quarter 55.8 / 52.5 and 77.6 / 66.2, at a tenth 37.0 / 44.6 and 60.1 / 57.6; 40 sequences on 4
// heads, 1.3 M, at a tenth 23.5 / 28.7 and 30.4 / 41.9: a table with far more room than its sequences take costs up to 12 us.
constexpr int64_t kApartKeys = 1000000;
bool prefix_apart(const PagedArgs& cache, bool mx4) {
  return mx4 && ((int64_t)cache.n_seqs * cache.table_stride << cache.page_shift) * cache.H_kv > kApartKeys;
}
constexpr int64_t align256(int64_t x) { return (x + 255) / 256 * 256; }

Choice choose(int64_t n_tokens, int n_seqs, int H_q, int H_kv, int64_t P, bool apart) {
  Choice c = {};
  const int64_t rows = n_tokens * (H_q / H_kv), mean = rows / n_seqs;
  // Rows of all sequences together against the prefix spare walks along it (`spared` keys of a head, 256 bytes each, in part from caches) and cost every row
  // a second set of pieces, apart from the first.  The line between the two is a fit to 220 random batches of 2 to 120 sequences, 1 to 32 rows each, 1 to 16
  // heads and 64 to 28 000 shared keys: the other side would be at most 13 % quicker, 0.4 % on average.  us together / each sequence by itself, with (spared keys
  // in thousands, rows x heads): 13.0 / 10.8 (34, 96), 57.1 / 29.2 (150, 21 840), 23.6 / 20.9 (257, 720),
  // 13.8 / 19.0 (321, 84), 20.5 / 22.5 (389, 1120), 26.9 / 28.7 (477, 3312), 35.3 / 54.7 (770, 624), 34.0 / 140.7 (6548, 936).
  // Sequences of more rows fill tiles: 24 x 60 rows 46.7 / 32.7.
  const int64_t spared = (n_seqs - (rows + 63) / 64) * P * H_kv;
  c.stacked = mean <= 32 && spared > 250000 + 20 * rows * H_kv;
  // Up to 1024 rows of all sequences go with the own keys in one launch (drafts of 48 streams 62.3, with the prefix in 256-row tiles 71.3; 256 streams
  // 93.6, 104), unless many own keys in 4 bits need one of their own (kApartKeys).
  c.tiles[0] = !c.stacked ? 0 : rows <= 16 ? 1 : rows <= 1024 && !apart ? 4 : 0;
  // Tiles as small as hold a sequence's rows, on average: 100 random batches, time with the smaller tile / with the larger, geometric mean: 16 or 32 rows
  // at 9 to 16 rows a sequence 0.95, 32 or 64 at 25 to 32 0.87, at 33 to 48 0.96, but up to 1.3 where the second tile's walk counts; the
  // other way round 16 against 32 at 17 to 24 1.15.  Together with the prefix's 64-row tiles the registers are theirs, and 32 rows are quicker from 9 on: 62.3,
  // with 16 68.6.
  // 256-row tiles, in which a key is read for four times as many rows, where there is work to spread them over the chip, by the keys known here: 102 random
  // batches of 129 to 2047 rows a sequence, 64-row tiles 0.66 to 1.18 of the time below 30 million rows x keys, from 100 million on 1.16 to 1.41; this line is
  // 0.7 % from the better side on average.  The sequences' own keys lie on the device: only new tokens count for them here, and rows cached earlier do not, so that
  // pieces of prompts behind long histories of their own take 64-row tiles where 256 would do: 4 x 512 rows to 30 000 own keys, 8 heads 259 us (in 256-row
  // tiles 193), 512 to 20 000, 16 heads 102 (85), 8 x 200 to 4000 72 (61); 2 x 1000 to 8000, 16 heads on 4, 100 (102).  Not up to 128 rows, which would be half a tile: 8 x 100 rows 50.2, in 64-row tiles 43.6.
  const int64_t work = rows * H_kv * (P + n_tokens / n_seqs);
  c.tiles[1] = mean <= (c.tiles[0] ? 8 : 16) ? 1 : mean <= 32 ? 2 : mean <= 128 || work < 30000000 ? 4 : 0;
  c.row_pieces = align256(n_tokens * H_q * (int64_t)sizeof(RowPieces));
  const int most = std::max(c.tiles[0], c.tiles[1]);
  for (int i = c.stacked ? 0 : 1; i < 2; ++i) {
    c.rows[i] = c.tiles[i] ? 16 * c.tiles[i] : kWideRows;
    c.shares[i] = 256 * (c.tiles[i] == 0 ? 2 : waves_per_simd(most));
    const int64_t tiles = H_kv * (i == 0 ? (rows + c.rows[i] - 1) / c.rows[i] : rows / c.rows[i] + n_seqs);
    c.slots[i] = c.stacked ? c.shares[i] + tiles : 2 * c.shares[i];
  }
  return c;
}
int64_t slot_bytes(const Choice& c, int i) { return align256(c.slots[i] * c.rows[i] * 8) + align256(c.slots[i] * c.rows[i] * kDHead * 4); }
int64_t plan_bytes(const Choice& c) {
  int64_t bytes = 0;
  for (int i = c.stacked ? 0 : 1; i < 2; ++i) bytes += c.row_pieces + slot_bytes(c, i);
  return bytes;
}

template <int NA, int NB, int KIND>
void start(const LineArgs& a, int shares, hipStream_t stream) {
  if (a.c.causal)
    hipLaunchKernelGGL((attention_cached_kernel<NA, NB, true, KIND>), dim3(shares), dim3(64 * kWaves), 0, stream, a);
  else
    hipLaunchKernelGGL((attention_cached_kernel<NA, NB, false, KIND>), dim3(shares), dim3(64 * kWaves), 0, stream, a);
}
template <int NA, int NB>
void start(const LineArgs& a, int shares, hipStream_t stream) {
  if constexpr (NA > 0) {      // (the sequences' part has no prefix)
    if (a.c.scales) return start<NA, NB, MX4_ALONE>(a, shares, stream);
  } else if (a.c.scales) {
    return a.c.P > 0 && a.part[1].with_prefix ? start<NA, NB, MX4_ROWS>(a, shares, stream) : start<NA, NB, MX4_ALONE>(a, shares, stream);
  }
  if (a.c.lse && a.finish)      // (pieces in their slots leave the sums to combine_kernel)
    start<NA, NB, ROWS_AND_SUMS>(a, shares, stream);
  else
    start<NA, NB, ROWS>(a, shares, stream);
}
template <int KIND>
void start_wide(const LineArgs& a, bool causal, int shares, hipStream_t stream) {
  if (causal)
    hipLaunchKernelGGL((attention_cached_wide_kernel<true, KIND>), dim3(shares), dim3(64 * kWideWaves), 0, stream, a);
  else
    hipLaunchKernelGGL((attention_cached_wide_kernel<false, KIND>), dim3(shares), dim3(64 * kWideWaves), 0, stream, a);
}

}  // namespace

int64_t cached_attention_workspace(int64_t n_tokens, int n_seqs, int H_q, int H_kv, int64_t P) {
  return std::max(plan_bytes(choose(n_tokens, n_seqs, H_q, H_kv, P, false)), plan_bytes(choose(n_tokens, n_seqs, H_q, H_kv, P, true)));
}
int64_t cached_attention_needs(const PagedArgs& cache, bool mx4, int64_t n_tokens, int H_q, int64_t P) {
  return plan_bytes(choose(n_tokens, cache.n_seqs, H_q, cache.H_kv, P, prefix_apart(cache, mx4)));
}

hipError_t launch_cached_attention(const CachedAttnArgs& args, hipStream_t stream) {
  if (args.n_tokens == 0) return hipSuccess;
  const int H_kv = args.cache.H_kv, H_q = H_kv * args.group;
  const Choice ch = choose(args.n_tokens, args.cache.n_seqs, H_q, H_kv, args.P, prefix_apart(args.cache, args.scales != nullptr));
  LineArgs a = {};
  a.c = args;
  a.H_q = H_q;
  a.group_magic = (uint32_t)((((uint64_t)1 << 32) + args.group - 1) / args.group);
  a.finish = !ch.stacked;
  a.min_length = kWaves;
  CombineArgs cb = {};
  cb.n_seqs = args.cache.n_seqs;
  cb.H_q = H_q;
  cb.n_tokens = args.n_tokens;
  cb.offsets = args.offsets;
  cb.o = args.o;
  cb.lse = args.lse;
  char* at = args.workspace;
  for (int i = ch.stacked ? 0 : 1; i < 2; ++i) {
    const int64_t rows = ch.slots[i] * ch.rows[i];
    a.part[i] = {ch.stacked && i == 0, !ch.stacked || i == 0, i == 1, (int32_t)ch.slots[i], (RowPieces*)at, (float2*)(at + ch.row_pieces),
                 (float*)(at + ch.row_pieces + align256(rows * 8))};
    at += ch.row_pieces + slot_bytes(ch, i);
    cb.part[cb.n_parts++] = {a.part[i].rows, a.part[i].slot_ml, a.part[i].slot_o, (int32_t)rows};
  }
  // Tiles of 256 rows: the part is all of the launch's line
  auto wide = [&](int i) {
    LineArgs w = a;
    w.part[0] = a.part[i];
    w.min_length = 2 * kWideUnit;
    // (the part of the prefix has no rows in 4 bits)
    const bool causal = args.causal && i == 1;
    if (i == 1 && args.scales)
      args.P > 0 && a.part[1].with_prefix ? start_wide<MX4_ROWS>(w, causal, ch.shares[i], stream) : start_wide<MX4_ALONE>(w, causal, ch.shares[i], stream);
    else if (args.lse && a.finish)
      start_wide<ROWS_AND_SUMS>(w, causal, ch.shares[i], stream);
    else
      start_wide<ROWS>(w, causal, ch.shares[i], stream);
  };
  if (ch.stacked && ch.tiles[0] == 0) wide(0);
  const int na = ch.tiles[0], nb = ch.tiles[1], shares = ch.shares[1];
  if (nb == 0)
    wide(1);
  else if (na == 0)
    nb == 1 ? start<0, 1>(a, shares, stream) : nb == 2 ? start<0, 2>(a, shares, stream) : start<0, 4>(a, shares, stream);
  else if (na == 1)
    start<1, 1>(a, shares, stream);
  else
    nb == 1 ? start<4, 1>(a, shares, stream) : start<4, 2>(a, shares, stream);    // (at most 32 rows a sequence together with the prefix)
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows = args.n_tokens * H_q;
  // Few rows have many pieces each, many rows fill the chip without a group's others.  Time of both kernels on 110 random batches, geometric mean: 16 groups / 4 up to
  // 512 rows 1.00, and above 1.03; 4 / 1 up to 2048 0.99, from there to 8192 1.03, to 32 768 1.08.  16 / 4 at 2048 to 8192: 1.10.
  if (rows <= 512)
    hipLaunchKernelGGL(combine_kernel<16>, dim3((unsigned)rows), dim3(256), 0, stream, cb);
  else if (rows <= 2048)
    hipLaunchKernelGGL(combine_kernel<4>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, cb);
  else
    hipLaunchKernelGGL(combine_kernel<1>, dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, stream, cb);
  return hipGetLastError();
}

}  // namespace httm
