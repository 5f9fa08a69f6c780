// Attention of a batch of sequences to a prefix that all of them share and to the pages of their own:
//   o = sum_j e^(scale q.k_j) v_j / sum_j e^(scale q.k_j),   j over prefix ++ own rows (causal: up to the token's own)
//
// Rows.  The query heads that share a key head and the tokens of a sequence are rows of one matrix: row r of sequence b and
// key head h is token offsets[b] + r / group, query head h * group + r % group.  A tile is R of these rows.
//
// The line.  The work of a launch is one line of units: for every key head, every sequence, every tile of its rows, the
// units of kUnit keys that the tile attends to, prefix first.  It is cut into equal shares, one per workgroup, wherever the
// cuts fall; lengths are read on the device, so a captured call follows the sequences as they grow.  A workgroup finds
// the start of its share by a scan over the sequences, and walks.  What a share holds of a tile is a piece; a piece that is
// not its whole tile leaves its maximum, sum and un-normalised product in the workspace, and combine_kernel adds
// the pieces of every row up, in the order of the keys: results are run-to-run identical.
//
// Prefix, computed once.  Where sequences have few rows each, the prefix is a launch of its own whose tiles are cut from the
// rows of all sequences together, so that its keys are read once per tile of the whole batch and not per
// sequence; combine_kernel joins it with the own keys.  Where a sequence fills tiles by itself, that would save nothing:
// there its tiles run over prefix and own keys in one go.
//
// A wave.  S^T = K Q^T with v_mfma_f32_16x16x32_bf16 (A = 16 keys x 32 channels, B = 32 channels x 16 rows): a lane has
// one row's scores of 4 of 16 keys, so that statistics are sums in a lane and two exchanges.  The weights go from the
// accumulators straight into the B operand of O^T += V^T P^T, which fixes the order of keys in an operand (lane group
// g: 4 g + 0..3 and 16 + 4 g + 0..3); V^T in that order are two transposing LDS reads of the row-major rows.  The
// waves of a workgroup take a share's units in turn and meet at the end of the piece.
//
// Softmax.  m is a running shift, not the maximum: it follows when a score is more than 2^kSlack above it, which
// after the first unit is rare, and a comparison per score pays for it.
#include <algorithm>

#include "dev_common.hpp"
#include "kernels.hpp"

namespace httm {

namespace {

constexpr int kUnit = 32;                       // keys
constexpr int kUnitBytes = kUnit * kRowBytes;
constexpr float kSlack = 10.f;
constexpr float kLowest = -3.402823466e38f;     // a finite shift for sums without a key

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Where the pieces of a row of q are, as rows of the workspace: the first in `first`, the i-th in base + i * stride
struct RowPieces {
  int32_t first, base, stride, n;   // n = 0: the row is written already
};

struct LineArgs {
  CachedAttnArgs c;
  int32_t H_q;
  int32_t stacked;        // one sequence that has the tokens of all of them
  int32_t with_prefix, with_own;
  int32_t finish;         // whole tiles are written to o; else every piece is left in its slot
  int32_t min_units;      // a share has at least so many
  int32_t max_slots;
  RowPieces* rows;        // [n_tokens * H_q]
  float2* slot_ml;        // [max_slots][R] shift (log2 units) and sum
  float* slot_o;          // [max_slots][R][64]
};

struct Pair {
  float a, b;
};
__device__ __forceinline__ Pair swap16(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t lo = r[0], hi = r[1];
  return {__uint_as_float(lo), __uint_as_float(hi)};
}
__device__ __forceinline__ Pair swap32(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t lo = r[0], hi = r[1];
  return {__uint_as_float(lo), __uint_as_float(hi)};
}
// over the four lane groups that share a row
__device__ __forceinline__ float groups_max(float x) {
  Pair p = swap16(x);
  p = swap32(fmaxf(p.a, p.b));
  return fmaxf(p.a, p.b);
}
__device__ __forceinline__ float groups_sum(float x) {
  Pair p = swap16(x);
  p = swap32(p.a + p.b);
  return p.a + p.b;
}
__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32) | (uint32_t)uniform((int)x));
}

// A sequence as the line sees it
struct Seq {
  int first, n;    // tokens
  int len;         // own keys
  int tiles;       // of R rows
  int units;       // of a tile, at least one: rows without keys are written too
};
template <int R>
__device__ __forceinline__ void count(const LineArgs& a, Seq& s) {
  const int keys = (a.with_prefix ? ((int)a.c.P + kUnit - 1) / kUnit : 0) + (s.len + kUnit - 1) / kUnit;
  s.tiles = (s.n * a.c.group + R - 1) / R;
  s.units = keys > 1 ? keys : 1;
}
// 64 sequences from `base` on, one per lane; those behind the last have no tokens
template <int R>
__device__ __forceinline__ Seq load_window(const LineArgs& a, int base, int lane) {
  const CachedAttnArgs& c = a.c;
  const int n_seq = a.stacked ? 1 : c.cache.n_seqs, b = base + lane, T = (int)c.n_tokens;
  Seq s = {};
  if (b < n_seq) {
    const int o0 = c.offsets[b], o1 = c.offsets[a.stacked ? c.cache.n_seqs : b + 1];
    const int len = a.with_own ? c.seq_lens[b] : 0;
    s.first = std::clamp(o0, 0, T);
    s.n = std::clamp(o1, s.first, T) - s.first;
    s.len = std::clamp(len, 0, c.cache.table_stride << c.cache.page_shift);
  }
  count<R>(a, s);
  return s;
}
template <int R>
__device__ __forceinline__ Seq of_lane(const LineArgs& a, const Seq& window, int l) {
  Seq s;
  s.first = __builtin_amdgcn_readlane(window.first, l);
  s.n = __builtin_amdgcn_readlane(window.n, l);
  s.len = __builtin_amdgcn_readlane(window.len, l);
  count<R>(a, s);
  return s;
}

// floor(x / y) for 0 <= x, 0 < y, both below 2^52: the compiler's 64-bit division takes some 200 instructions, in front of
// everything else that a workgroup does
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
  int64_t q = (int64_t)((double)x / (double)y);
  const int64_t r = x - q * y;
  q += r < 0 ? -1 : (r >= y ? 1 : 0);
  return uniform64(q);
}

// Where a share starts
struct Place {
  int h, b, tile, unit;
  int tile_id;      // of (h, b, tile) in the line
  int64_t at, end;  // units of the share, as positions on the line
  int64_t per_share, longer;    // units of a share; the first `longer` shares have one more
  int share;
  int base;         // first sequence of the window
  // the share that has unit x of the line
  __device__ __forceinline__ int share_of(int64_t x) const {
    const int64_t split = longer * (per_share + 1);
    return (int)(x < split ? quotient(x, per_share + 1) : longer + quotient(x - split, per_share));
  }
};
template <int R>
__device__ __forceinline__ bool find_share(const LineArgs& a, int lane, Place& p, Seq& window) {
  const int n_seq = a.stacked ? 1 : a.c.cache.n_seqs;
  const int lanes = n_seq < 64 ? n_seq : 64;
  window = load_window<R>(a, 0, lane);
  int64_t sum = (int64_t)window.tiles * window.units;
  int tiles = window.tiles;
  for (int i = 64; i < n_seq; i += 64) {
    const Seq s = load_window<R>(a, i, lane);
    sum += (int64_t)s.tiles * s.units;
    tiles += s.tiles;
  }
  for (int i = 1; i < lanes; i <<= 1) {
    sum += __shfl_xor(sum, i);
    tiles += __shfl_xor(tiles, i);
  }
  const int64_t per_head = uniform64(sum);
  const int tiles_per_head = uniform(tiles);
  if (per_head == 0) return false;
  const int64_t total = per_head * a.c.cache.H_kv;
  const int shares = (int)std::clamp<int64_t>(quotient(total, a.min_units), 1, gridDim.x);
  // workgroups go to the 8 XCDs in turn: shares next to each other, which read the same keys, go to one of them
  const int per_xcd = (shares + 7) / 8;
  p.share = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per_xcd || p.share >= shares) return false;
  p.per_share = quotient(total, shares);
  p.longer = total - p.per_share * shares;
  p.at = p.share * p.per_share + std::min<int64_t>(p.share, p.longer);
  p.end = p.at + p.per_share + (p.share < p.longer ? 1 : 0);
  p.h = (int)quotient(p.at, per_head);
  int64_t rest = p.at - p.h * per_head;
  int before = 0;
  for (p.base = 0;; p.base += 64) {
    if (p.base > 0) window = load_window<R>(a, p.base, lane);
    int64_t scan = (int64_t)window.tiles * window.units;
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
    const Seq s = of_lane<R>(a, window, l);
    rest -= uniform64(__shfl(scan, l)) - (int64_t)s.tiles * s.units;
    p.b = p.base + l;
    p.tile = (int)quotient(rest, s.units);
    p.unit = (int)(rest - (int64_t)p.tile * s.units);
    p.tile_id = p.h * tiles_per_head + before + uniform(__shfl(tscan, l)) - s.tiles + p.tile;
    return true;
  }
}

// V rows in LDS: chunk c of row r sits at position c ^ v_swizzle(r), so that the transposing reads find their rows in
// different banks.
__device__ __forceinline__ int v_swizzle(int row) { return ((row >> 1) & 3) << 1; }

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
  int limit[NQ];        // causal: own keys that the lane's row sees
};

// One unit of keys on its way to a wave
struct UnitData {
  u32x4 k[4];       // [key half * 2 + channel half]: the A operands
  u32x4 v[4];       // 8 rows each
};

// Rows of K or V: 16 from `at` on, of which the first `n` are there; the others are read as zeros, wherever they would be
__device__ __forceinline__ __amdgpu_buffer_rsrc_t half_rows(const char* at, int n) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)at, 0, n * kRowBytes, kRawBufferWord3);
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
        const bool seen = row0 + j < limit[qt];
#pragma unroll
        for (int r = 0; r < 4; ++r) o[ct][qt][r] += seen ? d[r] : 0.f;
      }
    }
  }
}

// Scores, statistics and product of a unit.  row0: its first key; end: keys from there on are masked in all rows (causal
// own keys: in some); ok: bit per half of 16 keys, whether it has a page.
template <int NQ, bool CAUSAL>
__device__ __forceinline__ void unit_step(WaveState<NQ>& w, const UnitData& d, bf16_t* sv, float c, int row0, int end, int ok, bool own,
                                          int lane) {
  const int l16 = lane & 15, grp = lane >> 4;
  const bool masked = ok != 3 || row0 + kUnit > end;
  const bool wild = CAUSAL && masked && own && __ballot(not_finite(d.v)) != 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 8 * i + (lane >> 3);
    *(u32x4*)(sv + r * kDHead + ((lane & 7) ^ v_swizzle(r)) * 8) = d.v[i];
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
      const int limit = (CAUSAL && own ? w.limit[qt] : end) - row0 - 4 * grp;
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
    const f32x4 &s0 = s[0][qt], &s1 = s[1][qt];
    top[qt] = fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])), fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
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
    add_seen<NQ>(w.o, av, p, w.limit, row0, lane);
  } else {
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) w.o[ct][qt] = mfma16(av[ct], p[qt], w.o[ct][qt]);
  }
}

constexpr int waves_per_simd(int nq) { return nq == 1 ? 3 : 2; }

template <int NQ, int KS, bool CAUSAL>
__global__ __launch_bounds__(64 * KS) __attribute__((amdgpu_waves_per_eu(waves_per_simd(NQ), waves_per_simd(NQ)))) void attention_cached_kernel(
    const LineArgs a) {
  constexpr int R = 16 * NQ;
  constexpr int DEPTH = 1;     // units of a wave on their way besides the one in work
  __shared__ __attribute__((aligned(16))) char s_mem[KS * kUnitBytes];
  __shared__ float2 s_ml[KS > 1 ? KS : 1][R];
  const CachedAttnArgs& c = a.c;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int l16 = lane & 15, grp = lane >> 4;
  bf16_t* sv = (bf16_t*)(s_mem + wave * kUnitBytes);
  Place p;
  Seq window;
  if (!find_share<R>(a, lane, p, window)) return;
  Seq s = of_lane<R>(a, window, p.b - p.base);
  const int prefix_units = a.with_prefix ? ((int)c.P + kUnit - 1) / kUnit : 0;
  const int64_t share_start = p.at;
  const int k_offset = l16 * kRowBytes + grp * 16, v_offset = lane * 16;

  while (p.at < p.end) {
    const int u0 = p.unit;
    const int u1 = (int)std::min<int64_t>(s.units, p.unit + (p.end - p.at));
    const int n_rows = s.n * c.group, r0 = p.tile * R;
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
          const int64_t at = ((((int64_t)g.page[i] * c.cache.H_kv + p.h) << c.cache.page_shift) + (row & ((1 << c.cache.page_shift) - 1))) * kRowBytes;
          k = c.cache.k_pages + at;
          v = c.cache.v_pages + at;
          n = there ? s.len - row : 0;
          ok &= there ? 3 : ~(1 << i);
        }
        n = std::clamp(n, 0, 16);
        const __amdgpu_buffer_rsrc_t kr = half_rows(k, n), vr = half_rows(v, n);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) d.k[2 * i + ks] = load_row(kr, k_offset + ks * 64);
#pragma unroll
        for (int e = 0; e < 2; ++e) d.v[2 * i + e] = load_row(vr, v_offset + e * 1024);
      }
      return ok;
    };

    WaveState<NQ> w;
    auto row_of = [&](int r, int& token) {     // the head of q, and the token
      const int i = r / c.group;
      token = s.first + i;
      return p.h * c.group + (r - i * c.group);
    };
    auto seen_by = [&](int r) { return CAUSAL ? std::clamp(s.len - s.n + r / c.group + 1, 0, s.len) : s.len; };
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      const int r = std::min(r0 + 16 * qt + l16, n_rows - 1);
      int token;
      const int head = row_of(r, token);
      const char* q = c.q.data + (token * c.q.token_stride + head * c.q.head_stride) * 2;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) w.qf[qt][ks] = *(const bf16x8*)(q + (ks * 4 + grp) * 16);
      if (CAUSAL) w.limit[qt] = seen_by(r);
      w.m[qt] = kLowest;
      w.l[qt] = 0.f;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) w.o[ct][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int least = uniform(seen_by(r0)), most = uniform(seen_by(std::min(r0 + R, n_rows) - 1));
    // keys behind the last one that a row of the tile sees are not read
    const int stop = std::min(u1, prefix_units + (most + kUnit - 1) / kUnit);
    // DEPTH units are on their way, the pages of the next one are asked for.  (The data moves through registers: two copies
    // of the step in the loop need more scalar registers than there are.)
    int unit = u0 + wave;
    UnitData d[DEPTH + 1];
    int ok[DEPTH + 1];
    Pages g = look_up(unit);
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      if (unit + i * KS < stop) ok[i] = fetch(unit + i * KS, g, d[i]);
      g = look_up(unit + (i + 1) * KS);
    }
#pragma unroll 1
    for (; unit < stop; unit += KS) {
      if (unit + DEPTH * KS < stop) ok[DEPTH] = fetch(unit + DEPTH * KS, g, d[DEPTH]);
      g = look_up(unit + (DEPTH + 1) * KS);
      const bool own = unit >= prefix_units;
      unit_step<NQ, CAUSAL>(w, d[0], sv, c.scale_log2, (own ? unit - prefix_units : unit) * kUnit, own ? least : (int)c.P, ok[0], own, lane);
#pragma unroll
      for (int i = 0; i < DEPTH; ++i) {
        d[i] = d[i + 1];
        ok[i] = ok[i + 1];
      }
    }

    // ---- the piece's end ---------------------------------------------------------------------------------
    const bool whole = u0 == 0 && u1 == s.units;
    const bool finish = a.finish && whole;
    int slot = -1;
    if (!finish) slot = a.finish ? 2 * p.share + (p.at == share_start ? 0 : 1) : p.share + p.tile_id;
    if (u0 == 0 && wave == 0) {
      RowPieces rp = {0, 0, 0, 0};
      if (!finish) {
        rp.n = p.share_of(p.at + s.units - 1) - p.share + 1;
        rp.first = slot * R;
        rp.base = (a.finish ? 2 * p.share : slot) * R;
        rp.stride = a.finish ? 2 * R : R;
      }
#pragma unroll
      for (int i = 0; i < (R + 63) / 64; ++i) {
        const int r = r0 + i * 64 + lane;
        if (i * 64 + lane < R && r < n_rows) {
          int token;
          const int head = row_of(r, token);
          const int in_tile = i * 64 + lane;
          a.rows[(int64_t)token * a.H_q + head] = {rp.first + in_tile, rp.base + in_tile, rp.stride, rp.n};
        }
      }
    }
    const bool store = finish || slot < a.max_slots;
    auto put = [&](int r, int channel, f32x4 o, float l) {    // r: row in the tile
      if (r0 + r >= n_rows || !store) return;
      if (finish) {
        const float f = l == 0.f ? 0.f : 1.f / l;
        int token;
        const int head = row_of(r0 + r, token);
        uint32_t* to = (uint32_t*)((char*)c.o + (((int64_t)token * a.H_q + head) * kDHead + channel) * 2);
        *(u32x2*)to = u32x2{pack_bf16x2(o[0] * f, o[1] * f), pack_bf16x2(o[2] * f, o[3] * f)};
      } else {
        *(f32x4*)(a.slot_o + ((int64_t)slot * R + r) * kDHead + channel) = o;
      }
    };
    if constexpr (KS == 1) {
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
        const float l = groups_sum(w.l[qt]);
        const int r = 16 * qt + l16;
        if (!finish && store && grp == 0 && r0 + r < n_rows) a.slot_ml[(int64_t)slot * R + r] = float2{w.m[qt], l};
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) put(r, 16 * ct + 4 * grp, w.o[ct][qt], l);
      }
    } else {
      float f[NQ];
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
        const float l = groups_sum(w.l[qt]);
        if (grp == 0) s_ml[wave][16 * qt + l16] = float2{w.m[qt], l};
      }
      __syncthreads();
      auto joined = [&](int r) {
        float m = s_ml[0][r].x, l = 0.f;
#pragma unroll
        for (int i = 1; i < KS; ++i) m = fmaxf(m, s_ml[i][r].x);
#pragma unroll
        for (int i = 0; i < KS; ++i) l += s_ml[i][r].y * __builtin_amdgcn_exp2f(s_ml[i][r].x - m);
        return float2{m, l};
      };
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) f[qt] = __builtin_amdgcn_exp2f(w.m[qt] - joined(16 * qt + l16).x);
      f32x4* so = (f32x4*)s_mem;      // [KS][R][4] of 16 channels
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) {
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) so[(wave * R + 16 * qt + l16) * 4 + grp] = w.o[ct][qt] * f[qt];
        __syncthreads();
        for (int i = threadIdx.x; i < R * 4; i += 64 * KS) {
          f32x4 o = so[i];
#pragma unroll
          for (int k = 1; k < KS; ++k) o += so[k * R * 4 + i];
          const float2 ml = joined(i >> 2);
          if (ct == 0 && (i & 3) == 0 && !finish && store && r0 + (i >> 2) < n_rows) a.slot_ml[(int64_t)slot * R + (i >> 2)] = ml;
          put(i >> 2, 16 * ct + 4 * (i & 3), o, ml.y);
        }
        __syncthreads();
      }
    }

    // ---- the next tile --------------------------------------------------------------------------------------
    p.at += u1 - u0;
    p.unit = 0;
    ++p.tile_id;
    if (p.at < p.end && ++p.tile == s.tiles) {
      p.tile = 0;
      do {
        if (++p.b == (a.stacked ? 1 : c.cache.n_seqs)) {
          p.b = 0;
          if (++p.h == c.cache.H_kv) return;
        }
        if (p.b < p.base || p.b >= p.base + 64) {
          p.base = p.b;
          window = load_window<R>(a, p.b, lane);
        }
        s = of_lane<R>(a, window, p.b - p.base);
      } while (s.tiles == 0);
    }
  }
}

// ---- joining the pieces --------------------------------------------------------------------------------------

struct Part {
  const RowPieces* rows;
  const float2* ml;
  const float* o;
  int32_t max_rows;
};
struct CombineArgs {
  Part part[2];           // in the order of the keys
  int32_t n_parts;
  int32_t n_seqs;
  int32_t H_q;
  int64_t n_tokens;
  const int32_t* offsets;
  void* o;
};

// 16 lanes have a piece's 64 channels; GP groups of them take a row's pieces in turn.
template <int GP>
__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a) {
  __shared__ f32x4 s_o[GP > 1 ? 256 : 1];
  __shared__ float2 s_ml[GP > 1 ? 16 : 1];
  const int group = threadIdx.x >> 4, l16 = threadIdx.x & 15;
  const int64_t row = GP == 1 ? (int64_t)blockIdx.x * 16 + group : blockIdx.x;
  const int64_t t = row / a.H_q;
  if (t >= a.n_tokens || t < a.offsets[0] || t >= a.offsets[a.n_seqs]) return;
  float m = kLowest, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  int pieces = 0;
  for (int i = 0; i < a.n_parts; ++i) {
    const Part& part = a.part[i];
    const RowPieces rp = part.rows[row];
    pieces += rp.n;
    for (int k = GP == 1 ? 0 : group; k < rp.n; k += GP) {
      const int at = k == 0 ? rp.first : rp.base + k * rp.stride;
      if (at < 0 || at >= part.max_rows) break;
      const float2 ml = part.ml[at];
      const f32x4 x = *(const f32x4*)(part.o + (int64_t)at * kDHead + 4 * l16);
      const float top = fmaxf(m, ml.x);
      const float f = __builtin_amdgcn_exp2f(m - top), g = __builtin_amdgcn_exp2f(ml.x - top);
      m = top;
      l = l * f + ml.y * g;
      o = o * f + x * g;
    }
  }
  if (pieces == 0) return;
  if constexpr (GP > 1) {
    if (l16 == 0) s_ml[group] = float2{m, l};
    s_o[threadIdx.x] = o;
    __syncthreads();
    if (group != 0) return;
    float top = s_ml[0].x;
#pragma unroll
    for (int i = 1; i < GP; ++i) top = fmaxf(top, s_ml[i].x);
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < GP; ++i) {
      const float f = __builtin_amdgcn_exp2f(s_ml[i].x - top);
      l += s_ml[i].y * f;
      o += s_o[i * 16 + l16] * f;
    }
  }
  const float f = l == 0.f ? 0.f : 1.f / l;
  *(u32x2*)((char*)a.o + (row * kDHead + 4 * l16) * 2) = u32x2{pack_bf16x2(o[0] * f, o[1] * f), pack_bf16x2(o[2] * f, o[3] * f)};
}

// ---- what runs -----------------------------------------------------------------------------------------------

struct Launch {
  int nq, ks;             // 16 * nq rows in a tile, ks waves
  bool stacked, with_prefix, with_own;
  int shares;
  int64_t slots;
};
struct Choice {
  Launch run[2];
  int n;
  bool finish;
  int64_t rows_bytes;     // RowPieces of a launch
};

constexpr int64_t align256(int64_t x) { return (x + 255) / 256 * 256; }

Choice choose(int64_t n_tokens, int n_seqs, int H_q, int H_kv, int64_t P) {
  Choice c = {};
  const int64_t rows = n_tokens * (H_q / H_kv), mean = rows / n_seqs;
  const bool stack = n_seqs > 1 && P > 0 && mean < 64;
  auto few = [&](int64_t n) { return n <= 16; };
  c.finish = !stack;
  c.rows_bytes = align256(n_tokens * H_q * (int64_t)sizeof(RowPieces));
  auto add = [&](int nq, int ks, bool stacked, bool prefix, bool own) {
    Launch& l = c.run[c.n++];
    l = {nq, ks, stacked, prefix, own, 0, 0};
    l.shares = ks == 1 ? 2048 : 512;
    const int64_t R = 16 * nq;
    const int64_t tiles = H_kv * (stacked ? (rows + R - 1) / R : rows / R + n_seqs);
    l.slots = c.finish ? 2 * l.shares : l.shares + tiles;
  };
  if (stack) {
    add(few(rows) ? 1 : 4, 4, true, true, false);
    add(few(mean) ? 1 : 4, few(mean) ? 1 : 4, false, false, true);
  } else {
    add(few(mean) ? 1 : 4, 4, false, P > 0, true);
  }
  return c;
}
int64_t slot_bytes(const Launch& l) { return align256(l.slots * 16 * l.nq * 8) + align256(l.slots * 16 * l.nq * kDHead * 4); }

template <int NQ, int KS>
void start(const LineArgs& a, int shares, hipStream_t stream) {
  if (a.c.causal && a.with_own)
    hipLaunchKernelGGL((attention_cached_kernel<NQ, KS, true>), dim3(shares), dim3(64 * KS), 0, stream, a);
  else
    hipLaunchKernelGGL((attention_cached_kernel<NQ, KS, false>), dim3(shares), dim3(64 * KS), 0, stream, a);
}

}  // namespace

int64_t cached_attention_workspace(int64_t n_tokens, int n_seqs, int H_q, int H_kv, int64_t P) {
  const Choice c = choose(n_tokens, n_seqs, H_q, H_kv, P);
  int64_t bytes = 0;
  for (int i = 0; i < c.n; ++i) bytes += c.rows_bytes + slot_bytes(c.run[i]);
  return bytes;
}

hipError_t launch_cached_attention(const CachedAttnArgs& args, hipStream_t stream) {
  if (args.n_tokens == 0) return hipSuccess;
  const int H_kv = args.cache.H_kv, H_q = H_kv * args.group;
  const Choice ch = choose(args.n_tokens, args.cache.n_seqs, H_q, H_kv, args.P);
  CombineArgs cb = {};
  cb.n_parts = ch.n;
  cb.n_seqs = args.cache.n_seqs;
  cb.H_q = H_q;
  cb.n_tokens = args.n_tokens;
  cb.offsets = args.offsets;
  cb.o = args.o;
  char* at = args.workspace;
  for (int i = 0; i < ch.n; ++i) {
    const Launch& l = ch.run[i];
    LineArgs a = {};
    a.c = args;
    a.H_q = H_q;
    a.stacked = l.stacked;
    a.with_prefix = l.with_prefix;
    a.with_own = l.with_own;
    a.finish = ch.finish;
    a.min_units = l.ks;
    a.max_slots = (int32_t)l.slots;
    const int R = 16 * l.nq;
    a.rows = (RowPieces*)at;
    a.slot_ml = (float2*)(at + ch.rows_bytes);
    a.slot_o = (float*)(at + ch.rows_bytes + align256(l.slots * R * 8));
    at += ch.rows_bytes + slot_bytes(l);
    cb.part[i] = {a.rows, a.slot_ml, a.slot_o, (int32_t)(l.slots * R)};
    if (l.nq == 1 && l.ks == 1)
      start<1, 1>(a, l.shares, stream);
    else if (l.nq == 1)
      start<1, 4>(a, l.shares, stream);
    else
      start<4, 4>(a, l.shares, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t rows = args.n_tokens * H_q;
  if (rows <= 2048)
    hipLaunchKernelGGL(combine_kernel<16>, dim3((unsigned)rows), dim3(256), 0, stream, cb);
  else
    hipLaunchKernelGGL(combine_kernel<1>, dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, stream, cb);
  return hipGetLastError();
}

}  // namespace httm
