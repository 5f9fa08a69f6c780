// A paged cache within a budget: what attention weight every key of a sequence gathers, and the keys with the least of it leave.
//
//   weigh   w_j <- decay w_j + sum over the step's rows r that see key j of e^(scale q_r.k_j - lse_r)
//   evict   of the keys between the first and the last ones those of highest w stay; the places that this leaves are filled from behind
#include <algorithm>

#include "attention_common.hpp"
#include "dev_common.hpp"
#include "kernels.hpp"
#include "mx4.hpp"

namespace httm {

namespace {

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32) | (uint32_t)uniform((int)x));
}

// floor(x / y) for 0 <= x, 0 < y, both below 2^52, for all lanes alike: the compiler's 64-bit division takes 130 instructions
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
  int64_t q = (int64_t)((double)x / (double)y);
  const int64_t r = x - q * y;
  q += r < 0 ? -1 : (r >= y ? 1 : 0);
  return uniform64(q);
}

// ---- weights ---------------------------------------------------------------------------------------------------
//
// The rows of a sequence and a key head are those of attention: r / group-th token, query head h * group + r % group.  S = Q K^T with
// v_mfma_f32_16x16x32_bf16, A = 16 rows and B = 16 keys of 32 channels: a lane has one key's scores of 4 of 16 rows, so that a key's sum is one register, and
// what is left of it at the end two exchanges.  A wave holds 64 keys and goes over rows.  Two kernels: where sequences have few rows
// every wave has keys of its own and keeps the rows of its head in registers from one item of 64 keys to the next; where
// they have many, the four waves of a workgroup share 64 keys and take tiles of rows in turn.  No sum depends on how the work falls: results are
// run-to-run identical.
//
// The work of a launch is a line: sequences, their key heads, the head's items of 64 keys, every item as long as it takes to go over the rows.
// It is cut into equal shares, for waves or workgroups, which take the items that begin in their share.
//
// Exponents: q.k in fp32, times scale * log2(e) minus lse * log2(e) in one rounding, exp2: off by 2^-23 of |lse| or so; sums in fp32.
//
// Measured, and what bounds it.  Few rows: a token each of 64 streams of 100 to 21 984 keys in 4 bits, 32 heads on 8, 63 us, 3.7 TB/s of what has to be moved:
// one item of 2.2 KB on its way for each of four waves a SIMD, half of whose time is waiting.  Many rows: 2 x 1374 tokens to 5496 to 13 740 keys in 16 bits, 16
// heads, 132 us, 0.45 PFLOP/s: 466 million pairs. By the counters a SIMD takes 656 clocks for 1024 of them. In 411 a vector instruction is in work: 78, of which 16 are
// exp2 of 8 clocks (8.6 measured alone, 24 us of all pairs'), 16 fma, 16 additions and 30 the walk over the rows, its addresses and choices. In 128 a product is (8 of 16). Waves
// wait for 57 % of their time: what bounds it is that rows, lse and addresses are taken anew for every 64 keys, and waiting for them. Loading scores a
// tile earlier changes nothing, staging the lse of a run of rows in the LDS instead of asking for every row's took 150 to 133.

constexpr int kWeighWaves = 4;
constexpr int kWeighKeys = 64;      // of an item
constexpr float kLog2e = 1.4426950408889634f;

// over the four lane groups that share a key
__device__ __forceinline__ float groups_sum(float x) {
  LanePair p = swap16(x);
  p = swap32(p.a + p.b);
  return p.a + p.b;
}

struct WeighSeq {
  int first, n, len;
  int items;            // of a key head
  int cost;             // of an item
};
// FRONT: what an item costs besides its rows, in tiles of 16; TURNS: waves that share the rows
template <int FRONT, int TURNS>
__device__ __forceinline__ WeighSeq weigh_seq(const WeighArgs& a, int b) {
  WeighSeq s = {0, 0, 0, 0, 1};
  if (b >= a.cache.n_seqs) return s;
  const int T = (int)a.n_tokens;
  s.first = std::clamp(a.offsets[b], 0, T);
  s.n = std::clamp(a.offsets[b + 1], s.first, T) - s.first;
  s.len = std::clamp(a.seq_lens[b], 0, a.cache.table_stride << a.cache.page_shift);
  s.items = (s.len + kWeighKeys - 1) / kWeighKeys;
  s.cost = FRONT + ((s.n * a.group + 15) / 16 + TURNS - 1) / TURNS;
  return s;
}
// The items of a share: [item, stop) of all key heads of sequence b, then those of the next one
struct WeighShare {
  int64_t at, end, begin;      // on the line; where sequence b begins
  int b;
};
template <int FRONT, int TURNS>
__device__ __forceinline__ bool find_weigh_share(const WeighArgs& a, int id, int shares, int lane, WeighShare& r) {
  auto length = [&](int base) {
    const WeighSeq s = weigh_seq<FRONT, TURNS>(a, base + lane);
    return (int64_t)s.items * a.cache.H_kv * s.cost;
  };
  int64_t total = 0;
  for (int base = 0; base < a.cache.n_seqs; base += 64) total += length(base);
  for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
  total = uniform64(total);
  const int64_t each = quotient(total, shares), more = total - each * shares;
  r.at = each * id + std::min<int64_t>(id, more);
  r.end = r.at + each + (id < more ? 1 : 0);
  if (r.at >= r.end) return false;
  r.begin = 0;
  for (int base = 0; base < a.cache.n_seqs; base += 64) {
    int64_t scan = length(base);
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t v = __shfl_up(scan, d);
      scan += lane >= d ? v : 0;
    }
    const uint64_t in = __ballot(r.begin + scan > r.at);
    if (in != 0) {
      const int l = __builtin_ctzll(in);
      r.b = base + l;
      r.begin += l ? uniform64(__shfl(scan, l - 1)) : 0;
      return true;
    }
    r.begin += uniform64(__shfl(scan, 63));
  }
  return false;
}
// r / group, as a product: exact for what rows there can be, 2^20 tokens of 64 heads
__device__ __forceinline__ int token_of(const WeighArgs& a, int r) { return a.group == 1 ? r : (int)__umulhi((uint32_t)r, a.group_magic); }

// 64 keys of a head on their way: 16 channels of four rows in a lane
template <bool MX4>
struct KeysOnTheirWay {
  u32x4 x[4][MX4 ? 1 : 2];      // codes in two words and the exponent in the third
  uint32_t there;               // bit per 16 keys, whether they have a page
  int pages[4];
  // the pages of the keys from j0 on, asked for before the rows
  __device__ __forceinline__ void look_up(const WeighArgs& a, int b, int len, int j0) {
    const auto* table = (const __attribute__((address_space(4))) int32_t*)(a.cache.table + (int64_t)b * a.cache.table_stride);
    const int shift = a.cache.page_shift;
    pages[0] = j0 < len ? table[j0 >> shift] : -1;     // (no length is beyond the table)
    if (shift < 6)
#pragma unroll
      for (int t = 1; t < 4; ++t) pages[t] = j0 + 16 * t < len ? table[(j0 + 16 * t) >> shift] : -1;
  }
  // rows [t0, t1) of 16 each, all on one page
  template <int T0, int T1>
  __device__ __forceinline__ void request_rows(const WeighArgs& a, int page, int row, int len, int h, int l16, int grp) {
    const PagedArgs& c = a.cache;
    const bool ok = page >= 0 && page < c.n_pages;
    there |= ok ? (1u << T1) - (1u << T0) : 0u;
    const int64_t first = (((int64_t)(ok ? page : 0) * c.H_kv + h) << c.page_shift) + (row & ((1 << c.page_shift) - 1));
    const int n = ok ? std::clamp(len - row, 0, 16 * (T1 - T0)) : 0;
    // (the compiler does not see that all lanes ask for the same rows: it would load for one lane after the other)
    auto rows = [&](const void* p, int bytes) {
      return __builtin_amdgcn_make_buffer_rsrc((void*)uniform64((int64_t)((char*)p + first * bytes)), 0, uniform(n * bytes), kRawBufferWord3);
    };
    if constexpr (MX4) {
      const __amdgpu_buffer_rsrc_t codes = rows(c.k_pages, kMxRowBytes), scales = rows(a.scales, kMxScaleBytes);
#pragma unroll
      for (int t = T0; t < T1; ++t) {
        const int in = l16 + 16 * (t - T0);
        const u32x2 k = __builtin_amdgcn_raw_buffer_load_b64(codes, in * kMxRowBytes + grp * 8, 0, 0);
        x[t][0][0] = k[0];
        x[t][0][1] = k[1];
        x[t][0][2] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(scales, in * kMxScaleBytes + 2 * (grp >> 1), 0, 0);
      }
    } else {
      const __amdgpu_buffer_rsrc_t keys = rows(c.k_pages, kRowBytes);
#pragma unroll
      for (int t = T0; t < T1; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) x[t][e] = __builtin_amdgcn_raw_buffer_load_b128(keys, (l16 + 16 * (t - T0)) * kRowBytes + grp * 32 + e * 16, 0, 0);
    }
  }
  __device__ __forceinline__ void request(const WeighArgs& a, int len, int h, int j0, int l16, int grp) {
    there = 0;
    if (a.cache.page_shift >= 6) {      // (items begin at multiples of 64)
      request_rows<0, 4>(a, pages[0], j0, len, h, l16, grp);
    } else {
      request_rows<0, 1>(a, pages[0], j0, len, h, l16, grp);
      request_rows<1, 2>(a, pages[1], j0 + 16, len, h, l16, grp);
      request_rows<2, 3>(a, pages[2], j0 + 32, len, h, l16, grp);
      request_rows<3, 4>(a, pages[3], j0 + 48, len, h, l16, grp);
    }
  }
  __device__ __forceinline__ void take(bf16x8 (&k)[4][2]) const {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        k[t][e] = __builtin_bit_cast(bf16x8, MX4 ? mx4_values(x[t][0][e], __uint_as_float(x[t][0][2] << 23)) : x[t][e & (MX4 ? 0 : 1)]);
  }
};
// 16 rows of a head: the A operands
__device__ __forceinline__ void load_queries(bf16x8 (&q)[2], const WeighArgs& a, const WeighSeq& s, int h, int r, int n_rows, int grp) {
  const int row = std::min(r, n_rows - 1), i = token_of(a, row);
  const char* at = a.q.data + ((int64_t)(s.first + i) * a.q.token_stride + (h * a.group + row - i * a.group) * a.q.head_stride) * 2;
#pragma unroll
  for (int e = 0; e < 2; ++e) q[e] = *(const bf16x8*)(at + grp * 32 + e * 16);
}
// The same of every 64th row from r on, as a walk: an address takes products that are four times as long as sums
struct QueryWalk {
  const char* head;          // row 0 of the head, the lane's channels
  int64_t at, last;          // bytes from there: of the row, and of the last one
  int64_t step, wrap;        // 64 rows on; a token on and the group's heads back
  int r, in, n_rows, group, rest;
  __device__ __forceinline__ QueryWalk(const WeighArgs& a, const WeighSeq& s, int h, int first, int n, int grp) {
    const int64_t ts = a.q.token_stride * 2, hs = a.q.head_stride * 2;
    const int i = token_of(a, first), j = token_of(a, n - 1), k = token_of(a, 64);
    group = a.group, n_rows = n, r = first;
    head = a.q.data + (int64_t)s.first * ts + (int64_t)h * group * hs + grp * 32;
    in = first - i * group;
    at = i * ts + in * hs;
    last = j * ts + (n - 1 - j * group) * hs;
    rest = 64 - k * group;
    step = k * ts + rest * hs;
    wrap = ts - group * hs;
  }
  // the row's operands (behind the last row: of the last one), and on to the next
  __device__ __forceinline__ void take(bf16x8 (&q)[2]) {
    const char* row = head + (r < n_rows ? at : last);
#pragma unroll
    for (int e = 0; e < 2; ++e) q[e] = *(const bf16x8*)(row + e * 16);
    r += 64;
    in += rest;
    at += step;
    if (in >= group) in -= group, at += wrap;
  }
};
// -lse of row r in base 2; minus infinity for a row that adds nothing: behind the last, or one that saw no key
__device__ __forceinline__ float load_lse(const WeighArgs& a, const WeighSeq& s, int h, int r, int n_rows) {
  const int row = std::min(r, n_rows - 1), i = token_of(a, row);
  const float x = a.lse[(int64_t)(s.first + i) * (a.cache.H_kv * a.group) + h * a.group + row - i * a.group];
  return r >= n_rows || x == -__builtin_inff() ? -__builtin_inff() : -x * kLog2e;
}
// A tile of rows against 64 keys: the scores, and what they give.  `sees` (MASKED): keys that a row sees, from the first of the 64 on
__device__ __forceinline__ void scores_of(f32x4 (&x)[4], const bf16x8 (&k)[4][2], const bf16x8 (&q)[2]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) x[t] = mfma16(q[0], k[t][0], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
  for (int t = 0; t < 4; ++t) x[t] = mfma16(q[1], k[t][1], x[t]);
}
template <bool MASKED, bool CAUSAL>
__device__ __forceinline__ void add_tile(float (&sum)[4], const f32x4 (&x)[4], const f32x4& lse, float scale_log2, const int (&sees)[4], int l16) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      p[e] = __builtin_amdgcn_exp2f(fmaf(x[t][e], scale_log2, lse[e]));
      if (MASKED && (CAUSAL ? 16 * t + l16 >= sees[e] : sees[e] == 0)) p[e] = 0.f;
    }
    sum[t] += (p[0] + p[1]) + (p[2] + p[3]);
  }
}
// Four rows alone, the first lane group's, against 64 keys: a quarter of the exponents where every group takes 16 of the keys.  Row e of the
// scores x[t] of lane group 0, for t = 0 .. 3, into lane group t
__device__ __forceinline__ float groups_apart(const f32x4 (&x)[4], int e) {
  auto bits = [&](int t) { return __float_as_uint(x[t][e]); };
  const auto lo = __builtin_amdgcn_permlane16_swap(bits(0), bits(1), false, false);
  const auto hi = __builtin_amdgcn_permlane16_swap(bits(2), bits(3), false, false);
  const uint32_t a = lo[0], b = hi[0];
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  const uint32_t y = r[0];
  return __uint_as_float(y);
}
// Sums of 64 keys into the weights: key `lane` of them to lane `lane`
__device__ __forceinline__ float key_of_lane(const float (&sum)[4], int grp) {
  float mine = 0.f;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const float x = groups_sum(sum[t]);
    mine = grp == t ? x : mine;
  }
  return mine;
}

// A weight with what came: of a key that was there before (else it has none; decay 0 forgets it, also where it is no number)
__device__ __forceinline__ float weight_with(const WeighArgs& a, bool before, float was, float mine) {
  return before && a.decay != 0.f ? fmaf(a.decay, was, mine) : mine;
}

// Few rows: NT tiles of them stay in registers
constexpr int few_waves(int nt) { return nt == 1 ? 4 : 2; }      // on a SIMD
template <bool MX4, int NT, bool CAUSAL>
__global__ __launch_bounds__(64 * kWeighWaves) __attribute__((amdgpu_waves_per_eu(few_waves(NT), few_waves(NT)))) void weigh_few_kernel(const WeighArgs a) {
  constexpr int kFront = 4;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), l16 = lane & 15, grp = lane >> 4;
  const int H = a.cache.H_kv;
  // (shares next to each other on one XCD: they read the same rows)
  const int id = (int)((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3)) * kWeighWaves + wave;
  WeighShare share;
  if (!find_weigh_share<kFront, 1>(a, id, (int)gridDim.x * kWeighWaves, lane, share)) return;
  const float scale_log2 = a.scale * kLog2e;

  struct Place {
    WeighSeq s;
    int64_t begin;     // of the sequence behind b on the line
    int64_t left;      // items of the sequence that the share still has, this one among them
    int b, h, chunk;
  };
  // the first item at or behind sequence b that the share has
  auto start = [&](Place& p) {
    for (; p.b < a.cache.n_seqs && p.begin < share.end; ++p.b) {
      p.s = weigh_seq<kFront, 1>(a, p.b);
      const int64_t all = (int64_t)p.s.items * H, from = share.at <= p.begin ? 0 : quotient(share.at - p.begin + p.s.cost - 1, p.s.cost);
      p.left = std::min<int64_t>(all, quotient(share.end - p.begin + p.s.cost - 1, p.s.cost)) - from;
      p.begin += all * p.s.cost;
      if (p.left <= 0) continue;
      p.h = (int)quotient(from, p.s.items);
      p.chunk = (int)(from - (int64_t)p.h * p.s.items);
      return true;
    }
    return false;
  };
  auto next = [&](Place& p) {
    if (--p.left == 0) {
      ++p.b;
      return start(p);
    }
    if (++p.chunk == p.s.items) p.chunk = 0, ++p.h;
    return true;
  };
  auto weight_at = [&](const Place& p) { return a.weights + ((int64_t)p.b * H + p.h) * a.columns + p.chunk * kWeighKeys + lane; };

  // The next item's keys are requested as soon as those of the item in work are turned into operands.  (Two items ahead take registers from the
  // waves: 64 streams 74 us, so 64.)
  KeysOnTheirWay<MX4> keys;
  float old = 0.f;
  Place here, ahead;
  ahead.b = share.b, ahead.begin = share.begin;
  bool more = start(ahead);
  bf16x8 q[NT][2];
  f32x4 lse[NT];
  int of_b = -1, of_h = -1;      // whose rows q holds
  auto request = [&] {
    if (!more) return;
    keys.look_up(a, ahead.b, ahead.s.len, ahead.chunk * kWeighKeys);
    keys.request(a, ahead.s.len, ahead.h, ahead.chunk * kWeighKeys, l16, grp);
    old = ahead.chunk * kWeighKeys + lane < ahead.s.len - ahead.s.n ? *weight_at(ahead) : 0.f;
  };
  request();
  while (more) {
    here = ahead;
    const int j0 = here.chunk * kWeighKeys, n_rows = here.s.n * a.group, before = here.s.len - here.s.n;
    const float was = old;
    const uint32_t there = keys.there;
    bf16x8 k[4][2];
    keys.take(k);
    more = next(ahead);
    request();
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    const bool stays = n_rows <= 16 * NT, four = NT == 1 && n_rows <= 4;
    for (int r0 = 0; r0 < n_rows; r0 += 16 * NT) {
      if (!stays || of_b != here.b || of_h != here.h) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          load_queries(q[i], a, here.s, here.h, r0 + 16 * i + l16, n_rows, grp);
#pragma unroll
          for (int e = 0; e < 4; ++e) lse[i][e] = load_lse(a, here.s, here.h, r0 + 16 * i + (four ? 0 : 4 * grp) + e, n_rows);
        }
        of_b = here.b, of_h = here.h;
      }
      if (four) {
        f32x4 x[4];
        scores_of(x, k, q[0]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(groups_apart(x, e), scale_log2, lse[0][e]));
          const int sees = CAUSAL ? before + token_of(a, e) + 1 - j0 : kWeighKeys;
          sum[0] += lse[0][e] == -__builtin_inff() || lane >= sees ? 0.f : p;
        }
        break;
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        if (i > 0 && r0 + 16 * i >= n_rows) break;
        // (rows that add nothing are masked as well: 0 times a key that is not finite would be no number)
        int sees[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = token_of(a, r0 + 16 * i + 4 * grp + e);
          sees[e] = lse[i][e] == -__builtin_inff() ? 0 : CAUSAL ? before + t + 1 - j0 : kWeighKeys;
        }
        f32x4 x[4];
        scores_of(x, k, q[i]);
        add_tile<true, CAUSAL>(sum, x, lse[i], scale_log2, sees, l16);
      }
    }
    float mine = four ? sum[0] : key_of_lane(sum, grp);
    if (!((there >> grp) & 1)) mine = 0.f;
    if (j0 + lane < here.s.len) *weight_at(here) = weight_with(a, j0 + lane < before, was, mine);
  }
}

// Many rows: the waves of a workgroup take tiles of them in turn.  Their lse lie in the LDS, a run of rows at a time.
template <bool MX4, bool CAUSAL>
__global__ __launch_bounds__(64 * kWeighWaves) __attribute__((amdgpu_waves_per_eu(4, 4))) void weigh_many_kernel(const WeighArgs a) {
  constexpr int kFront = 4, kRun = 4096;
  static_assert(16 * kWeighWaves == 64, "a wave's tiles are 64 rows apart");
  __shared__ __attribute__((aligned(16))) float s_lse[kRun];
  __shared__ float s_sum[kWeighWaves][kWeighKeys];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), l16 = lane & 15, grp = lane >> 4;
  const int H = a.cache.H_kv;
  const int id = blockIdx.x;
  WeighShare share;
  if (!find_weigh_share<kFront, kWeighWaves>(a, id, gridDim.x, lane, share)) return;
  const float scale_log2 = a.scale * kLog2e;
  for (int b = share.b; b < a.cache.n_seqs && share.begin < share.end; ++b) {
    const WeighSeq s = weigh_seq<kFront, kWeighWaves>(a, b);
    int64_t item = share.at <= share.begin ? 0 : quotient(share.at - share.begin + s.cost - 1, s.cost);
    const int64_t stop = std::min<int64_t>((int64_t)s.items * H, quotient(share.end - share.begin + s.cost - 1, s.cost));
    share.begin += (int64_t)s.items * H * s.cost;
    if (item >= stop) continue;
    const int n_rows = s.n * a.group, before = s.len - s.n;
    int h = (int)quotient(item, s.items), chunk = (int)(item - (int64_t)h * s.items);
    int run_of_h = -1;
    bool dead = false;      // whether a row of the run adds nothing
    KeysOnTheirWay<MX4> keys;
    keys.look_up(a, b, s.len, chunk * kWeighKeys);
    keys.request(a, s.len, h, chunk * kWeighKeys, l16, grp);
    for (; item < stop; ++item) {
      const int j0 = chunk * kWeighKeys;
      float* weight = a.weights + ((int64_t)b * H + h) * a.columns + j0 + lane;
      const float was = wave == 0 && j0 + lane < before ? *weight : 0.f;
      bf16x8 k[4][2];
      keys.take(k);
      const uint32_t there = keys.there;
      int next_chunk = chunk + 1, next_h = h;
      if (next_chunk == s.items) next_chunk = 0, ++next_h;
      if (item + 1 < stop) keys.look_up(a, b, s.len, next_chunk * kWeighKeys);
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
      // rows in front of the first that sees one of the keys are left out
      const int unseen = CAUSAL && j0 > before ? std::min((j0 - before) * a.group, n_rows) / 16 : 0;
      for (int run = unseen * 16 / kRun * kRun; run < n_rows; run += kRun) {
        if (run_of_h != h || n_rows > kRun) {
          __syncthreads();
          bool none = false;
          const int all = std::min(kRun, (n_rows - run + 15) / 16 * 16);
          for (int i = threadIdx.x; i < all; i += 4 * 64 * kWeighWaves) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = load_lse(a, s, h, run + i + e * 64 * kWeighWaves, n_rows);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int at = i + e * 64 * kWeighWaves;
              if (at < all) s_lse[at] = x[e];
              none |= x[e] == -__builtin_inff() && run + at < n_rows;
            }
          }
          dead = __syncthreads_or(none) != 0;
          run_of_h = h;
        }
        const int t1 = (std::min(run + kRun, n_rows) + 15) / 16;
        int tile = std::max(run / 16, unseen) + wave;
        if (tile >= t1) continue;
        QueryWalk walk(a, s, h, 16 * tile + l16, n_rows, grp);
        // the rows of a tile are on their way while the one before is in work (behind the last: rows that are there)
        bf16x8 q[2][2];
        auto step = [&](int now, int then) {
          const f32x4 lse = *(const f32x4*)(s_lse + 16 * tile - run + 4 * grp);
          walk.take(q[then]);
          f32x4 x[4];
          scores_of(x, k, q[now]);
          int sees[4] = {0, 0, 0, 0};
          if (dead || 16 * tile + 16 > n_rows || (CAUSAL && before + token_of(a, 16 * tile) + 1 < std::min(j0 + kWeighKeys, s.len))) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sees[e] = lse[e] == -__builtin_inff() ? 0 : CAUSAL ? before + token_of(a, 16 * tile + 4 * grp + e) + 1 - j0 : kWeighKeys;
            add_tile<true, CAUSAL>(sum, x, lse, scale_log2, sees, l16);
          } else {
            add_tile<false, CAUSAL>(sum, x, lse, scale_log2, sees, l16);
          }
          tile += kWeighWaves;
        };
        walk.take(q[0]);
        while (true) {
          step(0, 1);
          if (tile >= t1) break;
          step(1, 0);
          if (tile >= t1) break;
        }
      }
      if (item + 1 < stop) keys.request(a, s.len, next_h, next_chunk * kWeighKeys, l16, grp);
      s_sum[wave][lane] = key_of_lane(sum, grp);
      __syncthreads();
      if (wave == 0 && j0 + lane < s.len) {
        float mine = 0.f;
#pragma unroll
        for (int i = 0; i < kWeighWaves; ++i) mine += s_sum[i][lane];
        if (!((there >> grp) & 1)) mine = 0.f;
        *weight = weight_with(a, j0 + lane < before, was, mine);
      }
      __syncthreads();
      chunk = next_chunk, h = next_h;
    }
  }
}

// ---- eviction --------------------------------------------------------------------------------------------------

constexpr int kEvictRuns = 32;       // runs of 64 positions that a wave of the selection holds in the LDS
constexpr int kEvictBins = 2048, kEvictCopies = 2;

// In the order of the weights: NaN is below everything, zeros are alike
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  return w != w ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Moves of a key head of a sequence, in ascending order: how many (-1: none, and nothing else to do), how many of them from in front of row
// `keep`, where to, where from
struct Moves {
  int32_t* n;
  int32_t* near;
  int32_t* to;
  int32_t* from;
};
__device__ __forceinline__ Moves moves_of(const EvictArgs& a, int bh) {
  int32_t* n = (int32_t*)a.workspace + (int64_t)bh * (2 + 2 * (int64_t)a.keep);
  return {n, n + 1, n + 2, n + 2 + a.keep};
}
__device__ __forceinline__ int evict_length(const EvictArgs& a, int b) {
  return std::clamp(a.seq_lens[b], 0, a.cache.table_stride << a.cache.page_shift);
}

// Sum over the lanes up to this one, as data-parallel moves: within rows of 16, then what the rows before have
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);      // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);      // row_bcast:15 into rows 1 and 3, :31 into rows 2 and 3
  return x + __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
}

// (Measured: 64 sequences x 8 heads of 3300 to 4352 keys, 18 us of which 5 are waiting for lengths and weights, 6 the counts, 6 the two passes over what
// stays; 2 x 16 heads of 13 740 and 27 480 keys, on 32 CUs, 32 us.)
// What stays of a key head of a sequence, and what has to move: one workgroup, whose waves have a part of the positions each and its weights, as
// whole numbers in their order, in the LDS.  The threshold comes from counts over 11, 11 and 10 bits of them, as far as it takes until a bin stays or goes
// as a whole (two copies of the bins, by lane: most weights are within a few powers of two of each other, and counts of one bin wait for each other); the
// places of those alike with it and of the moves are sums over the waves before.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(const EvictArgs a) {
  constexpr int kWaves = THREADS / 64, kBinsEach = kEvictBins / THREADS;
  __shared__ uint32_t s_key[kEvictRuns * THREADS];
  __shared__ __attribute__((aligned(16))) uint32_t s_bins[kEvictBins * kEvictCopies];
  __shared__ __attribute__((aligned(16))) uint32_t s_count[5][kWaves];
  __shared__ uint32_t s_prefix, s_need, s_alike;
  const int b = blockIdx.x / a.cache.H_kv, h = blockIdx.x - b * a.cache.H_kv;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int len = evict_length(a, b);
  const Moves mv = moves_of(a, blockIdx.x);
  int32_t* kept = a.kept ? a.kept + (int64_t)blockIdx.x * a.keep : nullptr;
  const float* w = a.weights + (int64_t)blockIdx.x * a.columns;
  const bool over = len > a.keep;
  const int from = a.first, to = len - a.last, gap = a.keep - a.last;
  // a wave's part, in runs of 64 positions
  const int runs = over ? (to - from + THREADS - 1) / THREADS : 0;
  const int p0 = std::min(from + wave * runs * 64, to), p1 = std::min(p0 + runs * 64, to);
  uint32_t* keys = s_key + wave * kEvictRuns * 64 + lane;
#pragma unroll 8
  for (int i = 0; i < std::min(runs, kEvictRuns); ++i) keys[64 * i] = order_of(w[std::min(p0 + 64 * i + lane, len - 1)]);
  const int32_t* table = a.cache.table + (int64_t)b * a.cache.table_stride;
  bool hole = false;
  for (int i = threadIdx.x; i < (len + (1 << a.cache.page_shift) - 1) >> a.cache.page_shift; i += THREADS)
    hole |= table[i] < 0 || table[i] >= a.cache.n_pages;
  hole = __syncthreads_or(hole) != 0;
  if (hole || !over) {
    if (threadIdx.x == 0) {
      *mv.n = -1;
      if (h == 0) a.new_lens[b] = len;
    }
    if (kept)
      for (int d = threadIdx.x; d < a.keep; d += THREADS) kept[d] = !hole && d < len ? d : -1;
    return;
  }
  // f(position of the run, key of the lane) for the runs of the wave.  (Loops: straight code that is run once is fetched first, 3 us for a thousand
  // instructions.)
  auto each_run = [&](auto f) {
    const int held = std::min(runs, kEvictRuns);
    uint32_t next = keys[0];
    for (int i = 0; i < held; ++i) {
      const uint32_t x = next;
      next = keys[64 * std::min(i + 1, held - 1)];
      f(p0 + 64 * i, x);
    }
    for (int i = kEvictRuns; i < runs; ++i) f(p0 + 64 * i, order_of(w[std::min(p0 + 64 * i + lane, len - 1)]));
  };
  // Sum over the waves before this one, and over all
  struct Sums {
    uint32_t before, all;
  };
  auto sums_of = [&](int which) {
    Sums r = {0, 0};
#pragma unroll
    for (int i = 0; i < kWaves; i += 4) {
      const u32x4 x = *(const u32x4*)&s_count[which][i];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t n = (uint32_t)uniform((int)x[e]);
        r.before += i + e < wave ? n : 0;
        r.all += n;
      }
    }
    return r;
  };

  const bool any = gap > a.first;
  uint32_t need = (uint32_t)(gap - a.first), prefix = 0, alike_in_all = 0;
  for (int pass = 0; pass < 3 && any; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, top = pass == 1 ? 21 : 10;      // bits from `top` on are known
    const uint32_t mask = pass == 2 ? 1023 : 2047;
#pragma unroll
    for (int i = 0; i < kEvictBins * kEvictCopies / THREADS / 4; ++i) *(u32x4*)&s_bins[(i * THREADS + threadIdx.x) * 4] = u32x4{0, 0, 0, 0};
    __syncthreads();
    each_run([&](int p, uint32_t x) {
      if (p + lane < p1 && (pass == 0 || (x >> top) == (prefix >> top))) atomicAdd(&s_bins[((x >> shift) & mask) * kEvictCopies + (lane & 1)], 1u);
    });
    __syncthreads();
    // bins from above: the one in which the needed-th lies
    uint32_t n[kBinsEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kBinsEach; ++i) {
      const u32x2 x = *(const u32x2*)&s_bins[(kEvictBins - 1 - i - kBinsEach * (int)threadIdx.x) * kEvictCopies];
      n[i] = x[0] + x[1];
      sum += n[i];
    }
    const uint32_t scan = wave_scan(sum);
    if (lane == 63) s_count[0][wave] = scan;
    __syncthreads();
    uint32_t above = sums_of(0).before + scan - sum;
#pragma unroll
    for (int i = 0; i < kBinsEach; ++i) {
      if (above < need && above + n[i] >= need) {
        s_prefix = prefix | (uint32_t)(kEvictBins - 1 - i - kBinsEach * (int)threadIdx.x) << shift;
        s_need = need - above;
        s_alike = n[i];
      }
      above += n[i];
    }
    __syncthreads();
    prefix = s_prefix;
    need = s_need;
    alike_in_all = s_alike;
    if (alike_in_all == need) break;
  }
  // Stays: above the threshold, or among the first `need` that are alike with it (or all of them: all whose known bits are).  Bit per position of a run.
  const bool all_alike = alike_in_all == need;
  uint32_t rank = 0;      // of those alike, in front of the wave
  if (any && !all_alike) {
    uint32_t here = 0;
    each_run([&](int p, uint32_t x) { here += p + lane < p1 && x == prefix ? 1 : 0; });
    here = wave_scan(here);
    if (lane == 63) s_count[1][wave] = here;
    __syncthreads();
    rank = sums_of(1).before;
  }
  const uint32_t alike_before = rank;
  auto lanes_before = [](uint64_t set) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(set >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)set, 0)); };
  // (of the lane; by all lanes of a wave)
  auto stays_of = [&](int p, uint32_t x) {
    const bool in = p + lane < p1 && any;
    if (all_alike) return in && x >= prefix;
    const uint64_t alike = __ballot(in && x == prefix);
    const bool stays = in && (x > prefix || (x == prefix && rank + lanes_before(alike) < need));
    rank += __popcll(alike);
    return stays;
  };
  // Counts of the lane: what stays, in front of the gap's end, and between it and row `keep`
  uint32_t stay = 0, stay_below = 0, stay_near = 0;
  each_run([&](int p, uint32_t x) {
    const uint32_t one = stays_of(p, x) ? 1 : 0;
    stay += one;
    stay_below += p + lane < gap ? one : 0;
    stay_near += p + lane < a.keep ? one : 0;
  });
  stay = wave_scan(stay), stay_below = wave_scan(stay_below), stay_near = wave_scan(stay_near);
  if (lane == 63) s_count[2][wave] = std::clamp(gap - p0, 0, p1 - p0) - stay_below, s_count[3][wave] = stay - stay_below, s_count[4][wave] = stay_near - stay_below;
  __syncthreads();
  const Sums frees = sums_of(2);
  uint32_t free_at = frees.before, mover_at = sums_of(3).before;
  rank = alike_before;
  each_run([&](int p, uint32_t x) {
    const bool stays = stays_of(p, x), below = p + lane < gap;
    if (p < gap) {
      const bool is_free = !stays && below && p + lane < p1;
      const uint64_t set = __ballot(is_free);
      if (is_free) mv.to[free_at + lanes_before(set)] = p + lane;
      if (kept && stays && below) kept[p + lane] = p + lane;
      free_at += __popcll(set);
    }
    if (p + 64 > gap) {
      const bool moves = stays && !below;
      const uint64_t set = __ballot(moves);
      if (moves) mv.from[mover_at + lanes_before(set)] = p + lane;
      mover_at += __popcll(set);
    }
  });
  if (threadIdx.x == 0) {
    *mv.n = (int)frees.all;
    *mv.near = (int)sums_of(4).all;
    if (h == 0) a.new_lens[b] = a.keep;
  }
  if (kept) {
    for (int d = threadIdx.x; d < a.first; d += THREADS) kept[d] = d;
    for (int d = gap + threadIdx.x; d < a.keep; d += THREADS) kept[d] = d + len - a.keep;
    __threadfence_block();
    __syncthreads();
    constexpr int kAtOnce = 8;
    const int n = (int)frees.all;
    for (int i = threadIdx.x; i < n; i += kAtOnce * THREADS) {
      int place[kAtOnce], source[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) place[k] = mv.to[std::min(i + k * THREADS, n - 1)], source[k] = mv.from[std::min(i + k * THREADS, n - 1)];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
        if (i + k * THREADS < n) kept[place[k]] = source[k];
    }
  }
}

// Rows move by 16 lanes each: 16 bytes of the key and the value a lane; with 4 bits four lanes have those and one the exponents
constexpr int kMoveThreads = 512, kMoveRows = kMoveThreads / 16, kMoveAtOnce = 8;

template <bool MX4>
struct RowMover {
  const EvictArgs& a;
  int b, h, l16;
  int64_t weights;
  u32x4 x;
  float w;
  __device__ __forceinline__ int64_t at(int row) const {
    const PagedArgs& c = a.cache;
    const int64_t page = c.table[(int64_t)b * c.table_stride + (row >> c.page_shift)];
    return ((page * c.H_kv + h) << c.page_shift) + (row & ((1 << c.page_shift) - 1));
  }
  __device__ __forceinline__ void take(int row) {
    const int64_t r = at(row);
    if constexpr (MX4) {
      if (l16 < 4) x = *((const u32x4*)((l16 < 2 ? a.cache.k_pages : a.cache.v_pages) + r * kMxRowBytes) + (l16 & 1));
      if (l16 == 4) x[0] = *(const uint32_t*)(a.scales + r * kMxScaleBytes);
    } else {
      x = *((const u32x4*)((l16 < 8 ? a.cache.k_pages : a.cache.v_pages) + r * kRowBytes) + (l16 & 7));
    }
    if (l16 == 15) w = a.weights[weights + row];
  }
  __device__ __forceinline__ void put(int row) const {
    const int64_t r = at(row);
    if constexpr (MX4) {
      if (l16 < 4) *((u32x4*)((l16 < 2 ? a.cache.k_pages : a.cache.v_pages) + r * kMxRowBytes) + (l16 & 1)) = x;
      if (l16 == 4) *(uint32_t*)(a.scales + r * kMxScaleBytes) = x[0];
    } else {
      *((u32x4*)((l16 < 8 ? a.cache.k_pages : a.cache.v_pages) + r * kRowBytes) + (l16 & 7)) = x;
    }
    if (l16 == 15) a.weights[weights + row] = w;
  }
};
// The free places are filled, and the last rows go to the end.  Sources of the moves lie behind all places that they fill, so moves do not
// meet; those in front of row `keep` lie where the last rows go, and move first.  Where the last rows do not go over themselves the workgroups of a head
// take a part of that region each; else one of them takes all of it, and a batch is read before it is written.
// (Measured: 512 heads, a quarter of which move 256 + up to 256 rows in 16 bits, 25 MB, 15 us; 32 heads of 1374 + up to 4000 rows in 4 bits 22 to 26 us: chains of
// counts, places, pages and rows, each known when the one before has come.)
template <bool MX4>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(const EvictArgs a) {
  const int bh = blockIdx.x, b = bh / a.cache.H_kv, parts = gridDim.y, part = blockIdx.y;
  const int row0 = threadIdx.x >> 4;
  const Moves mv = moves_of(a, bh);
  const int n = *mv.n, near = *mv.near;
  if (n < 0) return;
  const RowMover<MX4> r = {a, b, bh - b * a.cache.H_kv, (int)(threadIdx.x & 15), (int64_t)bh * a.columns, {}, 0.f};
  const int gap = a.keep - a.last, shift = evict_length(a, b) - a.keep;
  const bool apart = shift >= a.last;
  const int each = apart ? (a.last + parts - 1) / parts : part == 0 ? a.last : 0;
  const int d0 = gap + (apart ? std::min(part * each, a.last) : 0), d1 = std::min(d0 + each, a.keep);
  // moves [i0, i1) whose source is in [lo, hi)
  auto fill = [&](int i0, int i1, int lo, int hi) {
    for (int i = i0; i < i1; i += kMoveRows * kMoveAtOnce) {
      RowMover<MX4> m[kMoveAtOnce] = {r, r, r, r, r, r, r, r};
      int source[kMoveAtOnce], place[kMoveAtOnce];
#pragma unroll
      for (int k = 0; k < kMoveAtOnce; ++k) {
        const int at = std::min(i + k * kMoveRows + row0, i1 - 1);
        source[k] = mv.from[at];
        place[k] = mv.to[at];
        if (i + k * kMoveRows + row0 >= i1 || source[k] < lo || source[k] >= hi) source[k] = -1;
      }
#pragma unroll
      for (int k = 0; k < kMoveAtOnce; ++k)
        if (source[k] >= 0) m[k].take(source[k]);
#pragma unroll
      for (int k = 0; k < kMoveAtOnce; ++k)
        if (source[k] >= 0) m[k].put(place[k]);
    }
  };
  if (d0 < d1) {
    fill(0, near, d0, d1);
    __syncthreads();
    for (int d = d0; d < d1; d += kMoveRows * kMoveAtOnce) {
      RowMover<MX4> m[kMoveAtOnce] = {r, r, r, r, r, r, r, r};
#pragma unroll
      for (int k = 0; k < kMoveAtOnce; ++k)
        if (d + k * kMoveRows + row0 < d1) m[k].take(shift + d + k * kMoveRows + row0);
      if (!apart) __syncthreads();
#pragma unroll
      for (int k = 0; k < kMoveAtOnce; ++k)
        if (d + k * kMoveRows + row0 < d1) m[k].put(d + k * kMoveRows + row0);
      if (!apart) __syncthreads();
    }
  }
  const int share = ((n - near + parts - 1) / parts + 7) / 8 * 8;
  const int i0 = std::min(near + part * share, n);
  fill(i0, std::min(i0 + share, n), 0, INT32_MAX);
}

template <bool MX4, bool CAUSAL>
void start_weigh(const WeighArgs& a, hipStream_t stream) {
  // Rows a sequence, on average: up to 64 stay in registers for every item of their head.
  const int64_t mean = a.n_tokens * a.group / a.cache.n_seqs;
  const dim3 block(64 * kWeighWaves);
  if (mean > 64)
    hipLaunchKernelGGL((weigh_many_kernel<MX4, CAUSAL>), dim3(1024), block, 0, stream, a);
  else if (mean > 16)
    hipLaunchKernelGGL((weigh_few_kernel<MX4, 4, CAUSAL>), dim3(256 * few_waves(4)), block, 0, stream, a);
  else
    hipLaunchKernelGGL((weigh_few_kernel<MX4, 1, CAUSAL>), dim3(256 * few_waves(1)), block, 0, stream, a);
}
template <bool MX4>
void start_moves(const EvictArgs& a, hipStream_t stream) {
  const unsigned heads = (unsigned)(a.cache.n_seqs * a.cache.H_kv);
  const unsigned parts = std::clamp(1024u / heads, 1u, 32u);
  hipLaunchKernelGGL(evict_move_kernel<MX4>, dim3(heads, parts), dim3(kMoveThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_cache_weigh(const WeighArgs& args, hipStream_t stream) {
  WeighArgs a = args;
  a.group_magic = (uint32_t)((((uint64_t)1 << 32) + a.group - 1) / a.group);
  if (a.scales)
    a.causal ? start_weigh<true, true>(a, stream) : start_weigh<true, false>(a, stream);
  else
    a.causal ? start_weigh<false, true>(a, stream) : start_weigh<false, false>(a, stream);
  return hipGetLastError();
}

int64_t cache_evict_workspace(int n_seqs, int H_kv, int keep) {
  return ((int64_t)n_seqs * H_kv * (2 + 2 * (int64_t)keep) * 4 + 255) / 256 * 256;
}

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t stream) {
  const dim3 heads((unsigned)(a.cache.n_seqs * a.cache.H_kv));
  // By what fits the LDS of a workgroup, of the rows that a sequence can have: the host knows the room in the page table alone.  256 / 1024 threads, selection and
  // moves, us: 64 sequences of 8 heads 4352 -> 4096 rows 35.6 / 42.8 (the workgroup with the larger LDS is alone on its CU), 1100 -> 1024 19.9 / 28.0, 8300 -> 8192 47.4 / 49.1,
  // 16 700 -> 16 384 103 / 80; 2 of 16 heads 4352 -> 4096 23.3 / 20.8, 27 480 -> 13 740 119 / 46.  So many short heads in a table with room for long ones lose
  // 7 or 8 us, and few heads of 8000 rows in a table with no more room 9 (33.4 / 24.4).
  if ((int64_t)a.cache.table_stride << a.cache.page_shift <= 256 * kEvictRuns)
    hipLaunchKernelGGL(evict_select_kernel<256>, heads, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(evict_select_kernel<1024>, heads, dim3(1024), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.scales ? start_moves<true>(a, stream) : start_moves<false>(a, stream);
  return hipGetLastError();
}

}  // namespace httm
