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
  const int64_t each = total / shares, more = total - each * shares;
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
  __device__ __forceinline__ void request(const WeighArgs& a, int b, int len, int h, int j0, int l16, int grp) {
    const PagedArgs& c = a.cache;
    const auto* table = (const __attribute__((address_space(4))) int32_t*)(c.table + (int64_t)b * c.table_stride);
    there = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int row = j0 + 16 * t;
      const int page = row < len ? table[row >> c.page_shift] : -1;     // (no length is beyond the table)
      const bool ok = page >= 0 && page < c.n_pages;
      there |= ok ? 1u << t : 0u;
      const int64_t first = (((int64_t)(ok ? page : 0) * c.H_kv + h) << c.page_shift) + (row & ((1 << c.page_shift) - 1));
      const int n = ok ? std::min(len - row, 16) : 0;
      auto rows = [&](const void* p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc((char*)p + first * bytes, 0, n * bytes, kRawBufferWord3); };
      if constexpr (MX4) {
        const u32x2 codes = __builtin_amdgcn_raw_buffer_load_b64(rows(c.k_pages, kMxRowBytes), l16 * kMxRowBytes + grp * 8, 0, 0);
        const uint32_t e = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(rows(c.scales, kMxScaleBytes), l16 * kMxScaleBytes + 2 * (grp >> 1), 0, 0);
        x[t][0] = u32x4{codes[0], codes[1], e, 0};
      } else {
#pragma unroll
        for (int e = 0; e < 2; ++e) x[t][e] = __builtin_amdgcn_raw_buffer_load_b128(rows(c.k_pages, kRowBytes), l16 * kRowBytes + grp * 32 + e * 16, 0, 0);
      }
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
// -lse of row r in base 2; minus infinity for a row that adds nothing: behind the last, or one that saw no key
__device__ __forceinline__ float load_lse(const WeighArgs& a, const WeighSeq& s, int h, int r, int n_rows) {
  const int row = std::min(r, n_rows - 1), i = token_of(a, row);
  const float x = a.lse[(int64_t)(s.first + i) * (a.cache.H_kv * a.group) + h * a.group + row - i * a.group];
  return r >= n_rows || x == -__builtin_inff() ? -__builtin_inff() : -x * kLog2e;
}
// What a tile of rows gives 64 keys.  `sees` (MASKED): keys that a row sees, from the first of the 64 on
template <bool MASKED>
__device__ __forceinline__ void add_tile(float (&sum)[4], const bf16x8 (&k)[4][2], const bf16x8 (&q)[2], const f32x4& lse, float scale_log2,
                                         const int (&sees)[4], int l16) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    f32x4 x = mfma16(q[0], k[t][0], f32x4{0.f, 0.f, 0.f, 0.f});
    x = mfma16(q[1], k[t][1], x);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float p = __builtin_amdgcn_exp2f(fmaf(x[e], scale_log2, lse[e]));
      if (MASKED && 16 * t + l16 >= sees[e]) p = 0.f;
      sum[t] += p;
    }
  }
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

// Few rows: NT tiles of them stay in registers
template <bool MX4, int NT, bool CAUSAL>
__global__ __launch_bounds__(64 * kWeighWaves) void weigh_few_kernel(const WeighArgs a) {
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
    int64_t left;      // items of the sequence that the share still has, this one among them
    int b, h, chunk;
  };
  // the first item at or behind sequence b that the share has
  auto start = [&](Place& p) {
    for (; p.b < a.cache.n_seqs && share.begin < share.end; ++p.b) {
      p.s = weigh_seq<kFront, 1>(a, p.b);
      const int64_t all = (int64_t)p.s.items * H, from = share.at <= share.begin ? 0 : (share.at - share.begin + p.s.cost - 1) / p.s.cost;
      p.left = std::min<int64_t>(all, (share.end - share.begin + p.s.cost - 1) / p.s.cost) - from;
      share.begin += all * p.s.cost;
      if (p.left <= 0) continue;
      p.h = uniform((int)(from / p.s.items));
      p.chunk = uniform((int)(from - (int64_t)p.h * p.s.items));
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
  auto old_weight = [&](const Place& p) {
    const int j = p.chunk * kWeighKeys + lane;
    return j < p.s.len - p.s.n ? *weight_at(p) : 0.f;
  };

  Place p;
  p.b = share.b;
  if (!start(p)) return;
  KeysOnTheirWay<MX4> keys;
  keys.request(a, p.b, p.s.len, p.h, p.chunk * kWeighKeys, l16, grp);
  float old = old_weight(p);
  bf16x8 q[NT][2];
  f32x4 lse[NT];
  int of_b = -1, of_h = -1;      // whose rows q holds
  while (true) {
    const Place here = p;
    const int j0 = here.chunk * kWeighKeys, n_rows = here.s.n * a.group, before = here.s.len - here.s.n;
    const KeysOnTheirWay<MX4> now = keys;
    const float was = old;
    const bool more = next(p);
    if (more) {
      keys.request(a, p.b, p.s.len, p.h, p.chunk * kWeighKeys, l16, grp);
      old = old_weight(p);
    }
    bf16x8 k[4][2];
    now.take(k);
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    const bool stays = n_rows <= 16 * NT;
    for (int r0 = 0; r0 < n_rows; r0 += 16 * NT) {
      if (!stays || of_b != here.b || of_h != here.h) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          load_queries(q[i], a, here.s, here.h, r0 + 16 * i + l16, n_rows, grp);
#pragma unroll
          for (int e = 0; e < 4; ++e) lse[i][e] = load_lse(a, here.s, here.h, r0 + 16 * i + 4 * grp + e, n_rows);
        }
        of_b = here.b, of_h = here.h;
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
        add_tile<true>(sum, k, q[i], lse[i], scale_log2, sees, l16);
      }
    }
    float mine = key_of_lane(sum, grp);
    if (!((now.there >> grp) & 1)) mine = 0.f;
    if (j0 + lane < here.s.len) *weight_at(here) = j0 + lane < before ? fmaf(a.decay, was, mine) : mine;
    if (!more) return;
  }
}

// Many rows: the waves of a workgroup take tiles of them in turn.  Their lse lie in the LDS, a run of rows at a time.
template <bool MX4, bool CAUSAL>
__global__ __launch_bounds__(64 * kWeighWaves) void weigh_many_kernel(const WeighArgs a) {
  constexpr int kFront = 4, kRun = 1024;
  __shared__ __attribute__((aligned(16))) float s_lse[kRun];
  __shared__ float s_sum[kWeighWaves][kWeighKeys];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), l16 = lane & 15, grp = lane >> 4;
  const int H = a.cache.H_kv;
  const int id = (int)((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3));
  WeighShare share;
  if (!find_weigh_share<kFront, kWeighWaves>(a, id, gridDim.x, lane, share)) return;
  const float scale_log2 = a.scale * kLog2e;
  for (int b = share.b; b < a.cache.n_seqs && share.begin < share.end; ++b) {
    const WeighSeq s = weigh_seq<kFront, kWeighWaves>(a, b);
    int64_t item = share.at <= share.begin ? 0 : (share.at - share.begin + s.cost - 1) / s.cost;
    const int64_t stop = std::min<int64_t>((int64_t)s.items * H, (share.end - share.begin + s.cost - 1) / s.cost);
    share.begin += (int64_t)s.items * H * s.cost;
    if (item >= stop) continue;
    const int n_rows = s.n * a.group, before = s.len - s.n;
    int h = uniform((int)(item / s.items)), chunk = uniform((int)(item - (int64_t)h * s.items));
    int run_of_h = -1;
    bool dead = false;      // whether a row of the run adds nothing
    for (; item < stop; ++item) {
      const int j0 = chunk * kWeighKeys;
      KeysOnTheirWay<MX4> keys;
      keys.request(a, b, s.len, h, j0, l16, grp);
      float* weight = a.weights + ((int64_t)b * H + h) * a.columns + j0 + lane;
      const float was = wave == 0 && j0 + lane < before ? *weight : 0.f;
      bf16x8 k[4][2];
      keys.take(k);
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
      // rows in front of the first that sees one of the keys are left out
      const int unseen = CAUSAL && j0 > before ? std::min((j0 - before) * a.group, n_rows) / 16 : 0;
      for (int run = unseen * 16 / kRun * kRun; run < n_rows; run += kRun) {
        if (run_of_h != h || n_rows > kRun) {
          __syncthreads();
          bool none = false;
          for (int i = threadIdx.x; i < kRun && run + i < (n_rows + 15) / 16 * 16; i += 64 * kWeighWaves) {
            s_lse[i] = load_lse(a, s, h, run + i, n_rows);
            none |= s_lse[i] == -__builtin_inff() && run + i < n_rows;
          }
          dead = __syncthreads_or(none) != 0;
          run_of_h = h;
        }
        const int t1 = (std::min(run + kRun, n_rows) + 15) / 16;
        int tile = std::max(run / 16, unseen) + wave;
        if (tile >= t1) continue;
        bf16x8 q[2];
        load_queries(q, a, s, h, 16 * tile + l16, n_rows, grp);
        for (; tile < t1; tile += kWeighWaves) {
          bf16x8 ahead[2];
          load_queries(ahead, a, s, h, 16 * (tile + kWeighWaves) + l16, n_rows, grp);
          const f32x4 lse = *(const f32x4*)(s_lse + 16 * tile - run + 4 * grp);
          int sees[4] = {0, 0, 0, 0};
          if (dead || 16 * tile + 16 > n_rows || (CAUSAL && before + token_of(a, 16 * tile) + 1 < std::min(j0 + kWeighKeys, s.len))) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sees[e] = lse[e] == -__builtin_inff() ? 0 : CAUSAL ? before + token_of(a, 16 * tile + 4 * grp + e) + 1 - j0 : kWeighKeys;
            add_tile<true>(sum, k, q, lse, scale_log2, sees, l16);
          } else {
            add_tile<false>(sum, k, q, lse, scale_log2, sees, l16);
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) q[e] = ahead[e];
        }
      }
      s_sum[wave][lane] = key_of_lane(sum, grp);
      __syncthreads();
      if (wave == 0 && j0 + lane < s.len) {
        float mine = 0.f;
#pragma unroll
        for (int i = 0; i < kWeighWaves; ++i) mine += s_sum[i][lane];
        if (!((keys.there >> grp) & 1)) mine = 0.f;
        *weight = j0 + lane < before ? fmaf(a.decay, was, mine) : mine;
      }
      __syncthreads();
      if (++chunk == s.items) chunk = 0, ++h;
    }
  }
}

// ---- eviction --------------------------------------------------------------------------------------------------

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;

// In the order of the weights: NaN is below everything, zeros are alike
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  return w != w ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Moves of a key head of a sequence: how many, where to, where from
struct Moves {
  int32_t* n;
  int32_t* to;
  int32_t* from;
};
__device__ __forceinline__ Moves moves_of(const EvictArgs& a, int bh) {
  int32_t* n = (int32_t*)a.workspace + (int64_t)bh * (1 + 2 * (int64_t)a.keep);
  return {n, n + 1, n + 1 + a.keep};
}
__device__ __forceinline__ int evict_length(const EvictArgs& a, int b) {
  return std::clamp(a.seq_lens[b], 0, a.cache.table_stride << a.cache.page_shift);
}
__device__ __forceinline__ int64_t cache_row(const PagedArgs& c, int b, int h, int row) {
  const int64_t page = c.table[(int64_t)b * c.table_stride + (row >> c.page_shift)];
  return ((page * c.H_kv + h) << c.page_shift) + (row & ((1 << c.page_shift) - 1));
}

// What stays of a key head of a sequence, and what has to move: one workgroup.  The threshold comes from four passes over 8 bits each of the weights' order,
// every wave of the workgroup with a part of the positions and counts of its own, so that the places of those alike and of the moves are
// sums over the waves before.
__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(const EvictArgs a) {
  __shared__ uint32_t s_hist[kEvictWaves][256];
  __shared__ uint32_t s_count[3][kEvictWaves];
  __shared__ uint32_t s_prefix, s_need, s_hole;
  const int b = blockIdx.x / a.cache.H_kv, h = blockIdx.x - b * a.cache.H_kv;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int len = evict_length(a, b);
  const Moves mv = moves_of(a, blockIdx.x);
  int32_t* kept = a.kept ? a.kept + (int64_t)blockIdx.x * a.keep : nullptr;
  if (threadIdx.x == 0) s_hole = 0;
  __syncthreads();
  const int32_t* table = a.cache.table + (int64_t)b * a.cache.table_stride;
  for (int i = threadIdx.x; i < (len + (1 << a.cache.page_shift) - 1) >> a.cache.page_shift; i += kEvictThreads)
    if (table[i] < 0 || table[i] >= a.cache.n_pages) s_hole = 1;
  __syncthreads();
  const bool hole = s_hole != 0;
  if (hole || len <= a.keep) {
    if (threadIdx.x == 0) {
      *mv.n = -1;
      if (h == 0) a.new_lens[b] = len;
    }
    if (kept)
      for (int d = threadIdx.x; d < a.keep; d += kEvictThreads) kept[d] = !hole && d < len ? d : -1;
    return;
  }
  const float* w = a.weights + (int64_t)blockIdx.x * a.columns;
  const int from = a.first, to = len - a.last, gap = a.keep - a.last;
  // a wave's part, in runs of 64 positions
  const int part = ((to - from + kEvictThreads - 1) / kEvictThreads) * 64;
  const int p0 = std::min(from + wave * part, to), p1 = std::min(p0 + part, to);

  uint32_t need = (uint32_t)(a.keep - a.first - a.last), prefix = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < kEvictWaves * 256; i += kEvictThreads) (&s_hist[0][0])[i] = 0;
    __syncthreads();
    for (int p = p0 + lane; p < p1; p += 64) {
      const uint32_t x = order_of(w[p]);
      if (shift == 24 || (x >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s_hist[wave][(x >> shift) & 255], 1u);
    }
    __syncthreads();
    if (threadIdx.x < 256) {
      uint32_t n = 0;
      for (int i = 0; i < kEvictWaves; ++i) n += s_hist[i][threadIdx.x];
      s_hist[0][threadIdx.x] = n;
    }
    __syncthreads();
    if (wave == 0) {
      // values from above: the bin in which the needed-th lies
      uint32_t n[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += n[i] = s_hist[0][255 - (4 * lane + i)];
      uint32_t scan = sum;
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t v = __shfl_up(scan, d);
        scan += lane >= d ? v : 0;
      }
      uint32_t above = scan - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (above < need && above + n[i] >= need) {
          s_prefix = prefix | (uint32_t)(255 - (4 * lane + i)) << shift;
          s_need = need - above;
        }
        above += n[i];
      }
    }
    if (need == 0) break;
    __syncthreads();
    prefix = s_prefix;
    need = s_need;
    __syncthreads();
  }
  // stays: above the threshold, or among the first `need` that are alike with it
  const bool any = a.keep - a.first - a.last > 0;
  auto ballot_of = [&](int p, uint64_t& above, uint64_t& alike) {
    const uint32_t x = p < p1 ? order_of(w[p]) : 0u;
    above = __ballot(p < p1 && any && x > prefix);
    alike = __ballot(p < p1 && any && x == prefix);
  };
  auto before_me = [&](int which, uint32_t mine) {
    if (lane == 0) s_count[which][wave] = mine;
    __syncthreads();
    uint32_t n = 0;
    for (int i = 0; i < wave; ++i) n += s_count[which][i];
    return (uint32_t)uniform((int)n);
  };
  uint32_t alike_here = 0;
  for (int p = p0; p < p1; p += 64) {
    uint64_t above, alike;
    ballot_of(p + lane, above, alike);
    alike_here += __popcll(alike);
  }
  const uint32_t alike_before = before_me(0, alike_here);
  auto stays_of = [&](int p, uint32_t& rank) {      // of a run; rank: of the first that is alike
    uint64_t above, alike;
    ballot_of(p + lane, above, alike);
    const uint32_t mine = rank + __popcll(alike & ((1ull << lane) - 1));
    rank += __popcll(alike);
    return above | __ballot(((alike >> lane) & 1) && mine < need);
  };
  uint32_t holes = 0, movers = 0, rank = alike_before;
  for (int p = p0; p < p1; p += 64) {
    const uint64_t stays = stays_of(p, rank), below = __ballot(p + lane < gap), in = __ballot(p + lane < p1);
    holes += __popcll(~stays & below & in);
    movers += __popcll(stays & ~below);
  }
  uint32_t hole_at = before_me(1, holes), mover_at = before_me(2, movers);
  rank = alike_before;
  for (int p = p0; p < p1; p += 64) {
    const uint64_t stays = stays_of(p, rank), below = __ballot(p + lane < gap), in = __ballot(p + lane < p1);
    const uint64_t h_set = ~stays & below & in, m_set = stays & ~below, me = 1ull << lane, lower = me - 1;
    if (h_set & me) mv.to[hole_at + __popcll(h_set & lower)] = p + lane;
    if (m_set & me) mv.from[mover_at + __popcll(m_set & lower)] = p + lane;
    if (kept && (stays & below & me)) kept[p + lane] = p + lane;
    hole_at += __popcll(h_set);
    mover_at += __popcll(m_set);
  }
  if (threadIdx.x == kEvictThreads - 1) *mv.n = (int)hole_at;
  if (h == 0 && threadIdx.x == 0) a.new_lens[b] = a.keep;
  if (kept) {
    for (int d = threadIdx.x; d < a.keep; d += kEvictThreads)
      if (d < from || d >= gap) kept[d] = d < from ? d : d + len - a.keep;
    __threadfence_block();
    __syncthreads();
    uint32_t n = 0;
    for (int i = 0; i < kEvictWaves; ++i) n += s_count[1][i];
    for (int i = threadIdx.x; i < (int)n; i += kEvictThreads) kept[mv.to[i]] = mv.from[i];
  }
}

// A row of keys, one of values and its weight on their way, by 16 lanes
template <bool MX4>
struct RowInLane {
  u32x4 x;
  float w;
  __device__ __forceinline__ void take(const EvictArgs& a, int b, int h, int64_t weights, int row, int l16) {
    const int64_t at = cache_row(a.cache, b, h, row);
    if constexpr (MX4) {
      if (l16 < 4) x = *((const u32x4*)((l16 < 2 ? a.cache.k_pages : a.cache.v_pages) + at * kMxRowBytes) + (l16 & 1));
      if (l16 == 4) x[0] = *(const uint32_t*)(a.cache.scales + at * kMxScaleBytes);
    } else {
      x = *((const u32x4*)((l16 < 8 ? a.cache.k_pages : a.cache.v_pages) + at * kRowBytes) + (l16 & 7));
    }
    if (l16 == 15) w = a.weights[weights + row];
  }
  __device__ __forceinline__ void put(const EvictArgs& a, int b, int h, int64_t weights, int row, int l16) const {
    const int64_t at = cache_row(a.cache, b, h, row);
    if constexpr (MX4) {
      if (l16 < 4) *((u32x4*)((l16 < 2 ? a.cache.k_pages : a.cache.v_pages) + at * kMxRowBytes) + (l16 & 1)) = x;
      if (l16 == 4) *(uint32_t*)(a.cache.scales + at * kMxScaleBytes) = x[0];
    } else {
      *((u32x4*)((l16 < 8 ? a.cache.k_pages : a.cache.v_pages) + at * kRowBytes) + (l16 & 7)) = x;
    }
    if (l16 == 15) a.weights[weights + row] = w;
  }
};

constexpr int kMoveThreads = 256, kMoveRows = kMoveThreads / 16;

// The places that are free are filled; sources lie behind all of them, so moves do not meet
template <bool MX4>
__global__ __launch_bounds__(kMoveThreads) void evict_fill_kernel(const EvictArgs a) {
  const int b = blockIdx.x / a.cache.H_kv, h = blockIdx.x - b * a.cache.H_kv, l16 = threadIdx.x & 15;
  const Moves mv = moves_of(a, blockIdx.x);
  const int64_t weights = (int64_t)blockIdx.x * a.columns;
  const int n = *mv.n;
  for (int i = blockIdx.y * kMoveRows + (threadIdx.x >> 4); i < n; i += gridDim.y * kMoveRows) {
    RowInLane<MX4> r;
    r.take(a, b, h, weights, mv.from[i], l16);
    r.put(a, b, h, weights, mv.to[i], l16);
  }
}
// The last rows go to the end, in order: towards the front, by one workgroup, which reads a batch before it writes it
template <bool MX4>
__global__ __launch_bounds__(kMoveThreads) void evict_tail_kernel(const EvictArgs a) {
  constexpr int kAtOnce = 8;
  const int b = blockIdx.x / a.cache.H_kv, h = blockIdx.x - b * a.cache.H_kv, l16 = threadIdx.x & 15;
  const int64_t weights = (int64_t)blockIdx.x * a.columns;
  if (*moves_of(a, blockIdx.x).n < 0) return;
  const int to = a.keep - a.last, from = evict_length(a, b) - a.last;
  for (int i0 = 0; i0 < a.last; i0 += kAtOnce * kMoveRows) {
    RowInLane<MX4> r[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = i0 + k * kMoveRows + (int)(threadIdx.x >> 4);
      if (i < a.last) r[k].take(a, b, h, weights, from + i, l16);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = i0 + k * kMoveRows + (int)(threadIdx.x >> 4);
      if (i < a.last) r[k].put(a, b, h, weights, to + i, l16);
    }
    __syncthreads();
  }
}

template <bool MX4, bool CAUSAL>
void start_weigh(const WeighArgs& a, hipStream_t stream) {
  const int64_t mean = a.n_tokens * a.group / a.cache.n_seqs;
  const dim3 block(64 * kWeighWaves);
  if (mean > 64)
    hipLaunchKernelGGL((weigh_many_kernel<MX4, CAUSAL>), dim3(1024), block, 0, stream, a);
  else if (mean > 16)
    hipLaunchKernelGGL((weigh_few_kernel<MX4, 4, CAUSAL>), dim3(1024), block, 0, stream, a);
  else
    hipLaunchKernelGGL((weigh_few_kernel<MX4, 1, CAUSAL>), dim3(1024), block, 0, stream, a);
}
template <bool MX4>
void start_moves(const EvictArgs& a, hipStream_t stream) {
  const unsigned heads = (unsigned)(a.cache.n_seqs * a.cache.H_kv);
  const unsigned parts = std::max(1u, std::min(64u, 2048u / heads));
  if (a.keep > a.first + a.last) hipLaunchKernelGGL(evict_fill_kernel<MX4>, dim3(heads, parts), dim3(kMoveThreads), 0, stream, a);
  if (a.last > 0) hipLaunchKernelGGL(evict_tail_kernel<MX4>, dim3(heads), dim3(kMoveThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_cache_weigh(const WeighArgs& args, hipStream_t stream) {
  WeighArgs a = args;
  a.group_magic = (uint32_t)((((uint64_t)1 << 32) + a.group - 1) / a.group);
  if (a.cache.scales)
    a.causal ? start_weigh<true, true>(a, stream) : start_weigh<true, false>(a, stream);
  else
    a.causal ? start_weigh<false, true>(a, stream) : start_weigh<false, false>(a, stream);
  return hipGetLastError();
}

int64_t cache_evict_workspace(int n_seqs, int H_kv, int keep) {
  return ((int64_t)n_seqs * H_kv * (1 + 2 * (int64_t)keep) * 4 + 255) / 256 * 256;
}

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)(a.cache.n_seqs * a.cache.H_kv)), dim3(kEvictThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.cache.scales ? start_moves<true>(a, stream) : start_moves<false>(a, stream);
  return hipGetLastError();
}

}  // namespace httm
