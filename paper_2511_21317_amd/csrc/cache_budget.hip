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
// The rows of a sequence and a key head are those of attention: r / group-th token, query head h * group + r % group.  A wave
// holds 64 keys as the A operands of S^T = K Q^T (v_mfma_f32_16x16x32_bf16) and goes over rows, 16 at a time: a lane has one row's scores of
// 4 of 16 keys, and adds what they come to up, key by key; the sum over the 16 lanes is taken once, at the end.
// Where sequences have few rows a wave goes over all of them; where they have many (SPLIT) the four waves of a
// workgroup share their 64 keys and take the rows in turn.  No sum depends on how the work falls: results are run-to-run identical.
//
// The work of a launch is a line: sequences, their key heads, the head's items of keys, every item as long as it takes to go over the rows.
// It is cut into equal shares, one per workgroup, which takes the items that begin in its share.

constexpr int kWeighWaves = 4;
constexpr int kWeighKeys = 64;      // of a wave
constexpr int kItemFront = 4;       // what an item costs besides its rows, in tiles of 16

struct WeighSeq {
  int first, n, len;
  int items;            // of a key head
  int cost;             // of an item
};
template <bool SPLIT>
__device__ __forceinline__ WeighSeq weigh_seq(const WeighArgs& a, int b) {
  constexpr int kItem = SPLIT ? kWeighKeys : kWeighKeys * kWeighWaves;
  WeighSeq s = {0, 0, 0, 0, 1};
  if (b >= a.cache.n_seqs) return s;
  const int T = (int)a.n_tokens;
  s.first = std::clamp(a.offsets[b], 0, T);
  s.n = std::clamp(a.offsets[b + 1], s.first, T) - s.first;
  s.len = std::clamp(a.seq_lens[b], 0, a.cache.table_stride << a.cache.page_shift);
  s.items = (s.len + kItem - 1) / kItem;
  const int tiles = (s.n * a.group + 15) / 16;
  s.cost = kItemFront + (SPLIT ? (tiles + kWeighWaves - 1) / kWeighWaves : tiles);
  return s;
}

template <bool MX4, bool SPLIT, bool CAUSAL>
__global__ __launch_bounds__(64 * kWeighWaves) void weigh_kernel(const WeighArgs a) {
  constexpr int kItem = SPLIT ? kWeighKeys : kWeighKeys * kWeighWaves;
  __shared__ float s_sum[kWeighWaves][kWeighKeys];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), l16 = lane & 15, grp = lane >> 4;
  const PagedArgs& c = a.cache;
  const int H = c.H_kv, H_q = H * a.group, n_seqs = c.n_seqs;

  // the share's positions [at, end), and the sequence that it begins in
  auto length = [&](int base) {
    const WeighSeq s = weigh_seq<SPLIT>(a, base + lane);
    return (int64_t)s.items * H * s.cost;
  };
  int64_t total = 0;
  for (int base = 0; base < n_seqs; base += 64) total += length(base);
  for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
  total = uniform64(total);
  const int64_t each = total / gridDim.x, more = total - each * gridDim.x;
  // (shares next to each other on one XCD: they read the same rows)
  const int id = (int)((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3));
  const int64_t at = each * id + std::min<int64_t>(id, more), end = at + each + (id < more ? 1 : 0);
  if (at >= end) return;
  int64_t begin = 0;       // of sequence b
  int b = 0;
  for (int base = 0; base < n_seqs; base += 64) {
    int64_t scan = length(base);
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t v = __shfl_up(scan, d);
      scan += lane >= d ? v : 0;
    }
    const uint64_t in = __ballot(begin + scan > at);
    if (in == 0) {
      begin += uniform64(__shfl(scan, 63));
      continue;
    }
    const int l = __builtin_ctzll(in);
    b = base + l;
    begin += l ? uniform64(__shfl(scan, l - 1)) : 0;
    break;
  }

  for (; b < n_seqs && begin < end; ++b) {
    const WeighSeq s = weigh_seq<SPLIT>(a, b);
    if (s.items == 0) continue;
    int64_t item = at <= begin ? 0 : (at - begin + s.cost - 1) / s.cost;
    const int64_t stop = std::min<int64_t>((int64_t)s.items * H, (end - begin + s.cost - 1) / s.cost);
    begin += (int64_t)s.items * H * s.cost;
    const int n_rows = s.n * a.group, tiles = (n_rows + 15) / 16, before = s.len - s.n;
    const int32_t* table = c.table + (int64_t)b * c.table_stride;
    for (; item < stop; ++item) {
      const int h = uniform((int)(item / s.items)), j0 = uniform((int)(item - (int64_t)h * s.items) * kItem + (SPLIT ? 0 : wave * kWeighKeys));
      if (!SPLIT && j0 >= s.len) continue;
      // keys: 16 channels of a row in a lane, in two operands
      bf16x8 k[4][2];
      uint32_t there = 0;
      {
        u32x2 codes[4];
        uint32_t exponents[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int row = j0 + 16 * t, index = row >> c.page_shift;
          const int page = row < s.len && index < c.table_stride ? table[index] : -1;
          const bool ok = page >= 0 && page < c.n_pages;
          there |= ok ? 1u << t : 0u;
          const int64_t first = (((int64_t)(ok ? page : 0) * H + h) << c.page_shift) + (row & ((1 << c.page_shift) - 1));
          const int n = ok ? std::min(s.len - row, 16) : 0;
          if constexpr (MX4) {
            codes[t] = __builtin_amdgcn_raw_buffer_load_b64(
                __builtin_amdgcn_make_buffer_rsrc(c.k_pages + first * kMxRowBytes, 0, n * kMxRowBytes, kRawBufferWord3), l16 * kMxRowBytes + grp * 8, 0, 0);
            exponents[t] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(
                __builtin_amdgcn_make_buffer_rsrc(c.scales + first * kMxScaleBytes, 0, n * kMxScaleBytes, kRawBufferWord3),
                l16 * kMxScaleBytes + 2 * (grp >> 1), 0, 0);
          } else {
            const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc(c.k_pages + first * kRowBytes, 0, n * kRowBytes, kRawBufferWord3);
#pragma unroll
            for (int e = 0; e < 2; ++e)
              k[t][e] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rows, l16 * kRowBytes + grp * 32 + e * 16, 0, 0));
          }
        }
        if constexpr (MX4)
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) k[t][e] = __builtin_bit_cast(bf16x8, mx4_values(codes[t][e], __uint_as_float(exponents[t] << 23)));
      }
      f32x4 sum[4] = {};
      // rows in front of the first that sees one of the keys are left out
      const int unseen = CAUSAL && j0 > before ? std::min((j0 - before) * a.group, n_rows) / 16 : 0;
      for (int tile = unseen + (SPLIT ? wave : 0); tile < tiles; tile += SPLIT ? kWeighWaves : 1) {
        const int r = std::min(16 * tile + l16, n_rows - 1);
        const int i = r / a.group, head = h * a.group + (r - i * a.group);
        const int64_t token = s.first + i;
        const char* q = a.q.data + (token * a.q.token_stride + head * a.q.head_stride) * 2;
        bf16x8 qf[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) qf[e] = *(const bf16x8*)(q + grp * 32 + e * 16);
        const float lse = a.lse[token * H_q + head];
        // keys that the lane's row sees, from j0 on: none behind the last row, and where it saw no key at all
        int sees = CAUSAL ? std::clamp(before + i + 1, 0, s.len) - j0 : s.len - j0;
        if (16 * tile + l16 >= n_rows || lse == -__builtin_inff()) sees = 0;
        const bool masked = __ballot(sees < std::min(kWeighKeys, s.len - j0)) != 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          f32x4 x = mfma16(k[t][0], qf[0], f32x4{0.f, 0.f, 0.f, 0.f});
          x = mfma16(k[t][1], qf[1], x);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // (the difference in one rounding: it is small where the weight counts, and then scaled)
            float p = __builtin_amdgcn_exp2f(fmaf(x[e], a.scale, -lse) * 1.4426950408889634f);
            if (masked && 16 * t + 4 * grp + e >= sees) p = 0.f;
            sum[t][e] += p;
          }
        }
      }
      // over the 16 lanes of a group: each is left with one key, 16 * (l16 >> 2) + 4 * grp + (l16 & 3)
      float mine = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = sum[t][e];
          for (int d = 1; d < 16; d <<= 1) x += __shfl_xor(x, d);
          if (l16 == 4 * t + e) mine = x;
        }
      const int in = 16 * (l16 >> 2) + 4 * grp + (l16 & 3);
      if constexpr (SPLIT) {
        s_sum[wave][in] = mine;
        __syncthreads();
        mine = 0.f;
#pragma unroll
        for (int i = 0; i < kWeighWaves; ++i) mine += s_sum[i][in];
        __syncthreads();
        if (wave != 0) continue;
      }
      const int j = j0 + in;
      if (j >= s.len) continue;
      if (!((there >> (in >> 4)) & 1)) mine = 0.f;
      float* w = a.weights + ((int64_t)b * H + h) * a.columns + j;
      *w = j < before ? fmaf(a.decay, *w, mine) : mine;
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

template <bool MX4, bool SPLIT>
void start_weigh(const WeighArgs& a, int shares, hipStream_t stream) {
  if (a.causal)
    hipLaunchKernelGGL((weigh_kernel<MX4, SPLIT, true>), dim3(shares), dim3(64 * kWeighWaves), 0, stream, a);
  else
    hipLaunchKernelGGL((weigh_kernel<MX4, SPLIT, false>), dim3(shares), dim3(64 * kWeighWaves), 0, stream, a);
}
template <bool MX4>
void start_moves(const EvictArgs& a, hipStream_t stream) {
  const unsigned heads = (unsigned)(a.cache.n_seqs * a.cache.H_kv);
  const unsigned parts = std::max(1u, std::min(64u, 2048u / heads));
  if (a.keep > a.first + a.last) hipLaunchKernelGGL(evict_fill_kernel<MX4>, dim3(heads, parts), dim3(kMoveThreads), 0, stream, a);
  if (a.last > 0) hipLaunchKernelGGL(evict_tail_kernel<MX4>, dim3(heads), dim3(kMoveThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_cache_weigh(const WeighArgs& a, hipStream_t stream) {
  const int64_t rows = a.n_tokens * a.group;
  const bool split = rows > 64 * (int64_t)a.cache.n_seqs;
  const int shares = 256 * 6;
  if (a.cache.scales)
    split ? start_weigh<true, true>(a, shares, stream) : start_weigh<true, false>(a, shares, stream);
  else
    split ? start_weigh<false, true>(a, shares, stream) : start_weigh<false, false>(a, shares, stream);
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
