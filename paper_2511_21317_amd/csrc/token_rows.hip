// The rows that a QKV projection leaves, on their way into the layer or into a paged cache: norms of queries and keys
// over their 64 channels and the rotation of channel pairs by the token's position, in one pass.
//
//   layer norm  (x - mean) / sqrt(mean((x - mean)^2) + eps) * w + b,   RMS norm  x / sqrt(mean(x^2) + eps) * w + b
//   rotation    (x, y) -> (x cos t - y sin t, y cos t + x sin t),   t = position * base^(-2 i / axis width)
//
// The kernel moves 128 bytes in and 128 out per row (256 in from fp32) and does some ten operations per element: it is bound
// by memory, or by one launch where there are few rows.
// Measured: 137 400 tokens of 3 x 16 heads, 1.7 GB, 310 us, 5.4 TB/s (a copy of 2 GiB reaches 4.96); 10 992 tokens 26 us; 522 tokens 5.9 us, of
// which 2.4 are a launch.
//
// Layout.  Eight lanes hold a row, 8 channels (16 bytes of bf16) each, so a wave has the same head of eight
// consecutive tokens: eight 128-byte lines in, and out to [H, N, 64] 1 KB in a piece.  The sums of a norm are sums in
// a lane and three exchanges.  A wave walks over several heads of its tokens: the angles depend on the token alone, and
// their 16 sines and cosines per lane cost as much issue time as a row's memory time, so they are made once.
//
// Angles.  In units of turns and modulo 1, which is all that sine and cosine see: position times a 64-bit fraction
// of a turn per step, wrapped by the integer product itself.  The fraction is off by less than 2^-60 turns (the products
// that make it 2^-58 of itself, its last bit 2^-65), the angle at position 2^31 by 2^-29; fp32 holds the wrapped angle to 2^-26.  v_sin_f32 and v_cos_f32 take turns.
#include <algorithm>

#include "dev_common.hpp"
#include "kernels.hpp"

namespace httm {

namespace {

constexpr int kWaves = 4;          // per workgroup
constexpr int kTokens = 8;         // per wave

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// 8 channels of a row as they lie in memory, and as numbers
template <int DT>
struct RawChunk {
  u32x4 w[DT == HTTM_FP32 ? 2 : 1];
};
template <int DT, bool NT>
__device__ __forceinline__ RawChunk<DT> load_chunk(const char* row, int chunk) {
  RawChunk<DT> r;
#pragma unroll
  for (int i = 0; i < (DT == HTTM_FP32 ? 2 : 1); ++i) {
    const u32x4* at = (const u32x4*)row + (DT == HTTM_FP32 ? 2 * chunk + i : chunk);
    r.w[i] = NT ? __builtin_nontemporal_load(at) : *at;
  }
  return r;
}
template <int DT>
__device__ __forceinline__ void to_f32(const RawChunk<DT>& r, float (&x)[8]) {
  if constexpr (DT == HTTM_FP32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(r.w[e >> 2][e & 3]);
  } else if constexpr (DT == HTTM_FP16) {
    const f32x8 y = __builtin_convertvector(__builtin_bit_cast(f16x8, r.w[0]), f32x8);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = y[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e & 1 ? bf16_hi(r.w[0][e >> 1]) : bf16_lo(r.w[0][e >> 1]);
  }
}
__device__ __forceinline__ u32x4 pack_chunk(const float (&x)[8]) {
  return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
}

// Exchanges between the eight lanes of a row as data-parallel moves, which take no trip through the LDS: lane ^ 1, ^ 2 (within
// four lanes), lane ^ 7 (mirrored eight)
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kXor3 = 0x1B, kXor7 = 0x141;

// Sum over the eight lanes of a row
__device__ __forceinline__ float row_sum(float x) {
  x += moved<kXor1>(x);
  x += moved<kXor2>(x);
  return x + moved<kXor7>(x);
}

// What a lane knows of its eight channels for all heads of its token
struct LaneRope {
  float cos[8], sin[8];   // sin carries the sign that the channel's partner enters with
  int partner;            // lane that holds the other channel of the pairs (halves of other than 1, 2 or 4 chunks)
  bool rotates;           // these channels are among the first rot_dim
};

__device__ __forceinline__ void make_rope(LaneRope& r, const NormRopeArgs& a, int64_t p, int lane, bool rotates, int in_axis) {
  r.rotates = rotates;
  const int half = a.axis_chunks >> 1;
  const bool halves = a.pairing == HTTM_ROPE_HALVES;
  const bool second = halves && in_axis >= half;
  r.partner = !rotates || !halves ? lane : (second ? lane - half : lane + half);
  const int first_pair = halves ? (second ? in_axis - half : in_axis) * 8 : in_axis * 4;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int pair = halves ? first_pair + e : first_pair + (e >> 1);
    const uint64_t frac = (uint64_t)p * a.turn[rotates ? pair & (kMaxPairs - 1) : 0];
    const float t = (float)(int32_t)(frac >> 32) * 2.3283064365386963e-10f;    // 2^-32
    const float c = __builtin_amdgcn_cosf(t), s = __builtin_amdgcn_sinf(t);
    const bool minus = halves ? !second : (e & 1) == 0;
    r.cos[e] = c;
    r.sin[e] = minus ? -s : s;
  }
}

// Where the other channel of a pair is: in the lane itself, or in the lane 1, 2, 4 or another number of chunks away
enum { PAIR_OWN, PAIR_1, PAIR_2, PAIR_4, PAIR_FAR };
__device__ __forceinline__ int pair_place(const NormRopeArgs& a) {
  const int half = a.axis_chunks >> 1;
  return a.pairing != HTTM_ROPE_HALVES ? PAIR_OWN : half == 1 ? PAIR_1 : half == 2 ? PAIR_2 : half == 4 ? PAIR_4 : PAIR_FAR;
}
template <int PLACE>
__device__ __forceinline__ void rotate_with(float (&x)[8], const LaneRope& r) {
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    y[e] = PLACE == PAIR_OWN ? x[e ^ 1] : PLACE == PAIR_1 ? moved<kXor1>(x[e]) : PLACE == PAIR_2 ? moved<kXor2>(x[e])
           : PLACE == PAIR_4 ? moved<kXor3>(moved<kXor7>(x[e])) : __shfl(x[e], r.partner);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = r.rotates ? fmaf(x[e], r.cos[e], y[e] * r.sin[e]) : x[e];
}
__device__ __forceinline__ void rotate(float (&x)[8], const LaneRope& r, int place) {
  switch (place) {
    case PAIR_OWN: return rotate_with<PAIR_OWN>(x, r);
    case PAIR_1: return rotate_with<PAIR_1>(x, r);
    case PAIR_2: return rotate_with<PAIR_2>(x, r);
    case PAIR_4: return rotate_with<PAIR_4>(x, r);
    default: return rotate_with<PAIR_FAR>(x, r);
  }
}

__device__ __forceinline__ void normalise(float (&x)[8], int norm, float eps, const float (&w)[8], const float (&b)[8]) {
  if (norm == HTTM_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += x[e];
    const float mean = row_sum(s) * (1.f / kDHead);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] -= mean;
  }
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(x[e], x[e], s);
  const float scale = 1.f / sqrtf(row_sum(s) * (1.f / kDHead) + eps);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = fmaf(x[e] * scale, w[e], b[e]);
}

// Where a token of the batch belongs in the cache
struct CachePlace {
  bool real;          // of a sequence, not padding
  bool in_cache;      // its row exists and has a page
  int64_t row;        // in its sequence
  int64_t page_row;   // page * H_kv * page_size + row in the page: add head * page_size
};
__device__ __forceinline__ CachePlace find_place(const NormRopeArgs& a, int64_t t, int lane) {
  CachePlace c = {false, false, 0, 0};
  // how many offsets are not above t: 64 at a time, one load for the whole wave.  us for 4096 tokens of 32 + 2 x 8 heads in 1 / 64 / 512 / 4096 sequences: 16.4 /
  // 17.0 / 22.8 / 64.9; one token each of 32 / 70 / 1000: 4.6 / 4.9 / 13.6
  int below = 0;
  const int n_off = a.cache.n_seqs + 1, mine = lane >> 3;
  for (int i = 0; i < n_off; i += 64) {
    const int off = i + lane < n_off ? a.offsets[i + lane] : INT32_MAX;
#pragma unroll
    for (int j = 0; j < kTokens; ++j) {
      const int64_t tj = __shfl((int)t, 8 * j);
      const int n = __popcll(__ballot(off <= tj));
      below += mine == j ? n : 0;
    }
  }
  const int b = below - 1;
  if (t >= a.N || b < 0 || b >= a.cache.n_seqs) return c;
  c.real = true;
  const int64_t most = (int64_t)a.cache.table_stride << a.cache.page_shift;
  const int64_t len = std::clamp<int64_t>(a.seq_lens[b], 0, most);
  c.row = len - a.offsets[b + 1] + t;
  if (c.row < 0 || c.row >= most) return c;
  const int64_t page = a.cache.table[(int64_t)b * a.cache.table_stride + (c.row >> a.cache.page_shift)];
  if (page < 0 || page >= a.cache.n_pages) return c;
  c.in_cache = true;
  c.page_row = ((page * a.cache.H_kv) << a.cache.page_shift) + (c.row & ((1 << a.cache.page_shift) - 1));
  return c;
}

// A wave's part of q, k or v: heads [head0, head1) of its eight tokens
template <int DT, bool APPEND, bool NT, int AHEAD>
__global__ __launch_bounds__(64 * kWaves) void norm_rope_kernel(const NormRopeArgs a, int heads_per_wave) {
  const int lane = threadIdx.x & 63, chunk = lane & 7;
  const int64_t t = (int64_t)blockIdx.x * kTokens + (lane >> 3);
  int wave = blockIdx.y * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = 0;
  for (; part < 3; ++part) {
    const int waves = (a.H[part] + heads_per_wave - 1) / heads_per_wave;
    if (wave < waves) break;
    wave -= waves;
  }
  if (part == 3) return;
  const int head0 = wave * heads_per_wave, heads = a.H[part];
  const int head1 = head0 + heads_per_wave < heads ? head0 + heads_per_wave : heads;
  constexpr int kBytes = DT == HTTM_FP32 ? 4 : 2;
  const int64_t tt = t < a.N ? t : a.N - 1;     // lanes of no token read the last one and write nothing
  const char* token = a.src[part].data + tt * a.src[part].token_stride * kBytes;
  const int64_t head_bytes = a.src[part].head_stride * kBytes;

  // AHEAD rows at a time are requested, next to those in work, without a condition: a head past the last is read as the last
  RawChunk<DT> next[AHEAD];
  auto request = [&](int head) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) next[i] = load_chunk<DT, NT>(token + (head + i < head1 ? head + i : head1 - 1) * head_bytes, chunk);
  };
  request(head0);

  CachePlace place = {true, false, 0, 0};
  if constexpr (APPEND) place = find_place(a, t, lane);
  const bool write = t < a.N && place.real && (!APPEND || part == 0 || place.in_cache);

  LaneRope rope = {};
  float w[8], b[8];
  const bool turns = a.axes > 0 && part < 2;
  const int pairs = pair_place(a);
  const float scale = part == 1 ? a.k_scale : 1.f;
  if (part < 2) {
    if (a.norm != HTTM_NORM_NONE) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = a.weight[part] ? a.weight[part][chunk * 8 + e] : 1.f;
        b[e] = a.bias[part] ? a.bias[part][chunk * 8 + e] : 0.f;
      }
    }
    if (turns) {
      int axis = 0, in_axis = chunk;
      while (axis < a.axes && in_axis >= a.axis_chunks) in_axis -= a.axis_chunks, ++axis;
      const bool rotates = axis < a.axes;
      int64_t p = 0;
      if (rotates) p = a.pos ? (int64_t)a.pos[tt * a.axes + axis] : a.first_pos + place.row;
      make_rope(rope, a, p, lane, rotates, rotates ? in_axis : 0);
    }
  }
  // first row of the output, and from one head to the next
  char* out = a.out[part];
  int64_t out_bytes = kRowBytes;
  if constexpr (!APPEND) {
    out += (head0 * a.N + t) * kRowBytes;
    out_bytes = a.N * kRowBytes;
  } else if (part == 0) {
    out += (t * a.H[0] + head0) * kRowBytes;
  } else {
    out = (part == 1 ? a.cache.k_pages : a.cache.v_pages) + (place.page_row + ((int64_t)head0 << a.cache.page_shift)) * kRowBytes;
    out_bytes = (int64_t)kRowBytes << a.cache.page_shift;
  }
  for (int head = head0; head < head1; head += AHEAD) {
    RawChunk<DT> raw[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) raw[i] = next[i];
    if (head + AHEAD < head1) request(head + AHEAD);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      u32x4 packed;
      if (part == 2 && DT == HTTM_BF16) {
        packed = raw[i].w[0];
      } else {
        float x[8];
        to_f32<DT>(raw[i], x);
        if (part < 2) {
          if (a.norm != HTTM_NORM_NONE) normalise(x, a.norm, a.eps, w, b);
          if (turns) rotate(x, rope, pairs);
          if (scale != 1.f) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= scale;
          }
        }
        packed = pack_chunk(x);
      }
      if (write && head + i < head1) {
        u32x4* to = (u32x4*)(out + (head - head0 + i) * out_bytes) + chunk;
        if constexpr (NT)
          __builtin_nontemporal_store(packed, to);
        else
          *to = packed;
      }
    }
  }
}

}  // namespace

template <int DT, bool APPEND, bool NT>
void start_norm_rope(const NormRopeArgs& a, int64_t groups, int heads_per_wave, hipStream_t stream) {
  int waves = 0;
  for (int h : a.H) waves += (h + heads_per_wave - 1) / heads_per_wave;
  const dim3 grid((unsigned)groups, (unsigned)((waves + kWaves - 1) / kWaves)), block(64 * kWaves);
  if (heads_per_wave == 1)
    hipLaunchKernelGGL((norm_rope_kernel<DT, APPEND, NT, 1>), grid, block, 0, stream, a, heads_per_wave);
  else if (heads_per_wave == 2)
    hipLaunchKernelGGL((norm_rope_kernel<DT, APPEND, NT, 2>), grid, block, 0, stream, a, heads_per_wave);
  else
    hipLaunchKernelGGL((norm_rope_kernel<DT, APPEND, NT, 4>), grid, block, 0, stream, a, heads_per_wave);
}
template <int DT>
void start_norm_rope(const NormRopeArgs& a, bool append, bool nt, int64_t groups, int heads_per_wave, hipStream_t stream) {
  if (append)
    start_norm_rope<DT, true, false>(a, groups, heads_per_wave, stream);
  else if (nt)
    start_norm_rope<DT, false, true>(a, groups, heads_per_wave, stream);
  else
    start_norm_rope<DT, false, false>(a, groups, heads_per_wave, stream);
}

hipError_t launch_norm_rope(const NormRopeArgs& a, int dtype, bool append, hipStream_t stream) {
  const int slots = a.H[0] + a.H[1] + a.H[2];
  if (a.N == 0 || slots == 0) return hipSuccess;
  const int64_t groups = (a.N + kTokens - 1) / kTokens;
  // Heads a wave takes one after the other.  More of them share the sines and cosines and keep more rows on their way; fewer fill the
  // chip when there are few rows.  us with 1 / 2 / 4 / 8 / 16: 1500 tokens of 48 heads 11.2 / 8.5 / 8.2 / - / -, 10992 - / - / 26.8 / 25.6 / 28.6
  const int64_t rows = groups * slots;     // (eight of them)
  const int per = rows < 2048 ? 1 : rows < 4096 ? 2 : (int)std::clamp<int64_t>(rows / 8192 / 4 * 4, 4, 16);
  // past the caches where the tensors do not fit there; us with / without: 137 400 tokens of 48 heads 313 / 337, 10 992 28.1 / 26.0.  Not for appended
  // rows, which the batch's attention reads next; by themselves 137 400 tokens take 291 / 309, 27 480 65.4 / 68.9, 22 003 54.2 / 50.9
  const bool nt = a.N * slots * kRowBytes > ((int64_t)128 << 20);
  if (dtype == HTTM_BF16)
    start_norm_rope<HTTM_BF16>(a, append, nt, groups, per, stream);
  else if (dtype == HTTM_FP16)
    start_norm_rope<HTTM_FP16>(a, append, nt, groups, per, stream);
  else
    start_norm_rope<HTTM_FP32>(a, append, nt, groups, per, stream);
  return hipGetLastError();
}

}  // namespace httm
