// Keys and values in 8 bits: writing tokens into the cache, reading them back, attention over it
// (asa_cache_write, asa_cache_read, asa_attn_cache).
//
// The cache lies in memory in the order in which the matrix instructions take their operands (asa.h): 32 tokens
// are D / 32 operand tiles of K and as many of V, 1 KB each, of which a lane takes 16 consecutive bytes.  A
// wavefront's load is one contiguous KB, from global memory or from LDS, without a swizzle and without a transposition.
//   K tile t: lane (h, r) holds token r, channels 32 t + 16 h .. + 15: two A operands of S^T = K Q^T, whose result gives
//             lane (h, query) the tokens 8 m + 4 h + j in register 4 m + j;
//   V tile t: lane (h, r) holds channel 32 t + r, tokens 8 m + 4 h + j in byte 4 m + j: two A operands of O^T = V^T P^T,
//             for which the registers of S^T are the B operand as they stand.
#include "asa_common.hpp"
#include "asa_extra.hpp"
#include "asa_tiles.hpp"

namespace asa {

namespace {

constexpr int kThreads = 256;
constexpr int kLeastExp = -100, kMostExp = 120;     // of a block's scale

// A sequence's share [from, to) of the positions of one call, inside the cache.
struct Span {
  int64_t from, to;
};
__device__ __forceinline__ Span span_of(const CacheArgs &a, int b, int block) {
  const int64_t start = a.start ? a.start[b] : 0;
  const int count = a.count ? min(max(a.count[b], 0), a.L) : a.L;
  const int64_t room = (int64_t)a.max_blocks * block;
  return Span{start, start + count < room ? start + count : room};
}

// One (side, sequence, key head, block of the cache) of a call, and the tokens [lo, hi) of it that the call deals with.
struct BlockItem {
  int side, b, h, j, lo, hi;
  int64_t row0;     // row of the call's tensor that token 0 of the block would be
  bool any;
};
__device__ __forceinline__ BlockItem block_item(const CacheArgs &a, int block, bool writing) {
  BlockItem it;
  int x = blockIdx.x;
  const int jb = x % a.reached;
  x /= a.reached;
  it.h = x % a.H;
  x /= a.H;
  it.b = x % a.B;
  it.side = x / a.B;
  const Span s = span_of(a, it.b, block);
  const int64_t from = s.from < 0 ? 0 : s.from;
  const int64_t j = from / block + jb, t0 = j * block;
  it.j = (int)j;
  it.row0 = t0 - s.from;
  it.lo = from > t0 ? (int)(from - t0) : 0;
  it.hi = s.to - t0 < block ? (int)(s.to > t0 ? s.to - t0 : 0) : block;
  it.any = it.lo < it.hi && !(writing && s.from < 0);
  return it;
}

__device__ __forceinline__ uint32_t magnitudes_max(uint32_t a, uint32_t b) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
  const u16x2 x = __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b));
  return __builtin_bit_cast(uint32_t, x);
}
__device__ __forceinline__ bool finite_bits(uint32_t magnitude) { return magnitude < 0x7f80u; }

__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
#if defined(__HIP_DEVICE_COMPILE__)
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
#else
  return 0;
#endif
}
__device__ __forceinline__ f32x4 decode4(uint32_t codes) {
#if defined(__HIP_DEVICE_COMPILE__)
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  return f32x4{lo[0], lo[1], hi[0], hi[1]};
#else
  return f32x4{};
#endif
}

// x / scale: exact by the reciprocal where the scale is a power of two, as those of the writer are (a division is ten
// instructions).  EXACT is the caller's branch on is_power_of_two(scale).
__device__ __forceinline__ bool is_power_of_two(float s) {
  const uint32_t bits = __builtin_bit_cast(uint32_t, s), e = bits >> 23;
  return (bits & 0x7fffffu) == 0 && e >= 1 && e <= 253;
}
template <bool EXACT>
struct Divider {
  float scale, reciprocal;
  __device__ __forceinline__ explicit Divider(float s)
      : scale(s), reciprocal(__builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, s))) {}
  __device__ __forceinline__ float operator()(float x) const { return EXACT ? x * reciprocal : x / scale; }
};

// bytes of a dword whose tokens t0 .. t0 + 3 lie in [lo, hi)
__device__ __forceinline__ uint32_t bytes_within(int t0, int lo, int hi) {
  const int a = min(max(lo - t0, 0), 4), b = min(max(hi - t0, 0), 4);
  return (uint32_t)(((1ull << (8 * b)) - 1) & ~((1ull << (8 * a)) - 1));
}

// byte address, in a block, of (token, 8 channels from 8 * chunk) in K's order, and of the dword of tokens
// 4 * quad .. + 3 of one channel in V's
template <int D>
__device__ __forceinline__ int k_place(int token, int chunk) {
  return token / 32 * (32 * D) + chunk / 2 * 512 + token % 32 * 16 + chunk % 2 * 8;
}
template <int D>
__device__ __forceinline__ int v_place(int quad, int channel) {
  return quad / 8 * (32 * D) + channel / 32 * 1024 + quad % 2 * 512 + channel % 32 * 16 + quad % 8 / 2 * 4;
}

// Where a block's 16-byte piece p lies in LDS while the block is put together: the pieces that the lanes of one store go to are
// a multiple of 8 apart, which without this is the same few banks.
__device__ __forceinline__ int image_piece(int p) { return p ^ ((p >> 3 & 7) | (p >> 6 & 1) << 3); }
__device__ __forceinline__ int image_at(int byte) { return image_piece(byte >> 4) << 4 | (byte & 15); }

// The four tokens `raw` (8 channels each) of a thread as codes in the block's image.
template <int D, bool EXACT>
__device__ __forceinline__ void encode_unit(const u32x4 (&raw)[4], bool odd, float scale, bool transposed, int quad, int chunk,
                                            unsigned char *image) {
  const Divider<EXACT> by(scale);
  float x[4][8];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float lo = __builtin_bit_cast(float, raw[j][w] << 16), hi = __builtin_bit_cast(float, raw[j][w] & 0xffff0000u);
      if (odd) {
        if (__builtin_isinf(lo)) lo = __builtin_nanf("");
        if (__builtin_isinf(hi)) hi = __builtin_nanf("");
      }
      x[j][2 * w] = by(lo);
      x[j][2 * w + 1] = by(hi);
    }
  if (transposed) {
#pragma unroll
    for (int c = 0; c < 8; ++c)
      *reinterpret_cast<uint32_t *>(image + image_at(v_place<D>(quad, chunk * 8 + c))) = encode4(x[0][c], x[1][c], x[2][c], x[3][c]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<uint2 *>(image + image_at(k_place<D>(quad * 4 + j, chunk))) =
          uint2{encode4(x[j][0], x[j][1], x[j][2], x[j][3]), encode4(x[j][4], x[j][5], x[j][6], x[j][7])};
  }
}
// The held codes among four, written again for another scale.
template <bool EXACT>
__device__ __forceinline__ uint32_t recoded(uint32_t codes, uint32_t which, float old_scale, float scale) {
  const Divider<EXACT> by(scale);
  const f32x4 was = decode4(codes);
  const uint32_t now = encode4(by(was[0] * old_scale), by(was[1] * old_scale), by(was[2] * old_scale), by(was[3] * old_scale));
  return (now & which) | (codes & ~which);
}

}  // namespace

template <int D, int BLOCK>
constexpr int cache_threads() { return BLOCK * D / 32 < kThreads ? BLOCK * D / 32 : kThreads; }   // 32 values a thread at least

// One workgroup for each block that new tokens go to: the rows come in 16 bytes to a lane (four tokens of 8
// channels in each thread), the block's maximum gives the scale, the codes are put into their order in LDS and leave
// 16 bytes to a lane.  Of a block that is not written whole the codes are read as well (on their way while the
// scale is formed): pieces of 16 bytes that hold new tokens and others are put together, and the tokens held are coded
// again where the scale grew.  Bound by HBM: 17 776 tokens of 2 x 48 heads of 64, K and V, 437 MB in, 219 MB out:
// 137 us (4.8 TB/s).  A single token for each of 128 (sequence, head) pairs: 6.9 us, a chain of start, row, maximum, codes.
template <int D, int BLOCK>
__global__ __launch_bounds__((cache_threads<D, BLOCK>())) void cache_write_kernel(const CacheArgs a) {
  constexpr int kThreads = cache_threads<D, BLOCK>(), kChunks = D / 8, kPer = BLOCK / 4 * kChunks / kThreads;
  constexpr int kPieces = BLOCK * D / 16 / kThreads;      // of 16 bytes, in a thread
  const BlockItem it = block_item(a, BLOCK, true);
  if (!it.any) return;
  const CacheSide &side = a.side[it.side];
  const int64_t slab = (int64_t)it.b * a.H + it.h;
  float *scale_at = side.scale + slab * a.max_blocks + it.j;
  unsigned char *codes = reinterpret_cast<unsigned char *>(side.codes) + (slab * a.max_blocks + it.j) * (BLOCK * D);
  const bf16 *rows = reinterpret_cast<const bf16 *>(side.rows) + it.b * side.view.sB + it.h * side.view.sH;
  const bool held = it.lo > 0;
  const float old_scale = held ? *scale_at : 0.f;

  u32x4 raw[kPer][4];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int u = threadIdx.x + i * kThreads, quad = u / kChunks, chunk = u % kChunks;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = quad * 4 + j;
      raw[i][j] = u32x4{0, 0, 0, 0};
      if (t >= it.lo && t < it.hi)
        raw[i][j] = *reinterpret_cast<const u32x4 *>(rows + (it.row0 + t) * side.view.sL + chunk * 8);
    }
  }
  // bytes that are kept, on their way while the scale is formed: of a block that is written whole there are none
  const bool whole = it.lo == 0 && it.hi == BLOCK;
  u32x4 old[kPieces];
  if (!whole) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) old[i] = *reinterpret_cast<const u32x4 *>(codes + (threadIdx.x + i * kThreads) * 16);
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int w = 0; w < 4; ++w) most = magnitudes_max(most, raw[i][j][w] & 0x7fff7fffu);
  const bool odd = !finite_bits(most & 0xffffu) || !finite_bits(most >> 16);     // an infinity or a NaN among mine
  uint32_t top = max(most & 0xffffu, most >> 16);
  if (odd) {
    top = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t lo = raw[i][j][w] & 0x7fffu, hi = raw[i][j][w] >> 16 & 0x7fffu;
          if (finite_bits(lo)) top = max(top, lo);
          if (finite_bits(hi)) top = max(top, hi);
        }
  }
  __shared__ uint32_t wave_top[kThreads / 64];
  __shared__ __align__(16) unsigned char image[BLOCK * D];
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s, 64));
  if (threadIdx.x % 64 == 0) wave_top[threadIdx.x / 64] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) top = max(top, wave_top[w]);

  // top = (1 + f) 2^x with f in its low 7 bits; 448 = (1 + 3/4) 2^8
  int e = (int)(top >> 7) - 127 - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0);
  e = min(max(e, kLeastExp), kMostExp);
  const float needed = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
  const float scale = held && old_scale > needed ? old_scale : needed;
  const bool recode = held && scale != old_scale;
  const bool exact = __builtin_amdgcn_readfirstlane(is_power_of_two(scale));

#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int u = threadIdx.x + i * kThreads, quad = u / kChunks, chunk = u % kChunks;
    if (quad * 4 + 3 < it.lo || quad * 4 >= it.hi) continue;
    if (exact) encode_unit<D, true>(raw[i], odd, scale, side.transposed, quad, chunk, image);
    else encode_unit<D, false>(raw[i], odd, scale, side.transposed, quad, chunk, image);
  }
  __syncthreads();
  if (threadIdx.x == 0) *scale_at = scale;

  if (whole) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int at = (threadIdx.x + i * kThreads) * 16;
      *reinterpret_cast<u32x4 *>(codes + at) = *reinterpret_cast<const u32x4 *>(image + image_at(at));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int piece = threadIdx.x + i * kThreads;
    const int t_first = piece / (2 * D) * 32 + (side.transposed ? piece / 32 % 2 * 4 : piece % 32);
    u32x4 value = *reinterpret_cast<const u32x4 *>(image + image_at(piece * 16));
    uint32_t any = 0;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      // (a piece of K is 16 channels of one token)
      const uint32_t fresh = side.transposed ? bytes_within(t_first + 8 * m, it.lo, it.hi)
                                             : (t_first >= it.lo && t_first < it.hi ? ~0u : 0u);
      const uint32_t again = !recode ? 0u : side.transposed ? bytes_within(t_first + 8 * m, 0, it.lo) : (t_first < it.lo ? ~0u : 0u);
      any |= fresh | again;
      uint32_t kept = old[i][m];
      if (again) kept = exact ? recoded<true>(kept, again, old_scale, scale) : recoded<false>(kept, again, old_scale, scale);
      value[m] = (value[m] & fresh) | (kept & ~fresh);
    }
    if (any) *reinterpret_cast<u32x4 *>(codes + piece * 16) = value;
  }
}

// One workgroup for each block that the call reads from; a thread writes 16 bytes of a row (K) or of four rows (V).  Bound by HBM:
// those tokens again, 219 MB in, 437 MB out: 118 us.
template <int D, int BLOCK>
__global__ __launch_bounds__((cache_threads<D, BLOCK>())) void cache_read_kernel(const CacheArgs a) {
  constexpr int kThreads = cache_threads<D, BLOCK>(), kChunks = D / 8;
  const BlockItem it = block_item(a, BLOCK, false);
  if (!it.any) return;
  const CacheSide &side = a.side[it.side];
  const int64_t slab = (int64_t)it.b * a.H + it.h;
  const float scale = side.scale[slab * a.max_blocks + it.j];
  const unsigned char *codes = reinterpret_cast<const unsigned char *>(side.codes) + (slab * a.max_blocks + it.j) * (BLOCK * D);
  bf16 *rows = reinterpret_cast<bf16 *>(side.rows) + it.b * side.view.sB + it.h * side.view.sH;
  // (all loads of a thread in front of the first use: the block is the cache's own, whichever of its tokens are asked for)
  if (side.transposed) {
    constexpr int kPer = BLOCK / 4 * kChunks / kThreads;
    uint32_t raw[kPer][8];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int u = threadIdx.x + i * kThreads, quad = u / kChunks, chunk = u % kChunks;
#pragma unroll
      for (int c = 0; c < 8; ++c) raw[i][c] = *reinterpret_cast<const uint32_t *>(codes + v_place<D>(quad, chunk * 8 + c));
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int u = threadIdx.x + i * kThreads, quad = u / kChunks, chunk = u % kChunks;
      f32x4 x[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) x[c] = decode4(raw[i][c]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = quad * 4 + j;
        u32x4 out;
#pragma unroll
        for (int w = 0; w < 4; ++w) out[w] = pack_bf16x2(x[2 * w][j] * scale, x[2 * w + 1][j] * scale);
        if (t >= it.lo && t < it.hi) *reinterpret_cast<u32x4 *>(rows + (it.row0 + t) * side.view.sL + chunk * 8) = out;
      }
    }
  } else {
    constexpr int kPer = BLOCK * kChunks / kThreads;
    uint2 raw[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int u = threadIdx.x + i * kThreads;
      raw[i] = *reinterpret_cast<const uint2 *>(codes + k_place<D>(u / kChunks, u % kChunks));
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int u = threadIdx.x + i * kThreads, t = u / kChunks, chunk = u % kChunks;
      const f32x4 lo = decode4(raw[i].x), hi = decode4(raw[i].y);
      const u32x4 out = {pack_bf16x2(lo[0] * scale, lo[1] * scale), pack_bf16x2(lo[2] * scale, lo[3] * scale),
                         pack_bf16x2(hi[0] * scale, hi[1] * scale), pack_bf16x2(hi[2] * scale, hi[3] * scale)};
      if (t >= it.lo && t < it.hi) *reinterpret_cast<u32x4 *>(rows + (it.row0 + t) * side.view.sL + chunk * 8) = out;
    }
  }
}

// ---------------------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------------------
namespace {

constexpr int kMaxSplits = kThreads;
constexpr int64_t kMostSums = (int64_t)1 << 28;           // values of the parts' sums: 1 GB of workspace at most
constexpr int64_t kFewRows = 4096;   // up to here the join has a workgroup for each row
constexpr float kLn2 = 0.6931471805599453f;
// What a row's maximum may grow by before its sums are brought down to it (log2 units).  Probabilities are then up to 2^8
// instead of 1, their rounding to bf16 is as near as before (though a row's largest is no longer exactly 1: where one key has
// nearly all the weight the result carries that rounding, 2^-9, beside its own), and the sums' D multiplications are rare
// instead of in nearly every step (4 680 queries on 32 760 keys, 12 heads of 128: 953 -> 925 us).
constexpr float kSlack = 8.f;
constexpr float kLeastScale = 7.8886091e-31f;     // 2^-100: probabilities down to 2^-26 times it are normal numbers
constexpr float kLeastFactor = 1.17549435e-38f;   // (a factor of zero would make NaN of a masked score)

// The two A operands that 16 codes of a tile are.
struct Operands {
  bf16x8 part[2];
};
__device__ __forceinline__ Operands widen(u32x4 codes) {
  Operands r;
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    bf16x2 x[4];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      x[2 * w] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * u + w], 1.0f, false);
      x[2 * w + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * u + w], 1.0f, true);
    }
    r.part[u] = bf16x8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
  }
#else
  r = Operands{};
#endif
  return r;
}
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

// A word that is the same for the whole wavefront and that the kernel does not write: read through the scalar cache, also
// behind written-out loads, whose memory clobber would make a vector load (and a wait for all copies in flight) of it.
template <typename T>
__device__ __forceinline__ T uniform_read(const T *p) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint64_t s = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x) |
                     ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32);
  return *reinterpret_cast<const __attribute__((address_space(4))) T *>(s);
#else
  return *p;
#endif
}

// Scales of a block as the inner loop wants them.
struct BlockScale {
  float c;          // of K, with the soft-max scale, in log2 units
  float log2_v;     // of V: the probabilities carry it, so that the accumulators need no scaling of their own ...
  float inv_v;      // ... and their sum takes it off again
  __device__ __forceinline__ BlockScale(const CacheAttnArgs &a, float k, float v) {
    c = fmaxf(a.scale_log2 * k, kLeastFactor);
    v = fmaxf(v, kLeastScale);
    log2_v = __builtin_amdgcn_logf(v);
    inv_v = __builtin_amdgcn_rcpf(v);     // (exact for a power of two, else within a last bit)
  }
};

// 32 rows (queries) of one wavefront: lane (h, r) holds row r's running maximum and its half of the denominator.
template <int D>
struct Rows {
  static constexpr int T = D / 32;
  bf16x8 q[T][2];
  f32x16 acc[T];     // O^T: register 4 g + j is channel 32 t + 8 g + 4 h + j
  float m, l;

  __device__ __forceinline__ void init(const bf16 *row, int half) {
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) q[t][u] = *reinterpret_cast<const bf16x8 *>(row + 32 * t + 16 * half + 8 * u);
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
    m = -__builtin_inff();
    l = 0.f;
  }

  // NG groups of 32 keys (MASKED: of which the first `left` > 0 keys exist); k(n, t), v(n, t): 16 codes of the lane in tile t
  template <int NG, bool MASKED, typename K, typename V>
  __device__ __forceinline__ void attend(const K &k, const V &v, const BlockScale &bs, int left, int half) {
    f32x16 s[NG];
#pragma unroll
    for (int n = 0; n < NG; ++n) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[n][i] = 0.f;
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const Operands kk = widen(k(n, t));
        s[n] = mfma(kk.part[0], q[t][0], s[n]);
        s[n] = mfma(kk.part[1], q[t][1], s[n]);
      }
    }
    if (MASKED) {
#pragma unroll
      for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * n + 8 * (i / 4) + 4 * half + i % 4 >= left) s[n][i] = -__builtin_inff();
    }
    float top = s[0][0];
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
    const float m_new = fmaxf(m, max_of_halves(top) * bs.c);
    const bool grown = m_new - m > kSlack;
    if (__ballot(grown)) {
      // (each row by its own maximum alone, so that its bits are the same whatever the wavefront's other rows hold)
      const float shrink = grown ? fast_exp2(m - m_new) : 1.f;
      l *= shrink;
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[t][i] *= shrink;
      m = grown ? m_new : m;
    }
    const float down = bs.log2_v - m;
    float sum = 0.f;
#pragma unroll
    for (int n = 0; n < NG; ++n) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[n][i] = fast_exp2(__builtin_fmaf(s[n][i], bs.c, down));
        sum += s[n][i];
      }
      bf16x8 p[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const u32x4 x = {pack_bf16x2(s[n][8 * u], s[n][8 * u + 1]), pack_bf16x2(s[n][8 * u + 2], s[n][8 * u + 3]),
                         pack_bf16x2(s[n][8 * u + 4], s[n][8 * u + 5]), pack_bf16x2(s[n][8 * u + 6], s[n][8 * u + 7])};
        p[u] = __builtin_bit_cast(bf16x8, x);
      }
#pragma unroll
      for (int t = 0; t < T; ++t) {
        u32x4 codes = v(n, t);
        if (MASKED) {       // what lies behind the last token may be a NaN
#pragma unroll
          for (int g = 0; g < 4; ++g) codes[g] &= bytes_within(32 * n + 8 * g + 4 * half, 0, left);
        }
        const Operands vv = widen(codes);
        acc[t] = mfma(vv.part[0], p[0], acc[t]);
        acc[t] = mfma(vv.part[1], p[1], acc[t]);
      }
    }
    l = __builtin_fmaf(sum, bs.inv_v, l);
  }
};

// Where a row of a unit (sequence, key head, block of queries, row tile) lies: rows of a block of queries go through the
// query heads that share the key head, and through the block's tokens in each.
struct Unit {
  int slab, b, h_kv, qb, tile, tokens, rows;   // rows: of this tile that exist (<= 0: none)
  __device__ __forceinline__ Unit(const CacheAttnArgs &a, int unit) {
    const int x = unit / a.tiles;
    tile = unit - x * a.tiles;
    slab = x / a.n_qblocks;
    qb = x - slab * a.n_qblocks;
    b = slab / a.H_kv;
    h_kv = slab - b * a.H_kv;
    tokens = min(a.block, a.L - qb * a.block);
    rows = min(tokens * a.group - tile * a.tile_rows, a.tile_rows);
  }
  // head and token of row r of the tile
  __device__ __forceinline__ void place(const CacheAttnArgs &a, int r, int &head, int &token) const {
    const int x = tile * a.tile_rows + r, g = x / tokens;
    head = h_kv * a.group + g;
    token = qb * a.block + x - g * tokens;
  }
};

// The blocks that a unit's split walks: positions [at, end) of the row's list, or of all blocks.
struct Walk {
  const int32_t *list;
  int at, end, length, n_blocks;
  __device__ __forceinline__ Walk(const CacheAttnArgs &a, const Unit &u, int split) {
    length = (int)min((int64_t)max(a.length[u.b], 0), (int64_t)a.max_blocks * a.block);
    n_blocks = (length + a.block - 1) / a.block;
    int n = n_blocks;
    list = nullptr;
    if (a.row_ptr) {
      const int room = a.n_qblocks * a.max_blocks;
      const int32_t *ptr = a.row_ptr + (int64_t)u.slab * (a.n_qblocks + 1) + u.qb;
      const int first = min(max(ptr[0], 0), room), last = min(max(ptr[1], first), room);
      list = a.col_idx + (int64_t)u.slab * room + first;
      n = min(last - first, a.max_blocks);      // (distinct blocks)
    }
    const int share = max((n + a.splits - 1) / a.splits, 1);
    at = (int)min((int64_t)split * share, (int64_t)n);
    end = min(at + share, n);
  }
  // what stands at a position; the block there, negative where the list names none that the sequence has
  __device__ __forceinline__ int entry(int position) const { return list ? uniform_read(list + position) : position; }
  __device__ __forceinline__ int block(int e) const { return e >= 0 && e < n_blocks ? e : -1; }
};

// Steps of KEYS keys along a walk, STRIDE apart: those that are full, one after the other; the one that the sequence ends
// in (there is one at most) is kept for the end, so that the loop over the others need not mask.
template <int BLOCK, int KEYS, int STRIDE>
struct Steps {
  static constexpr int kPerBlock = BLOCK / KEYS, kAhead = STRIDE > kPerBlock ? STRIDE / kPerBlock : 1;   // (in positions)
  const Walk &walk;
  const CacheAttnArgs &a;
  int64_t block0;
  int x, end, j;              // step, its block
  float k_scale, v_scale;     // of the block, on their way while the step before is worked on
  int last_x, last_j;
  int position, ahead;        // of the walk; the list's entry kAhead further on, on its way
  __device__ __forceinline__ Steps(const CacheAttnArgs &a_, const Walk &w, int64_t block0_, int first)
      : walk(w), a(a_), block0(block0_), end(w.end * kPerBlock), j(-1), k_scale(1.f), v_scale(1.f), last_x(-1), last_j(0),
        position(-1), ahead(0) {
    x = w.at * kPerBlock + first;
    if (x >= end) return;
    ahead = w.entry(x / kPerBlock);
    find(x);
  }
  __device__ __forceinline__ bool any() const { return x < end; }
  __device__ __forceinline__ void advance() { find(x + STRIDE); }
  __device__ __forceinline__ void find(int from) {
    for (x = from; x < end; x += STRIDE) {
      if (x / kPerBlock != position) {
        position = x / kPerBlock;
        j = __builtin_amdgcn_readfirstlane(walk.block(ahead));
        ahead = walk.entry(min(position + kAhead, walk.end - 1));
      }
      if (j < 0) continue;
      const int left = walk.length - keys_before();
      if (left >= KEYS) {
        scales();
        return;
      }
      if (left > 0) {
        last_x = x;
        last_j = j;
      }
    }
  }
  // the step that the sequence ends in becomes the current one
  __device__ __forceinline__ bool to_last() {
    if (last_x < 0) return false;
    x = last_x;
    j = last_j;
    scales();
    return true;
  }
  __device__ __forceinline__ void scales() {
    k_scale = uniform_read(a.k_scale + block0 + j);
    v_scale = uniform_read(a.v_scale + block0 + j);
  }
  __device__ __forceinline__ int keys_before() const { return j * BLOCK + x % kPerBlock * KEYS; }
  // byte address of the step's codes, of K and of V
  template <int D>
  __device__ __forceinline__ int64_t codes() const { return (block0 + j) * (BLOCK * D) + x % kPerBlock * (KEYS * D); }
};

// The result of 32 rows: a row of o and lse, or of the split's partial sums.
template <int D>
__device__ __forceinline__ void put_rows(const CacheAttnArgs &a, const Unit &u, int unit, int split, int row, int half,
                                         const f32x16 (&acc)[D / 32], float m, float l) {
  if (row >= u.rows) return;
  const bool nothing = l == 0.f && m == -__builtin_inff();
  if (a.splits > 1) {
    const int64_t at = ((int64_t)unit * a.splits + split) * a.rows_kept + row;
    float *ml = a.partial + (int64_t)a.units * a.splits * a.rows_kept * D + at * 2;
    if (half == 0) {
      ml[0] = m;
      ml[1] = l;
    }
    if (nothing) return;
    float *to = a.partial + at * D + 4 * half;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4 *>(to + 32 * t + 8 * g) = f32x4{acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]};
    return;
  }
  int head, token;
  u.place(a, row, head, token);
  const float f = nothing ? 0.f : 1.0f / l;
  bf16 *to = reinterpret_cast<bf16 *>(a.o) + u.b * a.ov.sB + head * a.ov.sH + token * a.ov.sL + 4 * half;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<uint2 *>(to + 32 * t + 8 * g) = uint2{pack_bf16x2(acc[t][4 * g] * f, acc[t][4 * g + 1] * f),
                                                             pack_bf16x2(acc[t][4 * g + 2] * f, acc[t][4 * g + 3] * f)};
  if (half == 0) a.lse[((int64_t)u.b * a.H + head) * a.L + token] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace

// Few rows (a token-by-token step): all of a tile's 32 rows in every wavefront, the keys shared out among the four.  What
// bounds it is the cache's bytes; a wavefront has the next 32 keys' 2 * 32 * D bytes in flight while it works on these.
// One token, 131 000 tokens, 12 heads of 128: 72 us = 5.6 TB/s.
template <int D, int BLOCK>
__global__ __launch_bounds__(kThreads, 2) void cache_attn_rows_kernel(const CacheAttnArgs a) {
  constexpr int T = D / 32, kWaves = kThreads / 64, kPitch = D + 4;
  __shared__ float wave_m[kWaves][32], wave_l[kWaves][32];
  __shared__ __align__(16) float half_acc[kWaves / 2][32 * kPitch];
  const int item = xcd_contiguous_work(blockIdx.x, a.units * a.splits);
  if (item < 0) return;
  const int unit = item / a.splits, split = item - unit * a.splits;
  const Unit u(a, unit);
  if (u.rows <= 0) return;
  const Walk walk(a, u, split);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, row = lane & 31;

  Rows<D> rows;
  {
    int head, token;
    u.place(a, min(row, u.rows - 1), head, token);
    rows.init(reinterpret_cast<const bf16 *>(a.q) + u.b * a.qv.sB + head * a.qv.sH + token * a.qv.sL, half);
  }
  struct Codes {
    u32x4 k[T], v[T];
  };
  auto fetch = [&](int64_t at, Codes &c) {
    const char *k = reinterpret_cast<const char *>(a.k) + at + lane * 16, *v = reinterpret_cast<const char *>(a.v) + at + lane * 16;
#pragma unroll
    for (int t = 0; t < T; ++t) c.k[t] = *reinterpret_cast<const u32x4 *>(k + t * 1024);
#pragma unroll
    for (int t = 0; t < T; ++t) c.v[t] = *reinterpret_cast<const u32x4 *>(v + t * 1024);
  };
  Codes now, coming;
  auto k_now = [&](int, int t) { return now.k[t]; };
  auto v_now = [&](int, int t) { return now.v[t]; };
  Steps<BLOCK, 32, kWaves> step(a, walk, (int64_t)u.slab * a.max_blocks, wave);
  if (step.any()) fetch(step.template codes<D>(), now);
  while (step.any()) {
    const BlockScale bs(a, step.k_scale, step.v_scale);
    step.advance();
    if (step.any()) fetch(step.template codes<D>(), coming);
    rows.template attend<1, false>(k_now, v_now, bs, 32, half);
    now = coming;
  }
  if (step.to_last()) {
    fetch(step.template codes<D>(), now);
    rows.template attend<1, true>(k_now, v_now, BlockScale(a, step.k_scale, step.v_scale), walk.length - step.keys_before(), half);
  }

  // the four wavefronts' parts of each row into one
  rows.l += swap_halves(rows.l);
  if (half == 0) {
    wave_m[wave][row] = rows.m;
    wave_l[wave][row] = rows.l;
  }
  __syncthreads();
  float m = -__builtin_inff(), l = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, wave_m[w][row]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float mw = wave_m[w][row], lw = wave_l[w][row];
    if (!(mw == -__builtin_inff() && lw == 0.f)) l = __builtin_fmaf(lw, fast_exp2(mw - m), l);
  }
  const float f = rows.m == -__builtin_inff() && rows.l == 0.f ? 0.f : fast_exp2(rows.m - m);
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) rows.acc[t][i] *= f;
#pragma unroll
  for (int step = kWaves / 2; step > 0; step /= 2) {
    if (wave >= step && wave < 2 * step && row < u.rows) {
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4 *>(&half_acc[wave - step][row * kPitch + 32 * t + 8 * g + 4 * half]) =
              f32x4{rows.acc[t][4 * g], rows.acc[t][4 * g + 1], rows.acc[t][4 * g + 2], rows.acc[t][4 * g + 3]};
    }
    __syncthreads();
    if (wave < step && row < u.rows) {
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 other = *reinterpret_cast<const f32x4 *>(&half_acc[wave][row * kPitch + 32 * t + 8 * g + 4 * half]);
#pragma unroll
          for (int i = 0; i < 4; ++i) rows.acc[t][4 * g + i] += other[i];
        }
    }
    __syncthreads();
  }
  if (wave == 0) put_rows<D>(a, u, unit, split, row, half, rows.acc, m, l);
}

// Many rows: two or four wavefronts of 32 rows each walk the listed blocks together, 64 keys at a time; the codes of the
// next 64 are copied to LDS meanwhile (two buffers), every wavefront widens what it reads.  Bound by the matrix and the
// vector pipe, which overlap little (64 keys x 32 rows at D 128: 1024 cycles of products, 512 of widening, 540 of soft-max):
// 4 680 queries on 32 760 tokens, 12 heads of 128: 895 to 920 us with the join, from card to card = 1020 to 1050 TFLOP/s; at D 64
// the vector pipe alone decides.
template <int D, int BLOCK, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void cache_attn_tile_kernel(const CacheAttnArgs a) {
  constexpr int kKeys = 64, kBytes = kKeys * D, kCopies = kBytes / 1024 / WAVES;
  __shared__ __align__(16) char stage[2][2][kBytes];
  const int item = xcd_contiguous_work(blockIdx.x, a.units * a.splits);
  if (item < 0) return;
  const int unit = item / a.splits, split = item - unit * a.splits;
  const Unit u(a, unit);
  if (u.rows <= 0) return;
  const Walk walk(a, u, split);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int row = wave * 32 + (lane & 31);

  Rows<D> rows;
  {
    int head, token;
    u.place(a, min(row, u.rows - 1), head, token);
    rows.init(reinterpret_cast<const bf16 *>(a.q) + u.b * a.qv.sB + head * a.qv.sH + token * a.qv.sL, half);
  }
  const uint32_t lane_off = (uint32_t)(wave * kCopies * 1024 + lane * 16);
  auto copy = [&](int64_t at, int buffer) {
    const char *k = reinterpret_cast<const char *>(a.k) + at, *v = reinterpret_cast<const char *>(a.v) + at;
    const uint32_t to = ASA_LDS_ADDR_OF(stage) + buffer * (2 * kBytes) + wave * kCopies * 1024;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      lds_dma16_sv(k, lane_off + i * 1024, to + i * 1024);
      lds_dma16_sv(v, lane_off + i * 1024, to + kBytes + i * 1024);
    }
  };
  auto arrived = [&]() {      // my copies, then everybody's
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#endif
    __syncthreads();
  };
  const bool mine = wave * 32 < u.rows;
  int buffer = 0;
  auto k_now = [&](int n, int t) { return *reinterpret_cast<const u32x4 *>(&stage[buffer][0][lane * 16 + n * 32 * D + t * 1024]); };
  auto v_now = [&](int n, int t) { return *reinterpret_cast<const u32x4 *>(&stage[buffer][1][lane * 16 + n * 32 * D + t * 1024]); };
  Steps<BLOCK, kKeys, 1> step(a, walk, (int64_t)u.slab * a.max_blocks, 0);
  if (step.any()) copy(step.template codes<D>(), 0);
  while (step.any()) {
    arrived();              // (nobody reads the other buffer any more, either)
    const BlockScale bs(a, step.k_scale, step.v_scale);
    step.advance();
    if (step.any()) copy(step.template codes<D>(), buffer ^ 1);
    if (mine) rows.template attend<2, false>(k_now, v_now, bs, kKeys, half);
    buffer ^= 1;
  }
  if (step.to_last()) {
    copy(step.template codes<D>(), buffer);      // (this one was read before the last barrier)
    arrived();
    if (mine)
      rows.template attend<2, true>(k_now, v_now, BlockScale(a, step.k_scale, step.v_scale), walk.length - step.keys_before(), half);
  }
  rows.l += swap_halves(rows.l);
  put_rows<D>(a, u, unit, split, row, half, rows.acc, rows.m, rows.l);
}

// Joins the parts of each row.  D / 4 lanes take a part's row.  With GROUPS such groups a row is one workgroup's work
// and each group takes every GROUPS-th part, joined through LDS (a row in 170 parts: 10 us; one group alone takes 110, a
// load's latency for each part); many rows of a few parts each are several to a workgroup.
template <int D, int GROUPS>
__global__ __launch_bounds__(kThreads) void cache_attn_join_kernel(const CacheAttnArgs a) {
  constexpr int kLanes = D / 4, kRows = kThreads / kLanes / GROUPS;
  static_assert(kMaxSplits == kThreads, "a thread for each part");
  __shared__ float factor[GROUPS > 1 ? kMaxSplits : 1], wave_m[kThreads / 64], wave_l[kThreads / 64];
  __shared__ __align__(16) f32x4 part[GROUPS > 1 ? GROUPS : 1][kLanes];
  const int64_t r = (int64_t)blockIdx.x * kRows + (GROUPS > 1 ? 0 : threadIdx.x / kLanes);
  const int sub = threadIdx.x % kLanes, group = GROUPS > 1 ? threadIdx.x / kLanes : 0;
  if (r >= (int64_t)a.units * a.rows_kept) return;
  const int unit = GROUPS > 1 ? (int)r / a.rows_kept : (int)(r / a.rows_kept);
  const int row = (int)(r - (int64_t)unit * a.rows_kept);
  const Unit u(a, unit);
  if (row >= u.rows) return;
  const int64_t first = (int64_t)unit * a.splits * a.rows_kept + row;
  const f32x2 *ml = reinterpret_cast<const f32x2 *>(a.partial + (int64_t)a.units * a.splits * a.rows_kept * D);
  float m = -__builtin_inff(), l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if constexpr (GROUPS > 1) {
    f32x2 mine = {-__builtin_inff(), 0.f};
    if ((int)threadIdx.x < a.splits) mine = ml[first + (int64_t)threadIdx.x * a.rows_kept];
    m = mine[0];
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor(m, s, 64));
    if (threadIdx.x % 64 == 0) wave_m[threadIdx.x / 64] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) m = fmaxf(m, wave_m[w]);
    // (a part without a key has left its sums unwritten: factor 0 and no read)
    const bool nothing = mine[0] == -__builtin_inff() && mine[1] == 0.f;
    const float f = nothing ? 0.f : fast_exp2(mine[0] - m);
    factor[threadIdx.x] = f;
    l = nothing ? 0.f : mine[1] * f;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) l += __shfl_xor(l, s, 64);
    if (threadIdx.x % 64 == 0) wave_l[threadIdx.x / 64] = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) l += wave_l[w];
#pragma unroll 4
    for (int s = group; s < a.splits; s += GROUPS) {
      const float fs = factor[s];
      if (fs == 0.f) continue;
      const f32x4 p = *reinterpret_cast<const f32x4 *>(a.partial + (first + (int64_t)s * a.rows_kept) * D + sub * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(p[i], fs, o[i]);
    }
    part[group][sub] = o;
    __syncthreads();
    if (group != 0) return;
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) o += part[g][sub];
  } else {
    // four parts at a time, their loads together
    for (int s0 = 0; s0 < a.splits; s0 += 4) {
      f32x2 x[4];
      f32x4 p[4];
      bool counts[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t at = first + (int64_t)min(s0 + e, a.splits - 1) * a.rows_kept;
        x[e] = ml[at];
        p[e] = *reinterpret_cast<const f32x4 *>(a.partial + at * D + sub * 4);
      }
      float top = m;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // (a part without a key has left its sums unwritten)
        counts[e] = s0 + e < a.splits && !(x[e][0] == -__builtin_inff() && x[e][1] == 0.f);
        if (counts[e]) top = fmaxf(top, x[e][0]);
      }
      const float kept = m == -__builtin_inff() && l == 0.f ? 0.f : fast_exp2(m - top);
      m = top;
      l *= kept;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= kept;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float f = fast_exp2(x[e][0] - top);
        if (!counts[e]) continue;
        l = __builtin_fmaf(x[e][1], f, l);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(p[e][i], f, o[i]);
      }
    }
  }
  int head, token;
  u.place(a, row, head, token);
  const float f = l == 0.f && m == -__builtin_inff() ? 0.f : 1.0f / l;
  bf16 *to = reinterpret_cast<bf16 *>(a.o) + u.b * a.ov.sB + head * a.ov.sH + token * a.ov.sL + sub * 4;
  *reinterpret_cast<uint2 *>(to) = uint2{pack_bf16x2(o[0] * f, o[1] * f), pack_bf16x2(o[2] * f, o[3] * f)};
  if (sub == 0) a.lse[((int64_t)u.b * a.H + head) * a.L + token] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------
// How many parts the keys of a row are cut into: the number with the least time by a model of the launch.  Cutting
// fills the chip and evens out its last round; each part costs the writing and reading of its sums.
//
// Tiles of many rows: a compute unit takes `fit` workgroups at once, k of them in fit / 3 + 2 k / 3 times one's time on a full
// unit (few wavefronts leave it idle); more than that as they come, or, where the cache's bytes are the time, in rounds.
// Measured (us, by parts): 43 tiles of 50 rows, 36 558 keys, d 128: 4: 251, 6: 200, 12: 140, 17: 112, 23: 103, 29: 121, 42: 114
// (the model takes 23); 36 tiles of 128 rows, 32 760 keys, d 128: 4: 214, 8: 131, 12: 101, 21: 103, 32: 121 (21); 156 of them: 1:
// 803, 3: 350, 5: 414, 8: 341, 12: 366 (8); 444: 1: 979, 2: 1014, 4: 910, 5: 933, 8: 954 (4); 16 tiles of 64 rows, 60 000 keys,
// d 64: 12: 112, 23: 72, 42: 51, 64: 44, 85: 49, 128: 47 (128); 1056 of them, 4 400 keys: 1: 149, 2: 143, 3: 137, 5: 142 (the
// model has 3 and 5 within 0.2 us of each other and takes 5).
// Few rows: the cache's bytes are all the time, and all workgroups should run at once.  One token, 131 000 keys, 12 key heads:
// 21: 77, 42 (504 workgroups, 512 fit): 77, 43: 104, 85: 81, 170: 88; 128 heads of up to 8 000 keys: 2: 51, 4: 39, 8: 42, 16: 49.
//
// The lengths are on the device: the keys that are counted here, the 256 of a part among them, are those that the cache has room
// for, or a quarter of them where there are lists.  A sequence that holds less is cut into as many parts, shorter or empty ones.
static int splits_of(const CacheAttnPlan &plan, const Problem &pb, int max_blocks, bool lists) {
  constexpr int kUnits = 256;                          // compute units
  const bool few = plan.tile_rows == 32, wide = pb.d == 128;
  const double keys = (double)max_blocks * pb.block * (lists ? 0.25 : 1.0);     // lists: what they may keep
  const int fit = few ? (wide ? 2 : 4) : wide ? (plan.tile_rows == 64 ? 4 : 3) : (plan.tile_rows == 64 ? 8 : 4);   // registers, LDS
  // a workgroup's time at its share of a full chip: its codes at 5.5 (tiles: 4.4) TB/s, or its products at 1000 / 600 TFLOP/s
  const double copies = 2.0 * keys * pb.d / ((few ? 5.5e12 : 4.4e12) / kUnits);
  const double products = 4.0 * plan.tile_rows * keys * pb.d / ((wide ? 1.0e15 : 0.6e15) / kUnits);
  const double part = 8.0 * plan.units * plan.rows_kept * pb.d / 8e12;
  auto together = [&](int64_t k) { return k == 0 ? 0.0 : fit / 3.0 + 2.0 * k / 3.0; };
  int best = 1;
  double best_time = 1e30;
  for (int s = 1; s <= kMaxSplits && (s == 1 || (s * 256.0 <= keys && plan.units * s * plan.rows_kept * pb.d <= kMostSums)); ++s) {
    const int64_t n = (plan.units * s + kUnits - 1) / kUnits, full = n / fit * fit;
    double time = s > 1 ? s * part + 3e-6 : 0.0;
    if (few) time += (double)((plan.units * s + kUnits * fit - 1) / (kUnits * fit)) * (fit * copies / s + 2e-6);
    else if (copies > products) time += ((double)full + together(n - full)) / s * copies;
    else time += (n < fit ? together(n) : (double)n) / s * products;
    if (time < best_time) {
      best_time = time;
      best = s;
    }
  }
  return best;
}

int plan_cache_attn(const Problem &pb, int H_kv, int max_blocks, bool lists, CacheAttnPlan *plan) {
  const int group = pb.H / H_kv;
  const int64_t rows = (int64_t)(pb.L < pb.block ? pb.L : pb.block) * group;   // of one list
  plan->n_qblocks = pb.Nb;
  plan->tile_rows = rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  plan->tiles = (int)((rows + plan->tile_rows - 1) / plan->tile_rows);
  plan->rows_kept = (int)(rows < plan->tile_rows ? rows : plan->tile_rows);
  plan->units = (int64_t)pb.B * H_kv * pb.Nb * plan->tiles;
  plan->splits = 1;
  if ((int64_t)pb.Nb * max_blocks >= ((int64_t)1 << 31)) return ASA_ERR_UNSUPPORTED;
  // (keys are cut only where there are far fewer units than this: kMostSums)
  if (!launch_fits((plan->units + kNumXcd - 1) / kNumXcd * kNumXcd, plan->tile_rows == 64 ? 128 : 256)) return ASA_ERR_UNSUPPORTED;
  plan->splits = splits_of(*plan, pb, max_blocks, lists);
  return ASA_OK;
}

size_t cache_attn_workspace_bytes(const Problem &pb, const CacheAttnPlan &plan) {
  if (plan.splits == 1) return 0;
  return (size_t)plan.units * plan.splits * plan.rows_kept * (pb.d + 2) * sizeof(float);
}

template <int D, int BLOCK>
static hipError_t launch_cache_attn_as(const CacheAttnArgs &a, hipStream_t st) {
  const int grid = xcd_grid(a.units * a.splits);
  if (a.tile_rows == 32) cache_attn_rows_kernel<D, BLOCK><<<grid, kThreads, 0, st>>>(a);
  else if (a.tile_rows == 64) cache_attn_tile_kernel<D, BLOCK, 2><<<grid, 128, 0, st>>>(a);
  else cache_attn_tile_kernel<D, BLOCK, 4><<<grid, 256, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  constexpr int kGroups = kThreads / (D / 4);
  const int64_t rows = (int64_t)a.units * a.rows_kept;
  if (rows <= kFewRows) cache_attn_join_kernel<D, kGroups><<<(int)rows, kThreads, 0, st>>>(a);
  else cache_attn_join_kernel<D, 1><<<(int)((rows + kGroups - 1) / kGroups), kThreads, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_cache_attn(const CacheAttnArgs &a, int D, hipStream_t st) {
  if (D == 128) return a.block == 128 ? launch_cache_attn_as<128, 128>(a, st) : launch_cache_attn_as<128, 64>(a, st);
  return a.block == 128 ? launch_cache_attn_as<64, 128>(a, st) : launch_cache_attn_as<64, 64>(a, st);
}

int plan_cache(const CacheArgs &a, int D, int block) {
  const int64_t workgroups = (int64_t)a.reached * a.H * a.B * a.n_sides;
  const int threads = block == 64 && D == 64 ? cache_threads<64, 64>() : kThreads;
  return launch_fits(workgroups, threads) ? ASA_OK : ASA_ERR_UNSUPPORTED;
}

template <int D, int BLOCK>
static hipError_t launch_cache_as(const CacheArgs &a, bool write, hipStream_t st) {
  const int grid = a.reached * a.H * a.B * a.n_sides;
  constexpr int threads = cache_threads<D, BLOCK>();
  if (write) cache_write_kernel<D, BLOCK><<<grid, threads, 0, st>>>(a);
  else cache_read_kernel<D, BLOCK><<<grid, threads, 0, st>>>(a);
  return hipGetLastError();
}
static hipError_t launch_cache(const CacheArgs &a, int D, int block, bool write, hipStream_t st) {
  if (D == 128) return block == 128 ? launch_cache_as<128, 128>(a, write, st) : launch_cache_as<128, 64>(a, write, st);
  return block == 128 ? launch_cache_as<64, 128>(a, write, st) : launch_cache_as<64, 64>(a, write, st);
}
hipError_t launch_cache_write(const CacheArgs &a, int D, int block, hipStream_t st) { return launch_cache(a, D, block, true, st); }
hipError_t launch_cache_read(const CacheArgs &a, int D, int block, hipStream_t st) { return launch_cache(a, D, block, false, st); }

}  // namespace asa
