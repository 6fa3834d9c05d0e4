// Norm of queries and keys for each head with the rotation by position in the same pass, forward and
// backward (asa_qk_norm_rope, asa_qk_norm_rope_bwd).
//
// A row is the D channels of one token and head.  A lane holds 8 channels (one 16-byte load and store), D / 8
// lanes a row; sums over a row are four additions through the lane permutes of the vector ALU, in fp32.  The work
// is 2 (forward) or 3 (backward) bf16 values per channel from and to HBM and nothing else, so what
// counts is that every wavefront has several loads in flight: a group of lanes takes one token and
// kHeads heads of it, whose rows it loads before it works on the first; they share the token's angles.
// At 32 760 tokens, 12 + 12 heads of 128 out of one projection: forward 79 us = 5.3 TB/s, a large copy's rate; backward
// 126 us = 4.9 TB/s and 4.7 us for the sums.  2 or 6 heads at once: 79, 82 us; with heads of 64 4 is best (95, 87, 88).
#include "asa_common.hpp"
#include "asa_extra.hpp"

namespace asa {

namespace {

constexpr int kHeads = 4;      // heads of a token that a group of lanes takes at once
constexpr int kThreads = 256;
constexpr int kMaxGroups = 512;    // workgroups of the backward for each of Q and K, each with a row of partial sums

enum Pairing { kAdjacent = ASA_ROPE_ADJACENT, kHalves = ASA_ROPE_HALVES, kNone = 2 };

// sum over the LANES (8 or 16) lanes of a row, in every one of them
template <int CTRL>
__device__ __forceinline__ float add_permuted(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
#else
  return x;
#endif
}
template <int LANES>
__device__ __forceinline__ float row_sum(float x) {
  x = add_permuted<0xB1>(x);                         // neighbour
  x = add_permuted<0x4E>(x);                         // other pair of the four
  x = add_permuted<0x141>(x);                        // mirrored in 8: the other four
  if (LANES == 16) x = add_permuted<0x140>(x);       // mirrored in 16: the other eight
  return x;
}

__device__ __forceinline__ void widen8(u32x4 raw, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __builtin_bit_cast(float, raw[i] << 16);
    x[2 * i + 1] = __builtin_bit_cast(float, raw[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 narrow8(const float (&x)[8]) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
  return r;
}

// What a lane needs to turn its 8 channels: ADJACENT has both channels of a pair, HALVES finds the others in
// the lane `partner`.
template <int PAIR>
struct Turn {
  bool on;
  float c[PAIR == kHalves ? 8 : 4], s[PAIR == kHalves ? 8 : 4];   // s with the sign that the lane's half takes
  int partner;

  template <int LANES>
  __device__ __forceinline__ void init(const NormArgs &a, int lane, int sub, int b, int l) {
    const int quarter = a.rot / 16;        // lanes of one half of the turned channels
    int64_t row = (int64_t)a.first_row + l;
    if (a.start) row += a.start[b];
    on = row >= 0 && row < a.table_rows && sub < 2 * quarter;
    const bool low = sub < quarter;
    partner = lane - sub + (on ? (low ? sub + quarter : sub - quarter) : sub);
    const int at = PAIR == kHalves ? (low ? sub : sub - quarter) * 8 : sub * 4;
    const int64_t first = on ? row * (a.rot / 2) + at : 0;
    constexpr int N = PAIR == kHalves ? 2 : 1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const f32x4 cc = *reinterpret_cast<const f32x4 *>(a.cos_table + first + 4 * i);
      const f32x4 ss = *reinterpret_cast<const f32x4 *>(a.sin_table + first + 4 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c[4 * i + j] = cc[j];
        s[4 * i + j] = PAIR == kHalves && low ? -ss[j] : ss[j];
      }
    }
  }
  // z turned; DIR = -1 turns back.  other: the partner lane's values (HALVES)
  template <int DIR>
  __device__ __forceinline__ void apply(float (&z)[8], const float (&other)[8]) const {
    if (PAIR == kNone) return;
    float y[8];
    if (PAIR == kAdjacent) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[2 * i] = z[2 * i] * c[i] - z[2 * i + 1] * (DIR * s[i]);
        y[2 * i + 1] = z[2 * i] * (DIR * s[i]) + z[2 * i + 1] * c[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = z[i] * c[i & (PAIR == kHalves ? 7 : 3)] + other[i] * (DIR * s[i & (PAIR == kHalves ? 7 : 3)]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = on ? y[i] : z[i];
  }
  __device__ __forceinline__ u32x4 from_partner(u32x4 raw) const {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (uint32_t)__shfl((int)raw[i], partner, 64);
    return r;
  }
};

// mean (0 for RMS) and 1 / deviation of a row; x becomes x - mean
template <int LANES, bool LAYER>
__device__ __forceinline__ float centre(float (&x)[8], float &mean, float eps) {
  constexpr float kPart = 1.0f / (LANES * 8);
  mean = 0.f;
  if (LAYER) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += x[i];
    mean = row_sum<LANES>(t) * kPart;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] -= mean;
  }
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) t = __builtin_fmaf(x[i], x[i], t);
  return rsqrtf(row_sum<LANES>(t) * kPart + eps);
}

template <int D>
__device__ __forceinline__ void load_params(const float *p, int sub, float otherwise, float (&out)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) out[i] = p ? p[sub * 8 + i] : otherwise;
}

}  // namespace

// Workgroup items: (tile of tokens, side, chunk of kHeads heads), a tile's chunks next to each other and on one XCD,
// so that the angles come from HBM once.
template <int D, int PAIR, bool LAYER>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(const NormArgs a) {
  constexpr int LANES = D / 8, kTokens = kThreads / LANES;
  const int chunks = a.side[0].chunks + a.side[1].chunks;
  const int item = xcd_contiguous_work(blockIdx.x, a.tiles * chunks);
  if (item < 0) return;
  const int tile = item / chunks, chunk_any = item - tile * chunks;
  const bool is_k = chunk_any >= a.side[0].chunks;
  const NormSide &side = a.side[is_k ? 1 : 0];
  const int head0 = (is_k ? chunk_any - a.side[0].chunks : chunk_any) * kHeads;

  const int lane = threadIdx.x & 63, sub = threadIdx.x % LANES;
  const int token = tile * kTokens + threadIdx.x / LANES;
  const bool there = token < a.tokens;
  const int t = there ? token : a.tokens - 1;
  const int b = t / a.L, l = t - b * a.L;

  const bf16 *src = reinterpret_cast<const bf16 *>(side.src) + b * side.in.sB + l * side.in.sL + sub * 8;
  bf16 *dst = reinterpret_cast<bf16 *>(side.dst) + b * side.out.sB + l * side.out.sL + sub * 8;
  u32x4 raw[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i)
    raw[i] = *reinterpret_cast<const u32x4 *>(src + (int64_t)min(head0 + i, side.heads - 1) * side.in.sH);

  Turn<PAIR> turn;
  if (PAIR != kNone) turn.template init<LANES>(a, lane, sub, b, l);
  float w[8], bias[8], w_other[8], bias_other[8];
  load_params<D>(side.w, sub, 1.f, w);
  load_params<D>(LAYER ? side.b : nullptr, sub, 0.f, bias);
  if (PAIR == kHalves) {
    load_params<D>(side.w, turn.partner % LANES, 1.f, w_other);
    load_params<D>(LAYER ? side.b : nullptr, turn.partner % LANES, 0.f, bias_other);
  }
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    if (head0 + i >= side.heads) break;
    float x[8], mean, other[8];
    widen8(raw[i], x);
    const float r = centre<LANES, LAYER>(x, mean, a.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = LAYER ? __builtin_fmaf(x[e] * r, w[e], bias[e]) : x[e] * r * w[e];
    if (PAIR == kHalves) {
      widen8(turn.from_partner(raw[i]), other);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        other[e] = LAYER ? __builtin_fmaf((other[e] - mean) * r, w_other[e], bias_other[e]) : other[e] * r * w_other[e];
    }
    turn.template apply<1>(x, other);
    if (there) *reinterpret_cast<u32x4 *>(dst + (int64_t)(head0 + i) * side.out.sH) = narrow8(x);
  }
}

// With dz the gradient turned back, xh the normalised row and gw = dz * weight:
//   dx = r (gw - xh mean(gw xh) [- mean gw]),   dweight = sum dz xh,   dbias = sum dz.
// The statistics are formed again from x (cheaper than reading them).  A workgroup walks a contiguous share of
// the (tile, chunk) items of Q or of K and keeps the two sums of its lanes' 8 channels in registers; they are joined
// through LDS at the end and written as one partial row, which norm_sums_kernel adds up in a fixed order.
template <int D, int PAIR, bool LAYER>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_bwd_kernel(const NormArgs a) {
  constexpr int LANES = D / 8, kTokens = kThreads / LANES;
  const bool is_k = (int)blockIdx.x >= a.side[0].groups;
  const NormSide &side = a.side[is_k ? 1 : 0];
  const int group = is_k ? blockIdx.x - a.side[0].groups : blockIdx.x;
  const int items = a.tiles * side.chunks;
  const int share = (items + side.groups - 1) / side.groups;

  const int lane = threadIdx.x & 63, sub = threadIdx.x % LANES;
  float w[8], dw[8] = {}, db[8] = {};
  load_params<D>(side.w, sub, 1.f, w);
  const int end = min((group + 1) * share, items);
  for (int item = group * share; item < end; ++item) {
    const int tile = item / side.chunks, head0 = (item - tile * side.chunks) * kHeads;
    const int token = tile * kTokens + threadIdx.x / LANES;
    const bool there = token < a.tokens;
    const int t = there ? token : a.tokens - 1;
    const int b = t / a.L, l = t - b * a.L;
    const bf16 *src = reinterpret_cast<const bf16 *>(side.src) + b * side.in.sB + l * side.in.sL + sub * 8;
    bf16 *dst = reinterpret_cast<bf16 *>(side.dst) + b * side.dx.sB + l * side.dx.sL + sub * 8;
    const bf16 *grad = reinterpret_cast<const bf16 *>(side.grad) + b * side.out.sB + l * side.out.sL + sub * 8;
    u32x4 raw[kHeads], raw_g[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      const int h = min(head0 + i, side.heads - 1);
      raw[i] = *reinterpret_cast<const u32x4 *>(src + (int64_t)h * side.in.sH);
      raw_g[i] = *reinterpret_cast<const u32x4 *>(grad + (int64_t)h * side.out.sH);
    }
    Turn<PAIR> turn;
    if (PAIR != kNone) turn.template init<LANES>(a, lane, sub, b, l);
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      if (head0 + i >= side.heads) break;
      float x[8], dz[8], mean, other[8];
      widen8(raw[i], x);
      widen8(raw_g[i], dz);
      const float r = centre<LANES, LAYER>(x, mean, a.eps);
      if (PAIR == kHalves) widen8(turn.from_partner(raw_g[i]), other);
      turn.template apply<-1>(dz, other);
      float along = 0.f, sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] *= r;
        dw[e] += there ? dz[e] * x[e] : 0.f;
        if (LAYER) db[e] += there ? dz[e] : 0.f;
        dz[e] *= w[e];
        along = __builtin_fmaf(dz[e], x[e], along);
        sum += dz[e];
      }
      along = row_sum<LANES>(along) * (1.0f / D);
      sum = LAYER ? row_sum<LANES>(sum) * (1.0f / D) : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = r * (dz[e] - __builtin_fmaf(x[e], along, sum));
      if (there) *reinterpret_cast<u32x4 *>(dst + (int64_t)(head0 + i) * side.dx.sH) = narrow8(x);
    }
  }

  __shared__ float sums[LAYER ? 2 : 1][kTokens][D];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sums[0][threadIdx.x / LANES][sub * 8 + e] = dw[e];
    if (LAYER) sums[LAYER ? 1 : 0][threadIdx.x / LANES][sub * 8 + e] = db[e];
  }
  __syncthreads();
  if (threadIdx.x < (LAYER ? 2 : 1) * D) {
    const int which = threadIdx.x / D, ch = threadIdx.x % D;
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < kTokens; ++i) total += sums[which][i][ch];
    side.partial[((int64_t)which * side.groups + group) * D + ch] = total;
  }
}

// out[ch] = sum over the workgroups' partial rows: 32 channels of one of the four sums for each workgroup, a quarter
// row to 8 threads, 128 rows at a time, then through LDS; always in the same order.
__global__ __launch_bounds__(1024) void norm_sums_kernel(const NormArgs a, int D) {
  const NormSide &side = a.side[blockIdx.y];
  const int which = blockIdx.z;
  float *out = which ? side.db : side.dw;
  if (!out) return;
  __shared__ float part[128][33];
  const int c = threadIdx.x % 8 * 4, s = threadIdx.x / 8;
  const float *p = side.partial + (int64_t)which * side.groups * D + blockIdx.x * 32 + c;
  f32x4 total = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kMaxGroups / 128; ++i) {      // (loads without a branch: all of them are in flight at once)
    const int g = s + i * 128;
    const f32x4 x = *reinterpret_cast<const f32x4 *>(p + (int64_t)min(g, side.groups - 1) * D);
#pragma unroll
    for (int j = 0; j < 4; ++j) total[j] += g < side.groups ? x[j] : 0.f;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) part[s][c + j] = total[j];
  for (int half = 64; half >= 32; half /= 2) {
    __syncthreads();
    for (int e = threadIdx.x; e < half * 32; e += 1024) part[e / 32][e % 32] += part[e / 32 + half][e % 32];
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) sum += part[i][threadIdx.x];
    out[blockIdx.x * 32 + threadIdx.x] = sum;
  }
}

// chunks, groups and tiles of a call; 0 = fits, else asa_status
int plan_norm(NormArgs *a, int D, bool backward) {
  const int64_t tokens = (int64_t)a->B * a->L;
  if (tokens >= ((int64_t)1 << 31) - 64) return ASA_ERR_UNSUPPORTED;
  const int per_tile = kThreads / (D / 8);
  a->tokens = (int)tokens;
  a->tiles = (int)((tokens + per_tile - 1) / per_tile);
  int64_t chunks = 0;
  for (NormSide &s : a->side) {
    s.chunks = (s.heads + kHeads - 1) / kHeads;
    chunks += s.chunks;
    const int64_t items = (int64_t)a->tiles * s.chunks;
    s.groups = (int)(items < kMaxGroups ? items : kMaxGroups);
  }
  // (the backward's workgroups walk: their places, rounded up to whole shares, are counted in 31 bits)
  const int64_t items = chunks * a->tiles, most = ((int64_t)1 << 31) - 2 * kMaxGroups;
  const bool fits = backward ? items < most : launch_fits((items + kNumXcd - 1) / kNumXcd * kNumXcd, kThreads);
  return fits ? ASA_OK : ASA_ERR_UNSUPPORTED;
}

size_t norm_partial_bytes(const NormSide &s, int D) { return (size_t)2 * s.groups * D * sizeof(float); }

template <int D, int PAIR, bool LAYER>
static hipError_t launch_norm_as(const NormArgs &a, bool backward, hipStream_t st) {
  if (!backward) {
    qk_norm_rope_kernel<D, PAIR, LAYER><<<xcd_grid(a.tiles * (a.side[0].chunks + a.side[1].chunks)), kThreads, 0, st>>>(a);
    return hipGetLastError();
  }
  qk_norm_rope_bwd_kernel<D, PAIR, LAYER><<<a.side[0].groups + a.side[1].groups, kThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  const bool wanted = a.side[0].dw || a.side[0].db || a.side[1].dw || a.side[1].db;
  if (e != hipSuccess || !wanted) return e;
  norm_sums_kernel<<<dim3(D / 32, a.side[1].heads ? 2 : 1, LAYER ? 2 : 1), 1024, 0, st>>>(a, D);
  return hipGetLastError();
}
template <int D, int PAIR>
static hipError_t launch_norm_kind(const NormArgs &a, bool layer, bool backward, hipStream_t st) {
  return layer ? launch_norm_as<D, PAIR, true>(a, backward, st) : launch_norm_as<D, PAIR, false>(a, backward, st);
}
template <int D>
static hipError_t launch_norm_pair(const NormArgs &a, bool layer, int pairing, bool backward, hipStream_t st) {
  if (a.rot == 0) return launch_norm_kind<D, kNone>(a, layer, backward, st);
  return pairing == ASA_ROPE_HALVES ? launch_norm_kind<D, kHalves>(a, layer, backward, st)
                                    : launch_norm_kind<D, kAdjacent>(a, layer, backward, st);
}
hipError_t launch_norm(const NormArgs &a, int D, bool layer, int pairing, bool backward, hipStream_t st) {
  return D == 128 ? launch_norm_pair<128>(a, layer, pairing, backward, st)
                  : launch_norm_pair<64>(a, layer, pairing, backward, st);
}

}  // namespace asa
