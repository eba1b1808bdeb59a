// The position rotation on the device: the angle of a pair, and 16 dimensions of
// a head rotated in registers.
//
// An angle in turns is p f / 2 pi modulo 1. With f / 2 pi held as a 64-bit fraction F
// the product p F modulo 2^64 is that remainder exactly (integers wrap where turns do),
// so that a position of a million is as good as one of ten: in fp32 p f would be off
// by 0.06 radians there. The fraction's upper 32 bits are split into the nearest quarter
// turn and the rest, whose sine and cosine are polynomials.
#pragma once

#include "cache_common.cuh"
#include "decode_internal.h"

namespace evisel {

// Positions on the (up to three) axes of token t of sequence b; `base` + i where neither `at` nor `first` is given.
__device__ __forceinline__ void positions_of(const RopeView& r, const PositionView& p, int b, int t, int base, int i,
                                             int (&pos)[3]) {
  if (p.at) {
    const int32_t* at = p.at + b * p.stride[1] + t;
    pos[0] = __ldg(at);
    pos[1] = r.border[0] < r.pairs ? __ldg(at + p.stride[0]) : 0;
    pos[2] = r.border[1] < r.pairs ? __ldg(at + 2 * p.stride[0]) : 0;
  } else {
    pos[0] = pos[1] = pos[2] = static_cast<int>(static_cast<unsigned>(p.first ? __ldg(p.first + b) : base) + static_cast<unsigned>(i));
  }
}

// Cosine and sine of turn / 2^32 turns, each within 2^-24 of those of the rest x as rounded (|x| <= pi / 4, off by
// 2^-23.3 at most). The polynomials in z = x^2 interpolate (sin x / x - 1) / z and (cos x - 1) / z at the Chebyshev
// points of [0, pi^2 / 16]. (With the library's sincospif in every head an append of 65,664 tokens and four heads took 77 us,
// 60 with these and a token's turns formed once for two heads.)
__device__ __forceinline__ float2 turned(uint32_t turn) {
  const uint32_t quarter = (turn + 0x20000000u) >> 30;
  const float x = static_cast<float>(static_cast<int32_t>(turn - (quarter << 30))) * 1.46291807926716e-9f;   // 2 pi / 2^32
  const float z = x * x;
  const float s = fmaf(x * z, fmaf(fmaf(-1.95878660e-4f, z, 8.33274797e-3f), z, -1.66666642e-1f), x);
  const float c = fmaf(fmaf(fmaf(fmaf(2.44637540e-5f, z, -1.38875889e-3f), z, 4.16666493e-2f), z, -0.5f), z, 1.f);
  const uint32_t odd = quarter & 1;
  const uint32_t re = __float_as_uint(odd ? s : c) ^ ((quarter + 1) & 2) << 30, im = __float_as_uint(odd ? c : s) ^ (quarter & 2) << 30;
  return make_float2(__uint_as_float(re), __uint_as_float(im));
}

// scale (cos, sin) of pair i; `sign` = -1 for the transposed matrix.
__device__ __forceinline__ float2 pair_turn(const RopeView& r, const int (&pos)[3], int i, float sign) {
  const int p = i < r.border[0] ? pos[0] : i < r.border[1] ? pos[1] : pos[2];
  const float2 t = turned(static_cast<uint32_t>(static_cast<uint64_t>(static_cast<int64_t>(p)) * r.turn[i] >> 32));
  return make_float2(t.x * r.scale, t.y * r.scale * sign);
}

// A head is shared by D / 16 lanes. Lane j < r / 16 has the 16-byte pieces lo and hi that hold
// pairs 8 j .. 8 j + 7; the others have two pieces of the rest.
__device__ __forceinline__ void lane_pieces(const RopeView& r, int j, int& lo, int& hi) {
  const int rot = r.pairs >> 3;                  // lanes that rotate
  const bool split = !r.interleaved && j < rot;
  lo = split ? j : 2 * j;
  hi = split ? j + rot : 2 * j + 1;
}

// Eight pairs of a lane's pieces, cs[e] the turn of pair 8 j + e.
template <class T, bool INTER>
__device__ __forceinline__ void rotate_pieces(uint4& lo, uint4& hi, const float2 (&cs)[8]) {
  float a[8], b[8], x[8], y[8];
  unpack8<T>(lo, a);
  unpack8<T>(hi, b);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float u = INTER ? (e < 4 ? a[(2 * e) & 7] : b[(2 * e) & 7]) : a[e];
    const float w = INTER ? (e < 4 ? a[(2 * e + 1) & 7] : b[(2 * e + 1) & 7]) : b[e];
    x[e] = u * cs[e].x - w * cs[e].y;
    y[e] = w * cs[e].x + u * cs[e].y;
  }
  if constexpr (INTER) {
    lo = make_uint4(T::pack(x[0], y[0]), T::pack(x[1], y[1]), T::pack(x[2], y[2]), T::pack(x[3], y[3]));
    hi = make_uint4(T::pack(x[4], y[4]), T::pack(x[5], y[5]), T::pack(x[6], y[6]), T::pack(x[7], y[7]));
  } else {
    lo = make_uint4(T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(x[4], x[5]), T::pack(x[6], x[7]));
    hi = make_uint4(T::pack(y[0], y[1]), T::pack(y[2], y[3]), T::pack(y[4], y[5]), T::pack(y[6], y[7]));
  }
}

constexpr int kHeadsAtOnce = 4;                  // passes whose loads are in flight together

// Heads [h0, h1) of the q and k heads of token t of sequence b, by one warp: the
// lanes form the token's turns once (mem: D / 2 entries of the warp's own) and every
// D / 16 lanes rotate a head, AT of them at a time.
template <class T, int D, bool INTER, int AT = kHeadsAtOnce>
__device__ __forceinline__ void rotate_token(const RopeView& r, const HeadsView& q, const HeadsView& k, int b, int t,
                                             const int (&pos)[3], float sign, int h0, int h1, float2* mem) {
  constexpr int LANES = D / 16, HEADS = 32 / LANES;
  const int lane = threadIdx.x & 31, j = lane % LANES;
  int lo, hi;
  lane_pieces(r, j, lo, hi);
  const uint16_t* q_in = static_cast<const uint16_t*>(q.in) + b * q.is[0] + t * q.is[1];
  const uint16_t* k_in = static_cast<const uint16_t*>(k.in) + b * k.is[0] + t * k.is[1];
  uint16_t* q_out = static_cast<uint16_t*>(q.out) + b * q.os[0] + t * q.os[1];
  uint16_t* k_out = static_cast<uint16_t*>(k.out) + b * k.os[0] + t * k.os[1];
  uint4 a[AT], c[AT];
  auto load = [&](int base) {
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const int h = base + i * HEADS;
      if (h < h1) {
        const uint4* row = reinterpret_cast<const uint4*>(h < q.heads ? q_in + h * q.is[2] : k_in + (h - q.heads) * k.is[2]);
        a[i] = row[lo];
        c[i] = row[hi];
      }
    }
  };
  int base = h0 + lane / LANES;
  load(base);                       // on their way while the turns are formed
  for (int i = lane; i < r.pairs; i += 32) mem[i] = pair_turn(r, pos, i, sign);
  __syncwarp();
  const bool rotates = 8 * j < r.pairs;
  float2 cs[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) cs[e] = rotates ? mem[8 * j + e] : make_float2(1.f, 0.f);
  while (base < h1) {
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const int h = base + i * HEADS;
      if (h < h1) {
        uint4* row = reinterpret_cast<uint4*>(h < q.heads ? q_out + h * q.os[2] : k_out + (h - q.heads) * k.os[2]);
        if (rotates) rotate_pieces<T, INTER>(a[i], c[i], cs);
        row[lo] = a[i];
        row[hi] = c[i];
      }
    }
    base += HEADS * AT;
    load(base);
  }
}

// Heads of a warp's share of a token: all of them where tokens fill the SMs by
// themselves, fewer (whole passes) where they do not.
inline int rotary_heads_per_warp(int64_t tokens, int heads, int head_dim, int n_sm) {
  const int pass = 512 / head_dim;
  const int64_t warps = static_cast<int64_t>(n_sm) * 32;
  const int64_t shares = tokens >= warps ? 1 : (warps + tokens - 1) / tokens;
  const int passes = (heads + pass - 1) / pass;
  const int64_t each = (passes + shares - 1) / shares;
  return static_cast<int>(each < 1 ? 1 : each) * pass;
}

}  // namespace evisel
