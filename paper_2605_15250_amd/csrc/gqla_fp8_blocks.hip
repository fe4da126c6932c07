// What fills the expanded caches: rows of new tokens appended to the 16-bit, fp32 or block-scaled 8-bit cache, and the 16-bit cache
// converted into the block-scaled one.
//
// Block scales.  The 32 tokens of a tile and the dims of one group, K or V, share one power of two 2^e: e is the smallest
// integer with amax <= 448 * 2^e (448: the largest E4M3 value), and a code is E4M3(x * 2^-e).  With amax's fp32 bits m * 2^k the rule is
// one addition: 448 = 1.75 * 2^8, so e = k - 8, plus one where the mantissa is above 0x600000, i.e. where adding 0x1fffff
// carries into the exponent.  A power of two loses nothing against a scale that maps amax to 448 exactly (codes are floating point),
// makes x * 2^-e exact, lets a block that was quantised to a smaller exponent move to a larger one without a second rounding (unless a
// code falls below 2^-6), and rides along for free in the instruction that widens codes (v_cvt_scalef32_pk_bf16_fp8).
#include "gqla_rows.h"

namespace gqla {

namespace {

constexpr int kBlockShift = 5, kBlock = 1 << kBlockShift;   // tokens that share a scale: the decode kernels' tile
constexpr int kExpMin = -100, kExpMax = 118;

__device__ __forceinline__ int block_exponent(uint32_t amax_bits) {
  return min(max((int)((amax_bits + 0x1fffffu) >> 23) - 127 - 8, kExpMin), kExpMax);
}
__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }
__device__ __forceinline__ int exponent_of(float scale) {
  return min(max((int)(__builtin_bit_cast(uint32_t, scale) >> 23 & 0xffu) - 127, kExpMin), kExpMax);
}

// maximum over the 64 lanes of values >= 0
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  auto step = [&](uint32_t o) { v = max(v, o); };
  step(__builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));  // row_shr:1
  step(__builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
  step(__builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
  step(__builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
  step(__builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));  // row_bcast:15 into rows 1 and 3
  step(__builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));  // row_bcast:31 into rows 2 and 3
  return __builtin_amdgcn_readlane(v, 63);
}

// |x| of two bf16 as 16-bit integers, whose order is the order of the magnitudes (infinities and NaN above all else)
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
__device__ __forceinline__ u16x2 max_abs(u16x2 m, uint32_t w) {
  return __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w & 0x7fff7fffu));
}
__device__ __forceinline__ u16x2 max_finite(u16x2 m, uint32_t w) {
  uint32_t a = w & 0x7fff7fffu;
  if ((a & 0xffffu) >= 0x7f80u) a &= 0xffff0000u;
  if (a >= 0x7f800000u) a &= 0xffffu;
  return __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, a));
}

// The block's exponent from the wave's words; `careful` says that some value needs more than a multiplication: an
// infinity (saturates), a NaN (stays one) or a magnitude beyond the largest scale (saturates).
template <class ForEach>
__device__ __forceinline__ int wave_exponent(ForEach&& words, bool& careful) {
  u16x2 m = {0, 0};
  words([&](uint32_t w) { m = max_abs(m, w); });
  uint32_t top = wave_max(max((uint32_t)m[0], (uint32_t)m[1]));
  careful = top >= 0x7f80u;
  if (careful) {
    m = u16x2{0, 0};
    words([&](uint32_t w) { m = max_finite(m, w); });
    top = wave_max(max((uint32_t)m[0], (uint32_t)m[1]));
  }
  const int e = block_exponent(top << 16);
  careful |= e == kExpMax;
  return e;
}

__device__ __forceinline__ float saturate(float x) { return x != x ? x : __builtin_amdgcn_fmed3f(x, -448.f, 448.f); }
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv, bool careful) {
  a *= inv; b *= inv; c *= inv; d *= inv;
  if (careful) { a = saturate(a); b = saturate(b); c = saturate(c); d = saturate(d); }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ float lo16(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
// 8 bf16 -> 8 codes
__device__ __forceinline__ u32x2 codes8(u32x4 v, float inv, bool careful) {
  return u32x2{codes4(lo16(v[0]), hi16(v[0]), lo16(v[1]), hi16(v[1]), inv, careful), codes4(lo16(v[2]), hi16(v[2]), lo16(v[3]), hi16(v[3]), inv, careful)};
}
// codes of a block whose exponent grows, factor = 2^(old - new) <= 1
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float factor) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * factor, a[1] * factor, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * factor, b[1] * factor, r, true);
}

// byte mask of word `w` (0 .. 3) of a 16-byte value vector whose half holds tokens 8 h + 16 u + i: bytes of tokens in [a, b)
__device__ __forceinline__ uint32_t token_bytes(int w, int h, int a, int b) {
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int tok = 16 * (w >> 1) + 8 * h + 4 * (w & 1) + k;
    if (tok >= a && tok < b) m |= 0xffu << (8 * k);
  }
  return m;
}

// ---- rows of new tokens ----------------------------------------------------------------------------------------------
// One wave per (sequence, block of 32 positions, group, K or V; 16-bit values of 256 dims are two waves' work): it alone owns what it
// writes, its scale included, so there is nothing to synchronise.  K: a lane takes one token and every second run of 8 dims, which are output vectors as they are.  V: a lane takes
// 4 dims (8 of 256 as codes) and the 16 tokens of an output vector, so that a load covers whole rows of two tokens and the turn from
// token-major to dim-major happens in registers; vectors that others share are stored element by element or, as codes, read, changed and
// written back.  At most four new tokens (a step): a lane takes four dims of each, and codes are stored byte by byte, with no read of
// what is there; only where the block's older codes need a larger exponent is this the long way again.
// More workgroups per block take 8 tokens each, or 2, and rotate: one sine and cosine per (token, pair) in LDS, shared by k_R and all
// heads of the queries; the angle is formed and reduced in double.
// Bound by HBM for prompts and by latency for a step: row bounds and lengths -> page (the rows on their way beside it) -> old scale -> stores.
// Eight ragged prompts of 500 to 4000 tokens, 8 groups: 56 us = 4.6 TB/s read and written (a copy reaches 4.95); 4 of 300 to
// 3000 into the 16-bit cache, (192, 256): 27 to 29 us = 3.6 to 3.9 TB/s (20 us where the last-level cache holds part of it); 64 sequences' two
// tokens x 128 heads 7.0 us; one token 3.7 us.
constexpr int kFew = 4;

template <int DH, int DV, bool BLOCKS>
__global__ void __launch_bounds__(256) append_rows_kernel(AppendRowsArgs a, int kv_groups, int turns_at_once) {
  constexpr int DR = 64;
  __shared__ float cs_tab[8 * DR];   // rotation: (cos, sin) of 8 tokens x 32 pairs
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool rotates = (int)blockIdx.y >= kv_groups;
  double theta = 0.0;
  if (rotates && a.log2_base > 0.0) theta = exp2(-2.0 * (int)(threadIdx.x & 31) / DR * a.log2_base) * 0.15915494309189535;
  RowSpan r;
  if (!find_rows<2>(a.first, a.seq_lens, a.B, a.total, a.s_q, 1, kBlockShift, blockIdx.x, r)) return;
  // positions p0 .. len - 1 are new; this block's share is [lo, hi)
  const int64_t p0 = (int64_t)r.len - r.n;
  const int64_t t0_wide = (max(p0, (int64_t)0) / kBlock + r.k) * kBlock;
  if (t0_wide >= r.len) return;
  const int t0 = (int)t0_wide;
  const int P = a.cache.page_size;
  const int lo = (int)max((int64_t)t0, p0), hi = (int)min((int64_t)t0 + kBlock, (int64_t)r.len);
  const int slot0 = t0 % P, T = slot0 / kBlock, gc = a.g;
  constexpr int EB = BLOCKS ? 1 : 2;
  const int64_t page_bytes = (int64_t)P * (gc * (DH + DV) * EB + DR * 2) + (BLOCKS ? (int64_t)gc * (P / kBlock) * 8 : 0);
  auto look_up = [&](char*& page) {   // false: there is no such page
    const int32_t pg = page_of_uniform(a.cache, r.b, t0 / P);
    page = (char*)a.cache.pool + (int64_t)max(pg, 0) * page_bytes;
    return pg >= 0;
  };
  char* page;

  if (rotates) {   // turns_at_once tokens
    const int s0 = t0 + turns_at_once * ((int)blockIdx.y - kv_groups);
    const int first_t = max(s0, lo), last_t = min(s0 + turns_at_once, hi);
    if (first_t >= last_t) return;
    const int tid = threadIdx.x, tok = tid >> 5;
    float sn = 0.f, cs = 1.f;
    if (a.log2_base > 0.0 && tok < turns_at_once) {
      double turns = (double)(s0 + tok) * theta;
      turns -= floor(turns);
      sincospif(2.0f * (float)turns, &sn, &cs);
    }
    *(f32x2*)(cs_tab + 2 * tid) = f32x2{cs, sn};
    __syncthreads();
    auto turn = [&](u32x4 v, int at) {   // 4 pairs, table entries at, at + 1, ...
      const f32x4 c0 = *(const f32x4*)(cs_tab + 2 * at), c1 = *(const f32x4*)(cs_tab + 2 * at + 4);
      auto one = [](uint32_t w, float c, float s) { return pack_bf16(lo16(w) * c - hi16(w) * s, lo16(w) * s + hi16(w) * c); };
      return u32x4{one(v[0], c0[0], c0[1]), one(v[1], c0[2], c0[3]), one(v[2], c1[0], c1[1]), one(v[3], c1[2], c1[3])};
    };
    const int64_t row0 = r.first + (first_t - p0);
    const int count = last_t - first_t, skip = first_t - s0;
    if (a.q_r) {
      const int per_token = a.h_q * 8, vecs = count * per_token;   // 16-byte vectors
      const u32x4* src = (const u32x4*)a.q_r + row0 * per_token;
      u32x4* dst = (u32x4*)a.q_rot + row0 * per_token;
      for (int base = tid; base < vecs; base += 4 * 256) {
        u32x4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (base + u * 256 < vecs) v[u] = src[base + u * 256];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int idx = base + u * 256;
          if (idx < vecs) dst[idx] = a.log2_base > 0.0 ? turn(v[u], (skip + idx / per_token) * 32 + 4 * (idx & 7)) : v[u];
        }
      }
    }
    if (tid < 8 * count && look_up(page)) {
      const int i = tid >> 3, c = tid & 7;
      const u32x4 v = *(const u32x4*)((const char*)a.k_r + ((row0 + i) * a.kr_stride + 8 * c) * 2);
      char* const plane = page + (int64_t)P * gc * (DH + DV) * EB;
      *(u32x4*)(plane + ((int64_t)c * P + slot0 + first_t - t0 + i) * 16) = a.log2_base > 0.0 ? turn(v, (skip + i) * 32 + 4 * c) : v;
    }
    return;
  }

  // K, then V: codes in one piece (the scale is the whole block's), 16 bits in pieces of 128 dims
  constexpr int VD = BLOCKS ? DV : 128, UNITS = 1 + DV / VD;
  const int item = blockIdx.y * 4 + wave;
  if (item >= UNITS * gc) return;
  const int j = item / UNITS, kind = item % UNITS > 0, v0 = max(item % UNITS - 1, 0) * VD;
  const int n_old = lo - t0;            // older tokens of the block
  const int n_hi = hi - t0;
  const int64_t row0 = r.first + (t0 - p0);   // row of the block's first token (where that is a new one)
  auto scale_at = [&] { return (float*)(page + (int64_t)P * (gc * (DH + DV) + DR * 2)) + ((int64_t)j * (P / kBlock) + T) * 2 + kind; };
  // the block's exponent from the new values and the older tokens'
  auto settle = [&](int e_new, int& e, int& e_old) {
    e_old = e_new;
    if (n_old > 0) e_old = exponent_of(*scale_at());
    e = max(e_new, e_old);
  };
  auto keep = [&](int e, int e_old) {
    if (lane == 0 && (n_old == 0 || e != e_old)) *scale_at() = pow2(e);
  };

  if (n_hi - n_old <= kFew) {           // a step's tokens: a lane takes dims 4 lane .. 4 lane + 3 of each
    const int dims = kind == 0 ? DH : v0 + VD, d = v0 + 4 * lane;
    const int64_t stride = kind == 0 ? a.k_stride : a.v_stride;
    const char* src = (const char*)(kind == 0 ? a.k_c : a.v) + ((row0 + n_old) * stride + (int64_t)j * (kind == 0 ? DH : DV) + d) * 2;
    u32x2 w[kFew];
#pragma unroll
    for (int i = 0; i < kFew; ++i) w[i] = d < dims && n_old + i < n_hi ? *(const u32x2*)(src + i * stride * 2) : u32x2{0, 0};
    asm volatile("" ::: "memory");      // (the rows are asked for ahead of the page)
    if (!look_up(page)) return;
    if constexpr (!BLOCKS) {
#pragma unroll
      for (int i = 0; i < kFew; ++i) {
        const int slot = slot0 + n_old + i;
        if (d >= dims || n_old + i >= n_hi) continue;
        if (kind == 0) {
          *(u32x2*)(page + (((int64_t)j * (DH / 8) + d / 8) * P + slot) * 16 + d % 8 * 2) = w[i];
        } else {
          uint16_t* dst = (uint16_t*)(page + (int64_t)P * gc * DH * 2 + (((int64_t)j * (P / 8) + slot / 8) * DV + d) * 16) + slot % 8;
#pragma unroll
          for (int k = 0; k < 4; ++k) dst[8 * k] = (uint16_t)(w[i][k >> 1] >> (16 * (k & 1)));
        }
      }
      return;
    } else {
      bool careful;
      const int e_new = wave_exponent([&](auto&& f) {
#pragma unroll
        for (int i = 0; i < kFew; ++i) {
          f(w[i][0]);
          f(w[i][1]);
        }
      }, careful);
      int e, e_old;
      settle(e_new, e, e_old);
      if (e == e_old) {                 // (else the older codes change as well: below)
        keep(e, e_old);
        const float inv = pow2(-e);
#pragma unroll
        for (int i = 0; i < kFew; ++i) {
          const int n = n_old + i;
          if (d >= dims || n >= n_hi) continue;
          const uint32_t c = codes4(lo16(w[i][0]), hi16(w[i][0]), lo16(w[i][1]), hi16(w[i][1]), inv, careful);
          if (kind == 0) {
            *(uint32_t*)(page + (((int64_t)j * (DH / 16) + d / 32 * 2 + d / 8 % 2) * P + slot0 + n) * 16 + d / 16 % 2 * 8 + d % 8) = c;
          } else {
            uint8_t* dst = (uint8_t*)(page + (int64_t)P * gc * DH + ((((int64_t)j * (P / kBlock) + T) * DV + d) * 2 + n / 8 % 2) * 16 + n / 16 * 8 + n % 8);
#pragma unroll
            for (int k = 0; k < 4; ++k) dst[32 * k] = (uint8_t)(c >> (8 * k));
          }
        }
        return;
      }
    }
  }

  if (kind == 0) {
    const int n = lane & 31, h = lane >> 5;
    const bool fresh = n >= n_old && n < n_hi;
    const char* src = (const char*)a.k_c + ((row0 + n) * a.k_stride + (int64_t)j * DH + 8 * h) * 2;
    u32x4 w[DH / 16];
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) w[c] = fresh ? *(const u32x4*)(src + c * 32) : u32x4{0, 0, 0, 0};   // dims 16 c + 8 h ..
    asm volatile("" ::: "memory");
    if (!look_up(page)) return;
    if constexpr (!BLOCKS) {
      char* dst = page + (((int64_t)j * (DH / 8) + h) * P + slot0 + n) * 16;
      if (fresh) {
#pragma unroll
        for (int c = 0; c < DH / 16; ++c) *(u32x4*)(dst + (int64_t)c * 32 * P) = w[c];
      }
    } else {
      bool careful;
      const int e_new = wave_exponent([&](auto&& f) {
#pragma unroll
        for (int c = 0; c < DH / 16; ++c)
#pragma unroll
          for (int k = 0; k < 4; ++k) f(w[c][k]);
      }, careful);
      int e, e_old;
      settle(e_new, e, e_old);
      keep(e, e_old);
      const float inv = pow2(-e);
      char* dst = page + (((int64_t)j * (DH / 16) + h) * P + slot0 + n) * 16;
      if (fresh) {
#pragma unroll
        for (int kp = 0; kp < DH / 32; ++kp) {
          const u32x2 x = codes8(w[2 * kp], inv, careful), y = codes8(w[2 * kp + 1], inv, careful);
          *(u32x4*)(dst + (int64_t)kp * 32 * P) = u32x4{x[0], x[1], y[0], y[1]};
        }
      } else if (e != e_old && n < n_old) {
        const float factor = pow2(max(e_old - e, -126));
#pragma unroll
        for (int kp = 0; kp < DH / 32; ++kp) {
          u32x4 x = *(const u32x4*)(dst + (int64_t)kp * 32 * P);
#pragma unroll
          for (int k = 0; k < 4; ++k) x[k] = rescale4(x[k], factor);
          *(u32x4*)(dst + (int64_t)kp * 32 * P) = x;
        }
      }
    }
  } else {
    constexpr int WPL = VD / 64;                 // 32-bit words (pairs of dims) per lane and token
    typedef __attribute__((ext_vector_type(WPL))) uint32_t words_t;
    const int dq = lane & 31, h = lane >> 5, d0 = v0 + 2 * WPL * dq;   // dims d0 ..
    const char* src = (const char*)a.v + (row0 * a.v_stride + (int64_t)j * DV + d0) * 2;
    words_t w[16];                               // token 16 (x / 8) + 8 h + x % 8
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const int n = 16 * (x >> 3) + 8 * h + (x & 7);
      w[x] = words_t{};
      if (n >= n_old && n < n_hi) w[x] = *(const words_t*)(src + n * a.v_stride * 2);
    }
    asm volatile("" ::: "memory");
    if (!look_up(page)) return;
    char* const plane = page + (int64_t)P * gc * DH * EB;
    if constexpr (!BLOCKS) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int n0 = 16 * u + 8 * h;           // tokens n0 .. n0 + 7 of this lane's vectors
        if (n0 + 8 <= n_old || n0 >= n_hi) continue;
        char* dst = plane + (((int64_t)j * (P / 8) + slot0 / 8 + 2 * u + h) * DV + d0) * 16;
        const bool whole = n0 >= n_old && n0 + 8 <= n_hi;
#pragma unroll
        for (int d = 0; d < 2 * WPL; ++d) {
          const uint32_t sel = d & 1 ? 0x07060302u : 0x05040100u;
          u32x4 o;
#pragma unroll
          for (int k = 0; k < 4; ++k) o[k] = __builtin_amdgcn_perm(w[8 * u + 2 * k + 1][d >> 1], w[8 * u + 2 * k][d >> 1], sel);
          if (whole) {
            *(u32x4*)(dst + d * 16) = o;
          } else {                               // the others' elements stay as they are
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (n0 + i >= n_old && n0 + i < n_hi) *(uint16_t*)(dst + d * 16 + 2 * i) = (uint16_t)(o[i >> 1] >> (16 * (i & 1)));
          }
        }
      }
    } else {
      bool careful;
      const int e_new = wave_exponent([&](auto&& f) {
#pragma unroll
        for (int x = 0; x < 16; ++x)
#pragma unroll
          for (int k = 0; k < WPL; ++k) f(w[x][k]);
      }, careful);
      int e, e_old;
      settle(e_new, e, e_old);
      keep(e, e_old);
      const float inv = pow2(-e);
      char* dst = plane + ((((int64_t)j * (P / kBlock) + T) * DV + d0) * 2 + h) * 16;
      const bool whole = n_old == 0 && n_hi == kBlock;
      uint32_t fresh[4], old[4];                 // byte masks of the vector's words
      if (!whole) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          fresh[k] = token_bytes(k, h, n_old, n_hi);
          old[k] = token_bytes(k, h, 0, n_old);
        }
      }
      const float factor = pow2(max(e_old - e, -126));
#pragma unroll
      for (int d = 0; d < 2 * WPL; ++d) {
        u32x4 o;
#pragma unroll
        for (int k = 0; k < 4; ++k) {            // tokens 16 (k / 2) + 8 h + 4 (k % 2) ..
          auto at = [&](int i) { const uint32_t x = w[8 * (k >> 1) + 4 * (k & 1) + i][d >> 1]; return d & 1 ? hi16(x) : lo16(x); };
          o[k] = codes4(at(0), at(1), at(2), at(3), inv, careful);
        }
        if (!whole) {
          const u32x4 x = *(const u32x4*)(dst + d * 32);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t was = x[k];
            if (e != e_old) was = (was & ~old[k]) | (rescale4(was, factor) & old[k]);
            o[k] = (was & ~fresh[k]) | (o[k] & fresh[k]);
          }
        }
        *(u32x4*)(dst + d * 32) = o;
      }
    }
  }
}

// fp32 rows: a workgroup per row, an element per thread and pass (any dims that are multiples of 8; for the small fp32 path).  Single floats of V
// are stored 32 bytes apart: 8 ragged prompts of 500 to 4000 tokens, 8 groups, 593 MB read and written: 237 us = 2.5 TB/s.
__global__ void __launch_bounds__(256) append_rows_f32_kernel(AppendRowsArgs a) {
  RowSpan r;
  if (!find_rows<0>(a.first, a.seq_lens, a.B, a.total, a.s_q, 1, 0, blockIdx.x, r) || r.k >= r.n) return;
  const int64_t t = (int64_t)r.len - r.n + r.k;
  if (t < 0) return;
  const int P = a.cache.page_size, gc = a.g, slot = (int)(t % P);
  const int64_t row = r.first + r.k;
  const int32_t pg = page_of_uniform(a.cache, r.b, (int)(t / P));
  const int nk = gc * a.d_h, nv = gc * a.d_v, half = a.d_r / 2;
  float* const page = (float*)a.cache.pool + (int64_t)(pg >= 0 ? pg : 0) * P * (nk + nv + a.d_r);
  if (pg >= 0) {
    const float* k = (const float*)a.k_c + row * a.k_stride;
    for (int i = threadIdx.x; i < nk; i += 256) page[((int64_t)(i / 8) * P + slot) * 8 + i % 8] = k[i];   // (j, d): vectors j d_h / 8 + d / 8
    const float* v = (const float*)a.v + row * a.v_stride;
    for (int i = threadIdx.x; i < nv; i += 256) {
      const int j = i / a.d_v, d = i % a.d_v;
      page[(int64_t)P * nk + (((int64_t)j * (P / 8) + slot / 8) * a.d_v + d) * 8 + slot % 8] = v[i];
    }
  }
  const float* kr = (const float*)a.k_r + row * a.kr_stride;
  const float* q = (const float*)a.q_r + row * a.h_q * a.d_r;
  float* q_to = (float*)a.q_rot + row * a.h_q * a.d_r;
  for (int p = threadIdx.x; p < half; p += 256) {
    float sn = 0.f, cs = 1.f;
    if (a.log2_base > 0.0) {
      double turns = (double)t * exp2(-2.0 * (double)p / (double)a.d_r * a.log2_base) * 0.15915494309189535;
      turns -= floor(turns);
      sincospif(2.0f * (float)turns, &sn, &cs);
    }
    auto turn = [&](float x, float y, float* to) {
      to[0] = x * cs - y * sn;
      to[1] = x * sn + y * cs;
    };
    if (pg >= 0) turn(kr[2 * p], kr[2 * p + 1], page + (int64_t)P * (nk + nv) + ((int64_t)(p / 4) * P + slot) * 8 + 2 * (p % 4));
    if (a.q_r)
      for (int i = 0; i < a.h_q; ++i) turn(q[i * a.d_r + 2 * p], q[i * a.d_r + 2 * p + 1], q_to + i * a.d_r + 2 * p);
  }
}

// ---- 16-bit expanded cache -> block scales ----------------------------------------------------------------------------------
// One wave per (page, tile of 32 tokens, group, K or V), a wave per tile for k_R behind them.  Both formats are made of
// vectors in the same order, so that loads and stores are runs of whole vectors.  Only bytes that belong to tokens t < L are written.
// Bound by HBM: 32 ragged sequences of 2049 to 6143 tokens, 8 groups (817 MB read and written) 168 us = 4.85 TB/s; 333 tokens 6 us.
template <int DH, int DV>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(QuantizeArgs a) {
  constexpr int DR = 64;
  const int lane = threadIdx.x & 63;
  const int p = blockIdx.x, b = blockIdx.y;
  const int L = a.seq_lens[b], P = a.src.page_size, gc = a.src.groups;
  if ((int64_t)p * P >= L) return;
  const int item = __builtin_amdgcn_readfirstlane(blockIdx.z * 4 + (threadIdx.x >> 6));
  const int tiles = P / kBlock;
  const int T = item % tiles, unit = item / tiles;   // unit: 2 j + kind, 2 g: k_R
  const int valid = (int)min((int64_t)kBlock, (int64_t)L - (int64_t)p * P - T * kBlock);
  if (valid <= 0 || unit > 2 * gc) return;
  const int32_t pg_in = page_of_uniform(a.src, b, p), pg_out = page_of_uniform(a.dst, b, p);
  if (pg_in < 0 || pg_out < 0) return;
  const char* in = (const char*)a.src.pool + (int64_t)pg_in * P * (gc * (DH + DV) + DR) * 2;
  char* out = (char*)a.dst.pool + (int64_t)pg_out * ((int64_t)P * (gc * (DH + DV) + DR * 2) + (int64_t)gc * tiles * 8);
  const int n = lane & 31, h = lane >> 5, slot = T * kBlock + n;
  if (unit == 2 * gc) {
    if (n >= valid) return;
#pragma unroll
    for (int c = 0; c < DR / 16; ++c) {
      const int64_t at = ((int64_t)(2 * c + h) * P + slot) * 16;
      *(u32x4*)(out + (int64_t)P * gc * (DH + DV) + at) = *(const u32x4*)(in + (int64_t)P * gc * (DH + DV) * 2 + at);
    }
    return;
  }
  const int j = unit >> 1;
  float* const scale_at = (float*)(out + (int64_t)P * (gc * (DH + DV) + DR * 2)) + ((int64_t)j * tiles + T) * 2 + (unit & 1);
  bool careful;
  if ((unit & 1) == 0) {
    const char* src = in + (((int64_t)j * (DH / 8) + h) * P + slot) * 16;
    u32x4 w[DH / 16];
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) w[c] = n < valid ? *(const u32x4*)(src + (int64_t)c * 32 * P) : u32x4{0, 0, 0, 0};
    const int e = wave_exponent([&](auto&& f) {
#pragma unroll
      for (int c = 0; c < DH / 16; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k) f(w[c][k]);
    }, careful);
    if (lane == 0) *scale_at = pow2(e);
    const float inv = pow2(-e);
    if (n >= valid) return;
    char* dst = out + (((int64_t)j * (DH / 16) + h) * P + slot) * 16;
#pragma unroll
    for (int kp = 0; kp < DH / 32; ++kp) {
      const u32x2 x = codes8(w[2 * kp], inv, careful), y = codes8(w[2 * kp + 1], inv, careful);
      *(u32x4*)(dst + (int64_t)kp * 32 * P) = u32x4{x[0], x[1], y[0], y[1]};
    }
  } else {
    const char* src = in + (int64_t)P * gc * DH * 2 + (((int64_t)j * (P / 8) + 4 * T + h) * DV + n) * 16;
    u32x4 w[DV / 32][2];
#pragma unroll
    for (int m = 0; m < DV / 32; ++m)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        w[m][u] = *(const u32x4*)(src + ((int64_t)2 * u * DV + 32 * m) * 16);
        if (valid < kBlock) {   // elements behind the last token may hold anything
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int t = 16 * u + 8 * h + 2 * k;
            if (t >= valid) w[m][u][k] = 0;
            else if (t + 1 >= valid) w[m][u][k] &= 0xffffu;
          }
        }
      }
    const int e = wave_exponent([&](auto&& f) {
#pragma unroll
      for (int m = 0; m < DV / 32; ++m)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int k = 0; k < 4; ++k) f(w[m][u][k]);
    }, careful);
    if (lane == 0) *scale_at = pow2(e);
    const float inv = pow2(-e);
    if (8 * h >= valid) return;
    char* dst = out + (int64_t)P * gc * DH + ((((int64_t)j * tiles + T) * DV + n) * 2 + h) * 16;
    const bool whole = 8 * h + 24 <= valid;
    uint32_t mine[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) mine[k] = whole ? ~0u : token_bytes(k, h, 0, valid);
#pragma unroll
    for (int m = 0; m < DV / 32; ++m) {
      const u32x2 x = codes8(w[m][0], inv, careful), y = codes8(w[m][1], inv, careful);
      u32x4 o = {x[0], x[1], y[0], y[1]};
      u32x4* to = (u32x4*)(dst + m * 1024);
      if (!whole) {
        const u32x4 was = *to;
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = (o[k] & mine[k]) | (was[k] & ~mine[k]);
      }
      *to = o;
    }
  }
}

template <int DH, int DV, bool BLOCKS>
hipError_t launch_append(const AppendRowsArgs& a, hipStream_t s) {
  const int kv = ((BLOCKS ? 2 : 1 + DV / 128) * a.g + 3) / 4;
  // Two tokens a workgroup where the rows are few, but more than a step's, so that many heads spread over the chip; eight otherwise, whose
  // table is read four times as often.  (128 heads, eight -> two) 150 rows 10.9 -> 5.9 us, 3700 26.7 -> 25.7, 6000 61.4 -> 58.4, 30000
  // 246 -> 247, 120000 958 -> 995; (32 heads) 750 7.1 -> 6.6, 6000 20.8 -> 20.9, 30000 97 -> 101.
  const int at_once = a.total > 4 * (int64_t)a.B && a.total <= 8192 && a.h_q >= 32 ? 2 : 8;
  append_rows_kernel<DH, DV, BLOCKS><<<dim3((unsigned)row_runs(a.total, 1, kBlockShift, 2, a.B), kv + kBlock / at_once), 256, 0, s>>>(a, kv, at_once);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append_rows_f32(const AppendRowsArgs& a, hipStream_t s) {
  append_rows_f32_kernel<<<(unsigned)a.total, 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_append_rows_bf16(const AppendRowsArgs& a, hipStream_t s) {
  return a.d_h == 192 ? launch_append<192, 256, false>(a, s) : launch_append<128, 128, false>(a, s);
}
hipError_t launch_append_rows_fp8_blocks(const AppendRowsArgs& a, hipStream_t s) {
  return a.d_h == 192 ? launch_append<192, 256, true>(a, s) : launch_append<128, 128, true>(a, s);
}
hipError_t launch_quantize_blocks(const QuantizeArgs& a, int d_h, hipStream_t s) {
  const int items = (2 * a.src.groups + 1) * (a.src.page_size / kBlock);
  const dim3 grid(a.src.max_pages, a.B, (items + 3) / 4);
  if (d_h == 192) quantize_blocks_kernel<192, 256><<<grid, 256, 0, s>>>(a);
  else quantize_blocks_kernel<128, 128><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace gqla
