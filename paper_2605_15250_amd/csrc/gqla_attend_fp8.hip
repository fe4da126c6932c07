// Attention of prompt chunks over the block-scaled 8-bit expanded cache: any number of query rows per sequence, causal.
//
// The query rows of a (sequence, group) are its tokens' heads, rho = t * G + head.  A workgroup of four waves takes 128 of them, 32 a
// wave, and walks the tokens they see in stages of 64, which LDS-DMA brings into a ring of buffers ahead of their use:
//   S^T[token][row] = K Q^T,   O^T[dim][row] += V^T P^T
// with one query row per lane throughout, a running maximum (moved only when outgrown) and an fp32 sum.
//   K Q^T: the codes go into the 8-bit matrix instruction as they lie, their block's power of two in its scale operand.  The queries are
//     the sum of two E4M3 terms, hi = E4M3(q 2^-e) and lo = E4M3((q 2^-e - hi) 2^4), e per row and 64 dims: 4 + 4 bits are the 8 of a
//     bf16, and what subnormal codes lose is below 2^-22 of the largest.  Two products at twice the rate cost what one in bf16 does, and
//     no key code is widened (32 conversions per tile and wave).
//   q_R k_R^T in bf16;  V^T P^T in bf16, value codes widened with their power of two, probabilities rounded to bf16.
// The cache's vectors are operand fragments; a stage in LDS is a row of 1 KB pieces, one per fragment, so that a request writes and a
// read takes 64 consecutive vectors (no bank is met twice).
// Few rows over a long context: the tokens are split into ranges, whose partial outputs a second kernel joins.
#include <algorithm>
#include <atomic>

#include "gqla_lds.h"
#include "gqla_rows.h"

namespace gqla {

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef const __attribute__((address_space(4))) f32x4* const_f32x4_ptr;

__device__ __forceinline__ bf16x8 widen_codes(uint32_t w0, uint32_t w1, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
  const u32x4 r = {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
  return __builtin_bit_cast(bf16x8, r);
}

constexpr int kWaves = 4, kRows = 32 * kWaves, kStage = 64;
constexpr float kRescale = 8.f;   // log2 units by which a maximum may outgrow the reference of the exponentials

template <int DH, int DV>
struct AttendTile {
  static constexpr int KC = DH / 32, KR = 4, MT = DV / 32;             // 1 KB pieces per 32 tokens: K codes, k_R, V codes
  static constexpr int kPieces = 2 * (KC + KR + MT), kPer = kPieces / kWaves;
  static constexpr int kBuffers = DV == 128 ? 3 : 2;
  static constexpr int kPitch = DV * 2 + 16;                           // of an output row on its way through LDS
  static constexpr int kLds = std::max(kBuffers * kPieces * 1024, kRows * kPitch);
  static_assert(2 * KC % kWaves == 0 && 2 * KR % kWaves == 0 && 2 * MT % kWaves == 0, "a wave's pieces are of known kinds");
};

template <int DH, int DV>
__global__ void __launch_bounds__(64 * kWaves, DV == 128 ? 2 : 1) attend_kernel(AttendArgs a, int n_tiles) {
  typedef AttendTile<DH, DV> Tile;
  constexpr int DR = 64, KC = Tile::KC, KR = Tile::KR, MT = Tile::MT, NB = Tile::kBuffers, PIECES = Tile::kPieces;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (workgroups go to the eight dies in turn: with g a multiple or a divisor of 8 a die keeps to its groups' keys and values; the
  // tiles with the most tokens in sight come first)
  const int j = blockIdx.x % a.g, split = blockIdx.x / a.g % a.splits, tile = n_tiles - 1 - (int)(blockIdx.x / (a.g * a.splits));
  RowSpan r;
  if (!find_rows<kRows, 1>(a.first, a.seq_lens, a.B, a.total, a.s_q, a.G, tile, r)) return;
  const int64_t rows = (int64_t)r.n * a.G, tile0 = (int64_t)r.k * kRows;
  if (tile0 >= rows) return;
  const int P = a.cache.page_size, gc = a.g;
  const int64_t cap = (int64_t)a.cache.max_pages * P;
  const int64_t p0 = (int64_t)r.len - r.n;                             // position of the sequence's first row
  auto visible = [&](int64_t rho) { return (int)min(max(p0 + rho / a.G + 1, (int64_t)0), cap); };   // tokens that a row sees
  const int64_t rho0 = tile0 + wave * 32, last = rows - 1;
  const int64_t rho = min(rho0 + n, last);                             // rows behind the last repeat it and are not stored
  const int t = (int)(rho / a.G), head = j * a.G + (int)(rho % a.G);
  const int vis = visible(rho);
  const int vis_min = visible(min(rho0, last)), vis_max = visible(min(rho0 + 31, last));   // of the wave
  const int stages = (int)(((int64_t)visible(min(tile0 + kRows - 1, last)) + kStage - 1) / kStage);
  const int per = (stages + a.splits - 1) / a.splits;
  const int st0 = min(split * per, stages), st1 = min(st0 + per, stages);

  // queries: content as two E4M3 terms per (row, 64 dims), the rotary part in bf16
  const int64_t row = (int64_t)r.first + t;
  i32x8 q_hi[KC / 2], q_lo[KC / 2];
  int q_e[KC / 2];
  bf16x8 qr[KR];
  {
    const char* pc = (const char*)a.q_c + ((row * a.h_q + head) * DH + 8 * h) * 2;
    const __bf16* pr = (const __bf16*)a.q_r + (row * a.h_q + head) * DR + 8 * h;
#pragma unroll
    for (int ks = 0; ks < KR; ++ks) qr[ks] = *(const bf16x8*)(pr + 16 * ks);
#pragma unroll
    for (int x = 0; x < KC / 2; ++x) {
      u32x4 w[4];                                                      // dims 64 x + 16 y + 8 h ..
#pragma unroll
      for (int y = 0; y < 4; ++y) w[y] = *(const u32x4*)(pc + (64 * x + 16 * y) * 2);
      uint32_t top = 0;
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int k = 0; k < 4; ++k) top = max(top, max(w[y][k] & 0x7fffu, w[y][k] >> 16 & 0x7fffu));
      {
        uint32_t r0, r1;   // one scale for the row's 64 dims: a scale operand covers 32 of them, 16 in either half-wave
        half_swap(top, top, r0, r1);
        top = max(r0, r1);
      }
      // smallest e with max |q| <= 448 * 2^e; infinities and NaN (which have to come out as such) leave the scale at its end
      const int e = min(max((int)(((top << 16) + 0x1fffffu) >> 23) - 127 - 8, -100), 120);
      const float inv = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
      q_e[x] = e + 127;
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          const float f0 = bf16_bits_to_float(w[y][k] & 0xffffu) * inv, f1 = bf16_bits_to_float(w[y][k] >> 16) * inv;
          const float f2 = bf16_bits_to_float(w[y][k + 1] & 0xffffu) * inv, f3 = bf16_bits_to_float(w[y][k + 1] >> 16) * inv;
          int c = __builtin_amdgcn_cvt_pk_fp8_f32(f0, f1, 0, false);
          c = __builtin_amdgcn_cvt_pk_fp8_f32(f2, f3, c, true);
          const auto b0 = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), b1 = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
          int l = __builtin_amdgcn_cvt_pk_fp8_f32((f0 - b0[0]) * 16.f, (f1 - b0[1]) * 16.f, 0, false);
          l = __builtin_amdgcn_cvt_pk_fp8_f32((f2 - b1[0]) * 16.f, (f3 - b1[1]) * 16.f, l, true);
          q_hi[x][2 * y + k / 2] = c;
          q_lo[x][2 * y + k / 2] = l;
        }
    }
  }

#pragma unroll
  for (int ks = 0; ks < KR; ++ks) asm volatile("" : "+v"(qr[ks]));      // (waited for here: a wait inside the loop would be one for the requests, too)

  // Where this wave's pieces of a stage begin in a page (32 bits: the host has seen to that), for its first slots; a stage further on
  // in the page adds 64 vectors of 16 bytes to those of K and k_R, 64 * DV bytes to those of V.
  uint32_t off[Tile::kPer];
#pragma unroll
  for (int i = 0; i < Tile::kPer; ++i) {
    const int piece = wave + kWaves * i;                               // [kind][32-token tile][fragment]
    if (kWaves * i < 2 * KC) {
      const int tt = piece / KC, kp = piece % KC;
      off[i] = ((j * (DH / 16) + 2 * kp + h) * P + 32 * tt + n) * 16;
    } else if (kWaves * i < 2 * (KC + KR)) {
      const int p = piece - 2 * KC, tt = p / KR, ks = p % KR;
      off[i] = P * gc * (DH + DV) + ((2 * ks + h) * P + 32 * tt + n) * 16;
    } else {
      const int p = piece - 2 * (KC + KR), tt = p / MT, mt = p % MT;
      off[i] = P * gc * DH + (((j * (P / 32) + tt) * DV + 32 * mt + n) * 2 + h) * 16;
    }
  }
  const uint32_t page_bytes = P * (gc * (DH + DV) + DR * 2) + gc * (P / 32) * 8;
  const uint32_t scale_off = P * (gc * (DH + DV) + DR * 2) + j * (P / 32) * 8;
  const char* const pool = (const char*)a.cache.pool;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem + wave * 1024;
  // A stage: its page (-1: not there) and first slot.  Looked up in order, a stage ahead of the requests.
  struct Stage {
    int32_t page, slot;
  };
  int next_page = st0 * kStage / P, next_slot = st0 * kStage % P;
  auto look_up = [&]() -> Stage {
    const Stage g = {page_of_uniform(a.cache, r.b, next_page), next_slot};
    next_slot += kStage;
    if (next_slot == P) {
      next_slot = 0;
      ++next_page;
    }
    return g;
  };
  auto page_of_stage = [&](Stage g) { return pool + (int64_t)max(g.page, 0) * page_bytes; };   // (one that is not there: any)
  auto request = [&](Stage g, int buf) __attribute__((always_inline)) {
    const char* page = page_of_stage(g);
    const char *kr = page + g.slot * 16, *v = page + g.slot * DV;
    const uint32_t lds = lds0 + buf * (PIECES * 1024);
#pragma unroll
    for (int i = 0; i < Tile::kPer; ++i)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                   :
                   : "s"(lds + kWaves * i * 1024), "v"(off[i]), "s"(kWaves * i < 2 * (KC + KR) ? kr : v)
                   : "memory");
  };
  auto scales_of = [&](Stage g) -> f32x4 {                              // K, V of the stage's first tile, K, V of its second
    return *(const_f32x4_ptr)(uintptr_t)(page_of_stage(g) + scale_off + g.slot / 32 * 8);
  };

  f32x16 o[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[mt][i] = 0.f;
  float m_run = GQLA_NEG_INF, l_run = 0.f;

  // 32 tokens from `tok` on, whose pieces begin at lds (k_R and V behind the K pieces of both tiles)
  auto attend_tile = [&](int tok, const char* k_lds, const char* r_lds, const char* v_lds, float sc_k, float sc_v) __attribute__((always_inline)) {
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
    const int k_e = (int)(__builtin_bit_cast(uint32_t, sc_k) >> 23);
#pragma unroll
    for (int x = 0; x < KC / 2; ++x) {
      const u32x4 k0 = *(const u32x4*)(k_lds + (2 * x) * 1024), k1 = *(const u32x4*)(k_lds + (2 * x + 1) * 1024);
      const i32x8 k = {(int)k0[0], (int)k0[1], (int)k0[2], (int)k0[3], (int)k1[0], (int)k1[1], (int)k1[2], (int)k1[3]};
      s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, q_hi[x], s, 0, 0, 0, k_e, 0, q_e[x]);
      s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, q_lo[x], s, 0, 0, 0, k_e, 0, q_e[x] - 4);
    }
#pragma unroll
    for (int ks = 0; ks < KR; ++ks) s = mfma32(*(const bf16x8*)(r_lds + ks * 1024), qr[ks], s);
    u32x4 v8[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) v8[mt] = *(const u32x4*)(v_lds + mt * 1024);
    // register i of lane (n, h): token tok + 8 (i / 4) + 4 h + i % 4
    if (tok + 32 > vis_min) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (tok + 8 * (i >> 2) + 4 * h + (i & 3) >= vis) s[i] = GQLA_NEG_INF;
      if (tok + 32 > vis_max) {   // codes of tokens that no row of the wave sees may be anything (NaN included)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (tok + 16 * (e >> 3) + 8 * h + (e & 7) >= vis_max) v8[mt][e >> 2] &= ~(0xffu << (8 * (e & 3)));
      }
    }
    float top = fmaxf(s[0], s[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) top = fmaxf(fmaxf(top, s[i]), s[i + 1]);
    top = pair_max(top) * a.scale_log2e;
    if (__builtin_amdgcn_ballot_w64(top > m_run + kRescale) != 0) {
      const float m_new = fmaxf(m_run, top);
      const float alpha = fast_exp2(m_run - (m_new == GQLA_NEG_INF ? 0.f : m_new));
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[mt][i] *= alpha;
    }
    const float m_use = m_run == GQLA_NEG_INF ? 0.f : m_run;
    float p[16], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = fast_exp2(__builtin_fmaf(s[i], a.scale_log2e, -m_use));
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += p[i];
    l_run += sum;
    bf16x8 pf[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      u32x4 w;
      uint32_t r0, r1;
      half_swap(pack_bf16(p[8 * kk], p[8 * kk + 1]), pack_bf16(p[8 * kk + 4], p[8 * kk + 5]), r0, r1);
      w[0] = r0;
      w[2] = r1;
      half_swap(pack_bf16(p[8 * kk + 2], p[8 * kk + 3]), pack_bf16(p[8 * kk + 6], p[8 * kk + 7]), r0, r1);
      w[1] = r0;
      w[3] = r1;
      pf[kk] = __builtin_bit_cast(bf16x8, w);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) o[mt] = mfma32(widen_codes(v8[mt][2 * kk], v8[mt][2 * kk + 1], sc_v), pf[kk], o[mt]);
  };

  if (st0 < st1) {
    Stage g[NB];                                                       // this stage and those ahead
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      g[i] = Stage{-1, 0};
      if (st0 + i < st1) g[i] = look_up();
    }
#pragma unroll
    for (int i = 0; i < NB - 1; ++i)
      if (st0 + i < st1) request(g[i], i);
    f32x4 sc = scales_of(g[0]);
    int buf = 0;
    for (int st = st0; st < st1; ++st) {
      // this stage's requests are the oldest: those of the NB - 2 stages behind it may be on their way still
      if (NB > 2 && st + 1 < st1) {
        static_assert(NB == 2 || Tile::kPer == 6, "the wait is written for this count");
        asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      __syncthreads();                                                 // every wave's share is there; the buffer before is free
      if (st + NB - 1 < st1) request(g[NB - 1], buf == 0 ? NB - 1 : buf - 1);
      const bool there = g[0].page >= 0;
#pragma unroll
      for (int i = 0; i + 1 < NB; ++i) g[i] = g[i + 1];
      const f32x4 now = sc;
      if (st + 1 < st1) sc = scales_of(g[0]);
      if (st + NB < st1) g[NB - 1] = look_up();
      const int tok = st * kStage;
      if (there) {                                                     // a page that is not there holds nothing
        const char* lds = smem + buf * (PIECES * 1024) + lane * 16;
        if (tok < vis_max) attend_tile(tok, lds, lds + 2 * KC * 1024, lds + 2 * (KC + KR) * 1024, now[0], now[1]);
        if (tok + 32 < vis_max)
          attend_tile(tok + 32, lds + KC * 1024, lds + (2 * KC + KR) * 1024, lds + (2 * (KC + KR) + MT) * 1024, now[2], now[3]);
      }
      buf = buf == NB - 1 ? 0 : buf + 1;
    }
  }

  const float l = pair_sum(l_run);
  const float inv = l == 0.f ? 0.f : 1.f / l;                          // 0: nothing visible
  const float lse = l == 0.f ? GQLA_NEG_INF : (m_run + fast_log2(l)) * kLn2;
  const bool row_ok = rho0 + n <= last;
  const int64_t at = row * a.h_q + head;
  if (a.splits == 1) {
    // through LDS, so that rows leave as runs of 16-byte vectors
    __syncthreads();                                                   // the ring is no longer read
    char* const mine = smem + wave * (32 * Tile::kPitch);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(u32x2*)(mine + n * Tile::kPitch + (32 * mt + 8 * q + 4 * h) * 2) =
            u32x2{pack_bf16(o[mt][4 * q] * inv, o[mt][4 * q + 1] * inv), pack_bf16(o[mt][4 * q + 2] * inv, o[mt][4 * q + 3] * inv)};
    if (a.lse && h == 0 && row_ok) a.lse[at] = lse;
    constexpr int LPR = DV / 8;                                        // lanes per row
    const int t_first = (int)(min(rho0, last) / a.G), rest = (int)(min(rho0, last) % a.G);
#pragma unroll
    for (int i = 0; i < 32 * LPR / 64; ++i) {
      const int nr = (i * 64 + lane) / LPR, c = lane % LPR;
      if (rho0 + nr > last) continue;
      const uint32_t k = (uint32_t)(rest + nr), dt = k / (uint32_t)a.G;
      const int64_t to = ((int64_t)r.first + t_first + dt) * a.h_q + j * a.G + (k - dt * a.G);
      *(u32x4*)((__bf16*)a.out + to * DV + 8 * c) = *(const u32x4*)(mine + nr * Tile::kPitch + c * 16);
    }
  } else if (row_ok) {
    const int64_t part = (int64_t)split * a.total * a.h_q + at;
    float* po = a.part_o + part * DV + 4 * h;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(f32x4*)(po + 32 * mt + 8 * q) = f32x4{o[mt][4 * q] * inv, o[mt][4 * q + 1] * inv, o[mt][4 * q + 2] * inv, o[mt][4 * q + 3] * inv};
    if (h == 0) a.part_lse[part] = lse;
  }
}

// Merge of the splits: DV / 4 threads per row, rows of sequences only (packed rows behind the last sequence stay as they are).
template <int DV>
__global__ void __launch_bounds__(256) attend_merge_kernel(AttendArgs a) {
  constexpr int VEC = DV / 4;
  const int64_t rows = (int64_t)a.total * a.h_q;
  const int64_t at = (int64_t)blockIdx.x * (256 / VEC) + threadIdx.x / VEC;
  const int v = threadIdx.x % VEC;
  if (at >= rows) return;
  const int row = (int)(at / a.h_q);
  const int begin = a.first ? min(max(a.first[0], 0), a.total) : 0, end = a.first ? min(max(a.first[a.B], 0), a.total) : a.total;
  if (row < begin || row >= end) return;
  float m = GQLA_NEG_INF;
  for (int s = 0; s < a.splits; ++s) m = fmaxf(m, a.part_lse[s * rows + at]);
  const float m_use = m == GQLA_NEG_INF ? 0.f : m;
  float den = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.splits; ++s) {
    const float w = __expf(a.part_lse[s * rows + at] - m_use);
    den += w;
    if (w > 0.f) acc += w * *(const f32x4*)(a.part_o + (s * rows + at) * DV + 4 * v);
  }
  const float inv = den > 0.f ? 1.f / den : 0.f;
  *(u32x2*)((__bf16*)a.out + at * DV + 4 * v) = u32x2{pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)};
  if (a.lse && v == 0) a.lse[at] = m + __logf(den);
}

// Dynamic LDS beyond 64 KB has to be allowed once per kernel and device.
template <int DH, int DV>
hipError_t allow_lds() {
  static std::atomic<uint64_t> done{0};   // a bit per device
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
  e = hipFuncSetAttribute((const void*)attend_kernel<DH, DV>, hipFuncAttributeMaxDynamicSharedMemorySize, AttendTile<DH, DV>::kLds);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <int DH, int DV>
hipError_t launch_attend(const AttendArgs& a, hipStream_t s) {
  constexpr int kLds = AttendTile<DH, DV>::kLds;
  hipError_t e = allow_lds<DH, DV>();
  if (e != hipSuccess) return e;
  const int64_t tiles = row_runs(a.total, a.G, kRows, 1, a.B);
  attend_kernel<DH, DV><<<(unsigned)(tiles * a.g * a.splits), 64 * kWaves, kLds, s>>>(a, (int)tiles);
  e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const int per = 256 / (DV / 4);
  attend_merge_kernel<DV><<<(unsigned)(((int64_t)a.total * a.h_q + per - 1) / per), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// Ranges of the context: as many as leave the chip's 256 units with about two workgroups each, none shorter than 256 tokens.
int attend_splits(int64_t total, int64_t batch, int h_q, int g, int d_h, int64_t max_tokens) {
  (void)d_h;
  const int64_t groups = row_runs(total, h_q / g, kRows, 1, batch) * g;
  const int64_t want = (512 + groups - 1) / groups, most = (max_tokens + 255) / 256;
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, most, 64}));
}

hipError_t launch_attend_fp8_blocks(const AttendArgs& a, hipStream_t s) {
  return a.d_h == 192 ? launch_attend<192, 256>(a, s) : launch_attend<128, 128>(a, s);
}

}  // namespace gqla
