// Attention of prompt chunks over the block-scaled 8-bit expanded cache: any number of query rows per sequence, causal.
//
// The query rows of a (sequence, group) are its tokens' heads, rho = t * G + head.  A workgroup of four waves takes 128 of them, 32 a
// wave (or 64, where 128 leave too few workgroups), and walks the tokens they see in stages of 64, which LDS-DMA brings into a ring of
// buffers ahead of their use:
//   S^T[token][row] = K Q^T,   O^T[dim][row] += V^T P^T
// with one query row per lane throughout, a running maximum (moved only when outgrown) and fp32 sums.
// Codes are widened to bf16 with their block's power of two, exactly, right before their products; probabilities are rounded to bf16, up to
// 2^-8 of each.  The output's denominator sums them as rounded: a token that dominates a row then carries its rounding on both sides (with the
// maximum lagging by up to 2^8 its probability is not 1).  The log-sum-exp takes the sum ahead of the rounding, as exact as fp32 has it.
// (The 8-bit matrix instruction takes key codes as they are, with the queries as the sum of two E4M3 terms: two prompts of 2500 to 4000 tokens x
// 128 heads then take 1042 us instead of 1107.  But it aligns the products of a sum to 2^-14 of the largest, where those in bf16 are
// summed in fp32: logits were 3e-4 off.)
// The cache's vectors are operand fragments; a stage in LDS is a row of 1 KB pieces, one per fragment, so that a request writes and a
// read takes 64 consecutive vectors (no bank is met twice).
// Few rows over a long context: the tokens are split into ranges, whose partial outputs a second kernel joins.
// Bound by the matrix cores on whole prompts: two of 2500 to 4000 tokens behind up to 500 x 128 heads 1108 to 1171 us = 1.01 to 1.07 PFLOP/s on
// different cards, pipes busy 55 % of the cycles (a large product of bf16 matrices reaches 1.15).  9 to 16 tokens x 32 heads over 20000 to
// 32000, two sequences: 31 us and 6 of the merge, 14 stages in a row per workgroup.  (Times further down that compare two forms were
// taken ahead of the second sum, which adds 3 % to whole prompts, 1 to 2 % to the rest.)
#include <algorithm>
#include <cmath>

#include "gqla_lds.h"
#include "gqla_rows.h"

namespace gqla {

namespace {

typedef const __attribute__((address_space(4))) f32x4* const_f32x4_ptr;

__device__ __forceinline__ bf16x8 widen_codes(uint32_t w0, uint32_t w1, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
  const u32x4 r = {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
  return __builtin_bit_cast(bf16x8, r);
}

// NaN codes are 0x7f and 0xff: bit 7 of their bytes, and a word with 0 in their place.
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t without_nans(uint32_t w) {
  const uint32_t bits = nan_codes(w);
  return w & ~(bits | (bits - (bits >> 7)));
}
// Which outputs of a 32x32 tile have a NaN in sight: the product of the indicators [code is NaN] and [row sees the token].  codes: value operand
// of two k-steps (byte e: token 16 (e / 8) + 8 h + e % 8); limit: tokens of the tile that this lane's row sees.  0 or NaN per output.
__device__ __forceinline__ f32x16 seen_nans(const u32x4& codes, int limit, int h) {
  f32x16 r;
#pragma unroll
  for (int i = 0; i < 16; ++i) r[i] = 0.f;
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    u32x4 sees;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int t = 16 * kk + 8 * h + 2 * k;
      sees[k] = (t < limit ? 0x3f80u : 0u) | (t + 1 < limit ? 0x3f800000u : 0u);
    }
    constexpr uint32_t kOne = 0x38;   // the code of 1
    r = mfma32(widen_codes((nan_codes(codes[2 * kk]) >> 7) * kOne, (nan_codes(codes[2 * kk + 1]) >> 7) * kOne, 1.f), __builtin_bit_cast(bf16x8, sees), r);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) r[i] = r[i] > 0.f ? __builtin_nanf("") : 0.f;
  return r;
}

constexpr int kWaves = 4, kRows = 32 * kWaves, kStage = 64;
constexpr float kRescale = 8.f;   // log2 units by which a maximum may outgrow the reference of the exponentials

template <int DH, int DV>
struct AttendTile {
  static constexpr int KC = DH / 32, KR = 4, MT = DV / 32;             // 1 KB pieces per 32 tokens: K codes, k_R, V codes
  static constexpr int kPieces = 2 * (KC + KR + MT), kPer = kPieces / kWaves;
  static constexpr int kPitch = DV * 2 + 16;                           // of an output row on its way through LDS
  static constexpr int kState = MT * 4096 + 768;                       // a wave's O^T, maxima and both sums on their way to another wave
  // Workgroups of a compute unit: registers allow three (two with value dims of 256), and two stages in the ring leave LDS for them.
  // (Three stages and two workgroups: a few rows over 20000 to 32000 tokens 41 us as well, 64 sequences of 2500 to 5000 158 us instead of 125.)
  static constexpr int kPerUnit = DV == 128 ? 3 : 2;
  static constexpr int kLds = std::max(2 * kPieces * 1024, std::max(kRows * kPitch, 2 * kState));
  static_assert(2 * KC % kWaves == 0 && 2 * KR % kWaves == 0 && 2 * MT % kWaves == 0, "a wave's pieces are of known kinds");
};

template <int DH, int DV>
__global__ void __launch_bounds__(64 * kWaves, (AttendTile<DH, DV>::kPerUnit)) attend_kernel(AttendArgs a, int n_tiles, int spread) {
  typedef AttendTile<DH, DV> Tile;
  constexpr int DR = 64, KC = Tile::KC, KR = Tile::KR, MT = Tile::MT, PIECES = Tile::kPieces;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Workgroups go to the eight dies in turn.  Many tiles of rows a sequence: with g a multiple or a divisor of 8 a die keeps to its groups'
  // keys and values, which its L2 then holds for all of them; the tiles with the most tokens in sight come first.  One tile (spread):
  // the groups of a (tile, range) stay on one die, for the k_R that they share.
  int j, unit;
  if (spread) {
    const int k = blockIdx.x >> 3;
    j = k % a.g;
    unit = k / a.g * 8 + (blockIdx.x & 7);
    if (unit >= n_tiles * a.splits) return;
  } else {
    j = blockIdx.x % a.g;
    unit = blockIdx.x / a.g;
  }
  const int split = unit % a.splits, tile = n_tiles - 1 - unit / a.splits;
  RowSpan r;
  if (!find_rows<1>(a.first, a.seq_lens, a.B, a.total, a.s_q, a.G, a.tile_shift, tile, r)) return;
  const int rows = r.n * a.G, tile0 = r.k << a.tile_shift;             // (the host has seen to 32 bits)
  if (tile0 >= rows) return;
  const int P = a.cache.page_size, gc = a.g;
  const int64_t cap = (int64_t)a.cache.max_pages * P;
  auto token = [&](int rho) { return (int)a.by_G(rho); };              // of the sequence's rows
  const int before = r.len - r.n;                                      // tokens ahead of the sequence's first row
  auto visible = [&](int rho) { return (int)min((int64_t)max(before + token(rho) + 1, 0), cap); };   // tokens that a row sees
  // Waves that would have no rows help the others: with at most 64 rows in the tile two teams, with at most 32 four, take the
  // tiles of 32 tokens in turn and join their states at the end.
  const int last = min(rows, tile0 + (1 << a.tile_shift)) - 1;
  const int team_bits = last - tile0 < 32 ? 2 : last - tile0 < 64 ? 1 : 0, row_waves = kWaves >> team_bits;
  const int team = wave >> (2 - team_bits), row_wave = wave & (row_waves - 1);
  const int rho0 = tile0 + row_wave * 32;
  const int rho = min(rho0 + n, last);                                 // rows behind the last repeat it and are not stored
  const int t = token(rho), head = j * a.G + rho - t * a.G;
  const int vis = (int)min((int64_t)max(before + t + 1, 0), cap);
  const int vis_min = visible(min(rho0, last)), vis_max = visible(min(rho0 + 31, last));   // of the wave
  const int stages = (int)(((int64_t)visible(last) + kStage - 1) / kStage);
  const int per = (stages + a.splits - 1) / a.splits;
  const int st0 = min(split * per, stages), st1 = min(st0 + per, stages);

  const int64_t row = (int64_t)r.first + t;
  bf16x8 qc[2 * KC], qr[KR];
  {
    const __bf16* pc = (const __bf16*)a.q_c + (row * a.h_q + head) * DH + 8 * h;
    const __bf16* pr = (const __bf16*)a.q_r + (row * a.h_q + head) * DR + 8 * h;
#pragma unroll
    for (int ks = 0; ks < 2 * KC; ++ks) qc[ks] = *(const bf16x8*)(pc + 16 * ks);
#pragma unroll
    for (int ks = 0; ks < KR; ++ks) qr[ks] = *(const bf16x8*)(pr + 16 * ks);
  }

  // Where this wave's pieces of a stage begin in a page (32 bits: the host has seen to that), for its first slots; a stage further on
  // in the page adds 64 vectors of 16 bytes to those of K and k_R, 64 * DV bytes to those of V.
  const uint32_t off_k = (h * P + n) * 16, off_v = (n * 2 + h) * 16;   // this lane's vector of a piece
  uint32_t piece_at[Tile::kPer];
#pragma unroll
  for (int i = 0; i < Tile::kPer; ++i) {
    const int piece = wave + kWaves * i;                               // [kind][32-token tile][fragment]
    if (kWaves * i < 2 * KC) {
      const int tt = piece / KC, kp = piece % KC;
      piece_at[i] = ((j * (DH / 16) + 2 * kp) * P + 32 * tt) * 16;
    } else if (kWaves * i < 2 * (KC + KR)) {
      const int p = piece - 2 * KC, tt = p / KR, ks = p % KR;
      piece_at[i] = P * gc * (DH + DV) + (2 * ks * P + 32 * tt) * 16;
    } else {
      const int p = piece - 2 * (KC + KR), tt = p / MT, mt = p % MT;
      piece_at[i] = P * gc * DH + ((j * (P / 32) + tt) * DV + 32 * mt) * 32;
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
                   : "s"(lds + kWaves * i * 1024), "v"(kWaves * i < 2 * (KC + KR) ? off_k : off_v), "s"((kWaves * i < 2 * (KC + KR) ? kr : v) + piece_at[i])
                   : "memory");
  };
  auto scales_of = [&](Stage g) -> f32x4 {                              // K, V of the stage's first tile, K, V of its second
    return *(const_f32x4_ptr)(uintptr_t)(page_of_stage(g) + scale_off + g.slot / 32 * 8);
  };

  Stage here = {-1, 0}, next = here;                                   // this stage; the next one, looked up a stage ahead of its request
  f32x4 sc = {1.f, 1.f, 1.f, 1.f};
  if (st0 < st1) {                                                     // the first stage comes while the queries do
    here = look_up();
    request(here, 0);
    sc = scales_of(here);
    if (st0 + 1 < st1) next = look_up();
  }
#pragma unroll
  for (int ks = 0; ks < 2 * KC; ++ks) asm volatile("" : "+v"(qc[ks]));
#pragma unroll
  for (int ks = 0; ks < KR; ++ks) asm volatile("" : "+v"(qr[ks]));      // (waited for here: a wait inside the loop would be one for the requests, too)

  f32x16 o[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[mt][i] = 0.f;
  bool had_nans = false;                                               // among values that only some of the wave's rows see
  float m_run = GQLA_NEG_INF, l_run = 0.f, d_run = 0.f;                // l, d: sums of the probabilities as they are, as rounded
  const int key_lane = (32 * h + (n & 19) + ((n & 4) << 1) + ((n & 8) >> 1)) * 16;

  // 32 tokens from `tok` on, whose pieces begin at lds (k_R and V behind the K pieces of both tiles).  Lane n takes the keys of token
  // n with bits 2 and 3 exchanged: register i of the scores in lane (n, h) is then token 16 (i / 8) + 8 h + i % 8, which is the token
  // order of the other operand's fragments, and probabilities need no exchange between the half-waves.
  auto attend_tile = [&](int tok, const char* k_lds, const char* r_lds, const char* v_lds, float sc_k, float sc_v) __attribute__((always_inline)) {
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int kp = 0; kp < KC; ++kp) {
      const u32x4 k8 = *(const u32x4*)(k_lds + kp * 1024);
      s = mfma32(widen_codes(k8[0], k8[1], sc_k), qc[2 * kp], s);
      s = mfma32(widen_codes(k8[2], k8[3], sc_k), qc[2 * kp + 1], s);
    }
#pragma unroll
    for (int ks = 0; ks < KR; ++ks) s = mfma32(*(const bf16x8*)(r_lds + ks * 1024), qr[ks], s);
    if (tok + 32 > vis_min) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (tok + 16 * (i >> 3) + 8 * h + (i & 7) >= vis) s[i] = GQLA_NEG_INF;
    }
    float top = fmaxf(s[0], s[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) top = fmaxf(fmaxf(top, s[i]), s[i + 1]);
    if (__builtin_amdgcn_ballot_w64(top * a.scale_log2e > m_run + kRescale) != 0) {
      const float m_new = fmaxf(m_run, pair_max(top) * a.scale_log2e);
      const float alpha = fast_exp2(m_run - (m_new == GQLA_NEG_INF ? 0.f : m_new));
      m_run = m_new;
      l_run *= alpha;
      d_run *= alpha;
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
    sum = 0.f;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const u32x4 w = {pack_bf16(p[8 * kk], p[8 * kk + 1]), pack_bf16(p[8 * kk + 2], p[8 * kk + 3]),
                       pack_bf16(p[8 * kk + 4], p[8 * kk + 5]), pack_bf16(p[8 * kk + 6], p[8 * kk + 7])};
      pf[kk] = __builtin_bit_cast(bf16x8, w);
#pragma unroll
      for (int k = 0; k < 4; ++k) sum = add_bf16_pair(w[k], sum);
    }
    d_run += sum;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      u32x4 v8 = *(const u32x4*)(v_lds + mt * 1024);
      if (tok + 32 > vis_min) {
        // a weight of 0 does not keep a NaN away from a row (0 * NaN = NaN): they are taken out, and the rows that see them get them at the end
        const uint32_t found = nan_codes(v8[0]) | nan_codes(v8[1]) | nan_codes(v8[2]) | nan_codes(v8[3]);
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(found != 0) != 0, 0)) {
          uint32_t seen = 0;                                           // (slots that no row sees may hold anything)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int count = min(max(vis_max - tok - 16 * (k >> 1) - 8 * h - 4 * (k & 1), 0), 4);
            seen |= nan_codes(v8[k]) & (uint32_t)((1ull << (8 * count)) - 1);
            v8[k] = without_nans(v8[k]);
          }
          had_nans |= __builtin_amdgcn_ballot_w64(seen != 0) != 0;
        }
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) o[mt] = mfma32(widen_codes(v8[2 * kk], v8[2 * kk + 1], sc_v), pf[kk], o[mt]);
    }
  };

  for (int st = st0; st < st1; ++st) {
    const int buf = (st - st0) & 1;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                                                   // every wave's share is there; the other buffer is free
    if (st + 1 < st1) request(next, buf ^ 1);
    const bool there = here.page >= 0;
    here = next;
    const f32x4 now = sc;
    if (st + 1 < st1) sc = scales_of(here);
    if (st + 2 < st1) next = look_up();
    const int tok = st * kStage;
    if (there) {                                                       // a page that is not there holds nothing
      const char *ring = smem + buf * (PIECES * 1024), *keys = ring + key_lane, *vals = ring + 2 * (KC + KR) * 1024 + lane * 16;
      // tile q of 32 tokens is team q mod teams's
      const int teams = 1 << team_bits, first = 2 * st & (teams - 1);
      if (tok < vis_max && team == first) attend_tile(tok, keys, keys + 2 * KC * 1024, vals, now[0], now[1]);
      if (tok + 32 < vis_max && team == (first + 1 & (teams - 1)))
        attend_tile(tok + 32, keys + KC * 1024, keys + (2 * KC + KR) * 1024, vals + MT * 1024, now[2], now[3]);
    }
  }
  if (__builtin_expect(had_nans, 0)) {                                 // what was taken out: those tiles' values once more
    for (int tok = max(vis_min & ~31, st0 * kStage); tok < min((int64_t)vis_max, (int64_t)st1 * kStage); tok += 32) {
      const int32_t pg = page_of_uniform(a.cache, r.b, tok / P);
      const char* codes = pool + (int64_t)max(pg, 0) * page_bytes + (uint32_t)(P * gc * DH + (j * (P / 32) + tok % P / 32) * DV * 32) + off_v;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) o[mt] += seen_nans(*(const u32x4*)(codes + mt * 1024), pg >= 0 ? vis - tok : 0, h);
    }
  }
  // the teams' states become one, half of them at a time
  for (int half = 1 << team_bits >> 1; half > 0; half >>= 1) {
    __syncthreads();                                                   // the ring, then the states before, are no longer read
    char* const state = smem + ((team & (half - 1)) * row_waves + row_wave) * Tile::kState;
    if (team >= half && team < 2 * half) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int q = 0; q < 4; ++q) *(f32x4*)(state + ((mt * 4 + q) * 64 + lane) * 16) = f32x4{o[mt][4 * q], o[mt][4 * q + 1], o[mt][4 * q + 2], o[mt][4 * q + 3]};
      *(float*)(state + MT * 4096 + lane * 4) = m_run;
      *(float*)(state + MT * 4096 + 256 + lane * 4) = l_run;
      *(float*)(state + MT * 4096 + 512 + lane * 4) = d_run;
    }
    __syncthreads();
    if (team < half) {
      const float m_other = *(const float*)(state + MT * 4096 + lane * 4), l_other = *(const float*)(state + MT * 4096 + 256 + lane * 4);
      const float m_new = fmaxf(m_run, m_other), m_use = m_new == GQLA_NEG_INF ? 0.f : m_new;
      const float mine = fast_exp2(m_run - m_use), other = fast_exp2(m_other - m_use);
      m_run = m_new;
      l_run = l_run * mine + l_other * other;
      d_run = d_run * mine + *(const float*)(state + MT * 4096 + 512 + lane * 4) * other;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 x = *(const f32x4*)(state + ((mt * 4 + q) * 64 + lane) * 16);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[mt][4 * q + i] = o[mt][4 * q + i] * mine + x[i] * other;
        }
    }
  }

  const float l = pair_sum(l_run), d = pair_sum(d_run);
  const float inv = d == 0.f ? 0.f : 1.f / d;                          // 0: nothing visible
  const float lse = l == 0.f ? GQLA_NEG_INF : (m_run + fast_log2(l)) * kLn2;
  const bool row_ok = rho0 + n <= last;
  const int64_t at = row * a.h_q + head;
  if (a.splits == 1) {
    // through LDS, so that rows leave as runs of 16-byte vectors
    __syncthreads();                                                   // the ring (or a state) is no longer read
    if (team > 0) return;
    char* const mine = smem + row_wave * (32 * Tile::kPitch);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(u32x2*)(mine + n * Tile::kPitch + (32 * mt + 8 * q + 4 * h) * 2) =
            u32x2{pack_bf16(o[mt][4 * q] * inv, o[mt][4 * q + 1] * inv), pack_bf16(o[mt][4 * q + 2] * inv, o[mt][4 * q + 3] * inv)};
    if (a.lse && h == 0 && row_ok) a.lse[at] = lse;
    constexpr int LPR = DV / 8;                                        // lanes per row
#pragma unroll
    for (int i = 0; i < 32 * LPR / 64; ++i) {
      const int nr = (i * 64 + lane) / LPR, c = lane % LPR;
      if (rho0 + nr > last) continue;
      const int tk = token(rho0 + nr);
      const int64_t to = ((int64_t)r.first + tk) * a.h_q + j * a.G + (rho0 + nr - tk * a.G);
      *(u32x4*)((__bf16*)a.out + to * DV + 8 * c) = *(const u32x4*)(mine + nr * Tile::kPitch + c * 16);
    }
  } else if (row_ok && team == 0) {
    const int64_t part = (int64_t)split * a.total * a.h_q + at;
    if (h == 0) a.part_lse[part] = lse;
    if (st0 >= st1) return;                                            // (nothing in this range: the weight of -inf is 0)
    float* po = a.part_o + part * DV + 4 * h;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(f32x4*)(po + 32 * mt + 8 * q) = f32x4{o[mt][4 * q] * inv, o[mt][4 * q + 1] * inv, o[mt][4 * q + 2] * inv, o[mt][4 * q + 3] * inv};
  }
}

// Joins the splits' partial outputs.  DV / 4 threads hold a row's vectors; as many slices of the splits as a workgroup has room for
// (slices, a power of two) are merged side by side, each with a running maximum, and meet in LDS.  Rows of sequences only:
// packed rows behind the last one stay as they are.
template <int DV>
__global__ void __launch_bounds__(256) attend_merge_kernel(AttendArgs a, int slices) {
  constexpr int VEC = DV / 4, GROUPS = 256 / VEC, AT_ONCE = 4;
  __shared__ f32x4 acc_lds[GROUPS][VEC];
  __shared__ float m_lds[GROUPS], den_lds[GROUPS];
  const int64_t rows = (int64_t)a.total * a.h_q;
  const int group = threadIdx.x / VEC, v = threadIdx.x % VEC, slice = group & (slices - 1);
  const int64_t at = (int64_t)blockIdx.x * (GROUPS / slices) + group / slices;
  const int begin = a.first ? min(max(a.first[0], 0), a.total) : 0, end = a.first ? min(max(a.first[a.B], 0), a.total) : a.total;
  const bool ok = at >= (int64_t)begin * a.h_q && at < (int64_t)end * a.h_q;
  float m = GQLA_NEG_INF, den = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (ok) {
    for (int s = slice; s < a.splits; s += AT_ONCE * slices) {
      float l[AT_ONCE];
      f32x4 x[AT_ONCE];
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const int su = s + u * slices;
        l[u] = GQLA_NEG_INF;
        x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (su < a.splits) l[u] = a.part_lse[su * rows + at];
      }
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u)
        if (l[u] != GQLA_NEG_INF) x[u] = *(const f32x4*)(a.part_o + ((s + u * slices) * rows + at) * DV + 4 * v);
      float m_new = m;
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) m_new = fmaxf(m_new, l[u]);
      const float m_use = m_new == GQLA_NEG_INF ? 0.f : m_new, old = __expf(m - m_use);
      m = m_new;
      den *= old;
      acc *= old;
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const float w = __expf(l[u] - m_use);
        den += w;
        acc += w * x[u];
      }
    }
  }
  if (slices > 1) {
    acc_lds[group][v] = acc;
    if (v == 0) {
      m_lds[group] = m;
      den_lds[group] = den;
    }
    __syncthreads();
    if (slice > 0) return;
    for (int s = 1; s < slices; ++s) m = fmaxf(m, m_lds[group + s]);
    const float m_use = m == GQLA_NEG_INF ? 0.f : m, mine = __expf(m_lds[group] - m_use);
    den *= mine;
    acc *= mine;
    for (int s = 1; s < slices; ++s) {
      const float w = __expf(m_lds[group + s] - m_use);
      den += w * den_lds[group + s];
      acc += w * acc_lds[group + s][v];
    }
  }
  if (!ok) return;
  const float inv = den == 0.f ? 0.f : 1.f / den;
  *(u32x2*)((__bf16*)a.out + at * DV + 4 * v) = u32x2{pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)};
  if (a.lse && v == 0) a.lse[at] = den == 0.f ? GQLA_NEG_INF : m + __logf(den);
}

// tiles of rows of a sequence, if all have as many
int64_t sequence_tiles(int64_t total, int64_t batch, int64_t G, int shift) {
  return std::max<int64_t>(1, (total * G + (batch << shift) - 1) / (batch << shift));
}

template <int DH, int DV>
hipError_t launch_attend(const AttendArgs& a, hipStream_t s) {
  static DynamicLds lds;
  hipError_t e = lds.allow((const void*)attend_kernel<DH, DV>, AttendTile<DH, DV>::kLds);
  if (e != hipSuccess) return e;
  const int64_t tiles = row_runs(a.total, a.G, a.tile_shift, 1, a.B), units = tiles * a.splits;
  // (spread: 64 sequences of 2500 to 5000 tokens, 8 groups, 4 to 8 rows of 4 heads each: 138 -> 123 us; 32 of 4000 to 6000, 4 rows of 16: 101 -> 93)
  const bool spread = sequence_tiles(a.total, a.B, a.G, a.tile_shift) == 1;
  attend_kernel<DH, DV><<<(unsigned)((spread ? (units + 7) / 8 * 8 : units) * a.g), 64 * kWaves, AttendTile<DH, DV>::kLds, s>>>(a, (int)tiles, spread);
  e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  // slices until there are 1024 workgroups (4 chunks of 100 to 512 tokens x 20 heads, two ranges: 67 -> 65 us against a slice per range)
  constexpr int kGroups = 256 / (DV / 4);
  int slices = 1;
  while (2 * slices <= a.splits && 2 * slices <= kGroups && (int64_t)a.total * a.h_q * slices < 1024 * kGroups) slices *= 2;
  const int per = kGroups / slices;
  attend_merge_kernel<DV><<<(unsigned)(((int64_t)a.total * a.h_q + per - 1) / per), 256, 0, s>>>(a, slices);
  return hipGetLastError();
}

}  // namespace

// Rows of a tile (2^7, or 2^6 for which two teams of waves share the tokens) and ranges that the tokens are split into: the pair with
// the smallest time by this model, in microseconds, of the 256 units, for sequences that all have max_tokens (the lengths are on the device):
//   N = groups * tiles * splits workgroups of ceil(stages / splits) stages each (2.5 more for their start and end);
//   a stage takes the k workgroups that share a unit stage[k] together.  k goes up to 3 (2 with value dims of 256);
//   up to N = 256 k the workgroups with the most tokens in sight end last, beyond that a unit has N / (256 k) turns of the mean number
//   of tokens in sight, and 0.15 of a turn in which units run out of work;
//   a merge costs 6.5 us and the partial outputs, written and read at 2.4 TB/s.
// The rates are fits to sweeps of 1 to 32 ranges and both tiles, off by 11 %; over 19 shapes the pair it takes is 1 % behind the best of the
// sweep, tiles of 128 rows alone 6 %.  (128 rows, 64 rows) 1 prompt of 1000 x 32 heads: 38, 29 us; 1 of 2500 x 16 heads in one group: 69, 60; 4 chunks
// of 100 to 512 x 20 heads in 5 groups over 1000 to 3000: 76 (4 ranges), 68 (2); 8 tokens x 128 heads over 20000: 38, 35 (32); 1 prompt of
// 3000 x 32 heads: 121, 124; 8 of 500 to 1000: 78, 87.  (ranges, at their better tile) 9 to 16 tokens x 32 heads, two over 20000 to
// 32000: 518 (1), 51 (16), 41 (32) us; 8 of 4 to 8 x 128 heads over 10000 to 20000: 372 (1), 100 (12), 121 (32); 8 chunks of 100 to 200 x 32 heads
// over 2500 to 5000: 142 (1), 144 (2), 151 (3); the same without a context: 23 (1), 39 (2).
void attend_shape(int64_t total, int64_t batch, int h_q, int g, int d_h, int64_t max_tokens, int32_t* splits, int32_t* tile_shift) {
  static constexpr double kStageTime[2][2][3] = {{{2.0, 2.65, 3.2}, {1.3, 1.7, 2.2}}, {{2.5, 3.25}, {1.7, 2.15}}};
  const int64_t G = h_q / g, stages = (max_tokens + kStage - 1) / kStage;
  const bool wide = d_h == 192, few = total * G <= 64 * batch;         // few: a tile of 128 is one of 64 or less
  const int per_unit = wide ? 2 : 3;
  const double part_us = (double)total * h_q * (wide ? 256 : 128) * 4 / 2.4e6;
  const double mean = std::max(0.5, 1 - 0.5 * total / ((double)batch * max_tokens));   // tokens that a row sees, of the most
  const int most = total * h_q >= (1 << 24) ? 1 : 64;                  // (the merge has a workgroup per row at the most)
  double best = INFINITY;
  *splits = 1;
  *tile_shift = 7;
  for (int shift = 7; shift >= (few ? 7 : 6); --shift) {
    const double* stage = kStageTime[wide][few || shift == 6];
    const double tiles = (double)(sequence_tiles(total, batch, G, shift) * batch * g);
    for (int s = 1; s <= most && (s == 1 || s <= stages); ++s) {
      const double n = tiles * s / 256, length = (double)((stages + s - 1) / s);
      const int k = (int)std::ceil(std::min(n, (double)per_unit));
      double us = n > k ? ((length * mean + 2.5) * n / k + 0.15 * (length + 2.5)) * stage[k - 1]
                        : (length + 2.5) * (mean + (1 - mean) / k) * stage[k - 1];
      if (s > 1) us += 6.5 + s * part_us;
      if (us < best) {
        best = us;
        *splits = s;
        *tile_shift = shift;
      }
    }
  }
}

hipError_t launch_attend_fp8_blocks(const AttendArgs& a, hipStream_t s) {
  return a.d_h == 192 ? launch_attend<192, 256>(a, s) : launch_attend<128, 128>(a, s);
}

}  // namespace gqla
