// Attention of prompt chunks over the block-scaled 8-bit expanded cache: any number of query rows per sequence, causal.
//
// The query rows of a (sequence, group) are its tokens' heads, rho = t * G + head: 32 of them per wave, kept as B operands in
// registers, against tiles of 32 cached tokens whose vectors are A operands as they lie in the cache (codes widened with their
// block's power of two):  S^T[token][row] = K Q^T,  O^T[dim][row] += V^T P^T,  one query row per lane throughout, with a running maximum
// and sum (in fp32, base 2).
#include <algorithm>

#include "gqla_rows.h"

namespace gqla {

namespace {

__device__ __forceinline__ bf16x8 widen_codes(uint32_t w0, uint32_t w1, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
  const u32x4 r = {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
  return __builtin_bit_cast(bf16x8, r);
}

constexpr int kAttendWaves = 4;

template <int DH, int DV>
__global__ void __launch_bounds__(64 * kAttendWaves) attend_kernel(AttendArgs a, int n_tiles) {
  constexpr int DR = 64, R = 32 * kAttendWaves;
  constexpr int KC = DH / 32, KR = DR / 16, MT = DV / 32;   // pairs of k-steps over the content dims, k-steps of k_R, 32-dim tiles of the output
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = blockIdx.x % a.g, split = blockIdx.x / a.g % a.splits, tile = n_tiles - 1 - (int)(blockIdx.x / (a.g * a.splits));
  RowSpan r;
  if (!find_rows<R, 1>(a.first, a.seq_lens, a.B, a.total, a.s_q, a.G, tile, r)) return;
  const int64_t rows = (int64_t)r.n * a.G, rho0 = (int64_t)r.k * R + wave * 32;
  if (rho0 >= rows) return;
  const int64_t rho = rho0 + n;
  const bool row_ok = rho < rows;
  const int t = (int)((row_ok ? rho : rows - 1) / a.G), head = j * a.G + (int)((row_ok ? rho : rows - 1) % a.G);
  const int P = a.cache.page_size, gc = a.g;
  const int64_t cap = (int64_t)a.cache.max_pages * P;
  const int64_t p0 = (int64_t)r.len - r.n;                       // position of the sequence's first row
  auto visible = [&](int64_t tok) { return (int)min(max(p0 + tok + 1, (int64_t)0), cap); };   // cached tokens that row `tok` sees
  const int vis = visible(t);
  const int vis_min = visible(rho0 / a.G), vis_max = visible((min(rho0 + 31, rows - 1)) / a.G);
  const int tiles = (int)(((int64_t)vis_max + 31) / 32), per = (tiles + a.splits - 1) / a.splits;
  const int tok_begin = split * per * 32, tok_end = (int)min((int64_t)tiles * 32, (int64_t)(split + 1) * per * 32);

  const int64_t row = (int64_t)r.first + t;
  bf16x8 qc[2 * KC], qr[KR];
  const __bf16* pc = (const __bf16*)a.q_c + (row * a.h_q + head) * DH + 8 * h;
  const __bf16* pr = (const __bf16*)a.q_r + (row * a.h_q + head) * DR + 8 * h;
#pragma unroll
  for (int ks = 0; ks < 2 * KC; ++ks) qc[ks] = *(const bf16x8*)(pc + 16 * ks);
#pragma unroll
  for (int ks = 0; ks < KR; ++ks) qr[ks] = *(const bf16x8*)(pr + 16 * ks);

  const int64_t page_bytes = (int64_t)P * (gc * (DH + DV) + DR * 2) + (int64_t)gc * (P / 32) * 8;
  f32x16 o[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[mt][i] = 0.f;
  float m_run = GQLA_NEG_INF, l_run = 0.f;

  for (int tok = tok_begin; tok < tok_end; tok += 32) {
    const int32_t pg = page_of_uniform(a.cache, r.b, tok / P);
    if (pg < 0) continue;                                        // a page that is not there holds nothing
    const char* page = (const char*)a.cache.pool + (int64_t)pg * page_bytes;
    const int slot0 = tok % P, T = slot0 / 32;
    typedef const __attribute__((address_space(4))) f32x2* const_ptr_t;
    const f32x2 sc = *(const_ptr_t)(uintptr_t)(page + (int64_t)P * (gc * (DH + DV) + 2 * DR) + ((int64_t)j * (P / 32) + T) * 8);
    const char* kb = page + (((int64_t)j * (DH / 16) + h) * P + slot0 + n) * 16;
    const char* rb = page + (int64_t)P * gc * (DH + DV) + ((int64_t)h * P + slot0 + n) * 16;
    const char* vb = page + (int64_t)P * gc * DH + ((((int64_t)j * (P / 32) + T) * DV + n) * 2 + h) * 16;
    u32x4 k8[KC], v8[MT];
    bf16x8 rf[KR];
#pragma unroll
    for (int kp = 0; kp < KC; ++kp) k8[kp] = *(const u32x4*)(kb + (int64_t)kp * 32 * P);
#pragma unroll
    for (int ks = 0; ks < KR; ++ks) rf[ks] = *(const bf16x8*)(rb + (int64_t)ks * 32 * P);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) v8[mt] = *(const u32x4*)(vb + mt * 1024);
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int kp = 0; kp < KC; ++kp) {
      s = mfma32(widen_codes(k8[kp][0], k8[kp][1], sc[0]), qc[2 * kp], s);
      s = mfma32(widen_codes(k8[kp][2], k8[kp][3], sc[0]), qc[2 * kp + 1], s);
    }
#pragma unroll
    for (int ks = 0; ks < KR; ++ks) s = mfma32(rf[ks], qr[ks], s);
    // register i of lane (n, h): token tok + 8 (i / 4) + 4 h + i % 4
    float sv[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sv[i] = s[i] * a.scale_log2e;
    if (tok + 32 > vis_min) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (tok + 8 * (i >> 2) + 4 * h + (i & 3) >= vis) sv[i] = GQLA_NEG_INF;
      // codes of tokens that no row sees may be anything (NaN included)
      if (tok + 32 > vis_max) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (tok + 16 * (e >> 3) + 8 * h + (e & 7) >= vis_max) v8[mt][e >> 2] &= ~(0xffu << (8 * (e & 3)));
      }
    }
    float top = sv[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, sv[i]);
    top = pair_max(top);
    const float m_new = fmaxf(m_run, top), m_use = m_new == GQLA_NEG_INF ? 0.f : m_new;
    const float alpha = fast_exp2(m_run - m_use);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[mt][i] *= alpha;
    bf16x8 pf[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sv[i] = fast_exp2(sv[i] - m_use);
      l_run += sv[i];
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      u32x4 w;
      uint32_t r0, r1;
      half_swap(pack_bf16(sv[8 * kk], sv[8 * kk + 1]), pack_bf16(sv[8 * kk + 4], sv[8 * kk + 5]), r0, r1);
      w[0] = r0;
      w[2] = r1;
      half_swap(pack_bf16(sv[8 * kk + 2], sv[8 * kk + 3]), pack_bf16(sv[8 * kk + 6], sv[8 * kk + 7]), r0, r1);
      w[1] = r0;
      w[3] = r1;
      pf[kk] = __builtin_bit_cast(bf16x8, w);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) o[mt] = mfma32(widen_codes(v8[mt][2 * kk], v8[mt][2 * kk + 1], sc[1]), pf[kk], o[mt]);
  }

  const float l = pair_sum(l_run);
  if (!row_ok) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;      // 0: nothing visible
  const float lse = l == 0.f ? GQLA_NEG_INF : (m_run + fast_log2(l)) * kLn2;
  const int64_t at = row * a.h_q + head;
  if (a.splits == 1) {
    __bf16* out = (__bf16*)a.out + at * DV + 4 * h;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(u32x2*)(out + 32 * mt + 8 * q) = u32x2{pack_bf16(o[mt][4 * q] * inv, o[mt][4 * q + 1] * inv), pack_bf16(o[mt][4 * q + 2] * inv, o[mt][4 * q + 3] * inv)};
    if (a.lse && h == 0) a.lse[at] = lse;
  } else {
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

template <int DH, int DV>
hipError_t launch_attend(const AttendArgs& a, hipStream_t s) {
  const int64_t tiles = row_runs(a.total, a.G, 32 * kAttendWaves, 1, a.B);
  attend_kernel<DH, DV><<<(unsigned)(tiles * a.g * a.splits), 64 * kAttendWaves, 0, s>>>(a, (int)tiles);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const int per = 256 / (DV / 4);
  attend_merge_kernel<DV><<<(unsigned)(((int64_t)a.total * a.h_q + per - 1) / per), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// Ranges of the context: as many as leave the chip's 256 units with about two workgroups each, none shorter than 256 tokens.
int attend_splits(int64_t total, int64_t batch, int h_q, int g, int d_h, int64_t max_tokens) {
  (void)d_h;
  const int64_t groups = row_runs(total, h_q / g, 32 * kAttendWaves, 1, batch) * g;
  const int64_t want = (512 + groups - 1) / groups, most = (max_tokens + 255) / 256;
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, most, 64}));
}

hipError_t launch_attend_fp8_blocks(const AttendArgs& a, hipStream_t s) {
  return a.d_h == 192 ? launch_attend<192, 256>(a, s) : launch_attend<128, 128>(a, s);
}

}  // namespace gqla
