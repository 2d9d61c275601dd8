// Attention over an MXFP4 cache for one query row of each of up to four users: with
// given queries (kf_kv_attend), and in a decode step, whose new keys and values it
// appends; and the merge of kf_kv_attend's splits, of caches of both types.
//
//   out_h = sum_t p_t v_t / sum_t p_t,  p_t = 2^(s_t - m),  s_t = q_h . k_t log2(e) / sqrt(hd)
//
// over the first len positions, a running maximum m per query head, 32-bit sums.
// A workgroup (split, KV head, row) takes whole pages of 64 positions for all G
// query heads of the KV head, so that each cached byte is read once per KV head
// and row; its waves take the split's pages in turn and keep states of their own
// until the end.  A lane loads a page's codes and exponents straight into the
// registers it computes from (kernels.h gives the order), the next page's K as soon
// as the scores have used this one's, and V after P V: nothing passes through LDS, and
// no wave waits for another.  (Registers for two whole pages, 244 of them, were slower.)
//
// Scores: S = K Q^T on 16x16x32 fp16 MFMAs, K decoded by the convert instruction
// that takes two E2M1 codes and the block's power of two (exact in fp16).  The 16
// columns of a tile hold 8 query heads twice, as two fp16 parts of each query
// value (columns 0-7 the rounded value, 8-15 what rounding left), so that a score
// is as exact as 22-bit queries give it at no more products than one part would
// take.  P V: O^T = V^T P^T alike, V decoded and multiplied by its positions' scales
// two at a time, the two halves of the columns holding the two parts of a
// probability.  The score tile's lane layout is the P^T operand's.
//
// Bound by the cache's bytes where it is long: two rows of 131072 and 100001 positions, 64 query and 8 KV heads of
// 128, 259 MB, 50 us (5.2 TB/s, 6 between its ramp and its tail); half the waves' time is
// waiting for memory, a quarter vector instructions (some 440 a page, 32 matrix ones).  Four rows of
// 1024 to 32768, 32 and 8 heads: 16.6 us, by the vector instructions of two waves a SIMD.  200 positions: 6.3 us, latency.
#include <cmath>
#include <type_traits>

#include "kernels.h"

namespace kf {

namespace {
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float ror8(float v) {  // the lane 8 apart within each row of 16
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xf, 0xf, false));
}
__device__ __forceinline__ float groups_max(float x) {  // over the four 16-lane groups
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float groups_sum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float exponent(uint32_t w, int byte) {  // 2^e of a stored K exponent
  return __uint_as_float(((w >> (8 * byte)) & 255u) << 23);
}

// 8 consecutive values of a query row.
__device__ __forceinline__ void load_q8(const void* q, int type, int64_t at, float (&f)[8]) {
  if (type == 0) {
    const v4f* p = reinterpret_cast<const v4f*>(reinterpret_cast<const float*>(q) + at);
    const v4f a = p[0], b = p[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    return;
  }
  const v4u w = *reinterpret_cast<const v4u*>(reinterpret_cast<const uint16_t*>(q) + at);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint16_t h = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
    f[i] = type == 1 ? __uint_as_float((uint32_t)h << 16) : (float)__builtin_bit_cast(_Float16, h);
  }
}
// An output value in fp32, bf16 or fp16 (nearest even).
__device__ __forceinline__ void store_out(void* out, int type, int64_t at, float v) {
  if (type == 0) reinterpret_cast<float*>(out)[at] = v;
  else if (type == 1) reinterpret_cast<__bf16*>(out)[at] = (__bf16)v;
  else reinterpret_cast<_Float16*>(out)[at] = (_Float16)v;
}

constexpr int kWaves = 4;
constexpr int kMostPages = kMxMaxSplit / kKvPage;
static_assert(kMostPages <= 64, "a lane holds the id of one page of the split");

template <int HD>
struct MxPage {
  v4u k[HD / 32], v[HD / 32];
  uint32_t ks;
  v4u vs[HD / 16];
};

// x[s][j] of d = grp hd/4 + 8 s + j, normalised (gains `gain`) and rotated to position pos; the RoPE partner
// d +- hd/2 lies in the lane 32 apart.
template <int HD>
__device__ __forceinline__ void norm_rope(const MxStepParams& p, float (&x)[HD / 32][8], int grp, int pos) {
  float ss = 0.f;
#pragma unroll
  for (int s = 0; s < HD / 32; ++s)
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += x[s][j] * x[s][j];
  const float rs = 1.0f / sqrtf(groups_sum(ss) / (float)HD + p.eps);
  const float sign = grp < 2 ? -1.0f : 1.0f;
#pragma unroll
  for (int s = 0; s < HD / 32; ++s) {
    const int d0 = grp * (HD / 4) + 8 * s;
    float gain[8], c[8], sn[8];
    load_q8(p.gq, 1, d0, gain);
    load_q8(p.rope_cos, 0, (int64_t)pos * (HD / 2) + d0 % (HD / 2), c);
    load_q8(p.rope_sin, 0, (int64_t)pos * (HD / 2) + d0 % (HD / 2), sn);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = x[s][j] * (rs * gain[j]);
      x[s][j] = a * c[j] + sign * __shfl_xor(a, 32) * sn[j];
    }
  }
}

// Row b's new key or value of KV head g to its position of the cache, by lanes 0 .. hd/8 - 1 of a wave, 8 values each.
template <int HD>
__device__ __forceinline__ void append(const MxStepParams& p, int b, int g, bool is_v, int lane) {
  constexpr int PER = HD / 8;
  if (lane >= PER) return;
  const int pos = p.a.len[b] - 1, t = pos % kKvPage, d0 = 8 * lane, blk = d0 / kMxBlock;
  uint8_t* rec = p.cache + (int64_t)kv_page(p.a.kv, p.a.users[b], pos / kKvPage) * p.a.kv.page_stride + (int64_t)g * mx_record(HD) +
                 (is_v ? mx_v(HD) : 0);
  uint8_t old[8];
  if (is_v) {  // the other nibble of each byte is a neighbouring position's
#pragma unroll
    for (int j = 0; j < 8; ++j) old[j] = rec[mx_v_byte(t, d0 + j)];
  }
  float x[8];
  if (!is_v && p.gk) {  // raw: its norm and RoPE are due
    load_q8(p.kraw, 0, ((int64_t)b * p.a.nkv + g) * HD + d0, x);
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += x[j] * x[j];
    for (int o = 1; o < PER; o <<= 1) ss += __shfl_xor(ss, o);
    const float rs = 1.0f / sqrtf(ss / (float)HD + p.eps);
    float gain[8], c[8], sn[8];
    load_q8(p.gk, 1, d0, gain);
    load_q8(p.rope_cos, 0, (int64_t)(pos + p.ahead.n[b]) * (HD / 2) + d0 % (HD / 2), c);
    load_q8(p.rope_sin, 0, (int64_t)(pos + p.ahead.n[b]) * (HD / 2) + d0 % (HD / 2), sn);
    const float sign = d0 < HD / 2 ? -1.f : 1.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = x[j] * (rs * gain[j]);
      x[j] = a * c[j] + sign * __shfl_xor(a, PER / 2) * sn[j];
    }
  } else {
    load_q8(is_v ? p.v16 : p.k16, 2, (((int64_t)b * p.a.nkv + g) * kKvPage + t) * HD + d0, x);
  }
  uint32_t pairs[4] = {f16_pair(x[0], x[1]), f16_pair(x[2], x[3]), f16_pair(x[4], x[5]), f16_pair(x[6], x[7])};
  bool bad = false;
  int e;
  const uint32_t w = mx_encode8(pairs, e, bad);
  raise_err(p.a.err_flag, bad, kErrF16Range);
  if (!is_v) {
    *reinterpret_cast<uint32_t*>(rec + mx_k_byte<HD>(t, d0)) = w;
    if (lane % 4 == 0) rec[mx_codes(HD) + mx_k_exp(t, blk)] = (uint8_t)(e + 127);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t c = (w >> (4 * j)) & 15u;
    rec[mx_v_byte(t, d0 + j)] = (uint8_t)(t & 1 ? (old[j] & 0x0f) | (c << 4) : (old[j] & 0xf0) | c);
  }
  if (lane % 4 == 0) reinterpret_cast<uint16_t*>(rec + mx_codes(HD))[mx_v_exp<HD>(t, blk)] = mx_v_scale(e);
}
}  // namespace

// P is MxAttnParams, or MxStepParams for a decode step: the workgroup whose split ends in the row's new position
// stores its key and value first (a launch of its own for that cost 5 us a layer).
template <int HD, class P>
__global__ __launch_bounds__(64 * kWaves, 3) void attn_mx_kernel(const P p) {
  constexpr bool STEP = std::is_same<P, MxStepParams>::value;
  constexpr int NS = HD / 32, NT = HD / 16, NB = HD / kMxBlock;
  constexpr int CODES = mx_codes(HD), REC = mx_record(HD), V = mx_v(HD);
  constexpr int SROW = HD + 4;  // a head's row of a wave's state in LDS
  __shared__ __attribute__((aligned(16))) float state[kWaves][8 * SROW];
  __shared__ float state_m[kWaves][8], state_l[kWaves][8];

  // grid.x: the splits of row 0, then of row 1, ..
  int split = blockIdx.x, b = 0;
  for (; b < kMaxBatch - 1 && split >= p.rows.n[b]; ++b) split -= p.rows.n[b];
  const int g = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = p.a.nq / p.a.nkv, hq0 = g * G;
  const int col = lane & 15, grp = lane >> 4, head = col & 7;
  const float keep = col >= 8 ? 1.0f : 0.0f;  // this lane's column holds the low parts

  const int len = p.a.len[b], u = p.a.users[b];
  const int page0 = split * (p.a.split / kKvPage);
  const int pages = min(p.a.split / kKvPage, (len + kKvPage - 1) / kKvPage - page0);
  auto put = [&](int h, int d, float v, float m, float l) {
    if (p.out) {
      store_out(p.out, p.io, ((int64_t)b * p.a.nq + hq0 + h) * HD + d, len ? v / l : 0.f);
      return;
    }
    const int64_t row = ((int64_t)b * p.a.nq + hq0 + h) * p.a.max_split + split;
    p.a.part_acc[row * HD + d] = v;
    if (d == 0) {
      p.a.part_ml[row * 2] = m;
      p.a.part_ml[row * 2 + 1] = l;
    }
  };
  if (pages <= 0) {  // a row without positions
    for (int e = tid; e < G * HD; e += 64 * kWaves) put(e / HD, e % HD, 0.f, -INFINITY, 0.f);
    return;
  }

  if constexpr (STEP) {
    if (page0 + pages == (len + kKvPage - 1) / kKvPage) {
      if (wave < 2) append<HD>(p, b, g, wave == 1, lane);
      // One workgroup reads the page.  Its waves share one vector cache, which takes their stores and loads in order: behind
      // the barrier a load finds what the other waves stored before it, and no wave waits for its stores' way to memory.
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    }
  }

  // Lane i holds the id of the split's page i.
  int pid = 0;
  if (lane < pages) pid = kv_page(p.a.kv, u, page0 + lane);
  const uint8_t* heads = p.rec + (int64_t)g * REC;
  MxPage<HD> pg;
  auto record = [&](int i) { return heads + (int64_t)__builtin_amdgcn_readlane(pid, i) * p.a.kv.page_stride; };
  auto load_k = [&](const uint8_t* rec) {
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) pg.k[j] = *reinterpret_cast<const v4u*>(rec + j * 1024 + lane * 16);
    pg.ks = *reinterpret_cast<const uint32_t*>(rec + CODES + ((HD == 128 ? grp : grp / 2) * 16 + col) * 4);
  };
  auto load_v = [&](const uint8_t* rec) {
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) pg.v[j] = *reinterpret_cast<const v4u*>(rec + V + j * 1024 + lane * 16);
#pragma unroll
    for (int j = 0; j < 2 * NB; ++j) pg.vs[j] = *reinterpret_cast<const v4u*>(rec + V + CODES + grp * NB * 32 + j * 16);
  };
  if (wave < pages) {
    load_k(record(wave));
    load_v(record(wave));
  }

  // The query operand, step s: d = grp hd/4 + 8 s .. + 7 of this column's head (columns past G repeat the
  // last one, and are not read).  Asked for after the page, so that one wait covers both.
  // In log2 units, times a power of two that puts the head's largest value near 2^10 (query_exponent).
  h8 qf[NS];
  float unscale;
  {
    float f[NS][8], top = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
      load_q8(p.q, p.q_type, ((int64_t)b * p.a.nq + hq0 + min(head, G - 1)) * HD + grp * (HD / 4) + 8 * s, f[s]);
    if constexpr (STEP) {
      if (p.gq) norm_rope<HD>(p, f, grp, len - 1 + p.ahead.n[b]);
    }
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, __builtin_fabsf(f[s][j]));
    const int e = query_exponent(groups_max(top));
    unscale = query_unscale(e);
    const float scale = p.a.scale_log2 * query_scale(e);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[s][j] *= scale;
      qf[s] = __builtin_bit_cast(h8, v4u{f16_part2(f[s][0], f[s][1], keep), f16_part2(f[s][2], f[s][3], keep),
                                         f16_part2(f[s][4], f[s][5], keep), f16_part2(f[s][6], f[s][7], keep)});
    }
  }

  v4f o[NT];  // O^T tile t: lane holds d = 16 t + 4 grp + r of its column's part
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = v4f{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;

  for (int i = wave; i < pages; i += kWaves) {
    const bool more = i + kWaves < pages;
    const uint8_t* next = record(more ? i + kWaves : i);
    v4f sc[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float scale = exponent(pg.ks, t);
      sc[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const uint32_t w = HD == 128 ? pg.k[t][s] : pg.k[t / 2][(t % 2) * 2 + s];
        const v4u kf = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3))};
        sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, kf), qf[s], sc[t], 0, 0, 0);
      }
    }
    if (more) load_k(next);  // K's registers are free from here on, V's after the last product
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[t][r] += ror8(sc[t][r]);
    const int left = len - (page0 + i) * kKvPage;  // positions of the page
    if (left < kKvPage) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (16 * t + 4 * grp + r >= left) sc[t][r] = -INFINITY;
    }
    float mb = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t) mb = fmaxf(mb, fmaxf(fmaxf(sc[t][0], sc[t][1]), fmaxf(sc[t][2], sc[t][3])));
    mb = groups_max(mb) * unscale;
    const float m_new = mb > m_run + kPartLazy ? mb : m_run;
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);  // 0 while m_run is -inf
    float ls = 0.f;
    uint32_t pw[8];  // pair k: positions 16 (k / 2) + 4 grp + 2 (k % 2), and the next
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[k / 2][2 * (k % 2)], unscale, -m_new) + kPartShift);
      const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[k / 2][2 * (k % 2) + 1], unscale, -m_new) + kPartShift);
      ls += x + y;
      pw[k] = f16_part2(x, y, keep);
    }
    l_run = l_run * alpha + ls;
    m_run = m_new;
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f)) {
#pragma unroll
      for (int t = 0; t < NT; ++t) o[t] *= alpha;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const h8 pf = __builtin_bit_cast(h8, v4u{pw[4 * s], pw[4 * s + 1], pw[4 * s + 2], pw[4 * s + 3]});
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint32_t w = pg.v[t / 2][(t % 2) * 2 + s];
        const h8 vs = __builtin_bit_cast(h8, pg.vs[2 * (t / 2) + s]);
        const h2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0) * __builtin_shufflevector(vs, vs, 0, 1),
                 v1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1) * __builtin_shufflevector(vs, vs, 2, 3),
                 v2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2) * __builtin_shufflevector(vs, vs, 4, 5),
                 v3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3) * __builtin_shufflevector(vs, vs, 6, 7);
        const v4u vf = {__builtin_bit_cast(uint32_t, v0), __builtin_bit_cast(uint32_t, v1), __builtin_bit_cast(uint32_t, v2),
                        __builtin_bit_cast(uint32_t, v3)};
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, vf), pf, o[t], 0, 0, 0);
      }
    }
    if (more) load_v(next);
  }
  l_run = groups_sum(l_run);

  // The waves' states meet in LDS; the two parts of a column are one head.
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    v4f x;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = o[t][r] + ror8(o[t][r]);
    if (col < 8) *reinterpret_cast<v4f*>(&state[wave][head * SROW + 16 * t + 4 * grp]) = x;
  }
  if (lane < 8) {
    state_m[wave][lane] = m_run;
    state_l[wave][lane] = l_run;
  }
  __syncthreads();
  for (int e = tid; e < G * HD; e += 64 * kWaves) {
    const int h = e / HD, d = e % HD;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, state_m[w][h]);
    float v = 0.f, l = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      // M is -inf only where every score was NaN (a query that is not finite): the sums stay NaN
      const float f = M == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(state_m[w][h] - M);
      v += f * state[w][h * SROW + d];
      l += f * state_l[w][h];
    }
    put(h, d, v, M, l);
  }
}

// Merge of a row's split partials into the output of kf_kv_attend; a row without
// positions gives zeros.  Workgroup (head, row): the splits' weights at once, in LDS, then each
// wave sums every fourth split, eight loads in flight.
template <int HD>
__global__ __launch_bounds__(256) void attend_merge_kernel(const MxAttnParams p) {
  constexpr int DPL = HD / 64, PRE = 8;
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ns = p.rows.n[b];
  const int64_t r0 = ((int64_t)b * p.a.nq + h) * p.a.max_split;
  const float* ml = p.a.part_ml + r0 * 2;
  const float* acc = p.a.part_acc + r0 * HD + lane * DPL;
  __shared__ float weight[kAttnMaxSplitCount];
  __shared__ float red[4][HD], red_m[4], red_l[4];
  // The wave's first splits are asked for with the maxima; past the last split it is read again, and not used.
  float pre[PRE][DPL];
#pragma unroll
  for (int k = 0; k < PRE; ++k)
#pragma unroll
    for (int i = 0; i < DPL; ++i) pre[k][i] = acc[(int64_t)min(wave + 4 * k, ns - 1) * HD + i];
  float M = -INFINITY;
  for (int s = tid; s < ns; s += 256) M = fmaxf(M, ml[2 * s]);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  if (lane == 0) red_m[wave] = M;
  __syncthreads();
  M = fmaxf(fmaxf(red_m[0], red_m[1]), fmaxf(red_m[2], red_m[3]));
  float l = 0.f;
  for (int s = tid; s < ns; s += 256) {
    // M is -inf where no split saw a key, or where every score was NaN: those sums stay NaN
    const float f = M == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ml[2 * s] - M);
    weight[s] = f;
    l += f * ml[2 * s + 1];
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) l += __shfl_xor(l, o);
  if (lane == 0) red_l[wave] = l;
  __syncthreads();
  float v[DPL] = {};
#pragma unroll
  for (int k = 0; k < PRE; ++k) {
    const bool mine = wave + 4 * k < ns;  // (weight 0 would make a NaN of an infinite sum)
    const float f = mine ? weight[wave + 4 * k] : 0.f;
#pragma unroll
    for (int i = 0; i < DPL; ++i) v[i] = mine ? v[i] + f * pre[k][i] : v[i];
  }
#pragma unroll 8
  for (int s = wave + 4 * PRE; s < ns; s += 4) {
    const float f = weight[s];
#pragma unroll
    for (int i = 0; i < DPL; ++i) v[i] += f * acc[(int64_t)s * HD + i];
  }
#pragma unroll
  for (int i = 0; i < DPL; ++i) red[wave][lane * DPL + i] = v[i];
  __syncthreads();
  if (tid < HD) {
    const float x = (red[0][tid] + red[1][tid]) + (red[2][tid] + red[3][tid]);
    l = (red_l[0] + red_l[1]) + (red_l[2] + red_l[3]);
    store_out(p.out, p.io, ((int64_t)b * p.a.nq + h) * HD + tid, p.a.len[b] ? x / l : 0.f);
  }
}

// ------------------------------------------------------------------ launchers
template <class P>
static hipError_t attn_mx(const P& p, int batch, hipStream_t s) {
  if (p.a.nq % p.a.nkv || p.a.nq / p.a.nkv > 8 || p.a.split % kKvPage || p.a.split > kMxMaxSplit) return hipErrorInvalidValue;
  int splits = 0;
  for (int b = 0; b < batch; ++b) {
    if (p.rows.n[b] < 1 || p.rows.n[b] > p.a.max_split) return hipErrorInvalidValue;
    splits += p.rows.n[b];
  }
  const dim3 grid(splits, p.a.nkv);
  if (p.a.hd == 128) hipLaunchKernelGGL((attn_mx_kernel<128, P>), grid, dim3(64 * kWaves), 0, s, p);
  else if (p.a.hd == 64) hipLaunchKernelGGL((attn_mx_kernel<64, P>), grid, dim3(64 * kWaves), 0, s, p);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}
hipError_t launch_attn_mx(const MxAttnParams& p, int batch, hipStream_t s) { return attn_mx(p, batch, s); }
hipError_t launch_attn_mx_step(const MxStepParams& p, int batch, hipStream_t s) { return attn_mx(p, batch, s); }

hipError_t launch_attend_merge(const MxAttnParams& p, int batch, hipStream_t s) {
  const dim3 grid(p.a.nq, batch);
  if (p.a.hd == 128) hipLaunchKernelGGL(attend_merge_kernel<128>, grid, dim3(256), 0, s, p);
  else if (p.a.hd == 64) hipLaunchKernelGGL(attend_merge_kernel<64>, grid, dim3(256), 0, s, p);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace kf
