// The attention weight that each cached position gets (kf_kv_weigh, and decode steps and
// prefill on tracked caches), added up per KV head:
//
//   w_g[t] += sum over rows r and heads h of g of p_rh(t),  p_rh(t) = 2^(s_rh(t) - M_rh) / L_rh
//
// A softmax's weights are known once its maximum M and sum L are, so there are two
// passes over the keys: weigh_max_kernel leaves (M, L) of each split of the positions,
// weigh_add_kernel joins them and adds.  A decode step's attention over an MXFP4 cache
// has left them, and the second pass is enough; over an fp16 cache it takes queries of
// 11 bits, where these have 22, and both passes are needed: p's sums of 1 hang on both
// having the same scores.  Values are not read.  A workgroup takes the pages of a
// split of one KV head for all of a user's columns (its rows times the G heads), whose
// queries it keeps in LDS as fp16 operands, two parts of fp32 ones; a wave takes a page
// at a time, its K operand in registers, decoded there from an MXFP4 cache.  In the
// first pass the tiles are K Q^T, whose lanes hold a column each, in the second Q K^T,
// whose lanes hold a position, so that both sums run along registers.  A position has
// one writer, so the order of all additions is fixed.
//
// What bounds it: one row a user reads K at 6.0 TB/s (131072 positions of 8 heads of 128
// in fp16: 45 + 46 us).  For 32 rows of 32 heads at 16384 positions (34 MB of keys, 5 us
// at 7 TB/s) the passes take 17 + 16 us, and 11.5 + 13 for one fp32 row each of four
// users at 32768, 16384, 8192 and 1024 MXFP4 positions (32 MB).  The rest is the way to
// the first product (launch, page table, queries, in the second pass the splits' sums:
// 5 us a pass, 9 with 128 columns) and, for many rows, the exponentials and their sums on
// the vector units.  So a wave's first page is asked for before the queries are prepared,
// and all of a round's loads of queries before the first is used (54 -> 33 us for the 32
// rows).
#include <algorithm>
#include <climits>

#include "kernels.h"

namespace kf {

namespace {
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// With many columns the preparation of their queries is what costs, so a workgroup has more waves to share it.  32 rows of
// 32 heads at 16384 positions: one workgroup of 8 waves a CU 17.8 + 16.0 us, two of 4 waves 20.6 + 22.0.
__host__ __device__ constexpr int waves_for(int cols) { return cols <= 32 ? 4 : 8; }

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

// Slot of 16-byte chunk c of a column's query: an operand read takes one chunk of 16 consecutive columns.
template <int HD>
__device__ __forceinline__ int q_slot(int col, int c) {
  return HD == 128 ? c ^ (col & 15) : c ^ ((col >> 1) & 7);
}

// What a workgroup works on.
struct Split {
  int u, z, g, page0, pages, rows, cols, row0;
};
__device__ __forceinline__ Split split_of(const WeighParams& p) {
  int id = blockIdx.x, u = 0;
  while (u < p.users - 1 && id >= p.user[u].splits * p.nkv) id -= p.user[u++].splits * p.nkv;
  const WeighUser& w = p.user[u];
  Split s;
  s.u = u;
  s.z = id % w.splits;
  s.g = id / w.splits;
  s.page0 = s.z * p.pages;
  s.pages = min(p.pages, (w.len + kKvPage - 1) / kKvPage - s.page0);
  s.row0 = w.row0;
  s.rows = w.rows;
  s.cols = w.rows * (p.nq / p.nkv);
  return s;
}

// The columns' queries as fp16 operands (two parts of fp32 ones, the second COLS columns on), times a power of two that puts a head's
// largest value near 2^13; scale[col] takes a score back, to log2 units.  Raw queries of qk_norm blocks are normalised
// and rotated first.
template <int HD, int PARTS, int COLS>
__device__ __forceinline__ void queries(const WeighParams& p, const Split& s, v4u* q, float* scale) {
  constexpr int PER = HD / 8, U = 4, kWaves = waves_for(COLS);
  const int G = p.nq / p.nkv, items = s.cols * PER;
  for (int it0 = threadIdx.x; it0 < items; it0 += 64 * kWaves * U) {
    v4u raw[U][PARTS];  // 8 values: fp32 (two parts of it to come) or 16 bits; all loads before the first use
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int it = min(it0 + u * 64 * kWaves, items - 1), col = it / PER, c = it % PER;
      const int64_t at = ((int64_t)p.row[s.row0 + col / G] * p.nq + s.g * G + col % G) * HD + 8 * c;
#pragma unroll
      for (int i = 0; i < PARTS; ++i) raw[u][i] = reinterpret_cast<const v4u*>(p.q)[at * PARTS / 8 + i];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int it = it0 + u * 64 * kWaves, col = it / PER, c = it % PER, r = s.row0 + min(col, s.cols - 1) / G;
      if (it >= items) break;  // (all PER threads of a column)
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint16_t h = (uint16_t)(raw[u][0][j / 2] >> (16 * (j % 2)));
        f[j] = PARTS == 2 ? __uint_as_float(raw[u][j / 4 % PARTS][j % 4])
                          : p.q_type == 1 ? __uint_as_float((uint32_t)h << 16) : (float)__builtin_bit_cast(_Float16, h);
      }
      if (p.gq) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) ss += f[j] * f[j];
        for (int o = 1; o < PER; o <<= 1) ss += __shfl_xor(ss, o);
        const float rs = 1.0f / sqrtf(ss / (float)HD + p.eps);
        float gain[8], cs[8], sn[8];
        const int64_t at = (int64_t)p.rot[r] * (HD / 2) + 8 * c % (HD / 2);
        load_q8(p.gq, 1, 8 * c, gain);
        load_q8(p.rope_cos, 0, at, cs);
        load_q8(p.rope_sin, 0, at, sn);
        const float sign = c < PER / 2 ? -1.f : 1.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float x = f[j] * (rs * gain[j]);
          f[j] = x * cs[j] + sign * __shfl_xor(x, PER / 2) * sn[j];
        }
      }
      float top = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, __builtin_fabsf(f[j]));
      for (int o = 1; o < PER; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
      const int e = query_exponent(top);
      const float k = query_scale(e);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] *= k;
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
        q[(part * COLS + col) * PER + q_slot<HD>(col, c)] = v4u{f16_part2(f[0], f[1], part), f16_part2(f[2], f[3], part),
                                                               f16_part2(f[4], f[5], part), f16_part2(f[6], f[7], part)};
      if (c == 0) scale[col] = p.scale_log2 * query_unscale(e);
    }
  }
}

// A page's keys as they lie, then its K operand: tile t, step s, lane (row lane % 16, group lane / 16).  The d of a step
// differ between the two kinds of cache; q_chunk gives the queries' same ones.
template <int HD, bool MX>
struct Keys {
  v4u w[MX ? HD / 32 : HD / 8];
  uint32_t e;
};
template <int HD, bool MX>
__device__ __forceinline__ void load_keys(const WeighParams& p, int user, int g, int page, Keys<HD, MX>& k) {
  const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
  const int64_t base = (int64_t)kv_page(p.kv, user, page) * p.kv.page_stride;
  if constexpr (MX) {
    const uint8_t* rec = p.rec + base + (int64_t)g * mx_record(HD);
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) k.w[j] = *reinterpret_cast<const v4u*>(rec + j * 1024 + lane * 16);
    k.e = *reinterpret_cast<const uint32_t*>(rec + mx_codes(HD) + ((HD == 128 ? grp : grp / 2) * 16 + r16) * 4);
  } else {
    const uint16_t* kc = p.kc + base + (int64_t)g * kKvPage * HD;
#pragma unroll
    for (int i = 0; i < HD / 8; ++i)
      k.w[i] = *reinterpret_cast<const v4u*>(kc + (16 * (i / (HD / 32)) + r16) * HD + 32 * (i % (HD / 32)) + 8 * grp);
  }
}
template <int HD, bool MX>
__device__ __forceinline__ void decode_keys(const Keys<HD, MX>& from, v4u (&k)[4][HD / 32]) {
  constexpr int NS = HD / 32;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const float sc = MX ? __uint_as_float(((from.e >> (8 * t)) & 255u) << 23) : 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      if constexpr (MX) {
        const uint32_t w = HD == 128 ? from.w[t][s] : from.w[t / 2][(t % 2) * 2 + s];
        k[t][s] = v4u{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 3))};
      } else {
        k[t][s] = from.w[t * NS + s];
      }
    }
  }
}
template <int HD, bool MX>
__device__ __forceinline__ int q_chunk(int s, int grp) {
  return MX ? grp * (HD / 32) + s : 4 * s + grp;
}
__device__ __forceinline__ v4f mfma16(v4u a, v4u b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
}  // namespace

template <int HD, bool MX, int PARTS, int COLS>
__global__ __launch_bounds__(64 * waves_for(COLS)) void weigh_max_kernel(const WeighParams p) {
  constexpr int NS = HD / 32, PER = HD / 8, kWaves = waves_for(COLS);
  __shared__ v4u q[PARTS * COLS * PER];
  __shared__ float scale[COLS], run_m[kWaves][COLS], run_l[kWaves][COLS];
  __shared__ int len[COLS];
  const Split s = split_of(p);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, grp = lane >> 4;
  const int G = p.nq / p.nkv, user = p.user[s.u].user;
  Keys<HD, MX> next;
  if (wave < s.pages) load_keys<HD, MX>(p, user, s.g, s.page0 + wave, next);
  queries<HD, PARTS, COLS>(p, s, q, scale);
  for (int c = tid; c < COLS; c += 64 * kWaves) {
    len[c] = c < s.cols ? p.len[s.row0 + c / G] : INT_MAX;  // (past them nothing is kept)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      run_m[w][c] = -INFINITY;
      run_l[w][c] = 0.f;
    }
  }
  __syncthreads();
  for (int i = wave; i < s.pages; i += kWaves) {
    const int page = s.page0 + i;
    v4u k[4][NS];
    decode_keys<HD, MX>(next, k);
    if (MX && i + kWaves < s.pages) load_keys<HD, MX>(p, user, s.g, page + kWaves, next);
    for (int ct = 0; ct * 16 < s.cols; ++ct) {
      const int col = ct * 16 + r16;
      v4f sc[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) sc[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          const v4u qf = q[(part * COLS + col) * PER + q_slot<HD>(col, q_chunk<HD, MX>(st, grp))];
#pragma unroll
          for (int t = 0; t < 4; ++t) sc[t] = mfma16(k[t][st], qf, sc[t]);
        }
      const int left = len[col] - page * kKvPage;
      if (__any(left < kKvPage)) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (16 * t + 4 * grp + r >= left) sc[t][r] = -INFINITY;
      }
      float mb = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) mb = fmaxf(mb, sc[t][r]);
      mb = groups_max(mb);
      const float ss = scale[col], m_old = run_m[wave][col], m_new = fmaxf(m_old, mb), ref = m_new == -INFINITY ? 0.f : m_new;
      float l = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) l += __builtin_amdgcn_exp2f((sc[t][r] - ref) * ss);
      l = groups_sum(l);
      l += run_l[wave][col] * __builtin_amdgcn_exp2f((m_old - ref) * ss);
      __builtin_amdgcn_wave_barrier();
      if (grp == 0) {
        run_m[wave][col] = m_new;
        run_l[wave][col] = l;
      }
    }
    // The lanes of all groups go on from what those of the first have stored.
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (!MX && i + kWaves < s.pages) load_keys<HD, MX>(p, user, s.g, page + kWaves, next);
  }
  __syncthreads();
  for (int c = tid; c < s.cols; c += 64 * kWaves) {
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, run_m[w][c]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = M == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((run_m[w][c] - M) * scale[c]);
      L += f * run_l[w][c];
    }
    const int64_t at = (((int64_t)s.row0 + c / G) * p.nq + s.g * G + c % G) * p.max_splits + s.z;
    p.part[2 * at] = M;
    p.part[2 * at + 1] = L;
  }
}

template <int HD, bool MX, int PARTS, int COLS>
__global__ __launch_bounds__(64 * waves_for(COLS)) void weigh_add_kernel(const WeighParams p) {
  constexpr int NS = HD / 32, PER = HD / 8, kWaves = waves_for(COLS);
  __shared__ v4u q[PARTS * COLS * PER];
  __shared__ float scale[COLS];
  __shared__ v4f of[COLS];      // M, scale, what a step's own M adds, and the positions (0: the column adds nothing)
  __shared__ float over[COLS];  // 1 / L (its logarithm in the exponent would be off by 2^-21 at 16384 positions)
  const Split s = split_of(p);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, grp = lane >> 4;
  const int G = p.nq / p.nkv;
  const WeighUser w = p.user[s.u];
  Keys<HD, MX> next;
  if (wave < s.pages) load_keys<HD, MX>(p, w.user, s.g, s.page0 + wave, next);
  // The splits' maxima and sums joined, `per` threads a column; the first of them come while the queries do.
  constexpr int U = 4;
  int per = 1;
  // (a step's users have one row each)
  const int splits = p.ml ? p.ml_n[p.row[s.row0]] : w.splits;
  while (per < 64 && 2 * per * s.cols <= 64 * kWaves && per < splits) per *= 2;
  const int c = tid / per, cc = min(c, s.cols - 1), r = s.row0 + cc / G;
  const float2* part = p.ml ? reinterpret_cast<const float2*>(p.ml) + ((int64_t)p.row[r] * p.nq + s.g * G + cc % G) * p.ml_splits
                            : reinterpret_cast<const float2*>(p.part) + ((int64_t)r * p.nq + s.g * G + cc % G) * p.max_splits;
  float2 x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) x[u] = part[min(tid % per + u * per, splits - 1)];
  queries<HD, PARTS, COLS>(p, s, q, scale);
  __syncthreads();
  if (c < COLS) {
    float M = -INFINITY, L = 0.f;
    const float unit = c < s.cols ? p.ml ? 1.0f : scale[c] : 0.f;  // of a maximum, to log2 units
    if (c < s.cols) {
      for (int z0 = tid % per; z0 < splits; z0 += U * per) {
        float m = M;
#pragma unroll
        for (int u = 0; u < U; ++u) m = fmaxf(m, x[u].x);
        // (M is -inf where every score was NaN: that sum stays NaN)
        L = M == -INFINITY ? L : L * __builtin_amdgcn_exp2f((M - m) * unit);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (z0 + u * per < splits) L += m == -INFINITY ? x[u].y : x[u].y * __builtin_amdgcn_exp2f((x[u].x - m) * unit);
        M = m;
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = part[min(z0 + (U + u) * per, splits - 1)];
      }
    }
    for (int o = 1; o < per; o <<= 1) {
      const float m2 = __shfl_xor(M, o), l2 = __shfl_xor(L, o), m = fmaxf(M, m2);
      L = m == -INFINITY ? L + l2 : L * __builtin_amdgcn_exp2f((M - m) * unit) + l2 * __builtin_amdgcn_exp2f((m2 - m) * unit);
      M = m;
    }
    const bool good = c < s.cols && M > -INFINITY && M < INFINITY && L > 0.f && L < INFINITY;
    if (tid % per == 0) {
      of[c] = v4f{p.ml ? 0.f : M, c < s.cols ? scale[c] : 0.f, p.ml ? p.ml_shift - M : 0.f,
                  __int_as_float(good ? p.len[s.row0 + c / G] : 0)};
      over[c] = good ? 1.0f / L : 0.f;
    }
  }
  for (int c = tid + 64 * kWaves / per; c < COLS; c += 64 * kWaves) {
    of[c] = v4f{0.f, 0.f, 0.f, 0.f};
    over[c] = 0.f;
  }
  __syncthreads();
  float* out = p.weights + ((int64_t)w.user * p.nkv + s.g) * p.stride;
  for (int i = wave; i < s.pages; i += kWaves) {
    const int page = s.page0 + i;
    v4u k[4][NS];
    decode_keys<HD, MX>(next, k);
    if (MX && i + kWaves < s.pages) load_keys<HD, MX>(p, w.user, s.g, page + kWaves, next);
    const int pos = page * kKvPage + lane;  // this lane's, in the end
    float old = 0.f;
    if (pos < w.len && pos < w.fresh) old = out[pos];
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int ct = 0; ct * 16 < s.cols; ++ct) {
      v4f sc[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) sc[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          const int col = ct * 16 + r16;
          const v4u qf = q[(part * COLS + col) * PER + q_slot<HD>(col, q_chunk<HD, MX>(st, grp))];
#pragma unroll
          for (int t = 0; t < 4; ++t) sc[t] = mfma16(qf, k[t][st], sc[t]);
        }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const v4f c = of[ct * 16 + 4 * grp + r];
        const float inv = over[ct * 16 + 4 * grp + r];
        const int left = __float_as_int(c.w) - page * kKvPage;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][r] - c.x, c.y, c.z));
          sum[t] = __builtin_fmaf(16 * t + r16 < left ? x : 0.f, inv, sum[t]);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) sum[t] = groups_sum(sum[t]);
    const float mine = grp == 0 ? sum[0] : grp == 1 ? sum[1] : grp == 2 ? sum[2] : sum[3];
    if (pos < w.len) out[pos] = old + mine;
    if (!MX && i + kWaves < s.pages) load_keys<HD, MX>(p, w.user, s.g, page + kWaves, next);
  }
}

// Rows of weights: dst[layer][head][0 .. n) from src, or zeros.
__global__ __launch_bounds__(256) void weights_move_kernel(const WeightRows dst, const WeightRows src, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int64_t g = blockIdx.y, l = blockIdx.z;
  dst.p[l * dst.layer + g * dst.head + i] = src.p ? src.p[l * src.layer + g * src.head + i] : 0.f;
}

// ------------------------------------------------------------------ launchers
template <int HD, bool MX, int PARTS, int COLS>
static hipError_t weigh(const WeighParams& p, int wgs, hipStream_t s) {
  if (!p.ml) hipLaunchKernelGGL((weigh_max_kernel<HD, MX, PARTS, COLS>), dim3(wgs), dim3(64 * waves_for(COLS)), 0, s, p);
  hipLaunchKernelGGL((weigh_add_kernel<HD, MX, PARTS, COLS>), dim3(wgs), dim3(64 * waves_for(COLS)), 0, s, p);
  return hipGetLastError();
}
template <int HD>
static hipError_t weigh_hd(const WeighParams& p, int cols, int wgs, hipStream_t s) {
  const bool mx = p.rec != nullptr, two = p.q_type == 0, few = cols <= 32;
  if (cols > kMaxWeighRows * kMaxGroup) return hipErrorInvalidValue;
  if (mx)
    return two ? (few ? weigh<HD, true, 2, 32>(p, wgs, s) : weigh<HD, true, 2, 256>(p, wgs, s))
               : (few ? weigh<HD, true, 1, 32>(p, wgs, s) : weigh<HD, true, 1, 256>(p, wgs, s));
  return two ? (few ? weigh<HD, false, 2, 32>(p, wgs, s) : weigh<HD, false, 2, 256>(p, wgs, s))
             : (few ? weigh<HD, false, 1, 32>(p, wgs, s) : weigh<HD, false, 1, 256>(p, wgs, s));
}
hipError_t launch_weigh(WeighParams p, int hd, int n_cu, int64_t part_floats, hipStream_t s) {
  static_assert(kMaxWeighRows * kMaxGroup <= 256, "columns");
  int64_t pages = 0, longest = 0;
  int cols = 0, rows = 0;
  for (int u = 0; u < p.users; ++u) {
    const int64_t n = (p.user[u].len + kKvPage - 1) / kKvPage;
    pages += n;
    longest = std::max(longest, n);
    cols = std::max(cols, p.user[u].rows * (p.nq / p.nkv));
    rows += p.user[u].rows;
  }
  if (!longest) return hipSuccess;
  // A page for each wave at least, and 8 waves a CU: the next page's codes come while this one is worked on, and more
  // workgroups prepare the queries more often (four 4-bit users, 58368 positions: 12.0 + 13.5 us, at 16 waves 13.6 + 16.2).
  const int64_t wgs = 8ll / waves_for(cols) * n_cu;
  int64_t per = std::max<int64_t>(waves_for(cols), (pages * p.nkv + wgs - 1) / wgs);
  const int64_t most = std::max<int64_t>(1, part_floats / (2ll * rows * p.nq));
  per = std::max(per, (longest + most - 1) / most);
  p.pages = (int)per;
  p.max_splits = 1;
  int grid = 0;
  for (int u = 0; u < p.users; ++u) {
    p.user[u].splits = std::max(1, (int)(((p.user[u].len + kKvPage - 1) / kKvPage + per - 1) / per));
    p.max_splits = std::max(p.max_splits, p.user[u].splits);
    grid += p.user[u].splits * p.nkv;
  }
  return hd == 128 ? weigh_hd<128>(p, cols, grid, s) : hd == 64 ? weigh_hd<64>(p, cols, grid, s) : hipErrorInvalidValue;
}

hipError_t launch_weights_move(const WeightRows& dst, const WeightRows& src, int n, int nkv, int layers, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  hipLaunchKernelGGL(weights_move_kernel, dim3((n + 255) / 256, nkv, layers), dim3(256), 0, s, dst, src, n);
  return hipGetLastError();
}

}  // namespace kf
