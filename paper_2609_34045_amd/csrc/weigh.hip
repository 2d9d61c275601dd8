// The attention weight that each cached position gets (kf_kv_weigh, and decode steps and
// prefill on tracked caches), added up per KV head:
//
//   w_g[t] += sum over rows r and heads h of g of p_rh(t),  p_rh(t) = 2^(s_rh(t) - M_rh) / L_rh
//
// A softmax's weights are known once its maximum M and sum L are, so there are two
// passes over the keys: weigh_max_kernel leaves (M, L) of each split of the positions,
// weigh_add_kernel joins them and adds.  Values are not read.  A workgroup takes the pages of a split
// of one KV head for all of a user's columns (its rows times the G heads), whose queries it keeps in LDS as fp16 operands,
// two parts of fp32 ones; a wave takes a page at a time, its K operand in registers, decoded there from an MXFP4 cache.
// In the first pass the tiles are K Q^T, whose lanes hold a column each, in the
// second Q K^T, whose lanes hold a position, so that both sums run along registers.
// A position has one writer, so the order of all additions is fixed.
#include <algorithm>

#include "kernels.h"

namespace kf {

namespace {
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;

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
  constexpr int PER = HD / 8;
  const int G = p.nq / p.nkv;
  for (int it = threadIdx.x; it < s.cols * PER; it += 64 * kWaves) {
    const int col = it / PER, c = it % PER, r = s.row0 + col / G;
    float f[8];
    load_q8(p.q, p.q_type, ((int64_t)p.row[r] * p.nq + s.g * G + col % G) * HD + 8 * c, f);
    if (p.gq) {
      float ss = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) ss += f[j] * f[j];
      for (int o = 1; o < PER; o <<= 1) ss += __shfl_xor(ss, o);
      const float rs = 1.0f / sqrtf(ss / (float)HD + p.eps);
      float gain[8], cs[8], sn[8];
      const int64_t at = (int64_t)(p.len[r] - 1) * (HD / 2) + 8 * c % (HD / 2);
      load_q8(p.gq, 1, 8 * c, gain);
      load_q8(p.rope_cos, 0, at, cs);
      load_q8(p.rope_sin, 0, at, sn);
      const float sign = c < PER / 2 ? -1.f : 1.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = f[j] * (rs * gain[j]);
        f[j] = a * cs[j] + sign * __shfl_xor(a, PER / 2) * sn[j];
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
      q[(part * COLS + col) * PER + q_slot<HD>(col, c)] =
          v4u{f16_part2(f[0], f[1], part), f16_part2(f[2], f[3], part), f16_part2(f[4], f[5], part), f16_part2(f[6], f[7], part)};
    if (c == 0) scale[col] = p.scale_log2 * query_unscale(e);
  }
}

// A page's K operand: tile t, step s, lane (row lane % 16, group lane / 16).  The d of a step differ between the two kinds
// of cache; q_chunk gives the queries' same ones.
template <int HD, bool MX>
__device__ __forceinline__ void load_keys(const WeighParams& p, int user, int g, int page, v4u (&k)[4][HD / 32]) {
  constexpr int NS = HD / 32;
  const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
  const int64_t base = (int64_t)kv_page(p.kv, user, page) * p.kv.page_stride;
  if constexpr (MX) {
    const uint8_t* rec = p.rec + base + (int64_t)g * mx_record(HD);
    v4u code[NS];
#pragma unroll
    for (int j = 0; j < NS; ++j) code[j] = *reinterpret_cast<const v4u*>(rec + j * 1024 + lane * 16);
    const uint32_t ke = *reinterpret_cast<const uint32_t*>(rec + mx_codes(HD) + ((HD == 128 ? grp : grp / 2) * 16 + r16) * 4);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float sc = __uint_as_float(((ke >> (8 * t)) & 255u) << 23);
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const uint32_t w = HD == 128 ? code[t][s] : code[t / 2][(t % 2) * 2 + s];
        k[t][s] = v4u{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 3))};
      }
    }
  } else {
    const uint16_t* kc = p.kc + base + (int64_t)g * kKvPage * HD;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int s = 0; s < NS; ++s) k[t][s] = *reinterpret_cast<const v4u*>(kc + (16 * t + r16) * HD + 32 * s + 8 * grp);
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
__global__ __launch_bounds__(64 * kWaves) void weigh_max_kernel(const WeighParams p) {
  constexpr int NS = HD / 32, PER = HD / 8;
  __shared__ v4u q[PARTS * COLS * PER];
  __shared__ float scale[COLS], run_m[kWaves][COLS], run_l[kWaves][COLS];
  __shared__ int len[COLS];
  const Split s = split_of(p);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, grp = lane >> 4;
  const int G = p.nq / p.nkv;
  queries<HD, PARTS, COLS>(p, s, q, scale);
  for (int c = tid; c < COLS; c += 64 * kWaves) {
    len[c] = c < s.cols ? p.len[s.row0 + c / G] : 0;
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
    load_keys<HD, MX>(p, p.user[s.u].user, s.g, page, k);
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
      float mb = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (16 * t + 4 * grp + r >= left) sc[t][r] = -INFINITY;
          mb = fmaxf(mb, sc[t][r]);
        }
      mb = groups_max(mb);
      const float ss = scale[col], m_old = run_m[wave][col], m_new = fmaxf(m_old, mb), ref = m_new == -INFINITY ? 0.f : m_new;
      float l = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) l += __builtin_amdgcn_exp2f((sc[t][r] - ref) * ss);
      l = groups_sum(l);
      l += run_l[wave][col] * __builtin_amdgcn_exp2f((m_old - ref) * ss);
      if (grp == 0) {
        run_m[wave][col] = m_new;
        run_l[wave][col] = l;
      }
    }
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
__global__ __launch_bounds__(64 * kWaves) void weigh_add_kernel(const WeighParams p) {
  constexpr int NS = HD / 32, PER = HD / 8;
  __shared__ v4u q[PARTS * COLS * PER];
  __shared__ float scale[COLS];
  __shared__ v4f of[COLS];  // M, scale, -log2 L and the positions (0: the column adds nothing)
  const Split s = split_of(p);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, grp = lane >> 4;
  const int G = p.nq / p.nkv;
  const WeighUser w = p.user[s.u];
  queries<HD, PARTS, COLS>(p, s, q, scale);
  __syncthreads();
  for (int c = tid; c < COLS; c += 64 * kWaves) {
    v4f x = {0.f, 0.f, 0.f, 0.f};
    if (c < s.cols) {
      const float* part = p.part + (((int64_t)s.row0 + c / G) * p.nq + s.g * G + c % G) * p.max_splits * 2;
      float M = -INFINITY, L = 0.f;
#pragma unroll 4
      for (int z = 0; z < w.splits; ++z) M = fmaxf(M, part[2 * z]);
#pragma unroll 4
      for (int z = 0; z < w.splits; ++z) L += part[2 * z + 1] * __builtin_amdgcn_exp2f((part[2 * z] - M) * scale[c]);
      const bool good = M > -INFINITY && M < INFINITY && L > 0.f && L < INFINITY;
      x = v4f{M, scale[c], -__builtin_amdgcn_logf(L), __int_as_float(good ? p.len[s.row0 + c / G] : 0)};
    }
    of[c] = x;
  }
  __syncthreads();
  float* out = p.weights + ((int64_t)w.user * p.nkv + s.g) * p.stride;
  for (int i = wave; i < s.pages; i += kWaves) {
    const int page = s.page0 + i;
    v4u k[4][NS];
    load_keys<HD, MX>(p, w.user, s.g, page, k);
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
        const int left = __float_as_int(c.w) - page * kKvPage;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][r] - c.x, c.y, c.z));
          sum[t] += 16 * t + r16 < left ? x : 0.f;
        }
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) sum[t] = groups_sum(sum[t]);
    const float mine = grp == 0 ? sum[0] : grp == 1 ? sum[1] : grp == 2 ? sum[2] : sum[3];
    if (pos < w.len) out[pos] = old + mine;
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
  hipLaunchKernelGGL((weigh_max_kernel<HD, MX, PARTS, COLS>), dim3(wgs), dim3(64 * kWaves), 0, s, p);
  hipLaunchKernelGGL((weigh_add_kernel<HD, MX, PARTS, COLS>), dim3(wgs), dim3(64 * kWaves), 0, s, p);
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
  // A page for each wave at least, and about two workgroups a CU.
  const int64_t wgs = 2ll * n_cu;
  int64_t per = std::max<int64_t>(kWaves, (pages * p.nkv + wgs - 1) / wgs);
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
