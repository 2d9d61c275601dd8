// Log probabilities of logit rows: a given token's, the distribution's entropy, and
// the most probable alternatives.
//
//   M = max z, S = sum e^(z - M), W = sum e^(z - M) (z - M)
//   log p(t) = (z_t - M) - ln S,  entropy = ln S - W / S
//
// One pass over the logits, which bounds it (4 bytes a value).  A workgroup takes a
// chunk of a row into registers: maximum, then the two sums, then the chunk's k
// largest.  Those: a value that k of a wave's 64 per-lane maxima reach is a lower bound of
// the k-th largest, and so is one that a quarter of k reach in each of the four waves (the
// closer one where the large values are spread, as they mostly are).  Both are found by a search
// over their upper bits whose steps are one compare and a count of its lanes.  The values that
// reach the larger bound, some 30 of 8192 for k = 20, go to LDS and are ranked by counting.
// Keys order values and, among equals, put the lower index first, so that they are
// distinct: (order-preserving bits of z, ~index).  Where equal values make the
// candidates too many the k largest keys are taken one by one.  A second, small launch joins
// a row's chunks: sums rescaled to the row's maximum, and the chunks' sorted lists merged
// in the same way.  Rows of one chunk need no second launch.
// 256 rows of 151936, k = 20: chunks 32 us (4.9 TB/s; some 20 vector instructions a value keep the ALU 65% busy), join
// 5.8 us.  200 rows of 128256 just written by the product: 18 us, 5.8 TB/s.
#include <cmath>

#include "kernels.h"

namespace kf {

namespace {
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int kT = 256;  // threads
constexpr int kMaxChunks = 128;  // of a row
static_assert(kMaxLogprobVocab <= kMaxChunks * kT * 32, "chunks of the longest row");
static_assert(kLogprobLeast >= 255 * 4 && kLogprobLeast >= kMaxChunks, "partials of a call of small chunks, and of a row");

// The order of values as that of unsigned numbers; -0 and 0 are equal.
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of_order(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
// 0 for a masked (-inf) logit, else its key.
__device__ __forceinline__ u64 key_of(float z, int index) {
  return z == -INFINITY ? 0 : (u64)order_of(z) << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float value_of(u64 key) { return value_of_order((uint32_t)(key >> 32)); }
// (fmaxf would quieten each operand first; NaN are looked for apart)
__device__ __forceinline__ float max3(float a, float b, float c) {
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(a) : "v"(a), "v"(b), "v"(c));
  return a;
}
// Over the wave, result in every lane: quad permutes and row mirrors within 16 lanes, then the 16-lane groups.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
}
template <class F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, F f) {
  v = f(v, dpp<0xB1>(v));
  v = f(v, dpp<0x4E>(v));
  v = f(v, dpp<0x141>(v));
  v = f(v, dpp<0x140>(v));
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = f(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return f(b[0], b[1]);
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  return wave_reduce(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}
__device__ __forceinline__ float wave_max(float v) {
  return __uint_as_float(wave_reduce(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}
__device__ __forceinline__ float wave_sum(float v) {
  return __uint_as_float(wave_reduce(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
__device__ __forceinline__ float block_max(float v, float* lds) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
  __syncthreads();
  return v;
}
__device__ __forceinline__ float block_sum(float v, float* lds) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = (lds[0] + lds[1]) + (lds[2] + lds[3]);
  __syncthreads();
  return v;
}

// A row's results from its sums and, in order, its k largest keys (0: no such value).
__device__ __forceinline__ void finish_row(const LogprobParams& p, int row, float M, float S, float W, const u64* keys) {
  const int tid = threadIdx.x;
  const bool some = M != -INFINITY;
  const float ls = some ? logf(S) : 0.f;
  if (tid == 0) {
    if (p.entropy) p.entropy[row] = some ? ls - W / S : 0.f;
    if (p.targets) {
      const int t = p.targets[row];
      float v;
      if (t == -1) {
        v = 0.f;
      } else if (t < 0 || t >= p.vocab) {
        v = __builtin_nanf("");
        raise_err(p.err_flag, true, kErrToken);
      } else {
        const float z = p.logits[row * p.stride + t] * (p.row_scale ? p.row_scale[row] : 1.0f);
        v = z == -INFINITY ? z : z != z || z == INFINITY ? __builtin_nanf("") : some ? (z - M) - ls : z;
      }
      p.logprob[row] = v;
    }
  }
  for (int i = tid; i < p.top; i += kT) {
    const u64 k = keys[i];
    p.top_ids[(int64_t)row * p.top + i] = k ? (int)~(uint32_t)k : -1;
    p.top_logprobs[(int64_t)row * p.top + i] = k ? (value_of(k) - M) - ls : -INFINITY;
  }
}
}  // namespace

// Chunk blockIdx.x of row blockIdx.y: VPT values a thread.
template <int VPT>
__global__ __launch_bounds__(kT) void logprob_chunk_kernel(const LogprobParams p) {
  constexpr int kSeg = 256;  // candidates of a wave
  __shared__ float red[4], red_s[4], red_w[4];
  __shared__ u64 cand[4][kSeg], best[kMaxTop], round[2][4];
  __shared__ uint32_t bound[4], quarter[4];
  __shared__ int count[4];
  const int row = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c0 = blockIdx.x * kT * VPT;
  const float* z = p.logits + row * p.stride;
  const bool wide = ((uintptr_t)z & 15) == 0;
  // Value 4 j + i of a thread: index c0 + 4 (256 j + tid) + i.
  float v[VPT];
#pragma unroll
  for (int j = 0; j < VPT / 4; ++j) {
    const int at = c0 + 4 * (kT * j + tid);
    if (wide && at + 4 <= p.vocab) {
      const v4f x = *reinterpret_cast<const v4f*>(z + at);
      v[4 * j] = x.x; v[4 * j + 1] = x.y; v[4 * j + 2] = x.z; v[4 * j + 3] = x.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * j + i] = at + i < p.vocab ? z[at + i] : -INFINITY;
    }
  }
  if (p.row_scale) {
    const float scale = p.row_scale[row];
#pragma unroll
    for (int i = 0; i < VPT; ++i) v[i] = v[i] == -INFINITY ? v[i] : v[i] * scale;  // (past the row's end: -inf stays)
  }
  float mine = v[0];  // the lane's largest
  bool bad = false;
#pragma unroll
  for (int i = 0; i < VPT; i += 2) {
    bad |= __builtin_isunordered(v[i], v[i + 1]);
    mine = max3(mine, v[i], v[i + 1]);
  }
  bad |= mine == INFINITY;
  if (bad) {  // NaN or +inf: skipped, and reported
    mine = -INFINITY;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (!(v[i] < INFINITY)) v[i] = -INFINITY;
      mine = fmaxf(mine, v[i]);
    }
  }
  raise_err(p.err_flag, bad, kErrNaNLogit);
  if (p.top) {  // the bounds, as far as sign, exponent and 8 bits of the mantissa give them
    uint32_t all = 0, part = 0;
    const uint32_t o = order_of(mine);
    for (int bit = 31; bit >= 15; --bit) {
      const uint32_t t = all | 1u << bit, q = part | 1u << bit;
      if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(o >= t)) >= p.top) all = t;
      if (4 * __builtin_popcountll(__builtin_amdgcn_ballot_w64(o >= q)) >= p.top) part = q;
    }
    if (lane == 0) {
      bound[wave] = all;
      quarter[wave] = part;
    }
    if (tid < kMaxTop) best[tid] = 0;
  }
  const float m = block_max(mine, red);
  float s = 0.f, w = 0.f;
  if (m != -INFINITY) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const float x = fmaxf(v[i] - m, -200.f);  // e^-200 is 0: a masked value adds nothing
      const float e = __expf(x);
      s += e;
      w += e * x;
    }
  }
  s = wave_sum(s);
  w = wave_sum(w);
  if (lane == 0) {
    red_s[wave] = s;
    red_w[wave] = w;
  }
  int n = 0;  // this wave's candidates
  if (p.top) {
    // no lower than the lowest finite value, so that masked values are no candidates
    const uint32_t least = max(max(max(bound[0], bound[1]), max(bound[2], bound[3])),
                               max(min(min(quarter[0], quarter[1]), min(quarter[2], quarter[3])), order_of(-__FLT_MAX__)));
    const float t = value_of_order(least);
    if (__builtin_amdgcn_ballot_w64(mine >= t)) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const u64 hit = __builtin_amdgcn_ballot_w64(v[i] >= t);
        if (!hit) continue;
        const int at = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(hit >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hit, 0));
        if (v[i] >= t && at < kSeg) cand[wave][at] = key_of(v[i], c0 + 4 * (kT * (i / 4) + tid) + i % 4);
        n += __builtin_popcountll(hit);
      }
    }
    if (lane == 0) count[wave] = n;
  }
  __syncthreads();
  s = (red_s[0] + red_s[1]) + (red_s[2] + red_s[3]);
  w = (red_w[0] + red_w[1]) + (red_w[2] + red_w[3]);
  if (p.top) {
    if (max(max(count[0], count[1]), max(count[2], count[3])) > kSeg) {
      u64 k0 = ~0ull;  // the last key taken, then the lane's largest below it
      for (int r = 0; r < p.top; ++r) {
        u64 next = 0;
        if (r == 0 || k0 == best[r - 1]) {  // the lane whose key was taken, and at first every lane
          // (read again: from the registers the loop would be unrolled, at the cost of a wave per SIMD)
          for (int i = 0; i < VPT; ++i) {
            const int at = c0 + 4 * (kT * (i / 4) + tid) + i % 4;
            float x = at < p.vocab ? z[at] : -INFINITY;
            if (p.row_scale && at < p.vocab) x *= p.row_scale[row];
            const u64 k = key_of(x < INFINITY ? x : -INFINITY, at);
            next = k < k0 && k > next ? k : next;
          }
          k0 = next;
        }
        const uint32_t hi = wave_max_u32((uint32_t)(k0 >> 32));
        const uint32_t lo = wave_max_u32((uint32_t)(k0 >> 32) == hi ? (uint32_t)k0 : 0);
        if (lane == 0) round[r & 1][wave] = (u64)hi << 32 | lo;
        __syncthreads();
        if (tid == 0) {
          const u64* q = round[r & 1];
          const u64 x = q[0] > q[1] ? q[0] : q[1], y = q[2] > q[3] ? q[2] : q[3];
          best[r] = x > y ? x : y;
        }
        __syncthreads();
      }
    } else {
      for (int c = lane; c < n; c += 64) {
        const u64 k = cand[wave][c];
        int r = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll 4
          for (int i = 0; i < count[q]; ++i) r += cand[q][i] > k;
        if (r < p.top) best[r] = k;
      }
      __syncthreads();
    }
  }
  if (gridDim.x == 1) {
    finish_row(p, row, m, s, w, best);
    return;
  }
  const int64_t part = (int64_t)row * gridDim.x + blockIdx.x;
  if (tid == 0) {
    p.part_sums[part * 4] = m;
    p.part_sums[part * 4 + 1] = s;
    p.part_sums[part * 4 + 2] = w;
  }
  for (int i = tid; i < p.top; i += kT) p.part_keys[part * p.top + i] = best[i];
}

// Row blockIdx.x from its chunks (at most kMaxChunks).
__global__ __launch_bounds__(kT) void logprob_join_kernel(const LogprobParams p) {
  constexpr int kFew = 6;
  __shared__ float red[4];
  __shared__ u64 heads[kMaxChunks * kMaxTop], cand[kT], best[kMaxTop];
  __shared__ uint32_t bound;
  __shared__ int count;
  const int row = blockIdx.x, tid = threadIdx.x, n = p.chunks, top = p.top;
  const float* sums = p.part_sums + (int64_t)row * n * 4;
  for (int i = tid; i < n * top; i += kT) heads[i] = p.part_keys[(int64_t)row * n * top + i];
  float m = -INFINITY, s = 0.f, w = 0.f;
  if (tid < n) {
    m = sums[tid * 4];
    s = sums[tid * 4 + 1];
    w = sums[tid * 4 + 2];
  }
  const float M = block_max(m, red);
  const float x = fmaxf(m - M, -200.f), f = tid < n && m != -INFINITY ? __expf(x) : 0.f;  // (NaN, of an empty row, gives -200)
  const float S = block_sum(f * s, red);
  const float W = block_sum(f * (w + s * x), red);
  // A bound of the k-th largest, as in a chunk: c keys of enough sorted lists reach it where their c-th does, c such that
  // two thirds of the lists are enough.  What reaches it is ranked by counting.  The few keys of a small k are
  // taken one by one instead, at 0.3 us each (with its chunks, 1 x 128256, k = 5: 8.5 us, ranked 8.8; k = 20: 13.1 and 11.0).
  const bool ranked = top > kFew;
  if (ranked) {
    if (tid < 64) {  // each lane has the lists of two chunks
      const int c = min((3 * top + 2 * n - 1) / (2 * n), top);
      const uint32_t o0 = tid < n ? (uint32_t)(heads[tid * top + c - 1] >> 32) : 0,
                     o1 = tid + 64 < n ? (uint32_t)(heads[(tid + 64) * top + c - 1] >> 32) : 0;
      uint32_t all = 0;
      for (int bit = 31; bit >= 15; --bit) {
        const uint32_t t = all | 1u << bit;
        const int lists = __builtin_popcountll(__builtin_amdgcn_ballot_w64(o0 >= t)) + __builtin_popcountll(__builtin_amdgcn_ballot_w64(o1 >= t));
        if (c * lists >= top) all = t;
      }
      if (tid == 0) {
        bound = max(all, 1u);  // masked values are no candidates
        count = 0;
      }
    }
    if (tid < kMaxTop) best[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n * top; i += kT) {
      const u64 k = heads[i];
      if ((uint32_t)(k >> 32) < bound) continue;
      const int at = atomicAdd(&count, 1);  // (their order does not matter: each counts the larger ones)
      if (at < kT) cand[at] = k;
    }
    __syncthreads();
    if (tid < count && count <= kT) {
      const u64 k = cand[tid];
      int r = 0;
#pragma unroll 8
      for (int i = 0; i < count; ++i) r += cand[i] > k;
      if (r < top) best[r] = k;
    }
  }
  if (tid < 64 && (!ranked || count > kT)) {  // few keys, or many equal values: each lane keeps the heads of two chunks' lists
    int at0 = 0, at1 = 0;
    const u64* l0 = heads + tid * top;
    const u64* l1 = heads + (tid + 64) * top;
    u64 h0 = top && tid < n ? l0[0] : 0, h1 = top && tid + 64 < n ? l1[0] : 0;
    for (int r = 0; r < top; ++r) {
      const u64 mine = h0 > h1 ? h0 : h1;
      // the largest value, then the largest key of its lanes (one, but for equal values)
      const uint32_t hi = wave_max_u32((uint32_t)(mine >> 32));
      const u64 lanes = __builtin_amdgcn_ballot_w64((uint32_t)(mine >> 32) == hi);
      uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, __builtin_ctzll(lanes));
      if (lanes & (lanes - 1)) lo = wave_max_u32((uint32_t)(mine >> 32) == hi ? (uint32_t)mine : 0);
      const u64 k = (u64)hi << 32 | lo;
      if (tid == 0) best[r] = k;
      if (mine == k && k) {
        if (h0 == k) h0 = ++at0 < top ? l0[at0] : 0;
        else h1 = ++at1 < top ? l1[at1] : 0;
      }
    }
  }
  __syncthreads();
  finish_row(p, row, M, S, W, best);
}

// Row blockIdx.x, bound by its latency: a thread's values wait in registers (rows of up to 32768; longer ones are
// read again).  K is a multiple of 64.
constexpr int kRowThreads = 512;
__global__ __launch_bounds__(kRowThreads) void rows_to_f16_kernel(const uint16_t* x, int K, float eps, uint16_t* x16, float* eps_rows,
                                                                 float* row_scale) {
  constexpr int kHeld = 8;  // 16-byte pieces
  __shared__ uint32_t red[kRowThreads / 64];
  __shared__ float red_s[kRowThreads / 64];
  const int tid = threadIdx.x, n = K / 8;
  const v4u* src = reinterpret_cast<const v4u*>(x + (int64_t)blockIdx.x * K);
  v4u* dst = reinterpret_cast<v4u*>(x16 + (int64_t)blockIdx.x * K);
  v4u v[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = tid + kRowThreads * j;
    v[j] = i < n ? src[i] : v4u{0u, 0u, 0u, 0u};
  }
  uint32_t top = 0;  // the magnitudes' bits, in the upper half
  auto seen = [&](const v4u& w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fff0000u, (w[i] & 0x7fffu) << 16));
  };
#pragma unroll
  for (int j = 0; j < kHeld; ++j) seen(v[j]);
  for (int i = tid + kRowThreads * kHeld; i < n; i += kRowThreads) seen(src[i]);
  top = wave_max_u32(top);
  if ((tid & 63) == 0) red[tid / 64] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kRowThreads / 64; ++w) top = max(top, red[w]);
  const float most = __uint_as_float(top);
  int e = top && most < INFINITY ? 14 - ilogbf(most) : 0;
  if (eps > 0.f) e = min(e, (126 - ilogbf(eps)) / 2);  // eps 4^e stays finite: smaller rows are nothing beside it
  float ss = 0.f;
  auto scaled = [&](v4u w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = ldexpf(__uint_as_float(w[i] << 16), e), b = ldexpf(__uint_as_float(w[i] & 0xffff0000u), e);
      ss += a * a + b * b;
      w[i] = f16_pair(a, b);
    }
    return w;
  };
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = tid + kRowThreads * j;
    if (i < n) dst[i] = scaled(v[j]);
  }
  for (int i = tid + kRowThreads * kHeld; i < n; i += kRowThreads) dst[i] = scaled(src[i]);
  const float eps_row = ldexpf(eps, 2 * e);
  if (tid == 0 && eps_rows) eps_rows[blockIdx.x] = eps_row;
  if (!row_scale) return;
  ss = wave_sum(ss);
  if ((tid & 63) == 0) red_s[tid / 64] = ss;
  __syncthreads();
  if (tid == 0) {
    ss = 0.f;
    for (int w = 0; w < kRowThreads / 64; ++w) ss += red_s[w];
    row_scale[blockIdx.x] = 1.0f / sqrtf(ss / (float)K + eps_row);
  }
}

// Values per thread: chunks of 8192 values where they give each CU a workgroup or cover a row that 2048 do not at once,
// else of 2048.  In chunks of 2048 and 8192, k = 20: 4 x 5000 11.5 and 7.0 us, 16 x 32000 12.8 and 14.0, 4 x 128256
// 13.5 and 14.1; 64 x 32000 14.5 and 14.1, 16 x 128256 15.3 and 14.6, 64 x 128256 26 and 19, 256 x 151936 72 and 37.
// (Workgroups of 1024 threads that take rows of up to 32768 alone were slower than two launches: 17 us and 12.)
int logprob_values(int rows, int vocab) {
  const int64_t large = (vocab + 8191) / 8192;
  if (vocab <= 2048) return 8;
  return large == 1 || rows * large >= 256 || (vocab + 2047) / 2048 > 128 ? 32 : 8;
}
int logprob_chunks(int vocab, int values) { return (vocab + kT * values - 1) / (kT * values); }

hipError_t launch_rows_to_f16(const uint16_t* x, int rows, int K, float eps, uint16_t* x16, float* eps_rows,
                              float* row_scale, hipStream_t s) {
  hipLaunchKernelGGL(rows_to_f16_kernel, dim3(rows), dim3(kRowThreads), 0, s, x, K, eps, x16, eps_rows, row_scale);
  return hipGetLastError();
}

hipError_t launch_logprobs(LogprobParams p, int rows, char* part, hipStream_t s) {
  if (p.vocab < 1 || p.vocab > kMaxLogprobVocab || rows < 1 || rows > kLogprobRows || p.top < 0 || p.top > kMaxTop ||
      (p.values != 8 && p.values != 32) || logprob_chunks(p.vocab, p.values) > kMaxChunks)
    return hipErrorInvalidValue;
  p.chunks = logprob_chunks(p.vocab, p.values);
  p.part_keys = reinterpret_cast<unsigned long long*>(part);
  p.part_sums = reinterpret_cast<float*>(part + (int64_t)rows * p.chunks * p.top * 8);
  const dim3 grid(p.chunks, rows);
  if (p.values == 32) hipLaunchKernelGGL(logprob_chunk_kernel<32>, grid, dim3(kT), 0, s, p);
  else hipLaunchKernelGGL(logprob_chunk_kernel<8>, grid, dim3(kT), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.chunks == 1) return e;
  hipLaunchKernelGGL(logprob_join_kernel, dim3(rows), dim3(kT), 0, s, p);
  return hipGetLastError();
}

}  // namespace kf
