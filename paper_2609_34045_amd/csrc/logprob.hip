// Log probabilities of logit rows: a given token's, the distribution's entropy, and
// the most probable alternatives.
//
//   M = max z, S = sum e^(z - M), W = sum e^(z - M) (z - M)
//   log p(t) = (z_t - M) - ln S,  entropy = ln S - W / S
//
// One pass over the logits, which bounds it (4 bytes a value).  A workgroup takes a
// chunk of a row into registers: maximum, then the two sums, then the chunk's k
// largest.  A key orders values and, among equals, puts the lower index first, so
// that keys are distinct: (order-preserving bits of z, ~index).  The k-th largest of
// a wave's 64 per-lane maxima is a lower bound of the chunk's k-th largest key (k
// keys reach it), at most k lanes of each wave hold keys that reach the largest of the four
// waves' bounds, and these few candidates are ranked by counting.  A second, small launch
// joins a row's chunks: sums rescaled to the row's maximum, and k rounds of the
// largest head of the chunks' sorted lists.  Rows of one chunk need no second launch.
#include <cmath>

#include "kernels.h"

namespace kf {

namespace {
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int kT = 256;  // threads

// 0 for a masked (-inf) or refused logit, else its key.
__device__ __forceinline__ u64 key_of(float z, int index) {
  if (z == -INFINITY) return 0;
  const uint32_t b = __float_as_uint(z + 0.0f);  // -0 and 0 are equal
  const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return (u64)o << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float value_of(u64 key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ u64 lane_key(u64 key, int lane) {
  return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)key, lane);
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
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
        const float z = p.logits[row * p.stride + t];
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
  __shared__ float red[4];
  __shared__ u64 bound[4], cand[4 * kMaxTop * VPT], best[kMaxTop];
  __shared__ int n_cand;
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
  bool bad = false;
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    if (!(v[i] < INFINITY)) {  // NaN or +inf: skipped, and reported
      v[i] = -INFINITY;
      bad = true;
    }
    m = fmaxf(m, v[i]);
  }
  raise_err(p.err_flag, bad, kErrNaNLogit);
  m = block_max(m, red);
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
  s = block_sum(s, red);
  w = block_sum(w, red);

  if (p.top) {
    u64 mine = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const u64 k = key_of(v[i], c0 + 4 * (kT * (i / 4) + tid) + i % 4);
      mine = k > mine ? k : mine;
    }
    int rank = 0;
    for (int l = 0; l < 64; ++l) rank += lane_key(mine, l) > mine;
    const u64 at = __builtin_amdgcn_ballot_w64(rank == p.top - 1 && mine != 0);
    if (lane == 0) bound[wave] = at ? lane_key(mine, __builtin_ctzll(at)) : 0;
    if (tid == 0) n_cand = 0;
    if (tid < kMaxTop) best[tid] = 0;
    __syncthreads();
    u64 least = 1;
#pragma unroll
    for (int i = 0; i < 4; ++i) least = bound[i] > least ? bound[i] : least;
    if (mine >= least) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const u64 k = key_of(v[i], c0 + 4 * (kT * (i / 4) + tid) + i % 4);
        if (k >= least) cand[atomicAdd(&n_cand, 1)] = k;
      }
    }
    __syncthreads();
    const int n = n_cand;  // at most top lanes of each wave reach the bound: 4 top VPT keys
    for (int c = tid; c < n; c += kT) {
      const u64 k = cand[c];
      int r = 0;
      for (int i = 0; i < n; ++i) r += cand[i] > k;
      if (r < p.top) best[r] = k;
    }
    __syncthreads();
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
  constexpr int kMaxChunks = 128;
  __shared__ float red[4];
  __shared__ u64 heads[kMaxChunks * kMaxTop], best[kMaxTop];
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
  if (tid < 64) {  // each lane keeps the heads of two chunks' lists
    int at0 = 0, at1 = 0;
    const u64* l0 = heads + tid * top;
    const u64* l1 = heads + (tid + 64) * top;
    u64 h0 = top && tid < n ? l0[0] : 0, h1 = top && tid + 64 < n ? l1[0] : 0;
    for (int r = 0; r < top; ++r) {
      const u64 mine = h0 > h1 ? h0 : h1;
      // the largest value, then among its lanes (one, but for equal values) the largest key
      uint32_t hi = (uint32_t)(mine >> 32);
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) {
        const uint32_t other = __shfl_xor(hi, o);
        hi = other > hi ? other : hi;
      }
      u64 lanes = __builtin_amdgcn_ballot_w64((uint32_t)(mine >> 32) == hi), k = 0;
      int who = 0;
      while (lanes) {
        const int l = __builtin_ctzll(lanes);
        lanes &= lanes - 1;
        const u64 c = lane_key(mine, l);
        if (c >= k) {
          k = c;
          who = l;
        }
      }
      if (tid == 0) best[r] = k;
      if (tid == who && k) {
        if (h0 == k) h0 = ++at0 < top ? l0[at0] : 0;
        else h1 = ++at1 < top ? l1[at1] : 0;
      }
    }
  }
  __syncthreads();
  finish_row(p, row, M, S, W, best);
}

// Values per thread: chunks of 8192 values where they fill the chip (two workgroups a
// CU) or cover a row at once, else of 2048.
static int values_per_thread(int rows, int vocab) {
  const int64_t large = (vocab + 8191) / 8192;
  return large == 1 || rows * large >= 512 || (vocab + 2047) / 2048 > 128 ? 32 : 8;
}

int logprob_chunks(int rows, int vocab) {
  const int c = kT * values_per_thread(rows, vocab);
  return (vocab + c - 1) / c;
}

int64_t logprob_part_bytes(int rows, int vocab, int top) {
  const int64_t n = (int64_t)rows * logprob_chunks(rows, vocab);
  return n * 16 + n * top * 8;
}

hipError_t launch_logprobs(LogprobParams p, int rows, char* part, hipStream_t s) {
  if (p.vocab < 1 || p.vocab > kMaxLogprobVocab || rows < 1 || rows > kLogprobRows || p.top < 0 || p.top > kMaxTop)
    return hipErrorInvalidValue;
  p.chunks = logprob_chunks(rows, p.vocab);
  p.part_keys = reinterpret_cast<unsigned long long*>(part);
  p.part_sums = reinterpret_cast<float*>(part + (int64_t)rows * p.chunks * p.top * 8);
  const dim3 grid(p.chunks, rows);
  if (values_per_thread(rows, p.vocab) == 32) hipLaunchKernelGGL(logprob_chunk_kernel<32>, grid, dim3(kT), 0, s, p);
  else hipLaunchKernelGGL(logprob_chunk_kernel<8>, grid, dim3(kT), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.chunks == 1) return e;
  hipLaunchKernelGGL(logprob_join_kernel, dim3(rows), dim3(kT), 0, s, p);
  return hipGetLastError();
}

}  // namespace kf
