// Kernels that keep some of a user's cached positions (kf_kv_accept, kf_kv_evict): the
// choice of the heaviest, and the gather of keys, values and weights.
//
// A list of ascending positions gives each new position i its old one, list[i] >= i.
// In place, a workgroup takes the new positions in order, a chunk at a time, reads the
// old ones of a chunk before it writes any of it, and never needs a position again that an
// earlier chunk wrote: those lie below the chunk, what it reads does not.
#include <algorithm>

#include "kernels.h"

namespace kf {

namespace {
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));

constexpr int kMoveThreads = 256;

// The old position of new position i (below p.n).
__device__ __forceinline__ int old_of(const KeepParams& p, const int* list, int i) {
  if (list) return list[i];
  return i < p.first ? i : p.first + p.node[i - p.first];
}
__device__ __forceinline__ const int* list_of(const KeepParams& p, int layer, int g) {
  return p.list ? p.list + ((int64_t)layer * p.nkv + g) * p.n : nullptr;
}
}  // namespace

// fp16 keys (blockIdx.z even) or values of one layer and KV head.  In place: one workgroup (grid.x = 1) over all
// new positions; else workgroup x takes chunk x.
template <int HD, bool INPLACE>
__global__ __launch_bounds__(kMoveThreads) void f16_keep_kernel(const KeepParams p) {
  constexpr int PER = HD / 8, ROWS = kMoveThreads / PER, U = 4, CHUNK = ROWS * U;  // 16-byte pieces per position
  const int g = blockIdx.y, layer = blockIdx.z >> 1, tid = threadIdx.x, r = tid / PER, d = (tid % PER) * 8;
  const uint16_t* src = reinterpret_cast<const uint16_t*>((blockIdx.z & 1 ? p.src.v : p.src.k) + layer * p.src.layer_bytes);
  uint16_t* dst = reinterpret_cast<uint16_t*>((blockIdx.z & 1 ? p.dst.v : p.dst.k) + layer * p.dst.layer_bytes);
  const int* list = list_of(p, layer, g);
  const int step = INPLACE ? CHUNK : CHUNK * gridDim.x;
  for (int c0 = p.from + (INPLACE ? 0 : blockIdx.x * CHUNK); c0 < p.n; c0 += step) {
    v4u x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = c0 + u * ROWS + r;
      if (i < p.n) x[u] = *reinterpret_cast<const v4u*>(src + kv_offset(p.src.pages, p.src_user, g, old_of(p, list, i), HD) + d);
    }
    if (INPLACE) __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = c0 + u * ROWS + r;
      if (i < p.n) *reinterpret_cast<v4u*>(dst + kv_offset(p.dst.pages, p.dst_user, g, i, HD) + d) = x[u];
    }
  }
}

// MXFP4 records of one layer and KV head, a page of new positions at a time: K's codes are whole bytes of a position,
// V's pass through LDS, a byte a value, as positions share theirs.
template <int HD, bool INPLACE>
__global__ __launch_bounds__(256) void mx_keep_kernel(const KeepParams p) {
  constexpr int CODES = mx_codes(HD), NB = HD / kMxBlock, KB = HD / 8;  // K code bytes of a position in one lane's run
  __shared__ __attribute__((aligned(16))) uint8_t nib[kKvPage * HD];
  const int g = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x;
  const int* list = list_of(p, layer, g);
  auto record = [&](const CacheRef& c, int user, int page) {
    return c.k + layer * c.layer_bytes + (int64_t)kv_page(c.pages, user, page) * c.pages.page_stride + (int64_t)g * mx_record(HD);
  };
  const int pages = (p.n + kKvPage - 1) / kKvPage, page0 = p.from / kKvPage;
  for (int page = page0 + (INPLACE ? 0 : blockIdx.x); page < pages; page += INPLACE ? 1 : gridDim.x) {
    const int a = max(p.from - page * kKvPage, 0), b = min(p.n - page * kKvPage, kKvPage);
    uint8_t* out = record(p.dst, p.dst_user, page);
    // thread (t, quarter q of the head): K codes, its part of the exponents and scales, and hd/4 V codes
    const int t = tid / 4, q = tid % 4;
    const bool in = t >= a && t < b;
    v4u kc = {0, 0, 0, 0};
    uint8_t ke = 0;
    uint16_t vs = 0;
    if (in) {
      const int from = old_of(p, list, page * kKvPage + t), s = from % kKvPage;
      const uint8_t* rec = record(p.src, p.src_user, from / kKvPage);
      const uint8_t* k = rec + mx_k_byte<HD>(s, q * (HD / 4));
      if (KB == 16) {
        kc = *reinterpret_cast<const v4u*>(k);
      } else {
        const v2u w = *reinterpret_cast<const v2u*>(k);
        kc.x = w.x;
        kc.y = w.y;
      }
      if (q < NB) {
        ke = rec[CODES + mx_k_exp(s, q)];
        vs = reinterpret_cast<const uint16_t*>(rec + mx_v(HD) + CODES)[mx_v_exp<HD>(s, q)];
      }
      const uint8_t* v = rec + mx_v(HD);
#pragma unroll 8
      for (int j = 0; j < HD / 4; ++j) {
        const int d = 4 * j + q;
        nib[t * HD + d] = (v[mx_v_byte(s, d)] >> (4 * (s & 1))) & 15;
      }
    }
    __syncthreads();  // in place: everything of the page's old positions is read
    if (in) {
      uint8_t* k = out + mx_k_byte<HD>(t, q * (HD / 4));
      if (KB == 16) *reinterpret_cast<v4u*>(k) = kc;
      else *reinterpret_cast<v2u*>(k) = v2u{kc.x, kc.y};
      if (q < NB) {
        out[CODES + mx_k_exp(t, q)] = ke;
        reinterpret_cast<uint16_t*>(out + mx_v(HD) + CODES)[mx_v_exp<HD>(t, q)] = vs;
      }
    }
    uint32_t* codes = reinterpret_cast<uint32_t*>(out + mx_v(HD));
    for (int w = tid; w < CODES / 4; w += 256) {  // dword of the V codes: positions 16 (2 s + j / 4) + 4 grp + j % 4 of one d
      const int lane = (w >> 2) & 63, d = 16 * (2 * (w >> 8) + ((w >> 1) & 1)) + (lane & 15), s = w & 1, grp = lane >> 4;
      uint32_t x = 0, mask = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int pos = 16 * (2 * s + j / 4) + 4 * grp + j % 4;
        if (pos < a || pos >= b) continue;
        x |= (uint32_t)nib[pos * HD + d] << (4 * j);
        mask |= 15u << (4 * j);
      }
      if (mask) codes[w] = mask == ~0u ? x : (codes[w] & ~mask) | x;
    }
    __syncthreads();
  }
}

// The weights, one workgroup a layer and KV head.
__global__ __launch_bounds__(1024) void weight_keep_kernel(const KeepParams p) {
  const int g = blockIdx.x, layer = blockIdx.y;
  const int* list = list_of(p, layer, g);
  const float* src = p.weights + (((int64_t)layer * p.users + p.src_user) * p.nkv + g) * p.stride;
  float* dst = p.weights + (((int64_t)layer * p.users + p.dst_user) * p.nkv + g) * p.stride;
  for (int c0 = p.from; c0 < p.n; c0 += 1024) {
    const int i = c0 + threadIdx.x;
    float x = 0.f;
    if (i < p.n) x = src[old_of(p, list, i)];
    __syncthreads();
    if (i < p.n) dst[i] = x;
  }
}

// Which positions to keep, one workgroup a layer and KV head: the m-th largest weight by its digits, most significant
// first (a histogram of the weights that agree so far, and where the m-th lies in it), then
// the positions above it, and of those equal to it the first, in order.
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kBins = 2048;
__device__ __forceinline__ uint32_t weight_key(float w) {  // ordered as the weights are; a NaN below all
  const uint32_t u = __float_as_uint(w + 0.f);
  return w != w ? 0u : u >> 31 ? ~u : u | 0x80000000u;
}
__global__ __launch_bounds__(kSelectThreads) void select_kernel(const SelectParams p) {
  __shared__ int hist[kBins];
  __shared__ int sums[kSelectWaves];
  __shared__ int found[2];
  __shared__ uint32_t counts[2][kSelectWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float* w = p.weights + blockIdx.y * p.layer + blockIdx.x * p.head;
  int* list = p.list + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * p.keep;
  const int lo = p.first, hi = p.len - p.last, m = p.keep - p.first - p.last;
  for (int i = tid; i < p.first; i += kSelectThreads) list[i] = i;
  for (int i = tid; i < p.last; i += kSelectThreads) list[p.keep - p.last + i] = hi + i;
  if (m == 0) return;
  uint32_t prefix = 0, known = 0;
  int need = m;  // of the weights that have the prefix, the need-th largest is the one looked for
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
    for (int b = tid; b < kBins; b += kSelectThreads) hist[b] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += kSelectThreads) {
      const uint32_t k = weight_key(w[i]);
      if ((k & known) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1);
    }
    __syncthreads();
    // thread t holds bins kBins - 1 - 2 t and the next lower
    const int a = hist[kBins - 1 - 2 * tid], b = hist[kBins - 2 - 2 * tid];
    int upto = a + b;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    for (int i = 0; i < wave; ++i) upto += sums[i];
    const int before = upto - a - b;
    if (before < need && need <= upto) {
      const bool second = before + a < need;
      found[0] = kBins - 1 - 2 * tid - second;
      found[1] = need - before - (second ? a : 0);
    }
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    known |= (uint32_t)(bins - 1) << shift;
    need = found[1];
    __syncthreads();
  }
  int above = 0, equal = 0;  // before this chunk
  for (int c0 = lo, turn = 0; c0 < hi; c0 += kSelectThreads, turn ^= 1) {
    const int i = c0 + tid;
    const uint32_t k = i < hi ? weight_key(w[i]) : 0u;
    const uint64_t gt = __ballot(i < hi && k > prefix), eq = __ballot(i < hi && k == prefix), below = (1ull << lane) - 1;
    if (lane == 0) counts[turn][wave] = (uint32_t)__popcll(gt) | (uint32_t)__popcll(eq) << 16;
    __syncthreads();
    uint32_t mine = 0, all = 0;
#pragma unroll
    for (int x = 0; x < kSelectWaves; ++x) {
      all += counts[turn][x];
      if (x < wave) mine += counts[turn][x];
    }
    const int g = above + (int)(mine & 0xffff) + __popcll(gt & below), e = equal + (int)(mine >> 16) + __popcll(eq & below);
    if ((gt >> lane & 1) || ((eq >> lane & 1) && e < need)) list[p.first + g + min(e, need)] = i;
    above += (int)(all & 0xffff);
    equal += (int)(all >> 16);
  }
}

// ------------------------------------------------------------------ launchers
hipError_t launch_select(const SelectParams& p, int nkv, int layers, hipStream_t s) {
  if (p.keep <= 0) return hipSuccess;
  hipLaunchKernelGGL(select_kernel, dim3(nkv, layers), dim3(kSelectThreads), 0, s, p);
  return hipGetLastError();
}
template <int HD>
static hipError_t keep(const KeepParams& p, int layers, hipStream_t s) {
  const bool in_place = p.dst.k == p.src.k && p.dst_user == p.src_user;
  const int n = p.n - p.from;
  if (p.src.mx) {
    const unsigned pages = (unsigned)((p.n + kKvPage - 1) / kKvPage - p.from / kKvPage);
    if (in_place) hipLaunchKernelGGL((mx_keep_kernel<HD, true>), dim3(1, p.nkv, layers), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((mx_keep_kernel<HD, false>), dim3(pages, p.nkv, layers), dim3(256), 0, s, p);
  } else {
    const int chunk = kMoveThreads / (HD / 8) * 4;
    if (in_place) hipLaunchKernelGGL((f16_keep_kernel<HD, true>), dim3(1, p.nkv, 2 * layers), dim3(kMoveThreads), 0, s, p);
    else
      hipLaunchKernelGGL((f16_keep_kernel<HD, false>), dim3((unsigned)((n + chunk - 1) / chunk), p.nkv, 2 * layers),
                         dim3(kMoveThreads), 0, s, p);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && p.weights) {
    hipLaunchKernelGGL(weight_keep_kernel, dim3(p.nkv, layers), dim3(1024), 0, s, p);
    e = hipGetLastError();
  }
  return e;
}
hipError_t launch_keep(const KeepParams& p, int hd, int layers, hipStream_t s) {
  if (p.n <= p.from) return hipSuccess;
  if (p.src.mx != p.dst.mx || (!p.list && (p.n - p.first > kMaxNodes || p.from < p.first))) return hipErrorInvalidValue;
  return hd == 128 ? keep<128>(p, layers, s) : hd == 64 ? keep<64>(p, layers, s) : hipErrorInvalidValue;
}

}  // namespace kf
