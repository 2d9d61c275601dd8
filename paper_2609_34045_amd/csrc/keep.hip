// Kernels that keep some of a user's cached positions (kf_kv_accept, kf_kv_evict): the
// choice of the heaviest, and the move of keys, values and weights.
//
// A list of ascending positions gives each new position i its old one, list[i] >= i.
// The moves go by pages of new positions: a workgroup reads the old ones of a page, for one KV head and layer, and
// writes them.  In place it must not write before the others have read what lies there.  A few pages (an
// accepted path) go four at a time in one workgroup, which reads them all and then writes: a page reads no position below
// its own.  Many go side by
// side: a workgroup takes a page by a ticket, in order, tells by a flag that it has read, and waits for the flags of the
// pages whose old positions lie in its own (one or two, by the counts that select_kernel leaves).  These have lower
// tickets, so they have started, and nothing waits before it has read: every wait ends.
//
// Bound by memory: 4096 of 16384 fp16 positions of four layers (8 heads of 128) 134 MB in 23 us, 5.9 TB/s.  In place 8001
// of 32000 MXFP4 positions of two layers 22 us (746 in one workgroup a head); 5 accepted of 60 tokens in four layers 4 us.
#include <algorithm>

#include "kernels.h"

namespace kf {

namespace {
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));

enum : int { kApart = 0, kInPlace = 1, kFew = 2 };  // another user's pages; in place, side by side; in place, in order

// The old position of new position i (below p.n).
__device__ __forceinline__ int old_of(const KeepParams& p, const int* list, int i) {
  if (list) return list[i];
  return i < p.first ? i : p.first + p.node[i - p.first];
}

// Values that are here at once, and not each where it is used.
template <int N>
__device__ __forceinline__ void pin(int (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// A page of fp16 keys and values on its way: thread tid has 16 bytes of every ROWS-th position of each.
// (With all list entries and page ids loaded before the rows, 23 us became 25, and an accepted path's 3.8 4.6.)
template <int HD>
struct PageF16 {
  static constexpr int PER = HD / 8, ROWS = 256 / PER, U = kKvPage / ROWS;
  v4u x[2][U];
  __device__ __forceinline__ void read(const KeepParams& p, int layer, int g, const int* list, int page, int a, int b) {
    const int tid = threadIdx.x % 256, d = tid % PER * 8;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = u * ROWS + tid / PER;
      if (t < a || t >= b) continue;
      const int64_t at = 2 * (kv_offset(p.src.pages, p.src_user, g, old_of(p, list, page * kKvPage + t), HD) + d) + layer * p.src.layer_bytes;
      x[0][u] = *reinterpret_cast<const v4u*>(p.src.k + at);
      x[1][u] = *reinterpret_cast<const v4u*>(p.src.v + at);
    }
  }
  __device__ __forceinline__ void write(const KeepParams& p, int layer, int g, int id, int a, int b) {  // to page id
    const int tid = threadIdx.x % 256, d = tid % PER * 8;
    const int64_t base = 2 * (id * p.dst.pages.page_stride + (int64_t)g * kKvPage * HD + d) + layer * p.dst.layer_bytes;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = u * ROWS + tid / PER;
      if (t < a || t >= b) continue;
      const int64_t at = base + 2 * t * HD;
      *reinterpret_cast<v4u*>(p.dst.k + at) = x[0][u];
      *reinterpret_cast<v4u*>(p.dst.v + at) = x[1][u];
    }
  }
};

// A page of MXFP4 records: K's codes are whole bytes of a position, V's pass through LDS, as positions share theirs: the
// V codes of the old pages as they are, where these are at most kSpan, or else a byte a value.  Thread (t, quarter q of
// the head) has K codes and its part of the exponents and scales.
template <int HD>
struct PageMx {
  static constexpr int CODES = mx_codes(HD), NB = HD / kMxBlock, kSpan = 8;
  static_assert(kSpan * CODES >= kKvPage * HD, "both forms");
  uint8_t* nib;  // kSpan CODES bytes in LDS
  int* at;       // [kKvPage] in LDS: the byte of each position's V code of d 0, and its nibble
  bool whole;    // the old pages' V codes are in LDS
  v4u kc;
  uint8_t ke;
  uint16_t vs;
  __device__ __forceinline__ void read(const KeepParams& p, int layer, int g, const int* list, int page, int a, int b) {
    const int tid = threadIdx.x % 256, t = tid / 4, q = tid % 4;
    int old[3];
    old[0] = old_of(p, list, page * kKvPage + min(max(t, a), b - 1));
    old[1] = old_of(p, list, page * kKvPage + a);
    old[2] = old_of(p, list, page * kKvPage + b - 1);
    pin(old);
    const int from = old[0], s = from % kKvPage;
    const int p0 = __builtin_amdgcn_readfirstlane(old[1]) / kKvPage, p1 = __builtin_amdgcn_readfirstlane(old[2]) / kKvPage;
    const int span = p1 - p0 + 1;
    whole = span <= kSpan;
    int id[kSpan + 1];
#pragma unroll
    for (int i = 0; i < kSpan; ++i) id[i] = kv_page(p.src.pages, p.src_user, min(p0 + i, p1));
    id[kSpan] = kv_page(p.src.pages, p.src_user, from / kKvPage);
    pin(id);
    const int64_t head = layer * p.src.layer_bytes + (int64_t)g * mx_record(HD);
    const uint8_t* rec = p.src.k + head + (int64_t)id[kSpan] * p.src.pages.page_stride;
    {
      const uint8_t* k = rec + mx_k_byte<HD>(s, q * (HD / 4));
      if (HD == 128) {
        kc = *reinterpret_cast<const v4u*>(k);
      } else {
        const v2u w = *reinterpret_cast<const v2u*>(k);
        kc.x = w.x;
        kc.y = w.y;
      }
      ke = rec[CODES + mx_k_exp(s, q % NB)];
      vs = reinterpret_cast<const uint16_t*>(rec + mx_v(HD) + CODES)[mx_v_exp<HD>(s, q % NB)];
    }
    v4u v[kSpan][CODES / 16 / 256 ? CODES / 16 / 256 : 1];
    if (whole) {
#pragma unroll
      for (int i = 0; i < kSpan; ++i) {
        if (i >= span) break;
        const v4u* src = reinterpret_cast<const v4u*>(p.src.k + head + (int64_t)id[i] * p.src.pages.page_stride + mx_v(HD));
#pragma unroll
        for (int j = 0; j * 256 < CODES / 16; ++j)
          if (j * 256 + tid < CODES / 16) v[i][j] = src[j * 256 + tid];
      }
    }
    if (t >= a && t < b) {
      if (whole) {
        if (q == 0) at[t] = ((from / kKvPage - p0) * CODES + mx_v_byte(s, 0)) * 2 + (s & 1);
      } else {
        const uint8_t* c = rec + mx_v(HD);
        uint8_t x[HD / 4];
#pragma unroll
        for (int j = 0; j < HD / 4; ++j) x[j] = c[mx_v_byte(s, 4 * j + q)];
#pragma unroll
        for (int j = 0; j < HD / 4; ++j) nib[t * HD + 4 * j + q] = (x[j] >> (4 * (s & 1))) & 15;
      }
    }
    if (whole) {
#pragma unroll
      for (int i = 0; i < kSpan; ++i) {
        if (i >= span) break;
#pragma unroll
        for (int j = 0; j * 256 < CODES / 16; ++j)
          if (j * 256 + tid < CODES / 16) reinterpret_cast<v4u*>(nib + i * CODES)[j * 256 + tid] = v[i][j];
      }
    }
  }
  __device__ __forceinline__ void write(const KeepParams& p, int layer, int g, int id, int a, int b) {
    const int tid = threadIdx.x % 256, t = tid / 4, q = tid % 4;
    uint8_t* out = p.dst.k + layer * p.dst.layer_bytes + (int64_t)id * p.dst.pages.page_stride + (int64_t)g * mx_record(HD);
    if (t >= a && t < b) {
      uint8_t* k = out + mx_k_byte<HD>(t, q * (HD / 4));
      if (HD == 128) *reinterpret_cast<v4u*>(k) = kc;
      else *reinterpret_cast<v2u*>(k) = v2u{kc.x, kc.y};
      if (q < NB) {
        out[CODES + mx_k_exp(t, q)] = ke;
        reinterpret_cast<uint16_t*>(out + mx_v(HD) + CODES)[mx_v_exp<HD>(t, q)] = vs;
      }
    }
    // Dword w = tid + 256 i of the V codes: positions 16 (2 s + j / 4) + 4 grp + j % 4 of d = d0 + 32 i.
    uint32_t* codes = reinterpret_cast<uint32_t*>(out + mx_v(HD));
    const int lane = (tid >> 2) & 63, d0 = 16 * ((tid >> 1) & 1) + (lane & 15), s = tid & 1, grp = lane >> 4;
    uint32_t mask = 0;
    int from[8], shift[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int pos = 16 * (2 * s + j / 4) + 4 * grp + j % 4;
      if (pos >= a && pos < b) mask |= 15u << (4 * j);
      const int w = whole && pos >= a && pos < b ? at[pos] : 0;
      from[j] = whole ? w / 2 + mx_v_byte(0, d0) : pos * HD + d0;
      shift[j] = whole ? 4 * (w & 1) : 0;
    }
    if (!mask) return;
#pragma unroll
    for (int i = 0; i < CODES / 4 / 256; ++i) {
      uint32_t x = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t c = nib[from[j] + i * (whole ? mx_v_byte(0, 32) : 32)];
        x |= (c >> shift[j] & 15u) << (4 * j);
      }
      const int w = tid + 256 * i;
      codes[w] = mask == ~0u ? x : (codes[w] & ~mask) | (x & mask);
    }
  }
};
template <int HD, bool MX>
struct PageOf : PageF16<HD> {};
template <int HD>
struct PageOf<HD, true> : PageMx<HD> {};
}  // namespace

// Replays of two graphs that move in place on one cache share the tickets and flags, and their caller orders them.  Should
// they run at once all the same, no ticket is taken for a page that is not there, and a wait ends after p.waits looks: such
// a page is left as it is, since what lies there may still have to be read, and the stage's error says so.
int keep_waits = 1 << 17;

// A page is 256 threads' work; a kFew workgroup has up to four such groups.
constexpr int groups_of(int mode) { return mode == kFew ? 4 : 1; }
template <int HD, bool MX, int MODE>
__global__ __launch_bounds__(256 * groups_of(MODE)) void keep_kernel(const KeepParams p) {
  constexpr int GROUPS = groups_of(MODE), NIB = MX ? PageMx<HD>::kSpan * PageMx<HD>::CODES : 16;
  __shared__ __attribute__((aligned(16))) uint8_t nib[GROUPS * NIB];
  __shared__ int at[MX ? GROUPS * kKvPage : 1];
  __shared__ int ticket;
  const int page0 = p.from / kKvPage, pages = (p.n + kKvPage - 1) / kKvPage;
  const int tid = threadIdx.x % 256, group = MODE == kFew ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
  PageOf<HD, MX> x;
  if constexpr (MX) {
    x.nib = nib + group * NIB;
    x.at = at + group * kKvPage;
  }
  // Workgroup (x, y): KV head and layer x, page y (kInPlace: the next page that none has), or (kFew) all pages, as many at a
  // time as it has groups.
  const int lg = blockIdx.x, g = lg % p.nkv, layer = lg / p.nkv;
  int nth = blockIdx.y;
  if (MODE == kInPlace) {
    if (tid == 0) ticket = __hip_atomic_fetch_add(&p.tickets[lg * kTicketStep], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    nth = ticket;
    if (nth >= pages - page0) {  // two replays at once
      raise_err(p.err_flag, tid == 0, kErrEvictions);
      return;
    }
  }
  const int* list = p.list ? p.list + (int64_t)lg * p.n : nullptr;
  const float* wsrc = p.weights ? p.weights + (((int64_t)layer * p.users + p.weights_src) * p.nkv + g) * p.stride : nullptr;
  float* wdst = p.weights ? p.weights + (((int64_t)layer * p.users + p.dst_user) * p.nkv + g) * p.stride : nullptr;
  const int first = page0 + (MODE == kFew ? 0 : nth), end = MODE == kFew ? pages : first + 1;
  for (int lead = first; lead < end; lead += MODE == kFew ? blockDim.x / 256 : 1) {
    const int page = lead + group;
    const bool none = MODE == kFew && page >= end;
    const int a = max(p.from - page * kKvPage, 0), b = min(p.n - page * kKvPage, kKvPage);
    // In place, but for a page that takes another's place, which no old key or value lies in.
    const int to = none ? 0 : kv_page(p.dst.pages, p.dst_user, page);
    const bool in_place = MODE != kApart && !none && kv_page(p.src.pages, p.src_user, page) == to;
    // a page whose last position stays where it is has all of them there
    const bool same = none || (in_place && old_of(p, list, page * kKvPage + b - 1) == page * kKvPage + b - 1);
    float w = 0.f;
    if (!same) {
      int wfrom[1] = {old_of(p, list, page * kKvPage + min(max(tid, a), b - 1))};
      x.read(p, layer, g, list, page, a, b);
      if (wsrc && tid < kKvPage) w = wsrc[wfrom[0]];
    }
    // Everything is here before anything behind this is written (and, in LDS, read).
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (MODE == kInPlace) {
      if (tid == 0) __hip_atomic_store(&p.flags[(int64_t)lg * p.pages + page], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (same) return;
    }
    auto waited = [&]() -> bool {  // for the pages with an old position in this one
      bool late = false;
      const int* flags = p.flags + (int64_t)lg * p.pages;
      const int* below = p.below + (int64_t)lg * (p.pages + 1);
      if (tid < 64) {
        const int r0 = below[page], r1 = below[page + 1];
        for (int i = max(r0 / kKvPage, page0) + tid; i < page && i * kKvPage < r1; i += 64) {
          bool set = false;
          for (int n = 0; n < p.waits && !set; ++n) {
            set = __hip_atomic_load(&flags[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (!set) __builtin_amdgcn_s_sleep(2);
          }
          late |= !set;
        }
      }
      late = __syncthreads_or(late);
      raise_err(p.err_flag, late && tid == 0, kErrEvictions);
      return !late;
    };
    if (MODE == kInPlace && in_place && !waited()) return;
    if (!same) {
      x.write(p, layer, g, to, a, b);
      if (MODE == kInPlace && !in_place && !waited()) return;  // (its weights lie here)
      if (wdst && tid >= a && tid < b) wdst[page * kKvPage + tid] = w;
    }
    if (MODE == kFew) __syncthreads();  // LDS is free again
  }
}

// Which positions to keep, one workgroup a layer and KV head: the m-th largest weight by its digits, most significant
// first (a histogram of the weights that agree so far, and where the m-th lies in it), then
// the positions above it, and of those equal to it the first, in order.  A wave has a run of pages, 64 positions at a
// time; with NV, the keys of its NV pages stay in registers (NV 0: they are read again at each pass).
// Bound by what one compute unit loads and counts: 300 positions 6 us, 16384 12, 32000 18.  Each wave lists its weights
// that share the first 11 bits (512 at most, else it goes through all again), so that the other two digits are looked for
// among few, and those few and a count give each wave its place in the list.
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kBins = 2048, kCopies = 4, kListed = 512;
// Sums over the lanes up to this one: of its 16, and of all.
template <int CTRL, int ROWS>
__device__ __forceinline__ int plus_lane(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int scan16(int x) {  // row_shr 1, 2, 4, 8
  return plus_lane<0x118, 0xf>(plus_lane<0x114, 0xf>(plus_lane<0x112, 0xf>(plus_lane<0x111, 0xf>(x))));
}
__device__ __forceinline__ int scan64(int x) {  // and row_bcast 15, 31
  return plus_lane<0x143, 0xc>(plus_lane<0x142, 0xa>(scan16(x)));
}
// The sum of the waves' values before this one's.
__device__ __forceinline__ int before_wave(const int* of, int wave, int lane) {
  const int x = of[lane % kSelectWaves];
  return __builtin_amdgcn_readlane(scan16(lane < wave ? x : 0), 15);
}
// Ordered as the weights are; 1 for a NaN, below all, and 0 stands for no weight.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  return w != w ? 1u : u >> 31 ? ~u : u | 0x80000000u;
}
template <int NV>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(const SelectParams p) {
  __shared__ __attribute__((aligned(16))) int hist[kBins * kCopies];  // a lane counts in copy lane % kCopies (many weights may be alike)
  __shared__ uint32_t listed[kSelectWaves][kListed];
  __shared__ int sums[kSelectWaves], of[2][kSelectWaves];
  __shared__ int found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float* w = p.weights + blockIdx.y * p.layer + blockIdx.x * p.head;
  const int64_t lg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  int* list = p.list + lg * p.keep;
  int* below = p.below + lg * (p.pages + 1);
  const int lo = p.first, hi = p.len - p.last, m = p.keep - p.first - p.last;
  // The wave's pages: positions c0 .. c0 + 64 per - 1.
  const int all = hi > lo ? (hi + kKvPage - 1) / kKvPage - lo / kKvPage : 0, per = NV ? NV : (all + kSelectWaves - 1) / kSelectWaves;
  const int c0 = (lo / kKvPage + wave * per) * kKvPage + lane;
  constexpr int U = NV ? NV : 8;  // pages at a time
  uint32_t held[U];
  auto load = [&](int j0) {
    float x[U];
#pragma unroll
    for (int j = 0; j < U; ++j) x[j] = w[min(max(c0 + (j0 + j) * kKvPage, lo), max(hi, 1) - 1)];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      asm volatile("" : "+v"(x[j]));  // (else each load goes behind a branch on its position, and waits for the one before)
      const int i = c0 + (j0 + j) * kKvPage;
      held[j] = i >= lo && i < hi ? weight_key(x[j]) : 0u;
    }
  };
  if constexpr (NV > 0) load(0);
  auto each = [&](auto what) {
    for (int j0 = 0; j0 < (NV ? 1 : per); j0 += U) {
      if constexpr (NV == 0) load(j0);
#pragma unroll
      for (int j = 0; j < U; ++j)
        if (NV || j0 + j < per) what(j0 + j, held[j]);
    }
  };
  for (int b = tid; b < kBins * kCopies; b += kSelectThreads) hist[b] = 0;
  for (int i = tid; i < p.first; i += kSelectThreads) list[i] = i;
  for (int i = tid; i < p.last; i += kSelectThreads) list[p.keep - p.last + i] = hi + i;
  // for a move in place (kInPlace): how many kept positions lie below each page (those between lo and hi later), no flag
  // set and no ticket taken
  for (int i = tid; i <= p.pages; i += kSelectThreads) {
    if (i < p.pages) p.flags[lg * p.pages + i] = 0;
    const int at = i * kKvPage;
    if (at <= lo) below[i] = at;
    else if (at >= hi) below[i] = min(p.first + m + at - hi, p.keep);
    else if (m == 0) below[i] = lo;
  }
  if (tid == 0) p.tickets[lg * kTicketStep] = 0;
  if (m == 0) return;
  __syncthreads();

  auto count = [&](uint32_t bin) { atomicAdd(&hist[bin * kCopies + lane % kCopies], 1); };
  int need = m;  // of the weights that have the prefix, the need-th largest is the one looked for
  // The bin that holds it, from the top; the histogram is empty again afterwards.
  auto find = [&]() {
    __syncthreads();
    int* mine = &hist[(kBins - 2 - 2 * tid) * kCopies];  // thread t: bins kBins - 1 - 2 t and the next lower
    int a = 0, b = 0;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      b += mine[i];
      a += mine[kCopies + i];
    }
    int upto = scan64(a + b);
    if (lane == 63) sums[wave] = upto;
#pragma unroll
    for (int i = 0; i < 2 * kCopies; ++i) mine[i] = 0;
    __syncthreads();
    upto += before_wave(sums, wave, lane);
    const int before = upto - a - b;
    if (before < need && need <= upto) {
      const bool second = before + a < need;
      found[0] = kBins - 1 - 2 * tid - second;
      found[1] = need - before - (second ? a : 0);
    }
    __syncthreads();
    need = found[1];
    return (uint32_t)found[0];
  };
  each([&](int, uint32_t k) { count(k >> 21); });
  uint32_t prefix = find() << 21;
  // The wave's weights with this prefix, listed (or, where they are too many, taken from all again), and how many lie above.
  int above = 0, n = 0;
  auto rank = [&](uint64_t x) {  // bits of the lower lanes
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(x >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)x, 0));
  };
  each([&](int, uint32_t k) {
    const bool mine = k >> 21 == prefix >> 21;
    above += __popcll(__ballot(k >> 21 > prefix >> 21));
    const uint64_t with = __ballot(mine);
    const int at = n + rank(with);
    if (mine && at < kListed) listed[wave][at] = k;
    n += __popcll(with);
  });
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (the lanes read each other's)
  __builtin_amdgcn_wave_barrier();
  auto each_listed = [&](auto what) {  // all 64 lanes, 0 where there is none
    if (n <= kListed) {
      for (int i = lane; i - lane < n; i += 64) {
        const uint32_t k = listed[wave][min(i, kListed - 1)];
        what(i < n ? k : 0u);
      }
    } else {
      each([&](int, uint32_t k) { what(k >> 21 == prefix >> 21 ? k : 0u); });
    }
  };
  auto digit = [&](int shift, int known, uint32_t bins) {
    each_listed([&](uint32_t k) {
      if (k && (k ^ prefix) >> known == 0) count(k >> shift & (bins - 1));
    });
    prefix |= find() << shift;
  };
  digit(10, 21, 2048);
  digit(0, 10, 1024);

  int equal = 0;  // (these and those above:) in the wave, in the waves before it, then before the position
  each_listed([&](uint32_t k) {
    above += __popcll(__ballot(k > prefix));
    equal += __popcll(__ballot(k == prefix));
  });
  if (lane == 0) {
    of[0][wave] = above;
    of[1][wave] = equal;
  }
  __syncthreads();
  above = before_wave(of[0], wave, lane);
  equal = before_wave(of[1], wave, lane);
  const int page0 = c0 / kKvPage;
  int* out = list + p.first;
  int counts = 0;  // lane j % 64: what lies below page j
  auto tell = [&](int j, int n) {
    const int page = page0 + j - n + 1 + lane;
    if (lane < n && page * kKvPage > lo && page * kKvPage < hi) below[page] = counts;
  };
  each([&](int j, uint32_t k) {
    const bool over = k > prefix;
    bool mine = over;
    const uint64_t eq = __ballot(k == prefix);
    const int before = above + min(equal, need);
    above += __popcll(__ballot(over));
    if (eq) {  // the first of these that are still needed
      const int left = need - equal;
      equal += __popcll(eq);
      mine |= k == prefix && rank(eq) < left;
    }
    if (mine) out[before + rank(__ballot(mine))] = c0 + j * kKvPage;
    if (lane == j % 64) counts = p.first + before;
    if (j % 64 == 63 || j == per - 1) tell(j, j % 64 + 1);
  });
}

// ------------------------------------------------------------------ launchers
hipError_t launch_select(const SelectParams& p, int nkv, int layers, hipStream_t s) {
  if (p.keep <= 0) return hipSuccess;
  const int pages = std::max((p.len - p.last + kKvPage - 1) / kKvPage - p.first / kKvPage, 0);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(nkv, layers), dim3(kSelectThreads), 0, s, p); };
  if (pages <= 4 * kSelectWaves) launch(select_kernel<4>);
  else if (pages <= 16 * kSelectWaves) launch(select_kernel<16>);
  else if (pages <= 32 * kSelectWaves) launch(select_kernel<32>);
  else launch(select_kernel<0>);
  return hipGetLastError();
}
template <int HD, bool MX>
static hipError_t keep(const KeepParams& p, hipStream_t s) {
  const unsigned pages = (unsigned)((p.n + kKvPage - 1) / kKvPage - p.from / kKvPage), heads = p.nkv * p.layers;
  const dim3 grid(heads, pages);  // (as one number, 1024 heads of 2^20 positions would be 2^32 threads, which a grid cannot have)
  if (!p.in_place) hipLaunchKernelGGL((keep_kernel<HD, MX, kApart>), grid, dim3(256), 0, s, p);
  else if (p.list) hipLaunchKernelGGL((keep_kernel<HD, MX, kInPlace>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((keep_kernel<HD, MX, kFew>), dim3(heads), dim3(256 * std::min(pages, (unsigned)groups_of(kFew))), 0, s, p);
  return hipGetLastError();
}
hipError_t launch_keep(const KeepParams& p, int hd, hipStream_t s) {
  if (p.n <= p.from) return hipSuccess;
  if (p.src.mx != p.dst.mx || (!p.list && (p.n - p.first > kMaxNodes || p.from < p.first))) return hipErrorInvalidValue;
  if (hd == 128) return p.src.mx ? keep<128, true>(p, s) : keep<128, false>(p, s);
  if (hd == 64) return p.src.mx ? keep<64, true>(p, s) : keep<64, false>(p, s);
  return hipErrorInvalidValue;
}

}  // namespace kf
