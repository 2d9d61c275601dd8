// Kernels that move KV cache contents: MXFP4 encoding and decoding, copies
// between users and caches, copies of shared pages.
//
// All of them are bound by the bytes they move; what they compute per value is a
// few instructions.  16384 positions of 8 heads of 128: bf16 rows encoded, 85 MB, 19 us (4.5 TB/s); decoded to
// fp32 rows, 152 MB, 26 us (5.8); a copy of 2 GiB moves 4.8 on this chip.  MXFP4: a block is 32 consecutive values x of a head, rounded
// to fp16.  With a = max |x|, e = (exponent of a rounded to one mantissa bit,
// nearest even) - 2, clamped: a / 2^e then rounds to at most 6, the largest
// E2M1 number, wherever the clamp does not bind.  Each x / 2^e is rounded to
// E2M1, nearest even, and saturates at 6.
#include <algorithm>

#include "kernels.h"

namespace kf {

namespace {
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));

enum : int { kRowsF32 = 0, kRowsBF16 = 1, kRowsF16 = 2, kPagesF16 = 3 };  // the first three are kf_dtype values

// 8 consecutive values of a row as fp16 pairs; `wide`: at is 16-byte aligned.
__device__ __forceinline__ void load8(const void* base, int type, int64_t at, bool wide, uint32_t (&x)[4]) {
  if (type == kRowsF32) {
    const float* p = reinterpret_cast<const float*>(base) + at;
    v4f a, b;
    if (wide) {
      a = __builtin_nontemporal_load(reinterpret_cast<const v4f*>(p));
      b = __builtin_nontemporal_load(reinterpret_cast<const v4f*>(p) + 1);
    } else {
      a = v4f{p[0], p[1], p[2], p[3]};
      b = v4f{p[4], p[5], p[6], p[7]};
    }
    x[0] = f16_pair(a.x, a.y);
    x[1] = f16_pair(a.z, a.w);
    x[2] = f16_pair(b.x, b.y);
    x[3] = f16_pair(b.z, b.w);
    return;
  }
  const uint16_t* p = reinterpret_cast<const uint16_t*>(base) + at;
  if (wide) {
    const v4u w = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = w[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
  }
  if (type != kRowsBF16) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = f16_pair(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u));
}

// Nibble i of word j to nibble j of word i, of 8 words.
__device__ __forceinline__ void transpose_nibbles(uint32_t (&r)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t a = r[j], b = r[j + 4];
    r[j] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    r[j + 4] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int j = k < 2 ? k : k + 2;
    const uint32_t a = r[j], b = r[j + 2];
    r[j] = __builtin_amdgcn_perm(b, a, 0x06020400u);
    r[j + 2] = __builtin_amdgcn_perm(b, a, 0x07030501u);
  }
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const uint32_t a = r[j], b = r[j + 1];
    r[j] = (a & 0x0f0f0f0fu) | (b & 0x0f0f0f0fu) << 4;
    r[j + 1] = (a >> 4 & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u);
  }
}
}  // namespace

struct MxEncodeParams {
  uint8_t* dst;  // MXFP4 records
  KvPages dp;
  int dst_user;
  int64_t dst_layer;  // bytes per layer
  const void *sk, *sv;
  int src_type;
  int wide;  // rows: sk and sv are 16-byte aligned
  KvPages sp;  // kPagesF16
  int src_user;
  int64_t src_layer;  // bytes per layer
  int pos0, n, nkv;
  int* err_flag;
};

// Workgroup (K or V of one KV head, page, layer), neighbouring workgroups taking the heads of the
// same positions, whose rows lie side by side in the source: encodes the page's positions that
// lie in [pos0, pos0 + n) and leaves the others as they are.  Four lanes hold a
// block, 8 values each.  K codes go out as they are made (8 codes are 4 bytes of a
// row); V codes, whose words hold 8 positions of one d, are exchanged through LDS, 8 x 8 at a
// time.  One workgroup owns all of a head's page, so no byte has two writers.
template <int HD>
__global__ __launch_bounds__(256) void mx_encode_kernel(const MxEncodeParams p) {
  constexpr int UPR = HD / 8;  // 8-value units per position
  constexpr int REC = mx_record(HD), CODES = mx_codes(HD);
  __shared__ uint32_t codes[kKvPage * UPR], turned[CODES / 4];
  const int page = p.pos0 / kKvPage + blockIdx.y, g = blockIdx.x >> 1, is_v = blockIdx.x & 1, tid = threadIdx.x;
  const int a = max(p.pos0 - page * kKvPage, 0), b = min(p.pos0 + p.n - page * kKvPage, kKvPage);
  const void* src = is_v ? p.sv : p.sk;
  bool bad = false;
  // Every load goes out before the first is used.
  constexpr int NU = kKvPage * UPR / 256;
  constexpr int NW = CODES / 4 / 256;
  uint32_t x[NU][4];
  uint32_t old[NW];  // the V codes of a page that is written in part
#pragma unroll
  for (int k = 0; k < NU; ++k) {
    const int u = tid + 256 * k, t = u / UPR, d0 = (u % UPR) * 8;
    if (t < a || t >= b) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[k][i] = 0;
    } else if (p.src_type == kPagesF16) {
      const char* base = reinterpret_cast<const char*>(src) + blockIdx.z * p.src_layer;
      load8(base, kRowsF16, kv_offset(p.sp, p.src_user, g, page * kKvPage + t, HD) + d0, true, x[k]);
    } else {
      load8(src, p.src_type, ((int64_t)(page * kKvPage + t - p.pos0) * p.nkv + g) * HD + d0, p.wide, x[k]);
    }
  }
  uint8_t* rec = p.dst + blockIdx.z * p.dst_layer + (int64_t)kv_page(p.dp, p.dst_user, page) * p.dp.page_stride +
                 (int64_t)g * REC + (is_v ? mx_v(HD) : 0);
  const bool whole = a == 0 && b == kKvPage;
  if (is_v && !whole) {
#pragma unroll
    for (int k = 0; k < NW; ++k) old[k] = reinterpret_cast<const uint32_t*>(rec)[tid + 256 * k];
  }
#pragma unroll
  for (int k = 0; k < NU; ++k) {
    const int u = tid + 256 * k, t = u / UPR, d0 = (u % UPR) * 8;
    int e;
    const uint32_t w = mx_encode8(x[k], e, bad);
    const bool live = t >= a && t < b;
    if (!is_v) {
      if (live) *reinterpret_cast<uint32_t*>(rec + mx_k_byte<HD>(t, d0)) = w;
    } else {
      codes[u] = w;
    }
    if (live && u % 4 == 0) {
      if (is_v) reinterpret_cast<uint16_t*>(rec + CODES)[mx_v_exp<HD>(t, d0 / kMxBlock)] = mx_v_scale(e);
      else rec[CODES + mx_k_exp(t, d0 / kMxBlock)] = (uint8_t)(e + 127);
    }
  }
  raise_err(p.err_flag, bad, kErrF16Range);
  if (!is_v) return;
  __syncthreads();
  if (tid < CODES / 32) {  // positions 16 (2 s + j / 4) + 4 grp + j % 4 of 8 values
    const int c = tid % UPR, s = (tid / UPR) & 1, grp = tid / (2 * UPR), d0 = 8 * c;
    uint32_t r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = codes[(16 * (2 * s + j / 4) + 4 * grp + j % 4) * UPR + c];
    transpose_nibbles(r);
#pragma unroll
    for (int i = 0; i < 8; ++i) turned[mx_v_byte(32 * s + 4 * grp, d0 + i) / 4] = r[i];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NW; ++k) {
    const int w = tid + 256 * k;  // dword of the V codes: 8 positions of one d
    uint32_t* out = reinterpret_cast<uint32_t*>(rec) + w;
    if (whole) {
      *out = turned[w];
      continue;
    }
    uint32_t mask = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = 16 * (2 * (w & 1) + j / 4) + 4 * ((w >> 6) & 3) + j % 4;
      if (t >= a && t < b) mask |= 15u << (4 * j);
    }
    if (mask) *out = (old[k] & ~mask) | (turned[w] & mask);
  }
}

struct MxDecodeParams {
  const uint8_t* src;
  KvPages sp;
  int src_user;
  int64_t src_layer;
  uint8_t *dk, *dv;  // fp32 rows [n][nkv][hd], or fp16 pages
  int wide;  // rows: dk and dv are 16-byte aligned
  KvPages dp;
  int dst_user;
  int64_t dst_layer;
  int pos0, n, nkv;
};

// The way back, exactly: workgroups as above.  V codes pass through LDS, where each
// thread collects the nibbles of its values.  A thread stores 16 bytes, beside its
// neighbours': 4 values of fp32 rows, 8 of fp16 pages.
template <int HD, bool PAGES>
__global__ __launch_bounds__(256) void mx_decode_kernel(const MxDecodeParams p) {
  constexpr int VPU = PAGES ? 8 : 4, UPR = HD / VPU;  // values per unit, units per position
  constexpr int REC = mx_record(HD), CODES = mx_codes(HD);
  __shared__ v4u codes[CODES / 16];
  const int page = p.pos0 / kKvPage + blockIdx.y, g = blockIdx.x >> 1, is_v = blockIdx.x & 1, tid = threadIdx.x;
  const int a = max(p.pos0 - page * kKvPage, 0), b = min(p.pos0 + p.n - page * kKvPage, kKvPage);
  const uint8_t* rec = p.src + blockIdx.z * p.src_layer + (int64_t)kv_page(p.sp, p.src_user, page) * p.sp.page_stride +
                       (int64_t)g * REC + (is_v ? mx_v(HD) : 0);
  constexpr int NU = kKvPage * UPR / 256;
  uint32_t kw[NU];
  float scale[NU];
  if (is_v) {
    for (int i = tid; i < CODES / 16; i += 256) codes[i] = reinterpret_cast<const v4u*>(rec)[i];
  }
#pragma unroll
  for (int k = 0; k < NU; ++k) {
    const int u = tid + 256 * k, t = u / UPR, d0 = (u % UPR) * VPU;
    if (is_v) {
      scale[k] = (float)reinterpret_cast<const _Float16*>(rec + CODES)[mx_v_exp<HD>(t, d0 / kMxBlock)];
    } else {
      const uint8_t* at = rec + mx_k_byte<HD>(t, d0);
      kw[k] = PAGES ? *reinterpret_cast<const uint32_t*>(at) : *reinterpret_cast<const uint16_t*>(at);
      scale[k] = __uint_as_float((uint32_t)rec[CODES + mx_k_exp(t, d0 / kMxBlock)] << 23);
    }
  }
  if (is_v) __syncthreads();
  const uint8_t* lds = reinterpret_cast<const uint8_t*>(codes);
#pragma unroll
  for (int k = 0; k < NU; ++k) {
    const int u = tid + 256 * k, t = u / UPR, d0 = (u % UPR) * VPU;
    if (t < a || t >= b) continue;
    uint32_t w = 0;
    if (is_v) {
#pragma unroll
      for (int i = 0; i < VPU; ++i) w |= (uint32_t)((lds[mx_v_byte(t, d0 + i)] >> (4 * (t & 1))) & 15) << (4 * i);
    } else {
      w = kw[k];
    }
    if constexpr (PAGES) {
      const h2 x0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale[k], 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale[k], 1),
               x2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale[k], 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale[k], 3);
      uint16_t* dst = reinterpret_cast<uint16_t*>((is_v ? p.dv : p.dk) + blockIdx.z * p.dst_layer) +
                      kv_offset(p.dp, p.dst_user, g, page * kKvPage + t, HD) + d0;
      *reinterpret_cast<v4u*>(dst) = v4u{__builtin_bit_cast(uint32_t, x0), __builtin_bit_cast(uint32_t, x1),
                                         __builtin_bit_cast(uint32_t, x2), __builtin_bit_cast(uint32_t, x3)};
    } else {
      const f2 x0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale[k], 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale[k], 1);
      float* dst = reinterpret_cast<float*>(is_v ? p.dv : p.dk) + ((int64_t)(page * kKvPage + t - p.pos0) * p.nkv + g) * HD + d0;
      if (p.wide) {
        __builtin_nontemporal_store(v4f{x0.x, x0.y, x1.x, x1.y}, reinterpret_cast<v4f*>(dst));
      } else {
        dst[0] = x0.x; dst[1] = x0.y; dst[2] = x1.x; dst[3] = x1.y;
      }
    }
  }
}

struct CopyParams {
  CacheRef dst, src;
  int dst_user, src_user, pos0, n;
};

// Workgroup (page, KV head, layer) of an MXFP4 copy: the dwords of the record, of
// which only what belongs to positions [a, b) is replaced.
template <int HD>
__global__ __launch_bounds__(256) void mx_copy_kernel(const CopyParams p) {
  constexpr int REC = mx_record(HD), CODES = mx_codes(HD);
  const int page = p.pos0 / kKvPage + blockIdx.x, g = blockIdx.y;
  const int a = max(p.pos0 - page * kKvPage, 0), b = min(p.pos0 + p.n - page * kKvPage, kKvPage);
  auto record = [&](const CacheRef& c, int user) {
    return c.k + blockIdx.z * c.layer_bytes + (int64_t)kv_page(c.pages, user, page) * c.pages.page_stride + (int64_t)g * REC;
  };
  const uint8_t* src = record(p.src, p.src_user);
  uint8_t* dst = record(p.dst, p.dst_user);
  if (a == 0 && b == kKvPage) {
    for (int i = threadIdx.x; i < REC / 16; i += 256) reinterpret_cast<v4u*>(dst)[i] = reinterpret_cast<const v4u*>(src)[i];
    return;
  }
  auto in = [&](int t) { return t >= a && t < b; };
  for (int i = threadIdx.x; i < REC / 4; i += 256) {
    const int is_v = i * 4 >= mx_v(HD), at = i * 4 - (is_v ? mx_v(HD) : 0);
    uint32_t mask = 0;
    if (at < CODES) {
      if (is_v) {  // 8 positions of one d
        const int grp = (at >> 8) & 3, s = (at >> 2) & 1;
        for (int j = 0; j < 8; ++j)
          if (in(16 * (2 * s + j / 4) + 4 * grp + j % 4)) mask |= 15u << (4 * j);
      } else {  // 8 values of one position
        const int tile = HD == 128 ? at >> 10 : 2 * (at >> 10) + ((at >> 3) & 1);
        if (in(16 * tile + ((at >> 4) & 15))) mask = ~0u;
      }
    } else if (is_v) {  // the scales of 2 positions
      const int w = (at - CODES) / 2, t = 16 * ((w >> 2) & 3) + 4 * ((w >> 4) / (HD / kMxBlock)) + w % 4;
      if (in(t)) mask |= 0xffffu;
      if (in(t + 1)) mask |= 0xffff0000u;
    } else {  // the exponents of 4 positions
      for (int j = 0; j < 4; ++j)
        if (in(16 * j + (((at - CODES) >> 2) & 15))) mask |= 255u << (8 * j);
    }
    if (!mask) continue;
    const uint32_t v = reinterpret_cast<const uint32_t*>(src)[i];
    uint32_t* out = reinterpret_cast<uint32_t*>(dst) + i;
    *out = mask == ~0u ? v : (*out & ~mask) | (v & mask);
  }
}

// fp16 to fp16: 16 bytes a thread, K and V of every layer in grid.y.
__global__ __launch_bounds__(256) void f16_copy_kernel(const CopyParams p, int64_t first, uint32_t total) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= total) return;
  const int hd = p.src.hd, nkv = p.src.nkv;
  const uint32_t row = i / (uint32_t)(hd / 8), d = (i - row * (uint32_t)(hd / 8)) * 8;
  const uint32_t t = row / (uint32_t)nkv, g = row - t * (uint32_t)nkv;
  const int pos = p.pos0 + (int)(first + t);
  const int64_t layer = blockIdx.y >> 1;
  const uint8_t* src = (blockIdx.y & 1 ? p.src.v : p.src.k) + layer * p.src.layer_bytes;
  uint8_t* dst = (blockIdx.y & 1 ? p.dst.v : p.dst.k) + layer * p.dst.layer_bytes;
  *reinterpret_cast<v4u*>(dst + 2 * (kv_offset(p.dst.pages, p.dst_user, (int)g, pos, hd) + d)) =
      *reinterpret_cast<const v4u*>(src + 2 * (kv_offset(p.src.pages, p.src_user, (int)g, pos, hd) + d));
}

__global__ __launch_bounds__(256) void page_copy_kernel(const CacheRef c, const PageCopies u, int64_t page_bytes, const KvTable table,
                                                        const KvTableUpdate t) {
  if (blockIdx.x + blockIdx.y + blockIdx.z == 0) kv_table_apply(table, t, threadIdx.x);
  const int arrays = c.mx ? 1 : 2;
  const int64_t layer = blockIdx.y / arrays;
  uint8_t* base = (blockIdx.y % arrays ? c.v : c.k) + layer * c.layer_bytes;
  const v4u* src = reinterpret_cast<const v4u*>(base + (int64_t)u.src[blockIdx.z] * page_bytes);
  v4u* dst = reinterpret_cast<v4u*>(base + (int64_t)u.dst[blockIdx.z] * page_bytes);
  for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < page_bytes / 16; i += (int64_t)gridDim.x * 256) dst[i] = src[i];
}

__global__ void table_share_kernel(const KvTable t, int src, int dst, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  t.page[dst + i] = t.page[src + i];
  t.version[dst + i]++;
}

// ------------------------------------------------------------------ launchers
static bool aligned16(const void* a, const void* b) { return (((uintptr_t)a | (uintptr_t)b) & 15) == 0; }
static unsigned pages_spanned(int pos0, int n) { return (unsigned)((pos0 + n - 1) / kKvPage - pos0 / kKvPage + 1); }

static hipError_t encode(const MxEncodeParams& p, int hd, int layers, hipStream_t s) {
  const dim3 grid(2 * p.nkv, pages_spanned(p.pos0, p.n), layers);
  if (hd == 128) hipLaunchKernelGGL(mx_encode_kernel<128>, grid, dim3(256), 0, s, p);
  else if (hd == 64) hipLaunchKernelGGL(mx_encode_kernel<64>, grid, dim3(256), 0, s, p);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}
template <bool PAGES>
static hipError_t decode(const MxDecodeParams& p, int hd, int layers, hipStream_t s) {
  const dim3 grid(2 * p.nkv, pages_spanned(p.pos0, p.n), layers);
  if (hd == 128) hipLaunchKernelGGL((mx_decode_kernel<128, PAGES>), grid, dim3(256), 0, s, p);
  else if (hd == 64) hipLaunchKernelGGL((mx_decode_kernel<64, PAGES>), grid, dim3(256), 0, s, p);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_mx_write(const CacheRef& c, int user, int pos0, const void* src_k, const void* src_v, int src_type,
                           int n, int* err_flag, hipStream_t s) {
  MxEncodeParams p{};
  p.dst = c.k;
  p.dp = c.pages;
  p.dst_user = user;
  p.sk = src_k;
  p.sv = src_v;
  p.src_type = src_type;
  p.wide = aligned16(src_k, src_v);
  p.pos0 = pos0;
  p.n = n;
  p.nkv = c.nkv;
  p.err_flag = err_flag;
  return encode(p, c.hd, 1, s);
}

hipError_t launch_mx_read(const CacheRef& c, int user, int pos0, float* dst_k, float* dst_v, int n, hipStream_t s) {
  MxDecodeParams p{};
  p.src = c.k;
  p.sp = c.pages;
  p.src_user = user;
  p.dk = reinterpret_cast<uint8_t*>(dst_k);
  p.dv = reinterpret_cast<uint8_t*>(dst_v);
  p.wide = aligned16(dst_k, dst_v);
  p.pos0 = pos0;
  p.n = n;
  p.nkv = c.nkv;
  return decode<false>(p, c.hd, 1, s);
}

hipError_t launch_cache_copy(const CacheRef& dst, int dst_user, const CacheRef& src, int src_user, int pos0, int n,
                             int layers, int* err_flag, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  if (dst.hd != src.hd || dst.nkv != src.nkv) return hipErrorInvalidValue;
  if (dst.mx && !src.mx) {
    MxEncodeParams p{};
    p.dst = dst.k;
    p.dp = dst.pages;
    p.dst_user = dst_user;
    p.dst_layer = dst.layer_bytes;
    p.sk = src.k;
    p.sv = src.v;
    p.src_type = kPagesF16;
    p.sp = src.pages;
    p.src_user = src_user;
    p.src_layer = src.layer_bytes;
    p.pos0 = pos0;
    p.n = n;
    p.nkv = src.nkv;
    p.err_flag = err_flag;
    return encode(p, src.hd, layers, s);
  }
  if (src.mx && !dst.mx) {
    MxDecodeParams p{};
    p.src = src.k;
    p.sp = src.pages;
    p.src_user = src_user;
    p.src_layer = src.layer_bytes;
    p.dk = dst.k;
    p.dv = dst.v;
    p.dp = dst.pages;
    p.dst_user = dst_user;
    p.dst_layer = dst.layer_bytes;
    p.pos0 = pos0;
    p.n = n;
    p.nkv = src.nkv;
    return decode<true>(p, src.hd, layers, s);
  }
  const CopyParams p{dst, src, dst_user, src_user, pos0, n};
  if (src.mx) {
    const dim3 grid(pages_spanned(pos0, n), src.nkv, layers);
    if (src.hd == 128) hipLaunchKernelGGL(mx_copy_kernel<128>, grid, dim3(256), 0, s, p);
    else if (src.hd == 64) hipLaunchKernelGGL(mx_copy_kernel<64>, grid, dim3(256), 0, s, p);
    else return hipErrorInvalidValue;
    return hipGetLastError();
  }
  // In pieces whose values a 32-bit index holds.
  const int64_t piece = std::max<int64_t>(1, (1LL << 30) / ((int64_t)src.nkv * src.hd));
  for (int64_t p0 = 0; p0 < n; p0 += piece) {
    const uint32_t total = (uint32_t)(std::min<int64_t>(piece, n - p0) * src.nkv * (src.hd / 8));
    hipLaunchKernelGGL(f16_copy_kernel, dim3((total + 255) / 256, 2 * layers), dim3(256), 0, s, p, p0, total);
  }
  return hipGetLastError();
}

hipError_t launch_page_copies(const CacheRef& c, const PageCopies& u, int layers, const KvTable& table,
                              const KvTableUpdate& t, hipStream_t s) {
  if (u.n < 1 || u.n > kPageCopyBatch) return hipErrorInvalidValue;
  const int64_t bytes = c.pages.page_stride * (c.mx ? 1 : 2);
  const unsigned wgs = (unsigned)std::min<int64_t>((bytes / 16 + 1023) / 1024, 64);
  hipLaunchKernelGGL(page_copy_kernel, dim3(wgs, layers * (c.mx ? 1 : 2), u.n), dim3(256), 0, s, c, u, bytes, table, t);
  return hipGetLastError();
}

hipError_t launch_kv_table_share(const KvTable& t, int src, int dst, int n, hipStream_t s) {
  hipLaunchKernelGGL(table_share_kernel, dim3((n + 255) / 256), dim3(256), 0, s, t, src, dst, n);
  return hipGetLastError();
}

}  // namespace kf
