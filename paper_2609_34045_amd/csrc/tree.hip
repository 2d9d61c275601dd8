// Attention of trees of drafted tokens over a cache (kf_kv_attend_tree): up to kMaxNodes
// tokens of each of up to four users, whose keys and values lie behind the user's len
// cached positions.
//
//   out_ih = sum_t p_t v_t / sum_t p_t,  p_t = 2^(s_t - m),  s_t = q_ih . k_t log2(e) / sqrt(hd),
//   t over [0, len) and len + a for i and each ancestor a of i
//
// The columns of a KV head are its tree's tokens times the G query heads of its
// group, token by token.  A workgroup takes a tile of them and a range of 64-key
// blocks (one page each), a wave 32 columns of the tile: S^T = K Q^T, softmax per lane,
// O^T += V^T P^T, all on 32x32x16 fp16 MFMAs.  K and V pass through LDS, so that the
// waves share what they read; the splits of a row meet in tree_merge_kernel.
//
// Probabilities are taken in two fp16 parts, each product with both: 22 bits, whatever the type.  PARTS: the same of the
// queries.  One for bf16 queries: times the power of two of their head, fp16 holds those down to 2^-27 of its largest
// exactly, and smaller ones to 2^-38 of that; two for fp32 and fp16 queries.
//
// What bounds it: the matrix and vector units, in turn.  128 fp32 tokens of 64 heads at 40001 positions (8 KV heads of
// 128): 336 GFLOP of products in 300 to 340 us, a large library product's rate; 64 bf16 tokens of 32 heads at 32768
// 66 us (51 GFLOP, 45 us at that rate; 10 are a launch's fixed part), where each unit is busy 53% of the time.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.h"

namespace kf {

namespace {
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s* lds_v4s;

__device__ __forceinline__ f32x16 mfma32(v4u a, v4u b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
// Over lanes l and l ^ 32.
__device__ __forceinline__ float max32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// 8 consecutive values of a query row of type IO (0 fp32, 1 bf16, 2 fp16).
template <int IO>
__device__ __forceinline__ void load_q8(const void* q, int64_t at, float (&f)[8]) {
  if constexpr (IO == 0) {
    const v4f* p = reinterpret_cast<const v4f*>(reinterpret_cast<const float*>(q) + at);
    const v4f a = p[0], b = p[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
    const v4u w = *reinterpret_cast<const v4u*>(reinterpret_cast<const uint16_t*>(q) + at);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint16_t h = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
      f[i] = IO == 1 ? __uint_as_float((uint32_t)h << 16) : (float)__builtin_bit_cast(_Float16, h);
    }
  }
}
// 4 consecutive output values in fp32, bf16 or fp16 (nearest even).
__device__ __forceinline__ void store_out4(void* out, int type, int64_t at, v4f v) {
  if (type == 0) {
    float* o = reinterpret_cast<float*>(out) + at;
    o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
    return;
  }
  uint16_t* o = reinterpret_cast<uint16_t*>(out) + at;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    o[i] = type == 1 ? __builtin_bit_cast(uint16_t, (__bf16)v[i]) : __builtin_bit_cast(uint16_t, (_Float16)v[i]);
}

constexpr int kKB = kKvPage;       // keys per block
constexpr int kNoToken = -2;       // the parent of a row that only pads

// Slot of 16-byte chunk c of key row r: a K fragment read takes one chunk of 16 consecutive rows (HD 64: 8
// same-parity rows among 16) per LDS cycle, a V transpose read 4 rows x 4 chunks; f(r) puts both on distinct
// 16-byte bank groups.
template <int HD>
__device__ __forceinline__ int kv_slot(int r, int c) {
  return HD == 128 ? c ^ (((r & 3) << 2) | ((r >> 2) & 3)) : c ^ ((((r >> 1) & 1) << 2) | ((r >> 2) & 3));
}
// Of chunk c (8 keys) of row d of a transposed V block.
__device__ __forceinline__ int vt_slot(int d, int c) { return c ^ ((d >> 1) & 7); }

// N times 16 bytes a lane from base + at[j] to the LDS bytes dst + 4096 j + 16 lane.  In assembly: the compiler would have
// every transpose read wait for all of these in flight, where the loop waits for those it needs (wait_loads).  (The scalar
// operands may come from a vector instruction just before, which a vector memory operation may read 5 states later.)
template <int N>
__device__ __forceinline__ void direct_loads(const char* base, const uint32_t (&at)[N], uint32_t dst) {
  static_assert(N == 2 || N == 4, "loads of a block");
  uint32_t m0;  // as it was, and is again afterwards
  if constexpr (N == 2)
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %2, %4\n\t"
        "s_add_u32 m0, m0, 4096\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %4\n\ts_mov_b32 m0, %0"
        : "=&s"(m0)
        : "s"(dst), "v"(at[0]), "v"(at[1]), "s"(base)
        : "memory", "scc");
  else
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %2, %6\n\t"
        "s_add_u32 m0, m0, 4096\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %6\n\t"
        "s_add_u32 m0, m0, 4096\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %6\n\t"
        "s_add_u32 m0, m0, 4096\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %6\n\ts_mov_b32 m0, %0"
        : "=&s"(m0)
        : "s"(dst), "v"(at[0]), "v"(at[1]), "v"(at[N - 2]), "v"(at[N - 1]), "s"(base)
        : "memory", "scc");
}
// Waits for this wave's vector memory operations, the direct loads among them.
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// What each token of a tree of n sees of it, 256 bits a token: itself and its ancestors, by doubling the
// way up.  A parent that is no earlier token counts as none.
__device__ __forceinline__ void see_ancestors(const int32_t* parents, int n, uint64_t (*see)[kMaxNodes / 64], int* up, int tid) {
  static_assert(kMaxNodes == 256, "a thread a token");
  int mine = -1;
  uint64_t bits[kMaxNodes / 64] = {};
  if (tid < n) {
    const int par = parents[tid];
    mine = par >= 0 && par < tid ? par : -1;
#pragma unroll
    for (int w = 0; w < kMaxNodes / 64; ++w)
      if (par != kNoToken && tid / 64 == w) bits[w] = 1ull << (tid % 64);
  }
  for (;;) {
#pragma unroll
    for (int w = 0; w < kMaxNodes / 64; ++w) see[tid][w] = bits[w];
    up[tid] = mine;
    if (!__syncthreads_or(mine >= 0)) return;  // (a barrier too)
    uint64_t theirs[kMaxNodes / 64] = {};
    int next = -1;
    if (mine >= 0) {
#pragma unroll
      for (int w = 0; w < kMaxNodes / 64; ++w) theirs[w] = see[mine][w];
      next = up[mine];
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kMaxNodes / 64; ++w) bits[w] |= theirs[w];
    mine = next;
  }
}
}  // namespace

template <int HD, bool MX, int PARTS>
__global__ __launch_bounds__(256, 2) void attn_tree_kernel(const TreeParams p) {
  constexpr int NT = kKB / 32;               // 32-key tiles per block
  constexpr int NS = HD / 16, DB = HD / 32;  // 16-wide d slices of S, 32-row d blocks of O^T
  constexpr int CPR = HD / 8;                // 16-byte chunks per key row
  constexpr int ROWB = HD * 2;               // bytes per key row
  constexpr int VTB = kKB * 2;               // bytes per row (one d) of a transposed V block
  constexpr int TILEB = kKB * ROWB;          // a block of K or V
  constexpr int RPI = 64 / CPR;              // key rows per 1 KB direct load
  constexpr int LPW = TILEB / 1024 / 4;      // direct loads per wave per block of K or V
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * TILEB];  // two stages: K, V behind it
  __shared__ uint64_t see[kMaxNodes][kMaxNodes / 64];
  __shared__ int up[kMaxNodes];
  __shared__ int again;  // some result is no number

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Consecutive workgroups go to the 8 XCDs in turn: numbering the work XCD by XCD keeps the tiles that read the
  // same keys on one L2.
  int id = blockIdx.x;
  if (gridDim.x % 8 == 0) id = (id % 8) * (gridDim.x / 8) + id / 8;
  int b = 0;
  while (b < p.trees - 1 && id >= p.tree[b].wgs) id -= p.tree[b++].wgs;
  const TreeOf tr = p.tree[b];
  const int G = p.nq / p.nkv, cols = tr.nodes * G;
  const int tile = id % tr.tiles, z = (id / tr.tiles) % tr.splits, g = id / (tr.tiles * tr.splits);
  const int total = tr.len + tr.nodes;
  const int blk0 = z * tr.blocks, blk1 = min(blk0 + tr.blocks, (total + kKB - 1) / kKB);
  const int c0 = (tile * 4 + wave) * 32;  // the wave's first column
  const bool live = c0 < cols;            // a wave without columns only loads
  const int half_sel = lane >> 5, rl = lane & 31;
  const int col = c0 + rl, node = min(col, cols - 1) / G;
  const int64_t head = ((int64_t)tr.row0 + node) * p.nq + g * G + min(col, cols - 1) % G;  // its row and query head

  // Page ids of pages [pb, pb + 64), lane i holding page pb + i's.
  int pb = blk0, pid = 0;
  auto load_pids = [&]() {
    pid = (p.kv.table && pb + lane < p.kv.ppu) ? p.kv.table[tr.user * p.kv.ppu + pb + lane] : 0;
    asm volatile("" : "+v"(pid));  // waited for here, and not at each use, where it would be a wait for every direct load
  };
  load_pids();
  // The bytes from one page's start to the KV head's place in page n.
  const bool paged = p.kv.table != nullptr;
  const int first_page = tr.user * p.kv.ppu;
  const uint32_t page_bytes = (uint32_t)p.kv.page_stride * (MX ? 1 : 2);
  auto page_at = [&](int n) -> uint64_t {
    if (paged && n >= pb + 64) {
      pb = n;
      load_pids();
    }
    const uint32_t id = paged ? __builtin_amdgcn_readlane(pid, n - pb) : first_page + n;
    return (uint64_t)id * page_bytes;
  };

  // ---- keys and values into the stages
  // fp16: load j of this wave fills rows RPI (4 j + wave) ..; lane l writes row RPI (4 j + wave) + l / CPR, slot l % CPR.
  // Rows past the last key are loaded from it, and masked.
  uint32_t dma[LPW];
#pragma unroll
  for (int j = 0; j < LPW; ++j) {
    const int r = RPI * (4 * j + wave) + lane / CPR;
    dma[j] = r * ROWB + kv_slot<HD>(r, lane % CPR) * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr)smem + 1024 * wave;
  const char* heads[2] = {reinterpret_cast<const char*>(p.kc) + (int64_t)g * kKvPage * ROWB,
                          reinterpret_cast<const char*>(p.vc) + (int64_t)g * kKvPage * ROWB};
  auto load_f16 = [&](int blk, int stage) {
    const uint64_t off = page_at(blk);
    const int last = total - 1 - blk * kKB;
    if (last >= kKB - 1) {
      direct_loads(heads[0] + off, dma, lds0 + 2 * stage * TILEB);
      direct_loads(heads[1] + off, dma, lds0 + (2 * stage + 1) * TILEB);
    } else {
      uint32_t at[LPW];
#pragma unroll
      for (int j = 0; j < LPW; ++j) {
        const int r = RPI * (4 * j + wave) + lane / CPR;
        at[j] = min(r, last) * ROWB + kv_slot<HD>(r, lane % CPR) * 16;
      }
      direct_loads(heads[0] + off, at, lds0 + 2 * stage * TILEB);
      direct_loads(heads[1] + off, at, lds0 + (2 * stage + 1) * TILEB);
    }
  };
  // MXFP4: jobs 0 .. hd/32 - 1 are 1 KB of K codes each, the others of V; wave w takes w
  // and w + 4.
  constexpr int JOBS = HD / 16 / 4, REC = mx_record(HD), CODES = mx_codes(HD), NB = HD / kMxBlock;
  const int r16 = lane & 15, grp = lane >> 4;
  v4u code[JOBS], vsc[2];
  uint32_t ke = 0;
  auto load_mx = [&](int blk) {
    const uint8_t* rec = p.rec + page_at(blk) + (int64_t)g * REC;
#pragma unroll
    for (int i = 0; i < JOBS; ++i) {
      const int job = wave + 4 * i;
      const bool is_v = job >= HD / 32;
      const int j = job % (HD / 32);
      code[i] = *reinterpret_cast<const v4u*>(rec + (is_v ? mx_v(HD) : 0) + j * 1024 + lane * 16);
      if (!is_v) ke = *reinterpret_cast<const uint32_t*>(rec + CODES + ((HD == 128 ? grp : grp / 2) * 16 + r16) * 4);
      else
#pragma unroll
        for (int k = 0; k < 2; ++k)
          vsc[k] = *reinterpret_cast<const v4u*>(rec + mx_v(HD) + CODES + (grp * NB + j) * 32 + 16 * k);
    }
  };
  auto store_mx = [&](uint8_t* stage) {
#pragma unroll
    for (int i = 0; i < JOBS; ++i) {
      const int job = wave + 4 * i;
      const int j = job % (HD / 32);
      if (job < HD / 32) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {  // 8 values of a key
          const int tile16 = HD == 128 ? j : 2 * j + w / 2, row = 16 * tile16 + r16;
          const int chunk = HD == 128 ? grp * 4 + w : grp * 2 + (w & 1);
          const float sc = __uint_as_float(((ke >> (8 * tile16)) & 255u) << 23);
          const v4u x = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], sc, 0)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], sc, 1)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], sc, 2)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], sc, 3))};
          *reinterpret_cast<v4u*>(stage + row * ROWB + kv_slot<HD>(row, chunk) * 16) = x;
        }
      } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) {  // positions 16 (2 (w & 1) + k / 4) + 4 grp + k % 4 of one d
          const int d = 16 * (2 * j + w / 2) + r16;
          const h8 vs = __builtin_bit_cast(h8, vsc[w & 1]);
          const h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], 1.0f, 0) * __builtin_shufflevector(vs, vs, 0, 1),
                   c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], 1.0f, 1) * __builtin_shufflevector(vs, vs, 2, 3),
                   e = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], 1.0f, 2) * __builtin_shufflevector(vs, vs, 4, 5),
                   f = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], 1.0f, 3) * __builtin_shufflevector(vs, vs, 6, 7);
          // A 16-key step's four groups lie 0 2 1 3, so that one read takes the two of a half of the lanes.
          uint8_t* at = stage + TILEB + d * VTB;
          const int c0 = 4 * (w & 1) + (grp & 1);
          *reinterpret_cast<v2u*>(at + vt_slot(d, c0) * 16 + (grp >> 1) * 8) =
              v2u{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c)};
          *reinterpret_cast<v2u*>(at + vt_slot(d, c0 + 2) * 16 + (grp >> 1) * 8) =
              v2u{__builtin_bit_cast(uint32_t, e), __builtin_bit_cast(uint32_t, f)};
        }
      }
    }
  };
  if (tid == 0) again = 0;
  if constexpr (MX) load_mx(blk0);
  else load_f16(blk0, 0);

  // Q^T fragments: this lane's column, d = 16 s + 8 half_sel .. +7, times a power of two that puts the head's largest
  // value near 2^13 (query_exponent): `sscale` takes a score back, to log2 units.
  v4u qf[PARTS][NS];
  float sscale;
  {
    float top = 0.f;
    float f[NS][8];
    auto load = [&](auto io) {  // the type's branch outside the loads: they go out together
#pragma unroll
      for (int s = 0; s < NS; ++s) load_q8<decltype(io)::value>(p.q, head * HD + 16 * s + 8 * half_sel, f[s]);
    };
    if constexpr (PARTS == 1) load(std::integral_constant<int, 1>());
    else if (p.io == 0) load(std::integral_constant<int, 0>());
    else load(std::integral_constant<int, 2>());
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, __builtin_fabsf(f[s][j]));
    const int e = query_exponent(max32(top));
    const float scale = query_scale(e);
    sscale = p.scale_log2 * query_unscale(e);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[s][j] *= scale;
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
        qf[part][s] = v4u{f16_part2(f[s][0], f[s][1], part), f16_part2(f[s][2], f[s][3], part),
                          f16_part2(f[s][4], f[s][5], part), f16_part2(f[s][6], f[s][7], part)};
    }
  }
  if (blk1 * kKB > tr.len) see_ancestors(p.parents + tr.row0, tr.nodes, see, up, tid);
  if constexpr (MX) store_mx(smem);

  f32x16 o[DB];
  float m_run, l_run;

  // ---- operands
  // Byte offsets of this lane's fragments within a block: K's of slice s and the first tile; V's of d block d, whose key step st (16 keys) takes
  // this half's keys 16 st + 4 half_sel + {0..3} and + 8 + {0..3}.  A transpose read (two of them, keys 8 apart): within
  // 16 lanes, lane 4 r + j reads 4 consecutive d of key row r, and lane c receives element c of the four rows.
  int koff[NS], voff[DB][2];
#pragma unroll
  for (int s = 0; s < NS; ++s) koff[s] = rl * ROWB + kv_slot<HD>(rl, 2 * s + half_sel) * 16;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if constexpr (MX) {  // step st: this with chunk bits 1 and 2 turned by st
        voff[d][e] = (32 * d + rl) * VTB + vt_slot(32 * d + rl, half_sel) * 16;
      } else {
        const int key = 8 * e + 4 * (grp >> 1) + ((lane >> 2) & 3), dd = 32 * d + 16 * (grp & 1) + 4 * (lane & 3);
        voff[d][e] = key * ROWB + kv_slot<HD>(key, dd >> 3) * 16 + (dd & 7) * 2;
      }
    }
  auto kread = [&](const uint8_t* ks, int i) {  // product i: key tile i % NT, slice i / NT
    return *reinterpret_cast<const v4u*>(ks + i % NT * 32 * ROWB + koff[i / NT]);
  };
  auto vread = [&](const uint8_t* vs, int i) {  // of step i / DB, d block i % DB
    if constexpr (MX) {
      return *reinterpret_cast<const v4u*>(vs + (voff[i % DB][0] ^ (i / DB * 32)));
    } else {
      const uint8_t* a0 = vs + voff[i % DB][0] + i / DB * 16 * ROWB;
      const uint8_t* a1 = vs + voff[i % DB][1] + i / DB * 16 * ROWB;
      const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)a0);
      const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)a1);
      const v2u l2 = __builtin_bit_cast(v2u, lo), h2v = __builtin_bit_cast(v2u, hi);
      return v4u{l2.x, l2.y, h2v.x, h2v.y};
    }
  };

  // Which of a block's 64 positions the column's token sees: those before len, and of the tree its own bits.
  auto mask = [&](int blk, f32x16 (&st)[NT]) {
    const int a0 = blk * kKB - tr.len;
    uint64_t sees;
    if (a0 < 0) {
      sees = (see[node][0] << -a0) | ((1ull << -a0) - 1);
    } else {
      const int w = a0 >> 6, sh = a0 & 63;
      sees = see[node][w] >> sh;
      if (sh && w + 1 < kMaxNodes / 64) sees |= see[node][w + 1] << (64 - sh);
    }
    sees >>= 4 * half_sel;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (!((uint32_t)(sees >> (32 * t)) >> (8 * (v >> 2) + (v & 3)) & 1u)) st[t][v] = -INFINITY;
  };
  bool odd = false;      // some value was no number, the same in every thread
  bool careful = false;  // the second time over the blocks, likewise
  // An infinity or NaN among the values that some tokens do not see would reach them as 0 times it: out of the
  // products with it, and into the sums of those that see it behind the loop.
  auto take_out = [&](uint8_t* vs) {
    constexpr int CPT = TILEB / 16 / 256;
    v4u* vt = reinterpret_cast<v4u*>(vs) + tid;
    bool some = false;
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      v4u x = vt[256 * i];
      bool here = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool lo = (x[e] & 0x7c00u) == 0x7c00u, hi = (x[e] & 0x7c000000u) == 0x7c000000u;
        here |= lo | hi;
        x[e] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
      }
      if (here) vt[256 * i] = x;
      some |= here;
    }
    odd |= __syncthreads_or(some);
  };

  f32x16 st[NT], zero;
#pragma unroll
  for (int v = 0; v < 16; ++v) zero[v] = 0.f;
  v4u pf[2][2 * NT];  // P^T fragments of a block's key steps, in two parts
  auto step = [&](int blk, auto parity) {
    constexpr int P = decltype(parity)::value;
    uint8_t* const stage = smem + P * 2 * TILEB;
    uint8_t* const next = smem + (1 - P) * 2 * TILEB;
    if constexpr (!MX) wait_loads();
    barrier();  // the block is here, and every wave is done with the one before
    const bool more = blk + 1 < blk1;
    if (more) {
      if constexpr (MX) load_mx(blk + 1);
      else load_f16(blk + 1, 1 - P);
    }
    const bool tail = blk * kKB + kKB > tr.len;  // positions of the tree, or past it
    if constexpr (!MX) {
      if (tail || careful) take_out(stage + TILEB);
    }
    if (live) {
      constexpr int NI = NT * NS, RING = 4;
      v4u ring[RING];  // K's operands a few reads ahead of their products
#pragma unroll
      for (int i = 0; i < RING; ++i) ring[i] = kread(stage, i);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
          st[i % NT] = mfma32(ring[i % RING], qf[part][i / NT], i / NT || part ? st[i % NT] : zero);
        if (i + RING < NI) ring[i % RING] = kread(stage, i + RING);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (!MX && PARTS == 2) {
        if (__builtin_expect(careful, 0)) {  // an infinite key's score is that of the first parts: with the second, of another sign or 0, it is NaN
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            f32x16 first = zero;
#pragma unroll
            for (int s = 0; s < NS; ++s) first = mfma32(kread(stage, s * NT + t), qf[0][s], first);
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (__builtin_fabsf(first[v]) == INFINITY) st[t][v] = first[v];
          }
        }
      }
      if (tail) mask(blk, st);
      // The reference of the softmax moves only when a block's maximum exceeds it by kPartLazy, so that O is rarely rescaled.
      float mb = -INFINITY;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) mb = fmaxf(mb, st[t][v]);
      mb = max32(mb);
      // Until a position is seen the maximum is -inf, and 0 stands in, so that nothing is added.
      const float m_new = (mb - m_run) * sscale > kPartLazy ? mb : m_run;
      const float m_ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f((m_run - m_ref) * sscale);
      m_run = m_new;
      // A probability is 2^(s sscale + c); c is rounded, to 2^-5 at scores of 2^20, the same way for all of a block, and
      // past those the distance from the reference is taken first, exact near it.
      float c = __builtin_fmaf(-m_ref, sscale, kPartShift);
      if (__ballot(!(__builtin_fabsf(c) < 0x1p20f))) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v) st[t][v] -= m_ref;
        c = kPartShift;
      }
      float ls = 0.f;
#pragma unroll
      for (int i = 0; i < 16 * NT; i += 2) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(st[i / 16][i % 16], sscale, c));
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(st[i / 16][i % 16 + 1], sscale, c));
        pf[0][i / 8][i / 2 % 4] = f16_pair(x, y);
        pf[1][i / 8][i / 2 % 4] = f16_part2(x, y, 1.0f);
        ls += x + y;
      }
      l_run = l_run * alpha + sum32(ls);
      if (__ballot(alpha != 1.0f)) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[d][v] *= alpha;
      }
      constexpr int NV = 2 * NT * DB, AHEAD = 8;
      v4u vr[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) vr[i] = vread(stage + TILEB, i);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int part = 0; part < 2; ++part) o[i % DB] = mfma32(vr[i % AHEAD], pf[part][i / DB], o[i % DB]);
        if (i + AHEAD < NV) vr[i % AHEAD] = vread(stage + TILEB, i + AHEAD);
      }
    }
    if constexpr (MX) {
      if (more) store_mx(next);
    }
  };
  for (;;) {
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[d][v] = 0.f;
    for (int blk = blk0; blk < blk1; blk += 2) {
      step(blk, std::integral_constant<int, 0>());
      if (blk + 1 < blk1) step(blk + 1, std::integral_constant<int, 1>());
    }
    // An fp16 cache may hold infinities (what did not fit), and two parts of which one is 0 or of another sign make NaN of
    // them: where a result is no number, all blocks once more, with infinite values taken out and infinite keys looked at.
    if (MX || careful) break;
    f32x16 sum = o[0];
#pragma unroll
    for (int d = 1; d < DB; ++d) sum += o[d];
    float all = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) all += sum[v];
    if (__ballot(!(__builtin_fabsf(all) < INFINITY)) && lane == 0) again = 1;
    __syncthreads();
    careful = __builtin_amdgcn_readfirstlane(again);
    if (__builtin_expect(!careful, 1)) break;
    if constexpr (!MX) {
      pb = blk0;
      load_pids();
      load_f16(blk0, 0);
    }
  }

  if constexpr (!MX) {
    if (odd) {
#pragma unroll 1
      for (int k = (careful ? blk0 : max(blk0, tr.len / kKB)) * kKB; k < min(blk1 * kKB, total); ++k) {
        const uint16_t* v = p.vc + kv_offset(p.kv, tr.user, g, k, HD) + 4 * half_sel;
        const int a = k - tr.len;
        if (a >= 0 && !(see[node][a >> 6] >> (a & 63) & 1)) continue;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint16_t x = v[32 * d + 8 * (e >> 2) + (e & 3)];
            if ((x & 0x7c00u) == 0x7c00u) o[d][e] += (float)__builtin_bit_cast(_Float16, x);
          }
      }
    }
  }
  if (col >= cols) return;
  if (tr.splits > 1) {
    const int64_t r = ((int64_t)tr.part0 + (int64_t)z * tr.nodes) * p.nq + (head - (int64_t)tr.row0 * p.nq);
    float* dst = p.part_acc + r * HD;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<v4f*>(dst + 32 * d + 8 * q + 4 * half_sel) =
            v4f{o[d][4 * q], o[d][4 * q + 1], o[d][4 * q + 2], o[d][4 * q + 3]};
    if (half_sel == 0) {
      p.part_ml[r * 2] = m_run * sscale;
      p.part_ml[r * 2 + 1] = l_run;
    }
    return;
  }
  const bool pad = p.parents[tr.row0 + node] == kNoToken;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v4f x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = pad ? 0.f : o[d][4 * q + e] / l_run;
      store_out4(p.out, p.io, head * HD + 32 * d + 8 * q + 4 * half_sel, x);
    }
}

// Merge of a row's splits: out = sum 2^(m_z - M) acc_z / sum 2^(m_z - M) l_z.  Workgroup (row, head): hd/4 threads times
// as many groups as fit take every so many splits.
template <int HD>
__global__ __launch_bounds__(256) void tree_merge_kernel(const TreeParams p) {
  constexpr int PER = HD / 4, GROUPS = 256 / PER, U = 4;
  const int64_t row = blockIdx.y;
  const int h = blockIdx.x, tid = threadIdx.x, d = tid % PER * 4, grp = tid / PER;
  int b = 0;
  while (b < p.trees - 1 && row >= p.tree[b + 1].row0) ++b;
  const TreeOf tr = p.tree[b];
  if (tr.splits == 1) return;  // written already
  __shared__ v4f acc[GROUPS][PER];
  __shared__ float red[GROUPS], lsum[GROUPS];
  const int64_t r0 = ((int64_t)tr.part0 + (row - tr.row0)) * p.nq + h, step = (int64_t)tr.nodes * p.nq;
  float M = -INFINITY;
  for (int z = tid; z < tr.splits; z += 256) M = fmaxf(M, p.part_ml[(r0 + z * step) * 2]);
  // over the lanes, then the waves
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  if ((tid & 63) == 0) red[tid >> 6] = M;
  __syncthreads();
  M = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  v4f x = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int z0 = grp; z0 < tr.splits; z0 += GROUPS * U) {
    v4f a[U];
    float m[U], s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = r0 + min(z0 + u * GROUPS, tr.splits - 1) * step;
      a[u] = *reinterpret_cast<const v4f*>(p.part_acc + r * HD + d);
      m[u] = p.part_ml[r * 2];
      s[u] = p.part_ml[r * 2 + 1];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (z0 + u * GROUPS >= tr.splits) break;
      // M is -inf where every score was NaN: those sums stay NaN
      const float f = M == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[u] - M);
      x += f * a[u];
      l += f * s[u];
    }
  }
  acc[grp][tid % PER] = x;
  if (tid % PER == 0) lsum[grp] = l;
  __syncthreads();
  if (tid >= PER) return;
  l = 0.f;
  x = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    x += acc[i][tid];
    l += lsum[i];
  }
  const bool pad = p.parents[row] == kNoToken;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = pad ? 0.f : x[i] / l;
  store_out4(p.out, p.io, (row * p.nq + h) * HD + d, x);
}

// ------------------------------------------------------------------ launchers
// Blocks per workgroup: about two workgroups a CU over all trees' tiles and blocks, as far as the partials (part_rows
// rows of nq heads) go.
void plan_trees(TreeParams& p, int n_cu, int64_t part_rows) {
  const int G = p.nq / p.nkv;
  int64_t work = 0, most = 1;
  for (int b = 0; b < p.trees; ++b) {
    TreeOf& t = p.tree[b];
    t.tiles = (t.nodes * G + 127) / 128;
    const int64_t n = ((int64_t)t.len + t.nodes + kKvPage - 1) / kKvPage;
    work += n * t.tiles * p.nkv;
    most = std::max(most, n);
  }
  const int64_t wgs = 2ll * n_cu;
  for (int64_t blocks = std::max<int64_t>(1, (work + wgs - 1) / wgs);; blocks = std::min(most, blocks + (blocks + 3) / 4)) {
    int64_t rows = 0;
    for (int b = 0; b < p.trees; ++b) {
      TreeOf& t = p.tree[b];
      t.blocks = (int)blocks;
      t.splits = std::max(1, (int)((((int64_t)t.len + t.nodes + kKvPage - 1) / kKvPage + blocks - 1) / blocks));
      t.wgs = t.tiles * t.splits * p.nkv;
      t.part0 = (int)rows;
      if (t.splits > 1) rows += (int64_t)t.splits * t.nodes;
    }
    if (rows <= part_rows || blocks >= most) return;
  }
}

template <int HD>
static hipError_t attn_tree(const TreeParams& p, hipStream_t s) {
  unsigned wgs = 0;
  bool split = false;
  for (int b = 0; b < p.trees; ++b) {
    wgs += p.tree[b].wgs;
    split |= p.tree[b].splits > 1;
  }
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(wgs), dim3(256), 0, s, p); };
  if (p.io == 1) p.rec ? launch(attn_tree_kernel<HD, true, 1>) : launch(attn_tree_kernel<HD, false, 1>);
  else p.rec ? launch(attn_tree_kernel<HD, true, 2>) : launch(attn_tree_kernel<HD, false, 2>);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && split) {
    hipLaunchKernelGGL(tree_merge_kernel<HD>, dim3(p.nq, p.rows), dim3(256), 0, s, p);
    e = hipGetLastError();
  }
  return e;
}
hipError_t launch_attn_tree(const TreeParams& p, int hd, hipStream_t s) {
  if (p.trees < 1 || p.nq % p.nkv || p.nq / p.nkv > kMaxGroup) return hipErrorInvalidValue;
  for (int b = 0; b < p.trees; ++b)
    if (p.tree[b].nodes < 1 || p.tree[b].nodes > kMaxNodes) return hipErrorInvalidValue;
  return hd == 128 ? attn_tree<128>(p, s) : hd == 64 ? attn_tree<64>(p, s) : hipErrorInvalidValue;
}

}  // namespace kf
