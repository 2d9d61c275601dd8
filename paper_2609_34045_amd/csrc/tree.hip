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
// PARTS: a column as one fp16 column (bf16 queries, which fp16 holds exactly, and one
// part of the probabilities: off by 2^-11 of each, an eighth of half a step of the bf16
// result), or as two, lanes 16 apart, the second with what rounding left in the first
// (fp32 and fp16 queries: 22 bits of queries and probabilities).
#include <algorithm>
#include <cmath>

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
// Over lanes l and l ^ 32, and l and l ^ 16.
__device__ __forceinline__ float max32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// 8 consecutive values of a query row of type 0 fp32, 1 bf16, 2 fp16.
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
constexpr int kCols = 128;         // columns of a workgroup's tile, in parts
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

__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0 | (0x7 << 4) | (0xF << 8)); }
__device__ __forceinline__ void barrier() {
  asm volatile("" ::: "memory");
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
  constexpr int KB = kKB, NT = KB / 32;      // 32-key tiles per block
  constexpr int NS = HD / 16, DB = HD / 32;  // 16-wide d slices of S, 32-row d blocks of O^T
  constexpr int CPR = HD / 8;                // 16-byte chunks per key row
  constexpr int ROWB = HD * 2;               // bytes per key row
  constexpr int VTB = KB * 2;                // bytes per row (one d) of a transposed V block
  constexpr int TILEB = KB * ROWB;           // one block of K or V
  constexpr int RPI = 64 / CPR;              // key rows per 1 KB direct load
  constexpr int LPW = TILEB / 1024 / 4;      // direct loads per wave per tile
  constexpr int WC = 32 / PARTS;             // columns per wave
  // Stage P: K at 2 P TILEB, V behind it.
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * TILEB];
  __shared__ uint64_t see[kMaxNodes][kMaxNodes / 64];
  __shared__ int up[kMaxNodes];

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
  const int blk0 = z * tr.blocks, blk1 = min(blk0 + tr.blocks, (total + KB - 1) / KB);
  const int c0 = tile * (kCols / PARTS) + wave * WC;  // the wave's first column
  const bool live = c0 < cols;                        // a wave without columns only loads
  const int col = c0 + (lane & (WC - 1)), half_sel = lane >> 5;
  const bool ok = col < cols;
  const int node = min(col, cols - 1) / G, h = g * G + min(col, cols - 1) % G;
  const float keep = PARTS == 2 && (lane & 16) ? 1.0f : 0.0f;  // this lane's column holds second parts
  const int64_t row = tr.row0 + node;

  if (blk1 * KB > tr.len) see_ancestors(p.parents + tr.row0, tr.nodes, see, up, tid);

  // Page ids of blocks [pb, pb + 64), lane i holding block pb + i's.
  int pb = blk0, pid = 0;
  auto load_pids = [&]() {
    pid = (p.kv.table && pb + lane < p.kv.ppu) ? p.kv.table[tr.user * p.kv.ppu + pb + lane] : 0;
  };
  load_pids();
  auto block_page = [&](int blk) -> int64_t {
    return p.kv.table ? __builtin_amdgcn_readlane(pid, blk - pb) : tr.user * p.kv.ppu + blk;
  };

  // Q^T fragments: this lane's column, d = 16 s + 8 half_sel .. +7, times a power of two that puts the head's largest
  // value near 2^13 (query_exponent): `sscale` takes a score back, to log2 units.
  v4u qf[NS];
  float sscale;
  {
    float top = 0.f;
    float f[NS][8];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      load_q8(p.q, p.io, (row * p.nq + h) * HD + 16 * s + 8 * half_sel, f[s]);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, __builtin_fabsf(f[s][j]));
    }
    const int e = query_exponent(max32(top));
    const float scale = query_scale(e);
    sscale = p.scale_log2 * query_unscale(e);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[s][j] *= scale;
      qf[s] = v4u{f16_part2(f[s][0], f[s][1], keep), f16_part2(f[s][2], f[s][3], keep), f16_part2(f[s][4], f[s][5], keep),
                  f16_part2(f[s][6], f[s][7], keep)};
    }
  }

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[d][v] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  // ---- a block's keys and values into a stage
  // fp16: load j of this wave fills rows RPI (4 j + wave) ..; lane l writes row RPI (4 j + wave) + l / CPR, slot l % CPR.
  // Rows past the last key are loaded from it, and masked.
  auto load_f16 = [&](int blk, uint8_t* stage) {
    const int last = total - 1 - blk * KB;
    const int64_t off = block_page(blk) * p.kv.page_stride + (int64_t)g * KB * HD;
    const char* kb = reinterpret_cast<const char*>(p.kc + off);
    const char* vb = reinterpret_cast<const char*>(p.vc + off);
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
      const int r = RPI * (4 * j + wave) + lane / CPR;
      const uint32_t at = min(r, last) * ROWB + kv_slot<HD>(r, lane % CPR) * 16;
      const char* ks = kb + at;
      const char* vs = vb + at;
      uint8_t* kd = stage + 1024 * (4 * j + wave);
      uint8_t* vd = stage + TILEB + 1024 * (4 * j + wave);
      __builtin_amdgcn_global_load_lds(ks, (lds_ptr)kd, 16, 0, 0);
      __builtin_amdgcn_global_load_lds(vs, (lds_ptr)vd, 16, 0, 0);
    }
  };
  // MXFP4: jobs 0 .. hd/32 - 1 are 1 KB of K codes each, the others of V; wave w takes w and w + 4.
  constexpr int JOBS = HD / 16 / 4, REC = mx_record(HD), CODES = mx_codes(HD), NB = HD / kMxBlock;
  const int r16 = lane & 15, grp = lane >> 4;
  v4u code[JOBS], vsc[2];
  uint32_t ke = 0;
  auto load_mx = [&](int blk) {
    const uint8_t* rec = p.rec + block_page(blk) * p.kv.page_stride + (int64_t)g * REC;
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
          const int tile16 = HD == 128 ? j : 2 * j + w / 2, key = 16 * tile16 + r16;
          const int chunk = HD == 128 ? grp * 4 + w : grp * 2 + (w & 1);
          const float sc = __uint_as_float(((ke >> (8 * tile16)) & 255u) << 23);
          const v4u x = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], sc, 0)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], sc, 1)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], sc, 2)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code[i][w], sc, 3))};
          *reinterpret_cast<v4u*>(stage + key * ROWB + kv_slot<HD>(key, chunk) * 16) = x;
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
          // A 16-key tile's four groups lie 0 2 1 3, so that one read takes the two of a half of the lanes.
          uint8_t* at = stage + TILEB + d * VTB;
          const int t0 = 2 * (w & 1);
          *reinterpret_cast<v2u*>(at + vt_slot(d, 2 * t0 + (grp & 1)) * 16 + (grp >> 1) * 8) =
              v2u{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c)};
          *reinterpret_cast<v2u*>(at + vt_slot(d, 2 * t0 + 2 + (grp & 1)) * 16 + (grp >> 1) * 8) =
              v2u{__builtin_bit_cast(uint32_t, e), __builtin_bit_cast(uint32_t, f)};
        }
      }
    }
  };

  // ---- the products
  // MFMA of d block d and key step (t, sidx): this half's keys 32 t + 16 sidx + 4 half_sel + {0..3} and + 8 + {0..3}.
  auto vread = [&](const uint8_t* vs, int d, int t, int sidx) {
    if constexpr (MX) {
      const int dd = 32 * d + (lane & 31);
      return *reinterpret_cast<const v4u*>(vs + dd * VTB + vt_slot(dd, 2 * (2 * t + sidx) + half_sel) * 16);
    } else {
      // ds_read_b64_tr_b16: within a group of 16 lanes, lane 4 r + j reads 4 consecutive d of key row r, and lane c
      // receives element c of the group's four rows.
      const int gq = lane >> 4, key = 4 * (gq >> 1) + ((lane >> 2) & 3), dd = 32 * d + 16 * (gq & 1) + 4 * (lane & 3);
      const uint8_t* base = vs + (32 * t + 16 * sidx) * ROWB;
      const uint8_t* a0 = base + key * ROWB + kv_slot<HD>(key, dd >> 3) * 16 + (dd & 7) * 2;
      const uint8_t* a1 = base + (key + 8) * ROWB + kv_slot<HD>(key + 8, dd >> 3) * 16 + (dd & 7) * 2;
      const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)a0);
      const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)a1);
      const v2u l2 = __builtin_bit_cast(v2u, lo), h2v = __builtin_bit_cast(v2u, hi);
      return v4u{l2.x, l2.y, h2v.x, h2v.y};
    }
  };
  auto pv = [&](const uint8_t* vs, const v4u (&pf)[NT][2]) {
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int sidx = 0; sidx < 2; ++sidx) o[d] = mfma32(vread(vs, d, t, sidx), pf[t][sidx], o[d]);
  };

  if (blk0 < blk1) {
    if constexpr (MX) {
      load_mx(blk0);
      store_mx(smem);
    } else {
      load_f16(blk0, smem);
    }
  }
  for (int blk = blk0; blk < blk1; ++blk) {
    uint8_t* stage = smem + ((blk - blk0) & 1) * 2 * TILEB;
    uint8_t* next = smem + (1 - ((blk - blk0) & 1)) * 2 * TILEB;
    if constexpr (!MX) wait_loads();
    __syncthreads();
    const bool more = blk + 1 < blk1;
    if (p.kv.table && blk + 1 >= pb + 64) {
      pb = blk + 1;
      load_pids();
    }
    if (more) {
      if constexpr (MX) load_mx(blk + 1);
      else load_f16(blk + 1, next);
    }
    const bool tail = blk * KB + KB > tr.len;  // positions of the tree, or past it

    f32x16 st[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) st[t][v] = 0.f;
    v4u pf[NT][2];
    if (live) {
      const int rl = lane & 31;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int s = 0; s < NS; ++s)
          st[t] = mfma32(*reinterpret_cast<const v4u*>(stage + (32 * t + rl) * ROWB + kv_slot<HD>(rl, 2 * s + half_sel) * 16),
                         qf[s], st[t]);
      if constexpr (PARTS == 2) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v) st[t][v] = sum16(st[t][v]);
      }
      if (tail) {
        // Which of the block's 64 positions the column's token sees: those before len, and of the tree its own bits.
        const int a0 = blk * KB - tr.len;
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
      }
      float mb = -INFINITY;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) mb = fmaxf(mb, st[t][v]);
      mb = max32(mb);
      // The maximum is kept as the products give it: the scores' distance from it is then exact near it, however large
      // they are.  Until a position is seen it is -inf, and 0 stands in, so that nothing is added.
      const float m_new = (mb - m_run) * sscale > kPartLazy ? mb : m_run;
      const float m_ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f((m_run - m_ref) * sscale);
      float ls = 0.f;
      const h2 ones = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int sidx = 0; sidx < 2; ++sidx) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int v = 8 * sidx + 2 * e;
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(st[t][v] - m_ref, sscale, kPartShift));
            const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(st[t][v + 1] - m_ref, sscale, kPartShift));
            if constexpr (PARTS == 2) {
              w[e] = f16_part2(x, y, keep);
              ls += x + y;
            } else {  // the sum of what the product takes
              w[e] = f16_pair(x, y);
              ls = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, w[e]), ones, ls, false);
            }
          }
          pf[t][sidx] = v4u{w[0], w[1], w[2], w[3]};
        }
      l_run = l_run * alpha + sum32(ls);
      m_run = m_new;
      if (__ballot(alpha != 1.0f)) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[d][v] *= alpha;
      }
    }
    bool odd = false;  // the same in every thread
    if constexpr (!MX) {
      if (tail) {
        // An infinity or NaN among the values that some tokens do not see would reach them as 0 times it.  It is taken out
        // of the product, and added where its probability is not 0, by products with where each sign (a NaN: both) lies.
        constexpr int CPT = TILEB / 16 / 256;
        v4u* vt = reinterpret_cast<v4u*>(stage + TILEB);
        v4u was[CPT];
        bool some = false;
        auto special = [](uint32_t hw) { return (hw & 0x7c00u) == 0x7c00u; };
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
          was[i] = vt[tid + 256 * i];
#pragma unroll
          for (int e = 0; e < 4; ++e) some |= special(was[i][e]) | special(was[i][e] >> 16);
        }
        odd = __syncthreads_or(some);
        if (odd) {
          // what: 0 finite values, 1 where an infinity or NaN adds +inf, 2 where -inf
          auto put = [&](v4u* dst, int what) {
#pragma unroll
            for (int i = 0; i < CPT; ++i) {
              v4u x;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                uint32_t r = 0;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const uint32_t hw = was[i][e] >> (16 * k) & 0xffffu;
                  const bool nan = (hw & 0x7fffu) > 0x7c00u;
                  const uint32_t y = what == 0 ? (special(hw) ? 0u : hw)
                                               : (special(hw) && (nan || (hw >> 15) == (uint32_t)(what - 1)) ? 0x3c00u : 0u);
                  r |= y << (16 * k);
                }
                x[e] = r;
              }
              dst[tid + 256 * i] = x;
            }
          };
          put(vt, 0);
          __syncthreads();
          if (live) pv(stage + TILEB, pf);
          __syncthreads();
          put(vt, 1);
          put(reinterpret_cast<v4u*>(stage), 2);  // K's place: its scores are taken
          __syncthreads();
          if (live) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
              for (int sign = 0; sign < 2; ++sign) {
                f32x16 x;
#pragma unroll
                for (int v = 0; v < 16; ++v) x[v] = 0.f;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                  for (int sidx = 0; sidx < 2; ++sidx)
                    x = mfma32(vread(sign ? stage : stage + TILEB, d, t, sidx), pf[t][sidx], x);
#pragma unroll
                for (int v = 0; v < 16; ++v)
                  if (x[v] != 0.f) o[d][v] += sign ? -INFINITY : INFINITY;
              }
          }
        }
      }
    }
    if (live && !odd) pv(stage + TILEB, pf);
    if constexpr (MX) {
      if (more) store_mx(next);
    }
  }
  if constexpr (PARTS == 2) {
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[d][v] = sum16(o[d][v]);
  }
  if (!ok || (PARTS == 2 && keep != 0.f)) return;
  if (tr.splits > 1) {
    const int64_t r = ((int64_t)tr.part0 + (int64_t)z * tr.nodes + node) * p.nq + h;
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
  const bool pad = p.parents[row] == kNoToken;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v4f x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = pad ? 0.f : o[d][4 * q + e] / l_run;
      store_out4(p.out, p.io, (row * p.nq + h) * HD + 32 * d + 8 * q + 4 * half_sel, x);
    }
}

// Merge of a row's splits, a thread per 4 values of a head: out = sum 2^(m_z - M) acc_z / sum 2^(m_z - M) l_z.
template <int HD>
__global__ __launch_bounds__(256) void tree_merge_kernel(const TreeParams p) {
  const int64_t e = blockIdx.x * 256ll + threadIdx.x;
  const int64_t row = e / (p.nq * (HD / 4));
  if (row >= p.rows) return;
  const int at = (int)(e % (p.nq * (HD / 4))), h = at / (HD / 4), d = at % (HD / 4) * 4;
  int b = 0;
  while (b < p.trees - 1 && row >= p.tree[b + 1].row0) ++b;
  const TreeOf tr = p.tree[b];
  if (tr.splits == 1) return;  // written already
  const int64_t r0 = ((int64_t)tr.part0 + (row - tr.row0)) * p.nq + h, step = (int64_t)tr.nodes * p.nq;
  float M = -INFINITY;
  for (int z = 0; z < tr.splits; ++z) M = fmaxf(M, p.part_ml[(r0 + z * step) * 2]);
  v4f x = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
#pragma unroll 4
  for (int z = 0; z < tr.splits; ++z) {
    const int64_t r = r0 + z * step;
    // M is -inf where every score was NaN: those sums stay NaN
    const float f = M == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(p.part_ml[r * 2] - M);
    x += f * *reinterpret_cast<const v4f*>(p.part_acc + r * HD + d);
    l += f * p.part_ml[r * 2 + 1];
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
  const int G = p.nq / p.nkv, per = kCols / (p.io == 1 ? 1 : 2);
  int64_t work = 0, most = 1;
  for (int b = 0; b < p.trees; ++b) {
    TreeOf& t = p.tree[b];
    t.tiles = (t.nodes * G + per - 1) / per;
    const int64_t n = ((int64_t)t.len + t.nodes + kKB - 1) / kKB;
    work += n * t.tiles * p.nkv;
    most = std::max(most, n);
  }
  const int64_t wgs = 2ll * n_cu;
  for (int64_t blocks = std::max<int64_t>(1, (work + wgs - 1) / wgs);; blocks = std::min(most, blocks + (blocks + 3) / 4)) {
    int64_t rows = 0;
    for (int b = 0; b < p.trees; ++b) {
      TreeOf& t = p.tree[b];
      t.blocks = (int)blocks;
      t.splits = std::max(1, (int)((((int64_t)t.len + t.nodes + kKB - 1) / kKB + blocks - 1) / blocks));
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
  if (p.rec) {
    if (p.io == 1) hipLaunchKernelGGL((attn_tree_kernel<HD, true, 1>), dim3(wgs), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((attn_tree_kernel<HD, true, 2>), dim3(wgs), dim3(256), 0, s, p);
  } else {
    if (p.io == 1) hipLaunchKernelGGL((attn_tree_kernel<HD, false, 1>), dim3(wgs), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((attn_tree_kernel<HD, false, 2>), dim3(wgs), dim3(256), 0, s, p);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && split) {
    const int64_t n = (int64_t)p.rows * p.nq * (HD / 4);
    hipLaunchKernelGGL(tree_merge_kernel<HD>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, p);
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
