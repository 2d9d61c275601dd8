// Internal interface between the stage runtime (stage.hip) and the gfx950 kernels.
// Nothing here is exported from the shared library.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kf {

constexpr int kMaxBatch = 4;
constexpr int kMaxGroup = 8;     // query heads per KV head
constexpr int kAttnMinSplit = 16;   // keys per split-KV workgroup, lower bound
constexpr int kAttnMaxSplit = 1024; // keys per split-KV workgroup, upper bound
// Output rows per workgroup of the head-split output projection (128 and 64 measured
// slower: every workgroup repeats its head's merge of the split partials).
constexpr int kOprojRows = 256;
constexpr int kAttnMaxSplitCount = 1024;  // split-KV workgroups per (row, KV head), upper bound
constexpr int kHeadRowsKept = 12;  // rows of the LM head per workgroup, for fp16 input rows of batch 2-4
// Decode attention on the matrix cores: workgroups of kAttnMfmaWaves waves over
// splits of any multiple of kAttnMfmaAlign keys (16-key blocks, one page or
// less each).
#ifndef KF_ATTN_WAVES
#define KF_ATTN_WAVES 4
#endif
constexpr int kAttnMfmaWaves = KF_ATTN_WAVES;
constexpr int kAttnMfmaAlign = 16;

// Bits of the stage's sticky device error flag (reported and cleared by kf_stage_sync).
enum : int {
  kErrToken = 1,      // a token id outside [0, vocab): its hidden row became NaN
  kErrF16Range = 2,   // an activation, key or value stored in fp16 was at or beyond 65520 in magnitude
  kErrNaNLogit = 4,   // a logit was NaN (the argmax skips it; a row of NaN gives token -1)
};

// fp32 to fp16 bits (round to nearest even), noting in `bad` a value that fp16
// cannot hold (|v| >= 65520 rounds to infinity; an infinite input counts too).
__device__ __forceinline__ uint16_t f16_checked(float v, bool& bad) {
  bad |= __builtin_fabsf(v) >= 65520.0f;
  return __builtin_bit_cast(uint16_t, (_Float16)v);
}
__device__ __forceinline__ void raise_err(int* flag, bool bad, int bit) {
  if (bad && flag) atomicOr(flag, bit);
}

// KV cache pages.  One layer's K (and, alike, V) is an array of pages of kKvPage
// positions, each page [kv_head][kKvPage][hd] fp16.  Position t of user u lies
// at slot t % kKvPage of the page with id table[u * ppu + t / kKvPage] (a paged
// cache, whose pages come from a shared pool), or u * ppu + t / kKvPage (a
// cache without a table: each user's ppu pages reserved in order).
constexpr int kKvPage = 64;
struct KvPages {
  const int* table;     // [max_users][ppu] page ids, or NULL
  int ppu;              // pages per user
  int64_t page_stride;  // elements per page: nkv * kKvPage * hd
};
__device__ __forceinline__ int kv_page(const KvPages& kp, int user, int i) {
  return kp.table ? kp.table[user * kp.ppu + i] : user * kp.ppu + i;
}
// Element offset of (user, kv head g, position t) in a layer's K or V.
__device__ __forceinline__ int64_t kv_offset(const KvPages& kp, int user, int g, int t, int hd) {
  return (int64_t)kv_page(kp, user, t / kKvPage) * kp.page_stride + ((int64_t)g * kKvPage + t % kKvPage) * hd;
}

// MXFP4 caches (KF_KV_MXFP4).  A page holds one record per KV head, K codes, K
// exponents, V codes, V exponents; KvPages::page_stride counts bytes there.  A
// block of kMxBlock values along the head has one exponent e in [kMxExpMin,
// kMxExpMax] and E2M1 codes: value = 2^e times 0, 0.5, 1, 1.5, 2, 3, 4 or 6 with a
// sign.  With that range every stored value is an fp16 number.  K's exponents are bytes
// e + 127, of which the convert instruction's fp32 scale is made by a shift.  V's are
// 2^e in fp16: a register of V operands holds two positions, so the products with their
// two scales are one packed instruction where the pair lies ready, at 1/32 more bytes
// (of bytes each lane would have to expand two a pair).
// Codes and exponents lie in the order in which the attention's lanes take them
// (mx_* below), so that each of its loads is 16 contiguous bytes a lane.
constexpr int kMxBlock = 32;
constexpr int kMxExpMin = -23, kMxExpMax = 13;
__host__ __device__ constexpr int mx_codes(int hd) { return kKvPage * hd / 2; }           // bytes, K or V
__host__ __device__ constexpr int mx_exps(int hd) { return kKvPage * hd / kMxBlock; }     // exponents, K or V
__host__ __device__ constexpr int mx_v(int hd) { return mx_codes(hd) + mx_exps(hd); }     // byte where V begins
__host__ __device__ constexpr int mx_record(int hd) { return mx_v(hd) + mx_codes(hd) + 2 * mx_exps(hd); }
// Position t of the page as a matrix-core operand sees it: tile t / 16, and within
// it row t % 16 of K; for V, 16-lane group (t / 4) % 4 and element t % 4.
// Byte of the K code of (t, d); its nibble is d % 2.  A lane (row, group) takes hd / 4 consecutive d.
template <int HD>
__host__ __device__ constexpr int mx_k_byte(int t, int d) {
  const int tile = t / 16, row = t % 16, grp = d / (HD / 4), x = d % (HD / 4);
  return HD == 128 ? (tile * 64 + grp * 16 + row) * 16 + x / 2
                   : ((tile / 2) * 64 + grp * 16 + row) * 16 + (tile % 2) * 8 + x / 2;
}
// Byte of the exponent of K block blk at t.
__host__ __device__ constexpr int mx_k_exp(int t, int blk) { return (blk * 16 + t % 16) * 4 + t / 16; }
// Byte of the V code of (t, d); its nibble is t % 2.  A lane (d % 16, group) takes its 16 positions of two 16-wide d tiles.
__host__ __device__ constexpr int mx_v_byte(int t, int d) {
  const int dt = d / 16;
  return ((dt / 2) * 64 + ((t / 4) % 4) * 16 + d % 16) * 16 + (dt % 2) * 8 + (t / 16) * 2 + (t % 4) / 2;
}
// Index of the scale (fp16) of V block blk at t.
template <int HD>
__host__ __device__ constexpr int mx_v_exp(int t, int blk) {
  return (((t / 4) % 4) * (HD / kMxBlock) + blk) * 16 + (t / 16) * 4 + t % 4;
}
__device__ __forceinline__ uint16_t mx_v_scale(int e) {  // 2^e
  return (uint16_t)(e >= -14 ? (e + 15) << 10 : 1 << (e + 24));
}

// Two fp32 values as packed fp16 bits (nearest even; what fp16 cannot hold becomes infinite).
__device__ __forceinline__ uint32_t f16_pair(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, h2));
}
// One fp16 part of each of a pair of finite values, which two parts hold to 22 bits: the rounded values for keep 0, what
// rounding left for keep 1.
__device__ __forceinline__ uint32_t f16_part2(float a, float b, float keep) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  const h2 hi = __builtin_convertvector(f2{a, b}, h2);
  return f16_pair(__builtin_fmaf(-keep, (float)hi.x, a), __builtin_fmaf(-keep, (float)hi.y, b));
}
// Attention with given queries (kf_kv_attend, and decode steps on MXFP4 caches) takes probabilities relative to a maximum
// that moves only when a tile's exceeds it by kPartLazy (log2 units), so that O is rarely rescaled, and times 2^kPartShift:
// the largest lies in [2^12, 2^14], within fp16, and two fp16 parts, whose finest step is 2^-24, hold every one above
// 2^-14 to 22 bits (one of a long flat tail beside a peak too: without the shift those below 2^-14 of the peak would keep
// 10).  The shift is added after the subtraction, which is exact near the maximum however large the scores are.
constexpr float kPartShift = 12.0f, kPartLazy = 2.0f;
// Queries go into two fp16 parts times a power of two, 2^(13 - e) with e the exponent of the head's largest value (in
// [-90, 127]), so that they neither overflow, up to the largest fp32 number, nor lose bits below the normal range.
__device__ __forceinline__ int query_exponent(float top) {
  const int e = (int)(__float_as_uint(top) >> 23) - 127;
  return e < -90 ? -90 : e > 127 ? 127 : e;
}
__device__ __forceinline__ float query_scale(int e) { return __uint_as_float((uint32_t)(127 + 13 - e) << 23); }
__device__ __forceinline__ float query_unscale(int e) { return __uint_as_float((uint32_t)(127 - 13 + e) << 23); }
// 8 of a block's values as fp16 pairs, the other 24 in the 3 lanes beside (lanes 4 k .. 4 k + 3
// hold a block): their E2M1 codes, and the block's exponent.  A NaN is stored as 0, an infinity as the
// largest magnitude; both are noted in `bad`.  The convert instruction rounds to nearest even
// and saturates at 6.
__device__ __forceinline__ uint32_t mx_encode8(uint32_t (&x)[4], int& e, bool& bad) {
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  typedef uint16_t u2 __attribute__((ext_vector_type(2)));
  auto most = [&]() {  // of the magnitudes' bits, whose order is the values'
    u2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u2, x[i] & 0x7fff7fffu));
    return (uint32_t)(m.x > m.y ? m.x : m.y);
  };
  uint32_t top = most();
  if (top >= 0x7c00u) {
    bad = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t h = (x[i / 2] >> (16 * (i % 2))) & 0xffffu, a = h & 0x7fffu;
      const uint32_t v = a > 0x7c00u ? 0u : a == 0x7c00u ? h - 1u : h;  // infinity - 1 is 65504
      x[i / 2] = i % 2 ? (x[i / 2] & 0xffffu) | v << 16 : (x[i / 2] & 0xffff0000u) | v;
    }
    top = most();
  }
  // over the four lanes, by two quad permutes
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, false));
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, false));
  // adding half a unit of the one kept mantissa bit carries into the exponent where the rounding does
  const float t = (float)__builtin_bit_cast(_Float16, (uint16_t)top);
  e = (int)((__builtin_bit_cast(uint32_t, t) + 0x200000u) >> 23) - 127 - 2;
  e = e < kMxExpMin ? kMxExpMin : e > kMxExpMax ? kMxExpMax : e;
  const float scale = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(0u, __builtin_bit_cast(h2, x[0]), scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(h2, x[1]), scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(h2, x[2]), scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(h2, x[3]), scale, 3);
}

// Optional per-launch marker around each kernel (instrumentation hook of the runtime).
struct Tracer {
  void* ctx = nullptr;
  void (*fn)(void* ctx, int cls, int begin) = nullptr;
  void begin(int cls) const {
    if (fn) fn(ctx, cls, 1);
  }
  void end(int cls) const {
    if (fn) fn(ctx, cls, 0);
  }
};

enum GemvEpi : int {
  kEpiQKV = 0,     // RoPE on q and k, q -> fp32 workspace, k and v -> fp16 cache at the row's position
  kEpiResid = 1,   // x[b][row] += y (fp32 residual stream), optional copy to the hidden output
  kEpiSwiGLU = 2,  // a[b][j] = silu(gate_j) * up_j
  kEpiLMHead = 3,  // optional fp32 logits, per-workgroup (max, lowest index) partials
};

// Element type of a residual GEMV's optional copy output.
enum { kOut2F32 = 0, kOut2BF16 = 1, kOut2F16 = 2 };

// One decode GEMV launch: y[b][n] = sum_k W[n][k] * in[b][k] (* gain[k] * rsqrt(mean(in^2)+eps) if norm).
struct GemvParams {
  const uint16_t* w0;  // fp16 matrix rows (QKV: [q;k;v] rows; SwiGLU: gate; others: the matrix)
  const uint16_t* w1;  // SwiGLU: up rows; unused otherwise
  const uint16_t* gain;  // RMSNorm gain [K] when the launch normalises its input
  const float* in;     // [B][K] fp32
  int K;               // reduction length (multiple of 8)
  int N;               // output rows (logical)
  float eps;
  int batch;

  // kEpiResid
  float* x;            // [B][N] residual stream, updated in place
  void* out2;          // optional [B][N] copy of the updated rows, element type out2_type
  int out2_type;       // kOut2F32, kOut2BF16 (a bf16 hidden output) or kOut2F16 (the next GEMV's input)

  // kEpiQKV
  float* q;            // [B][nq*hd]
  uint16_t* kc;        // K cache of this layer (fp16 bits), pages as in KvPages
  uint16_t* vc;
  KvPages kv;
  int nq, nkv, hd;
  const float* rope_cos;  // [max_ctx][hd/2]
  const float* rope_sin;
  int users[kMaxBatch];
  int pos[kMaxBatch];
  // Blocks with per-head q/k norms: when set, q goes to `q` and k to kraw
  // ([B][nkv][hd] fp32) as projected (after the attention RMSNorm), without
  // RoPE; the decode attention finishes both.  v goes to the cache as usual.
  float* kraw;

  // kEpiSwiGLU
  float* act;          // [B][N] with N = F: fp32, or fp16 when act16 is set
  int act16;
  // Input rows `in` stored as fp16 (the down projection's input at batch > 1), else fp32.
  int in16;

  // Launches with the stage input as their input rows (instead of `in`): the
  // first layer's QKV and the LM head.  Exactly one of src / tokens is set.
  const void* src;         // [B][K] hidden input, fp32 or (src_bf16) bf16
  int src_bf16;
  const int32_t* tokens;   // [B] token ids: rows of `embed` [vocab][K] bf16
  const uint16_t* embed;
  int vocab;
  float* x_init;           // optional [B][K]: workgroup 0 stores the input rows here (residual stream)
  int* err_flag;           // sticky error bits (kErrToken, kErrF16Range, kErrNaNLogit); every launch sets it

  // kEpiLMHead
  float* logits;       // optional [B][N]
  float* part_val;     // [B][n_wg]
  int* part_idx;       // [B][n_wg]
  int n_wg;
  const float* eps_rows;  // [B] or NULL: eps of each row, for input rows that were scaled (launch_rows_to_f16)
};

struct AttnParams {
  const float* q;      // [B][nq*hd] rotated queries
  uint16_t* kc;        // layer base (fp16 bits), pages as in KvPages (written only for the new key of qk-norm blocks)
  const uint16_t* vc;
  float* part_acc;     // [B][nq][max_split][hd]
  float* part_ml;      // [B][nq][max_split][2]
  KvPages kv;
  int nq, nkv, hd;
  int split;           // keys per workgroup
  int n_split;         // workgroups per (row, kv head): the most of any row
  int max_split;       // allocated split capacity
  float scale_log2;    // log2(e) / sqrt(hd)
  int users[kMaxBatch];
  int len[kMaxBatch];  // keys visible to row b: position + 1
  // Blocks with per-head q/k norms: q holds the projections as they come from
  // the QKV GEMV (no RoPE).  Every workgroup RMS-normalises (gains gq, eps) and
  // rotates the query heads it scores; the workgroup whose split holds row b's
  // new position does the same for the new key (kraw, gains gk), stores it to the
  // cache and scores it from registers.  kraw NULL: q is already rotated and the
  // new key is in the cache.
  const float* kraw;      // [B][nkv][hd]
  const uint16_t* gq;     // [hd] bf16
  const uint16_t* gk;
  const float* rope_cos;  // [max_ctx][hd/2]
  const float* rope_sin;
  float eps;
  int* err_flag;          // sticky error bits: kErrF16Range for an fp16 store out of range
};

// Attention over an MXFP4 cache (attend.hip): a's queries and cache pointers are not
// used, its KvPages count bytes, its splits are whole pages, and rows have as many as they
// need (1 at least).  With `out` set (one split a row, or the merge) the result goes
// there; else the partials go to a's arrays, as the fp16 kernel's do.
constexpr int kMxMaxSplit = 4096;  // keys per workgroup, upper bound
struct RowSplits {
  int n[kMaxBatch];  // partials of each row
};
struct MxAttnParams {
  AttnParams a;
  RowSplits rows;
  const uint8_t* rec;  // layer base
  const void* q;       // [B][nq][hd] rotated queries
  int q_type;          // and their type, 0 fp32, 1 bf16, 2 fp16 (the kf_dtype values)
  void* out;           // [B][nq][hd] of type io, or NULL
  int io;
};
// The same in a decode step, which appends each row's new key and value at its last position (a.len - 1).
struct MxStepParams : MxAttnParams {  // q: fp32; normalised and rotated here when gq is set
  uint8_t* cache;  // = rec
  // row b's key (rotated) and value, as the QKV launch left them: fp16 page b, at the position's slot
  const uint16_t *k16, *v16;
  const float* kraw;        // [B][nkv][hd]: the raw keys instead, when gk is set
  const uint16_t *gq, *gk;  // per-head norm gains [hd] bf16, or NULL
  const float *rope_cos, *rope_sin;
  float eps;
};

// Launchers (return hipGetLastError() of the launch).
hipError_t launch_attn_mx(const MxAttnParams& p, int batch, hipStream_t s);
// p.out from the partials of either cache type's attention.
hipError_t launch_attend_merge(const MxAttnParams& p, int batch, hipStream_t s);
hipError_t launch_attn_mx_step(const MxStepParams& p, int batch, hipStream_t s);
int gemv_grid(int epi, int rows_per_wg, const GemvParams& p);
hipError_t launch_gemv(int epi, int rows_per_wg, int chunks_in_flight, bool norm, const GemvParams& p, hipStream_t s);
// The same launch with the stage input (p.src or p.tokens) as its input rows.
hipError_t launch_gemv_src(int epi, int rows_per_wg, int chunks_in_flight, bool norm, const GemvParams& p,
                           hipStream_t s);
hipError_t launch_attn_decode(const AttnParams& p, int batch, hipStream_t s);
// The same with given queries, p.q of q_type (a kf_dtype value), and queries and probabilities in two fp16 parts each.
hipError_t launch_attn_given(const AttnParams& p, int batch, int q_type, hipStream_t s);
// Head h of row b merged from the attention partials in p, to o16[b][h*hd:(h+1)*hd]
// (fp16) or, with o16 NULL, to o32[b][h*hd:(h+1)*hd] (fp32).
// rows: how many partials each row has, or NULL for p.n_split.
hipError_t launch_attn_merge(const AttnParams& p, const RowSplits* rows, uint16_t* o16, float* o32, int batch, hipStream_t s);
// x[b][0:N) += W_o o_b with o_b merged from the attention partials in p (W_o [N][nq*hd] fp16).
hipError_t launch_oproj_heads(const AttnParams& p, const uint16_t* w, float* x, int N, int batch, hipStream_t s);
hipError_t launch_argmax_final(const float* part_val, const int* part_idx, int n_wg, int rows, int32_t* token,
                               float* max_logit, hipStream_t s);
// In place over n elements: bf16 weights to fp16 (round to nearest even); *bad |= 1
// if a finite weight is beyond the fp16 range.
hipError_t launch_weights_to_f16(uint16_t* w, int64_t n, int* bad, hipStream_t s);
// Sets *flag when some w[r][k] g[k] (bf16 w [n / K][K], bf16 g [K]) has no finite fp16 rounding.
hipError_t launch_gain_fold_check(const uint16_t* w, int64_t n, int K, const uint16_t* g, int* flag, hipStream_t s);
// In place: bf16 w[r][k] -> fp16 w[r][k] g[k] (the gain folded into the columns); *bad on an fp16 overflow.
hipError_t launch_weights_to_f16_gain(uint16_t* w, int64_t n, int K, const uint16_t* g, int* bad, hipStream_t s);
// Positions [pos0, pos0 + n) of one user in one layer (k, v: the layer's base)
// from / to [n][nkv][hd] rows.  src_type: 0 fp32, 1 bf16, 2 fp16 (the kf_dtype values).
hipError_t launch_kv_write(uint16_t* k, uint16_t* v, const KvPages& kp, int user, int pos0, const void* src_k,
                           const void* src_v, int src_type, int n, int nkv, int hd, hipStream_t s);
hipError_t launch_kv_read(const uint16_t* k, const uint16_t* v, const KvPages& kp, int user, int pos0, float* dst_k,
                          float* dst_v, int n, int nkv, int hd, hipStream_t s);
// The page table of a paged cache as its updates see it: each entry has the number of the update that it holds, so that
// one that a captured graph replays after later ones changes nothing.
struct KvTable {
  int* page;
  uint32_t* version;
};
// page[idx[i]] = val[i] for i < n (n <= kKvTableBatch) where version[idx[i]] is before ver[i], which it becomes; a val of
// -1 brings the version alone.
constexpr int kKvTableBatch = 32;
struct KvTableUpdate {
  int n;
  int idx[kKvTableBatch];
  int val[kKvTableBatch];
  uint32_t ver[kKvTableBatch];
};
__device__ __forceinline__ void kv_table_apply(const KvTable& t, const KvTableUpdate& u, int i) {
  if (i >= u.n || (int32_t)(u.ver[i] - t.version[u.idx[i]]) <= 0) return;
  if (u.val[i] >= 0) t.page[u.idx[i]] = u.val[i];
  t.version[u.idx[i]] = u.ver[i];
}
hipError_t launch_kv_table_update(const KvTable& t, const KvTableUpdate& u, hipStream_t s);
// page[dst + i] = page[src + i] for i < n, as each entry's next update: a user that shares another's pages.
hipError_t launch_kv_table_share(const KvTable& t, int src, int dst, int n, hipStream_t s);

// Log probabilities of rows of logits (logprob.hip).
constexpr int kMaxTop = 32;
constexpr int kMaxLogprobVocab = 1 << 20;
constexpr int kLogprobRows = 32768;  // rows of one launch
struct LogprobParams {
  const float* logits;  // [rows][stride]
  int64_t stride;
  int vocab;
  const float* row_scale;  // [rows] or NULL: the logits are these times what is stored
  const int32_t* targets;  // [rows] or NULL
  float* logprob;          // [rows], with targets
  float* entropy;          // [rows] or NULL
  int top;
  int32_t* top_ids;        // [rows][top]
  float* top_logprobs;
  int* err_flag;
  int values;  // per thread (logprob_values of all rows of the call, so that its launches give the bits of one)
  // set by the launcher: partial results of rows of several chunks
  int chunks;
  unsigned long long* part_keys;  // [rows][chunks][top]
  float* part_sums;               // [rows][chunks][4]
};
// x16 = x 2^e of bf16 rows [rows][K], with e so that a row's largest value lies in [2^14, 2^15): every value above
// 2^-29 of the row's largest is exact.  What RMSNorm multiplies x16 by is row_scale = 1 / sqrt(mean x16^2 + eps 4^e);
// eps_rows = eps 4^e.  Either may be NULL.
hipError_t launch_rows_to_f16(const uint16_t* x, int rows, int K, float eps, uint16_t* x16, float* eps_rows,
                              float* row_scale, hipStream_t s);
// How a call's rows are cut: values per thread, of 256 threads a chunk, and the chunks of a row.  More than one have a partial
// result each in a workspace.  Smaller chunks are for calls of fewer than 256 large ones, so that kLogprobLeast partials hold
// any such call whole, and a row of any other.  kLogprobMost, 18 MB, are as fast as more: rows past them are other launches.
int logprob_values(int rows, int vocab);
int logprob_chunks(int vocab, int values);
constexpr int kLogprobLeast = 1024, kLogprobMost = 65536;
constexpr int64_t kLogprobPartBytes = 16 + kMaxTop * 8;  // a partial's, for any number of alternatives
hipError_t launch_logprobs(LogprobParams p, int rows, char* part, hipStream_t s);

// A cache as the copying kernels see it (cache.hip): fp16 K and V arrays, or one array of MXFP4 records at k.
struct CacheRef {
  uint8_t* k;
  uint8_t* v;           // fp16 caches only
  KvPages pages;
  int64_t layer_bytes;  // of k (and, alike, v)
  int mx;
  int nkv, hd;
};
// As launch_kv_write / launch_kv_read, for one layer (c.k: its base) of an MXFP4 cache.  A value is rounded to fp16
// first, so that an MXFP4 cache holds the same whether a position was written, appended or copied from an fp16 cache.
hipError_t launch_mx_write(const CacheRef& c, int user, int pos0, const void* src_k, const void* src_v, int src_type,
                           int n, int* err_flag, hipStream_t s);
hipError_t launch_mx_read(const CacheRef& c, int user, int pos0, float* dst_k, float* dst_v, int n, hipStream_t s);
// Positions [pos0, pos0 + n) of src_user to the same ones of dst_user, in every one of `layers` layers.
hipError_t launch_cache_copy(const CacheRef& dst, int dst_user, const CacheRef& src, int src_user, int pos0, int n,
                             int layers, int* err_flag, hipStream_t s);
// Whole pages src[i] to dst[i] for i < n (n <= kPageCopyBatch), in every layer, and the table entries in u.
constexpr int kPageCopyBatch = 32;
struct PageCopies {
  int n;
  int src[kPageCopyBatch];
  int dst[kPageCopyBatch];
};
hipError_t launch_page_copies(const CacheRef& c, const PageCopies& copies, int layers, const KvTable& table,
                              const KvTableUpdate& u, hipStream_t s);

}  // namespace kf
