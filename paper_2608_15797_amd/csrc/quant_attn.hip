// Attention over a context kept in 4 bits and the sequence's own rows, for one
// or several query tokens per sequence.
//
// The tokens of sequence s are the n = ctx_len[s / C] slots of its context and
// then the u = len[s] slots of its own cache; its nq queries belong to the
// last nq of these, so query t sees the first n + u - (nq - 1 - t) of them.
#include <hip/hip_runtime.h>

#include "kvr_device.h"
#include "kvr_internal.h"
#include "quant_common.h"

namespace kvr {

namespace {

constexpr float kNegInf = -__builtin_huge_valf();
constexpr int kThreads = 256;

// Own row j of a unit: the new rows come from the caller's arrays (another
// workgroup may be storing them), the others from the cache.
struct OwnRows {
  const float *cache, *fresh;
  int first;  // first new row; none where fresh is NULL
  __device__ __forceinline__ const float *row(int j, int D) const {
    return fresh && j >= first ? fresh + (size_t)(j - first) * D : cache + (size_t)j * D;
  }
};

__device__ __forceinline__ int own_len(const QuantAttnParams &p, int s) {
  return p.ok ? min(max(p.len[s], 0), p.ocap) : 0;
}
__device__ __forceinline__ int ctx_len(const QuantAttnParams &p, int c) { return min(max(p.ctx_len[c], 0), p.cap); }

// The new rows of a unit into its cache (and their positions), by THREADS threads.
template <typename T, int D, int THREADS>
__device__ __forceinline__ void store_new(const QuantAttnParams &p, int unit, int s, int u) {
  if (p.k_new == nullptr) return;
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  constexpr int W = D * sizeof(T) / 16;  // 16-byte words per row
  const int first = u - p.nq;
  for (int e = threadIdx.x; e < p.nq * W; e += THREADS) {
    const int t = e / W, j = first + t;
    if (j < 0) continue;
    const size_t from = ((size_t)unit * p.nq + t) * W + e % W, to = ((size_t)unit * p.ocap + j) * W + e % W;
    static_cast<u32x4 *>(p.ok)[to] = static_cast<const u32x4 *>(p.k_new)[from];
    static_cast<u32x4 *>(p.ov)[to] = static_cast<const u32x4 *>(p.v_new)[from];
  }
  if (p.pos && p.new_pos)
    for (int t = threadIdx.x; t < p.nq; t += THREADS)
      if (first + t >= 0) p.pos[(size_t)unit * p.ocap + first + t] = p.new_pos[(size_t)s * p.nq + t];
}

// float32: vector kernel, one workgroup per (sequence, layer, KV head), 16 of
// its rows and a share of its keys. 32 keys at a time are expanded to float32
// rows in LDS; a thread has two of the 16 x 32 logits, then one column of the
// output for some of the rows. Shares leave records (max, sum, -, -, o) that
// quant_vector_join joins. Bound by latency in small calls, by the vector
// units' float32 rate in long ones.
constexpr int kVecKeys = 32, kVecRows = 16;

__host__ __device__ __forceinline__ int vector_blocks(const QuantAttnParams &p) {
  return (p.nq * p.G + kVecRows - 1) / kVecRows;
}
template <int D>
constexpr int kVecRec = 4 + D;

template <int D, int NG>
__global__ __launch_bounds__(kThreads) void quant_attn_vector(QuantAttnParams p) {
  using Q = QTile<D, NG>;
  constexpr int CH = D / 8, PITCH = D + 4, KG = kThreads / D, RPT = kVecRows / KG;
  __shared__ __align__(16) float qs[kVecRows][D];
  __shared__ __align__(16) float kt[kVecKeys][PITCH], vt[kVecKeys][PITCH];
  __shared__ float prob[kVecRows][kVecKeys + 1];
  __shared__ float row_m[kVecRows], row_l[kVecRows], row_f[kVecRows];
  __shared__ int row_lim[kVecRows];
  const int blocks = vector_blocks(p), per = p.nq * p.G;
  const int share = blockIdx.x % p.shares, ub = blockIdx.x / p.shares, block = ub % blocks, unit = ub / blocks;
  const int lh = p.L * p.Hkv, s = unit / lh, c = s / p.C;
  const int tid = threadIdx.x, r0 = block * kVecRows, nrow = min(kVecRows, per - r0);
  const int n = ctx_len(p, c), u = own_len(p, s);
  if (share == 0 && block == 0 && p.ok) store_new<float, D, kThreads>(p, unit, s, u);
  const float *q = static_cast<const float *>(p.q) + ((size_t)unit * per + r0) * D;
  for (int e = tid; e < kVecRows * D; e += kThreads) qs[e / D][e % D] = e < nrow * D ? q[e] : 0.f;
  if (tid < kVecRows) {
    row_m[tid] = kNegInf;
    row_l[tid] = 0.f;
    // Keys that the row sees, of context and own together.
    row_lim[tid] = (int)((long)n + u - (p.nq - 1 - (r0 + tid) % p.nq));
  }
  const char *ctx = static_cast<const char *>(p.data) + ((size_t)c * lh + unit % lh) * p.ntiles * Q::BYTES;
  const size_t own0 = (size_t)unit * p.ocap * D, new0 = (size_t)unit * p.nq * D;
  const float *fk = static_cast<const float *>(p.k_new), *fv = static_cast<const float *>(p.v_new);
  const OwnRows K{static_cast<const float *>(p.ok) + own0, fk ? fk + new0 : nullptr, u - p.nq};
  const OwnRows V{static_cast<const float *>(p.ov) + own0, fv ? fv + new0 : nullptr, u - p.nq};
  const int d = tid % D, kg = tid / D, key = tid % kVecKeys, rg = tid / kVecKeys;
  const int sees_all = (int)((long)n + u - (p.nq - 1));  // keys before it are seen by every row
  float o[RPT];
#pragma unroll
  for (int i = 0; i < RPT; i++) o[i] = 0.f;

  // Chunks: the context's tiles, then the own rows in 32s.
  const int held = (n + kVecKeys - 1) / kVecKeys, all = held + (u + kVecKeys - 1) / kVecKeys;
  const int t0 = (int)((long)all * share / p.shares), t1 = (int)((long)all * (share + 1) / p.shares);
  for (int t = t0; t < t1; t++) {
    const bool own = t >= held;
    const int first = own ? n + (t - held) * kVecKeys : t * kVecKeys;  // token of the chunk's first key
    const int live = min(kVecKeys, own ? n + u - first : n - first);
    const char *tile = ctx + (size_t)t * Q::BYTES;
    __syncthreads();
    // A thread's pieces of eight values: all their loads, then the values.
    constexpr int PIECES = 2 * kVecKeys * CH / kThreads;
    float x[PIECES][8];
    if (own) {
      float4_t w[PIECES][2];
#pragma unroll
      for (int i = 0; i < PIECES; i++) {
        const int e = tid + i * kThreads, k = e / CH % kVecKeys;
        const float *row = (e >= kVecKeys * CH ? V : K).row(first - n + min(k, live - 1), D) + e % CH * 8;
#pragma unroll
        for (int h = 0; h < 2; h++) w[i][h] = reinterpret_cast<const float4_t *>(row)[h];
      }
#pragma unroll
      for (int i = 0; i < PIECES; i++)
#pragma unroll
        for (int j = 0; j < 8; j++) x[i][j] = w[i][j >> 2][j & 3];
    } else {
      uint32_t w[PIECES];
      float sc[PIECES], z[PIECES];
#pragma unroll
      for (int i = 0; i < PIECES; i++) {
        const int e = tid + i * kThreads, k = e / CH % kVecKeys, ch = e % CH;
        const bool val = e >= kVecKeys * CH;
        const int grp = ch * 8 / Q::GROUP, at = val ? Q::VS + Q::vparam(k, grp) : Q::KS + Q::kparam(k, grp);
        sc[i] = f16_at(tile + at);
        z[i] = f16_at(tile + at + (Q::KZ - Q::KS));
        if (!val) {
          w[i] = *reinterpret_cast<const uint32_t *>(tile + Q::kword(k, ch));
        } else {
          w[i] = 0;
#pragma unroll
          for (int j = 0; j < 4; j++) w[i] |= (uint32_t)(uint8_t)tile[Q::vbyte(k, ch * 4 + j)] << (8 * j);
        }
      }
#pragma unroll
      for (int i = 0; i < PIECES; i++)
#pragma unroll
        for (int j = 0; j < 8; j++) x[i][j] = fmaf(sc[i], (float)((w[i] >> (4 * j)) & 15u), z[i]);
    }
#pragma unroll
    for (int i = 0; i < PIECES; i++) {
      const int e = tid + i * kThreads, k = e / CH % kVecKeys;
#pragma unroll
      for (int j = 0; j < 8; j++) x[i][j] = k < live ? x[i][j] : 0.f;
      float4_t *to = reinterpret_cast<float4_t *>(&(e >= kVecKeys * CH ? vt : kt)[k][e % CH * 8]);
      to[0] = (float4_t){x[i][0], x[i][1], x[i][2], x[i][3]};
      to[1] = (float4_t){x[i][4], x[i][5], x[i][6], x[i][7]};
    }
    __syncthreads();
    // Logits of key `key` and rows rg, rg + 8; a row's 32 are in one half wave.
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int r = rg + 8 * h;
      if (8 * h >= nrow) break;  // the rows past the last are not stored
      float4_t a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
      for (int i = 0; i < D / 4; i++) {
        const float4_t x = reinterpret_cast<const float4_t *>(kt[key])[i];
        const float4_t y = reinterpret_cast<const float4_t *>(qs[r])[i];
#pragma unroll
        for (int j = 0; j < 4; j++) a[j] = fmaf(x[j], y[j], a[j]);
      }
      const bool seen = key < live && first + key < row_lim[r];
      const float x = seen ? ((a[0] + a[1]) + (a[2] + a[3])) * p.scale * kLog2e : kNegInf;
      float m = x;
#pragma unroll
      for (int k = 16; k >= 1; k >>= 1) m = fmaxf(m, shfl_xor(m, k));
      const float was = row_m[r], mn = fmaxf(was, m), ref = mn == kNegInf ? 0.f : mn;
      const float e = seen ? exp2f(x - ref) : 0.f;
      float sum = e;
#pragma unroll
      for (int k = 16; k >= 1; k >>= 1) sum += shfl_xor(sum, k);
      prob[r][key] = e;
      if (key == 0) {
        const float f = was == kNegInf ? 0.f : exp2f(was - mn);
        row_f[r] = f;
        row_m[r] = mn;
        row_l[r] = row_l[r] * f + sum;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RPT; i++) o[i] *= row_f[kg * RPT + i];
    if (first + kVecKeys <= sees_all) {
#pragma unroll 4
      for (int k = 0; k < kVecKeys; k++) {
        const float v = vt[k][d];
#pragma unroll
        for (int i = 0; i < RPT; i++) o[i] = fmaf(prob[kg * RPT + i][k], v, o[i]);
      }
    } else {
      // A row takes nothing from keys it does not see, whatever they hold.
      for (int k = 0; k < live; k++) {
        const float v = vt[k][d];
#pragma unroll
        for (int i = 0; i < RPT; i++)
          o[i] = first + k < row_lim[kg * RPT + i] ? fmaf(prob[kg * RPT + i][k], v, o[i]) : o[i];
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RPT; i++) {
    const int r = kg * RPT + i;
    if (r >= nrow) continue;
    if (p.shares == 1) {
      static_cast<float *>(p.out)[((size_t)unit * per + r0 + r) * D + d] = row_l[r] == 0.f ? 0.f : o[i] / row_l[r];
    } else {
      float *rec = p.ws + ((size_t)blockIdx.x * kVecRows + r) * kVecRec<D>;
      rec[4 + d] = o[i];
      if (d == 0) {
        rec[0] = row_m[r];
        rec[1] = row_l[r];
      }
    }
  }
}

// The records of one row's shares; one thread per column.
template <int D>
__global__ __launch_bounds__(D) void quant_vector_join(QuantAttnParams p) {
  const int blocks = vector_blocks(p), per = p.nq * p.G;
  const int unit = blockIdx.x / per, row = blockIdx.x % per, d = threadIdx.x;
  const float *rec = p.ws + (((size_t)unit * blocks + row / kVecRows) * p.shares * kVecRows + row % kVecRows) * kVecRec<D>;
  const size_t pitch = (size_t)kVecRows * kVecRec<D>;
  float m = kNegInf, den = 0.f, o = 0.f;
#pragma unroll 8
  for (int k = 0; k < p.shares; k++) m = fmaxf(m, rec[k * pitch]);
  const float ref = m == kNegInf ? 0.f : m;
#pragma unroll 8
  for (int k = 0; k < p.shares; k++) {
    const float l = rec[k * pitch + 1], f = l == 0.f ? 0.f : exp2f(rec[k * pitch] - ref);
    den = fmaf(l, f, den);
    o = fmaf(rec[k * pitch + 4 + d], f, o);
  }
  static_cast<float *>(p.out)[((size_t)unit * per + row) * D + d] = den == 0.f ? 0.f : o / den;
}

// ---------------------------------------------------------------------------
// bfloat16: matrix products straight from the codes.
//
// A unit (context, layer, KV head) has R = C nq G query rows, in blocks of 16.
// With k_j = z + s n (per group) the logit of a key is
//   q.k = sum_groups s (q.n) + z (sum of q in the group),
// and the output of column d is
//   sum_j p_j v_jd = sum_j (p_j s_j) n_jd + sum_j p_j z_j,
// so the codes themselves are matrix operands, and scales and offsets touch
// one number per key and group. A code placed in the low bits of a float16 is
// the subnormal n 2^-24 (or n 2^-20 four bits up), which the matrix cores take
// as exactly that; expanding eight codes costs one shift and four ands.
//   S^T = K.Q^T : A = codes of 16 keys x 32 d, B = q in float16, per row scaled
//     by a power of two so that bfloat16's values stay exact (2^-25 of the
//     row's largest). A product per group, then an fma by the keys' scales.
//     The offsets' part is one more product over the groups' sums of q, held
//     as three float16 terms.
//   O = P.V : P is float16 (the layout of S^T is the A operand's), P s its
//     product with the scales of a group, B = codes. One more product has the
//     offsets as columns and a column of ones: the sums of p, as rounded.
// Rounding p and p s to float16 costs 2^-11 each, below the bfloat16 output's
// 2^-8; sums stay in float32.
//
// Work: the tiles of all units, one after the other, are cut into equal spans,
// one wave each, as many as the chip holds at once; a wave leaves one partial
// record per unit that its span touches. The lengths are read on the device,
// so the cut follows them. A second kernel joins the records with the
// sequence's own rows.

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;

__device__ __forceinline__ rsrc_t make_rsrc(const void *p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), (short)0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2_t){a, b}, half2_t));
}
__device__ __forceinline__ uint32_t mul_f16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, a) * __builtin_bit_cast(half2_t, b));
}
__device__ __forceinline__ float4_t mfma_f16(u32x4 a, u32x4 b, float4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ float4_t mfma_f16_k16(u32x2 a, u32x2 b, float4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(half4_t, a), __builtin_bit_cast(half4_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ float4_t mfma_bf16(u32x4 a, u32x4 b, float4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
// Lane 0's value as a scalar.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A partial record of one query row: (max, sum, -, -) in the log2 domain, then
// o / sum as D float16.
template <int D>
constexpr int kRecFloats = 4 + D / 2;

// The running reference of a row's exponents is moved where a logit exceeds it
// by more than kSlack (log2), to kHead below the largest: p stays at most 16,
// so that p s fits float16 (s <= 2184.6), and is rarely far below 1, where
// float16 gets coarse. The first tile of a piece sets it: a row that sees no
// key there sees none later.
constexpr float kSlack = 4.0f, kHead = 1.0f;

__device__ __forceinline__ int ctx_tiles(const QuantAttnParams &p, int c) {
  return c < p.P ? (ctx_len(p, c) + kQuantTile - 1) / kQuantTile : 0;
}

// The workspace: the cut (1 + P ints, to a multiple of 16 bytes), the records.
__host__ __device__ __forceinline__ size_t cut_floats(int P) { return ((size_t)P + 4) / 4 * 4; }
__device__ __forceinline__ float *records(const QuantAttnParams &p) { return p.ws + cut_floats(p.P); }

// How the tiles are cut: all units in order, `span` tiles to a wave. The host
// has refused contexts of 2^31 tiles and more.
struct Cut {
  int span, total;  // in tiles
  int first, sum;   // lane: tiles of context `lane`; of contexts 0 .. lane
};

// Inclusive sum over the lanes: within rows of 16 (by 1, 2, 4, 8), then the
// last lanes of rows 0 and 2 into 1 and 3, then that of row 1 into 2 and 3.
__device__ __forceinline__ int scan_lanes(int t) {
  t += __builtin_amdgcn_update_dpp(0, t, 0x111, 0xf, 0xf, true);
  t += __builtin_amdgcn_update_dpp(0, t, 0x112, 0xf, 0xf, true);
  t += __builtin_amdgcn_update_dpp(0, t, 0x114, 0xf, 0xf, true);
  t += __builtin_amdgcn_update_dpp(0, t, 0x118, 0xf, 0xf, true);
  t += __builtin_amdgcn_update_dpp(0, t, 0x142, 0xa, 0xf, false);
  t += __builtin_amdgcn_update_dpp(0, t, 0x143, 0xc, 0xf, false);
  return t;
}
// Lane i's value as a scalar.
__device__ __forceinline__ int lane_value(int x, int i) { return __builtin_amdgcn_readlane(x, i); }

__device__ __forceinline__ Cut cut_of(const QuantAttnParams &p, int lane) {
  Cut cut;
  cut.first = ctx_tiles(p, lane);
  cut.sum = scan_lanes(cut.first);
  int sum = lane_value(cut.sum, kWave - 1);
  for (int c0 = kWave; c0 < p.P; c0 += kWave)
    sum += lane_value(scan_lanes(ctx_tiles(p, c0 + lane)), kWave - 1);
  cut.total = sum * p.L * p.Hkv;
  cut.span = max((int)(((uint32_t)cut.total + p.nwaves - 1) / (uint32_t)p.nwaves), 1);
  return cut;
}

// The cut for the second kernel, before the records: the span, then the tiles
// before each context.
__device__ __forceinline__ void store_cut(const QuantAttnParams &p, const Cut &cut, int lane) {
  int *to = reinterpret_cast<int *>(p.ws);
  if (lane == 0) to[0] = cut.span;
  int t = cut.first, sc = cut.sum, at = 0;
  for (int c0 = 0;;) {
    if (c0 + lane < p.P) to[1 + c0 + lane] = at + sc - t;
    at += lane_value(sc, kWave - 1);
    c0 += kWave;
    if (c0 >= p.P) break;
    t = ctx_tiles(p, c0 + lane);
    sc = scan_lanes(t);
  }
}

typedef __attribute__((address_space(3))) void lds_void_t;

// s_waitcnt vmcnt(N), other counters unconstrained.
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt field");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
  asm volatile("" ::: "memory");  // no read of LDS moves before it
}

// s_waitcnt lgkmcnt(0): this wave's reads of LDS have been answered.
__device__ __forceinline__ void wait_lds() {
  __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));
  asm volatile("" ::: "memory");
}

// A wave's ring of tiles in LDS. A tile is one block of memory, loaded as it
// lies by LOADS instructions of 1 KiB (past the end of a unit: zeros, without
// a memory access); the operands are read from there.
template <int D, int NG>
struct Ring {
  static constexpr int LOADS = (QTile<D, NG>::BYTES + 1023) / 1024;
  static constexpr int SLOT = QTile<D, NG>::BYTES;
};

template <int D, int NG>
__device__ __forceinline__ void load_tile(char *slot, const char *tile, bool live, int lane) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
  for (int i = 0; i < Ring<D, NG>::LOADS; i++) {
    // The last instruction's lanes past the tile would write zeros behind it.
    constexpr int BYTES = QTile<D, NG>::BYTES;
    const rsrc_t r = make_rsrc(tile + i * 1024, live ? BYTES - i * 1024 : 0);
    if ((i + 1) * 1024 <= BYTES || i * 1024 + lane * 16 < BYTES)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t *)(slot + i * 1024), 16, lane * 16, 0, 0, kStreamLoad);
  }
#endif  // the host pass has no buffer-to-LDS loads
}

// With three row blocks and more the keys' values themselves are expanded, z +
// s n as float16 (off by 2^-12 of an element at most): 15 packed instructions
// per eight elements against five for the codes, but per key and row one fma
// after the product instead of two and one per group. 16 contexts shared by 8
// candidates of 6 heads 348 -> 321 us, 35 rows 328 -> 297.
template <int RB>
constexpr bool kKeyValues = RB >= 3;

// The query operands of one row block and what is summed for it.
template <int D, int NG>
struct Block {
  u32x4 q[D / 32];      // B operand of step i
  u32x2 qz;             // B operand of the offsets' product
  float unit;           // logits (log2) = unit (2^24 codes' part + offsets' part)
  float nref;           // minus the exponents' reference of the lane's row
  int limit;            // visible keys of the lane's row
  float4_t o[D / 16];   // rows 4 g + 0..3, column n of instance b
  float4_t z;           // the same rows; column: group's offsets, NG: sum of p
};

// Four code operands of a code word: codes 0 and 4 (times 2^-24), 1 and 5 (times 2^-20), 2 and 6, 3 and 7.
__device__ __forceinline__ u32x4 expand(uint32_t w) {
  const uint32_t h = w >> 8;
  return (u32x4){w & 0x000f000fu, w & 0x00f000f0u, h & 0x000f000fu, h & 0x00f000f0u};
}

// z + s n of a code word's elements, in the order of expand(): n from 1024 + n
// (the mantissa of a float16), exactly.
__device__ __forceinline__ u32x4 expand_values(uint32_t w, f16_t s, f16_t z) {
  const half2_t s2 = {s, s}, z2 = {z, z}, base = {(f16_t)1024.f, (f16_t)1024.f};
  uint32_t bias = 0x64006400u;
  asm("" : "+v"(bias));  // in a vector register: one and-or instruction per pair
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const half2_t n = __builtin_bit_cast(half2_t, ((w >> (4 * i)) & 0x000f000fu) | bias) - base;
    out[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(n, s2, z2));
  }
  return out;
}

template <int D, int NG, bool VALUES>
__device__ __forceinline__ void load_queries(Block<D, NG> &b, const QuantAttnParams &p, const bf16_t *row, int lane) {
  const int g = lane >> 4;
  float x[D / 32][8];
  float big = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; i++) {
    u32x4 w = {0u, 0u, 0u, 0u};
    if (row) w = *reinterpret_cast<const u32x4 *>(row + 32 * i + 8 * g);
#pragma unroll
    for (int e = 0; e < 4; e++) {
      x[i][2 * e] = bf16_lo(w[e]);
      x[i][2 * e + 1] = bf16_hi(w[e]);
      big = fmaxf(big, fmaxf(fabsf(x[i][2 * e]), fabsf(x[i][2 * e + 1])));
    }
  }
  big = fmaxf(big, shfl_xor(big, 16));
  big = fmaxf(big, shfl_xor(big, 32));
  // The row times 2^-e lies in [2^8, 2^9) at its largest.
  int e = 0;
  if (big > 0.f && big < __builtin_huge_valf()) e = ilogbf(big) - 8;
  float sum[NG];
#pragma unroll
  for (int k = 0; k < NG; k++) sum[k] = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; i++) {
#pragma unroll
    for (int k = 0; k < 8; k++) {
      x[i][k] = ldexpf(x[i][k], -e);
      sum[i * NG / (D / 32)] += x[i][k];
    }
    b.q[i][0] = pack_f16(x[i][0], x[i][4]);
    constexpr float kHigh = VALUES ? 1.f : 0.0625f;  // of codes placed four bits up
    b.q[i][1] = pack_f16(x[i][1] * kHigh, x[i][5] * kHigh);
    b.q[i][2] = pack_f16(x[i][2], x[i][6]);
    b.q[i][3] = pack_f16(x[i][3] * kHigh, x[i][7] * kHigh);
  }
  float mine = 0.f;  // the sum of group g
#pragma unroll
  for (int k = 0; k < NG; k++) {
    sum[k] += shfl_xor(sum[k], 16);
    sum[k] += shfl_xor(sum[k], 32);
    mine = k == g ? sum[k] : mine;
  }
  const float hi = (float)(f16_t)mine, mid = (float)(f16_t)(mine - hi);
  b.qz[0] = pack_f16(hi, mid);
  b.qz[1] = pack_f16(mine - hi - mid, 0.f);
  b.unit = ldexpf(p.scale * kLog2e, e);
}

template <int D, int NG>
__device__ __forceinline__ void clear(Block<D, NG> &b) {
  b.nref = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; i++) b.o[i] = (float4_t){0.f, 0.f, 0.f, 0.f};
  b.z = (float4_t){0.f, 0.f, 0.f, 0.f};
}

// The key in a tile of slot 8 g + e of the values' order.
__device__ __forceinline__ int slot_key(int g, int e) { return e < 4 ? 4 * g + e : 16 + 4 * g + e - 4; }

// The last tile of a context: slots past the last hold anything, so their value
// scales and offsets become 0 in LDS (p = 0 times a NaN would reach every row).
template <int D, int NG>
__device__ __forceinline__ void clear_dead_slots(char *slot, int live, int lane) {
  using Q = QTile<D, NG>;
#pragma unroll
  for (int e = lane; e < 32 * NG; e += kWave) {
    const int i = e & 7, g = (e >> 3) & 3;  // slot 8 g + i of a group
    if (slot_key(g, i) >= live) {
      *reinterpret_cast<uint16_t *>(slot + Q::VS + 2 * e) = 0;
      *reinterpret_cast<uint16_t *>(slot + Q::VZ + 2 * e) = 0;
    }
  }
}

// Between the phases of a tile: what a phase loads from LDS is not held in
// registers through the one before it.
__device__ __forceinline__ void phase() { __builtin_amdgcn_sched_barrier(0); }

// One tile for RB row blocks; key0: the tile's first key; tail: some row does
// not see some of its keys.
template <int D, int NG, int RB>
__device__ __forceinline__ void tile_step(Block<D, NG> (&blk)[RB], const char *slot, int key0, bool tail,
                                          bool first, const int *limits, int lane) {
  using Q = QTile<D, NG>;
  const int n = lane & 15, g = lane >> 4;
  float4_t d[RB][2];  // logits less the rows' references (log2)
#pragma unroll
  for (int t = 0; t < 2; t++) {
    constexpr int PER = D / 32 / NG;  // products per group
    const u32x4 code = *reinterpret_cast<const u32x4 *>(slot + (D == 128 ? t * 1024 : 0) + lane * 16);
    if constexpr (kKeyValues<RB>) {
      const f16_t *sk = reinterpret_cast<const f16_t *>(slot + Q::KS) + (16 * t + n) * NG;
      const f16_t *zk = reinterpret_cast<const f16_t *>(slot + Q::KZ) + (16 * t + n) * NG;
      u32x4 ka[D / 32];
#pragma unroll
      for (int i = 0; i < D / 32; i++) ka[i] = expand_values(code[D == 128 ? i : 2 * t + i], sk[i / PER], zk[i / PER]);
#pragma unroll
      for (int i = 0; i < D / 32; i++)  // the blocks' products between the steps of one
#pragma unroll
        for (int b = 0; b < RB; b++)
          d[b][t] = mfma_f16(ka[i], blk[b].q[i], i == 0 ? (float4_t){0.f, 0.f, 0.f, 0.f} : d[b][t]);
    } else {
      uint32_t z = *reinterpret_cast<const uint16_t *>(slot + Q::KZ + t * 32 * NG + (n * NG + (NG == 4 ? g : g & (NG - 1))) * 2);
      if (NG < 4) z = g < NG ? z : 0u;
      const u32x2 kz = {z | (z << 16), z};
      uint32_t ks[2 * NG];  // scales of keys 4 g .. 4 g + 3: [key][group] float16
#pragma unroll
      for (int i = 0; i < 2 * NG; i++) ks[i] = *reinterpret_cast<const uint32_t *>(slot + Q::KS + t * 32 * NG + g * 8 * NG + i * 4);
      u32x4 ka[D / 32];
#pragma unroll
      for (int i = 0; i < D / 32; i++) ka[i] = expand(code[D == 128 ? i : 2 * t + i]);
#pragma unroll
      for (int b = 0; b < RB; b++) {
        const Block<D, NG> &B = blk[b];
        const float4_t zt = mfma_f16_k16(kz, B.qz, (float4_t){0.f, 0.f, 0.f, 0.f});
        float xs[4];
#pragma unroll
        for (int k = 0; k < NG; k++) {
          float4_t a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < PER; i++) a = mfma_f16(ka[k * PER + i], B.q[k * PER + i], a);
#pragma unroll
          for (int j = 0; j < 4; j++) {
            const int at = j * NG + k;
            const half2_t h = __builtin_bit_cast(half2_t, ks[at >> 1]);
            const float sc = (float)h[at & 1];
            xs[j] = k == 0 ? a[j] * sc : fmaf(a[j], sc, xs[j]);
          }
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
          d[b][t][j] = fmaf(fmaf(xs[j], 0x1p24f, zt[j]), B.unit, B.nref);
        }
      }
    }
  }
  if constexpr (kKeyValues<RB>) {
#pragma unroll
    for (int b = 0; b < RB; b++)
#pragma unroll
      for (int t = 0; t < 2; t++)
#pragma unroll
        for (int j = 0; j < 4; j++) d[b][t][j] = fmaf(d[b][t][j], blk[b].unit, blk[b].nref);
  }
  phase();
  u32x4 vz = *reinterpret_cast<const u32x4 *>(slot + Q::VZ + (n & (NG - 1)) * 64 + g * 16);
  if (tail) {
    asm volatile("");  // a branch, not selects in every tile
#pragma unroll
    for (int b = 0; b < RB; b++)
#pragma unroll
      for (int t = 0; t < 2; t++)
#pragma unroll
        for (int j = 0; j < 4; j++)
          d[b][t][j] = key0 + 16 * t + 4 * g + j < (RB <= 2 ? blk[b].limit : limits[16 * b + n]) ? d[b][t][j] : kNegInf;
  }
  // Column NG holds ones; what the columns after it hold is not used.
#pragma unroll
  for (int r = 0; r < 4; r++) vz[r] = n == NG ? 0x3c003c00u : vz[r];
  u32x4 p[RB];
#pragma unroll
  for (int b = 0; b < RB; b++) {
    Block<D, NG> &B = blk[b];
    float top = kNegInf;
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int j = 0; j < 4; j++) top = fmaxf(top, d[b][t][j]);
    if (first || __any(top > kSlack)) {
      top = fmaxf(top, shfl_xor(top, 16));
      top = fmaxf(top, shfl_xor(top, 32));
      const bool move = first ? top > kNegInf : top > kSlack;
      const float up = move ? top - kHead : 0.f;
      const float f = first ? 1.f : fast_exp2(-up);
      B.nref -= up;
#pragma unroll
      for (int t = 0; t < 2; t++)
#pragma unroll
        for (int j = 0; j < 4; j++) d[b][t][j] -= up;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const float fj = __shfl(f, 4 * g + j, kWave);
#pragma unroll
        for (int i = 0; i < D / 16; i++) B.o[i][j] *= fj;
        B.z[j] *= fj;
      }
    }
#pragma unroll
    for (int t = 0; t < 2; t++) {
      p[b][2 * t] = pack_f16(fast_exp2(d[b][t][0]), fast_exp2(d[b][t][1]));
      p[b][2 * t + 1] = pack_f16(fast_exp2(d[b][t][2]), fast_exp2(d[b][t][3]));
    }
    B.z = mfma_f16(p[b], vz, B.z);
  }
  phase();
  // Values: half h of the codes has instances 4 h .. 4 h + 3, in GH groups.
#pragma unroll
  for (int h = 0; h < D / 64; h++) {
    constexpr int IPG = Q::GROUP / 16, GH = 4 / IPG;  // instances per group
    u32x4 vs[GH];
#pragma unroll
    for (int i = 0; i < GH; i++) vs[i] = *reinterpret_cast<const u32x4 *>(slot + Q::VS + (h * GH + i) * 64 + g * 16);
    const u32x4 code = *reinterpret_cast<const u32x4 *>(slot + Q::VC + h * 1024 + lane * 16);
    u32x4 vb[4];
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const u32x4 x = expand(code[r]);
#pragma unroll
      for (int i = 0; i < 4; i++) vb[i][r] = x[i];
    }
#pragma unroll
    for (int b = 0; b < RB; b++) {
      u32x4 ps;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const int inst = 4 * h + i;
        if (i % IPG == 0) {
#pragma unroll
          for (int r = 0; r < 4; r++) ps[r] = mul_f16(p[b][r], vs[i / IPG][r]);
        }
        blk[b].o[inst] = mfma_f16(ps, vb[i], blk[b].o[inst]);
      }
    }
  }
}

// Waves per SIMD and tiles in a wave's ring. Registers hold two waves of up to
// three row blocks at D = 128, more of fewer at D = 64 (18.2 us against 18.7
// for 61 contexts of up to 2000). Two waves' rings of four 5 KiB tiles are all
// of a CU's LDS: 32 contexts of 16384 in groups of 64 take 620, 656 and 588 us
// with rings of two, three and four tiles, 590 with three waves of two.
constexpr int ctx_waves(int D, int RB) { return D == 128 || RB >= 3 ? 2 : RB == 2 ? 3 : 4; }
constexpr int ctx_depth(int D, int RB) { return D == 128 && RB >= 3 ? 3 : 4; }

// Context kernel: one wave per span.
template <int D, int NG, int RB>
__global__ __launch_bounds__(kWave) __attribute__((amdgpu_waves_per_eu(ctx_waves(D, RB)))) void quant_ctx(QuantAttnParams p) {
  using Q = QTile<D, NG>;
  constexpr int DEPTH = ctx_depth(D, RB), LOADS = Ring<D, NG>::LOADS, SLOT = Ring<D, NG>::SLOT;
  // With the ring, beyond two blocks (registers): the visible keys of each row.
  // One array: of two, the compiler waits for every load into the ring before
  // it reads any of it (16 contexts shared by 8 candidates of 6 heads 320 us,
  // 288 so).
  __shared__ __align__(1024) char ring[DEPTH * SLOT + (RB <= 2 ? 0 : RB * 64)];
  int *limits = reinterpret_cast<int *>(ring + DEPTH * SLOT);
  const int lane = threadIdx.x, n = lane & 15, g = lane >> 4;
  // The row groups of a span run eight workgroups apart, on one XCD.
  const int xcd = blockIdx.x & 7, k8 = blockIdx.x >> 3;
  const int w = (k8 / p.row_groups) * 8 + xcd, rg = k8 % p.row_groups;
  if (w >= p.nwaves) return;
  const Cut cut = cut_of(p, lane);
  if (blockIdx.x == 0) store_cut(p, cut, lane);
  if ((long)w * cut.span >= cut.total) return;
  int pos = w * cut.span;
  const int end = min(pos + cut.span, cut.total);
  const int lh = p.L * p.Hkv, rows = p.C * p.nq * p.G, per = p.nq * p.G;
  // The context that holds the first tile, and the tiles before it.
  int c = 0, at = 0, t = cut.first, sc = cut.sum;
  for (;;) {
    const uint64_t past = __ballot((at + sc) * lh > pos);
    if (past) {
      const int i = uniform(__ffsll((long long)past) - 1);
      c += i;
      at += lane_value(sc - t, i);
      break;
    }
    at += lane_value(sc, kWave - 1);
    c += kWave;
    t = ctx_tiles(p, c + lane);
    sc = scan_lanes(t);
  }
  int n_ctx = uniform(ctx_len(p, c)), tiles = (n_ctx + kQuantTile - 1) / kQuantTile;
  int u = (pos - at * lh) / tiles;  // unit within the context
  int tile = (pos - at * lh) % tiles;
  Block<D, NG> blk[RB];
  while (pos < end) {
    const int last = min(tiles, tile + (end - pos));
    const int l = u / p.Hkv, h = u % p.Hkv;
    const char *base = static_cast<const char *>(p.data) + ((size_t)c * lh + u) * p.ntiles * Q::BYTES;
    // The first tiles are on their way while the queries are made ready.
#pragma unroll
    for (int i = 0; i < DEPTH - 1; i++)
      load_tile<D, NG>(ring + i * SLOT, base + (size_t)(tile + i) * Q::BYTES, tile + i < last, lane);
    int least = n_ctx;
#pragma unroll
    for (int i = 0; i < RB; i++) {
      const int r = (rg * RB + i) * 16 + n;
      const bf16_t *row = nullptr;
      int limit = n_ctx;
      if (r < rows) {
        const int s = c * p.C + r / per, rr = r % per;
        row = static_cast<const bf16_t *>(p.q) + ((((size_t)s * p.L + l) * p.Hkv + h) * per + rr) * D;
        if (p.nq > 1) limit = (int)min((long)n_ctx, (long)n_ctx + own_len(p, s) - (p.nq - 1 - rr % p.nq));
      }
      load_queries<D, NG, kKeyValues<RB>>(blk[i], p, row, lane);
      clear<D, NG>(blk[i]);
      if (RB <= 2) blk[i].limit = limit;
      else limits[16 * i + n] = limit;
      if (p.nq > 1) {
#pragma unroll
        for (int x = 8; x >= 1; x >>= 1) limit = min(limit, shfl_xor(limit, x));
        least = min(least, uniform(limit));
      }
    }
    // The queries' loads are done, so that the waits below count tiles alone
    // (and with them the first tiles', which were issued before).
    wait_vm<0>();
    int at_slot = 0;
    for (int t = tile; t < last; t++) {
      const int next = at_slot == 0 ? DEPTH - 1 : at_slot - 1, tn = t + DEPTH - 1;
      wait_lds();  // the slot's tile has been read
      load_tile<D, NG>(ring + next * SLOT, base + (size_t)tn * Q::BYTES, tn < last, lane);
      wait_vm<LOADS *(DEPTH - 1)>();
      if ((t + 1) * Q::KEYS > n_ctx) clear_dead_slots<D, NG>(ring + at_slot * SLOT, n_ctx - t * Q::KEYS, lane);
      tile_step<D, NG, RB>(blk, ring + at_slot * SLOT, t * Q::KEYS, (t + 1) * Q::KEYS > least, t == tile, limits, lane);
      at_slot = at_slot + 1 == DEPTH ? 0 : at_slot + 1;
    }
    wait_vm<0>();  // the zeros behind the last tile, before the ring starts again
    wait_lds();
    // The records of this piece.
    float *rec = records(p) + ((size_t)w + (size_t)c * lh + u) * rows * kRecFloats<D>;
#pragma unroll
    for (int i = 0; i < RB; i++) {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int r = (rg * RB + i) * 16 + 4 * g + j;
        const float den = __shfl(blk[i].z[j], (lane & 48) + NG, kWave);
        const float ref = -__shfl(blk[i].nref, 4 * g + j, kWave);
        const float inv = den > 0.f ? 1.0f / den : 0.f;
        float off_j[NG];
#pragma unroll
        for (int k = 0; k < NG; k++) off_j[k] = __shfl(blk[i].z[j], (lane & 48) + k, kWave);
        if (r < rows) {
          float *to = rec + (size_t)r * kRecFloats<D>;
          if (n == 0) *reinterpret_cast<float2_t *>(to) = (float2_t){den == 0.f ? kNegInf : ref, den};
#pragma unroll
          for (int x = 0; x < D / 32; x++) {
            const float o = off_j[x * 32 / Q::GROUP];
            reinterpret_cast<uint32_t *>(to + 4)[x * 16 + n] =
                pack_f16((blk[i].o[2 * x][j] * 0x1p24f + o) * inv, (blk[i].o[2 * x + 1][j] * 0x1p20f + o) * inv);
          }
        }
      }
    }
    pos += last - tile;
    tile = 0;
    if (++u == lh && pos < end) {
      u = 0;
      do {
        c++;
        n_ctx = uniform(ctx_len(p, c));
      } while (n_ctx == 0);  // pos < end: a later context has tiles
      tiles = (n_ctx + kQuantTile - 1) / kQuantTile;
    }
  }
}

// One chunk of 32 own keys as a lane holds it: the rows of K as the A operand
// (keys n and 16 + n, d = 32 i + 8 g + 0..7), of V the 8 keys of the lane's
// slots at d = n D / 16 ...
template <int D>
struct OwnChunk {
  u32x4 k[2][D / 32];
  uint32_t v[8][D / 32];
};

// The own rows of a unit and the query rows r0 .. r0 + nrow - 1 of its
// sequence. Rows before `first` are in the cache, the new ones after it in the
// caller's array (another workgroup may be storing them). Both are read as
// buffers that end with them, so rows past the last live one are zeros,
// whatever their slots hold.
struct OwnUnit {
  const bf16_t *k, *v, *fk, *fv;
  int u, first, nq, r0, nrow;
  float sl2;
};

template <int D>
__device__ __forceinline__ OwnUnit own_unit(const QuantAttnParams &p, int unit, int u, int r0, int nrow) {
  const size_t own0 = (size_t)unit * p.ocap * D, new0 = (size_t)unit * p.nq * D;
  return OwnUnit{static_cast<const bf16_t *>(p.ok) + own0, static_cast<const bf16_t *>(p.ov) + own0,
                 static_cast<const bf16_t *>(p.k_new) + new0, static_cast<const bf16_t *>(p.v_new) + new0,
                 u, p.k_new ? u - p.nq : u, p.nq, r0, nrow, p.scale * kLog2e};
}

// The rows of a chunk that are in the cache; the bounds check takes the whole
// offset, so a chunk's place goes into the base. A chunk reads 32 rows, so a
// buffer of those is enough, and its bytes fit 32 bits in any cache.
template <int D>
__device__ __forceinline__ rsrc_t held_rows(const bf16_t *rows, const OwnUnit &w, int key0) {
  // A scalar: bounds in vector registers would put a loop around every load.
  return make_rsrc(rows + (size_t)key0 * D, (uint32_t)uniform(min(max(w.first - key0, 0), 32)) * (2 * D));
}

// ONE: a single query token, so at most one new row, the last: its lanes' words
// are loaded beside (registers: 20 words instead of a second chunk).
template <int D, bool ONE>
__device__ __forceinline__ void load_keys(OwnChunk<D> &c, const OwnUnit &w, int key0, int lane) {
  constexpr int ROW = 2 * D;
  const int n = lane & 15, g = lane >> 4;
  const rsrc_t held = held_rows<D>(w.k, w, key0);
#pragma unroll
  for (int t = 0; t < 2; t++)
#pragma unroll
    for (int i = 0; i < D / 32; i++)
      c.k[t][i] = __builtin_amdgcn_raw_buffer_load_b128(held, n * ROW + g * 16 + t * 16 * ROW + i * 64, 0, kStreamLoad);
  if (key0 + 32 <= w.first || key0 >= w.u || w.first == w.u) return;
  const rsrc_t fresh = make_rsrc(w.fk, w.nq * ROW);
  if constexpr (ONE) {
    const int key = w.first - key0;
    const uint32_t off = n == (key & 15) ? g * 16 : 0x40000000u;
    u32x4 x[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; i++) x[i] = __builtin_amdgcn_raw_buffer_load_b128(fresh, off + i * 64, 0, kStreamLoad);
    // Masks, not branches: a load that one path does not take up is waited for
    // where the paths meet, and with it the loads before.
#pragma unroll
    for (int t = 0; t < 2; t++) {
      const uint32_t mask = t == key >> 4 ? ~0u : 0u;
#pragma unroll
      for (int i = 0; i < D / 32; i++) c.k[t][i] |= x[i] & mask;
    }
  } else {
    // Rows before the first new one get an offset past the end.
#pragma unroll
    for (int t = 0; t < 2; t++) {
      const uint32_t off = (uint32_t)((key0 + 16 * t + n - w.first) * ROW);
#pragma unroll
      for (int i = 0; i < D / 32; i++)
        c.k[t][i] |= __builtin_amdgcn_raw_buffer_load_b128(fresh, off + (g * 16 + i * 64), 0, kStreamLoad);
    }
  }
}

template <int D, bool ONE>
__device__ __forceinline__ void load_values(OwnChunk<D> &c, const OwnUnit &w, int key0, int lane) {
  constexpr int ROW = 2 * D;
  const int n = lane & 15, g = lane >> 4;
  auto get = [&](rsrc_t r, uint32_t off, uint32_t (&x)[D / 32], bool add) {
    if constexpr (D == 128) {
      const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, off + n * 16, 0, kStreamLoad);
#pragma unroll
      for (int i = 0; i < 4; i++) x[i] = add ? x[i] | v[i] : v[i];
    } else {
      const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(r, off + n * 8, 0, kStreamLoad);
#pragma unroll
      for (int i = 0; i < 2; i++) x[i] = add ? x[i] | v[i] : v[i];
    }
  };
  const rsrc_t held = held_rows<D>(w.v, w, key0);
#pragma unroll
  for (int e = 0; e < 8; e++) get(held, slot_key(g, e) * ROW, c.v[e], false);
  if (key0 + 32 <= w.first || key0 >= w.u || w.first == w.u) return;
  const rsrc_t fresh = make_rsrc(w.fv, w.nq * ROW);
  if constexpr (ONE) {
    const int key = w.first - key0, slot = 4 * (key >> 4) + (key & 3);
    uint32_t x[D / 32];
    get(fresh, g == ((key >> 2) & 3) ? 0u : 0x40000000u, x, false);
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const uint32_t mask = e == slot ? ~0u : 0u;
#pragma unroll
      for (int i = 0; i < D / 32; i++) c.v[e][i] |= x[i] & mask;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; e++) get(fresh, (uint32_t)((key0 + slot_key(g, e) - w.first) * ROW), c.v[e], true);
  }
}

// Where the records of context c's units are: what is loaded of it, and the
// waves w0 .. w1 of the context kernel that left records of unit u.
struct RecordPlan {
  int span, before, len;
  __device__ __forceinline__ RecordPlan(const QuantAttnParams &p, int c) {
    const int *cut = reinterpret_cast<const int *>(p.ws);
    span = cut[0];
    before = cut[1 + c];
    len = p.ctx_len[c];
  }
};
struct Records {
  int w0, w1;
};
__device__ __forceinline__ Records records_of(const QuantAttnParams &p, const RecordPlan &plan, int u) {
  const int tiles = (min(max(uniform(plan.len), 0), p.cap) + kQuantTile - 1) / kQuantTile;
  const uint32_t span = uniform(plan.span), first = uniform(plan.before) * p.L * p.Hkv + u * tiles;
  const int w0 = first / span;
  return Records{w0, tiles > 0 ? (int)((first + tiles - 1) / span) : w0 - 1};
}

// What a wave has of the own rows: 16 query rows (lane's row: n), running
// maximum and sum per row, o as rows 4 g + 0..3 at d = n D / 16 + b.
template <int D>
struct OwnState {
  u32x4 q[D / 32];
  int limit;  // keys that the lane's row sees
  float m, den;
  float4_t o[D / 16];
};

template <int D>
__device__ __forceinline__ void own_begin(OwnState<D> &st, const QuantAttnParams &p, const OwnUnit &w, int unit, int lane) {
  const int n = lane & 15, g = lane >> 4, r = w.r0 + min(n, w.nrow - 1);
  const bf16_t *row = static_cast<const bf16_t *>(p.q) + ((size_t)unit * p.nq * p.G + r) * D;
#pragma unroll
  for (int i = 0; i < D / 32; i++) st.q[i] = *reinterpret_cast<const u32x4 *>(row + 32 * i + 8 * g);
  st.limit = w.u - (p.nq - 1 - r % p.nq);
  st.m = kNegInf;
  st.den = 0.f;
#pragma unroll
  for (int b = 0; b < D / 16; b++) st.o[b] = (float4_t){0.f, 0.f, 0.f, 0.f};
}

// The B operand of instance b from the values of the lane's 8 slots.
template <int D>
__device__ __forceinline__ u32x4 value_operand(const uint32_t (&v)[8][D / 32], int b) {
  u32x4 w;
#pragma unroll
  for (int r = 0; r < 4; r++)
    w[r] = __builtin_amdgcn_perm(v[2 * r + 1][b / 2], v[2 * r][b / 2], b & 1 ? 0x07060302u : 0x05040100u);
  return w;
}

// One chunk at key0; `next` follows it.
template <int D, bool ONE>
__device__ __forceinline__ void own_step(OwnState<D> &st, OwnChunk<D> &ch, const OwnUnit &w, int key0, int next,
                                         int lane) {
  const int g = lane >> 4;
  float x[2][4], top = kNegInf;
#pragma unroll
  for (int t = 0; t < 2; t++) {
    float4_t a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 32; i++) a = mfma_bf16(ch.k[t][i], st.q[i], a);
#pragma unroll
    for (int j = 0; j < 4; j++) {
      x[t][j] = key0 + 16 * t + 4 * g + j < st.limit ? a[j] * w.sl2 : kNegInf;
      top = fmaxf(top, x[t][j]);
    }
  }
  load_keys<D, ONE>(ch, w, next, lane);
  top = fmaxf(top, shfl_xor(top, 16));
  top = fmaxf(top, shfl_xor(top, 32));
  const float mn = fmaxf(st.m, top), ref = mn == kNegInf ? 0.f : mn;
  if (__any(mn > st.m)) {
    const float f = fast_exp2(st.m - ref);
    st.den *= f;
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const float fj = __shfl(f, 4 * g + j, kWave);
#pragma unroll
      for (int b = 0; b < D / 16; b++) st.o[b][j] *= fj;
    }
  }
  st.m = mn;
  u32x4 hi, lo;
#pragma unroll
  for (int t = 0; t < 2; t++)
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      const float e0 = fast_exp2(x[t][j] - ref), e1 = fast_exp2(x[t][j + 1] - ref);
      st.den += e0 + e1;
      const uint32_t h = pack_bf16x2(e0, e1);
      hi[2 * t + j / 2] = h;
      lo[2 * t + j / 2] = pack_bf16x2(e0 - bf16_lo(h), e1 - bf16_hi(h));
    }
  // Rows that only later queries see may hold a value that is not finite, which
  // would reach the others as 0 times it: those get a product per query token.
  const int sees_all = w.u - (w.nq - 1);
  bool split = false;
  if (!ONE && key0 + 32 > sees_all && w.nq > 1) {
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      bool any = false;
#pragma unroll
      for (int i = 0; i < D / 32; i++) {
        const uint32_t v = ch.v[e][i];
        any |= (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
      }
      odd |= any && key0 + slot_key(g, e) >= sees_all;
    }
    split = __any(odd);
  }
  if (ONE || !split) {
#pragma unroll
    for (int b = 0; b < D / 16; b++) {
      const u32x4 v = value_operand<D>(ch.v, b);
      st.o[b] = mfma_bf16(lo, v, mfma_bf16(hi, v, st.o[b]));
    }
    load_values<D, ONE>(ch, w, next, lane);
    return;
  }
#pragma unroll 1
  for (int t = 0; t < w.nq; t++) {
    const int lim = w.u - (w.nq - 1 - t);
    uint32_t see[4];
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int k0 = key0 + slot_key(g, 2 * r);
      see[r] = (k0 < lim ? 0xffffu : 0u) | (k0 + 1 < lim ? 0xffff0000u : 0u);
    }
#pragma unroll
    for (int b = 0; b < D / 16; b++) {
      u32x4 v = value_operand<D>(ch.v, b);
#pragma unroll
      for (int r = 0; r < 4; r++) v[r] &= see[r];
      const float4_t acc = mfma_bf16(lo, v, mfma_bf16(hi, v, st.o[b]));
#pragma unroll
      for (int j = 0; j < 4; j++) st.o[b][j] = (w.r0 + 4 * g + j) % w.nq == t ? acc[j] : st.o[b][j];
    }
  }
  load_values<D, ONE>(ch, w, next, lane);
}

// The chunks key0, key0 + stride, .. of a unit. A chunk's keys make way for the
// next one's once they are multiplied, its values likewise, so that those are
// under way meanwhile. p is split into two bfloat16 terms, so that its rounding
// (2^-17) stays out of the result.
template <int D, bool ONE>
__device__ __forceinline__ void own_attend(OwnState<D> &st, OwnChunk<D> &ch, const OwnUnit &w, int key0, int stride,
                                           int lane) {
  for (; key0 < w.u; key0 += stride) own_step<D, ONE>(st, ch, w, key0, key0 + stride, lane);
}

// Joins (mr, lr, values x whose sum of weights is lr after the factor scale) to a row's (m, den, o).
template <int EL>
__device__ __forceinline__ void fold(float &m, float &den, float (&o)[EL], float mr, float lr, float scale,
                                     const float (&x)[EL]) {
  const float mn = fmaxf(m, mr);
  const float fa = m == kNegInf ? 0.f : fast_exp2(m - mn), fb = lr == 0.f ? 0.f : fast_exp2(mr - mn);
  m = mn;
  den = den * fa + lr * fb;
  const float sb = scale * fb;
#pragma unroll
  for (int e = 0; e < EL; e++) o[e] = fmaf(x[e], sb, o[e] * fa);
}

// Elements sub EL .. of a record's values.
template <int EL>
__device__ __forceinline__ void record_values(const float *rec, int sub, float (&x)[EL]) {
  const f16_t *h = reinterpret_cast<const f16_t *>(rec + 4) + sub * EL;
#pragma unroll
  for (int e = 0; e < EL; e++) x[e] = (float)h[e];
}

template <int EL>
__device__ __forceinline__ void put_row(bf16_t *row, int sub, const float (&o)[EL], float den) {
  const float inv = den == 0.f ? 0.f : 1.0f / den;
  uint32_t *to = reinterpret_cast<uint32_t *>(row) + sub * (EL / 2);
#pragma unroll
  for (int e = 0; e < EL; e += 2) to[e / 2] = pack_bf16x2(o[e] * inv, o[e + 1] * inv);
}

// Second kernel, many units: a wave per (sequence, layer, KV head) and 16 of
// its rows attends to the own rows, 32 keys at a time, and joins the context's
// records as it holds its result: 16 lanes per row, four rows per lane.
template <int D, int NG, bool ONE>
__global__ __launch_bounds__(kWave) __attribute__((amdgpu_waves_per_eu(ONE ? 3 : 2))) void quant_join_wave(QuantAttnParams p) {
  constexpr int EL = D / 16;
  const int per = p.nq * p.G, blocks = (per + 15) / 16;
  const int unit = blockIdx.x / blocks, r0 = blockIdx.x % blocks * 16;
  const int lh = p.L * p.Hkv, s = unit / lh, c = s / p.C;
  const int lane = threadIdx.x, n = lane & 15, g = lane >> 4;
  const RecordPlan plan(p, c);
  const int u = uniform(own_len(p, s)), nrow = min(16, per - r0);
  OwnState<D> st;
  st.m = kNegInf;
  st.den = 0.f;
#pragma unroll
  for (int b = 0; b < D / 16; b++) st.o[b] = (float4_t){0.f, 0.f, 0.f, 0.f};
  const OwnUnit w = own_unit<D>(p, unit, u, r0, nrow);
  OwnChunk<D> ch;
  if (u > 0) {
    // The queries first: a wait for them in the loop would be one for all before.
    own_begin<D>(st, p, w, unit, lane);
    load_keys<D, ONE>(ch, w, 0, lane);
    load_values<D, ONE>(ch, w, 0, lane);
  }
  const Records here = records_of(p, plan, unit % lh);
  own_attend<D, ONE>(st, ch, w, 0, 32, lane);
  if (p.ok && r0 == 0) store_new<bf16_t, D, kWave>(p, unit, s, u);
  st.den += shfl_xor(st.den, 16);
  st.den += shfl_xor(st.den, 32);
  const int rows = p.C * per;
  const float *rec = records(p) + (((size_t)here.w0 + (size_t)c * lh + unit % lh) * rows + (s % p.C * per + r0)) * kRecFloats<D>;
  float m[4], den[4], o[4][EL];
#pragma unroll
  for (int j = 0; j < 4; j++) {
    m[j] = __shfl(st.m, 4 * g + j, kWave);
    den[j] = __shfl(st.den, 4 * g + j, kWave);
#pragma unroll
    for (int e = 0; e < EL; e++) o[j][e] = st.o[e][j];
  }
  for (int k = here.w0; k <= here.w1; k++, rec += (size_t)rows * kRecFloats<D>) {
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const float *r = rec + (size_t)min(4 * g + j, nrow - 1) * kRecFloats<D>;
      const float2_t ml = *reinterpret_cast<const float2_t *>(r);
      float x[EL];
      record_values<EL>(r, n, x);
      fold<EL>(m[j], den[j], o[j], ml[0], ml[1], ml[1], x);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; j++)
    if (4 * g + j < nrow)
      put_row<EL>(static_cast<bf16_t *>(p.out) + ((size_t)unit * per + r0 + 4 * g + j) * D, n, o[j], den[j]);
}

constexpr int kOwnWaves = 4;

// Second kernel, few units: a workgroup per (sequence, layer, KV head) and rpw
// of its rows. Its four waves attend to the own rows, 32 keys each in turn; then
// all of them join these and the context's records: 16 lanes per row, the
// records of a row dealt to the groups of 16.
template <int D, int NG>
__global__ __launch_bounds__(kOwnWaves *kWave) __attribute__((amdgpu_waves_per_eu(2))) void quant_join(QuantAttnParams p) {
  constexpr int NT = kOwnWaves * kWave, SLOTS = NT / 16, EL = D / 16;  // elements per thread of the join
  __shared__ float so[kOwnWaves][16][D];
  __shared__ float sm[SLOTS][2];
  __shared__ float wm[kOwnWaves][16], wl[kOwnWaves][16];
  const int per = p.nq * p.G, blocks = (per + p.rpw - 1) / p.rpw;
  const int unit = blockIdx.x / blocks, r0 = blockIdx.x % blocks * p.rpw;
  const int lh = p.L * p.Hkv, s = unit / lh, c = s / p.C;
  const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave), n = lane & 15, g = lane >> 4;
  const RecordPlan plan(p, c);
  const int u = uniform(own_len(p, s)), nrow = min(p.rpw, per - r0);

  const OwnUnit w = own_unit<D>(p, unit, u, r0, nrow);
  OwnState<D> st;
  OwnChunk<D> ch;
  if (u > 0) {
    own_begin<D>(st, p, w, unit, lane);
    load_keys<D, false>(ch, w, wave * 32, lane);
    load_values<D, false>(ch, w, wave * 32, lane);
  }
  const Records here = records_of(p, plan, unit % lh);
  if (p.ok && r0 == 0) store_new<bf16_t, D, NT>(p, unit, s, u);

  if (u > 0) {
    own_attend<D, false>(st, ch, w, wave * 32, kOwnWaves * 32, lane);
    st.den += shfl_xor(st.den, 16);
    st.den += shfl_xor(st.den, 32);
    if (g == 0) {
      wm[wave][n] = st.m;
      wl[wave][n] = st.den;
    }
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
      for (int b = 0; b < D / 16; b += 4)
        *reinterpret_cast<float4_t *>(&so[wave][4 * g + j][n * EL + b]) =
            (float4_t){st.o[b][j], st.o[b + 1][j], st.o[b + 2][j], st.o[b + 3][j]};
  }
  __syncthreads();

  // Join. Thread: row r0 + slot % rpw, records part, part + parts, .. of it,
  // elements sub EL ..
  const int slot = tid / 16, sub = tid % 16, parts = SLOTS / p.rpw;
  const int row = slot % p.rpw, part = slot / p.rpw;
  float m = kNegInf, den = 0.f, o[EL];
#pragma unroll
  for (int e = 0; e < EL; e++) o[e] = 0.f;
  if (row < nrow && part == 0 && u > 0) {
#pragma unroll
    for (int w = 0; w < kOwnWaves; w++) {
      float x[EL];
#pragma unroll
      for (int e = 0; e < EL; e++) x[e] = so[w][row][sub * EL + e];
      fold<EL>(m, den, o, wm[w][row], wl[w][row], 1.f, x);
    }
  }
  if (row < nrow) {
    const int rows = p.C * per, r = s % p.C * per + r0 + row;
    const float *rec = records(p) + (((size_t)(here.w0 + part) + (size_t)c * lh + unit % lh) * rows + r) * kRecFloats<D>;
#pragma unroll 4
    for (int k = here.w0 + part; k <= here.w1; k += parts, rec += (size_t)parts * rows * kRecFloats<D>) {
      const float2_t ml = *reinterpret_cast<const float2_t *>(rec);
      float x[EL];
      record_values<EL>(rec, sub, x);
      fold<EL>(m, den, o, ml[0], ml[1], ml[1], x);
    }
  }
  if (parts > 1) {
    // Halves of the groups join the others, down to one per row.
    float *po = &so[0][0][0];
    for (int half = parts / 2;; half /= 2) {
      __syncthreads();
      if (part < 2 * half) {
#pragma unroll
        for (int e = 0; e < EL; e++) po[slot * D + sub * EL + e] = o[e];
        if (sub == 0) {
          sm[slot][0] = m;
          sm[slot][1] = den;
        }
      }
      __syncthreads();
      if (part < half) {
        float x[EL];
        const int from = slot + half * p.rpw;
#pragma unroll
        for (int e = 0; e < EL; e++) x[e] = po[from * D + sub * EL + e];
        fold<EL>(m, den, o, sm[from][0], sm[from][1], 1.f, x);
      }
      if (half == 1) break;
    }
  }
  if (part == 0 && row < nrow)
    put_row<EL>(static_cast<bf16_t *>(p.out) + ((size_t)unit * per + r0 + row) * D, sub, o, den);
}

constexpr int kChipCus = 256, kChipSimds = 4 * kChipCus;
// Row blocks a wave takes at once; more rows go to further waves over the same
// tiles. Two waves per SIMD hold three at D = 128 (a fourth, one wave per SIMD,
// takes 267 us where two waves of two take 233, for 64 rows over 16 contexts of
// 8192 x 28 heads), four at D = 64 (131 us as two of two, 121).
constexpr int max_blocks(int D) { return D == 128 ? 3 : 4; }
// Fewer where tiles x blocks are at most this many times one (two): a wave's
// chain is shorter, and its tiles come from the L2. 48 rows, one block and
// three: 512 tiles 13.8 us and 16.9, 3584 25 and 36, 15136 42 (two) and 50;
// 64512 tiles 145 us with one and 116 with three.
constexpr double kBlockTiles = 65536;

// Plan of a call, from shapes alone.
void plan(QuantAttnParams *p) {
  if (p->dtype == 0) {
    // float32: shares of the chunks, up to 1024 workgroups. 32 units of 2 and 3
    // chunks: 26 us with one chunk each, 31 with two, 44 with all.
    const long groups = (long)p->S * p->L * p->Hkv * vector_blocks(*p);
    const long chunks = p->ntiles + (p->ocap + kVecKeys - 1) / kVecKeys;
    const long most = chunks < 64 ? chunks : 64, want = 1024 / groups;
    const long n = want < most ? want : most;
    p->shares = n < 1 ? 1 : (int)n;
    return;
  }
  const int rows = p->C * p->nq * p->G, blocks = (rows + 15) / 16;
  const double tiles = (double)p->P * p->L * p->Hkv * p->ntiles;
  int most_blocks = max_blocks(p->D);
  while (most_blocks > 1 && tiles * blocks <= (most_blocks - 1) * kBlockTiles) most_blocks--;
  p->row_groups = (blocks + most_blocks - 1) / most_blocks;
  p->rb = (blocks + p->row_groups - 1) / p->row_groups;
  const int waves = kChipSimds * ctx_waves(p->D, p->rb);
  const int most = waves / p->row_groups > 64 ? waves / p->row_groups : 64;
  p->nwaves = tiles < most ? (int)tiles : most;
  // The join: a wave per 16 rows where that fills the chip, or is more than a
  // workgroup per CU with about two records per unit (336 units 10.3 us, 14.4 as
  // workgroups; with seven records 20 and 16); else workgroups, of fewer rows
  // where they stay one per CU (each reads all the own rows: 132 units of 12
  // rows 13.6 us, 17 with twice as many, 27 with four times).
  const int per = p->nq * p->G;
  const long units = (long)p->S * p->L * p->Hkv, waves16 = units * ((per + 15) / 16);
  const bool few_records = p->nwaves <= 2.0 * p->P * p->L * p->Hkv;
  p->join_waves = waves16 >= kChipSimds || (waves16 > kChipCus && few_records);
  int rpw = 16;
  while (rpw > 1 && units * ((per + rpw / 2 - 1) / (rpw / 2)) <= kChipCus) rpw /= 2;
  p->rpw = rpw;
}

template <int D, int NG, int RB>
void launch_ctx(const QuantAttnParams &p, hipStream_t stream) {
  const uint32_t groups = (uint32_t)(p.nwaves + 7) / 8 * 8 * p.row_groups;
  hipLaunchKernelGGL((quant_ctx<D, NG, RB>), dim3(groups), dim3(kWave), 0, stream, p);
}

template <int D, int NG>
void launch_bf16(const QuantAttnParams &p, hipStream_t stream) {
  switch (p.rb) {
    case 1: launch_ctx<D, NG, 1>(p, stream); break;
    case 2: launch_ctx<D, NG, 2>(p, stream); break;
    case 3: launch_ctx<D, NG, 3>(p, stream); break;
    default:
      if constexpr (D == 64) launch_ctx<D, NG, 4>(p, stream);
  }
  const int per = p.nq * p.G, rpw = p.join_waves ? 16 : p.rpw;
  const dim3 groups((uint32_t)p.S * p.L * p.Hkv * ((per + rpw - 1) / rpw));
  if (p.join_waves && p.nq == 1) hipLaunchKernelGGL((quant_join_wave<D, NG, true>), groups, dim3(kWave), 0, stream, p);
  else if (p.join_waves) hipLaunchKernelGGL((quant_join_wave<D, NG, false>), groups, dim3(kWave), 0, stream, p);
  else hipLaunchKernelGGL((quant_join<D, NG>), groups, dim3(kOwnWaves * kWave), 0, stream, p);
}

template <int D, int NG>
void launch_any(const QuantAttnParams &p, hipStream_t stream) {
  if (p.dtype == 0) {
    const uint32_t units = (uint32_t)p.S * p.L * p.Hkv;
    hipLaunchKernelGGL((quant_attn_vector<D, NG>), dim3(units * vector_blocks(p) * p.shares), dim3(kThreads), 0, stream,
                       p);
    if (p.shares > 1) hipLaunchKernelGGL((quant_vector_join<D>), dim3(units * p.nq * p.G), dim3(D), 0, stream, p);
  } else {
    launch_bf16<D, NG>(p, stream);
  }
}

}  // namespace

size_t quant_attn_workspace_bytes(const QuantAttnParams &params) {
  QuantAttnParams p = params;
  plan(&p);
  if (p.dtype == 0) {
    if (p.shares == 1) return 0;
    return (size_t)p.S * p.L * p.Hkv * vector_blocks(p) * p.shares * kVecRows * (4 + p.D) * sizeof(float);
  }
  // A wave's piece of a unit has record wave + unit.
  const size_t pieces = (size_t)p.nwaves + (size_t)p.P * p.L * p.Hkv;
  return (cut_floats(p.P) + pieces * p.C * p.nq * p.G * (4 + p.D / 2)) * sizeof(float);
}

hipError_t launch_quant_attn(const QuantAttnParams &params, hipStream_t stream) {
  QuantAttnParams p = params;
  plan(&p);
  if (p.D == 128) {
    if (p.group == 32) launch_any<128, 4>(p, stream);
    else launch_any<128, 2>(p, stream);
  } else {
    if (p.group == 32) launch_any<64, 2>(p, stream);
    else launch_any<64, 1>(p, stream);
  }
  return hipGetLastError();
}

}  // namespace kvr
