// The 4-bit cache written and read back: rows quantised and appended, and
// rows given back as the values they stand for.
//
// Both kernels are copies bound by memory: a row of D bf16 values and its D /
// 2 + 4 NG bytes, K and V each.
#include <hip/hip_runtime.h>

#include "kvr_device.h"
#include "kvr_internal.h"
#include "quant_common.h"

namespace kvr {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
// Waves of an append's workgroup: a wave per KiB of codes, K and V.
template <int D>
constexpr int kAppendWaves = D / 32;

// Eight consecutive values of a row.
__device__ __forceinline__ void load8(const bf16_t *p, float (&x)[8]) {
  const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
#pragma unroll
  for (int i = 0; i < 4; i++) {
    x[2 * i] = bf16_lo(w[i]);
    x[2 * i + 1] = bf16_hi(w[i]);
  }
}
__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; h++) {
    const float4_t w = __builtin_nontemporal_load(reinterpret_cast<const float4_t *>(p) + h);
#pragma unroll
    for (int i = 0; i < 4; i++) x[4 * h + i] = w[i];
  }
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; i++) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
  __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(p));
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; h++) {
    const float4_t w = {x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
    __builtin_nontemporal_store(w, reinterpret_cast<float4_t *>(p) + h);
  }
}

// A NaN becomes 0 and an infinity the limit: a group has no code for them, and
// a cache without them is one whose masked rows cannot reach a result.
__device__ __forceinline__ float storable(float x) {
  x = x != x ? 0.f : x;
  return fminf(fmaxf(x, -kQuantLimit), kQuantLimit);
}

// A lane's view of a tile: four chunks of eight consecutive values, K or V. The
// four lanes of a quad hold the neighbouring chunks, so that a group of 32 is
// one chunk index over the quad and a group of 64 two of them.
//   K: word w of the 16 bytes that an attention lane reads. D = 128: key n, d =
//      32 c + 8 g; D = 64: keys n (c < 2) and 16 + n, d = 32 (c & 1) + 8 g.
//   V, half h: keys k and k + 1 of the slots 2 r, 2 r + 1 of row g, d = 32 (2 h
//      + (c & 1)) + 8 q.
template <int D>
struct Lane {
  int key[4];  // of chunk c, within the tile
  int d[4];
  int g, r;    // V: the slots 8 g + 2 r and the one after
  __device__ __forceinline__ Lane(bool val, int part, int lane) {
    const int q = lane & 3, x = lane >> 2;
    g = val ? x >> 2 : q;
    r = x & 3;
#pragma unroll
    for (int c = 0; c < 4; c++) {
      if (val) {
        key[c] = 4 * g + 2 * (r & 1) + 16 * (r >> 1) + (c >> 1);
        d[c] = 32 * (2 * part + (c & 1)) + 8 * q;
      } else {
        key[c] = D == 128 ? 16 * part + x : 16 * (c >> 1) + x;
        d[c] = 32 * (D == 128 ? c : c & 1) + 8 * q;
      }
    }
  }
};

// The values of lanes 0, 1, 2 or 3 of each quad, or of the lane beside.
template <int CTRL>
__device__ __forceinline__ float quad(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
constexpr int kNext = 0xb1, kOther = 0x4e;  // lanes 1 0 3 2, lanes 2 3 0 1

__device__ __forceinline__ float lesser(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float greater(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Least and largest value of each chunk (a NaN stays one).
__device__ __forceinline__ void bounds(const float (&x)[4][8], float (&lo)[4], float (&hi)[4]) {
#pragma unroll
  for (int c = 0; c < 4; c++) {
    lo[c] = lesser(lesser(lesser(x[c][0], x[c][1]), lesser(x[c][2], x[c][3])),
                   lesser(lesser(x[c][4], x[c][5]), lesser(x[c][6], x[c][7])));
    hi[c] = greater(greater(greater(x[c][0], x[c][1]), greater(x[c][2], x[c][3])),
                    greater(greater(x[c][4], x[c][5]), greater(x[c][6], x[c][7])));
  }
}

// Writes a tile's rows [j0, j1), K by the first waves and V by the others. A
// workgroup per tile of 32 slots that a unit's new rows may touch; a lane
// quantises 32 values, and computes the scale and offset of one group for its
// quad.
// Bound by memory where rows are many: 4096 rows of 28 layers x 8 x 4 heads
// (1.88 GB in, 0.53 out) .
template <typename T, int D, int NG>
__global__ __launch_bounds__(kAppendWaves<D> *kWave) void quant_append_kernel(QuantAppendParams p, int tiles) {
  using Q = QTile<D, NG>;
  constexpr int PARTS = kAppendWaves<D> / 2, PAIR = Q::GROUP == 64;
  __shared__ uint32_t turn[PARTS][256];
  const int unit = blockIdx.x / tiles;  // (s * L + l) * Hkv + h
  const int lh = p.L * p.Hkv, s = unit / lh;
  const int from = p.src_index ? p.src_index[s] : s;
  if (from < 0 || from >= p.S_src) return;
  const int n = max(p.len[s], 0);
  const int count = p.count ? min(p.count[s], p.T) : p.T;
  const int tile = n / Q::KEYS + blockIdx.x % tiles;
  const int first = tile * Q::KEYS;
  const int j0 = max(n, first);
  const int j1 = (int)min((long)min((long)n + count, (long)p.cap), (long)first + Q::KEYS);
  if (j0 >= j1) return;
  const bool full = j1 - j0 == Q::KEYS;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const bool val = wave >= PARTS;
  const int part = val ? wave - PARTS : wave, q = lane & 3;
  const Lane<D> at(val, part, lane);
  const T *src = static_cast<const T *>(val ? p.v : p.k) + (((size_t)from * lh + unit % lh) * p.T + (first - n)) * (long)D;
  float x[4][8];
  bool live[4];
#pragma unroll
  for (int c = 0; c < 4; c++) {
    live[c] = first + at.key[c] >= j0 && first + at.key[c] < j1;
    if (live[c]) {
      load8(src + (long)at.key[c] * D + at.d[c], x[c]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) x[c][i] = 0.f;
    }
  }
  float lo[4], hi[4];
  bounds(x, lo, hi);
  bool plain = true;
#pragma unroll
  for (int c = 0; c < 4; c++) plain = plain && lo[c] >= -kQuantLimit && hi[c] <= kQuantLimit;
  if (__any(!plain)) {
#pragma unroll
    for (int c = 0; c < 4; c++)
#pragma unroll
      for (int i = 0; i < 8; i++) x[c][i] = storable(x[c][i]);
    bounds(x, lo, hi);
  }
  if (PAIR) {
#pragma unroll
    for (int c = 0; c < 4; c += 2) {
      lo[c] = lo[c + 1] = lesser(lo[c], lo[c + 1]);
      hi[c] = hi[c + 1] = greater(hi[c], hi[c + 1]);
    }
  }
  float mlo = 0.f, mhi = 0.f;  // of chunk q's group
#pragma unroll
  for (int c = 0; c < 4; c++) {
    lo[c] = lesser(lo[c], quad<kNext>(lo[c]));
    lo[c] = lesser(lo[c], quad<kOther>(lo[c]));
    hi[c] = greater(hi[c], quad<kNext>(hi[c]));
    hi[c] = greater(hi[c], quad<kOther>(hi[c]));
    mlo = q == c ? lo[c] : mlo;
    mhi = q == c ? hi[c] : mhi;
  }
  const f16_t zh = (f16_t)mlo;
  const float z = (float)zh, span = mhi - z;
  float step = span * (1.0f / 15.0f);
  asm volatile("" : "+v"(step));  // rounded to float32 here: no product straight into float16
  const f16_t sh = span > 0.f ? (f16_t)step : (f16_t)0.f;
  const float sc = (float)sh, inv = sc > 0.f ? 1.0f / sc : 0.f;
  const float zc[4] = {quad<0x00>(z), quad<0x55>(z), quad<0xaa>(z), quad<0xff>(z)};
  const float ic[4] = {quad<0x00>(inv), quad<0x55>(inv), quad<0xaa>(inv), quad<0xff>(inv)};
  uint32_t w[4];
#pragma unroll
  for (int c = 0; c < 4; c++) {
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
      // Adding 2^23 rounds to a whole number, ties to even, in the low bits.
      const float u = __builtin_amdgcn_fmed3f((x[c][i] - zc[c]) * ic[c], 0.f, 15.f);
      b[i] = __float_as_uint(u + 8388608.0f);
    }
    uint32_t t[4];
#pragma unroll
    for (int i = 0; i < 4; i++) t[i] = (b[2 * i + 1] << 4) | b[2 * i];  // the low byte: two codes
    w[c] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(t[3], t[2], 0x0c0c0400u),
                                 __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0400u), 0x05040100u);
  }

  char *out = static_cast<char *>(p.data) + ((size_t)unit * p.ntiles + tile) * Q::BYTES;
  // Scale and offset of chunk q's group, once per group.
  bool mine = false;
  int key = 0, d = 0;
#pragma unroll
  for (int c = 0; c < 4; c++)
    if (q == c) {
      mine = live[c] && !(PAIR && (c & 1));
      key = at.key[c];
      d = at.d[c] - 8 * q;
    }
  if (mine) {
    const int to = val ? Q::vparam(key, d / Q::GROUP) : Q::kparam(key, d / Q::GROUP);
    *reinterpret_cast<f16_t *>(out + (val ? Q::VS : Q::KS) + to) = sh;
    *reinterpret_cast<f16_t *>(out + (val ? Q::VZ : Q::KZ) + to) = zh;
  }
  if (!val) {
    char *to = out + part * 1024 + (at.g * 16 + (lane >> 2)) * 16;
    if (full) {
      *reinterpret_cast<u32x4 *>(to) = (u32x4){w[0], w[1], w[2], w[3]};
    } else {
#pragma unroll
      for (int c = 0; c < 4; c++)
        if (live[c]) reinterpret_cast<uint32_t *>(to)[c] = w[c];
    }
    return;
  }
  // V: byte m of the words (k, even i), (k, odd i), (k + 1, even), (k + 1, odd) is column 4 q + m.
  const uint32_t a0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), a1 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const uint32_t b0 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), b1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  const uint32_t col[4] = {__builtin_amdgcn_perm(b0, a0, 0x05040100u), __builtin_amdgcn_perm(b0, a0, 0x07060302u),
                           __builtin_amdgcn_perm(b1, a1, 0x05040100u), __builtin_amdgcn_perm(b1, a1, 0x07060302u)};
  char *to = out + Q::VC + part * 1024;
  if (full) {
    uint32_t *mat = turn[part];  // this wave's alone
#pragma unroll
    for (int m = 0; m < 4; m++) mat[(at.g * 16 + 4 * q + m) * 4 + at.r] = col[m];
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    __builtin_amdgcn_wave_barrier();
    reinterpret_cast<u32x4 *>(to)[lane] = reinterpret_cast<const u32x4 *>(mat)[lane];
  } else {
#pragma unroll
    for (int m = 0; m < 4; m++) {
      uint16_t *half = reinterpret_cast<uint16_t *>(to + (at.g * 16 + 4 * q + m) * 16 + at.r * 4);
      if (live[0]) half[0] = (uint16_t)col[m];
      if (live[2]) half[1] = (uint16_t)(col[m] >> 16);
    }
  }
}

// One workgroup per tile of a destination's live slots.
template <typename T, int D, int NG>
__global__ __launch_bounds__(kThreads) void quant_read_kernel(QuantReadParams p, int tiles) {
  using Q = QTile<D, NG>;
  constexpr int CH = D / 8, LANES = Q::GROUP / 8;
  const int unit = blockIdx.x / tiles, tile = blockIdx.x % tiles;
  const int lh = p.L * p.Hkv, s = unit / lh;
  const int from = p.src_index ? p.src_index[s] : s;
  if (from < 0 || from >= p.S_src) return;
  const int j0 = tile * Q::KEYS;
  const int j1 = min(min(p.len[s], min(p.cap, p.cap_dst)), j0 + Q::KEYS);
  if (j0 >= j1) return;
  const char *in = static_cast<const char *>(p.data) + (((size_t)from * lh + unit % lh) * p.ntiles + tile) * Q::BYTES;
  const size_t row0 = (size_t)unit * p.cap_dst + j0;
  const int items = (j1 - j0) * CH;
  for (int it = threadIdx.x; it < 2 * items; it += kThreads) {
    const bool val = it >= items;
    const int e = val ? it - items : it;
    const int key = e / CH, c = e % CH;
    const int at = val ? Q::vparam(key, c / LANES) : Q::kparam(key, c / LANES);
    const float sc = f16_at(in + (val ? Q::VS : Q::KS) + at), z = f16_at(in + (val ? Q::VZ : Q::KZ) + at);
    uint32_t w = 0;
    if (!val) {
      w = *reinterpret_cast<const uint32_t *>(in + Q::kword(key, c));
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++) w |= (uint32_t)(uint8_t)in[Q::vbyte(key, c * 4 + i)] << (8 * i);
    }
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = fmaf(sc, (float)((w >> (4 * i)) & 15u), z);
    store8(static_cast<T *>(val ? p.v : p.k) + (row0 + key) * D + c * 8, x);
  }
}

template <typename T, int D, int NG>
void append_launch(const QuantAppendParams &p, hipStream_t stream) {
  // T rows touch at most this many tiles of 32, whatever the first one's place.
  const int tiles = (p.T - 1 + kQuantTile - 1) / kQuantTile + 1;
  const int units = p.S * p.L * p.Hkv;
  hipLaunchKernelGGL((quant_append_kernel<T, D, NG>), dim3((uint32_t)units * (uint32_t)tiles),
                     dim3(kAppendWaves<D> * kWave), 0, stream, p, tiles);
}

template <typename T, int D, int NG>
void read_launch(const QuantReadParams &p, hipStream_t stream) {
  const int tiles = (p.cap < p.cap_dst ? p.cap : p.cap_dst) / kQuantTile + 1;
  const int units = p.S * p.L * p.Hkv;
  hipLaunchKernelGGL((quant_read_kernel<T, D, NG>), dim3((uint32_t)units * (uint32_t)tiles), dim3(kThreads), 0, stream,
                     p, tiles);
}

}  // namespace

#define KVR_QUANT_DISPATCH(FN, p, f32, D, group, stream)             \
  do {                                                               \
    if (D == 128 && group == 32) {                                   \
      if (f32) FN<float, 128, 4>(p, stream); else FN<bf16_t, 128, 4>(p, stream); \
    } else if (D == 128) {                                           \
      if (f32) FN<float, 128, 2>(p, stream); else FN<bf16_t, 128, 2>(p, stream); \
    } else if (group == 32) {                                        \
      if (f32) FN<float, 64, 2>(p, stream); else FN<bf16_t, 64, 2>(p, stream);   \
    } else {                                                         \
      if (f32) FN<float, 64, 1>(p, stream); else FN<bf16_t, 64, 1>(p, stream);   \
    }                                                                \
  } while (0)

hipError_t launch_quant_append(const QuantAppendParams &p, hipStream_t stream) {
  KVR_QUANT_DISPATCH(append_launch, p, p.dtype == 0, p.D, p.group, stream);
  return hipGetLastError();
}

hipError_t launch_quant_read(const QuantReadParams &p, hipStream_t stream) {
  KVR_QUANT_DISPATCH(read_launch, p, p.dtype == 0, p.D, p.group, stream);
  return hipGetLastError();
}

}  // namespace kvr
