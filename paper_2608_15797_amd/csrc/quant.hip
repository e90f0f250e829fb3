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

// One workgroup per tile of 32 slots that a unit's new rows may touch. A
// thread takes 8 consecutive values; the LANES = group / 8 lanes of a group
// find its least and largest value together.
template <typename T, int D, int NG>
__global__ __launch_bounds__(kThreads) void quant_append_kernel(QuantAppendParams p, int tiles) {
  using Q = QTile<D, NG>;
  constexpr int CH = D / 8, LANES = Q::GROUP / 8;
  const int unit = blockIdx.x / tiles;  // (s * L + l) * Hkv + h
  const int lh = p.L * p.Hkv, s = unit / lh;
  const int from = p.src_index ? p.src_index[s] : s;
  if (from < 0 || from >= p.S_src) return;
  const int n = max(p.len[s], 0);
  const int count = p.count ? min(p.count[s], p.T) : p.T;
  const int tile = n / Q::KEYS + blockIdx.x % tiles;
  const int j0 = max(n, tile * Q::KEYS);
  const int j1 = (int)min((long)min((long)n + count, (long)p.cap), (long)(tile + 1) * Q::KEYS);
  if (j0 >= j1) return;
  const size_t row0 = ((size_t)from * lh + unit % lh) * p.T;
  char *out = static_cast<char *>(p.data) + ((size_t)unit * p.ntiles + tile) * Q::BYTES;
  const int items = (j1 - j0) * CH;  // of K, then as many of V
  for (int it = threadIdx.x; it < 2 * items; it += kThreads) {
    const bool val = it >= items;
    const int e = val ? it - items : it;
    const int j = j0 + e / CH, c = e % CH, key = j - tile * Q::KEYS;
    const T *src = static_cast<const T *>(val ? p.v : p.k) + (row0 + (j - n)) * D + c * 8;
    float x[8];
    load8(src, x);
    float lo = 0.f, hi = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      x[i] = storable(x[i]);
      lo = i ? fminf(lo, x[i]) : x[i];
      hi = i ? fmaxf(hi, x[i]) : x[i];
    }
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) {
      lo = fminf(lo, shfl_xor(lo, m));
      hi = fmaxf(hi, shfl_xor(hi, m));
    }
    const f16_t zh = (f16_t)lo;
    const float z = (float)zh, span = hi - z;
    float step = span * (1.0f / 15.0f);
    asm volatile("" : "+v"(step));  // rounded to float32 here: no product straight into float16
    const f16_t sh = span > 0.f ? (f16_t)step : (f16_t)0.f;
    const float sc = (float)sh, inv = sc > 0.f ? 1.0f / sc : 0.f;
    uint32_t n8[8];
#pragma unroll
    for (int i = 0; i < 8; i++) n8[i] = (uint32_t)fminf(fmaxf(rintf((x[i] - z) * inv), 0.f), 15.f);
    if (!val) {
      uint32_t w = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) w |= n8[i] << (4 * i);
      *reinterpret_cast<uint32_t *>(out + Q::kword(key, c)) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++)
        out[Q::vbyte(key, c * 4 + i)] = (char)(n8[2 * i] | (n8[2 * i + 1] << 4));
    }
    if (c % LANES == 0) {
      const int at = val ? Q::vparam(key, c / LANES) : Q::kparam(key, c / LANES);
      *reinterpret_cast<f16_t *>(out + (val ? Q::VS : Q::KS) + at) = sh;
      *reinterpret_cast<f16_t *>(out + (val ? Q::VZ : Q::KZ) + at) = zh;
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
  hipLaunchKernelGGL((quant_append_kernel<T, D, NG>), dim3((uint32_t)units * (uint32_t)tiles), dim3(kThreads), 0,
                     stream, p, tiles);
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
