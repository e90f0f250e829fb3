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
constexpr int kMaxG = 16;

__device__ __forceinline__ float as_f32(bf16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ float as_f32(float x) { return x; }
__device__ __forceinline__ void put(bf16_t *p, float x) { *p = (bf16_t)(pack_bf16x2(x, x) & 0xffffu); }
__device__ __forceinline__ void put(float *p, float x) { *p = x; }

// Own row j of a unit: the new rows come from the caller's arrays (another
// workgroup may be storing them), the others from the cache.
template <typename T>
struct OwnRows {
  const T *cache, *fresh;
  int first;  // first new row; none where fresh is NULL
  __device__ __forceinline__ const T *row(int j, int D) const {
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

// Vector kernel, the float32 path: one workgroup per (sequence, layer, KV
// head, query token). Chunks of one key per thread: the thread's key is
// expanded and multiplied with the G query rows (in LDS), the probabilities go
// to LDS, and each thread sums one column d over every KG-th key of the chunk.
template <typename T, int D, int NG>
__global__ __launch_bounds__(kThreads) void quant_attn_vector(QuantAttnParams p) {
  using Q = QTile<D, NG>;
  constexpr int KG = kThreads / D, NW = kThreads / kWave;
  __shared__ float qs[kMaxG][D];
  __shared__ float prob[kMaxG][kThreads];
  __shared__ float red[kMaxG][NW];
  const int t = blockIdx.x % p.nq, unit = blockIdx.x / p.nq;
  const int lh = p.L * p.Hkv, s = unit / lh, h = unit % p.Hkv, l = unit / p.Hkv % p.L;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, G = p.G;
  const int c = s / p.C, n = ctx_len(p, c), u = own_len(p, s);
  const long seen = (long)n + u - (p.nq - 1 - t);  // keys query t attends to
  if (t == 0 && p.ok) store_new<T, D, kThreads>(p, unit, s, u);
  const size_t qrow = (((size_t)s * p.L + l) * p.Hq + (size_t)h * G) * p.nq + t;  // + g nq
  for (int e = tid; e < G * D; e += kThreads)
    qs[e / D][e % D] = as_f32(static_cast<const T *>(p.q)[(qrow + (size_t)(e / D) * p.nq) * D + e % D]);
  __syncthreads();

  const char *ctx = static_cast<const char *>(p.data) + ((size_t)c * lh + unit % lh) * p.ntiles * Q::BYTES;
  const size_t own0 = (size_t)unit * p.ocap * D, new0 = (size_t)unit * p.nq * D;
  const T *fk = static_cast<const T *>(p.k_new), *fv = static_cast<const T *>(p.v_new);
  const OwnRows<T> K{static_cast<const T *>(p.ok) + own0, fk ? fk + new0 : nullptr, u - p.nq};
  const OwnRows<T> V{static_cast<const T *>(p.ov) + own0, fv ? fv + new0 : nullptr, u - p.nq};
  float m[kMaxG], den[kMaxG], o[kMaxG];
#pragma unroll
  for (int g = 0; g < kMaxG; g++) {
    m[g] = kNegInf;
    den[g] = o[g] = 0.f;
  }
  const int d = tid % D, kg = tid / D;
  for (long c0 = 0; c0 < seen; c0 += kThreads) {
    const long key = c0 + tid;
    float x[kMaxG];
#pragma unroll
    for (int g = 0; g < kMaxG; g++) x[g] = 0.f;
    if (key < seen) {
      const bool held = key < n;
      const char *tile = ctx + (held ? key / Q::KEYS : 0) * Q::BYTES;
      const int kt = (int)(key % Q::KEYS);
      const T *krow = held ? nullptr : K.row((int)(key - n), D);
      for (int ch = 0; ch < D / 8; ch++) {
        float k8[8];
        if (held) {
          const uint32_t w = *reinterpret_cast<const uint32_t *>(tile + Q::kword(kt, ch));
          const int at = Q::kparam(kt, ch * 8 / Q::GROUP);
          const float sc = f16_at(tile + Q::KS + at), z = f16_at(tile + Q::KZ + at);
#pragma unroll
          for (int i = 0; i < 8; i++) k8[i] = fmaf(sc, (float)((w >> (4 * i)) & 15u), z);
        } else {
#pragma unroll
          for (int i = 0; i < 8; i++) k8[i] = as_f32(krow[ch * 8 + i]);
        }
#pragma unroll
        for (int g = 0; g < kMaxG; g++)
          if (g < G) {
#pragma unroll
            for (int i = 0; i < 8; i++) x[g] = fmaf(qs[g][ch * 8 + i], k8[i], x[g]);
          }
      }
    }
#pragma unroll
    for (int g = 0; g < kMaxG; g++)
      if (g < G) {
        x[g] = key < seen ? x[g] * p.scale * kLog2e : kNegInf;
        const float wm = wave_max(x[g]);
        if (lane == 0) red[g][wave] = wm;
      }
    __syncthreads();
    float keep[kMaxG];
#pragma unroll
    for (int g = 0; g < kMaxG; g++)
      if (g < G) {
        float mn = m[g];
#pragma unroll
        for (int w = 0; w < NW; w++) mn = fmaxf(mn, red[g][w]);
        // Logits of -inf alone leave the reference at -inf: as softmax has it, NaN.
        keep[g] = m[g] == kNegInf ? 0.f : exp2f(m[g] - mn);
        m[g] = mn;
        prob[g][tid] = key < seen ? exp2f(x[g] - mn) : 0.f;
      }
    __syncthreads();
    const int keys = (int)min((long)kThreads, seen - c0);
#pragma unroll
    for (int g = 0; g < kMaxG; g++)
      if (g < G) {
        o[g] *= keep[g];
        den[g] *= keep[g];
      }
    for (int j = kg; j < keys; j += KG) {
      const long kj = c0 + j;
      float v;
      if (kj < n) {
        const char *tile = ctx + kj / Q::KEYS * Q::BYTES;
        const int kt = (int)(kj % Q::KEYS), at = Q::vparam(kt, d / Q::GROUP);
        const uint32_t b = (uint8_t)tile[Q::vbyte(kt, d / 2)];
        v = fmaf(f16_at(tile + Q::VS + at), (float)(d & 1 ? b >> 4 : b & 15u), f16_at(tile + Q::VZ + at));
      } else {
        v = as_f32(V.row((int)(kj - n), D)[d]);
      }
#pragma unroll
      for (int g = 0; g < kMaxG; g++)
        if (g < G) {
          const float w = prob[g][j];
          o[g] = fmaf(w, v, o[g]);
          den[g] += w;
        }
    }
    __syncthreads();
  }
  // The KG partial sums of a column.
  float *part = &prob[0][0];
#pragma unroll
  for (int g = 0; g < kMaxG; g++)
    if (g < G) {
      part[tid] = o[g];
      part[kThreads + tid] = den[g];
      __syncthreads();
      if (kg == 0) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int k = 0; k < KG; k++) {
          a += part[k * D + d];
          b += part[kThreads + k * D + d];
        }
        put(static_cast<T *>(p.out) + (qrow + (size_t)g * p.nq) * D + d, seen > 0 ? a / b : 0.f);
      }
      __syncthreads();
    }
}

template <typename T, int D, int NG>
void launch_vector(const QuantAttnParams &p, hipStream_t stream) {
  const dim3 grid((uint32_t)p.S * p.L * p.Hkv * p.nq);
  hipLaunchKernelGGL((quant_attn_vector<T, D, NG>), grid, dim3(kThreads), 0, stream, p);
}

template <typename T>
void launch_type(const QuantAttnParams &p, hipStream_t stream) {
  if (p.D == 128) {
    if (p.group == 32) launch_vector<T, 128, 4>(p, stream);
    else launch_vector<T, 128, 2>(p, stream);
  } else {
    if (p.group == 32) launch_vector<T, 64, 2>(p, stream);
    else launch_vector<T, 64, 1>(p, stream);
  }
}

}  // namespace

size_t quant_attn_workspace_bytes(const QuantAttnParams &) { return 0; }

hipError_t launch_quant_attn(const QuantAttnParams &p, hipStream_t stream) {
  if (p.dtype == 0) launch_type<float>(p, stream);
  else launch_type<bf16_t>(p, stream);
  return hipGetLastError();
}

}  // namespace kvr
