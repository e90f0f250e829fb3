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

// Waves of a workgroup: one per KiB of a tile's codes, K and V.
template <int D>
constexpr int kTileWaves = D / 32;

// New rows per unit up to which a thread takes eight values of a row instead of
// a workgroup a tile. Lone tokens of 1792 units: 3.0 us against 6.9, eight 5.5
// against 11.8; 16 rows of 7168 units: 31 against 43, 32 rows 58 against 57.
constexpr int kFewRows = 16, kRowThreads = 256;

// Eight consecutive values of a row, as loaded.
template <typename T>
struct Raw8;
template <>
struct Raw8<bf16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const bf16_t *p) {
    w = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    }
  }
};
template <>
struct Raw8<float> {
  float4_t w[2];
  __device__ __forceinline__ void load(const float *p) {
#pragma unroll
    for (int h = 0; h < 2; h++) w[h] = __builtin_nontemporal_load(reinterpret_cast<const float4_t *>(p) + h);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = w[i >> 2][i & 3];
  }
};

// Read-back values, past the caches: 28 x 2 x 64 units of 150 rows (275 MB of
// values) take 46 us one after another against 64 with ordinary stores; where
// the caches are full of another kernel's writes, 75 against 73.
__device__ __forceinline__ void store16(bf16_t *p, const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; i++) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
  __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(p));
}
__device__ __forceinline__ void store16(float *p, const float (&x)[4]) {
  const float4_t w = {x[0], x[1], x[2], x[3]};
  __builtin_nontemporal_store(w, reinterpret_cast<float4_t *>(p));
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

// A wave's own LDS, between its lanes' writes and reads.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Word c of the result: byte c of each of the four words.
__device__ __forceinline__ u32x4 transpose4(const uint32_t (&w)[4]) {
  const uint32_t a0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), a1 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const uint32_t b0 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), b1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  return (u32x4){__builtin_amdgcn_perm(b0, a0, 0x05040100u), __builtin_amdgcn_perm(b0, a0, 0x07060302u),
                 __builtin_amdgcn_perm(b1, a1, 0x05040100u), __builtin_amdgcn_perm(b1, a1, 0x07060302u)};
}

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

// Scale and offset of a group with these bounds.
struct Group {
  f16_t sh, zh;
  float z, inv;
  __device__ __forceinline__ Group(float lo, float hi) {
    zh = (f16_t)lo;
    z = (float)zh;
    const float span = hi - z;
    float step = span * (1.0f / 15.0f);
    asm volatile("" : "+v"(step));  // rounded to float32 here: no product straight into float16
    sh = span > 0.f ? (f16_t)step : (f16_t)0.f;
    const float sc = (float)sh;
    inv = sc > 0.f ? 1.0f / sc : 0.f;
  }
};

// The codes of eight values, the first in the low bits.
__device__ __forceinline__ uint32_t codes(const float (&x)[8], float z, float inv) {
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; i++) {
    // Adding 2^23 rounds to a whole number, ties to even, in the low bits.
    const float u = __builtin_amdgcn_fmed3f((x[i] - z) * inv, 0.f, 15.f);
    b[i] = __float_as_uint(u + 8388608.0f);
  }
  uint32_t t[4];
#pragma unroll
  for (int i = 0; i < 4; i++) t[i] = (b[2 * i + 1] << 4) | b[2 * i];  // the low byte: two codes
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(t[3], t[2], 0x0c0c0400u),
                               __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0400u), 0x05040100u);
}

// Writes a tile's rows [j0, j1), K by the first waves and V by the others. A
// workgroup per tile of 32 slots that a unit's new rows may touch; a lane
// quantises 32 values, and computes the scale and offset of one group for its
// quad.
// Bound by memory where rows are many: 4096 rows of 8 x 28 x 4 units (1.88 GB in,
// 0.53 out) take 434 us, 5.5 TB/s; a thread per eight values, 637 us.
template <typename T, int D, int NG>
__global__ __launch_bounds__(kTileWaves<D> *kWave) void quant_append_kernel(QuantAppendParams p, int tiles) {
  using Q = QTile<D, NG>;
  constexpr int PARTS = kTileWaves<D> / 2, PAIR = Q::GROUP == 64;
  __shared__ __align__(16) uint32_t turn[PARTS][256];
  const int unit = blockIdx.x / tiles;  // (s * L + l) * Hkv + h
  const int lh = p.L * p.Hkv, s = unit / lh;
  const int from = p.src_index ? p.src_index[s] : s;
  if (from < 0 || from >= p.S_src) return;
  const int n = max(p.len[s], 0);
  const int count = p.count ? min(p.count[s], p.T) : p.T;
  const int end = (int)min((long)n + count, (long)p.cap);  // the slots [n, end)
  const int tile = n / Q::KEYS + blockIdx.x % tiles, first = tile * Q::KEYS;
  if (max(n, first) >= end) return;
  const bool full = first >= n && first + Q::KEYS <= end;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const bool val = wave >= PARTS;
  const int part = val ? wave - PARTS : wave, q = lane & 3;
  const Lane<D> at(val, part, lane);
  // Row j of the slots; rows before the first new one are not read.
  const T *src = static_cast<const T *>(val ? p.v : p.k) + ((long)((size_t)from * lh + unit % lh) * p.T - n) * (long)D;
  Raw8<T> raw[4];
  bool live[4];
#pragma unroll
  for (int c = 0; c < 4; c++) {
    const int j = first + at.key[c];
    live[c] = j >= n && j < end;
    raw[c] = Raw8<T>{};
    if (live[c]) raw[c].load(src + (long)j * D + at.d[c]);
  }
  float x[4][8];
#pragma unroll
  for (int c = 0; c < 4; c++) raw[c].get(x[c]);
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
  const Group grp(mlo, mhi);
  const f16_t sh = grp.sh, zh = grp.zh;
  const float zc[4] = {quad<0x00>(grp.z), quad<0x55>(grp.z), quad<0xaa>(grp.z), quad<0xff>(grp.z)};
  const float ic[4] = {quad<0x00>(grp.inv), quad<0x55>(grp.inv), quad<0xaa>(grp.inv), quad<0xff>(grp.inv)};
  uint32_t w[4];
#pragma unroll
  for (int c = 0; c < 4; c++) w[c] = codes(x[c], zc[c], ic[c]);

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
  const u32x4 col = transpose4(w);
  char *to = out + Q::VC + part * 1024;
  if (full) {
    uint32_t *mat = turn[part];  // this wave's alone
#pragma unroll
    for (int m = 0; m < 4; m++) mat[(at.g * 16 + 4 * q + m) * 4 + at.r] = col[m];
    wave_sync();
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

// The same for few rows per unit: a thread per eight values, the rows of the
// units one after another, so that no lane waits for rows that are not there.
template <typename T, int D, int NG>
__global__ __launch_bounds__(kRowThreads) void quant_append_rows(QuantAppendParams p) {
  using Q = QTile<D, NG>;
  constexpr int CH = D / 8, LANES = Q::GROUP / 8;
  const size_t it = (size_t)blockIdx.x * kRowThreads + threadIdx.x;
  const int c = (int)(it % CH);
  const bool val = it / CH % 2;
  const size_t row = it / (2 * CH);  // ((s * L + l) * Hkv + h) * T + t
  const int lh = p.L * p.Hkv;
  const int unit = (int)(row / p.T), t = (int)(row % p.T), s = unit / lh;
  if (s >= p.S) return;  // whole groups
  const int from = p.src_index ? p.src_index[s] : s;
  const int n = max(p.len[s], 0);
  const int count = p.count ? min(p.count[s], p.T) : p.T;
  if (from < 0 || from >= p.S_src || t >= count || (long)n + t >= p.cap) return;
  const T *src = static_cast<const T *>(val ? p.v : p.k) + (((size_t)from * lh + unit % lh) * p.T + t) * D + c * 8;
  Raw8<T> raw;
  raw.load(src);
  float x[8];
  raw.get(x);
  float lo = 0.f, hi = 0.f;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    x[i] = storable(x[i]);
    lo = i ? lesser(lo, x[i]) : x[i];
    hi = i ? greater(hi, x[i]) : x[i];
  }
#pragma unroll
  for (int m = 1; m < LANES; m <<= 1) {
    lo = lesser(lo, shfl_xor(lo, m));
    hi = greater(hi, shfl_xor(hi, m));
  }
  const Group grp(lo, hi);
  const uint32_t w = codes(x, grp.z, grp.inv);
  const int key = (n + t) % Q::KEYS;
  char *out = static_cast<char *>(p.data) + ((size_t)unit * p.ntiles + (n + t) / Q::KEYS) * Q::BYTES;
  if (!val) {
    *reinterpret_cast<uint32_t *>(out + Q::kword(key, c)) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) out[Q::vbyte(key, c * 4 + i)] = (char)(w >> (8 * i));
  }
  if (c % LANES == 0) {
    const int at = val ? Q::vparam(key, c / LANES) : Q::kparam(key, c / LANES);
    *reinterpret_cast<f16_t *>(out + (val ? Q::VS : Q::KS) + at) = grp.sh;
    *reinterpret_cast<f16_t *>(out + (val ? Q::VZ : Q::KZ) + at) = grp.zh;
  }
}

// A workgroup per tile of a destination's live slots. A wave loads a KiB of
// codes, in the append's lanes, and the scales and offsets of its quads'
// groups; through LDS a lane gets the words, each with its group's scale and
// offset, of four chunks such that a store covers whole lines (64-byte pieces
// of 16 rows, as the codes lie, take 509 us for 4096 rows of 28 x 8 x 4 heads).
template <typename T, int D, int NG>
__global__ __launch_bounds__(kTileWaves<D> *kWave) void quant_read_kernel(QuantReadParams p, int tiles) {
  using Q = QTile<D, NG>;
  constexpr int PARTS = kTileWaves<D> / 2, LANES = Q::GROUP / 8;
  __shared__ __align__(16) uint32_t turn[PARTS][256];
  __shared__ uint32_t words[2 * PARTS][256 + 64];
  __shared__ uint32_t params[2 * PARTS][256 / LANES];
  const int unit = blockIdx.x / tiles, tile = blockIdx.x % tiles;
  const int lh = p.L * p.Hkv, s = unit / lh;
  const int from = p.src_index ? p.src_index[s] : s;
  if (from < 0 || from >= p.S_src) return;
  const int end = min(p.len[s], min(p.cap, p.cap_dst));
  if (tile * Q::KEYS >= end) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, q = lane & 3;
  const bool val = wave >= PARTS;
  const int part = val ? wave - PARTS : wave;
  const Lane<D> at(val, part, lane);
  // The wave's keys and d: from key0 and d0, chunks of a key side by side.
  const int log_cpr = D == 128 && !val ? 4 : 3, key0 = val || D == 64 ? 0 : 16 * part, d0 = val ? 64 * part : 0;
  const char *in = static_cast<const char *>(p.data) + (((size_t)from * lh + unit % lh) * p.ntiles + tile) * Q::BYTES;
  T *out = static_cast<T *>(val ? p.v : p.k) + (size_t)unit * p.cap_dst * D;
  int key = 0, d = 0;  // of chunk q
#pragma unroll
  for (int c = 0; c < 4; c++)
    if (q == c) {
      key = at.key[c];
      d = at.d[c] - 8 * q;
    }
  const int param = val ? Q::VS + Q::vparam(key, d / Q::GROUP) : Q::KS + Q::kparam(key, d / Q::GROUP);
  const int code = (val ? Q::VC : 0) + part * 1024 + (val ? lane * 16 : (at.g * 16 + (lane >> 2)) * 16);
  static_assert(Q::KZ - Q::KS == Q::VZ - Q::VS, "offsets after the scales");
  u32x4 c4 = *reinterpret_cast<const u32x4 *>(in + code);
  const uint32_t sh = *reinterpret_cast<const uint16_t *>(in + param);
  const uint32_t zh = *reinterpret_cast<const uint16_t *>(in + param + (Q::KZ - Q::KS));
  // Chunk q's group, by the chunk's place.
  params[wave][(((key - key0) << log_cpr) + (d - d0) / 8) / LANES] = sh | (zh << 16);
  if (val) {
    uint32_t *mat = turn[part];
    reinterpret_cast<u32x4 *>(mat)[lane] = c4;
    wave_sync();
    uint32_t col[4];
#pragma unroll
    for (int m = 0; m < 4; m++) col[m] = mat[(at.g * 16 + 4 * q + m) * 4 + at.r];
    c4 = transpose4(col);
  }
#pragma unroll
  for (int c = 0; c < 4; c++) {
    const int e = ((at.key[c] - key0) << log_cpr) + (at.d[c] - d0) / 8;
    words[wave][e + (e >> 4) * 4] = c4[c];  // four words of padding in 16 keep the banks apart
  }
  wave_sync();
  // 16 bytes of values per lane and store: a word's eight codes, float32: half of them.
  constexpr int VALS = 16 / sizeof(T), HALVES = 8 / VALS;
#pragma unroll
  for (int c = 0; c < 4 * HALVES; c++) {
    const int e = (c * kWave + lane) / HALVES, half = (c * kWave + lane) % HALVES;
    const uint32_t word = words[wave][e + (e >> 4) * 4] >> (half * 16), pz = params[wave][e / LANES];
    const float sc = (float)__builtin_bit_cast(f16_t, (uint16_t)pz);
    const float z = (float)__builtin_bit_cast(f16_t, (uint16_t)(pz >> 16));
    const uint32_t even = word & 0x0f0f0f0fu, odd = (word >> 4) & 0x0f0f0f0fu;
    float x[VALS];
#pragma unroll
    for (int m = 0; m < VALS / 2; m++) {
      x[2 * m] = fmaf(sc, (float)((even >> (8 * m)) & 0xffu), z);
      x[2 * m + 1] = fmaf(sc, (float)((odd >> (8 * m)) & 0xffu), z);
    }
    const int j = tile * Q::KEYS + key0 + (e >> log_cpr);
    if (j < end) store16(out + (size_t)j * D + d0 + (e & ((1 << log_cpr) - 1)) * 8 + half * VALS, x);
  }
}

template <typename T, int D, int NG>
void append_launch(const QuantAppendParams &p, hipStream_t stream) {
  if (p.T <= kFewRows) {
    const size_t threads = (size_t)p.S * p.L * p.Hkv * p.T * 2 * (D / 8);
    hipLaunchKernelGGL((quant_append_rows<T, D, NG>), dim3((uint32_t)((threads + kRowThreads - 1) / kRowThreads)),
                       dim3(kRowThreads), 0, stream, p);
    return;
  }
  // T rows touch at most this many tiles of 32, whatever the first one's place.
  const int tiles = (p.T - 1 + kQuantTile - 1) / kQuantTile + 1;
  const uint32_t units = (uint32_t)p.S * p.L * p.Hkv;
  hipLaunchKernelGGL((quant_append_kernel<T, D, NG>), dim3(units * tiles), dim3(kTileWaves<D> * kWave), 0, stream, p,
                     tiles);
}

template <typename T, int D, int NG>
void read_launch(const QuantReadParams &p, hipStream_t stream) {
  const int tiles = ((p.cap < p.cap_dst ? p.cap : p.cap_dst) - 1) / kQuantTile + 1;
  const uint32_t units = (uint32_t)p.S * p.L * p.Hkv;
  hipLaunchKernelGGL((quant_read_kernel<T, D, NG>), dim3(units * tiles), dim3(kTileWaves<D> * kWave), 0, stream, p,
                     tiles);
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
