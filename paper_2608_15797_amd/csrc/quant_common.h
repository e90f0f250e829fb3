// The 4-bit cache: its layout, shared by the kernels that write, read and
// attend over it.
//
// A row of D values is cut into NG = D / group groups of 32 or 64. A group
// with offset z and scale s (float16 each) and codes n (0 .. 15) stands for
// z + s n (include/kvr.h has the steps that find them). The slots of a
// (sequence, layer, KV head) unit lie in tiles of 32, one contiguous block of
// tile_bytes each, so that a unit is one stream of memory: K codes, V codes,
// K scales, K offsets, V scales, V offsets.
//
// The order inside a tile is the operand order of the attention's matrix
// products (attention of a tile: quant_attn.hip), in which a lane (n = lane &
// 15, g = lane >> 4) holds 16 consecutive bytes per 1 KiB load:
//   K codes: the A operand of a 16x16x32 product holds keys n and d = 32 i +
//     8 g + 0..7; the eight codes of (key, i, g) are one word, code e at bits
//     4 e. D = 128: a lane's 16 bytes are its words i = 0..3 of one key, 1 KiB
//     per 16 keys. D = 64: the words i = 0, 1 of key n, then of key 16 + n.
//   V codes: the B operand holds keys in the order of slot(key) = 8 g + e and
//     one column n of instance b, where instances 2 i and 2 i + 1 have d = 32 i
//     + 2 n and the d after it. The codes of (key, n, instances 4 h .. 4 h + 3)
//     are one 16-bit unit, and a lane's 16 bytes of half h its 8 keys' units.
//   K scales, K offsets: [32 keys][NG]; V scales, V offsets: [NG][32 slots].
// Every byte belongs to one row, so rows are written without reading.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvr_device.h"
#include "kvr_internal.h"

namespace kvr {
namespace {

typedef _Float16 f16_t;

template <int D, int NG>
struct QTile {
  static constexpr int KEYS = kQuantTile;
  static constexpr int VC = 16 * D;                 // V codes
  static constexpr int KS = 32 * D;                 // K scales
  static constexpr int KZ = KS + 64 * NG;           // K offsets
  static constexpr int VS = KZ + 64 * NG;           // V scales
  static constexpr int VZ = VS + 64 * NG;           // V offsets
  static constexpr int BYTES = VZ + 64 * NG;
  static constexpr int GROUP = D / NG;

  // Place of a key in the value operand's order.
  __device__ static __forceinline__ int slot(int key) {
    return 8 * ((key >> 2) & 3) + 4 * (key >> 4) + (key & 3);
  }
  // The word of the K codes of d = 8 c .. 8 c + 7.
  __device__ static __forceinline__ int kword(int key, int c) {
    const int i = c >> 2, g = c & 3, n = key & 15, t = key >> 4;
    return D == 128 ? t * 1024 + (g * 16 + n) * 16 + i * 4 : (g * 16 + n) * 16 + t * 8 + i * 4;
  }
  // The byte of the V codes of d = 2 x (low bits) and 2 x + 1.
  __device__ static __forceinline__ int vbyte(int key, int x) {
    const int i = x >> 4, n = x & 15, s = slot(key), g = s >> 3, e = s & 7;
    return VC + (i >> 1) * 1024 + (g * 16 + n) * 16 + e * 2 + (i & 1);
  }
  __device__ static __forceinline__ int kparam(int key, int grp) { return (key * NG + grp) * 2; }
  __device__ static __forceinline__ int vparam(int key, int grp) { return (grp * 32 + slot(key)) * 2; }
};

__device__ __forceinline__ float f16_at(const char *p) { return (float)*reinterpret_cast<const f16_t *>(p); }

}  // namespace
}  // namespace kvr
