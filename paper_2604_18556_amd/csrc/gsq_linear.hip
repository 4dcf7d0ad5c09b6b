// The packed layer in use: its bytes laid out for the matrix instructions, and the product of grouped
// rows with it.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gsq_product_any.hpp"

namespace gsq {
namespace {

// Where code j (0 .. 31) of a lane is kept in its `bits` words.  Four codes that are neighbours lie at
// the same place in the four bytes of a word, so that one mask takes out four byte-wide indices:
//   1 bit:  bit 8 (j % 4) + j / 4
//   2 bits: word j / 16, bits 8 (j % 4) + 2 (j / 4 % 4)
//   3 bits: the lower two as for 2 bits, the third in word 2 as for 1 bit
//   4 bits: word j / 8, bits 8 (j % 4) + 4 (j / 4 % 2)
__host__ __device__ __forceinline__ void place_code(uint32_t* words, int bits, int j, uint32_t code) {
  const int byte = 8 * (j & 3), quad = j >> 2;
  if (bits == 1) {
    words[0] |= code << (byte + quad);
  } else if (bits == 4) {
    words[quad >> 1] |= code << (byte + 4 * (quad & 1));
  } else {
    words[quad >> 2] |= (code & 3) << (byte + 2 * (quad & 3));
    if (bits == 3) words[2] |= (code >> 2) << (byte + quad);
  }
}
__device__ __forceinline__ uint32_t code_at(const uint32_t* words, int bits, int j) {
  const int byte = 8 * (j & 3), quad = j >> 2;
  if (bits == 1) return words[0] >> (byte + quad) & 1;
  if (bits == 4) return words[quad >> 1] >> (byte + 4 * (quad & 1)) & 15;
  const uint32_t low = words[quad >> 2] >> (byte + 2 * (quad & 3)) & 3;
  return bits == 2 ? low : low | (words[2] >> (byte + quad) & 1) << 2;
}

// A field of at most 8 bits from little-endian bits; the next byte is read only if the field reaches it.
__device__ __forceinline__ uint32_t bit_field(const uint8_t* p, int64_t bit, int width) {
  const int64_t at = bit >> 3;
  const int shift = (int)(bit & 7);
  uint32_t v = p[at] >> shift;
  if (shift + width > 8) v |= (uint32_t)p[at + 1] << (8 - shift);
  return v & ((1u << width) - 1);
}

// Code of weight w (its index over all layers) in the packed bytes.
__device__ __forceinline__ uint32_t packed_code(const uint8_t* p, int layout, int bits, int64_t w) {
  if (layout == GSQ_LAYOUT_SUPERBLOCK) return bit_field(p + (w >> 8) * 110 + 14, (w & 255) * 3, 3);
  if (layout == GSQ_LAYOUT_BASE3) {
    uint32_t v = p[w / 5];
    for (int j = (int)(w % 5); j; --j) v /= 3;
    return v % 3;
  }
  return bit_field(p, w * bits, bits);
}

__device__ __forceinline__ uint16_t two_bytes(const uint8_t* p) { return p[0] | (uint16_t)(p[1] << 8); }

// One thread per lane of a unit: its 32 codes.
__global__ __launch_bounds__(256) void k_unpack_codes(const uint8_t* __restrict__ packed, int layout,
                                                      int packed_bits, PackedLayer L, int64_t lanes,
                                                      uint32_t* __restrict__ codes) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= lanes) return;
  const int lane = (int)(at & 63);
  const int64_t unit = at >> 6;
  const int kb = (int)(unit % L.blocks);
  const int64_t tile = unit / L.blocks;
  const int64_t e = tile / L.tiles;
  const int64_t o = (tile % L.tiles) * 16 + (lane & 15), i0 = (int64_t)kb * 128 + (lane >> 4) * 32;
  uint32_t words[4] = {0, 0, 0, 0};
  if (o < L.O)
    for (int j = 0; j < 32 && i0 + j < L.I; ++j) {
      const uint32_t c = packed_code(packed, layout, packed_bits, (e * L.O + o) * L.I + i0 + j);
      place_code(words, L.bits, j, min(c, (uint32_t)L.n_levels - 1));
    }
  for (int k = 0; k < L.bits; ++k) codes[at * L.bits + k] = words[k];
}

// One thread per kept scale (groups x tiles x per x 16 channels), zero where there is no channel or group.
__global__ __launch_bounds__(256) void k_unpack_scales(const uint8_t* __restrict__ packed, int layout,
                                                       PackedLayer L, int64_t at_byte, int64_t count,
                                                       uint16_t* __restrict__ scales) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= count) return;
  const int64_t tile = at / 16 / L.scale_groups;
  const int64_t g = at / 16 % L.scale_groups;
  const int64_t e = tile / L.tiles, o = (tile % L.tiles) * 16 + (at & 15);
  uint16_t v = 0;
  if (o < L.O && g < L.I / L.gs) {
    const int64_t k = (e * L.O + o) * (L.I / L.gs) + g;
    v = two_bytes(layout == GSQ_LAYOUT_SUPERBLOCK ? packed + k * 110 : packed + at_byte + 2 * k);
  }
  scales[at] = v;
}

__global__ __launch_bounds__(256) void k_unpack_sub(const uint8_t* __restrict__ packed, PackedLayer L,
                                                    int64_t count, uint8_t* __restrict__ sub) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= count) return;
  const int64_t per = L.scale_groups * 16;
  const int64_t tile = at / 16 / per, g = at / 16 % per;
  const int64_t e = tile / L.tiles, o = (tile % L.tiles) * 16 + (at & 15);
  uint32_t v = 0;
  if (o < L.O && g < L.I / 16) {
    const int64_t rec = (e * L.O + o) * (L.I / 256) + g / 16;
    v = bit_field(packed + rec * 110 + 2, (g & 15) * 6, 6);
  }
  sub[at] = (uint8_t)v;
}

// scale * level rounded to fp32, for a second rounding to the type of x.  The empty asm keeps the compiler
// from joining product and conversion into one instruction, which would round once.
__device__ __forceinline__ float scaled_level(float scale, float level) {
  float p = scale * level;
  asm("" : "+v"(p));
  return p;
}

// Weight (n, k) of one group: scale * level in fp32, rounded to the type of x.
template <class E>
struct PackedWeights {
  const PackedLayer& L;
  int64_t tile0;       // first tile of the group
  static constexpr bool kFast = true;
  __device__ __forceinline__ E at(int n, int k) const {
    if (n >= L.O || k >= L.I) return (E)0;
    const int64_t tile = tile0 + n / 16;
    const int lane = (k % 128) / 32 * 16 + n % 16;
    const uint32_t* words = L.codes + ((tile * L.blocks + k / 128) * 64 + lane) * L.bits;
    const uint32_t c = code_at(words, L.bits, k % 32);
    float s = (float)__builtin_bit_cast(_Float16, L.scales[(tile * L.scale_groups + k / L.gs) * 16 + n % 16]);
    if (L.sub) s *= (float)L.sub[(tile * L.scale_groups * 16 + k / 16) * 16 + n % 16];
    return (E)scaled_level(s, L.levels[c]);
  }
};

template <class T>
__global__ __launch_bounds__(256) void k_packed_any(PackedLayer L, GroupRows rows,
                                                    const typename T::elem* __restrict__ x,
                                                    typename T::elem* __restrict__ y) {
  using E = typename T::elem;
  PanelPlace at;
  if (!find_panel(rows, kAnyTile, blockIdx.x, at)) return;
  const int64_t first = at.first + (int64_t)at.panel * kAnyTile;
  const int e = at.group, ms = (int)min(at.end - first, (int64_t)kAnyTile);
  const AlongK<E> a{x + first * L.I, L.I, ms, L.I};
  tile_any<T>(a, PackedWeights<E>{L, (int64_t)e * L.tiles}, 0, blockIdx.y * kAnyTile, L.I,
              [&](int m, int n, float v) {
                if (m < ms && n < L.O) y[(first + m) * L.O + n] = (E)v;
              });
}

}  // namespace

hipError_t launch_unpack_layer(const gsq_config& cfg, const uint8_t* packed, const PackedLayer& L,
                               hipStream_t s) {
  const auto blocks = [](int64_t n) { return (unsigned)((n + 255) / 256); };
  const int64_t tiles = (int64_t)cfg.batch * L.tiles, weights = (int64_t)cfg.batch * L.O * L.I;
  const int packed_bits = cfg.layout == GSQ_LAYOUT_SUPERBLOCK ? 3 : L.bits;
  const int64_t lanes = tiles * L.blocks * 64, scales = tiles * L.scale_groups * 16;
  k_unpack_codes<<<blocks(lanes), 256, 0, s>>>(packed, cfg.layout, packed_bits, L, lanes,
                                               const_cast<uint32_t*>(L.codes));
  const int64_t at_byte = cfg.layout == GSQ_LAYOUT_BASE3 ? (weights + 4) / 5 : weights * packed_bits / 8;
  k_unpack_scales<<<blocks(scales), 256, 0, s>>>(packed, cfg.layout, L, at_byte, scales,
                                                 const_cast<uint16_t*>(L.scales));
  if (L.sub)
    k_unpack_sub<<<blocks(scales * 16), 256, 0, s>>>(packed, L, scales * 16, const_cast<uint8_t*>(L.sub));
  return hipGetLastError();
}

hipError_t launch_packed_product(const PackedLayer& L, int dtype, const GroupRows& rows, const void* x,
                                 void* y, hipStream_t s) {
  if (rows.rows == 0) return hipSuccess;
  const dim3 grid(most_panels(rows, kAnyTile), (L.O + kAnyTile - 1) / kAnyTile);
  if (dtype == GSQ_DT_BF16)
    k_packed_any<Bf16><<<grid, 256, 0, s>>>(L, rows, static_cast<const __bf16*>(x), static_cast<__bf16*>(y));
  else
    k_packed_any<F16><<<grid, 256, 0, s>>>(L, rows, static_cast<const _Float16*>(x), static_cast<_Float16*>(y));
  return hipGetLastError();
}

}  // namespace gsq
