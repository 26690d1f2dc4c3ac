// The microscaled cache format on the device.
//
// A row of D elements is D / 32 blocks.  A block is one scale byte b, standing for 2^(b - 127), and 32 elements: e4m3 bytes
// (MXFP8), or e2m1 nibbles (MXFP4), two to a byte, the even element in the low one.  A scale is a power of two and an element
// has at most four significant bits, so every value of the cache is a bf16 number exactly: products of queries with it are
// those of a bf16 cache that holds the same values, and nothing is rounded when it is read.
#pragma once

#include "common.cuh"

namespace quoka {

constexpr int kMxBlock = 32;
constexpr int kMxExpMin = -64, kMxExpMax = 15;    // exponents of a scale, as quoka_append_kv_mx writes them
constexpr uint32_t kMxNanScale = 255;             // a block with a value that is not finite reads back as NaN

constexpr int kNoNan = 0x7FFFFFFF;                   // no position, or key, that sees a value that is not finite
// Formats of a cache that an attention kernel is made for: 0 bf16, QUOKA_KV_MXFP8, QUOKA_KV_MXFP4, and bf16 rows unpacked from either.
constexpr int kUnpacked = 3;
template <int FMT>
constexpr bool kIsMx = FMT == QUOKA_KV_MXFP8 || FMT == QUOKA_KV_MXFP4;
template <int FMT>
constexpr int kMxBits = FMT == QUOKA_KV_MXFP8 ? 8 : 4;

// e4m3's codes 0x7F and 0xFF are no numbers.  quoka_append_kv_mx does not write them; reading back and the scalar kernels give NaN for them,
// the others take them for whatever their conversion makes of the bits.
constexpr uint32_t kE4m3Nan = 0x7Fu;
// Whether a word of four codes has one.
__device__ __forceinline__ bool e4m3_has_nan(uint32_t w) { return (((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0u; }

// The value of an element: its bits at the place of an fp32 number's exponent and fraction are the value times a power of two
// (subnormals too), which the multiplication takes off.
template <int FMT>
__device__ __forceinline__ float mx_element(uint32_t code) {
  if constexpr (FMT == QUOKA_KV_MXFP8)
    return (code & 0x7Fu) == kE4m3Nan ? __uint_as_float(0x7FC00000u) : __uint_as_float((code & 0x80u) << 24 | (code & 0x7Fu) << 20) * 0x1p120f;
  else
    return __uint_as_float((code & 8u) << 28 | (code & 7u) << 22) * 0x1p126f;
}

// 2^(b - 127), NaN for the scale byte of a block that is not finite.
__device__ __forceinline__ float mx_scale(uint32_t b) {
  return b == kMxNanScale ? __uint_as_float(0x7FC00000u) : b == 0 ? 0x1p-127f : __uint_as_float(b << 23);
}

// 8 elements in order as bf16 pairs, their bits at the place of a bf16 number's exponent and fraction: the values divided by 2^120, 2^126.
template <int FMT>
__device__ __forceinline__ void mx_bits_bf16x8(uint32_t w0, uint32_t w1, uint32_t (&o)[4]) {
  if constexpr (FMT == QUOKA_KV_MXFP8) {
    o[0] = __byte_perm(w0, w0, 0x1100); o[1] = __byte_perm(w0, w0, 0x3322);
    o[2] = __byte_perm(w1, w1, 0x1100); o[3] = __byte_perm(w1, w1, 0x3322);
  } else {
    const uint32_t lo = w0 << 4;
    o[0] = __byte_perm(lo, w0, 0x4400); o[1] = __byte_perm(lo, w0, 0x5511);
    o[2] = __byte_perm(lo, w0, 0x6622); o[3] = __byte_perm(lo, w0, 0x7733);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)                          // (what stands below an element's bits is masked off)
    o[i] = (o[i] & 0x80008000u) | (FMT == QUOKA_KV_MXFP8 ? o[i] >> 4 & 0x07F007F0u : o[i] >> 6 & 0x01C001C0u);
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// 2^(b - 127) twice, NaN for the scale byte of a block that is not finite.
__device__ __forceinline__ uint32_t mx_scale_bf16x2(uint32_t b) { return (b == kMxNanScale ? 0x7FC0u : b == 0 ? 0x0040u : b << 7) * 0x10001u; }
// 8 elements as bf16 values, exactly, whatever the scale: half the instructions of eight floats rounded to bf16
// (4 sequences of 20011 to 32768 rows, 8 heads, d 128, MXFP4 read back, one call after the other: 101 us so, 91 this way).
template <int FMT>
__device__ __forceinline__ uint4 mx_values_bf16x8(uint32_t w0, uint32_t w1, uint32_t scale2) {
  uint32_t o[4];
  mx_bits_bf16x8<FMT>(w0, w1, o);
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = mul_bf16x2(mul_bf16x2(o[i], FMT == QUOKA_KV_MXFP8 ? 0x7B807B80u : 0x7E807E80u), scale2);
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// Exponent of a block's scale from the bits of its largest magnitude (finite): the smallest e with amax <= M 2^e, M = 1.75 2^8 or
// 1.5 2^2: a fraction above M's carries into the exponent.
template <int FMT>
__device__ __forceinline__ int mx_scale_exponent(uint32_t amax_bits) {
  constexpr uint32_t kCarry = FMT == QUOKA_KV_MXFP8 ? 0x1FFFFFu : 0x3FFFFFu;
  const int e = (int)((amax_bits + kCarry) >> 23) - 127 - (FMT == QUOKA_KV_MXFP8 ? 8 : 2);
  return min(max(e, kMxExpMin), kMxExpMax);
}

// Two values, already divided by their scale, to elements (round to nearest even, saturating): a in the lower one.
template <int FMT>
__device__ __forceinline__ uint32_t mx_encode2(float a, float b) {
  if constexpr (FMT == QUOKA_KV_MXFP8) {
    uint16_t h;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h) : "f"(b), "f"(a));
    return h;
  } else {
    uint32_t w;
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tmov.b32 %0, {t, t, t, t};\n\t}" : "=r"(w) : "f"(b), "f"(a));
    return w & 0xFFu;
  }
}

// Index of a row's first scale byte: the cache's layout without head_dim, D / 32 bytes per row.
template <int D, bool FIRST = false>
__device__ __forceinline__ int64_t mx_scale_index(const DevParams& P, int s, int h, int t) {
  return kv_norm_index<FIRST>(P, s, h, t) * (D / kMxBlock);
}

}  // namespace quoka
