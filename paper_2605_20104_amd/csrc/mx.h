// The 4-bit cache: microscaled e2m1 elements (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign; codes 0..7, 8 for the sign), 32 along the head
// dimension to a scale 2^(byte - 127).
//
// A run holds the 16 tokens of one page and one KV head in 17 D / 2 bytes: 16 D / 2 bytes of elements, then D / 32 rows of 16
// scale bytes, one per token.  The order of the elements is that of the matrix cores' operands, so that attention loads
// a page's keys, and its values, with one 16-byte load per lane and rearranges nothing:
//   keys    token after token.  Lane l of v_mfma_scale_f32_16x16x128 takes row (token) l % 16, elements 32 (l / 16) .. + 32.
//   values  [token / 4][part 0..15][token % 4][D / 16 elements of the part].  Lane l of v_mfma_f32_16x16x32 takes one row (element
//           of the head dimension) l % 16 of four tokens; with the rows of its D / 16 tiles dealt as part * D / 16 + tile,
//           all that a lane takes of a token stands side by side and has one scale.
#pragma once
#include "common.h"

namespace graft {

constexpr int mx_run_bytes(int D) { return D * 17 / 2; }
constexpr int mx_scales_at(int D) { return 8 * D; }

// Byte of a token's part (its D / 16 elements, D / 32 bytes; parts 0..15) within a run.
template <int D> __device__ __forceinline__ int mx_part_at(bool values, int token, int part) {
    constexpr int UNIT = D / 32;
    return values ? (((token >> 2) * 16 + part) * 4 + (token & 3)) * UNIT : token * (D / 2) + part * UNIT;
}
template <int D> __device__ __forceinline__ int mx_scale_at(int token, int block) { return mx_scales_at(D) + block * 16 + token; }

// The scale byte of a block whose largest magnitude has the bits `top`: m 2^E becomes 4 m 2^(E - 2), or 2 m 2^(E - 1) where
// m > 1.75, so that the largest element comes to lie within (3.5, 7] and, at 6 or below, loses at most a seventh.  (rms error of
// N(0,1) data: 0.1119 with this border, 0.1155 with the largest kept at 6 or below, 0.1151 with no second case.)  Bytes are held
// within 2..252: what the elements stand for is finite and normal in float32 and bfloat16.  255, NaN, where an element is no number.
constexpr unsigned MX_NAN = 255;
constexpr unsigned MX_TOO_LARGE = 253;             // from here on: elements that bfloat16 does not hold, or NaN
__device__ __forceinline__ unsigned mx_scale_byte(unsigned top) {
    const int e = static_cast<int>((top + 0x1FFFFFu) >> 23) - 2;
    const unsigned byte = static_cast<unsigned>(e < 2 ? 2 : e > 252 ? 252 : e);
    return top >= 0x7F800000u ? MX_NAN : byte;
}
__device__ __forceinline__ float mx_scale(unsigned byte) { return __uint_as_float(byte << 23); }    // (255: the conversions make NaN of it)

int device_compute_units();                       // (tree_attn.hip)

}  // namespace graft
