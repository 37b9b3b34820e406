// The 4-bit cache: 32 consecutive columns of a row share a power of two, a byte E that stands for 2^(E - 127); a value is
// one of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} times it: codes 0 to 7, the sign in bit 3, two to a byte, the even column in the
// low half.  Codes [.., D / 2] bytes, scales [.., D / 32] bytes.  E = 255 makes NaN of all 32.
// The chip converts between this and bf16 itself, two values an instruction, the scale (of which it looks at the exponent
// alone) and the rounding to the nearest, ties to the even code, beyond 6 to 6, with it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sb {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int KV4_BLOCK = 32;          // columns of a scale
constexpr int KV4_ROWS = 32;           // a cache has room for a multiple of so many rows
constexpr int KV4_LEAST = 7;           // smallest scale byte written: 2^-120, so that neither a value nor its half is subnormal

// values of byte B of w
template <int B> __device__ __forceinline__ uint32_t kv4_pair(uint32_t w, uint32_t scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, __builtin_bit_cast(float, scale), B));
}

// Scale byte of a block whose largest magnitude has the bf16 bits `top`: the smallest power of two with top <= 7 of it.  Up to 7
// a value is at most half a step of its neighbourhood from the grid (6 and 8, which is not there), so the largest one loses no
// more than others of its size.
__device__ __forceinline__ uint32_t kv4_scale(uint32_t top)
{
    if (top >= 0x7f80u) return 255u;
    const int e = (int)(top >> 7) - 2 + ((top & 0x7fu) > 0x60u);
    return (uint32_t)max(e, KV4_LEAST);
}

}  // namespace sb
