// Rows of bf16 keys and values into a 4-bit cache (sb_kv4.h says how they are held there) and back.
//
// Bound by HBM: 2 D bytes of a row and D / 2 + D / 32 of its 4-bit form.  A thread has eight columns, so that a wave reads (or
// writes) 1 KB side by side; the four threads of a block of 32 columns find its largest magnitude among them.  4096 rows of B4 Hkv8 d128, 85 MB
// a launch: stored in 16.3 us, loaded in 15.2, 5.2 and 5.6 TB/s (a large copy: 5.1); a row each of 32 entries and 8 heads 2.2 us, the shortest launch.
#include "sb_kernels.h"
#include "sb_kv4.h"
#include "sb_mma.h"

namespace sb {
namespace {

constexpr int NTHR = 256;

// the larger magnitude (bf16 bits without the sign) of this lane's and of the one that CTRL names
template <int CTRL> __device__ __forceinline__ uint32_t max_with(uint32_t x)
{
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true));
}

// x: eight bf16 values of a block that four neighbouring lanes hold
__device__ __forceinline__ uint32_t quantise(const u32x4 x, uint32_t& scale)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
    top = max_with<0xB1>(top);             // quad_perm: 1, 0, 3, 2
    top = max_with<0x4E>(top);             // 2, 3, 0, 1
    scale = kv4_scale(top);
    const float s = __builtin_bit_cast(float, scale << 23);
    const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x0), s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x1), s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x2), s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x3), s, 3);
    return w;
}

// grid (rows, entry * kv head, k or v)
template <int D>
__global__ void __launch_bounds__(NTHR)
kv4_store_kernel(const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, uint8_t* __restrict__ kc, uint8_t* __restrict__ ks,
                 uint8_t* __restrict__ vc, uint8_t* __restrict__ vs, const int* __restrict__ pos, int Hkv, int n, int Tcap)
{
    constexpr int TPR = D / 8;
    const int bkv = blockIdx.y;
    const long i = (long)blockIdx.x * (blockDim.x / TPR) + threadIdx.x / TPR;
    const int c = threadIdx.x % TPR;
    const long at = i + (pos ? pos[bkv / Hkv] : 0);
    if (i >= n || at < 0 || at >= Tcap) return;
    const uint16_t* x = blockIdx.z ? v : k;
    uint8_t* codes = blockIdx.z ? vc : kc;
    uint8_t* scales = blockIdx.z ? vs : ks;
    uint32_t scale;
    const uint32_t w = quantise(*reinterpret_cast<const u32x4*>(x + ((long)bkv * n + i) * D + 8 * c), scale);
    const long row = (long)bkv * Tcap + at;
    *reinterpret_cast<uint32_t*>(codes + row * (D / 2) + 4 * c) = w;
    if (c % 4 == 0) scales[row * (D / KV4_BLOCK) + c / 4] = (uint8_t)scale;
}

template <int D>
__global__ void __launch_bounds__(NTHR)
kv4_load_kernel(const uint8_t* __restrict__ kc, const uint8_t* __restrict__ ks, const uint8_t* __restrict__ vc, const uint8_t* __restrict__ vs,
                uint16_t* __restrict__ k, uint16_t* __restrict__ v, const int* __restrict__ pos, int Hkv, int n, int Tcap)
{
    constexpr int TPR = D / 8;
    const int bkv = blockIdx.y;
    const long i = (long)blockIdx.x * (blockDim.x / TPR) + threadIdx.x / TPR;
    const int c = threadIdx.x % TPR;
    if (i >= n) return;
    const long at = i + (pos ? pos[bkv / Hkv] : 0);
    u32x4 x = {0u, 0u, 0u, 0u};
    if (at >= 0 && at < Tcap) {
        const long row = (long)bkv * Tcap + at;
        const uint32_t w = *reinterpret_cast<const uint32_t*>((blockIdx.z ? vc : kc) + row * (D / 2) + 4 * c);
        const uint32_t s = (uint32_t)(blockIdx.z ? vs : ks)[row * (D / KV4_BLOCK) + c / 4] << 23;
        x = u32x4{kv4_pair<0>(w, s), kv4_pair<1>(w, s), kv4_pair<2>(w, s), kv4_pair<3>(w, s)};
    }
    *reinterpret_cast<u32x4*>((blockIdx.z ? v : k) + ((long)bkv * n + i) * D + 8 * c) = x;
}

// threads of a workgroup: no more than a head's rows need, in whole waves
template <int D> int threads_for(int n) { return (int)std::min<long>(NTHR, ((long)n * (D / 8) + 63) / 64 * 64); }

template <int D>
hipError_t store_d(const uint16_t* k, const uint16_t* v, uint8_t* kc, uint8_t* ks, uint8_t* vc, uint8_t* vs,
                   const int* pos, int B, int Hkv, int n, int Tcap, hipStream_t stream)
{
    const int t = threads_for<D>(n), rows = t / (D / 8);
    hipLaunchKernelGGL((kv4_store_kernel<D>), dim3((unsigned)((n + (long)rows - 1) / rows), (unsigned)(B * Hkv), 2u), dim3(t), 0, stream,
                       k, v, kc, ks, vc, vs, pos, Hkv, n, Tcap);
    return hipGetLastError();
}

template <int D>
hipError_t load_d(const uint8_t* kc, const uint8_t* ks, const uint8_t* vc, const uint8_t* vs, uint16_t* k, uint16_t* v,
                  const int* pos, int B, int Hkv, int n, int Tcap, hipStream_t stream)
{
    const int t = threads_for<D>(n), rows = t / (D / 8);
    hipLaunchKernelGGL((kv4_load_kernel<D>), dim3((unsigned)((n + (long)rows - 1) / rows), (unsigned)(B * Hkv), 2u), dim3(t), 0, stream,
                       kc, ks, vc, vs, k, v, pos, Hkv, n, Tcap);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_store(const uint16_t* k, const uint16_t* v, uint8_t* kc, uint8_t* ks, uint8_t* vc, uint8_t* vs,
                            const int* pos, int B, int Hkv, int n, int Tcap, int d, hipStream_t stream)
{
    if (d == 32) return store_d<32>(k, v, kc, ks, vc, vs, pos, B, Hkv, n, Tcap, stream);
    if (d == 64) return store_d<64>(k, v, kc, ks, vc, vs, pos, B, Hkv, n, Tcap, stream);
    return store_d<128>(k, v, kc, ks, vc, vs, pos, B, Hkv, n, Tcap, stream);
}

hipError_t launch_kv4_load(const uint8_t* kc, const uint8_t* ks, const uint8_t* vc, const uint8_t* vs, uint16_t* k, uint16_t* v,
                           const int* pos, int B, int Hkv, int n, int Tcap, int d, hipStream_t stream)
{
    if (d == 32) return load_d<32>(kc, ks, vc, vs, k, v, pos, B, Hkv, n, Tcap, stream);
    if (d == 64) return load_d<64>(kc, ks, vc, vs, k, v, pos, B, Hkv, n, Tcap, stream);
    return load_d<128>(kc, ks, vc, vs, k, v, pos, B, Hkv, n, Tcap, stream);
}

}  // namespace sb
