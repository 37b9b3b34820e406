// Eviction: of every (entry, kv head) the `recent` newest rows and the highest scores among the others stay, `keep` in all, in their
// order (the weights of stick-breaking attention depend on the order of the keys and on nothing else of their positions, so
// what is left is a cache as any other).
//
//   select   a workgroup per (entry, kv head): the smallest score that stays, by its bits from the highest eight down (radix
//            selection: a histogram in LDS each), then the places of the rows that stay by prefix sums.  Reads the scores five times, from L2 but the first.
//   move     the rows of every array to their places: bound by HBM, 2 x the bytes that stay.
#include "sb_kernels.h"

namespace sb {
namespace {

constexpr int SEL_THREADS = 1024;
constexpr int SEL_NW = SEL_THREADS / 64;
constexpr int MOVE_THREADS = 256;
constexpr int MOVE_ROWS = 64;          // rows of a workgroup

struct Arrays {
    const uint8_t* src[EVICT_ARRAYS];
    uint8_t* dst[EVICT_ARRAYS];
    int row_bytes[EVICT_ARRAYS];
    int n;
};

// order of scores as whole numbers: -0 is 0, NaN is above everything
__device__ __forceinline__ uint32_t rank_of(float x)
{
    if (x != x) return 0xffffffffu;
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(SEL_THREADS)
evict_select_kernel(const float* __restrict__ score, const int* __restrict__ lens, float* __restrict__ score_out,
                    int* __restrict__ index, int* __restrict__ lens_out, int Hkv, int T, int Tcap, int Tcap_out, int keep, int recent)
{
    __shared__ uint32_t hist[256];
    __shared__ uint32_t s_prefix, s_left;
    __shared__ int s_more[2][SEL_NW], s_ties[2][SEL_NW];
    const int bkv = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int len = lens ? min(max(lens[bkv / Hkv], 0), T) : T;
    const int kept = min(len, keep);
    const float* const x = score + (long)bkv * Tcap;
    float* const out = score_out + (long)bkv * Tcap_out;
    int* const at = index + (long)bkv * keep;
    if (tid == 0 && bkv % Hkv == 0) lens_out[bkv / Hkv] = kept;
    for (int i = kept + tid; i < keep; i += SEL_THREADS) at[i] = -1;
    const int older = len > keep ? max(0, len - recent) : 0;      // rows that have to compete
    const int few = kept - (len - older);                         // and how many of them stay
    // the rows that stay in any case come last
    for (int i = older + tid; i < len; i += SEL_THREADS) {
        at[few + i - older] = i;
        out[few + i - older] = x[i];
    }
    if (few == 0) return;

    uint32_t prefix = 0, left = (uint32_t)few;                    // bits known so far; how many stay of those that share them
#pragma unroll
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < older; i += SEL_THREADS) {
            const uint32_t u = rank_of(x[i]);
            if (shift == 24 || (u ^ prefix) >> (shift + 8 & 31) == 0) {
                const uint32_t bin = (u >> shift) & 255u;
                // equal scores in droves (zeros) would come one after the other
                const uint32_t first = __builtin_amdgcn_readfirstlane(bin);
                const unsigned long long here = __builtin_amdgcn_ballot_w64(true), same = __builtin_amdgcn_ballot_w64(bin == first);
                if (here == same) {
                    if (lane == __builtin_ctzll(here)) atomicAdd(&hist[first], (uint32_t)__builtin_popcountll(here));
                } else {
                    atomicAdd(&hist[bin], 1u);
                }
            }
        }
        __syncthreads();
        if (wave == 0) {                                          // the bin, from the highest down, that holds the left-th
            uint32_t h[4], own = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) own += h[i] = hist[255 - 4 * lane - i];
            uint32_t before = own;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const uint32_t up = __shfl_up(before, d);
                if (lane >= d) before += up;
            }
            before -= own;
            if (before < left && before + own >= left) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (before < left && before + h[i] >= left) {
                        s_prefix = prefix | (uint32_t)(255 - 4 * lane - i) << shift;
                        s_left = left - before;
                    }
                    before += h[i];
                }
            }
        }
        __syncthreads();
        prefix = s_prefix;
        left = s_left;
    }

    // places: those above `prefix`, and the first `left` equal to it
    int put = 0, ties = 0;
    for (int i0 = 0, par = 0; i0 < older; i0 += SEL_THREADS, par ^= 1) {
        const int i = i0 + tid;
        const float v = i < older ? x[i] : 0.0f;
        const uint32_t u = i < older ? rank_of(v) : 0u;
        const bool more = i < older && u > prefix, tie = i < older && u == prefix;
        const unsigned long long bm = __builtin_amdgcn_ballot_w64(more), bt = __builtin_amdgcn_ballot_w64(tie);
        if (lane == 0) {
            s_more[par][wave] = __builtin_popcountll(bm);
            s_ties[par][wave] = __builtin_popcountll(bt);
        }
        __syncthreads();
        const unsigned long long below = (1ull << lane) - 1;
        int m = 0, t = 0, all_m = 0, all_t = 0;
#pragma unroll
        for (int w = 0; w < SEL_NW; ++w) {
            if (w < wave) {
                m += s_more[par][w];
                t += s_ties[par][w];
            }
            all_m += s_more[par][w];
            all_t += s_ties[par][w];
        }
        m += __builtin_popcountll(bm & below);
        t += ties + __builtin_popcountll(bt & below);              // ties before this one
        if (more || (tie && t < (int)left)) {
            const int p = put + m + min(t, (int)left);
            at[p] = i;
            out[p] = v;
        }
        put += all_m;
        ties += all_t;
    }
}

template <class V> __device__ __forceinline__ void move_rows(const uint8_t* src, uint8_t* dst, const int* from, int rows, int row_bytes)
{
    const unsigned per = (unsigned)row_bytes / sizeof(V);
    const unsigned n = (unsigned)rows * per;
    for (unsigned i = threadIdx.x; i < n; i += MOVE_THREADS) {
        const unsigned r = i / per, c = i % per;
        *reinterpret_cast<V*>(dst + (long)r * row_bytes + c * sizeof(V)) = *reinterpret_cast<const V*>(src + (long)from[r] * row_bytes + c * sizeof(V));
    }
}

__global__ void __launch_bounds__(MOVE_THREADS)
evict_move_kernel(const Arrays a, const int* __restrict__ index, const int* __restrict__ lens, int Hkv, int T, int Tcap, int Tcap_out, int keep)
{
    __shared__ int from[MOVE_ROWS];
    const int bkv = blockIdx.y, r0 = blockIdx.x * MOVE_ROWS;
    const int len = lens ? min(max(lens[bkv / Hkv], 0), T) : T;
    const int rows = min(MOVE_ROWS, min(len, keep) - r0);
    if (rows <= 0) return;
    if ((int)threadIdx.x < rows) from[threadIdx.x] = index[(long)bkv * keep + r0 + threadIdx.x];
    __syncthreads();
    for (int j = 0; j < a.n; ++j) {
        const int rb = a.row_bytes[j];
        const uint8_t* src = a.src[j] + (long)bkv * Tcap * rb;
        uint8_t* dst = a.dst[j] + ((long)bkv * Tcap_out + r0) * rb;
        if (rb % 16 == 0) move_rows<uint4>(src, dst, from, rows, rb);
        else if (rb % 4 == 0) move_rows<uint32_t>(src, dst, from, rows, rb);
        else if (rb % 2 == 0) move_rows<uint16_t>(src, dst, from, rows, rb);
        else move_rows<uint8_t>(src, dst, from, rows, rb);
    }
}

}  // namespace

hipError_t launch_evict(const float* score, const int* lens, const void* const* src, void* const* dst, const int* row_bytes, int arrays,
                        float* score_out, int* index, int* lens_out, int B, int Hkv, int T, int Tcap, int Tcap_out, int keep, int recent, hipStream_t stream)
{
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)(B * Hkv)), dim3(SEL_THREADS), 0, stream,
                       score, lens, score_out, index, lens_out, Hkv, T, Tcap, Tcap_out, keep, recent);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || arrays == 0) return e;
    Arrays a = {};
    a.n = arrays;
    for (int i = 0; i < arrays; ++i) {
        a.src[i] = static_cast<const uint8_t*>(src[i]);
        a.dst[i] = static_cast<uint8_t*>(dst[i]);
        a.row_bytes[i] = row_bytes[i];
    }
    hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)((std::min(keep, T) + MOVE_ROWS - 1) / MOVE_ROWS), (unsigned)(B * Hkv)), dim3(MOVE_THREADS), 0, stream,
                       a, index, lens, Hkv, T, Tcap, Tcap_out, keep);
    return hipGetLastError();
}

}  // namespace sb
