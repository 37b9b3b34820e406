// Eviction: of every (entry, kv head) the `recent` newest rows and the highest scores among the others stay, `keep` in all, in their
// order (the weights of stick-breaking attention depend on the order of the keys and on nothing else of their positions, so
// what is left is a cache as any other).
//
//   select   a workgroup per (entry, kv head): the smallest score that stays, by its bits from the highest eleven down (radix
//            selection: a histogram in LDS each), then the places of the rows that stay by prefix sums.  Up to 65536 scores stay in registers
//            throughout, more are read again for each step, from L2.  Bound by the latency of its steps: 16384 scores of 128 heads 16.5 us, 1111 of 24
//            6.0; 65536 of 8 heads, in all with their rows, 78 -> 65 us in registers.
//   move     the rows of every array to their places: bound by HBM, 2 x the bytes that stay.  8192 of 16384 4-bit rows of 128 heads at d = 128, 285 MB: 53 us,
//            5.4 TB/s (a large copy: 5.1).
// (Moved by the workgroups that select, the rows would wait for the slowest of them, and 128 workgroups do not fill the chip.)
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

// sum of x over the lanes below this one (by DPP: row_shr 1, 2, 4, 8, then row_bcast 15 and 31), and over all in `total`
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t dpp_or_zero(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ uint32_t wave_prefix(uint32_t x, uint32_t& total)
{
    uint32_t inc = x;
    inc += dpp_or_zero<0x111, 0xF>(inc);
    inc += dpp_or_zero<0x112, 0xF>(inc);
    inc += dpp_or_zero<0x114, 0xF>(inc);
    inc += dpp_or_zero<0x118, 0xF>(inc);
    inc += dpp_or_zero<0x142, 0xA>(inc);
    inc += dpp_or_zero<0x143, 0xC>(inc);
    total = (uint32_t)__builtin_amdgcn_readlane((int)inc, 63);
    return inc - x;
}

// PER scores a thread at a time, in registers; ONE: that is all of them
template <int PER, bool ONE>
__global__ void __launch_bounds__(SEL_THREADS)
evict_select_kernel(const float* __restrict__ score, const int* __restrict__ lens, float* __restrict__ score_out,
                    int* __restrict__ index, int* __restrict__ lens_out, int Hkv, int T, int Tcap, int Tcap_out, int keep, int recent)
{
    constexpr int BLOCK = PER * SEL_THREADS;
    constexpr int BINS = 2 * SEL_THREADS;
    __shared__ uint32_t hist[BINS];
    __shared__ uint32_t s_wave[SEL_NW], s_prefix, s_left, s_whole;
    __shared__ uint32_t s_count[PER * SEL_NW + 1];                // per 64 scores in turn: those above the threshold, and (<< 16) equal to it
    const int bkv = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int len = lens ? min(max(lens[bkv / Hkv], 0), T) : T;
    const int kept = min(len, keep);
    const float* const x = score + (long)bkv * Tcap;
    float* const out = score_out + (long)bkv * Tcap_out;
    int* const at = index + (long)bkv * keep;
    const int older = len > keep ? max(0, len - recent) : 0;      // rows that have to compete
    const int few = kept - (len - older);                         // and how many of them stay
    uint32_t key[PER];                                            // 0: none
    auto read = [&](int i0) __attribute__((always_inline)) {
        float v[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int i = i0 + j * SEL_THREADS + tid;
            v[j] = i < older ? x[i] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) key[j] = i0 + j * SEL_THREADS + tid < older ? rank_of(v[j]) : 0u;
    };
    if (few > 0) read(0);
    if (tid == 0 && bkv % Hkv == 0) lens_out[bkv / Hkv] = kept;
    for (int i = kept + tid; i < keep; i += SEL_THREADS) at[i] = -1;
    // the rows that stay in any case come last
    for (int i = older + tid; i < len; i += SEL_THREADS) {
        at[few + i - older] = i;
        out[few + i - older] = x[i];
    }
    if (few == 0) return;

    uint32_t prefix = 0, left = (uint32_t)few;                    // bits known so far; how many stay of those that share them
    bool whole = false;                                           // all of those: no more bits are needed
#pragma unroll
    for (int step = 0; step < 3; ++step) {
        const int shift = step == 0 ? 21 : step == 1 ? 10 : 0;    // 11, 11 and 10 bits
        if (whole) break;
        hist[tid] = hist[tid + SEL_THREADS] = 0;
        __syncthreads();
        for (int i0 = 0; i0 < older; i0 += BLOCK) {
            if (!ONE && (step > 0 || i0 > 0)) read(i0);
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const uint32_t u = key[j];
                const bool mine = u != 0 && (step == 0 || (u ^ prefix) >> (step == 1 ? 21 : 10) == 0);
                const unsigned long long here = __builtin_amdgcn_ballot_w64(mine);
                if (mine) {
                    const uint32_t bin = (u >> shift) & (step == 2 ? 1023u : 2047u);
                    // equal scores in droves (zeros) would come one after the other: those like the first lane's go as one
                    const uint32_t first = __builtin_amdgcn_readfirstlane(bin);
                    const unsigned long long same = __builtin_amdgcn_ballot_w64(bin == first);
                    if (bin != first) atomicAdd(&hist[bin], 1u);
                    else if (lane == __builtin_ctzll(here)) atomicAdd(&hist[first], (uint32_t)__builtin_popcountll(same));
                }
            }
            if (ONE) break;
        }
        __syncthreads();
        // the bin, from the highest down, that holds the left-th
        const uint32_t h0 = hist[BINS - 1 - 2 * tid], h1 = hist[BINS - 2 - 2 * tid];
        uint32_t total;
        uint32_t before = wave_prefix(h0 + h1, total);
        if (lane == 0) s_wave[wave] = total;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < SEL_NW; ++w) before += w < wave ? s_wave[w] : 0u;
        if (before < left && before + h0 + h1 >= left) {
            const bool second = before + h0 < left;
            s_prefix = prefix | (uint32_t)(BINS - 1 - 2 * tid - second) << shift;
            s_left = left - before - (second ? h0 : 0u);
            s_whole = s_left == (second ? h1 : h0);
        }
        __syncthreads();
        prefix = s_prefix;
        left = s_left;
        whole = s_whole != 0;
    }
    if (whole) {                                                  // everything from there up stays (prefix is above zero: a rank is 2^22 at least)
        --prefix;
        left = 0;
    }

    // places: those above `prefix`, and the first `left` equal to it
    uint32_t put = 0, ties = 0;
    for (int i0 = 0; i0 < older; i0 += BLOCK) {
        if (!ONE) read(i0);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const unsigned long long m = __builtin_amdgcn_ballot_w64(key[j] > prefix), t = __builtin_amdgcn_ballot_w64(key[j] == prefix);
            if (lane == 0) s_count[j * SEL_NW + wave] = (uint32_t)__builtin_popcountll(m) | (uint32_t)__builtin_popcountll(t) << 16;
        }
        __syncthreads();
        if (wave == 0) {
            constexpr int EACH = PER * SEL_NW / 64;
            uint32_t c[EACH], own = 0, total;
#pragma unroll
            for (int i = 0; i < EACH; ++i) own += c[i] = s_count[EACH * lane + i];
            uint32_t before = wave_prefix(own, total);
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                s_count[EACH * lane + i] = before;
                before += c[i];
            }
            if (lane == 0) s_count[PER * SEL_NW] = total;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const bool more = key[j] > prefix, tie = key[j] == prefix;
            const unsigned long long m = __builtin_amdgcn_ballot_w64(more), t = __builtin_amdgcn_ballot_w64(tie), below = (1ull << lane) - 1;
            const uint32_t c = s_count[j * SEL_NW + wave];
            const uint32_t above = put + (c & 0xffffu) + (uint32_t)__builtin_popcountll(m & below);
            const uint32_t equal = ties + (c >> 16) + (uint32_t)__builtin_popcountll(t & below);
            if (more || (tie && equal < left)) {
                const uint32_t p = above + min(equal, left);
                const int i = i0 + j * SEL_THREADS + tid;
                at[p] = i;
                out[p] = x[i];
            }
        }
        if (ONE) return;
        const uint32_t total = s_count[PER * SEL_NW];
        put += total & 0xffffu;
        ties += total >> 16;
        __syncthreads();                                          // (everyone has read it)
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
    auto select = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)(B * Hkv)), dim3(SEL_THREADS), 0, stream,
                           score, lens, score_out, index, lens_out, Hkv, T, Tcap, Tcap_out, keep, recent);
    };
    if (T <= 4 * SEL_THREADS) select(evict_select_kernel<4, true>);
    else if (T <= 16 * SEL_THREADS) select(evict_select_kernel<16, true>);
    else if (T <= 64 * SEL_THREADS) select(evict_select_kernel<64, true>);
    else select(evict_select_kernel<16, false>);
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
