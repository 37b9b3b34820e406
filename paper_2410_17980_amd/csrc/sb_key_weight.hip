// The weight that a prompt's queries give each key: score_out[i] = score[i] + sum over query rows j and heads of the group of A[i,j]
// (Eq. 1).  The queries are the last rows of their entry, all of it or a window at its end.
//
// Logits and weights as in the forward; in place of A V the sum of A over the queries.  A unit is 32 query rows of one head; units of
// the heads of a group at the same rows are neighbours, as they read the same keys.  A workgroup takes NW units, sweeps 64-key tiles
// from the last unit's diagonal towards key 0, and leaves the sums over its queries, one number a key, in the workspace; a second
// launch adds the workgroups up in a fixed order.  It stops where the stick of all its rows is used up (CARRY_EXHAUSTED), and notes how far it came.
#include "sb_kernels.h"
#include "sb_mma.h"

namespace sb {
namespace {

constexpr int NW = 4;                  // waves of a workgroup, a unit each
constexpr int TK = 64;                 // keys of a tile
constexpr int SUM_THREADS = 256;

template <int CTRL> __device__ __forceinline__ float dpp(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}

// Sums over the 32 lanes of a half-wave of 16 values: lane n gets the sum of value key_of_lane(n).  Each step
// hands half of the values that are left to the partner lane and adds the partner's share of the other half.
__device__ __forceinline__ int key_of_lane(int n)
{
    return ((n >> 4) & 1) * 8 + ((n >> 3) & 1) * 4 + ((n >> 2) & 1) * 2 + ((n >> 1) & 1);
}
__device__ __forceinline__ float sums_of_lanes(const float (&v)[16], int n)
{
    float a[8], b[4], c[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        auto sw = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(int, v[i]), __builtin_bit_cast(int, v[i + 8]), false, false);
        a[i] = __builtin_bit_cast(float, (int)sw[0]) + __builtin_bit_cast(float, (int)sw[1]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = ((n & 8) ? a[i + 4] : a[i]) + dpp<0x128>((n & 8) ? a[i] : a[i + 4]);        // row_ror:8
#pragma unroll
    for (int i = 0; i < 2; ++i) c[i] = ((n & 4) ? b[i + 2] : b[i]) + dpp<0x141>((n & 4) ? b[i] : b[i + 2]);        // row_half_mirror
    const float d = ((n & 2) ? c[1] : c[0]) + dpp<0x1B>((n & 2) ? c[0] : c[1]);                                    // quad_perm 3, 2, 1, 0
    return d + dpp<0xB1>(d);                                                                                       // quad_perm 1, 0, 3, 2
}

struct Args {
    const uint16_t *q, *k;
    const int *lens, *qlens;           // or nullptr: T, Tq
    const float* score;                // or nullptr: zero
    float* score_out;
    float* part;                       // [entry * kv head][workgroup][Tpad]
    int* reach;                        // [entry * kv head][workgroup][2]: first key written, one past the last
    int H, Hkv, G, Tq, T, Tcap, Tpad, groups;
};

__device__ __forceinline__ int length_of(const int* lens, int b, int most)
{
    return lens ? min(max(lens[b], 0), most) : most;
}

template <int D>
__global__ void __launch_bounds__(64 * NW, 2)
key_weight_kernel(const Args a, int BHkv, int first_wg)
{
    constexpr int ROW = 2 * D, CPR = ROW / 16, BLK_ROWS = 1024 / ROW;
    constexpr int TILE = TK * ROW, NPW = TILE / 1024 / NW;
    __shared__ __attribute__((aligned(1024))) char tiles[2 * TILE];
    __shared__ __attribute__((aligned(16))) float csum[2][NW][TK];
    __shared__ __attribute__((aligned(16))) int s_done[2][NW];

    const int wg = first_wg + blockIdx.x;
    const int bkv = wg % BHkv, grp = a.groups - 1 - wg / BHkv;         // the longest first
    const int b = bkv / a.Hkv;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int len = length_of(a.lens, b, a.T), qlen = length_of(a.qlens, b, a.Tq);
    const int off = len - qlen;                                         // position of query row 0
    int* const reach = a.reach + ((long)bkv * a.groups + grp) * 2;

    const int unit = grp * NW + wave;
    const int strip = unit / a.G, head = (bkv % a.Hkv) * a.G + unit % a.G;
    // keys below `sees` are visible to this lane's query; to all of the strip's below `all`, to one at least below `some`
    const int row = 32 * strip + n;
    const int sees = row < qlen ? off + row : 0;
    const int all = max(0, off + 32 * strip);
    const int some = 32 * strip < qlen ? max(0, off + min(32 * strip + 32, qlen) - 1) : 0;
    const int last_strip = min((grp * NW + NW - 1) / a.G, (qlen - 1) / 32);            // of the workgroup, with rows in it
    const int top = grp * NW / a.G * 32 < qlen ? max(0, off + min(32 * last_strip + 32, qlen) - 1) : 0;
    if (top == 0) {
        if (tid == 0) reach[0] = reach[1] = 0;
        return;
    }

    const float c2 = SB_LOG2E / sqrtf((float)D);
    bf16x8 qf[D / 16];                         // zero where there is no row: what lies there may be anything
    {
        const uint16_t* x = a.q + (((long)b * a.H + head) * a.Tq + min(row, a.Tq - 1)) * D + 8 * hh;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            u32x4 y = *reinterpret_cast<const u32x4*>(x + 16 * s);
            if (row >= qlen) y = u32x4{0u, 0u, 0u, 0u};
            qf[s] = __builtin_bit_cast(bf16x8, y);
        }
    }
    const uint16_t* const kg = reinterpret_cast<const uint16_t*>(scalar_base(a.k + (long)bkv * a.Tcap * D));
    int goff[NPW];
#pragma unroll
    for (int i = 0; i < NPW; ++i) {
        const int r = (wave * NPW + i) * BLK_ROWS + lane / CPR;
        goff[i] = r * ROW + (((lane % CPR) ^ swz_perm<D>(r)) << 4);
    }
    auto stage = [&](int jt, int st) __attribute__((always_inline)) {
        const uint16_t* src = kg + (long)jt * TK * D;
        char* dst = tiles + st * TILE + wave * NPW * 1024;
        if ((jt + 1) * TK <= len) dma16_to_lds_run(src, goff, dst);
        else dma16_to_lds_run_clamped<ROW, BLK_ROWS>(src, goff, wave * NPW * BLK_ROWS + lane / CPR, len - 1 - jt * TK, dst);
    };
    const uint32_t smem0 = lds_offset(tiles);
    uint32_t aoff[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) aoff[s] = smem0 + tile_off_perm<D>(perm_row(n), 2 * s + hh);

    // a row that is not there has nothing of its stick left
    float carry = row < qlen ? 0.0f : 1e9f;
    const int jt0 = (top - 1) / TK;
    float* const part = a.part + ((long)bkv * a.groups + grp) * a.Tpad;
    auto flush = [&](int jt, int par) __attribute__((always_inline)) {
        if (tid < TK) part[(long)jt * TK + tid] = (csum[par][0][tid] + csum[par][1][tid]) + (csum[par][2][tid] + csum[par][3][tid]);
    };
    stage(jt0, 0);
    int jt = jt0, par = 0;
    for (;; --jt, par ^= 1) {
        dma_wait<0>();
        barrier_lds();
        if (jt < jt0) {
            flush(jt + 1, par ^ 1);
            if (jt < 0 || waves_done(s_done[par ^ 1])) break;
        }
        if (jt > 0) stage(jt - 1, par ^ 1);
#pragma unroll
        for (int half = 1; half >= 0; --half) {
            const int base = jt * TK + 32 * half;
            float w[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) w[r] = 0.0f;
            if (base < some && __builtin_amdgcn_ballot_w64(!(carry >= CARRY_EXHAUSTED)) != 0) {
                f32x16 s;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, lds_load16(aoff[i] + par * TILE + 32 * half * ROW)), qf[i], s, 0, 0, 0);
                const bool mask = base + 32 > all;
                const int visible = sees - base - 16 * hh;
                // Eq. 1's product in the lane, from 2^-60 on: w[r] = W_r e_r, W_{r+1} = W_r + w[r]
                float W = 0x1p-60f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float e = fast_exp2(s[r] * c2);
                    if (mask) e = r < visible ? e : 0.0f;
                    w[r] = W * e;
                    W += w[r];
                }
                float lo, hi;
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(W < 0x1p80f)) == 0, 1)) {
                    both_halves(fast_log2(W) + 60.0f, lo, hi);
                    const float kf = fast_exp2(60.0f - (carry + hi + (hh == 0 ? lo : 0.0f)));
#pragma unroll
                    for (int r = 0; r < 16; ++r) w[r] *= kf;
                } else {                       // in the log form
                    float run = 0.0f;
#pragma unroll
                    for (int r = 15; r >= 0; --r) {
                        const float x = !mask || r < visible ? s[r] * c2 : -INFINITY;
                        run += sp2(x);
                        w[r] = x - run;
                    }
                    both_halves(run, lo, hi);
                    const float take = carry + (hh == 0 ? hi : 0.0f);
#pragma unroll
                    for (int r = 0; r < 16; ++r) w[r] = fast_exp2(w[r] - take);
                }
                carry += lo + hi;
            }
            const float sum = sums_of_lanes(w, n);
            if ((n & 1) == 0) csum[par][wave][32 * half + 16 * hh + key_of_lane(n)] = sum;
        }
        const int done = __builtin_amdgcn_ballot_w64(!(carry >= CARRY_EXHAUSTED)) == 0 ? -1 : 0;
        if (lane == 0) s_done[par][wave] = done;
    }
    if (tid == 0) {
        reach[0] = (jt + 1) * TK;
        reach[1] = (jt0 + 1) * TK;
    }
}

__global__ void __launch_bounds__(SUM_THREADS)
key_weight_sum_kernel(const Args a)
{
    const int bkv = blockIdx.y, key = blockIdx.x * SUM_THREADS + threadIdx.x;
    const int len = length_of(a.lens, bkv / a.Hkv, a.T);
    if (blockIdx.x * SUM_THREADS >= len) return;
    const float* part = a.part + (long)bkv * a.groups * a.Tpad;
    const int* reach = a.reach + (long)bkv * a.groups * 2;
    float s = 0.0f;
    for (int g = 0; g < a.groups; ++g) {
        const int lo = reach[2 * g], hi = reach[2 * g + 1];
        if (key >= lo && key < hi) s += part[(long)g * a.Tpad + key];
    }
    if (key < len) {
        const long at = (long)bkv * a.Tcap + key;
        a.score_out[at] = (a.score ? a.score[at] : 0.0f) + s;
    }
}

int groups_of(int H, int Hkv, int Tq) { return (int)(((long)((Tq + 31) / 32) * (H / Hkv) + NW - 1) / NW); }
int pad_of(int T) { return (T + TK - 1) / TK * TK; }

}  // namespace

size_t key_weight_workspace_bytes(int B, int H, int Hkv, int Tq, int T)
{
    return sizeof(float) * (size_t)B * Hkv * groups_of(H, Hkv, Tq) * ((size_t)pad_of(T) + 2);
}

hipError_t launch_key_weight(const uint16_t* q, const uint16_t* k, const int* lens, const int* qlens, const float* score, float* score_out,
                             float* workspace, int B, int H, int Hkv, int Tq, int T, int Tcap, int d, hipStream_t stream)
{
    Args a = {q, k, lens, qlens, score, score_out, workspace, nullptr, H, Hkv, H / Hkv, Tq, T, Tcap, pad_of(T), groups_of(H, Hkv, Tq)};
    a.reach = reinterpret_cast<int*>(workspace + (size_t)B * Hkv * a.groups * a.Tpad);
    const int BHkv = B * Hkv;
    auto go = [&](unsigned wgs, int first) {
        const dim3 grid(wgs), threads(64 * NW);
        if (d == 32) hipLaunchKernelGGL((key_weight_kernel<32>), grid, threads, 0, stream, a, BHkv, first);
        else if (d == 64) hipLaunchKernelGGL((key_weight_kernel<64>), grid, threads, 0, stream, a, BHkv, first);
        else hipLaunchKernelGGL((key_weight_kernel<128>), grid, threads, 0, stream, a, BHkv, first);
    };
    const hipError_t e = launch_workgroups((long)BHkv * a.groups, 64 * NW, go);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(key_weight_sum_kernel, dim3((unsigned)((T + SUM_THREADS - 1) / SUM_THREADS), (unsigned)BHkv), dim3(SUM_THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace sb
