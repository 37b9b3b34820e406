// The weight that a prompt's queries give each key: score_out[i] = score[i] + sum over query rows j and heads of the group of A[i,j]
// (Eq. 1).  The queries are the last rows of their entry, all of it or a window at its end.
//
// Logits as in the forward, S^T = K Q^T by the 32x32x16 MFMA, a lane 16 keys of one query; Eq. 1's product along the keys in the lane,
// and what is left of a query's stick carried from 32 keys to the next as it is, not by its logarithm: a weight here is a result in
// fp32, and the logarithm of a carry around 30 would be off by 2^-20 of it (the forward's weights go on to a product in bf16).  As in sb_decode_kv4.hip, many small weights would be
// lost beside a 1: the keys of a tile carry P = prod (1 + e) - 1, and the tiles' shares of the stick are multiplied in 64 bits.  From
// less than 2^-126 of the stick on, no weight is more than a subnormal number: the row counts as exhausted and what is farther gets nothing from it.
// In place of A V the sum of A over the queries.  A unit is 32 query rows of one head; units of the heads of a group at the
// same rows are neighbours, as they read the same keys.  What a workgroup's queries give the keys, one number a key, goes into
// the workspace, with how far it reaches; a last launch adds the workgroups up in a fixed order.
//   key_weight_kernel        a unit a wave, or two where there are plenty; 64-key tiles through LDS for all of a workgroup, from the last unit's diagonal towards
//                            key 0.  Few units at many keys are also split over chunks of keys: a first launch finds what each chunk leaves of the sticks, a
//                            second one the weights
//   key_weight_small_kernel  one unit a workgroup, its waves 32 keys each, side by side
// Bound by vector instructions: for 32 x 32 weights 16 exponentials a lane and some 110 others, next to the D / 16 matrix products.  B1 H32 Hkv8 T8192 d128,
// 1.05 million such squares, all far 405 us, a third of the kv heads 186, none 40 (384 all far with 1 + P and fp32 in place of P and 64 bits); the products alone are 216 us at the 1271 TFLOP/s that a product of 8192^3 reaches
// here (109 at the chip's peak), the exponentials alone 109 at 2.4 GHz.  Three and four tiles of K under way instead of two, or four waves a unit, gain nothing (402 -> 482 with four, before that).
#include <climits>
#include <type_traits>
#include "sb_kernels.h"
#include "sb_mma.h"
#include "sb_plan_key_weight.h"

namespace sb {
namespace {

using namespace key_weight;

constexpr int SNW = 8;                 // waves of a small kernel's workgroup
constexpr int SUM_DEEP = 4;            // groups that a wave of the last launch asks for at once

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
    float* part;                       // [entry * kv head][group][Tpad]; a group is a workgroup's units, groups first .. first + groups - 1
    int* reach;                        // [entry * kv head][group][chunks][2]: first key written, one past the last
    double* left;                      // [entry * kv head][unit][chunks][32]: the share of the stick that a chunk leaves of each query's
    int H, Hkv, G, Tq, T, Tcap, Tpad, groups, chunks, C, first;
};

__device__ __forceinline__ int length_of(const int* lens, int b, int most)
{
    return lens ? min(max(lens[b], 0), most) : most;
}

constexpr float LEAST = 0x1p-126f;     // of the stick
__device__ __forceinline__ bool none_left(double stick) { return __builtin_amdgcn_ballot_w64(!(stick < LEAST)) == 0; }

// One query's share of 32 keys, a half-wave 16 of them, N times (two subtiles of keys, or two queries): with the stick whole before a subtile's nearest
// key, the weight of key r is w[r] * mine, and `all` is what its 32 leave, 1 / (1 + sum).  MASK: keys from `visible` on are not seen.  (N = 2: one's instructions fill the
// other's waits.)
struct Taken { float all, sum; };
// (1 + p) (1 + q) - 1
__device__ __forceinline__ float plus(float p, float q) { return __builtin_fmaf(p, q, p + q); }
// of one's keys and the next, farther ones'
__device__ __forceinline__ Taken both(Taken x, Taken y) { return {x.all * y.all, plus(x.sum, y.sum)}; }
// What is left once these keys have been passed.  Where they take half of the stick or more, the last bits of the sum count no more, and it may be anything.
__device__ __forceinline__ double passed(double stick, Taken t)
{
    return stick * (t.all > 0.5f ? 1.0 - (double)(t.all * t.sum) : (double)t.all);
}
template <bool MASK, int N>
__device__ __forceinline__ void weights(const f32x16 (&s)[N], float c2, const int (&visible)[N], int hh, float (&w)[N][16], float (&mine)[N], Taken (&t)[N])
{
    // w[r] = (1 + P_r) e_r, P_{r+1} = P_r + w[r], e = sigma / (1 - sigma): 1 + P_r = prod_{r' < r} 1 / (1 - sigma_r')
    float P[N], most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) P[i] = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float e = fast_exp2(s[i][r] * c2);
            if (MASK) e = r < visible[i] ? e : 0.0f;
            w[i][r] = __builtin_fmaf(P[i], e, e);
            P[i] += w[i][r];
        }
#pragma unroll
    for (int i = 0; i < N; ++i) most += P[i];
    // what the lane's keys leave, and what makes w the weight where the stick is whole before the lane's nearest key
    float left[N], norm[N];
#pragma unroll
    for (int i = 0; i < N; ++i) left[i] = norm[i] = __builtin_amdgcn_rcpf(1.0f + P[i]);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(most < 0x1p40f)) != 0, 0)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            // (norm times what is left before the lane could be subnormal where the weight is not)
#pragma unroll
            for (int r = 0; r < 16; ++r) w[i][r] *= norm[i];
            norm[i] = 1.0f;
            if (!(P[i] < 0x1p120f)) {          // in the log form
                float run = 0.0f;
#pragma unroll
                for (int r = 15; r >= 0; --r) {
                    const float x = !MASK || r < visible[i] ? s[i][r] * c2 : -INFINITY;
                    run += sp2(x);
                    w[i][r] = fast_exp2(x - run);
                }
                left[i] = fast_exp2(-run);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float lo, hi, p, q;                    // (the upper half's keys are nearer)
        both_halves(left[i], lo, hi);
        both_halves(P[i], p, q);
        t[i] = {lo * hi, plus(p, q)};
        mine[i] = hh ? norm[i] : norm[i] * hi;
    }
}

// the other half-wave's copy
__device__ __forceinline__ double other_half(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)u, 32), hi = (uint32_t)__shfl_xor((int)(uint32_t)(u >> 32), 32);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// the unit's rows and what they see
struct Unit {
    int head, strip, sees, all, some;  // this lane's query sees the keys below `sees`, all of the unit's those below `all`, one at least those below `some`
    bool there;
};
__device__ __forceinline__ Unit unit_of(const Args& a, int unit, int bkv, int off, int qlen, int n)
{
    Unit u;
    u.strip = unit / a.G;
    u.head = (bkv % a.Hkv) * a.G + unit % a.G;
    const int row = 32 * u.strip + n;
    u.there = row < qlen;
    u.sees = u.there ? off + row : 0;
    u.all = max(0, off + 32 * u.strip);
    u.some = 32 * u.strip < qlen ? max(0, off + min(32 * u.strip + 32, qlen) - 1) : 0;
    return u;
}

template <int D> struct Cfg {
    static constexpr int ROW = 2 * D, CPR = ROW / 16, BLK_ROWS = 1024 / ROW;
    static constexpr int SUB = 32 * ROW;                // bytes of 32 rows
    static constexpr int LOADS = SUB / 1024;            // loads of a wave for 32 rows
};

// 32 rows to LDS, swizzled, those past `last` as that one; every lane's offsets in off
template <int D> __device__ __forceinline__ void sub_offsets(int (&off)[Cfg<D>::LOADS], int lane)
{
    using C = Cfg<D>;
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) {
        const int r = i * C::BLK_ROWS + lane / C::CPR;
        off[i] = r * C::ROW + (((lane % C::CPR) ^ swz_perm<D>(r)) << 4);
    }
}
template <int D> __device__ __forceinline__ void sub_to_lds(const uint16_t* src, const int (&off)[Cfg<D>::LOADS], int last, const char* dst, int lane)
{
    using C = Cfg<D>;
    if (last >= 31) dma16_to_lds_run(src, off, dst);
    else {
        int o[C::LOADS];
#pragma unroll
        for (int i = 0; i < C::LOADS; ++i) o[i] = off[i] - max(i * C::BLK_ROWS + lane / C::CPR - last, 0) * C::ROW;
        dma16_to_lds_run(src, o, dst);
    }
}

// B operand of the logits from 32 rows of q in LDS; zero where there is no row: what lies there may be anything
template <int D> __device__ __forceinline__ void read_q(bf16x8 (&qf)[D / 16], uint32_t at, int n, int hh, bool there)
{
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        u32x4 y = lds_load16(at + tile_off_perm<D>(n, 2 * s + hh));
        if (!there) y = u32x4{0u, 0u, 0u, 0u};
        qf[s] = __builtin_bit_cast(bf16x8, y);
    }
}

// of N in all: NU units' with the subtiles of keys at `at` and from there down
template <int D, int NU, int N> __device__ __forceinline__ void logits(f32x16 (&s)[N], const bf16x8 (&qf)[NU][D / 16], const uint32_t (&aoff)[D / 16], uint32_t at)
{
    static_assert(NU == 1 || NU == N, "one unit, or one subtile");
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[j][r] = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
            s[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, lds_load16(aoff[i] + at - (NU == 1 ? j : 0) * Cfg<D>::SUB)), qf[NU == 1 ? 0 : j][i], s[j], 0, 0, 0);
}

// WHAT: 0 the weights of all keys, 1 what a chunk of keys leaves of the sticks, 2 the weights of a chunk
// NU: units of a wave.  One: it takes both halves of a tile at once.  Two: a half for both units, which read K once and add their weights up before they
// are summed over the lanes (a unit's vector instructions are a fifth fewer, but a tile takes a workgroup longer).
template <int D, int WHAT, int NU>
__global__ void __launch_bounds__(64 * NW, 2)
key_weight_kernel(const Args a, int BHkv, int first_wg)
{
    using C = Cfg<D>;
    constexpr int TILE = 2 * C::SUB, NPW = TILE / 1024 / NW;
    __shared__ __attribute__((aligned(1024))) char tiles[2 * TILE];         // of K; before that, the units' q
    static_assert(2 * TILE == NW * C::SUB, "room for q");
    __shared__ __attribute__((aligned(16))) float csum[2][NW][TK];
    __shared__ __attribute__((aligned(16))) int s_done[2][NW];

    // The longest first; kv heads turn as workgroups go round the chip, so that a CU does not get the same one, which may be the one that reaches far, each time
    const int wg = first_wg + blockIdx.x, chunk = WHAT ? blockIdx.y : 0;
    const int turn = wg / BHkv, at = a.groups - 1 - turn, grp = a.first + at;
    const int bkv = (wg % BHkv + (int)((long)turn * BHkv / 256 % BHkv)) % BHkv;
    const int b = bkv / a.Hkv;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int len = length_of(a.lens, b, a.T), qlen = length_of(a.qlens, b, a.Tq);
    const int off = len - qlen;                                         // position of query row 0
    const int unit = (grp * NW + wave) * NU;
    int* const reach = a.reach + (((long)bkv * a.groups + at) * a.chunks + chunk) * 2;
    double* const left = a.left + (((long)bkv * a.groups * NW + unit) * a.chunks) * 32 + n;       // of chunk 0
    Unit u[NU];
    double stick[NU];
    int all_see = INT_MAX, some_see = 0;                                // (as Unit's)
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        u[i] = unit_of(a, unit + i, bkv, off, qlen, n);
        stick[i] = u[i].there ? 1.0 : 0.0;
        all_see = min(all_see, u[i].all);
        some_see = max(some_see, u[i].some);
    }
    auto left_of = [&]() __attribute__((always_inline)) { return NU == 1 ? stick[0] : stick[0] + stick[NU - 1]; };
    const int last_strip = min(((grp + 1) * NW * NU - 1) / a.G, (qlen - 1) / 32);            // of the workgroup, with rows in it
    const int lo = WHAT ? chunk * a.C : 0;
    int top = grp * NW * NU / a.G * 32 < qlen ? max(0, off + min(32 * last_strip + 32, qlen) - 1) : 0;
    if (WHAT) top = min(top, lo + a.C);
    if (top <= lo) {
        if (WHAT == 1 && hh == 0) left[chunk * 32] = stick[0];
        if (WHAT != 1 && tid == 0) reach[0] = reach[1] = 0;
        return;
    }
    int qoff[C::LOADS];
    sub_offsets<D>(qoff, lane);
    auto fetch_q = [&](const Unit& u) __attribute__((always_inline)) {
        const int r0 = min(32 * u.strip, (a.Tq - 1) / 32 * 32);
        sub_to_lds<D>(a.q + (((long)b * a.H + u.head) * a.Tq + r0) * D, qoff, a.Tq - 1 - r0, tiles + wave * C::SUB, lane);
    };
    fetch_q(u[0]);
    if constexpr (WHAT == 2) {
        // what the nearer chunks left: every second one a half-wave's, eight loads at once
        constexpr int EACH = 8;
        double mine = 1.0;
        for (int c = a.chunks - 1 - hh; c > chunk; c -= 2 * EACH) {
            double x[EACH];
#pragma unroll
            for (int i = 0; i < EACH; ++i) x[i] = left[max(c - 2 * i, chunk + 1) * 32];
#pragma unroll
            for (int i = 0; i < EACH; ++i) mine *= c - 2 * i > chunk ? x[i] : 1.0;
        }
        stick[0] *= mine * other_half(mine);
        const int done = none_left(stick[0]) ? -1 : 0;
        if (lane == 0) s_done[0][wave] = done;
        barrier_lds();
        if (waves_done(s_done[0])) {
            if (tid == 0) reach[0] = reach[1] = 0;
            dma_wait<0>();
            return;
        }
    }

    const float c2 = SB_LOG2E / sqrtf((float)D);
    const uint32_t smem0 = lds_offset(tiles);
    bf16x8 qf[NU][D / 16];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        if (i > 0) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // (the rows before have been read)
            fetch_q(u[i]);
        }
        dma_wait<0>();
        read_q<D>(qf[i], smem0 + wave * C::SUB, n, hh, u[i].there);
    }
    barrier_lds();
    const uint16_t* const kg = reinterpret_cast<const uint16_t*>(scalar_base(a.k + (long)bkv * a.Tcap * D));
    int goff[NPW];
#pragma unroll
    for (int i = 0; i < NPW; ++i) {
        const int r = (wave * NPW + i) * C::BLK_ROWS + lane / C::CPR;
        goff[i] = r * C::ROW + (((lane % C::CPR) ^ swz_perm<D>(r)) << 4);
    }
    auto stage = [&](int jt, int st) __attribute__((always_inline)) {
        const uint16_t* src = kg + (long)jt * TK * D;
        char* dst = tiles + st * TILE + wave * NPW * 1024;
        if ((jt + 1) * TK <= len) dma16_to_lds_run(src, goff, dst);
        else dma16_to_lds_run_clamped<C::ROW, C::BLK_ROWS>(src, goff, wave * NPW * C::BLK_ROWS + lane / C::CPR, len - 1 - jt * TK, dst);
    };
    uint32_t aoff[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) aoff[s] = smem0 + tile_off_perm<D>(perm_row(n), 2 * s + hh);

    const int jt0 = (top - 1) / TK, jend = lo / TK;
    float* const part = a.part + ((long)bkv * a.groups + at) * a.Tpad;
    auto flush = [&](int jt, int par) __attribute__((always_inline)) {
        if (tid < TK) part[(long)jt * TK + tid] = (csum[par][0][tid] + csum[par][1][tid]) + (csum[par][2][tid] + csum[par][3][tid]);
    };
    stage(jt0, 0);
    int jt = jt0;
    // tile jt, in buffer PAR; whether another follows
    auto tile = [&](auto buffer) __attribute__((always_inline)) {
        constexpr int par = decltype(buffer)::value;
        dma_wait<0>();
        barrier_lds();
        if (jt < jt0) {
            if (WHAT != 1) flush(jt + 1, par ^ 1);
            if (jt < jend || waves_done(s_done[par ^ 1])) return false;
        }
        if (jt > jend) stage(jt - 1, par ^ 1);
        float sum[2] = {0.0f, 0.0f};                       // of the nearer half, of the farther
#pragma unroll
        for (int half = 0; half < NU; ++half) {            // (one unit: both at once)
            const int base = jt * TK + 32 - 32 * half;
            if ((NU == 1 ? base - 32 : base) >= some_see || none_left(left_of())) continue;
            f32x16 s[2];
            float w[2][16];
            float mine[2];
            Taken t[2];
            logits<D, NU>(s, qf, aoff, par * TILE + (1 - half) * C::SUB);
            const int seen[2] = {u[0].sees - base - 16 * hh, (NU == 1 ? u[0].sees + 32 : u[NU - 1].sees) - base - 16 * hh};
            if (base + 32 > all_see) weights<true>(s, c2, seen, hh, w, mine, t);
            else weights<false>(s, c2, seen, hh, w, mine, t);
            if constexpr (NU == 1) {
                if constexpr (WHAT != 1) {
                    mine[0] *= (float)stick[0];
                    mine[1] *= (float)stick[0] * t[0].all;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) w[i][r] *= mine[i];
                        sum[i] = sums_of_lanes(w[i], n);
                    }
                }
                stick[0] = passed(stick[0], both(t[0], t[1]));
            } else {
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    mine[i] *= (float)stick[i];
                    stick[i] = passed(stick[i], t[i]);
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) w[0][r] = w[0][r] * mine[0] + w[1][r] * mine[1];
                sum[half] = sums_of_lanes(w[0], n);
            }
        }
        if (WHAT != 1 && (n & 1) == 0) {
            csum[par][wave][32 + 16 * hh + key_of_lane(n)] = sum[0];
            csum[par][wave][16 * hh + key_of_lane(n)] = sum[1];
        }
        const int done = none_left(left_of()) ? -1 : 0;
        if (lane == 0) s_done[par][wave] = done;
        --jt;
        return true;
    };
    while (tile(std::integral_constant<int, 0>()) && tile(std::integral_constant<int, 1>())) {}
    if (WHAT == 1 && hh == 0) left[chunk * 32] = stick[0];
    if (WHAT != 1 && tid == 0) {
        reach[0] = (jt + 1) * TK;
        reach[1] = (jt0 + 1) * TK;
    }
}

template <int D>
__global__ void __launch_bounds__(64 * SNW, 2)
key_weight_small_kernel(const Args a)
{
    using C = Cfg<D>;
    __shared__ __attribute__((aligned(1024))) char rows[SNW * C::SUB];      // 32 of K a wave
    __shared__ __attribute__((aligned(1024))) char qrows[C::SUB];
    __shared__ __attribute__((aligned(16))) Taken prod[2][SNW][32];         // per round parity: a wave's keys
    const int at = a.groups - 1 - (int)blockIdx.x, unit = a.first + at, bkv = blockIdx.y;
    const int b = bkv / a.Hkv;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int len = length_of(a.lens, b, a.T), qlen = length_of(a.qlens, b, a.Tq);
    const Unit u = unit_of(a, unit, bkv, len - qlen, qlen, n);
    int* const reach = a.reach + ((long)bkv * a.groups + at) * 2;
    double stick = u.there ? 1.0 : 0.0;
    if (u.some == 0) {
        if (tid == 0) reach[0] = reach[1] = 0;
        return;
    }

    const float c2 = SB_LOG2E / sqrtf((float)D);
    int off[C::LOADS];
    sub_offsets<D>(off, lane);
    const uint16_t* const kg = reinterpret_cast<const uint16_t*>(scalar_base(a.k + (long)bkv * a.Tcap * D));
    const char* const mine_at = rows + wave * C::SUB;
    auto fetch = [&](int base) __attribute__((always_inline)) {
        base = max(base, 0);
        sub_to_lds<D>(kg + (long)base * D, off, len - 1 - base, mine_at, lane);
    };
    // q: every wave some of the loads
    if (wave < C::LOADS) {
        const int r = wave * C::BLK_ROWS + lane / C::CPR, r0 = 32 * u.strip;
        dma16_to_lds_saddr(a.q + (((long)b * a.H + u.head) * a.Tq + r0) * D,
                           min(r, a.Tq - 1 - r0) * C::ROW + (((lane % C::CPR) ^ swz_perm<D>(r)) << 4), qrows + wave * 1024);
    }
    const int hi0 = (u.some + 31) & ~31;
    int hi = hi0;
    fetch(hi - 32 * (wave + 1));
    uint32_t aoff[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) aoff[s] = lds_offset(mine_at) + tile_off_perm<D>(perm_row(n), 2 * s + hh);
    dma_wait<C::LOADS>();
    barrier_lds();
    bf16x8 qf[1][D / 16];
    read_q<D>(qf[0], lds_offset(qrows), n, hh, u.there);

    float* const part = a.part + ((long)bkv * a.groups + at) * a.Tpad;
    for (int par = 0; hi > 0; par ^= 1) {
        const int base = hi - 32 * (wave + 1);
        dma_wait<0>();
        f32x16 s[1];
        logits<D, 1>(s, qf, aoff, 0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // (the rows have been read)
        if (hi > 32 * SNW) fetch(base - 32 * SNW);
        float w[1][16];
        float mine[1] = {0.0f};
        Taken t[1] = {{1.0f, 0.0f}};
        if (base >= 0) {
            if (base + 32 > u.all) weights<true>(s, c2, {u.sees - base - 16 * hh}, hh, w, mine, t);
            else weights<false>(s, c2, {0}, hh, w, mine, t);
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) w[0][r] = 0.0f;
        }
        if (hh == 0) prod[par][wave][n] = t[0];
        barrier_lds();
        float before = (float)stick;
        Taken round = {1.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < SNW; ++j) {
            if (j == wave) before *= round.all;
            round = both(round, prod[par][j][n]);
        }
        stick = passed(stick, round);
        if (base >= 0) {
            mine[0] *= before;
#pragma unroll
            for (int r = 0; r < 16; ++r) w[0][r] *= mine[0];
            const float sum = sums_of_lanes(w[0], n);
            if ((n & 1) == 0) part[base + 16 * hh + key_of_lane(n)] = sum;
        }
        hi -= 32 * SNW;
        if (none_left(stick)) break;
    }
    if (tid == 0) {
        reach[0] = max(hi, 0);
        reach[1] = hi0;
    }
    dma_wait<0>();                             // (rows asked for before the end was known)
}

// Groups by wave in turn, 64 keys a workgroup: a wave asks for four groups' numbers at a time, and how far a group reaches is the same for all its lanes.
template <int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
key_weight_sum_kernel(const Args a)
{
    __shared__ float sums[WAVES][64];
    const int bkv = blockIdx.y, lane = threadIdx.x & 63, key = blockIdx.x * 64 + lane;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int len = length_of(a.lens, bkv / a.Hkv, a.T);
    if ((int)blockIdx.x * 64 >= len) return;
    const float* part = a.part + (long)bkv * a.groups * a.Tpad + key;
    const int2* reach = reinterpret_cast<const int2*>(a.reach) + (long)bkv * a.groups * a.chunks + blockIdx.x * 64 / a.C;
    float s = 0.0f;
    for (int g0 = wave; g0 < a.groups; g0 += SUM_DEEP * WAVES) {
        int2 r[SUM_DEEP];
        float x[SUM_DEEP];
#pragma unroll
        for (int i = 0; i < SUM_DEEP; ++i) r[i] = reach[(long)min(g0 + i * WAVES, a.groups - 1) * a.chunks];
#pragma unroll
        for (int i = 0; i < SUM_DEEP; ++i) {
            x[i] = 0.0f;
            if (g0 + i * WAVES < a.groups && key >= r[i].x && key < r[i].y) x[i] = part[(long)(g0 + i * WAVES) * a.Tpad];
        }
#pragma unroll
        for (int i = 0; i < SUM_DEEP; ++i) s += x[i];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && key < len) {
        s = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += sums[w][lane];
        const long at = (long)bkv * a.Tcap + key;
        a.score_out[at] = (a.score ? a.score[at] : 0.0f) + s;
    }
}

template <int D> hipError_t launch_d(const Args& a, const Plan& p, int BHkv, hipStream_t stream)
{
    if (p.small) {
        hipLaunchKernelGGL((key_weight_small_kernel<D>), dim3((unsigned)a.groups, (unsigned)BHkv), dim3(64 * SNW), 0, stream, a);
        return hipGetLastError();
    }
    if (a.chunks == 1)
        return launch_workgroups((long)BHkv * a.groups, 64 * NW, [&](unsigned wgs, int first) {
            if (p.pairs) hipLaunchKernelGGL((key_weight_kernel<D, 0, 2>), dim3(wgs), dim3(64 * NW), 0, stream, a, BHkv, first);
            else hipLaunchKernelGGL((key_weight_kernel<D, 0, 1>), dim3(wgs), dim3(64 * NW), 0, stream, a, BHkv, first);
        });
    const dim3 grid((unsigned)(BHkv * a.groups), (unsigned)a.chunks), threads(64 * NW);
    hipLaunchKernelGGL((key_weight_kernel<D, 1, 1>), grid, threads, 0, stream, a, BHkv, 0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((key_weight_kernel<D, 2, 1>), grid, threads, 0, stream, a, BHkv, 0);
    return hipGetLastError();
}

}  // namespace

size_t key_weight_workspace_bytes(int B, int H, int Hkv, int Tq, int T)
{
    return sizeof(float) * plan_of(B, H, Hkv, Tq, T).floats(B * Hkv);
}

hipError_t launch_key_weight(const uint16_t* q, const uint16_t* k, const int* lens, const int* qlens, const float* score, float* score_out,
                             float* workspace, int B, int H, int Hkv, int Tq, int T, int Tcap, int d, hipStream_t stream)
{
    const Plan p = plan_of(B, H, Hkv, Tq, T);
    const int BHkv = B * Hkv, most = p.at_once(BHkv);
    Args a = {q, k, lens, qlens, score, score_out, workspace, nullptr, nullptr, H, Hkv, H / Hkv, Tq, T, Tcap, p.Tpad, most, p.chunks, p.C, 0};
    a.left = reinterpret_cast<double*>(workspace + (size_t)BHkv * most * p.Tpad);
    a.reach = reinterpret_cast<int*>(a.left + BHkv * p.left_of());
    for (; a.first < p.groups; a.first += most) {
        a.groups = std::min(most, p.groups - a.first);
        hipError_t e = d == 32 ? launch_d<32>(a, p, BHkv, stream) : d == 64 ? launch_d<64>(a, p, BHkv, stream) : launch_d<128>(a, p, BHkv, stream);
        if (e != hipSuccess) return e;
        // no more waves than have a group to add (B4 H16 T8192 d64, 128 rows, 4 groups: 9 us in all with one wave, 15.5 with eight)
        auto sum = [&](auto kernel, int waves) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)((T + 63) / 64), (unsigned)BHkv), dim3(64 * waves), 0, stream, a);
        };
        if (a.groups <= SUM_DEEP) sum(key_weight_sum_kernel<1>, 1);
        else if (a.groups <= 2 * SUM_DEEP) sum(key_weight_sum_kernel<2>, 2);
        else sum(key_weight_sum_kernel<8>, 8);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        a.score = score_out;                               // the groups before
    }
    return hipSuccess;
}

}  // namespace sb
