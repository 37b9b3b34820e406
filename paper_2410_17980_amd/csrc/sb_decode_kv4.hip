// Single-token decode on a 4-bit cache (sb_kv4.h): one new query per (entry, head) against the entry's keys and values, and the
// weight that its heads give every key, added to the key's score.
//
// One pass over the cache, 2 (D / 2 + D / 32) bytes a key and kv head (136 at D = 128, 512 in bf16).  Chunks of keys combine as in
// sb_decode.hip: a chunk's weights are taken as if nothing nearer were there, and are shifted afterwards by what the nearer chunks
// took (Eq. 2).
//   near launch      grid (kv head, block of query heads): the nearest keys, all of a short cache
//   far launch       grid (chunk, kv head, block of query heads): the keys before those; returns at once where the nearest keys
//                    have used up the stick (CARRY_EXHAUSTED: every farther weight is zero in fp32)
//   combine launch   a workgroup per query head adds the chunks up in a fixed order; with scores, one per (kv head, chunk)
//                    shifts the weights of its keys, sums them over the group's heads and adds the score
//
// A workgroup takes its keys from the nearest down in rounds of R tiles of 32 per wave, wave 0 the nearest.
//   logits   z[key][head] = K q: 16x16x32 bf16 MFMA, A = 16 rows of K, B = the query heads of the group.  A lane loads the D / 8
//            bytes of its row that make up one A operand after the other (the order of the columns is free as long as q comes in
//            the same one), and converts them in registers, the scale with them.  Rows go to the MFMAs so that a lane gets eight
//            consecutive keys of a head.
//   weights  where the MFMA leaves the logits: Eq. 1's product over the lane's eight keys, then across the four lanes of a tile,
//            the tiles and the waves (by LDS, one barrier a round).  What is left of the stick is carried as it is, not by its
//            logarithm: the keys' scores are results in fp32.  From less than 2^-126 of it on, weights are subnormal at most and count as zero.
//   output   O^T[c][head] += V^T w: a lane's eight weights are the B operand as they lie; it loads D / 16 columns of those same
//            eight rows of V, converts, and an in-register transposition (one v_perm per packed pair) makes the A operands.
// The 16 columns of the MFMAs are more than most groups have heads.  Their copies of a head take a tile each (R of them), which
// divides the vector instructions of the weights by R, and the upper 8 bits of a weight or the 8 below (o gets 16 bits of a weight; o itself has
// 8), which halves the MFMAs of the output; the columns of a head are added up at the end.
#include "sb_kernels.h"
#include "sb_kv4.h"
#include "sb_mma.h"

namespace sb {
namespace {

constexpr int GMAX = 16;               // query heads of a group per workgroup: the columns of the MFMA
constexpr int KW = 32;                 // keys of a tile
constexpr int NEAR_NW = 8, FAR_NW = 4;
constexpr int NEAR = KW * NEAR_NW;     // keys of a near launch that has a far one behind it
constexpr float LEAST = 0x1p-126f;     // of the stick
constexpr int ALONE = 2048;            // a cache is the near launch's alone up to here
constexpr int MAXSLOT = 128;           // chunks, the nearest keys among them: two per lane of a wave
constexpr long FAR_WGS = 4096;         // workgroups of the far launch, all heads together
constexpr int MOST_GROUP = 1024;       // query heads of a kv head where scores are wanted
constexpr int COMBINE_THREADS = 256;

struct Args {
    const uint16_t* q;
    const uint8_t *kc, *ks, *vc, *vs;
    const uint16_t* rb;
    const int* lens;                   // rows per entry, or nullptr: T
    const float* score;                // nullptr: zero
    float* score_out;                  // nullptr: not wanted
    uint16_t* o;
    float* m;
    float *part_o, *part_a, *part_l;   // [heads][slots][D], [heads][slots]: slot 0 the nearest; share of the stick that it leaves, and -log2 of that where m is wanted
    float* wl;                         // [heads][Tcap]: weights inside their chunk, where scores are combined
    int T, Tcap, Hkv, G, near, C, slots;
    int lg;                            // log2 of the columns that a copy of the heads takes
};

__device__ __forceinline__ int length_of(const Args& a, int b)
{
    return a.lens ? min(max(a.lens[b], 0), a.T) : a.T;
}
__device__ __forceinline__ int up32(int n) { return (n + 31) & ~31; }

template <int CTRL> __device__ __forceinline__ float dpp(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
// sum over the 16 lanes of a row, in all of them
__device__ __forceinline__ float row_sum(float x)
{
    x += dpp<0xB1>(x);                 // quad_perm 1, 0, 3, 2
    x += dpp<0x4E>(x);                 // quad_perm 2, 3, 0, 1
    x += dpp<0x141>(x);                // row_half_mirror
    return x + dpp<0x140>(x);          // row_mirror
}
__device__ __forceinline__ float wave_sum(float x)
{
    x = row_sum(x);
    float a, b;
    both_halves(x + __shfl_xor(x, 16), a, b);
    return a + b;
}

// product over the lanes below this one, and over all in `total`
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_or_one(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0x3f800000, __builtin_bit_cast(int, x), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float wave_prefix(float v, float& total)
{
    v *= dpp_or_one<0x111, 0xF>(v);                       // row_shr:1, 2, 4, 8
    v *= dpp_or_one<0x112, 0xF>(v);
    v *= dpp_or_one<0x114, 0xF>(v);
    v *= dpp_or_one<0x118, 0xF>(v);
    v *= dpp_or_one<0x142, 0xA>(v);                       // row_bcast:15 into rows 1 and 3
    v *= dpp_or_one<0x143, 0xC>(v);                       // row_bcast:31 into rows 2 and 3
    total = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
    return dpp_or_one<0x138, 0xF>(v);                     // wave_shr:1
}

// `even`: v of this lane's column in row 0 (lanes 0 .. 31) or 2 (32 .. 63), `odd`: in row 1 or 3
__device__ __forceinline__ void both_rows(float v, float& even, float& odd)
{
    auto sw = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), false, false);
    even = __builtin_bit_cast(float, (int)sw[0]);
    odd = __builtin_bit_cast(float, (int)sw[1]);
}

// what a lane loads of a tile
template <int D> struct KTile {
    uint32_t k[2][D / 32];             // rows 8 (l16 / 4) + 4 h + l16 % 4: columns lq D / 4 .. + D / 4 - 1
    uint32_t s[2];                     // and their scale
};
template <int D> struct VTile {
    uint32_t v[8];                     // rows 8 lq + i: columns D / 16 l16 .. + D / 16 - 1
    uint32_t s[D / 16];                // scales of the eight rows, bytes as they lie
};

template <class V> __device__ __forceinline__ V load_as(const uint8_t* p)
{
    V x;
    __builtin_memcpy(&x, p, sizeof(V));
    return x;
}
// N words from p on
template <int N> __device__ __forceinline__ void load_words(uint32_t (&w)[N], const uint8_t* p)
{
    if constexpr (N == 1) {
        w[0] = load_as<uint32_t>(p);
    } else if constexpr (N == 2) {
        const uint2 x = load_as<uint2>(p);
        w[0] = x.x;
        w[1] = x.y;
    } else {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const u32x4 x = load_as<u32x4>(p + 4 * j);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[j + i] = x[i];
        }
    }
}

template <int D> __device__ __forceinline__ void fetch_k(KTile<D>& t, const uint8_t* kc, const uint8_t* ks, int base, int l16, int lq)
{
    constexpr int ROW = D / 2, SROW = D / KV4_BLOCK;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = base + 8 * (l16 >> 2) + 4 * h + (l16 & 3);
        load_words(t.k[h], kc + (long)row * ROW + lq * (ROW / 4));
        t.s[h] = ks[(long)row * SROW + lq * SROW / 4];
    }
}
template <int D> __device__ __forceinline__ void fetch_v(VTile<D>& t, const uint8_t* vc, const uint8_t* vs, int base, int l16, int lq)
{
    constexpr int ROW = D / 2, SROW = D / KV4_BLOCK;
    const long row = base + 8 * lq;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint8_t* p = vc + (row + i) * ROW + l16 * (ROW / 16);
        t.v[i] = D == 128 ? load_as<uint32_t>(p) : D == 64 ? load_as<uint16_t>(p) : *p;
    }
    load_words(t.s, vs + row * SROW);
}

// scale of row i, of this lane's columns (exponent bits; what stands below them does not count)
template <int D> __device__ __forceinline__ uint32_t v_scale(const VTile<D>& t, int i, int l16)
{
    constexpr int PER = 128 / D;       // rows in a word
    // byte of the row's first block: i % PER * D / 32; of this lane's block: + l16 D / 16 / 32
    const int sh = 24 - 8 * ((i % PER) * (D / KV4_BLOCK)) - 8 * (l16 * (D / 16) / KV4_BLOCK);
    return (t.s[i / PER] << sh) >> 1;
}

// R: tiles of a wave and round.  PIECES: the columns' copies take a weight's upper and lower bits; without, two MFMAs do
template <int D, bool FAR, int R, bool PIECES>
__global__ void __launch_bounds__(64 * (FAR ? FAR_NW : NEAR_NW), 2)
decode_kv4_kernel(const Args a)
{
    constexpr int NW = FAR ? FAR_NW : NEAR_NW;
    constexpr int NTHR = 64 * NW;
    constexpr int NT = NW * R;             // tiles of a round
    constexpr int KEYS = KW * NT;
    constexpr int CW = D / 16;             // columns of V per lane
    constexpr int CH = D / 4;              // 16-byte chunks of a head's columns
    __shared__ __attribute__((aligned(16))) float tot[2][GMAX][NT];      // per round parity: what a tile leaves of the stick
    __shared__ float s_log[NW][GMAX];
    __shared__ __attribute__((aligned(16))) f32x4 ored[NW * GMAX * CH];

    const int bkv = FAR ? blockIdx.y : blockIdx.x;     // entry * Hkv + kv head
    const int g0 = blockIdx.z * GMAX;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, lq = lane >> 4;
    const int b = bkv / a.Hkv;
    const int len = length_of(a, b), end = up32(len);
    const int slot = FAR ? (int)blockIdx.x + (a.near > 0) : 0;
    const int top = FAR ? end - a.near - (int)blockIdx.x * a.C : end;
    const int lo = max(0, FAR ? top - a.C : top - a.near);
    const long hq0 = (long)bkv * a.G + g0;
    const int live = min(GMAX, a.G - g0);
    // this lane's column: head l16 % 2^lg, copy l16 / 2^lg
    const int hc = l16 & ((1 << a.lg) - 1), copy = l16 >> a.lg;
    const int mytile = R == 1 ? 0 : copy & (R - 1);
    const bool lower = PIECES && (copy / R & 1);
    const bool first = copy < R && hc < live;          // one column for each tile and head
    const long head = hq0 + min(hc, live - 1);
    const float c2 = SB_LOG2E / sqrtf((float)D);

    if constexpr (FAR) {
        if (top <= 0) return;
        if (!a.m && a.near > 0 && __builtin_amdgcn_ballot_w64(!(a.part_a[head * a.slots] < LEAST)) == 0) return;
    }

    const uint8_t* const kc = a.kc + (long)bkv * a.Tcap * (D / 2);
    const uint8_t* const vc = a.vc + (long)bkv * a.Tcap * (D / 2);
    const uint8_t* const ks = a.ks + (long)bkv * a.Tcap * (D / KV4_BLOCK);
    const uint8_t* const vs = a.vs + (long)bkv * a.Tcap * (D / KV4_BLOCK);

    bf16x8 qw[D / 32];                     // B operand
#pragma unroll
    for (int s = 0; s < D / 32; ++s) qw[s] = *reinterpret_cast<const bf16x8*>(a.q + head * D + lq * (D / 4) + 8 * s);

    f32x4 acc[CW];                         // O^T: row 4 lq + r of MFMA e is column CW (4 lq + r) + e, column l16
#pragma unroll
    for (int e = 0; e < CW; ++e) acc[e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float stick = 1.0f, logs = 0.0f;       // left by the keys already passed; -log2 of what this lane's own keys left
    int par = 0, hi = top;
    KTile<D> kt[R];
    VTile<D> vt[R];
    // tile j of this wave; where that is below lo there is none, and the last one is loaded
    auto base_of = [&](int j) __attribute__((always_inline)) { return hi - KW * (wave * R + j + 1); };
    auto valid_of = [&](int j) __attribute__((always_inline)) { return base_of(j) < lo ? 0 : len - base_of(j); };

    // one round; whether another follows
    auto round = [&]() __attribute__((always_inline)) {
        const bool more = hi - KEYS > lo;
        // ---- logits of the lane's eight keys, in base 2
        float x[8];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int valid = valid_of(j);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
                const uint32_t s = kt[j].s[h] << 23;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const uint32_t w = kt[j].k[h][i];
                    const u32x4 p = {kv4_pair<0>(w, s), kv4_pair<1>(w, s), kv4_pair<2>(w, s), kv4_pair<3>(w, s)};
                    z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p), qw[i], z, 0, 0, 0);
                }
                if (valid < KW)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[r] = 8 * lq + 4 * h + r < valid ? z[r] : -INFINITY;
#pragma unroll
                for (int r = 0; r < 4; ++r) x[4 * h + r] = j == 0 || mytile == j ? z[r] : x[4 * h + r];
            }
        }
        if (more) {
#pragma unroll
            for (int j = 0; j < R; ++j) fetch_k<D>(kt[j], kc, ks, max(base_of(j) - KEYS, lo), l16, lq);
        }
        // ---- the lane's chain: w[i] = e_i prod_{i' < i} (1 + e_i'), e = sigma / (1 - sigma); norm makes it the weight where the stick is whole
        // before the lane's nearest key, `leave` is what the eight keys leave
        float w[8], norm, leave;
        float W = 1.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] *= c2;
            w[i] = W * fast_exp2(x[i]);
            W += w[i];
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(W < 0x1p120f)) == 0, 1)) {
            norm = leave = __builtin_amdgcn_rcpf(W);
            if (a.m) logs += fast_log2(W);
        } else {                           // in the log form
            float run = 0.0f;
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                run += sp2(x[i]);
                w[i] = fast_exp2(x[i] - run);
            }
            norm = 1.0f;
            leave = fast_exp2(-run);
            logs += run;
        }
        // ---- across the four lanes of a tile (the odd one of a pair and the upper half are nearer), the tiles and waves
        float even, odd, lowhalf, upphalf;
        both_rows(leave, even, odd);
        both_halves(even * odd, lowhalf, upphalf);
        norm *= ((lq & 1) ? 1.0f : odd) * (lq < 2 ? upphalf : 1.0f);
        if (lq == 0 && first) tot[par][hc][wave * R + mytile] = lowhalf * upphalf;
        barrier_lds();
        float before = stick;
        const int mine = wave * R + mytile;
#pragma unroll
        for (int j = 0; j < NT; j += 4) {
            const f32x4 p = *reinterpret_cast<const f32x4*>(&tot[par][min(hc, live - 1)][j]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                before *= j + i < mine ? p[i] : 1.0f;
                stick *= p[i];
            }
        }
        norm *= before;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] *= norm;
        if (a.score_out) {
            const int base = hi - KW * (mine + 1);
            if (a.wl) {
                if (first && base >= lo) {
                    float* p = a.wl + (hq0 + hc) * a.Tcap + base + 8 * lq;
                    *reinterpret_cast<f32x4*>(p) = f32x4{w[0], w[1], w[2], w[3]};
                    *reinterpret_cast<f32x4*>(p + 4) = f32x4{w[4], w[5], w[6], w[7]};
                }
            } else if constexpr (!FAR) {   // (R = 1)
                f32x4 s[2];
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i / 4][i % 4] = row_sum(first ? w[i] : 0.0f);
                if (l16 < 2 && base >= lo) {
                    const int key = base + 8 * lq + 4 * l16;
                    const long at = (long)bkv * a.Tcap + key;
                    const f32x4 own = l16 ? s[1] : s[0];
                    if (key + 4 <= len) {
                        const f32x4 was = a.score ? *reinterpret_cast<const f32x4*>(a.score + at) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                        *reinterpret_cast<f32x4*>(a.score_out + at) = was + own;
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (key + r < len) a.score_out[at + r] = (a.score ? a.score[at + r] : 0.0f) + own[r];
                    }
                }
            }
        }
        // ---- output
        bf16x8 w0, w1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w0[i] = (__bf16)w[i];
            const float rest = w[i] - (float)w0[i];
            if (PIECES) w0[i] = (__bf16)(lower ? rest : w[i]);
            else w1[i] = (__bf16)rest;
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int valid = valid_of(j);
            bf16x8 wb = w0;
            if (R > 1) {
                u32x4 y = __builtin_bit_cast(u32x4, w0);
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = mytile == j ? y[i] : 0u;
                wb = __builtin_bit_cast(bf16x8, y);
            }
            uint32_t pv[8][CW / 2];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t s = v_scale<D>(vt[j], i, l16);
                if (valid < KW && 8 * lq + i >= valid) s = 0x3f800000u;        // (whatever lies there, a zero weight makes it zero)
                const uint32_t v = vt[j].v[i];
                pv[i][0] = kv4_pair<0>(v, s);
                if constexpr (CW >= 4) pv[i][1] = kv4_pair<1>(v, s);
                if constexpr (CW >= 8) {
                    pv[i][2] = kv4_pair<2>(v, s);
                    pv[i][3] = kv4_pair<3>(v, s);
                }
            }
#pragma unroll
            for (int e = 0; e < CW; ++e) {
                u32x4 y;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    y[i] = __builtin_amdgcn_perm(pv[2 * i + 1][e >> 1], pv[2 * i][e >> 1], (e & 1) ? 0x07060302u : 0x05040100u);
                const bf16x8 av = __builtin_bit_cast(bf16x8, y);
                if (!PIECES) acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, w1, acc[e], 0, 0, 0);
                acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, wb, acc[e], 0, 0, 0);
            }
        }
        if (more) {
#pragma unroll
            for (int j = 0; j < R; ++j) fetch_v<D>(vt[j], vc, vs, max(base_of(j) - KEYS, lo), l16, lq);
        }
        hi -= KEYS;
        par ^= 1;
        return more && (FAR || a.m || __builtin_amdgcn_ballot_w64(!(stick < LEAST)) != 0);
    };
    if (hi > lo) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            fetch_k<D>(kt[j], kc, ks, max(base_of(j), lo), l16, lq);
            fetch_v<D>(vt[j], vc, vs, max(base_of(j), lo), l16, lq);
        }
        while (round()) {}
    }
    // keys that no stick was left for keep their scores
    if (!FAR && a.score_out && !a.wl && a.score_out != a.score)
        for (int i = lo + tid; i < hi; i += NTHR) a.score_out[(long)bkv * a.Tcap + i] = a.score ? a.score[(long)bkv * a.Tcap + i] : 0.0f;
    if (!FAR && a.wl && a.slots == 1)                      // (read by the combination)
        for (int g = 0; g < live; ++g)
            for (int i = lo + tid; i < hi; i += NTHR) a.wl[(hq0 + g) * a.Tcap + i] = 0.0f;

    // ---- the columns' and waves' shares: a lane holds 4 CW columns of V of its column, CW chunks of 16 bytes, their places xor-ed with the column
    {
        f32x4* const r = ored + (wave * GMAX + l16) * CH;
#pragma unroll
        for (int j = 0; j < CW; ++j) {
            f32x4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = acc[(4 * j + i) % CW][(4 * j + i) / CW];
            r[(CW * lq + j) ^ (l16 & 7)] = y;
        }
    }
    if (wave == 0 && lq == 0 && first && mytile == 0) tot[par][hc][0] = stick;
    if (a.m) {
        float even, odd, lowhalf, upphalf;
        both_rows(logs, even, odd);
        both_halves(even + odd, lowhalf, upphalf);
        if (lq == 0) s_log[wave][l16] = lowhalf + upphalf;
    }
    barrier_lds();
    constexpr int COPIES = R * (PIECES ? 2 : 1);           // columns of a head
    for (int i = tid; i < live * CH; i += NTHR) {
        const int g = i / CH, c = i % CH;
        f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < NW; ++w)
#pragma unroll
            for (int k = 0; k < COPIES; ++k) {
                const int col = g + (k << a.lg);
                s += ored[(w * GMAX + col) * CH + (c ^ (col & 7))];
            }
        const float left = tot[par][g][0];
        float log = 0.0f;
        if (a.m && c == 0)
            for (int w = 0; w < NW; ++w)
                for (int k = 0; k < R; ++k) log += s_log[w][g + (k << a.lg)];
        const long h = hq0 + g;
        if (!FAR && (a.slots == 1 || (!a.m && left < LEAST))) {
            typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
            if (a.rb) {
                const uint16_t* e = a.rb + ((bkv % a.Hkv) * (long)a.G + g0 + g) * D + 4 * c;
#pragma unroll
                for (int k = 0; k < 4; ++k) s[k] += left * __builtin_bit_cast(float, (uint32_t)e[k] << 16);
            }
            *reinterpret_cast<bf16x4*>(a.o + h * D + 4 * c) = bf16x4{(__bf16)s[0], (__bf16)s[1], (__bf16)s[2], (__bf16)s[3]};
            if (a.m && c == 0) a.m[h] = -log * SB_LN2;
        }
        if (a.part_o) {
            *reinterpret_cast<f32x4*>(a.part_o + (h * a.slots + slot) * D + 4 * c) = s;
            if (c == 0) {
                a.part_a[h * a.slots + slot] = left;
                if (a.m) a.part_l[h * a.slots + slot] = log;
            }
        }
    }
}

// slots of an entry that hold keys
__device__ __forceinline__ int slots_of(const Args& a, int end)
{
    return (a.near > 0) + (max(0, end - a.near) + a.C - 1) / a.C;
}

template <int D>
__global__ void __launch_bounds__(COMBINE_THREADS)
decode_kv4_combine_kernel(const Args a, int H, int heads)
{
    constexpr int NV = D / 4;              // a thread adds four columns of every NG-th slot
    constexpr int NG = COMBINE_THREADS / NV;
    __shared__ __attribute__((aligned(16))) float ored[NG][D];
    __shared__ float f[MOST_GROUP];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if ((int)blockIdx.x < heads) {
        const long bh = blockIdx.x;
        const int n = slots_of(a, up32(length_of(a, (int)(bh / H))));
        const float* pa = a.part_a + bh * a.slots;
        if (!a.m && a.near > 0 && pa[0] < LEAST) return;               // finished by the near launch
        if (a.slots == 1) return;                                      // (so is every head)
        // slot i gets what the nearer (lower) slots left
        const int c4 = tid % NV, grp = tid / NV;
        const f32x4* po = reinterpret_cast<const f32x4*>(a.part_o + bh * a.slots * D) + c4;
        // all of a thread's share is in flight at once
        constexpr int N = MAXSLOT / NG;
        f32x4 x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = grp + i * NG < n ? po[(grp + i * NG) * NV] : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        float p[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) p[e] = 2 * lane + e < n ? pa[2 * lane + e] : 1.0f;
        float left;
        const float before = wave_prefix(p[0] * p[1], left);
        if (wave == 0) {
            f[2 * lane] = before;
            f[2 * lane + 1] = before * p[0];
        }
        __syncthreads();
        f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < N; ++i) s += f[grp + i * NG] * x[i];
        *reinterpret_cast<f32x4*>(&ored[grp][4 * c4]) = s;
        __syncthreads();
        if (tid < D) {
            float r = 0.0f;
#pragma unroll
            for (int g = 0; g < NG; ++g) r += ored[g][tid];
            if (a.rb) r += left * __builtin_bit_cast(float, (uint32_t)a.rb[(bh % H) * D + tid] << 16);
            const __bf16 val = (__bf16)r;
            a.o[bh * D + tid] = __builtin_bit_cast(uint16_t, val);
        }
        if (a.m && wave == 1) {
            float log = 0.0f;
#pragma unroll
            for (int e = 0; e < 2; ++e) log += 2 * lane + e < n ? a.part_l[bh * a.slots + 2 * lane + e] : 0.0f;
            log = wave_sum(log);
            if (lane == 0) a.m[bh] = -log * SB_LN2;
        }
        return;
    }
    // ---- scores of one slot's keys
    const int bkv = ((int)blockIdx.x - heads) / a.slots, slot = ((int)blockIdx.x - heads) % a.slots;
    const int len = length_of(a, bkv / a.Hkv), end = up32(len);
    if (slot >= slots_of(a, end)) return;
    const bool is_near = a.near > 0 && slot == 0;
    const int top = is_near ? end : end - a.near - (slot - (a.near > 0)) * a.C;
    const int lo = max(0, top - (is_near ? a.near : a.C));
    const long hq0 = (long)bkv * a.G;
    bool any = false;
    for (int g = wave; g < a.G; g += COMBINE_THREADS / 64) {
        const float* pa = a.part_a + (hq0 + g) * a.slots;
        float x = 1.0f;
        for (int i = lane; i < slot; i += 64) x *= pa[i];
        wave_prefix(x, x);
        // the far launch left out the blocks of heads that are all exhausted
        bool there = true;
        if (!a.m && a.near > 0 && slot > 0) {
            const int g0 = g / GMAX * GMAX;
            there = __builtin_amdgcn_ballot_w64(!(a.part_a[(hq0 + min(g0 + (lane & 15), min(a.G, g0 + GMAX) - 1)) * a.slots] < LEAST)) != 0;
        }
        x = there ? x : 0.0f;
        any |= x != 0.0f;
        if (lane == 0) f[g] = x;
    }
    if (!__syncthreads_or(any) && a.score_out == a.score) return;
    for (int i = lo + tid; i < min(top, len); i += COMBINE_THREADS) {
        float s = a.score ? a.score[(long)bkv * a.Tcap + i] : 0.0f;
        for (int g = 0; g < a.G; ++g)
            if (f[g] != 0.0f) s = __builtin_fmaf(f[g], a.wl[(hq0 + g) * a.Tcap + i], s);
        a.score_out[(long)bkv * a.Tcap + i] = s;
    }
}

struct Split {
    int near, C, slots;
};
// The nearest keys in the near launch, the rest in chunks of whole rounds.  With m wanted every key is read whatever the nearest
// ones take: they need no launch of their own.
Split split_of(long wgs, int T, bool want_m)
{
    if (T <= ALONE) return {(T + 31) & ~31, KW * FAR_NW, 1};
    Split s = {want_m ? 0 : NEAR, 0, 0};
    constexpr int unit = KW * FAR_NW;
    const int far = T + KW - 1 - s.near;
    const long want = std::min((long)MAXSLOT - 1, std::max(1L, FAR_WGS / wgs));
    s.C = (int)(((far + want - 1) / want + unit - 1) / unit * unit);
    s.slots = (far + s.C - 1) / s.C + (s.near > 0);
    return s;
}

Split split_for(int B, int H, int Hkv, int T, bool want_m)
{
    const int nz = (H / Hkv + GMAX - 1) / GMAX;
    return split_of((long)B * Hkv * nz, T, want_m);
}

template <int D>
hipError_t launch_d(Args a, int B, int H, float* workspace, hipStream_t stream)
{
    const long heads = (long)B * H;
    const unsigned bkv = (unsigned)(B * a.Hkv), nz = (unsigned)((a.G + GMAX - 1) / GMAX);
    const bool combine = a.slots > 1 || (a.score_out && a.G > GMAX);
    if (combine) {
        a.part_o = workspace;
        a.part_a = a.part_o + heads * a.slots * D;
        a.part_l = a.part_a + heads * a.slots;
        if (a.score_out) a.wl = a.part_a + ((2 * heads * a.slots + 3) & ~3L);
    }
    hipError_t e = hipSuccess;
    while (1 << a.lg < std::min(a.G, GMAX)) ++a.lg;
    if (a.near > 0) {
        const dim3 grid(bkv, 1u, nz), threads(64 * NEAR_NW);
        if (a.lg == 4) hipLaunchKernelGGL((decode_kv4_kernel<D, false, 1, false>), grid, threads, 0, stream, a);
        else hipLaunchKernelGGL((decode_kv4_kernel<D, false, 1, true>), grid, threads, 0, stream, a);
        if ((e = hipGetLastError()) != hipSuccess || !combine) return e;
    }
    if (a.slots > (a.near > 0)) {
        const dim3 grid((unsigned)(a.slots - (a.near > 0)), bkv, nz), threads(64 * FAR_NW);
        if (a.lg == 4) hipLaunchKernelGGL((decode_kv4_kernel<D, true, 1, false>), grid, threads, 0, stream, a);
        else if (a.lg == 3) hipLaunchKernelGGL((decode_kv4_kernel<D, true, 1, true>), grid, threads, 0, stream, a);
        else if (a.lg == 2) hipLaunchKernelGGL((decode_kv4_kernel<D, true, 2, true>), grid, threads, 0, stream, a);
        else hipLaunchKernelGGL((decode_kv4_kernel<D, true, 4, true>), grid, threads, 0, stream, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const unsigned more = a.score_out ? bkv * (unsigned)a.slots : 0u;
    hipLaunchKernelGGL((decode_kv4_combine_kernel<D>), dim3((unsigned)heads + more), dim3(COMBINE_THREADS), 0, stream, a, H, (int)heads);
    return hipGetLastError();
}

}  // namespace

int decode_kv4_most_group() { return MOST_GROUP; }

// room for either split
size_t decode_kv4_workspace_bytes(int B, int H, int Hkv, int T, int Tcap, int d, bool scores)
{
    const long heads = (long)B * H;
    const long slots = std::max(split_for(B, H, Hkv, T, false).slots, split_for(B, H, Hkv, T, true).slots);
    size_t n = (size_t)heads * slots * d + (size_t)((2 * heads * slots + 3) & ~3L);
    if (scores) n += (size_t)heads * Tcap;
    return sizeof(float) * n;
}

hipError_t launch_decode_kv4(const uint16_t* q, const uint8_t* kc, const uint8_t* ks, const uint8_t* vc, const uint8_t* vs, const uint16_t* rb,
                             const int* lens, const float* score, float* score_out, uint16_t* o, float* m, float* workspace,
                             int B, int H, int Hkv, int T, int Tcap, int d, hipStream_t stream)
{
    const Split s = split_for(B, H, Hkv, T, m != nullptr);
    const Args a = {q, kc, ks, vc, vs, rb, lens, score, score_out, o, m, nullptr, nullptr, nullptr, nullptr, T, Tcap, Hkv, H / Hkv, s.near, s.C, s.slots, 0};
    if (d == 32) return launch_d<32>(a, B, H, workspace, stream);
    if (d == 64) return launch_d<64>(a, B, H, workspace, stream);
    return launch_d<128>(a, B, H, workspace, stream);
}

}  // namespace sb
