// Single-token decode on a 4-bit cache (sb_kv4.h): one new query per (entry, head) against the entry's keys and values, and the
// weight that its heads give every key, added to the key's score.
//
// One pass over the cache, 2 (D / 2 + D / 32) bytes a key and kv head (136 at D = 128, 512 in bf16).  Chunks of keys combine as in
// sb_decode.hip: a chunk's weights are taken as if nothing nearer were there, and are shifted afterwards by what the nearer chunks
// took (Eq. 2).
//   near launch      grid (kv head, block of query heads): the nearest keys, all of a short cache
//   far launch       grid (chunk, kv head, block of query heads): the keys before those; returns at once where the nearest keys
//                    have used up the stick (LEAST, below)
//   combine launch   a workgroup per query head adds the chunks up in a fixed order; with scores, one per (kv head, chunk)
//                    shifts the weights of its keys, sums them over the group's heads and adds the score
//
// A workgroup takes its keys from the nearest down in rounds of R tiles of 32 per wave, wave 0 the nearest.
//   logits   z[key][head] = K q: 16x16x32 bf16 MFMA, A = 16 rows of K, B = the query heads of the group.  A lane reads the D / 8
//            bytes of its row that make up one A operand after the other (the order of the columns is free as long as q comes in
//            the same one), and converts them in registers, the scale with them.  Rows go to the MFMAs so that a lane gets eight
//            consecutive keys of a head.
//   weights  where the MFMA leaves the logits: Eq. 1's product over the lane's eight keys, then across the four lanes of a tile,
//            the tiles and the waves (by LDS, one barrier a round).  The keys' scores are results in fp32, so what is left of the stick is carried as it is, not by its
//            logarithm.  Many small weights would be lost where it is near 1: there their own sum P = prod (1 + e) - 1, e = sigma / (1 - sigma), is what is carried, up to a round of keys,
//            and the rounds' shares of the stick are multiplied in 64 bits, as T / 256 factors that are alike round the same way (in fp32 throughout, T = 524288 and logits around
//            -16: 3 % of the far weights, all of m).  That takes 2 to 8 % (B32 H16 T1800 d64, all far, 20.3 -> 21.9 us, d128 29.5 -> 29.8, B8 H16 T16384 d64 37.7 -> 39.5).  From less than 2^-126 of the stick on, weights are subnormal at most and count as zero.
//   output   O^T[c][head] += V^T w: a lane's eight weights are the B operand as they lie; it loads D / 16 columns of those same
//            eight rows of V, converts, and an in-register transposition (one v_perm per packed pair) makes the A operands.
// Codes and scales come through LDS as whole rows, every wave its own, one round ahead: K's place is asked for again as soon as a round
// has its logits, V's behind its output.  (Straight to registers it is 14 loads a tile, and 26 registers a tile to hold them: all heads far, B8 H16 T16384, d = 128, 64, 32:
// 69, 52, 37 us, through LDS with the same rounds 65, 44, 36, both before what is said of small weights and parts here.)  A near launch of more workgroups than the chip holds takes half
// as many waves a workgroup, two tiles each: B32 H16 T2000 d128 10.5 -> 8.9 us with no head far, 32.4 -> 21.3 with a third, B40 H16 T1800 d64 9.2 -> 7.7, 21.5 -> 18.1; smaller ones lose by it
// (B16 H8 T2000 d128 5.5 -> 6.3, 16.9 -> 18.2, B32 H16 T1800 d64 6.9 -> 6.8, 16.5 -> 17.1).
// V meets a weight in three parts of eight bits, bf16 each: 24 bits, all that it has, as in sb_decode.hip.  (Two parts, 16 bits, took 1 to 3 % less: B8 H16 T16384 d128, all far,
// 55.5 / 55.9 us, B32 H16 T1800 d64 19.4 / 20.0.)
// The 16 columns of the MFMAs are more than most groups have heads.  Their copies of a head take a tile each (two with up to four heads, R), which
// halves the vector instructions of the weights (four tiles gain nothing more), and the parts of a weight (PIECES of them), so that one MFMA does for a tile with up to four heads,
// two with up to eight, three beyond; the columns of a head are added up at the end.
#include "sb_kernels.h"
#include "sb_kv4.h"
#include "sb_mma.h"
#include "sb_split_kv4.h"

namespace sb {
namespace {

using namespace kv4;

constexpr float LEAST = 0x1p-126f;     // of the stick
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
    float* part_o;                     // [heads][slots][D]: slot 0 the nearest
    double* part_a;                    // [heads][slots]: share of the stick that a slot leaves
    float* part_l;                     // and -log2 of it, where m is wanted
    float* wl;                         // [heads][rows]: weights inside their chunk, where scores are combined; T rows, in whole tiles
    int T, rows, Tcap, Hkv, G, near, C, slots;
    int lg;                            // log2 of the columns that a copy of the heads takes
};

__device__ __forceinline__ int length_of(const Args& a, int b)
{
    return a.lens ? min(max(a.lens[b], 0), a.T) : a.T;
}
__device__ __forceinline__ int up32(int n) { return (n + 31) & ~31; }

// The entry and kv head of a near workgroup.  A CU gets workgroups i, i + 256, ..: with 16 kv heads, the same head of several entries, and heads that reach far would come
// together.  So the heads of an entry turn by one for each 256 workgroups in front of it (B32 H16 T1800 d64, a third of the heads far, 20.6 -> 16.4 us, d128 25.2 -> 21.7,
// d32 18.9 -> 15.4; none far 7.3 -> 7.3, 8.8 -> 9.0, 6.8 -> 6.8; all far 21.3 -> 21.9, 29.3 -> 30.1, 19.9 -> 19.9).
__device__ __forceinline__ int turned(int wg, int Hkv)
{
    const int first = wg / Hkv * Hkv;
    return first < 256 ? wg : first + (wg - first + first / 256) % Hkv;
}

template <int CTRL> __device__ __forceinline__ float dpp(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
template <int CTRL> __device__ __forceinline__ uint32_t dpp_word(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
// x += what CTRL's lanes have
template <int CTRL> __device__ __forceinline__ void add_columns(float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] += dpp<CTRL>(x[i]);
}
__device__ __forceinline__ float wave_sum(float x)
{
    x += dpp<0xB1>(x);
    x += dpp<0x4E>(x);
    x += dpp<0x141>(x);
    x += dpp<0x140>(x);
    float a, b;
    both_halves(x + __shfl_xor(x, 16), a, b);
    return a + b;
}

// product over the lanes below this one, and over all in `total`
template <int CTRL, int ROWS> __device__ __forceinline__ double dpp_or_one(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0x3ff00000, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xF, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_prefix(double v, double& total)
{
    v *= dpp_or_one<0x111, 0xF>(v);                       // row_shr:1, 2, 4, 8
    v *= dpp_or_one<0x112, 0xF>(v);
    v *= dpp_or_one<0x114, 0xF>(v);
    v *= dpp_or_one<0x118, 0xF>(v);
    v *= dpp_or_one<0x142, 0xA>(v);                       // row_bcast:15 into rows 1 and 3
    v *= dpp_or_one<0x143, 0xC>(v);                       // row_bcast:31 into rows 2 and 3
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, 63), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), 63);
    total = __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    return dpp_or_one<0x138, 0xF>(v);                     // wave_shr:1
}

// (1 + p) (1 + q) - 1
__device__ __forceinline__ float plus(float p, float q) { return __builtin_fmaf(p, q, p + q); }

// log2(1 + p), to some roundings of itself; below 1 / 4 by 2 atanh(p / (2 + p)), whose next term is 3e-9 of it
__device__ __forceinline__ float log2_1p(float p)
{
    const float s = p * __builtin_amdgcn_rcpf(2.0f + p), y = s * s;
    const float near_one = 2.0f * SB_LOG2E * (s + s * y * (1.0f / 3.0f + y * (1.0f / 5.0f + y * (1.0f / 7.0f))));
    return p < 0.25f ? near_one : fast_log2(1.0f + p);
}

// `even`: v of this lane's column in row 0 (lanes 0 .. 31) or 2 (32 .. 63), `odd`: in row 1 or 3
__device__ __forceinline__ void both_rows(float v, float& even, float& odd)
{
    auto sw = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), false, false);
    even = __builtin_bit_cast(float, (int)sw[0]);
    odd = __builtin_bit_cast(float, (int)sw[1]);
}

// A wave's R tiles in LDS, keys ascending: codes of K, of V, scales of K, of V.  A row's place is p = row ^ x, a 16-byte chunk of its
// codes lies at chunk ^ y, with x and y made of bits 3 and 4 of the row so that neither the rows of K's operands nor those of V's meet in a bank.
template <int D, int R> struct Place {
    static constexpr int ROW = D / 2, SROW = D / KV4_BLOCK, CPR = ROW / 16;
    static constexpr int CODES = KW * R * ROW, SCALES = KW * R * SROW;
    static constexpr int V = CODES, KS = 2 * CODES, VS = 2 * CODES + SCALES;
    static constexpr int BYTES = 2 * (CODES + SCALES);
    static constexpr int CODE_LOADS = (CODES + 1023) / 1024, LOADS = CODE_LOADS + 1;     // of a wave, for either of K and V
    static constexpr int ROWS_A_LOAD = 1024 / ROW;
    // x and y of a row
    static __device__ __forceinline__ int x_of(int row)
    {
        const int a = row >> 3 & 3;
        return D == 128 ? a : D == 64 ? (a >> 1) << 2 | (a & 1) : (a >> 1) << 2;
    }
    static __device__ __forceinline__ int y_of(int row) { return D == 128 ? row >> 3 & 3 : D == 64 ? row >> 3 & 1 : 0; }
};

// bytes of LDS as a T
template <class T> __device__ __forceinline__ T lds_read(uint32_t at)
{
    return *(__attribute__((address_space(3))) const T*)(uintptr_t)at;
}
template <int N> __device__ __forceinline__ void lds_words(uint32_t (&w)[N], uint32_t at)
{
    if constexpr (N == 1) {
        w[0] = lds_read<uint32_t>(at);
    } else if constexpr (N == 2) {
        const unsigned long long x = lds_read<unsigned long long>(at);
        w[0] = (uint32_t)x;
        w[1] = (uint32_t)(x >> 32);
    } else {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const u32x4 x = lds_load16(at + 4 * j);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[j + i] = x[i];
        }
    }
}

// the upper halves of two numbers' bits, each a bf16, in one word; what is left of the numbers in their place
__device__ __forceinline__ uint32_t upper_halves(float& a, float& b)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, a), v = __builtin_bit_cast(uint32_t, b);
    a -= __builtin_bit_cast(float, u & 0xffff0000u);
    b -= __builtin_bit_cast(float, v & 0xffff0000u);
    return __builtin_amdgcn_perm(v, u, 0x07060302u);
}

template <bool NT> __device__ __forceinline__ void dma16(uint64_t base, int off, uint32_t lds)
{
    if constexpr (NT) dma16_to_lds_at_nt(base, off, lds);
    else dma16_to_lds_at(base, off, lds);
}

// R: tiles of a wave and round.  PIECES: how many of the three parts of a weight the copies of a head's column take
template <int D, bool FAR, int NW, int R, int PIECES>
__global__ void __launch_bounds__(64 * NW, 2)
decode_kv4_kernel(const Args a)
{
    constexpr int NTHR = 64 * NW;
    constexpr int NT = NW * R;             // tiles of a round
    constexpr int KEYS = KW * NT;
    constexpr int CW = D / 16;             // columns of V per lane
    constexpr int CH = D / 4;              // 16-byte chunks of a head's columns
    __shared__ __attribute__((aligned(16))) float tot[2][GMAX][NT];      // per round parity: what a tile leaves of the stick
    __shared__ __attribute__((aligned(16))) float sums[2][GMAX][NT];     // and P of its keys
    __shared__ float s_log[NW][GMAX];
    __shared__ double s_left[GMAX];
    using P = Place<D, R>;
    constexpr int SHARES = NW * GMAX * CH * 16;
    __shared__ __attribute__((aligned(1024))) char smem[NW * P::BYTES > SHARES ? NW * P::BYTES : SHARES];
    __shared__ __attribute__((aligned(16))) float was[FAR ? 4 : KEYS];   // scores of the round's keys, every wave its own
    f32x4* const ored = reinterpret_cast<f32x4*>(smem);                  // once the keys are done

    const int bkv = FAR ? (int)blockIdx.y : turned((int)blockIdx.x, a.Hkv);      // entry * Hkv + kv head
    const int g0 = blockIdx.z * GMAX;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, lq = lane >> 4;
    const int b = (int)(FAR ? blockIdx.y : blockIdx.x) / a.Hkv;
    const int len = length_of(a, b), end = up32(len);
    const int slot = FAR ? (int)blockIdx.x + (a.near > 0) : 0;
    const int top = FAR ? end - a.near - (int)blockIdx.x * a.C : end;
    const int lo = max(0, FAR ? top - a.C : top - a.near);
    const long hq0 = (long)bkv * a.G + g0;
    const int live = min(GMAX, a.G - g0);
    // this lane's column: head l16 % 2^lg, copy l16 / 2^lg
    const int hc = l16 & ((1 << a.lg) - 1), copy = l16 >> a.lg;
    const int mytile = R == 1 ? 0 : copy & (R - 1);
    const int piece = copy / R;
    const bool first = copy < R && hc < live;          // one column for each tile and head
    const long head = hq0 + min(hc, live - 1);
    const float c2 = SB_LOG2E / sqrtf((float)D);

    if constexpr (FAR) {
        if (top <= 0) return;
        if (!a.m && a.near > 0 && __builtin_amdgcn_ballot_w64(!(a.part_a[head * a.slots] < LEAST)) == 0) return;
    }

    bf16x8 qw[D / 32];                     // B operand
#pragma unroll
    for (int s = 0; s < D / 32; ++s) qw[s] = *reinterpret_cast<const bf16x8*>(a.q + head * D + lq * (D / 4) + 8 * s);

    f32x4 acc[CW];                         // O^T: row 4 lq + r of MFMA e is column CW (4 lq + r) + e, column l16
#pragma unroll
    for (int e = 0; e < CW; ++e) acc[e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    double stick = 1.0, logs = 0.0;        // left by the keys already passed; -log2 of what this lane's own keys left
    int par = 0, hi = top;

    // ---- rows to LDS, whole rows of the wave's R tiles at a time; where a tile is below lo there is none, and the last one is loaded
    const uint64_t kc = scalar_base(a.kc + (long)bkv * a.Tcap * P::ROW), vc = scalar_base(a.vc + (long)bkv * a.Tcap * P::ROW);
    const uint64_t ks = scalar_base(a.ks + (long)bkv * a.Tcap * P::SROW), vs = scalar_base(a.vs + (long)bkv * a.Tcap * P::SROW);
    const uint32_t mem = lds_offset(smem) + wave * P::BYTES;
    auto fetch = [&](uint64_t codes, uint64_t scales, uint32_t at, uint32_t scales_at, int first_row) __attribute__((always_inline)) {
        const uint64_t cb = codes + (int64_t)first_row * P::ROW, sb = scales + (int64_t)first_row * P::SROW;
        const int least = lo - first_row;
#pragma unroll
        for (int i = 0; i < P::CODE_LOADS; ++i) {
            const int p = i * P::ROWS_A_LOAD + lane / P::CPR, row = p ^ P::x_of(p);
            const int off = max(row, least) * P::ROW + (((lane % P::CPR) ^ P::y_of(p)) << 4);
            if (P::CODES >= 1024 || lane < P::CODES / 16) dma16<FAR>(cb, off, at + i * 1024);
        }
        if (lane < P::SCALES / 16) dma16<FAR>(sb, max(lane * (16 / P::SROW), least) * P::SROW, scales_at);
    };
    auto first_row_of = [&](int top) __attribute__((always_inline)) { return top - KW * R * (wave + 1); };
    auto fetch_k = [&](int top) __attribute__((always_inline)) { fetch(kc, ks, mem, mem + P::KS, first_row_of(top)); };
    const bool adds = !FAR && a.score && !a.wl;            // to scores, that come the same way, behind V
    const uint64_t sc = adds ? scalar_base(reinterpret_cast<const uint8_t*>(a.score + (long)bkv * a.Tcap)) : 0;
    const uint32_t scores = lds_offset(reinterpret_cast<const char*>(was)) + wave * R * KW * 4;
    auto fetch_v = [&](int top) __attribute__((always_inline)) {
        fetch(vc, vs, mem + P::V, mem + P::VS, first_row_of(top));
        if (!FAR && adds && lane < R * KW / 4) dma16<FAR>(sc + (int64_t)first_row_of(top) * 4, max(4 * lane, lo - first_row_of(top)) * 4, scores);
    };
    // where this lane's words are, in a wave's lowest tile (keys ascending: tile j of this wave is R - 1 - j tiles on)
    auto place = [&](int row, int byte) __attribute__((always_inline)) {
        return (row ^ P::x_of(row)) * P::ROW + (((byte >> 4) ^ P::y_of(row)) << 4 | (byte & 15));
    };
    uint32_t kat[2], vat[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) kat[h] = mem + place(8 * (l16 >> 2) + 4 * h + (l16 & 3), lq * (D / 8));
#pragma unroll
    for (int i = 0; i < 8; ++i) vat[i] = mem + P::V + place(8 * lq + i, l16 * (D / 32));
    const uint32_t ksat = mem + P::KS + (8 * (l16 >> 2) + (l16 & 3)) * P::SROW + lq * P::SROW / 4, vsat = mem + P::VS + 8 * lq * P::SROW;
    const uint32_t vrot = 9 + 8 * (l16 * (D / 16) / KV4_BLOCK);          // rotation that takes a scale byte to bits 30 .. 23
    // rows of tile j of this wave
    auto valid_of = [&](int j) __attribute__((always_inline)) {
        const int base = hi - KW * (wave * R + j + 1);
        return base < lo ? 0 : len - base;
    };

    // one round; whether another follows
    auto round = [&]() __attribute__((always_inline)) {
        const bool more = hi - KEYS > lo;
        // ---- logits of the lane's eight keys, in base 2
        // K has landed, V was asked for behind it
        if (!FAR && adds) dma_wait<P::LOADS + 1>();
        else dma_wait<P::LOADS>();
        float x[8];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int valid = valid_of(j), on = R - 1 - j;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
                uint32_t k[D / 32];
                lds_words(k, kat[h] + on * KW * P::ROW);
                const uint32_t s = (uint32_t)lds_read<uint8_t>(ksat + (on * KW + 4 * h) * P::SROW) << 23;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const u32x4 p = {kv4_pair<0>(k[i], s), kv4_pair<1>(k[i], s), kv4_pair<2>(k[i], s), kv4_pair<3>(k[i], s)};
                    z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p), qw[i], z, 0, 0, 0);
                }
                if (__builtin_expect(valid < KW, 0)) {
                    asm volatile("");      // (a branch, not two instructions a logit)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[r] = 8 * lq + 4 * h + r < valid ? z[r] : -INFINITY;
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) x[4 * h + r] = j == 0 || mytile == j ? z[r] : x[4 * h + r];
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (the rows have been read)
        if (more) fetch_k(hi - KEYS);
        // ---- the lane's chain: w[i] = e_i prod_{i' < i} (1 + e_i'), their sum P; norm makes it the weight where the stick is whole
        // before the lane's nearest key, `leave` is what the eight keys leave
        float w[8], norm, leave, P = 0.0f, run = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] *= c2;
            const float e = fast_exp2(x[i]);
            w[i] = __builtin_fmaf(P, e, e);
            P = __builtin_fmaf(P, 1.0f + e, e);            // (P + w would make the chain twice as long)
        }
        norm = leave = __builtin_amdgcn_rcpf(1.0f + P);
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(P < 0x1p40f)) != 0, 0)) {
            // (norm times what is left before the lane could be subnormal where the weight is not)
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] *= norm;
            norm = 1.0f;
            if (!(P < 0x1p120f)) {         // in the log form
#pragma unroll
                for (int i = 7; i >= 0; --i) {
                    run += sp2(x[i]);
                    w[i] = fast_exp2(x[i] - run);
                }
                leave = fast_exp2(-run);
            }
        }
        if (a.m) logs += P < 0x1p120f ? log2_1p(P) : run;
        // ---- across the four lanes of a tile (the odd one of a pair and the upper half are nearer), the tiles and waves
        float even, odd, lowhalf, upphalf;
        both_rows(P, even, odd);
        both_halves(plus(even, odd), lowhalf, upphalf);
        P = plus(lowhalf, upphalf);
        both_rows(leave, even, odd);
        both_halves(even * odd, lowhalf, upphalf);
        norm *= ((lq & 1) ? 1.0f : odd) * (lq < 2 ? upphalf : 1.0f);
        const int mine = wave * R + mytile;
        if (lq == 0 && first) {
            tot[par][hc][mine] = lowhalf * upphalf;
            sums[par][hc][mine] = P;
        }
        barrier_lds();
        const int row = min(hc, live - 1);
        float before = (float)stick, left = 1.0f;
#pragma unroll
        for (int j = 0; j < NT; j += 4) {
            const f32x4 p = *reinterpret_cast<const f32x4*>(&tot[par][row][j]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (j + i == mine) before *= left;
                left *= p[i];
            }
        }
        norm *= before;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] *= norm;
        // the round's P (a quarter of the tiles for each of a column's lanes); where the round takes half of the stick or more its last bits count no more, and it may be anything
        P = sums[par][row][NT / 4 * lq];
        if (NT == 8) P = plus(P, sums[par][row][2 * lq + 1]);
        both_rows(P, even, odd);
        both_halves(plus(even, odd), lowhalf, upphalf);
        P = plus(lowhalf, upphalf);
        stick *= left > 0.5f ? 1.0 - (double)(P * left) : (double)left;
        // ---- output
        // a weight is the sum of three bf16, of eight bits each: nothing of it is lost
        u32x4 w0, w1, w2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a0 = w[2 * i], a1 = w[2 * i + 1];
            w0[i] = upper_halves(a0, a1);
            w1[i] = upper_halves(a0, a1);
            w2[i] = upper_halves(a0, a1);
            if (PIECES > 1) w0[i] = piece == 0 ? w0[i] : w1[i];
            if (PIECES > 2) w0[i] = piece < 2 ? w0[i] : w2[i];
            // two tiles a wave, two copies for each: the third part goes to where the other tile's first one would be
            if (PIECES == 2) w2[i] = piece == 0 ? R == 2 ? dpp_word<0x124>(w2[i]) : w2[i] : 0u;        // row_ror:4, to a copy of the other tile
        }
        if (more) dma_wait<P::LOADS>();    // V has landed
        else dma_wait<0>();
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int valid = valid_of(j), on = R - 1 - j;
            u32x4 wb = w0;
            if (R > 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) wb[i] = mytile == j ? wb[i] : PIECES == 2 ? w2[i] : 0u;
            }
            // scales of the eight rows, bytes as they lie: of row i, the byte of this lane's columns to the exponent's place (what stands beside it does not count)
            constexpr int PER = 128 / D;   // rows in a word
            uint32_t sw[D / 16];
            lds_words(sw, vsat + on * KW * P::SROW);
            if (__builtin_expect(valid < KW, 0)) {
                asm volatile("");
                // whatever lies in rows that are not there: a zero weight makes it zero once it is finite
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (8 * lq + i >= valid) sw[i / PER] = PER == 1 ? 0x7f7f7f7fu : (sw[i / PER] & ~(((1u << (32 / PER)) - 1) << (i % PER * (32 / PER)))) | (0x7f7f7f7fu & (((1u << (32 / PER)) - 1) << (i % PER * (32 / PER))));
            }
            uint32_t pv[8][CW / 2];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t s = __builtin_amdgcn_alignbit(sw[i / PER], sw[i / PER], vrot + 8 * (i % PER) * P::SROW);
                const uint32_t at = vat[i] + on * KW * P::ROW;
                const uint32_t v = D == 128 ? lds_read<uint32_t>(at) : D == 64 ? lds_read<uint16_t>(at) : lds_read<uint8_t>(at);
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
                if (R * PIECES < 3) acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8, w2), acc[e], 0, 0, 0);
                if (PIECES == 1) acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8, w1), acc[e], 0, 0, 0);
                acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8, wb), acc[e], 0, 0, 0);
            }
        }
        // (stores go ahead of the next round's loads of V: what waits for K waits for nothing behind them)
        if (a.score_out) {
            if (a.wl) {
                const int base = hi - KW * (mine + 1);
                if (first && base >= lo) {
                    float* p = a.wl + (hq0 + hc) * a.rows + base + 8 * lq;
                    *reinterpret_cast<f32x4*>(p) = f32x4{w[0], w[1], w[2], w[3]};
                    *reinterpret_cast<f32x4*>(p + 4) = f32x4{w[4], w[5], w[6], w[7]};
                }
            } else if constexpr (!FAR) {
                // over the heads, 2^lg neighbouring columns; each tile's sums are then in the first column of its copy
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = hc < live ? w[i] : 0.0f;
                if (a.lg > 0) add_columns<0xB1>(w);        // quad_perm 1, 0, 3, 2
                if (a.lg > 1) add_columns<0x4E>(w);        // quad_perm 2, 3, 0, 1
                if (a.lg > 2) add_columns<0x141>(w);       // row_half_mirror
                if (a.lg > 3) add_columns<0x140>(w);       // row_mirror
                const int base = hi - KW * (mine + 1), key = base + 8 * lq;
                if (first && hc == 0 && base >= lo) {
                    const long at = (long)bkv * a.Tcap + key;
                    const uint32_t mine_was = scores + ((R - 1 - mytile) * KW + 8 * lq) * 4;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (key + 4 * h + 4 <= len) {
                            f32x4 x = {w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]};
                            if (adds) x += __builtin_bit_cast(f32x4, lds_load16(mine_was + 16 * h));
                            *reinterpret_cast<f32x4*>(a.score_out + at + 4 * h) = x;
                        } else {
#pragma unroll
                            for (int r = 4 * h; r < 4 * h + 4; ++r)
                                if (key + r < len) a.score_out[at + r] = (adds ? lds_read<float>(mine_was + 4 * r) : 0.0f) + w[r];
                        }
                    }
                }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) fetch_v(hi - KEYS);
        hi -= KEYS;
        par ^= 1;
        return more && (FAR || a.m || __builtin_amdgcn_ballot_w64(!(stick < LEAST)) != 0);
    };
    if (hi > lo) {
        fetch_k(hi);
        fetch_v(hi);
        while (round()) {}
    }
    dma_wait<0>();                         // keys asked for before the end was known
    barrier_lds();                         // (theirs is the place of the shares)
    // keys that no stick was left for keep their scores
    if (!FAR && a.score_out && !a.wl && a.score_out != a.score)
        for (int i = lo + tid; i < hi; i += NTHR) a.score_out[(long)bkv * a.Tcap + i] = a.score ? a.score[(long)bkv * a.Tcap + i] : 0.0f;
    if (!FAR && a.wl && a.slots == 1)                      // (read by the combination)
        for (int g = 0; g < live; ++g)
            for (int i = lo + tid; i < hi; i += NTHR) a.wl[(hq0 + g) * a.rows + i] = 0.0f;

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
    if (wave == 0 && lq == 0 && first && mytile == 0) s_left[hc] = stick;
    if (a.m) {
        float even, odd, lowhalf, upphalf;
        both_rows((float)logs, even, odd);
        both_halves(even + odd, lowhalf, upphalf);
        if (lq == 0) s_log[wave][l16] = lowhalf + upphalf;
    }
    barrier_lds();
    constexpr int COPIES = R * PIECES;                     // columns of a head
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
        const double left = s_left[g];
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
                for (int k = 0; k < 4; ++k) s[k] += (float)left * __builtin_bit_cast(float, (uint32_t)e[k] << 16);
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
        const double* pa = a.part_a + bh * a.slots;
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
        double p[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) p[e] = 2 * lane + e < n ? pa[2 * lane + e] : 1.0;
        double left;
        const double before = wave_prefix(p[0] * p[1], left);
        if (wave == 0) {
            f[2 * lane] = (float)before;
            f[2 * lane + 1] = (float)(before * p[0]);
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
            if (a.rb) r += (float)left * __builtin_bit_cast(float, (uint32_t)a.rb[(bh % H) * D + tid] << 16);
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
        const double* pa = a.part_a + (hq0 + g) * a.slots;
        double before = 1.0;
        for (int i = lane; i < slot; i += 64) before *= pa[i];
        wave_prefix(before, before);
        // the far launch left out the blocks of heads that are all exhausted
        bool there = true;
        if (!a.m && a.near > 0 && slot > 0) {
            const int g0 = g / GMAX * GMAX;
            there = __builtin_amdgcn_ballot_w64(!(a.part_a[(hq0 + min(g0 + (lane & 15), min(a.G, g0 + GMAX) - 1)) * a.slots] < LEAST)) != 0;
        }
        const float x = there ? (float)before : 0.0f;
        any |= x != 0.0f;
        if (lane == 0) f[g] = x;
    }
    if (!__syncthreads_or(any) && a.score_out == a.score) return;
    const long row = (long)bkv * a.Tcap;
    for (int i = lo + 4 * tid; i < min(top, len); i += 4 * COMBINE_THREADS) {
        f32x4 s = a.score ? *reinterpret_cast<const f32x4*>(a.score + row + i) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int g = 0; g < a.G; ++g)
            if (f[g] != 0.0f) s += f[g] * *reinterpret_cast<const f32x4*>(a.wl + (hq0 + g) * a.rows + i);
        if (i + 4 <= len) {
            *reinterpret_cast<f32x4*>(a.score_out + row + i) = s;
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (i + r < len) a.score_out[row + i + r] = s[r];
        }
    }
}

// Workgroups of the near launch that one round of the chip holds: eight waves of 147 to 152 registers and 69 KB, 116 to 127 and 36 KB, 92 to 111 and 20 KB.
constexpr long round_of(int d) { return d == 128 ? 256 : 512; }

// the heads' weights meet in a launch of their own
inline bool combined(long slots, int G) { return slots > 1 || G > GMAX; }

template <int D>
hipError_t launch_d(Args a, int B, int H, float* workspace, hipStream_t stream)
{
    const long heads = (long)B * H;
    const unsigned bkv = (unsigned)(B * a.Hkv), nz = (unsigned)((a.G + GMAX - 1) / GMAX);
    const bool combine = a.slots > 1 || (a.score_out && combined(a.slots, a.G));
    if (combine) {
        a.part_o = workspace;
        a.part_a = reinterpret_cast<double*>(a.part_o + heads * a.slots * D);
        a.part_l = reinterpret_cast<float*>(a.part_a + heads * a.slots);
        if (a.score_out) a.wl = a.part_o + heads * a.slots * D + ((3 * heads * a.slots + 3) & ~3L);
    }
    hipError_t e = hipSuccess;
    while (1 << a.lg < std::min(a.G, GMAX)) ++a.lg;
    if (a.near > 0) {
        const dim3 grid(bkv, 1u, nz);
        const bool wide = a.lg < 3 && (long)bkv * nz > round_of(D);
        auto go = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), 0, stream, a); };
        if (a.lg == 4) go(decode_kv4_kernel<D, false, NEAR_NW, 1, 1>, NEAR_NW);
        else if (a.lg == 3) go(decode_kv4_kernel<D, false, NEAR_NW, 1, 2>, NEAR_NW);
        else if (!wide) go(decode_kv4_kernel<D, false, NEAR_NW, 1, 3>, NEAR_NW);
        else if (a.lg == 2) go(decode_kv4_kernel<D, false, NEAR_NW / 2, 2, 2>, NEAR_NW / 2);
        else go(decode_kv4_kernel<D, false, NEAR_NW / 2, 2, 3>, NEAR_NW / 2);
        if ((e = hipGetLastError()) != hipSuccess || !combine) return e;
    }
    if (a.slots > (a.near > 0)) {
        const dim3 grid((unsigned)(a.slots - (a.near > 0)), bkv, nz);
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * FAR_NW), 0, stream, a); };
        if (a.lg == 4) go(decode_kv4_kernel<D, true, FAR_NW, 1, 1>);
        else if (a.lg == 3) go(decode_kv4_kernel<D, true, FAR_NW, 1, 2>);
        else if (a.lg == 2) go(decode_kv4_kernel<D, true, FAR_NW, 2, 2>);
        else go(decode_kv4_kernel<D, true, FAR_NW, 2, 3>);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const unsigned more = a.score_out ? bkv * (unsigned)a.slots : 0u;
    hipLaunchKernelGGL((decode_kv4_combine_kernel<D>), dim3((unsigned)heads + more), dim3(COMBINE_THREADS), 0, stream, a, H, (int)heads);
    return hipGetLastError();
}

}  // namespace

int decode_kv4_most_group() { return MOST_GROUP; }

// room for either split
size_t decode_kv4_workspace_bytes(int B, int H, int Hkv, int T, int d, bool scores)
{
    const long heads = (long)B * H;
    const long slots = std::max(split_for(B, H, Hkv, T, d, false).slots, split_for(B, H, Hkv, T, d, true).slots);
    size_t n = (size_t)heads * slots * d + (size_t)((3 * heads * slots + 3) & ~3L);
    if (scores && combined(slots, H / Hkv)) n += (size_t)heads * ((T + KW - 1) / KW * KW);
    return sizeof(float) * n;
}

hipError_t launch_decode_kv4(const uint16_t* q, const uint8_t* kc, const uint8_t* ks, const uint8_t* vc, const uint8_t* vs, const uint16_t* rb,
                             const int* lens, const float* score, float* score_out, uint16_t* o, float* m, float* workspace,
                             int B, int H, int Hkv, int T, int Tcap, int d, hipStream_t stream)
{
    const Split s = split_for(B, H, Hkv, T, d, m != nullptr);
    const Args a = {q, kc, ks, vc, vs, rb, lens, score, score_out, o, m, nullptr, nullptr, nullptr, nullptr, T, (T + KW - 1) / KW * KW, Tcap, Hkv, H / Hkv, s.near, s.C, s.slots, 0};
    if (d == 32) return launch_d<32>(a, B, H, workspace, stream);
    if (d == 64) return launch_d<64>(a, B, H, workspace, stream);
    return launch_d<128>(a, B, H, workspace, stream);
}

}  // namespace sb
