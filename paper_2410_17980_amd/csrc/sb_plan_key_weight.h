// How a call of the key weights is laid out over launches and workgroups, and what it needs of a workspace.
#pragma once
#include <stddef.h>
#include <algorithm>

namespace sb {
namespace key_weight {

constexpr int NW = 4;                  // waves of a workgroup, a unit (32 query rows of a head) each
constexpr int TK = 64;                 // keys of a tile

// Numbers in the workspace at a time: 2 GiB (chunks of keys, 384 groups at most, take less).  B1 H32 Hkv8 T131072 d128 takes four times two launches, 10.3 ms
// with a third of the kv heads far, 34.4 with all; with 8 GiB at once 9.7 and 33.4.
constexpr long MOST_PART = 1L << 29;

struct Plan {
    bool small, pairs;
    int groups, chunks, C;
    int Tpad;
    // groups at a time: their numbers go through the workspace, which for all of them would grow with T^2
    int at_once(int BHkv) const
    {
        const long most = chunks > 1 ? groups : std::max(1L, std::min<long>(groups, MOST_PART / ((long)BHkv * Tpad)));
        const long times = (groups + most - 1) / most;
        return (int)((groups + times - 1) / times);
    }
    size_t left_of() const { return chunks > 1 ? (size_t)groups * NW * chunks * 32 : 0; }
    size_t floats(int BHkv) const { return (size_t)BHkv * ((size_t)at_once(BHkv) * (Tpad + 2 * (size_t)chunks) + 2 * left_of()); }
};
// What a plan takes, from measurements (all heads far; us).  One unit a workgroup: 1.25 for a round of 256 keys, of the longest unit alone where the
// units fit the chip, 256 of them at a time beyond.  Four units: 1.4 for a tile of 64 keys of the longest, or 0.45 ns a subtile of all, whichever is more.  Chunks of
// keys in two launches: 8 more, 0.8 ns a subtile.  Measured with all heads far, one unit / four units / chunks (768 workgroups):
//   B4 H12 Hkv4 T2048 d128, whole prompt 78 / 56;  B8 H16 T2048 d64 173 / 101;  B1 H12 Hkv4 T3000 d64 39 / 56 / 70;  B1 H4 T4000 d128 40 / 85 / 54;
//   B2 H16 Hkv8 T700 d128 16.5 / 19 / 20;  64 rows of B1 H32 Hkv8 T16384 d128 93 / 315 / 39;  one row of B1 H32 Hkv8 T4000 d128 27 / 82 / 16
// Two units a wave where the longest workgroup's tiles, 2.1 each, take no longer than all the work does with a third of the kv heads far.  One / two, a third
// far, then all:  B16 H16 T2048 d32 109 / 97, 181 / 153;  B2 H64 Hkv8 T4096 d64 148 / 139, 339 / 287;  B8 H32 Hkv8 T2048 d128 108 / 114, 224 / 213;
//   B8 H16 T4096 d64 174 / 174, 352 / 310;  not B8 H16 T2048 d64 66 / 66, 101 / 89;  B1 H32 Hkv8 T8192 d128 184 / 271, 409 / 412
inline Plan plan_of(int B, int H, int Hkv, int Tq, int T)
{
    const int G = H / Hkv, units = (Tq + 31) / 32 * G, Tpad = (T + TK - 1) / TK * TK;
    const double all = (double)B * Hkv * units, mean = (T - 0.5 * Tq) / T;            // share of the keys that a query sees in the mean
    const double subtiles = all * mean * T / 32.0;
    const double small = 1.25 * (T / 256 + 1) * std::max(1.0, all * mean / 256.0);
    Plan p = {false, false, (units + NW - 1) / NW, 1, Tpad, Tpad};
    const long wgs = (long)B * Hkv * p.groups;
    const int tiles = Tpad / TK;
    const int want = (int)std::max(1L, std::min<long>(tiles / 2, 768 / wgs));
    if (small <= (want > 1 ? 8.0 + 0.0008 * subtiles : std::max(1.4 * tiles, 0.00045 * subtiles))) {
        p.small = true;
        p.groups = units;
    } else if (want > 1) {
        p.C = (tiles + want - 1) / want * TK;
        p.chunks = (T + p.C - 1) / p.C;
        if (p.chunks == 1) p.C = Tpad;
    } else if (2.1 * tiles <= 0.00015 * subtiles) {
        p.pairs = true;
        p.groups = (units + 2 * NW - 1) / (2 * NW);
    }
    return p;
}

}  // namespace key_weight
}  // namespace sb
