// How a call of decode on a 4-bit cache splits its keys over launches and workgroups.
#pragma once
#include <algorithm>

namespace sb {
namespace kv4 {

constexpr int GMAX = 16;               // query heads of a group per workgroup: the columns of the MFMA
constexpr int KW = 32;                 // keys of a tile
constexpr int NEAR_NW = 8, FAR_NW = 4;
constexpr int NEAR = KW * NEAR_NW;     // keys of a near launch that has a far one behind it
constexpr int MAXSLOT = 128;           // chunks, the nearest keys among them: two per lane of a wave
constexpr long FAR_WGS = 2048;         // workgroups of the far launch, all heads together

// The cache is the near launch's alone where its rounds (1.6 us each at d = 128, 1.2 below, as long as all its workgroups run at once) take no
// longer than the two other launches; beyond one workgroup a CU near and far heads share the CUs, and what a launch in front costs weighs more.
// Alone / three launches, us, no head far, then a third of the kv heads, then all:
//   256 workgroups at most  d = 128 B16 H8 T2800 5.9 / 13.0, 21.8 / 18.1, 21.9 / 22.6;  not T4000 6.2 / 14.0, 30.9 / 19.3, 30.6 / 27.2;  d = 64 not T4000 5.8 / 13.2, 25.1 / 16.8, 25.3 / 20.2
//   more  d = 128  B20 H16 T4000 8.3 / 13.3, 35 / 39, 46 / 43;  B32 H16 T4000 8.7 / 14.5, 36 / 39, 56 / 60, not T6500 8.9 / 14.1, 54 / 53, 86 / 89;  B32 H32 T2000 14.6 / 16.9, 37 / 42, 58 / 63,
//                  T4000 15.1 / 16.9, 58 / 60, 105 / 104;  B64 H32 T4000 29 / 24, 101 / 147, 196 / 190
//         d = 64   B20 H16 T4000 7.2 / 13.1, 27 / 29, 38 / 31;  B32 H16 T4000 7.4 / 13.5, 27 / 29, 42 / 41, not T6500 7.2 / 12.9, 41 / 39, 65 / 57;  B64 H32 T5000 14.7 / 17.8, 71 / 122, 141 / 143
//         d = 32   B32 H16 T4000 6.7 / 12.8, 25 / 26, 35 / 33;  B32 H32 T4000 7.6 / 13.9, 32 / 37, 46 / 51
// Where m is wanted every key is read anyway, alone / spread (below): d = 128 B4 H8 T700 8.9 / 8.8, B32 H16 T2000 30.8 / 33.0;  not B4 H8 T1300 13.7 / 9.0, B16 H8 T1300 13.9 / 12.3
inline int alone_up_to(long wgs, bool want_m)
{
    if (want_m) return wgs <= 256 ? 4 * NEAR : 8 * NEAR;
    return wgs <= 256 ? 13 * NEAR : 16 * NEAR;
}

// A small cache is spread over the chip, every key read, in two launches: 7.5 us and 0.19 us per MB beyond 6.  The limits lie where what is lost where no head is
// far is at most two thirds of what is gained where a third of the kv heads are.  Alone / spread, us, no head far, then a third:
//   d = 128  B4 H8 T1300 (6 MB) 6.1 / 8.3, 13.3 / 8.4;  T2800 (12 MB) 6.0 / 9.8, 21.5 / 9.9;  not T700 6.4 / 8.0, 8.6 / 8.3;  B16 H8 T1300 (23 MB) 6.2 / 11.6, 13.7 / 11.6
//   d = 64   B4 H8 T2000 (4 MB) 6.0 / 7.4, 14.1 / 7.5;  not T1300 5.8 / 7.4, 11.3 / 7.5 (the limit is from times of 9.7);  B16 H8 T2000 (17 MB) 5.4 / 10.2, 14.2 / 10.3
//   d = 32   B4 H8 T2800 (3 MB) 5.7 / 7.5, 17.0 / 7.5;  not T1300 5.7 / 7.2, 10.8 / 7.2 (the same)
// and beyond what the near launch takes alone, three launches / spread: B16 H8 T4000 d64 (35 MB) 12.9 / 14.8, 16.3 / 14.8;  not d128 (70 MB) 13.1 / 21.5, 18.7 / 21.7
inline bool spread_small(double cache_bytes, int T, int d)
{
    const int rounds = (T + NEAR - 1) / NEAR;
    return cache_bytes <= std::min(35e6, 1e6 * ((d == 128 ? 3.5 : 2.5) * (rounds - 1) - 11.5));
}

struct Split {
    int near, C, slots;
};
// The nearest keys in the near launch, the rest in chunks of whole rounds.  With m wanted, or spread, the nearest keys need no launch of their own, and no chunk writes the outputs:
// they come of two chunks at least.  Where the chip has so many workgroups that a head would get but one chunk, the near launch takes it, all keys, alone.
// FAR_WGS 1024 / 2048 / 4096, a third of the kv heads far: B8 H16 T16384 d128 38.9 / 30.5 / 31.3 us, d = 32 29.4 / 22.0 / 20.6, B16 H32 Hkv8 T4096 d128 20.9 / 20.6 / 18.8;
// all far 58.8 / 58.5 / 61.4, 30.5 / 31.7 / 34.2, 26.9 / 30.0 / 30.1.
inline Split split_of(long wgs, double cache_bytes, int T, int d, bool want_m)
{
    const long want = std::min((long)MAXSLOT - 1, std::max(1L, FAR_WGS / wgs));
    const bool spread = !want_m && want > 1 && spread_small(cache_bytes, T, d);
    if ((T <= alone_up_to(wgs, want_m) && !spread) || (want_m && want == 1)) return {(T + 31) & ~31, KW * FAR_NW, 1};
    Split s = {want_m || spread ? 0 : NEAR, 0, 0};
    constexpr int unit = 2 * KW * FAR_NW;
    const int far = T + KW - 1 - s.near;
    s.C = (int)(((far + want - 1) / want + unit - 1) / unit * unit);
    s.slots = (far + s.C - 1) / s.C + (s.near > 0);
    return s;
}

inline Split split_for(int B, int H, int Hkv, int T, int d, bool want_m)
{
    const int nz = (H / Hkv + GMAX - 1) / GMAX;
    return split_of((long)B * Hkv * nz, (double)B * Hkv * T * (d + d / 16), T, d, want_m);
}

}  // namespace kv4
}  // namespace sb
