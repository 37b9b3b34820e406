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

// The cache is the near launch's alone where its rounds (1.4 us each at d = 128, 1.0 below, as long as all its workgroups run at once) take no
// longer than the two other launches; beyond one workgroup a CU near and far heads share the CUs, and what a launch in front costs weighs more.
// Alone / three launches, us, no head far, then a third of the kv heads, then all:
//   256 workgroups at most  d = 128 B16 H8 T2800 5.8 / 10.1, 19.8 / 16.0, 20.4 / 21.6;  not T4000 5.2 / 10.0, 27.3 / 16.7, 27.7 / 25.8;  d = 64 not T4000 5.6 / 13.4, 23.0 / 15.3, 23.1 / 19.4
//   more  d = 128  B20 H16 T4000 7.6 / 13.3, 33 / 36, 42 / 42;  B32 H16 T4000 8.5 / 13.9, 34 / 36, 54 / 58, not T6500 8.5 / 14.1, 51 / 50, 85 / 84;  B32 H32 T2000 14.7 / 17.2, 37 / 40, 55 / 60,
//                  T4000 14.4 / 17.5, 58 / 58, 105 / 100;  B64 H32 T4000 27 / 24, 97 / 135, 194 / 187
//         d = 64   B20 H16 T4000 6.6 / 12.9, 25 / 27, 35 / 29;  B32 H16 T4000 6.9 / 13.4, 26 / 26, 38 / 39, not T6500 6.8 / 13.5, 42 / 36, 59 / 53;  B64 H32 T5000 14.2 / 18.4, 65 / 108, 133 / 132
//         d = 32   B32 H16 T4000 6.4 / 12.3, 25 / 23, 32 / 29;  B32 H32 T4000 7.0 / 13.9, 28 / 32, 41 / 44
// Where m is wanted every key is read anyway, alone / spread (below): d = 128 B4 H8 T700 7.8 / 7.9, B32 H16 T2000 29.7 / 30.6;  not B4 H8 T1300 12.3 / 8.1, B16 H8 T1300 12.5 / 11.0
inline int alone_up_to(long wgs, bool want_m)
{
    if (want_m) return wgs <= 256 ? 4 * NEAR : 8 * NEAR;
    return wgs <= 256 ? 13 * NEAR : 16 * NEAR;
}

// A small cache is spread over the chip, every key read, in two launches: 8 us and 0.16 us per MB beyond 6.  The limits lie where what is lost where no head is
// far is at most two thirds of what is gained where a third of the kv heads are.  Alone / spread, us, no head far, then a third:
//   d = 128  B4 H8 T1300 (6 MB) 5.2 / 8.1, 12.2 / 8.1;  T2800 (12 MB) 5.3 / 9.4, 19.3 / 9.3;  not T700 5.4 / 8.1, 7.9 / 8.0;  B16 H8 T1300 (23 MB) 5.2 / 11.0, 12.3 / 11.0
//   d = 64   B4 H8 T2000 (4 MB) 5.9 / 10.0, 12.7 / 10.0;  not T1300 6.1 / 9.7, 10.5 / 9.7;  B16 H8 T2000 (17 MB) 5.7 / 10.8, 13.2 / 10.9
//   d = 32   B4 H8 T2800 (3 MB) 5.8 / 9.8, 15.6 / 9.1;  not T1300 5.5 / 9.9, 9.9 / 9.8
// and beyond what the near launch takes alone, three launches / spread: B16 H8 T4000 d64 (35 MB) 13.4 / 14.3, 15.3 / 14.2;  not d128 (70 MB) 10.0 / 20.9, 16.7 / 20.8
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
// FAR_WGS 1024 / 2048 / 4096, a third of the kv heads far: B8 H16 T16384 d128 38.5 / 30.0 / 30.6 us, d = 32 30.6 / 23.4 / 21.1, B16 H32 Hkv8 T4096 d128 21.2 / 19.5 / 23.1.
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
