// Buckets of a bias by relative position (rk_block.h): the distances where they begin.  Plain C++, so that tests ask it on the host.
#pragma once
#include <climits>
#include <cmath>
#include <cstdint>

namespace rkb {

// n^a m^b as 32-bit limbs, the lowest first.
struct big {
    uint32_t limb[64] = {1};
    int size = 1;
    void times(uint32_t m, int power)
    {
        for (; power > 0; --power) {
            uint64_t carry = 0;
            for (int i = 0; i < size; ++i) {
                carry += (uint64_t)limb[i] * m;
                limb[i] = (uint32_t)carry;
                carry >>= 32;
            }
            if (carry) limb[size++] = (uint32_t)carry;
        }
    }
    bool reaches(const big &o) const
    {
        if (size != o.size) return size > o.size;
        for (int i = size - 1; i >= 0; --i)
            if (limb[i] != o.limb[i]) return limb[i] > o.limb[i];
        return true;
    }
};

// The least distances of buckets 1 .. count - 1: of bucket exact + i, the least n with (n / exact)^wide >= (far / exact)^i.  A
// product of roots is within 1e-16 of that power's root; a whole number as near as 1e-12 is decided by whole numbers.
// `room` entries are set, those past the buckets to INT_MAX.
inline void set_borders(int *border, int room, int count, int max_distance)
{
    const int exact = count / 2, wide = count - exact;
    for (int i = 0; i < exact; ++i) border[i] = i + 1;
    const double root = std::pow((double)max_distance / exact, 1.0 / wide);
    double at = exact;
    for (int i = 1; i < wide; ++i) {
        at *= root;
        const double whole = std::nearbyint(at);
        int n = (int)std::ceil(at);
        if (std::fabs(at - whole) < 1e-12 * at) {
            big a, b;
            a.times((uint32_t)whole, wide);
            a.times((uint32_t)exact, i);
            b.times((uint32_t)max_distance, i);
            b.times((uint32_t)exact, wide);
            n = (int)whole + (a.reaches(b) ? 0 : 1);
        }
        border[exact + i - 1] = n;
    }
    for (int i = count - 1; i < room; ++i) border[i] = INT_MAX;
}

}  // namespace rkb
