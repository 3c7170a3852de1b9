// In which unit the attention over an 8-bit cache sums its values (pv_kernels_kv8_attention.hip).  Whole numbers only, the same in every lane.
//
// The accumulators are multiples of 2^E: a key adds 2^15 * weight * code * 2^(ev - E) to them, ev the exponent of its values' scale, 2^15 * weight * 2^(ev - E) rounded to f16.  E is the largest
// exponent so far, unless a group of 16 keys is so far below that f16 would round its weights: then the groups are gone through one after the other, each in its own unit.  The unit then falls, and what has
// been summed grows by as much, so it never falls by more than 2^64 below the largest exponent of all groups so far: 2^15 * 448 * 2^30 keys * 2^64 < 2^118, which 32 bits hold (a block of
// zeros has the smallest scale there is, 2^-100).  Values of scales that lie further below add nothing; they need no pass of their own.
#pragma once

#define KV8_NO_SCALE (-1000)                // exponent of a group that does not exist
#define KV8_FALL 64

// Four groups' exponents against the unit E, and top, the largest exponent so far: the unit that the groups are summed in, and dv, ev - E.  Where they are too far apart, `only` one group is looked at at a time,
// from 0 to 3 (-1: all; the others' dv is 0).
__device__ inline void kv8_next_unit(const int (&ev)[4], int &E, int &top, int (&dv)[4], int &only)
{
    const int e0 = ev[0], e1 = ev[1], e2 = ev[2], e3 = ev[3], high = max(max(max(e0, e1), max(e2, e3)), E);
    int lowest = -1000000;
    bool one = false;
    top = max(top, high);
    if (only < 0 && min(min(e0, e1), min(e2, e3)) - high >= -14) E = high;      // (few scalar instructions in most calls: they take a wave's turns as others do)
    else {
        const int least = top - KV8_FALL;
        auto far = [&](int e) { return (int)(e >= least) & (int)(e - high < -14); };
        if (only < 0 && (far(e0) | far(e1) | far(e2) | far(e3))) only = 0;
        one = only >= 0;
        const int mine = only == 0 ? e0 : only == 1 ? e1 : only == 2 ? e2 : e3;
        E = !one ? high : mine < least ? max(E, least) : mine;
        lowest = -KV8_FALL;
    }
    dv[0] = max(e0 - E, lowest); dv[1] = max(e1 - E, lowest); dv[2] = max(e2 - E, lowest); dv[3] = max(e3 - E, lowest);
    if (one) {
#pragma unroll
        for (int i = 0; i < 4; ++i) dv[i] = i != only ? 0 : dv[i];
    }
}
