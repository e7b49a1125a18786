// Arithmetic of the search for a nucleus' end, in host and device code alike, so that it can be checked without a GPU.
#pragma once
#include <math.h>
#include <stdint.h>
#include <string.h>

#ifdef __CUDACC__
#define ARDIFF_BOTH __host__ __device__ __forceinline__
#else
#define ARDIFF_BOTH inline
#endif

namespace ardiff {

// Logits in their order as whole numbers, and back: key_of(x) < key_of(y) just where x < y, both zeros are one number, and no number between
// two logits' is without a logit, so that a range of numbers and the range of the logits at its ends hold the same ones.
ARDIFF_BOTH unsigned key_of(float x) {
    uint32_t b;
    memcpy(&b, &x, 4);
    return b & 0x80000000u ? 0u - b : b | 0x80000000u;
}
ARDIFF_BOTH float value_of(unsigned k) {
    const uint32_t b = k & 0x80000000u ? k & 0x7fffffffu : 0u - k;
    float x;
    memcpy(&x, &b, 4);
    return x;
}

// How many elements of weight w, next to `sure`, it takes to reach `enough`: `in` + 1 if there are not that many, 1 if none is needed.
// The first estimate is held between these before it is stepped, so that every step is one of fp64's own whole numbers: where `sure` is
// far above `enough` the quotient is negative and, for a small w, so large that adding 1 to it changes nothing.
ARDIFF_BOTH double needed(double enough, double sure, double w, unsigned in) {
    double need = fmin(fmax(ceil((enough - sure) / w), 1.0), (double)in + 1.0);
    while (need > 1.0 && sure + (need - 1.0) * w >= enough) need -= 1.0;
    while (need <= (double)in && sure + need * w < enough) need += 1.0;
    return need;
}

}  // namespace ardiff
