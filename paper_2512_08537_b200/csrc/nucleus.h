// Arithmetic of the search for a nucleus' end, in host and device code alike, so that it can be checked without a GPU.
#pragma once
#include <math.h>
#include <stdint.h>

#ifdef __CUDACC__
#define ARDIFF_BOTH __host__ __device__ __forceinline__
#else
#define ARDIFF_BOTH inline
#endif

namespace ardiff {

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
