// The end of a ring of stages that was given up: what is still to be waited for, so that nothing is on its way into shared memory when its CTA
// leaves.  Device code; it compiles as plain C++ too.
#pragma once

#ifdef __CUDACC__
#define VP_DRAIN __device__ __forceinline__
#else
#define VP_DRAIN inline
#endif

// A stage's barrier ends its phase with one arrival of each maker and the bytes that were asked for with them; stage q of the sequence uses
// barrier q % stages, phase q / stages.  made[i]: stages that maker i has arrived for; the first `loaders` makers ask for bytes.  None of them
// goes on any more.  Only the last `stages` that anyone has asked bytes for can be unfinished (a barrier is used again when its stage
// has been read); arrivals that they lack are made here, and then their phases end with their bytes.
template <typename Arrive, typename Wait>
VP_DRAIN void drain_ring(const unsigned long long* made, int makers, int loaders, int stages, Arrive arrive, Wait wait) {
    unsigned long long asked = 0;
    for (int i = 0; i < loaders; i++) asked = made[i] > asked ? made[i] : asked;
    for (unsigned long long q = asked > (unsigned)stages ? asked - stages : 0; q < asked; q++) {
        const int at = (int)(q % stages);
        for (int i = 0; i < makers; i++)
            if (made[i] <= q) arrive(at);
        wait(at, (unsigned)(q / stages) & 1);
    }
}
