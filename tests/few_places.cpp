// Goes through the loads that the layer for a few tokens makes of tokens in LDS, for every width, and prints the first one that leaves its row.
#include <cstdio>
#include <cstdlib>

#include "few_places.hpp"

using namespace tperm;

// Elements from the row's start to behind the last one that a load of 8 at element i reads.  all: the steps that are requested are there as a whole.
static uint32_t reaches(bool all, uint32_t i, uint32_t width) { return (all ? i : start_in(i, width)) + 8; }

int main() {
    uint64_t loads = 0;
    for (uint32_t width = 1; width <= 2100; ++width)
        for (uint32_t steps = 1; steps <= 2; ++steps)
            for (uint32_t waves = 1; waves <= 8; waves *= 2)
                for (uint32_t wave = 0; wave < waves; ++wave) {
                    const uint32_t block = steps * kFourBitDepth;
                    uint32_t i = wave * block;
                    for (; i < width; i += waves * block) {
                        const bool all = i + block <= width;        // else the row's end is in it
                        for (uint32_t t = 0; t < steps; ++t)
                            for (uint32_t piece = 0; piece < 8; ++piece)
                                for (uint32_t j = 0; j < 4; ++j, ++loads) {
                                    const uint32_t at = i + t * kFourBitDepth + piece * 32 + j * 8, end = reaches(all, at, width);
                                    if (end > staged_pitch(width)) {
                                        std::printf("width %u, %u steps, wavefront %u of %u: element %u reads to %u of %u\n", width, steps, wave, waves, at, end, staged_pitch(width));
                                        return 1;
                                    }
                                }
                    }
                }
    std::printf("ok: %llu loads\n", (unsigned long long)loads);
    return 0;
}
