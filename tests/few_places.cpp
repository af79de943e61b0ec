// Goes through the loads that the layer for a few tokens makes of tokens in LDS, for every width, and of hidden rows between its kernels, for many lengths, and
// prints the first one that leaves its row or finds other channels than it should.
#include <cstdio>
#include <vector>

#include "few_places.hpp"

using namespace tperm;

// Elements from the row's start to behind the last one that a load of 8 at element i reads.  all: the steps that are requested are there as a whole.
static uint32_t reaches(bool all, uint32_t i, uint32_t width) { return (all ? i : start_in(i, width)) + 8; }

// Channels of a lane's quads, and that every place of a row is one channel's.
static bool hidden_rows(uint64_t* loads) {
    for (uint32_t each : {4u, 8u, 32u})
        for (uint32_t hidden = 1; hidden <= 1300; ++hidden) {
            const uint32_t pitch = hidden_pitch(hidden, each), step = 8 * each;
            bool good = pitch >= hidden && pitch < hidden + step && pitch % step == 0;
            std::vector<uint32_t> channel(pitch, pitch);
            for (uint32_t c = 0; c < pitch; ++c) {
                const uint32_t at = hidden_place(c, each);
                good = good && at < pitch && at % 4 == c % 4 && channel[at] == pitch;
                if (good) channel[at] = c;
            }
            // a wavefront's steps, up to eight requested at once
            for (uint32_t i = 0; good && i < pitch + 7 * step; i += step)
                for (uint32_t piece = 0; piece < 8; ++piece)
                    for (uint32_t quad = 0; quad < each / 4; ++quad, ++*loads) {
                        const uint32_t at = start_in(i, hidden) + hidden_piece(piece) + hidden_quad(quad);
                        good = good && at % 4 == 0 && at + 4 <= pitch && (i >= hidden || channel[at] == i + piece * each + quad * 4);
                    }
            if (!good) {
                std::printf("hidden rows of %u, pieces of %u\n", hidden, each);
                return false;
            }
        }
    return true;
}

int main(int argc, char**) {
    uint64_t loads = 0;
    if (argc == 1 && !hidden_rows(&loads)) return 1;     // with an argument: tokens alone
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
