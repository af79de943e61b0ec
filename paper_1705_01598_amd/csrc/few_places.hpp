// Where loads of rows start: arithmetic without device code, which the host can go through as well.
#pragma once
#include <stdint.h>

namespace tperm {

constexpr uint32_t kFourBitDepth = 256;     // elements of a row in 4 bits that a wavefront takes in a step

// Elements of a row of `depth` are taken from i on, where there are any: what starts behind the row's end loads the row's first ones, and counts as zeros.
constexpr uint32_t start_in(uint32_t i, uint32_t depth) { return i < depth ? i : 0u; }

// Elements of a row in LDS: whole steps, filled up with zeros, and 16 bytes more so that rows start at different banks.  A step that is not there
// (a wavefront requests two at once) has no such zeros; its loads go by start_in.
constexpr uint32_t staged_pitch(uint32_t width) { return (width + kFourBitDepth - 1) / kFourBitDepth * kFourBitDepth + 8; }

// A hidden row between the two kernels, in binary32: steps of 8 pieces of `each` channels, of which a lane takes one, four channels (a quad) to a load.
// The quads that the lanes of a load take stand side by side, those of even pieces in front, since paired tiles take even and odd pieces in turn: whole lines, or
// halves of them (in the channels' order a load takes 16 bytes of every 32, of 4-bit matrices of every 128: second kernel of 64 tokens x 8 of 128 experts,
// 2048 -> 2 x 1024 bfloat16, 97 us for 92).
constexpr uint32_t hidden_piece(uint32_t piece) { return (piece % 2 * 4 + piece / 2) * 4; }
constexpr uint32_t hidden_quad(uint32_t quad) { return quad * 32; }
// Where channel c stands, and a row's length: whole steps, zeros behind the last channel.
constexpr uint32_t hidden_place(uint32_t c, uint32_t each) {
    const uint32_t step = 8 * each;
    return c / step * step + hidden_quad(c % each / 4) + hidden_piece(c % step / each) + c % 4;
}
constexpr uint32_t hidden_pitch(uint32_t hidden, uint32_t each) { return (hidden + 8 * each - 1) / (8 * each) * (8 * each); }

}  // namespace tperm
