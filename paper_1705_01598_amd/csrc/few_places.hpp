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

}  // namespace tperm
