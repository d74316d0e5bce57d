// What the norms (norm.hip, layernorm.hip) share: where a row's values lie in its lanes'
// registers, its largest width, and the parts of a backward.
#pragma once
#include "seq.h"

namespace gorila {

constexpr int MAX_ROW = 65536;

// A row in the registers of its LANES lanes, QUADS runs of four values each.  W: values
// a load (8: two quads of bf16 side by side; 4; 1: no alignment).
template <int W, int LANES>
__device__ __forceinline__ int column(int l, int i) {
    return W == 8 ? (l + (i >> 1) * LANES) * 8 + (i & 1) * 4 : (l + i * LANES) * 4;
}

// Workgroups of a backward, a part each: two of eight waves a compute unit.
constexpr int NORM_PARTS = 512;

}  // namespace gorila
