// qnn_f8_matmul: the plan for a size, and the launches of its parts.
#pragma once

#include "f8.h"

namespace qnn {

enum class F8Kernel { Rows, Rows64, Tile128, Tile256 };
struct F8Plan {
    F8Kernel kernel;
    int splits;     // parts that K is in, each written down (tiles)
    float us;       // estimated time
    bool padded;    // rows that are no whole 16-byte pieces are copied into padded ones first
    size_t x_bytes, w_bytes, bytes; // of the workspace: those copies, and all with the sums of parts
};
F8Plan f8_plan(int64_t M, int64_t N, int64_t K, int type);

inline int64_t f8_padded(int64_t K) { return (K + 15) / 16 * 16; }

// x and w (or their padded copies) have rows of whole 16-byte pieces
void launch_f8_tiles(const F8Args &a, const F8Plan &plan, float *parts, hipStream_t s);
void launch_f8_pad(const F8Args &a, uint8_t *x, uint8_t *w, hipStream_t s);

} // namespace qnn
