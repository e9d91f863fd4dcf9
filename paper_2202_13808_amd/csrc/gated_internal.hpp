// What the sources of the gated projection share (internal header).
#pragma once

#include "common.hpp"
#include "dropit_layers.h"

namespace dropit {

struct WideArgs {
    const void *w, *x;          // weights [2 * hidden][c_in]; token operand [tokens][K]
    int64_t tokens;
    int hidden, c_in;
    int K;                      // forward: c_in, backward: 2 * hidden
    int act;
    const void *bias;
    void *out, *pre;            // forward: h and pre (or null); backward: dx
    int row_tiles, token_tiles; // set by the launch
};

// gated_wide.hip: bf16 products on 256-row tiles
bool gated_wide_takes(int64_t tokens, int c_in, int hidden, bool forward);
dropit_status launch_gated_wide(const WideArgs &a, bool forward, hipStream_t stream);

}  // namespace dropit
