// What the sources of the gated projection share (internal header).
#pragma once

#include "common.hpp"
#include "dropit_layers.h"

namespace dropit {

struct WideArgs {
    const void *w, *x;          // weights [2 * hidden][w_pitch]; token operand [tokens][x_pitch]: pitches in elements, of 8
    int w_pitch, x_pitch;
    int64_t tokens;
    int hidden, c_in;
    int K;                      // forward: c_in (its padding counts: zeros), backward: 2 * hidden
    int act;
    const void *bias;
    void *out, *pre;            // forward: h and pre (or null); backward: dx
    float *partial;             // splits > 1: [splits][tokens][width], width = 2 * hidden (forward) or c_in (backward)
    int splits;
    int row_tiles, token_tiles; // set by the launch
};

// gated_wide.hip: bf16 products on 256-row tiles.  The plan says whether a product (of rows in whole 16-byte units) is one for
// it, how many tokens its tiles have, into how many slices the sum is cut and what it is expected to take; with more than one
// slice, the launch writes partial sums and no outputs.
struct WidePlan {
    bool takes;
    int fn, splits;
    double us;
};
WidePlan gated_wide_plan(int64_t tokens, int64_t c_in, int64_t hidden, bool forward);
dropit_status launch_gated_wide(const WideArgs &a, const WidePlan &plan, bool forward, hipStream_t stream);

// gated_tokens.hip: the forward pass for few tokens
bool gated_tokens_takes(int64_t tokens, int64_t c_in, int64_t hidden, dropit_dtype dt);
dropit_status launch_gated_tokens(const void *x, int64_t tokens, int c_in, dropit_dtype dt, const void *w, const void *bias,
                                  int hidden, int act, void *h, void *pre, hipStream_t stream);

}  // namespace dropit
