// serve_view.hpp -- what the operators around a verification (serve_api.hip) read of a handle.
#pragma once
#include <stdint.h>

struct stand_handle;

namespace stand {

struct ServeView {
    int B, N, D, V, logits_dtype, device, cus;
    const unsigned long long *anc;  // device, [N][anc_words]: ancestor-or-self bit sets of the tree
    int anc_words;
    int *last_hip;                  // where a HIP error of a call is kept
};

__attribute__((visibility("hidden"))) ServeView serve_view(stand_handle *h);

}  // namespace stand
