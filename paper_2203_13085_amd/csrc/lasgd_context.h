// What the library's other translation units see of a context.  The definitions are in lasgd.hip.
#pragma once
#include "../../include/lasgd.h"

namespace lasgd {

struct ContextView {
    int32_t K, n_tensors;
    int device;
    bool bf16;
    bool all_bound;
    const int64_t *numel;          // [n_tensors]
    void *const *params, *const *grads;    // [K][n_tensors], as bound
};

__attribute__((visibility("hidden"))) ContextView view_of(const lasgd_ctx *c);

// Keeps the text for lasgd_last_error and hands back st.
__attribute__((visibility("hidden"), format(printf, 3, 4))) lasgd_status refuse(lasgd_ctx *c, lasgd_status st, const char *fmt, ...);

} // namespace lasgd
