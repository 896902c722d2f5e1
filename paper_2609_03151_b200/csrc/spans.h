// Host-side argument checks of calls that take several tables of device pointers: presence, alignment, overlap.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "plan.h"

// Device buffers of one call, inputs and outputs, in the order they are added.  `slot` ties an output to the one input
// that it may be (exactly, same address): a step that reads a vector whole before it writes it can run in place.
struct SpanSet {
    static constexpr int kMax = 10 * BASP_MAX_RANKS;
    struct Span { uintptr_t p; size_t n; int slot; };
    Span in[kMax], out[kMax];
    int n_in = 0, n_out = 0;

    static int check(const void *p, unsigned align) {
        if (!p) return BASP_ERR_NULL;
        return ((uintptr_t)p & (align - 1)) ? BASP_ERR_ALIGN : BASP_OK;
    }
    int add_in(const void *p, size_t bytes, unsigned align = 16, int slot = -1) {
        in[n_in++] = Span{(uintptr_t)p, bytes, slot};
        return check(p, align);
    }
    int add_out(const void *p, size_t bytes, unsigned align = 16, int slot = -1) {
        out[n_out++] = Span{(uintptr_t)p, bytes, slot};
        return check(p, align);
    }
    static bool meet(const Span &a, const Span &b) { return a.p < b.p + b.n && b.p < a.p + a.n; }
    // BASP_ERR_ALIAS where an output overlaps another output, or an input that it may not be
    int overlaps() const {
        for (int i = 0; i < n_out; ++i) {
            for (int j = 0; j < i; ++j)
                if (meet(out[i], out[j])) return BASP_ERR_ALIAS;
            for (int j = 0; j < n_in; ++j)
                if (meet(out[i], in[j]) && !(out[i].slot >= 0 && out[i].slot == in[j].slot && out[i].p == in[j].p))
                    return BASP_ERR_ALIAS;
        }
        return BASP_OK;
    }
};

// BASP_TRY(expr): leave the calling function with the first error code
#define BASP_TRY(expr)                       \
    do {                                     \
        const int rc_ = (expr);              \
        if (rc_ != BASP_OK) return rc_;      \
    } while (0)
