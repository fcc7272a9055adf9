// Checks of arguments that the entry points of rows_api.hip and maps_api.hip share.
#pragma once
#include <stdint.h>
#include <stddef.h>
#include "corr.h"

namespace {

bool known(corr_dtype t) { return t == CORR_TYPE_F32 || t == CORR_TYPE_BF16 || t == CORR_TYPE_F16; }
bool known(corr_activation a) { return a >= CORR_ACT_NONE && a <= CORR_ACT_SIGMOID; }
bool known(corr_norm n) { return n >= CORR_NORM_NONE && n <= CORR_NORM_LAYER; }
bool on(const void* p, int border) { return ((uintptr_t)p & (uintptr_t)(border - 1)) == 0; }

// The bytes [at, end) of a matrix, in rows of `row` bytes `stride` apart, to compare with another's.
struct Range { uintptr_t at, end, row, stride; };
Range range(const void* p, int64_t rows, int64_t cols, int64_t stride, int es) {
    if (!p || rows <= 0) return {0, 0, 0, 0};
    return {(uintptr_t)p, (uintptr_t)p + (uintptr_t)((rows - 1) * stride + cols) * es, (uintptr_t)cols * es, (uintptr_t)stride * es};
}
bool overlap(const Range& a, const Range& b) {
    if (a.at >= b.end || b.at >= a.end) return false;
    if (a.stride != b.stride || !a.stride) return true;
    const uintptr_t off = b.at >= a.at ? (b.at - a.at) % a.stride : (a.stride - (a.at - b.at) % a.stride) % a.stride;
    return off < a.row || off + b.row > a.stride;        // else columns beside each other in one buffer
}
template <int NO, int NI>
bool any_overlap(const Range (&out)[NO], const Range (&in)[NI]) {
    for (int i = 0; i < NO; ++i) {
        for (const Range& r : in) if (overlap(out[i], r)) return true;
        for (int j = 0; j < i; ++j) if (overlap(out[i], out[j])) return true;
    }
    return false;
}

struct Carver {                           // pieces of the workspace on 256-byte borders
    size_t used = 0;
    size_t take(size_t bytes) { const size_t at = used; used = (used + bytes + 255) & ~(size_t)255; return at; }
};

}  // namespace
