// Argument checks and workspace carving shared by the entry points' translation units (host code).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/la.h"
#include "la_plan.h"

namespace la_check {
using la_plan::align256;

inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// Aliasing: no buffer that a call writes may overlap any other buffer of the call.
struct Span {
    const void *p;
    size_t bytes;
};
inline bool overlap(const Span &a, const Span &b) {
    if (a.p == nullptr || b.p == nullptr || a.bytes == 0 || b.bytes == 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return x < y + b.bytes && y < x + a.bytes;
}
// outs: written (or read and written); ins: read only
template <size_t NO, size_t NI>
bool aliased(const Span (&outs)[NO], const Span (&ins)[NI]) {
    for (size_t i = 0; i < NO; ++i) {
        for (size_t j = i + 1; j < NO; ++j)
            if (overlap(outs[i], outs[j])) return true;
        for (size_t j = 0; j < NI; ++j)
            if (overlap(outs[i], ins[j])) return true;
    }
    return false;
}

struct Carver {
    char *base;
    size_t off;
    void *take(size_t bytes) {
        void *p = base + off;
        off += align256(bytes);
        return p;
    }
};

inline int hip_status(hipError_t e) { return e == hipSuccess ? LA_OK : LA_ERR_HIP; }

}  // namespace la_check
