// Host-side helpers of the entry points.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <cstdio>
#include <cstdlib>

namespace eora {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

// Set EORA_VERBOSE=1 to have a refused launch explain itself on stderr.
inline bool failed(hipError_t e, const char* what)
{
    if (e == hipSuccess) return false;
    static const bool verbose = getenv("EORA_VERBOSE") != nullptr;      // read once per process
    if (verbose) fprintf(stderr, "eora: %s: %s\n", what, hipGetErrorString(e));
    return true;
}

}  // namespace eora
