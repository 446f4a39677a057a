// Shared parts of the gated delta rule's kernels.
#pragma once

#include "common.hpp"
#include "libspyke_readout.h"

namespace spk {
namespace delta {

struct Args {
    int dtype, B, L, Hk, Hv, dk, dv;
    float scale;
};

// Sizes and flags of a call; SPK_OK or the recorded error.
int check(const Args &a, const char *name);

// The batch call over chunks of samples, and the bytes of its workspace.
size_t chunk_workspace(const Args &a);
int chunk_forward(const void *q, const void *k, const void *v, const float *g, const float *beta, const Args &a,
                  const int32_t *lengths, const float *state_in, void *out, float *state_out, void *ws, hipStream_t st,
                  const char *name);

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// bfloat16 elements are carried as uint16_t.
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
template <class E>
__device__ __forceinline__ E from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ uint16_t from_float<uint16_t>(float v) {
    return __builtin_bit_cast(uint16_t, (__bf16)v);  // to nearest, ties to even
}

}  // namespace delta
}  // namespace spk
