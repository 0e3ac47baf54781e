// lif_types.hpp -- the element types of the sequence and answer operators
// (float32, bfloat16, float16): conversion to and from float32, and loads and
// stores of several contiguous elements by one lane.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/lif.h"

namespace lif {

using bf16 = __bf16;
using f16 = _Float16;

template <typename T> __device__ __forceinline__ float to_f32(T v) { return (float)v; }

// One rounding to nearest even.
template <typename T> __device__ __forceinline__ T from_f32(float v) { return (T)v; }

// Calls fn with a value of the element type that `dtype` names; false for a
// type there is none of.
template <typename Fn> bool with_dtype(int dtype, Fn&& fn)
{
    switch (dtype) {
        case LIF_F32: fn(float()); return true;
        case LIF_BF16: fn(bf16()); return true;
        case LIF_F16: fn(f16()); return true;
        default: return false;
    }
}

}  // namespace lif
