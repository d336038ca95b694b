// A norm of symar_norm as its kernels have it, the same in the library and in a host program that replays it.
#pragma once
#include "symar.h"

namespace symar {

struct Side {
    const void *weight, *bias;
    float eps;
    int   kind, wide, plus_one;            // wide: weight and bias are float32
};

// The kernels read weight and bias by their pointers alone: a norm that is none has none of them, whatever the caller left there.
inline Side side_of(const symar_norm_side_t &s)
{
    if (s.kind == SYMAR_NORM_NONE) return Side{nullptr, nullptr, 0.0f, SYMAR_NORM_NONE, 0, 0};
    return Side{s.weight, s.bias, s.eps, s.kind, s.dtype == SYMAR_F32, s.plus_one};
}

}  // namespace symar
