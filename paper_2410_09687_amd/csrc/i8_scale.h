// The sums of the integer products to fp32, v s_t s_o: the same steps in every kernel.
#pragma once
#include <hip/hip_runtime.h>

namespace moin {

// A token's scale.  The scales' product may leave fp32's range where the result does not, so the sum is taken times s_t, then times s_o: a sum that is not 0 has a
// magnitude of 1 to 2^31 and scales are 2^-126 at least, so v s_t is a normal number as long as s_t is below 2^97.  Larger ones (rows with values beyond 2e31) go
// in divided by 2^32, and the result is multiplied by that.
__device__ __forceinline__ float i8_result(int v, float s, float far, float so) { return (float)v * s * so * far; }
struct I8Token {
    float s, far;
    __device__ __forceinline__ explicit I8Token(float st) : s(st >= 0x1p97f ? st * 0x1p-32f : st), far(st >= 0x1p97f ? 0x1p32f : 1.f) {}
    __device__ __forceinline__ float operator()(int v, float so) const { return i8_result(v, s, far, so); }
};

}  // namespace moin
