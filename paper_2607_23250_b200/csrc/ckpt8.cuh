// The 8-bit checkpoint format, for the kernels that write and read it.
//
// A run of 32 values along the head dimension shares an exponent byte E = max(exponent field of its largest magnitude, 7);
// x is held as the integer rint(x 2^(133 - E)), ties to even, at most 127 in magnitude, and stands for that integer times
// 2^(E - 133).  Powers of two: neither scaling rounds, the integers have seven bits, so what is read back is exact in bf16 and in
// the product sums of fp32, and the one rounding is the integer's, half a step at most: 2^-7 of the largest power of two not
// above the run's largest magnitude.  (A bf16 below 2^E' x 2 is at most 255 / 128 x 2^E', so only 127.5 could round to
// 128; clamped, it is half a step off as well.)  E = 255: the run holds an infinity or a NaN and reads as NaN.  With E >= 7
// the factor 2^(133 - E) is a finite fp32 number; values below 2^-127 of such runs read as zero.
// An absolute scale per run (its largest magnitude / 127) would make the step up to two times finer, round what is read back once
// more, to bf16, and take four bytes a run instead of one.
#pragma once
#include <stdint.h>

#include "ptx.cuh"

namespace libra {

constexpr int kRun = 32;             // values that share an exponent
constexpr uint32_t kRunNaN = 255;

__device__ __forceinline__ float run_down(uint32_t e) { return __uint_as_float((260u - e) << 23); }   // 2^(133 - E)
__device__ __forceinline__ float run_up(uint32_t e) {                                                    // 2^(E - 133)
    return e == kRunNaN ? __uint_as_float(0x7fffffffu) : __uint_as_float((e - 6u) << 23);
}
// Four held integers of a word as floats: 2^23 + 128 + q is put together from bytes (a conversion instruction an element
// runs at a quarter of this rate).
__device__ __forceinline__ void held_floats(uint32_t w, float* f) {
    const uint32_t u = w ^ 0x80808080u;   // q + 128
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7540 + i)) - 8388736.0f;
}

}  // namespace libra
