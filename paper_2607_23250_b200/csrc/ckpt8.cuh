// The 8-bit checkpoint format, for the kernels that write and read it.
//
// A run of 32 values along the head dimension shares an exponent byte E = max(exponent field of its largest magnitude, 7);
// x is held as the integer rint(x 2^(133 - E)), ties to even, at most 127 in magnitude, and stands for that integer times
// 2^(E - 133).  Powers of two: neither scaling rounds, the integers have seven bits, so what is read back is exact in bf16 and in
// the product sums of fp32, and the one rounding is the integer's, half a step at most: 2^-7 of the largest power of two not
// above the run's largest magnitude.  (A bf16 below 2^E' x 2 is at most 255 / 128 x 2^E', so only 127.5 could round to
// 128; clamped, it is half a step off as well.)  E = 255: the run holds an infinity or a NaN and reads as NaN.  With E >= 7
// the factor 2^(133 - E) is a finite fp32 number; values below 2^-127 of such runs read as zero.
// (The published MXINT8 layout, integers in blocks of 32 with a power of two each, with a floor on the exponent.)
// An absolute scale per run (its largest magnitude / 127) would make the step up to two times finer, round what is read back once
// more, to bf16, and take four bytes a run instead of one.
#pragma once
#include <stdint.h>

#include "../../include/libra.h"
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

// How warps share a call's tensors: kWarpRuns runs of one of them each; read back four lanes a run, 16 bytes of bf16 and 8 of integers a
// lane and step; the runs' exponents are one 32-byte access.
constexpr int kSteps = 4;                       // runs a lane takes part in
constexpr int kWarpRuns = 8 * kSteps;
// Of a warp of the kernel that restores q, k and v among the row statistics: its CTAs have the registers of that kernel, so fewer
// warps fit an SM.  Both together, 65536 tokens, 8 / 2 heads of 128: 111 us with one share a warp, 103 with two, 90 with four (0.51 GB).
constexpr int kRestoreShares = 4;

struct CkptTensor {
    uint4* x;               // bf16, 8 values each
    uint2* q;               // integers, 8 each
    uint8_t* e;             // exponents
    int64_t runs;
    uint32_t chunks;        // warps' shares of it
};

// The tensor of warp w's share and its first run (selected, not indexed: an index into a kernel's arguments would copy them to
// local memory).
template <int N>
__device__ __forceinline__ CkptTensor share_of(const CkptTensor (&all)[N], uint32_t w, int64_t& run0) {
    CkptTensor t = all[0];
#pragma unroll
    for (int k = 1; k < N; ++k)
        if (w >= t.chunks) { w -= t.chunks; t = all[k]; }
    if (w >= t.chunks) t.runs = 0;
    run0 = (int64_t)w * kWarpRuns;
    return t;
}
// Reads the shares M w .. M w + M - 1 back as bf16 (all of one tensor: its shares are counted in multiples of M), the loads of all of
// them first.
template <int M, int N>
__device__ __forceinline__ void unpack_shares(const CkptTensor (&all)[N], uint32_t w_) {
    int64_t run0;
    const CkptTensor t = share_of(all, M * w_, run0);
    if (run0 >= t.runs) return;
    const int lane = threadIdx.x & 31;
    const int64_t at = run0 * 4 + lane;
    uint2 q[M * kSteps];
    uint32_t mine[M];
#pragma unroll
    for (int u = 0; u < M * kSteps; ++u) {
        q[u] = make_uint2(0, 0);
        if (run0 + 8 * u + (lane >> 2) < t.runs) q[u] = __ldcs(t.q + at + 32 * u);
    }
#pragma unroll
    for (int k = 0; k < M; ++k) mine[k] = run0 + 32 * k + lane < t.runs ? t.e[run0 + 32 * k + lane] : 7u;
#pragma unroll
    for (int u = 0; u < M * kSteps; ++u) {
        const float up = run_up(__shfl_sync(0xffffffffu, mine[u / kSteps], 8 * (u % kSteps) + (lane >> 2)));
        float f[8];
        held_floats(q[u].x, f);
        held_floats(q[u].y, f + 4);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(f[2 * i] * up, f[2 * i + 1] * up);
        if (run0 + 8 * u + (lane >> 2) < t.runs) t.x[at + 32 * u] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// One tensor of a call: null everywhere = left out.  Returns false where only some of its pointers are given or misaligned.
inline bool set_tensor(CkptTensor& t, const void* x, const void* q, const void* e, int64_t values, int shares = 1) {
    t = {};
    if (!x && !q && !e) return true;
    if (!x || !q || !e || (((uintptr_t)x | (uintptr_t)q) & 15)) return false;
    t.x = (uint4*)x;
    t.q = (uint2*)q;
    t.e = (uint8_t*)e;
    t.runs = values / kRun;
    t.chunks = (uint32_t)((t.runs + shares * kWarpRuns - 1) / (shares * kWarpRuns) * shares);   // (the last ones may be empty)
    return true;
}

// q, k and v of a checkpoint and where they are restored.
inline bool set_restore(CkptTensor (&t)[3], const libra_ckpt8* c, void* q, void* k, void* v, const libra_dims* dims) {
    const int64_t row = dims->total_tokens * dims->head_dim;
    return set_tensor(t[0], q, c->q, c->q_exp, row * dims->hq, kRestoreShares) &&
           set_tensor(t[1], k, c->k, c->k_exp, row * dims->hkv, kRestoreShares) &&
           set_tensor(t[2], v, c->v, c->v_exp, row * dims->hkv, kRestoreShares);
}

}  // namespace libra
