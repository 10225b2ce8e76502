// 8-bit activation checkpoints: q, k, v and out of an attention layer, written after its forward pass and read by its backward
// pass (format: ckpt8.cuh).
//
// Both directions are bound by memory: 2 bytes a value on one side, 33 / 32 on the other.  A warp takes kWarpRuns runs of 32
// values: four lanes a run, 16 bytes of bf16 and 8 of integers a lane, all loads issued before the first is used, and
// the runs' exponent bytes as one 32-byte access.  The tensors of a call share a launch.
#include "common.h"
#include "ckpt8.cuh"

namespace libra {

constexpr int kCkptThreads = 256;

struct CkptArgs {
    CkptTensor t[4];
};

__global__ void __launch_bounds__(kCkptThreads) k_ckpt8_pack(const __grid_constant__ CkptArgs a) {
    grid_dep_wait();
    int64_t run0;
    const CkptTensor t = share_of(a.t, blockIdx.x * (kCkptThreads / 32) + (threadIdx.x >> 5), run0);
    if (run0 >= t.runs) return;
    const int lane = threadIdx.x & 31;
    const int64_t at = run0 * 4 + lane;         // this lane's eight values of step 0
    uint4 x[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        x[u] = make_uint4(0, 0, 0, 0);
        if (run0 + 8 * u + (lane >> 2) < t.runs) x[u] = __ldcs(t.x + at + 32 * u);
    }
    uint32_t mine = 0;                          // exponent of run `lane`
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&x[u]);
        uint32_t m = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
        m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 2));
        uint32_t e = max(m & 0xffffu, m >> 16) >> 7;
        e = e < 7 ? 7 : e;
        const float down = run_down(e);
        uint32_t q[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t b[4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // 1.5 2^23 + y has rint(y) in its low bits, ties to even
                const float lo = __uint_as_float(w[2 * i + j] << 16) * down, hi = __uint_as_float(w[2 * i + j] & 0xffff0000u) * down;
                b[2 * j] = __float_as_uint(fminf(fmaxf(lo, -127.f), 127.f) + 12582912.0f);
                b[2 * j + 1] = __float_as_uint(fminf(fmaxf(hi, -127.f), 127.f) + 12582912.0f);
            }
            q[i] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
        }
        const uint32_t got = __shfl_sync(0xffffffffu, e, (lane & 7) * 4);
        if ((lane >> 3) == u) mine = got;
        if (run0 + 8 * u + (lane >> 2) < t.runs) __stcs(t.q + at + 32 * u, make_uint2(q[0], q[1]));
    }
    if (run0 + lane < t.runs) t.e[run0 + lane] = (uint8_t)mine;
}

__global__ void __launch_bounds__(kCkptThreads) k_ckpt8_unpack(const __grid_constant__ CkptArgs a) {
    grid_dep_wait();
    unpack_share(a.t, blockIdx.x * (kCkptThreads / 32) + (threadIdx.x >> 5));
}

// Memory that a kernel on this device may touch (there is no plan that names the device).
static bool on_device(const void* p, int dev) {
    cudaPointerAttributes at;
    if (cudaPointerGetAttributes(&at, p) != cudaSuccess) { cudaGetLastError(); return false; }
    return at.type == cudaMemoryTypeManaged || (at.type == cudaMemoryTypeDevice && at.device == dev);
}

// pack: x -> held, else held -> x.
static int run_ckpt8(bool pack, const void* const (&x)[4], const libra_ckpt8* c, const libra_dims* dims, cudaStream_t s) {
    if (!c || !dims || dims->total_tokens <= 0 || dims->hq <= 0 || dims->hkv <= 0) return LIBRA_ERR_INVALID_ARG;
    if (dims->head_dim != 64 && dims->head_dim != 128 && dims->head_dim != 256) return LIBRA_ERR_UNSUPPORTED;
    const void* const q[4] = {c->q, c->k, c->v, c->out};
    const void* const e[4] = {c->q_exp, c->k_exp, c->v_exp, c->out_exp};
    const int64_t rows = dims->total_tokens;
    for (const int heads : {dims->hq, dims->hkv})
        if ((long double)rows * heads * dims->head_dim >= 2.0e12L) return LIBRA_ERR_OVERFLOW;   // (a warp's share is numbered in 32 bits)
    CkptArgs a = {};
    int64_t warps = 0;
    for (int k = 0; k < 4; ++k) {
        const int heads = k == 0 || k == 3 ? dims->hq : dims->hkv;
        // a tensor that is not asked for is left out, whether or not the checkpoint has it
        if (!set_tensor(a.t[k], x[k], x[k] ? q[k] : nullptr, x[k] ? e[k] : nullptr, rows * heads * dims->head_dim))
            return LIBRA_ERR_INVALID_ARG;
        warps += a.t[k].chunks;
    }
    if (warps == 0) return LIBRA_OK;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return LIBRA_ERR_NO_DEVICE; }
    for (const CkptTensor& t : a.t)
        if (t.chunks && !(on_device(t.x, dev) && on_device(t.q, dev) && on_device(t.e, dev))) return LIBRA_ERR_INVALID_ARG;
    const int64_t blocks = (warps + kCkptThreads / 32 - 1) / (kCkptThreads / 32);
    if (blocks > INT32_MAX / 16) return LIBRA_ERR_OVERFLOW;
    count_launch();
    const cudaError_t err = launch_dependent(pack ? k_ckpt8_pack : k_ckpt8_unpack, (unsigned)blocks, kCkptThreads, 0, s, a);
    if (err != cudaSuccess) cudaGetLastError();   // not the next call's
    return err == cudaSuccess ? LIBRA_OK : LIBRA_ERR_CUDA;
}

}  // namespace libra

using namespace libra;

extern "C" int libra_ckpt8_pack(const void* q_dev, const void* k_dev, const void* v_dev, const void* out_dev,
                                const libra_ckpt8* ckpt, const libra_dims* dims, void* stream) {
    return run_ckpt8(true, {q_dev, k_dev, v_dev, out_dev}, ckpt, dims, (cudaStream_t)stream);
}

extern "C" int libra_ckpt8_unpack(const libra_ckpt8* ckpt, void* q_dev, void* k_dev, void* v_dev, void* out_dev,
                                  const libra_dims* dims, void* stream) {
    return run_ckpt8(false, {q_dev, k_dev, v_dev, out_dev}, ckpt, dims, (cudaStream_t)stream);
}
