// 8-bit activation checkpoints: q, k, v and out of an attention layer, written after its forward pass and read by its backward
// pass (format: ckpt8.cuh).
//
// Both directions are bound by memory: 2 bytes a value on one side, 33 / 32 on the other.  A warp takes kWarpRuns runs of 32
// values, issues all of its loads before the first is used and takes the runs' exponent bytes as one 32-byte access.  The tensors
// of a call share a launch.  There and back, 131072 tokens, 32 / 8 heads of 128: 598 + 596 us, 6.8 TB/s.
#include "common.h"
#include "ckpt8.cuh"

namespace libra {

constexpr int kCkptThreads = 256;

struct CkptArgs {
    CkptTensor t[4];
};

// Eight values as integers: 1.5 2^23 + y has rint(y) in its low bits, ties to even.
__device__ __forceinline__ uint2 quant8(const uint4& x, float down) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&x);
    uint32_t q[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t b[4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float lo = __uint_as_float(w[2 * i + j] << 16) * down, hi = __uint_as_float(w[2 * i + j] & 0xffff0000u) * down;
            b[2 * j] = __float_as_uint(fminf(fmaxf(lo, -127.f), 127.f) + 12582912.0f);
            b[2 * j + 1] = __float_as_uint(fminf(fmaxf(hi, -127.f), 127.f) + 12582912.0f);
        }
        q[i] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    }
    return make_uint2(q[0], q[1]);
}
// Two lanes a run: 16 bytes of integers a lane.  (Four lanes a run, as in unpack_shares, with streaming loads and stores: 660 us for
// 131072 tokens, 32 / 8 heads of 128; so with them 631, without 598, 6.8 TB/s; blocks of 1024 threads 830.)
__global__ void __launch_bounds__(kCkptThreads) k_ckpt8_pack(const __grid_constant__ CkptArgs a) {
    grid_dep_wait();
    int64_t run0;
    const CkptTensor t = share_of(a.t, blockIdx.x * (kCkptThreads / 32) + (threadIdx.x >> 5), run0);
    if (run0 >= t.runs) return;
    const int lane = threadIdx.x & 31;
    uint4 x[2][2];                              // two lanes a run, 16 values of it each, two steps
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        x[u][0] = x[u][1] = make_uint4(0, 0, 0, 0);
        if (run0 + 16 * u + (lane >> 1) < t.runs) {
            const uint4* src = t.x + (run0 + 16 * u) * 4 + 2 * lane;
            x[u][0] = __ldg(src);
            x[u][1] = __ldg(src + 1);
        }
    }
    uint32_t mine = 0;                          // exponent of run `lane`
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(&x[u][k]);
            m = __vmaxu2(m, __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu)));
        }
        m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 1));
        uint32_t e = max(m & 0xffffu, m >> 16) >> 7;
        e = e < 7 ? 7 : e;
        const float down = run_down(e);
        const uint2 q0 = quant8(x[u][0], down), q1 = quant8(x[u][1], down);
        const uint32_t got = __shfl_sync(0xffffffffu, e, (lane & 15) * 2);
        if ((lane >> 4) == u) mine = got;
        if (run0 + 16 * u + (lane >> 1) < t.runs) 
            reinterpret_cast<uint4*>(t.q)[(run0 + 16 * u) * 2 + lane] = make_uint4(q0.x, q0.y, q1.x, q1.y);
    }
    if (run0 + lane < t.runs) t.e[run0 + lane] = (uint8_t)mine;
}

__global__ void __launch_bounds__(kCkptThreads) k_ckpt8_unpack(const __grid_constant__ CkptArgs a) {
    grid_dep_wait();
    unpack_shares<1>(a.t, blockIdx.x * (kCkptThreads / 32) + (threadIdx.x >> 5));
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
