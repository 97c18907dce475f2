// Shared helpers of the policy-network operators (embedding, query/key norm and rotation, attention).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "rapid_common.cuh"
#include "rapid_policy_ops.h"

namespace rapid {
namespace policy {

static_assert(sizeof(rapid_embed_desc_t) == 48 && sizeof(rapid_qk_desc_t) == 88 && sizeof(rapid_attn_desc_t) == 104, "bindings rely on these");

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t elem_size(int32_t dtype) { return dtype == RAPID_BF16 ? 2 : 4; }

// Whether two byte ranges share a byte.
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

// Bytes from the first element of `n` rows of `width` elements at pitch `ld` to the end of the last.
inline size_t extent(int64_t n, int64_t width, int64_t ld, size_t es) { return ((size_t)(n - 1) * ld + width) * es; }

// Two matrices of `na` and `nb` rows, `wa` and `wb` bytes wide, at pitches of `pa` and `pb` bytes: do they share a byte?  Matrices of
// one pitch may lie side by side in the same rows (queries, keys and values of one projection); of two pitches, they have to be
// apart altogether.
inline bool matrices_overlap(const void* a, int64_t na, int64_t wa, int64_t pa, const void* b, int64_t nb, int64_t wb, int64_t pb) {
    if (!overlap(a, extent(na, wa, pa, 1), b, extent(nb, wb, pb, 1))) return false;
    if (pa != pb) return true;
    int64_t off = ((int64_t)reinterpret_cast<uintptr_t>(b) - (int64_t)reinterpret_cast<uintptr_t>(a)) % pa;
    if (off < 0) off += pa;
    return off < wa || off + wb > pa;
}
// The same for `n` rows each, widths and pitches in elements of `es` bytes.
inline bool rows_overlap(const void* a, int64_t wa, int64_t lda, const void* b, int64_t wb, int64_t ldb, int64_t n, size_t es) {
    const int64_t e = (int64_t)es;
    return matrices_overlap(a, n, wa * e, lda * e, b, n, wb * e, ldb * e);
}

// sm_100 only.  Returns the SM count of the current device through *sm_count.
inline rapid_status_t check_device(int* sm_count) {
    int dev = 0, major = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return RAPID_ERR_CUDA;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(sm_count, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return RAPID_ERR_CUDA;
    return major == 10 ? RAPID_OK : RAPID_ERR_UNSUPPORTED;
}

// A kernel whose last resort is "gave up waiting" reports through here; see rapid_stats_t.
inline cudaError_t clear_stats(rapid_stats_t* stats, cudaStream_t st) {
    return stats ? cudaMemsetAsync(stats, 0, sizeof(rapid_stats_t), st) : cudaSuccess;
}

#ifdef __CUDACC__

// Eight consecutive elements as floats, and back; bf16: one 16-byte access, float: two.
template <class T>
struct Vec8;
template <>
struct Vec8<uint16_t> {
    uint4 u;
    __device__ __forceinline__ void load(const uint16_t* p) { u = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = bf16_lo(w[i]);
            f[2 * i + 1] = bf16_hi(w[i]);
        }
    }
    __device__ __forceinline__ static void store(uint16_t* p, const float (&f)[8]) {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                                  pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
    }
};
template <>
struct Vec8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = reinterpret_cast<const float4*>(p)[0];
        b = reinterpret_cast<const float4*>(p)[1];
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    }
    __device__ __forceinline__ static void store(float* p, const float (&f)[8]) {
        reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void from_float(float* p, float x) { *p = x; }
__device__ __forceinline__ void from_float(uint16_t* p, float x) { *p = (uint16_t)pack_bf16x2(x, 0.f); }

#endif  // __CUDACC__

}  // namespace policy
}  // namespace rapid
