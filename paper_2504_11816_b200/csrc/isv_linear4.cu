// Decode linear layers with 4-bit weights and a 16-bit scale per (row, group of k): y = x . w^T for a few tokens.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <new>

#include "../../include/isv.h"

namespace isv {
int set_error(int code, const char *msg);
}

namespace {

int err(int code, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return isv::set_error(code, buf);
}

// Makes a device current for the length of a call.
struct OnDevice {
    int before = -1;
    cudaError_t e;
    explicit OnDevice(int dev) {
        e = cudaGetDevice(&before);
        if (e == cudaSuccess && before != dev) e = cudaSetDevice(dev);
        else if (e == cudaSuccess) before = -1;
    }
    ~OnDevice() {
        if (before >= 0) cudaSetDevice(before);
    }
};

struct Linear4Params {
    const uint8_t *w;          // [N][K / 2]
    const uint16_t *scales;    // [N][K / group]
    const uint16_t *x;
    uint16_t *y;
    float *y_f32;
    int32_t M, N, K, group, bf16;
};

__device__ __forceinline__ float to_f32(uint16_t b, int bf16) {
    return bf16 ? __bfloat162float(__ushort_as_bfloat16(b)) : __half2float(__ushort_as_half(b));
}

// One warp per output value.
__global__ void linear4_kernel(Linear4Params p) {
    const long long id = (long long)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
    const int lane = threadIdx.x % 32;
    if (id >= (long long)p.M * p.N) return;
    const int m = (int)(id % p.M), n = (int)(id / p.M);
    float sum = 0.f;
    for (int g = 0; g < p.K / p.group; ++g) {
        float part = 0.f;
        for (int i = lane; i < p.group / 2; i += 32) {
            const int k = g * p.group + 2 * i;
            const uint8_t b = p.w[(size_t)n * (p.K / 2) + k / 2];
            part += (float)((b & 15) - 8) * to_f32(p.x[(size_t)m * p.K + k], p.bf16);
            part += (float)((b >> 4) - 8) * to_f32(p.x[(size_t)m * p.K + k + 1], p.bf16);
        }
        sum += part * to_f32(p.scales[(size_t)n * (p.K / p.group) + g], p.bf16);
    }
    for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane) return;
    const size_t at = (size_t)m * p.N + n;
    if (p.y_f32) p.y_f32[at] = sum;
    if (p.y) p.y[at] = p.bf16 ? __bfloat16_as_ushort(__float2bfloat16(sum)) : __half_as_ushort(__float2half(sum));
}

}  // namespace

struct isv_linear4 {
    int N = 0, K = 0, group = 0, max_M = 0, device = 0;
    bool bf16 = false;
    uint8_t *w = nullptr;
    uint16_t *scales = nullptr;
};

extern "C" {

int isv_linear4_free(isv_linear4 *l) {
    if (!l) return err(ISV_EINVAL, "null handle");
    OnDevice on(l->device);
    cudaDeviceSynchronize();   // calls may have been made on any stream
    cudaFree(l->w);
    cudaFree(l->scales);
    delete l;
    return ISV_OK;
}

int isv_linear4_create(isv_linear4 **out, const void *w4_dev, const void *scales_dev, int32_t N, int32_t K, int32_t group,
                       int32_t dtype, int32_t max_M, void *stream) {
    if (!out) return err(ISV_EINVAL, "out is null");
    *out = nullptr;
    if (!w4_dev || !scales_dev) return err(ISV_EINVAL, "isv_linear4_create: weights and scales are required");
    if (reinterpret_cast<uintptr_t>(scales_dev) & 1u) return err(ISV_EINVAL, "isv_linear4_create: scales must be 2-byte aligned");
    if (group != 32 && group != 64 && group != 128) return err(ISV_EINVAL, "isv_linear4_create: group (%d) must be 32, 64 or 128", group);
    if (N < 1 || N > (1 << 24)) return err(ISV_EINVAL, "isv_linear4_create: bad N (%d)", N);
    if (K < group || K % group != 0 || K > (1 << 20)) return err(ISV_EINVAL, "isv_linear4_create: K (%d) must be a multiple of the group (%d)", K, group);
    if (max_M < 1 || max_M > 64) return err(ISV_EINVAL, "isv_linear4_create: max_M (%d) must be in [1, 64]", max_M);
    if (dtype != ISV_F16 && dtype != ISV_BF16) return err(ISV_EINVAL, "dtype must be ISV_F16 or ISV_BF16");
    isv_linear4 *l = new (std::nothrow) isv_linear4();
    if (!l) return err(ISV_EINVAL, "out of host memory");
    l->N = N; l->K = K; l->group = group; l->max_M = max_M; l->bf16 = dtype == ISV_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const size_t wb = (size_t)N * (K / 2), sb = (size_t)N * (K / group) * 2;
    cudaError_t e = cudaGetDevice(&l->device);
    if (e == cudaSuccess) e = cudaMalloc((void **)&l->w, wb);
    if (e == cudaSuccess) e = cudaMalloc((void **)&l->scales, sb);
    if (e == cudaSuccess) e = cudaMemcpyAsync(l->w, w4_dev, wb, cudaMemcpyDeviceToDevice, st);
    if (e == cudaSuccess) e = cudaMemcpyAsync(l->scales, scales_dev, sb, cudaMemcpyDeviceToDevice, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) {
        cudaGetLastError();
        isv_linear4_free(l);
        return err(e == cudaErrorMemoryAllocation ? ISV_ENOMEM_DEVICE : ISV_ECUDA, "isv_linear4_create: %s", cudaGetErrorString(e));
    }
    *out = l;
    return ISV_OK;
}

int isv_linear4_forward(isv_linear4 *l, const void *x_dev, void *y_dev, float *y_f32_dev, int32_t M, void *stream) {
    if (!l) return err(ISV_EINVAL, "null handle");
    if (!x_dev || (!y_dev && !y_f32_dev)) return err(ISV_EINVAL, "x and one of y / y_f32 must be given");
    if (reinterpret_cast<uintptr_t>(x_dev) & 15u) return err(ISV_EINVAL, "x must be 16-byte aligned");
    if (M < 1 || M > l->max_M) return err(ISV_EINVAL, "M (%d) must be in [1, %d]", M, l->max_M);
    if ((reinterpret_cast<uintptr_t>(y_dev) & 1u) || (reinterpret_cast<uintptr_t>(y_f32_dev) & 3u))
        return err(ISV_EINVAL, "outputs must be aligned to their elements");
    Linear4Params p{};
    p.w = l->w; p.scales = l->scales; p.x = static_cast<const uint16_t *>(x_dev);
    p.y = static_cast<uint16_t *>(y_dev); p.y_f32 = y_f32_dev;
    p.M = M; p.N = l->N; p.K = l->K; p.group = l->group; p.bf16 = l->bf16;
    OnDevice on(l->device);
    if (on.e != cudaSuccess) return err(ISV_ECUDA, "isv_linear4_forward: %s", cudaGetErrorString(on.e));
    linear4_kernel<<<(unsigned)(((long long)M * l->N + 3) / 4), 128, 0, static_cast<cudaStream_t>(stream)>>>(p);
    cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ISV_OK : err(ISV_ECUDA, "isv_linear4_forward: %s", cudaGetErrorString(e));
}

}  // extern "C"
