// RMSNorm over rows and its backward pass (ee_rms_norm, ee_rms_norm_backward):
//   r = 1 / sqrt(mean x^2 + eps),  y = x r g
//   dx = r (g dy - x r^2 mean(g dy x)),  dg = sum over rows of dy x r
// Both are bound by reading their inputs and writing their result once.  A CTA
// takes rows blockIdx, blockIdx + grid, ...; a thread keeps the same columns in
// every row, so that its share of the gain's gradient stays in registers until
// the end, and loads the next row's columns before it reduces this one's.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ee_internal.h"

namespace ee {
namespace {

constexpr int kNormThreads = 512;  // at most
constexpr unsigned kFull = 0xffffffffu;

struct Rows {
    const void* p;
    int64_t ld;
    int type;
};

__device__ __forceinline__ int bytes_of(int type) { return type == EE_FP32 ? 4 : 2; }

// Columns [8 j, 8 j + 8) of a row of d; columns past d read as 0.
__device__ __forceinline__ void load8(const void* row, int type, int j, int d, float (&x)[8]) {
    const int c = 8 * j;
    const char* p = (const char*)row + (int64_t)c * bytes_of(type);
    if (c + 8 <= d && ((uintptr_t)p & 15) == 0) {
        uint4 a = *(const uint4*)p;
        if (type == EE_FP32) {
            const uint4 b = *(const uint4*)(p + 16);
            x[0] = __uint_as_float(a.x), x[1] = __uint_as_float(a.y), x[2] = __uint_as_float(a.z);
            x[3] = __uint_as_float(a.w), x[4] = __uint_as_float(b.x), x[5] = __uint_as_float(b.y);
            x[6] = __uint_as_float(b.z), x[7] = __uint_as_float(b.w);
        } else {
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (type == EE_BF16) {
                    x[2 * i] = __uint_as_float(w[i] << 16);
                    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                } else {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                    x[2 * i] = f.x, x[2 * i + 1] = f.y;
                }
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = 0.f;
        if (c + i < d) {
            if (type == EE_FP32) x[i] = ((const float*)p)[i];
            else if (type == EE_BF16) x[i] = __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
            else x[i] = __half2float(((const __half*)p)[i]);
        }
    }
}

__device__ __forceinline__ void store8(void* row, int type, int j, int d, const float (&x)[8]) {
    const int c = 8 * j;
    char* p = (char*)row + (int64_t)c * bytes_of(type);
    if (type == EE_FP32) {
        if (c + 8 <= d && ((uintptr_t)p & 15) == 0) {
            ((float4*)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
            ((float4*)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
        } else {
            for (int i = 0; i < 8; ++i)
                if (c + i < d) ((float*)p)[i] = x[i];
        }
        return;
    }
    uint4 v;
    uint16_t* h = (uint16_t*)&v;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        h[i] = type == EE_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(x[i])) : __half_as_ushort(__float2half_rn(x[i]));
    if (c + 8 <= d && ((uintptr_t)p & 15) == 0) *(uint4*)p = v;
    else
        for (int i = 0; i < 8; ++i)
            if (c + i < d) ((uint16_t*)p)[i] = h[i];
}

__device__ __forceinline__ const char* row_of(const Rows& t, int64_t r) {
    return (const char*)t.p + r * t.ld * bytes_of(t.type);
}

// Sum over the CTA; `sh` holds two sets of warp sums used in turn, so that one
// barrier per call is enough.
__device__ __forceinline__ float cta_sum(float v, float (&sh)[2][kNormThreads / 32], int turn) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    if ((threadIdx.x & 31) == 0) sh[turn & 1][threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < (int)(blockDim.x >> 5); ++i) v += sh[turn & 1][i];
    return v;
}

// CPT: chunks of 8 columns per thread, chunk i of a thread being
// threadIdx.x + i blockDim.x.
template <int CPT>
__global__ void __launch_bounds__(kNormThreads)
    k_rms_norm(Rows x, Rows gain, Rows y, float* __restrict__ rstd, int64_t rows, int d, float eps) {
    __shared__ float sh[2][kNormThreads / 32];
    float g[CPT][8], nx[CPT][8];
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        load8(gain.p, gain.type, threadIdx.x + i * blockDim.x, d, g[i]);
        load8(row_of(x, blockIdx.x), x.type, threadIdx.x + i * blockDim.x, d, nx[i]);
    }
    int turn = 0;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x, ++turn) {
        float v[CPT][8], ss = 0.f;
#pragma unroll
        for (int i = 0; i < CPT; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] = nx[i][e];
                ss = fmaf(v[i][e], v[i][e], ss);
            }
        if (r + gridDim.x < rows)
#pragma unroll
            for (int i = 0; i < CPT; ++i)
                load8(row_of(x, r + gridDim.x), x.type, threadIdx.x + i * blockDim.x, d, nx[i]);
        const float s = 1.f / sqrtf(cta_sum(ss, sh, turn) / (float)d + eps);
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= s * g[i][e];
            store8((void*)row_of(y, r), y.type, threadIdx.x + i * blockDim.x, d, v[i]);
        }
        if (rstd && threadIdx.x == 0) rstd[r] = s;
    }
}

template <int CPT>
__global__ void __launch_bounds__(kNormThreads)
    k_rms_norm_backward(Rows dy, Rows x, Rows gain, const float* __restrict__ rstd, Rows dx, float* __restrict__ part,
                        int64_t rows, int d) {
    __shared__ float sh[2][kNormThreads / 32];
    float g[CPT][8], dg[CPT][8], nx[CPT][8], ny[CPT][8];
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        const int j = threadIdx.x + i * blockDim.x;
        load8(gain.p, gain.type, j, d, g[i]);
        load8(row_of(x, blockIdx.x), x.type, j, d, nx[i]);
        load8(row_of(dy, blockIdx.x), dy.type, j, d, ny[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) dg[i][e] = 0.f;
    }
    float ns = rstd[blockIdx.x];
    int turn = 0;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x, ++turn) {
        const float s = ns;
        float xh[CPT][8], gy[CPT][8], dot = 0.f;
#pragma unroll
        for (int i = 0; i < CPT; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xh[i][e] = nx[i][e] * s;
                dg[i][e] = fmaf(ny[i][e], xh[i][e], dg[i][e]);
                gy[i][e] = ny[i][e] * g[i][e];
                dot = fmaf(gy[i][e], xh[i][e], dot);
            }
        if (r + gridDim.x < rows) {
            ns = rstd[r + gridDim.x];
#pragma unroll
            for (int i = 0; i < CPT; ++i) {
                load8(row_of(x, r + gridDim.x), x.type, threadIdx.x + i * blockDim.x, d, nx[i]);
                load8(row_of(dy, r + gridDim.x), dy.type, threadIdx.x + i * blockDim.x, d, ny[i]);
            }
        }
        if (!dx.p) continue;
        const float m = cta_sum(dot, sh, turn) / (float)d;
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) gy[i][e] = s * (gy[i][e] - xh[i][e] * m);
            store8((void*)row_of(dx, r), dx.type, threadIdx.x + i * blockDim.x, d, gy[i]);
        }
    }
    if (part)
#pragma unroll
        for (int i = 0; i < CPT; ++i)
            store8(part + (int64_t)blockIdx.x * d, EE_FP32, threadIdx.x + i * blockDim.x, d, dg[i]);
}

// dg = sum of the CTAs' shares, in their order: 32 columns per CTA, 32 groups of
// shares.
__global__ void __launch_bounds__(1024) k_sum_parts(const float* __restrict__ part, int n, int d, float* __restrict__ out) {
    __shared__ float sh[32][33];
    const int c = blockIdx.x * 32 + threadIdx.x;
    float v = 0.f;
    if (c < d)
        for (int i = threadIdx.y; i < n; i += 32) v += part[(int64_t)i * d + c];
    sh[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y == 0 && c < d) {
        v = 0.f;
        for (int i = 0; i < 32; ++i) v += sh[i][threadIdx.x];
        out[c] = v;
    }
}

int fail(int code, const char* msg) { return set_last_error(code, msg); }
int cuda_status(cudaError_t e) { return e == cudaSuccess ? EE_OK : fail(EE_ECUDA, cudaGetErrorString(e)); }
bool type_ok(int t) { return t == EE_BF16 || t == EE_FP16 || t == EE_FP32; }
size_t elem(int t) { return t == EE_FP32 ? 4 : 2; }

int check_rows(const void* p, int type, int64_t rows, int d, int64_t ld) {
    if (!type_ok(type)) return fail(EE_EINVAL, "unknown element type");
    if (rows < 0 || d < 1 || d > EE_MAX_NORM) return fail(EE_EINVAL, "bad number of rows or width");
    if (ld < d) return fail(EE_EINVAL, "rows overlap: the row stride is below the width");
    if (rows && !p) return fail(EE_EINVAL, "NULL argument");
    if ((uintptr_t)p % elem(type)) return fail(EE_EINVAL, "a tensor is not aligned to its type");
    return EE_OK;
}

// Threads and chunks per thread: one chunk up to 256 threads (2048 columns).
struct Plan {
    int threads, cpt, grid;
};
int plan(int64_t rows, int d, Plan* p) {
    const int chunks = (d + 7) / 8;
    p->cpt = chunks <= 256 ? 1 : chunks <= 512 ? 2 : 4;
    p->threads = ((chunks + p->cpt - 1) / p->cpt + 31) / 32 * 32;
    int dev = 0, n_sm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev);
    p->grid = (int)std::min<int64_t>(rows, (int64_t)n_sm * std::max(1, 1024 / p->threads));
    return cuda_status(e);
}

}  // namespace
}  // namespace ee

using namespace ee;

extern "C" {

int ee_rms_norm(const void* x, int x_type, int64_t rows, int d, int64_t ld_x, const void* gain, int gain_type, float eps,
                void* y, int y_type, int64_t ld_y, float* rstd, void* stream) {
    int rc = check_rows(x, x_type, rows, d, ld_x);
    if (rc == EE_OK) rc = check_rows(y, y_type, rows, d, ld_y);
    if (rc == EE_OK) rc = check_rows(gain, gain_type, 1, d, d);
    if (rc != EE_OK) return rc;
    if (!(eps >= 0.f)) return fail(EE_EINVAL, "eps must not be negative");
    if (!rows) return EE_OK;
    Plan p;
    if ((rc = plan(rows, d, &p)) != EE_OK) return rc;
    const Rows X{x, ld_x, x_type}, G{gain, 0, gain_type}, Y{y, ld_y, y_type};
    cudaStream_t s = (cudaStream_t)stream;
    if (p.cpt == 1) k_rms_norm<1><<<p.grid, p.threads, 0, s>>>(X, G, Y, rstd, rows, d, eps);
    else if (p.cpt == 2) k_rms_norm<2><<<p.grid, p.threads, 0, s>>>(X, G, Y, rstd, rows, d, eps);
    else k_rms_norm<4><<<p.grid, p.threads, 0, s>>>(X, G, Y, rstd, rows, d, eps);
    return cuda_status(cudaGetLastError());
}

int ee_rms_norm_scratch_bytes(int64_t rows, int d, size_t* bytes) {
    if (!bytes || rows < 0 || d < 1 || d > EE_MAX_NORM) return fail(EE_EINVAL, "bad argument");
    Plan p;
    const int rc = plan(rows, d, &p);
    if (rc != EE_OK) return rc;
    *bytes = 4 * (size_t)p.grid * d;
    return EE_OK;
}

int ee_rms_norm_backward(const void* dy, int dy_type, int64_t ld_dy, const void* x, int x_type, int64_t rows, int d,
                         int64_t ld_x, const void* gain, int gain_type, const float* rstd, void* dx, int64_t ld_dx,
                         float* dgain, void* scratch, size_t scratch_bytes, void* stream) {
    int rc = check_rows(x, x_type, rows, d, ld_x);
    if (rc == EE_OK) rc = check_rows(dy, dy_type, rows, d, ld_dy);
    if (rc == EE_OK && dx) rc = check_rows(dx, x_type, rows, d, ld_dx);
    if (rc == EE_OK) rc = check_rows(gain, gain_type, 1, d, d);
    if (rc != EE_OK) return rc;
    if (!dx && !dgain) return fail(EE_EINVAL, "neither gradient is asked for");
    cudaStream_t s = (cudaStream_t)stream;
    if (!rows) return dgain ? cuda_status(cudaMemsetAsync(dgain, 0, 4 * (size_t)d, s)) : EE_OK;
    if (!rstd) return fail(EE_EINVAL, "NULL argument");
    Plan p;
    if ((rc = plan(rows, d, &p)) != EE_OK) return rc;
    if (dgain && (!scratch || scratch_bytes < 4 * (size_t)p.grid * d)) return fail(EE_ENOMEM, "scratch too small");
    if ((uintptr_t)scratch % 16) return fail(EE_EINVAL, "scratch must be 16-byte aligned");
    const Rows Y{dy, ld_dy, dy_type}, X{x, ld_x, x_type}, G{gain, 0, gain_type}, D{dx, ld_dx, x_type};
    float* part = dgain ? (float*)scratch : nullptr;
    if (p.cpt == 1) k_rms_norm_backward<1><<<p.grid, p.threads, 0, s>>>(Y, X, G, rstd, D, part, rows, d);
    else if (p.cpt == 2) k_rms_norm_backward<2><<<p.grid, p.threads, 0, s>>>(Y, X, G, rstd, D, part, rows, d);
    else k_rms_norm_backward<4><<<p.grid, p.threads, 0, s>>>(Y, X, G, rstd, D, part, rows, d);
    if (dgain) k_sum_parts<<<(d + 31) / 32, dim3(32, 32), 0, s>>>(part, p.grid, d, dgain);
    return cuda_status(cudaGetLastError());
}

}  // extern "C"
