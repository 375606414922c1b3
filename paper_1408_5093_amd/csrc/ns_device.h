// ns_device.h -- what the two paths of the Newton-Schulz iteration share
// (muon.hip: tiled products; muon_small.hip: matrices with a side of at most
// 128): the two-term elements, the input with its momentum, the norm.
#pragma once

#include <math.h>

#include "tile_gemm.h"

namespace caffe_hip {

typedef _Float16 halfx4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------ pair matrices
// Element (row, k): line k / 32 of the row, its high half at byte 2 (k % 32),
// its low half 64 bytes on.  k a multiple of 4.
__device__ __forceinline__ size_t pair_off(size_t pitch, int row, int k)
{
    return (size_t)row * pitch + (size_t)(k >> 5) * 128 + (k & 31) * 2;
}

__device__ __forceinline__ void store_pair4(char* M, size_t off, const float (&v)[4])
{
    halfx4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        h[e] = (_Float16)v[e];
        l[e] = (_Float16)(v[e] - (float)h[e]);
    }
    *(halfx4*)(M + off) = h;
    *(halfx4*)(M + off + 64) = l;
}

__device__ __forceinline__ void load_pair4(const char* M, size_t off, float (&v)[4])
{
    const halfx4 h = *(const halfx4*)(M + off), l = *(const halfx4*)(M + off + 64);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] = (float)h[e] + (float)l[e];
}

// u (the matrix to orthogonalise) is g, or with momentum
// v <- mu v + g (written) and u = nesterov ? g + mu v : v.
struct NsInput {
    const void* g;
    float* v;       // null: u = g
    float mu;
    int nesterov;
    int bf16;       // g is bfloat16 (v null)
    int64_t count;  // elements of one matrix
};

template <int VEC>
__device__ __forceinline__ void load_vec(const NsInput& in, int64_t at, float (&g)[VEC])
{
    if (in.bf16) {
        const uint16_t* p = (const uint16_t*)in.g + at;
        if constexpr (VEC == 4) {
            const u16x4 x = *(const u16x4*)p;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                g[e] = bf16_to_f32(x[e]);
        } else {
            g[0] = bf16_to_f32(*p);
        }
    } else {
        const float* p = (const float*)in.g + at;
        if constexpr (VEC == 4) {
            const floatx4 x = *(const floatx4*)p;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                g[e] = x[e];
        } else {
            g[0] = *p;
        }
    }
}

template <int VEC>
__device__ __forceinline__ void load_u(const NsInput& in, int64_t at, bool update, float (&u)[VEC])
{
    load_vec<VEC>(in, at, u);
    if (in.v) {
        float* p = in.v + at;
        float v[VEC];
        if constexpr (VEC == 4) {
            const floatx4 x = *(const floatx4*)p;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = x[e];
        } else {
            v[0] = *p;
        }
        if (update) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                v[e] = in.mu * v[e] + u[e];
            if constexpr (VEC == 4)
                *(floatx4*)p = floatx4{v[0], v[1], v[2], v[3]};
            else
                *p = v[0];
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            u[e] = in.nesterov ? u[e] + in.mu * v[e] : v[e];
    }
}

// The sum over a workgroup of WAVES waves, in a fixed order, on every thread.
template <int WAVES>
__device__ __forceinline__ double block_sum(double s)
{
    __shared__ double part[WAVES];
    for (int off = 32; off > 0; off >>= 1)
        s += __shfl_xor(s, off, 64);
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = part[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w)
        s += part[w];
    return s;
}

// 1 / (||u|| + eps) from ||u||^2: 0 for a zero matrix, NaN where an element is
// NaN or infinite.
__device__ __forceinline__ double inv_from(double sum, double eps)
{
    return sum == 0.0 ? 0.0 : (sum < INFINITY ? 1.0 / (sqrt(sum) + eps) : NAN);
}

// ... from its parts, added in a fixed order
template <int WAVES>
__device__ __forceinline__ double inv_norm(const double* part, int parts, double eps)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 64 * WAVES)
        s += part[i];
    return inv_from(block_sum<WAVES>(s), eps);
}

// ------------------------------------------- matrices with a side <= 128
struct NsSmall {
    NsInput in;
    const double* norm;
    int norm_parts;
    double eps;
    int m, n, tall, chunks, n_pad, parts;
    float* part;  // [batch][parts][LD][LD]
    char* p_img;  // [batch] P's LDS image
    float* xs;    // [batch][n_pad][LD]: X between two segments, transposed
};
struct NsSteps {  // exponents of the operands' scales by step, of X by segment
    float a, b, c;
    int segments;
    int8_t length[kNsMaxSteps], er[kNsMaxSteps], eq[kNsMaxSteps], et[kNsMaxSteps],
        ep[kNsMaxSteps], ex[kNsMaxSteps];
};
struct NsOut {
    float* out_f32;
    uint16_t* out_bf16;
    float* w;
    const float* lr_dev;
    float lr, decay, step_scale;
};
void ns_small_sizes(int m, int n, NsPlan* q);
hipError_t launch_ns_small(const NsPlan& q, const NsInput& in, const NsArgs& x, char* ws,
                           hipStream_t s);

}  // namespace caffe_hip
