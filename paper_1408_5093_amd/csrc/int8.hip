// int8.hip -- rows held as 8-bit integers with a scale each, and the inner
// product of such rows: top[n][k] = (sum_c q[n][c] p[k][c]) s[n] t[k] + bias[k].
//
// The sum runs on the 8-bit matrix instructions and is exact in 32 bits
// (C <= 2^17 and |q p| <= 2^14); only its scaling is rounded, in float.
#include <algorithm>
#include <type_traits>

#include "tile_gemm.h"

namespace caffe_hip {

namespace {

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

// The whole number next to x / s, halves to the even one, exactly: the
// rounded quotient t = fl(x / s) lies on the same side of every half as x / s
// or on the half itself, and then the remainder x - t s (exact in one fma)
// says on which side the quotient was.
__device__ __forceinline__ int round_quotient(float x, float s)
{
    const float t = x / s;
    float r = rintf(t);
    const float d = t - r;  // exact
    if (fabsf(d) == 0.5f) {
        const float rem = fmaf(-t, s, x);
        // toward the side of the quotient (s > 0); the even one at rem = 0
        if (rem > 0.f && d > 0.f)
            r += 1.f;
        else if (rem < 0.f && d < 0.f)
            r -= 1.f;
    }
    return (int)fminf(fmaxf(r, -127.f), 127.f);
}

template <typename T, int VEC>
__device__ __forceinline__ void load4(const T* p, int left, float (&x)[4])
{
    if constexpr (VEC == 4) {
        if (left <= 0) {
            x[0] = x[1] = x[2] = x[3] = 0.f;
        } else if constexpr (std::is_same<T, float>::value) {
            const floatx4 v = *(const floatx4*)p;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = v[e];
        } else {
            const u16x4 v = *(const u16x4*)p;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = bf16_to_f32(v[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (e >= left)
                x[e] = 0.f;
            else if constexpr (std::is_same<T, float>::value)
                x[e] = p[e];
            else
                x[e] = bf16_to_f32(p[e]);
        }
    }
}

// scale = max|x| / 127 (float), q = the whole numbers next to x / scale, the
// row padded with zeros to the pitch.  A zero row, or one whose scale
// vanishes, has scale 0 and zeros; one with a NaN or an infinity has scale
// NaN and zeros (the absolute values' bits order them above every number).
// LANES threads take a row, each CH chunks of four kept in registers; longer
// rows are read again.  Bound by HBM.
template <typename T, int VEC, int LANES, int CH>
__global__ void __launch_bounds__(256)
quantize_rows_kernel(const T* __restrict__ x, int64_t rows, int cols, int pitch,
                     int8_t* __restrict__ q, float* __restrict__ scale)
{
    constexpr int RPB = 256 / LANES;
    __shared__ uint32_t part[4];
    const int lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / LANES;
    const bool live = row < rows;
    const T* p = x + row * cols;
    float v[CH][4];
    uint32_t top = 0;
    auto look = [&](const float(&y)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            top = max(top, __builtin_bit_cast(uint32_t, y[e]) & 0x7FFFFFFFu);
    };
#pragma unroll
    for (int h = 0; h < CH; ++h) {
        const int c = (h * LANES + lane) * 4;
        load4<T, VEC>(p + c, live ? cols - c : 0, v[h]);
        look(v[h]);
    }
    for (int c = (CH * LANES + lane) * 4; live && c < cols; c += LANES * 4) {
        float y[4];
        load4<T, VEC>(p + c, cols - c, y);
        look(y);
    }
    for (int off = 32; off > 0; off >>= 1)
        top = max(top, (uint32_t)__shfl_xor((int)top, off, 64));
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0)
            part[threadIdx.x >> 6] = top;
        __syncthreads();
        top = max(max(part[0], part[1]), max(part[2], part[3]));
    }
    if (!live)
        return;
    const bool bad = top >= 0x7F800000u;
    const float s = bad ? NAN : __builtin_bit_cast(float, top) / 127.f;
    const bool some = s > 0.f;
    if (lane == 0)
        scale[row] = s;
    int8_t* o = q + row * (int64_t)pitch;
    auto put = [&](int c, const float(&y)[4]) {
        uint32_t w = 0;
        if (some) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w |= (uint32_t)(uint8_t)round_quotient(y[e], s) << (8 * e);
        }
        *(uint32_t*)(o + c) = w;
    };
#pragma unroll
    for (int h = 0; h < CH; ++h) {
        const int c = (h * LANES + lane) * 4;
        if (c < pitch)
            put(c, v[h]);
    }
    for (int c = (CH * LANES + lane) * 4; c < pitch; c += LANES * 4) {
        float y[4];
        load4<T, VEC>(p + c, cols - c, y);
        put(c, y);
    }
}

template <typename T, int VEC>
void quantize_rows(const T* x, int64_t rows, int cols, int pitch, int8_t* q, float* scale,
                   hipStream_t s)
{
    if (cols <= 1024)
        hipLaunchKernelGGL(HIP_KERNEL_NAME(quantize_rows_kernel<T, VEC, 64, 4>),
                           dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, x, rows, cols, pitch,
                           q, scale);
    else if (cols <= 4096)
        hipLaunchKernelGGL(HIP_KERNEL_NAME(quantize_rows_kernel<T, VEC, 256, 4>),
                           dim3((unsigned)rows), dim3(256), 0, s, x, rows, cols, pitch, q, scale);
    else
        hipLaunchKernelGGL(HIP_KERNEL_NAME(quantize_rows_kernel<T, VEC, 256, 16>),
                           dim3((unsigned)rows), dim3(256), 0, s, x, rows, cols, pitch, q, scale);
}

// ------------------------------------------------------------------ products
struct Ip8Params {
    const int8_t *x, *w;
    const float *xs, *ws, *bias;
    float* out_f32;
    uint16_t* out_bf16;
    int N, K, relu;
    uint32_t pitch;  // bytes of a row of x or w, a multiple of 128
};

__device__ __forceinline__ float ip8_finish(int acc, float s, float t, float bias, int relu)
{
    const float z = (float)acc * s * t + bias;
    return z > 0.f ? z : (relu ? 0.f : z);
}

typedef TileNT<OpInt8, 2, 2, 1, 1, 3, false> Ip8Tile64;

template <class Tile>
__global__ void __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd)
ip8_tile_kernel(const Ip8Params p)
{
    const int mt = (p.N + Tile::TM - 1) / Tile::TM;
    const int nt = (p.K + Tile::TN - 1) / Tile::TN;
    // consecutive tiles on one XCD, in bands of four tile rows
    const int chunk = gridDim.x >> 3;
    const int t = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
    if (t >= mt * nt)
        return;
    const int band = t / (4 * nt), h = min(4, mt - 4 * band), r = t - band * 4 * nt;
    const int m0 = (4 * band + r % h) * Tile::TM, n0 = r / h * Tile::TN;
    typename Tile::acc_t acc[Tile::kMI][Tile::kNI];
    Tile::run(p.x + (size_t)m0 * p.pitch, (uint32_t)min(Tile::TM, p.N - m0) * p.pitch, p.pitch,
              p.w + (size_t)n0 * p.pitch, (uint32_t)min(Tile::TN, p.K - n0) * p.pitch, p.pitch, 0,
              (int)(p.pitch / 128), acc);
    Tile::each(acc, [&](int di, int dj, int(&v)[4]) {
        const int i = m0 + di, j = n0 + dj;
        if (j >= p.K)
            return;
        const float t = p.ws[j], bias = p.bias ? p.bias[j] : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (i + e >= p.N)
                continue;
            const float z = ip8_finish(v[e], p.xs[i + e], t, bias, p.relu);
            const size_t at = (size_t)(i + e) * p.K + j;
            if (p.out_bf16)
                p.out_bf16[at] = f32_to_bf16_rne(z);
            else
                p.out_f32[at] = z;
        }
    });
}

template <class Tile>
hipError_t launch_ip8_tile(const Ip8Params& p, hipStream_t s)
{
    const int64_t tiles = (int64_t)((p.N + Tile::TM - 1) / Tile::TM) *
                          ((p.K + Tile::TN - 1) / Tile::TN);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ip8_tile_kernel<Tile>),
                       dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(Tile::kThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const void* x, int bf16, int64_t rows, int cols, int pitch,
                                int8_t* q, float* scale, hipStream_t s)
{
    if (rows == 0)
        return hipSuccess;
    if (bf16) {
        if (cols % 4 == 0)
            quantize_rows<uint16_t, 4>((const uint16_t*)x, rows, cols, pitch, q, scale, s);
        else
            quantize_rows<uint16_t, 1>((const uint16_t*)x, rows, cols, pitch, q, scale, s);
    } else {
        if (cols % 4 == 0)
            quantize_rows<float, 4>((const float*)x, rows, cols, pitch, q, scale, s);
        else
            quantize_rows<float, 1>((const float*)x, rows, cols, pitch, q, scale, s);
    }
    return hipGetLastError();
}

hipError_t launch_inner_product_int8(const Ip8Args& a, char* ws, hipStream_t s)
{
    if (a.N == 0)
        return hipSuccess;
    Ip8Params p{};
    p.w = a.weight;
    p.ws = a.weight_scale;
    p.bias = a.bias;
    p.out_f32 = a.top_bf16 ? nullptr : (float*)a.top;
    p.out_bf16 = a.top_bf16 ? (uint16_t*)a.top : nullptr;
    p.N = a.N;
    p.K = a.K;
    p.relu = a.relu;
    p.pitch = (uint32_t)a.pitch;
    if (a.bottom_type == kIp8BottomInt8) {
        p.x = (const int8_t*)a.bottom;
        p.xs = a.bottom_scale;
    } else {
        int8_t* q = (int8_t*)ws;
        float* qs = (float*)(ws + (size_t)a.N * a.pitch);
        const hipError_t e = launch_quantize_rows(a.bottom, a.bottom_type == kIp8BottomBf16, a.N,
                                                  a.C, a.pitch, q, qs, s);
        if (e != hipSuccess)
            return e;
        p.x = q;
        p.xs = qs;
    }
    return launch_ip8_tile<Ip8Tile64>(p, s);
}

}  // namespace caffe_hip
