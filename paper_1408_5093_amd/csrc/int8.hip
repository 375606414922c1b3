// int8.hip -- rows held as 8-bit integers with a scale each, and the inner
// product of such rows: top[n][k] = (sum_c q[n][c] p[k][c]) s[n] t[k] + bias[k].
//
// The sum runs on the 8-bit matrix instructions and is exact in 32 bits
// (C <= 2^17, |q p| <= 127^2); only its scaling is rounded, in float.
#include <algorithm>
#include <type_traits>

#include "tile_gemm.h"

namespace caffe_hip {

namespace {

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

// The whole number next to x / s, halves to the even one, exactly.  x * inv,
// inv = fl(1 / s), is within 127 * 2^-23 < 2^-16 of the quotient, so its
// rounding is the quotient's unless it lies within 2^-15 of a half.  There the
// rounded quotient t = fl(x / s) decides: it is on the same side of the half as
// x / s, or on the half itself, and then the remainder x - t s says on which
// side the quotient was.  The remainder is a multiple of half a unit of s and
// at most 2^8 of them, exact in one fma where that half is a float: x and s
// below 2^-100 are taken 2^64 times.
__device__ __forceinline__ int round_quotient(float x, float s, float inv)
{
    const float near = x * inv;
    float r = rintf(near);
    if (!(fabsf(fabsf(near - r) - 0.5f) > 0x1p-15f)) {  // (also where inv overflows)
        const float up = s < 0x1p-100f ? 0x1p64f : 1.f;  // exact: |x| < 2^8 s
        const float xs = x * up, ss = s * up, t = xs / ss;
        r = rintf(t);
        const float d = t - r;  // exact
        if (fabsf(d) == 0.5f) {
            const float rem = fmaf(-t, ss, xs);
            // toward the side of the quotient (s > 0); the even one at rem = 0
            if (rem > 0.f && d > 0.f)
                r += 1.f;
            else if (rem < 0.f && d < 0.f)
                r -= 1.f;
        }
    }
    return (int)fminf(fmaxf(r, -127.f), 127.f);
}

// A row's scale from its largest absolute value's bits: NaN if that is not a
// number or infinite.
__device__ __forceinline__ float row_scale(uint32_t top)
{
    return top >= 0x7F800000u ? NAN : __builtin_bit_cast(float, top) / 127.f;
}

// four values as 8-bit numbers (zeros unless the scale is positive)
__device__ __forceinline__ uint32_t round_row4(const float (&x)[4], float s)
{
    uint32_t w = 0;
    if (s > 0.f) {
        const float inv = 1.f / s;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w |= (uint32_t)(uint8_t)round_quotient(x[e], s, inv) << (8 * e);
    }
    return w;
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
__global__ void __launch_bounds__(LANES > 256 ? LANES : 256)
quantize_rows_kernel(const T* __restrict__ x, int64_t rows, int cols, int pitch,
                     int8_t* __restrict__ q, float* __restrict__ scale)
{
    constexpr int RPB = LANES > 256 ? 1 : 256 / LANES;
    __shared__ uint32_t part[LANES > 64 ? LANES / 64 : 1];
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
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w)
            top = max(top, part[w]);
    }
    if (!live)
        return;
    const float s = row_scale(top);
    if (lane == 0)
        scale[row] = s;
    int8_t* o = q + row * (int64_t)pitch;
    auto put = [&](int c, const float(&y)[4]) { *(uint32_t*)(o + c) = round_row4(y, s); };
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
    // few long rows: a thousand threads to each (20 x 9216: 6.5 us with 256)
    if (rows <= 512 && cols > 1024)
        hipLaunchKernelGGL(HIP_KERNEL_NAME(quantize_rows_kernel<T, VEC, 1024, 4>),
                           dim3((unsigned)rows), dim3(1024), 0, s, x, rows, cols, pitch, q, scale);
    else if (cols <= 1024)
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

// 32 x 32 by four waves that share the reduction, 64 x 64 and 128 x 128 by 2 x 2
// waves, 256 x 256 by eight
typedef TileShared<OpInt8Line, 4, false> Ip8Tile32;
typedef TileNT<OpInt8Line, 2, 2, 1, 1, 5, false> Ip8Tile64;
typedef TileNT<OpInt8Line, 2, 2, 2, 2, 2, false> Ip8Tile128;
typedef TileNT<OpInt8Half, 4, 2, 2, 4, 2, false> Ip8Tile256;

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
    const bool vec = p.K % 4 == 0;
    Tile::each(acc, [&](int di, int dj, int(&v)[4]) {
        const int i = m0 + di, j = n0 + dj, jc = min(j, p.K - 1);
        const float t = p.ws[jc], bias = p.bias ? p.bias[jc] : 0.f;
        float z[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            z[e] = ip8_finish(v[e], p.xs[min(i + e, p.N - 1)], t, bias, p.relu);
        if (vec) {  // four outputs of a sample to a lane
            quad_transpose(z);
            const int n = i + (threadIdx.x & 3), k = j - (threadIdx.x & 3);
            if (n >= p.N || k >= p.K)
                return;
            const size_t at = (size_t)n * p.K + k;
            if (p.out_bf16)
                *(u32x2*)(p.out_bf16 + at) = u32x2{f32x2_to_bf16x2_rne(z[0], z[1]),
                                                   f32x2_to_bf16x2_rne(z[2], z[3])};
            else
                *(floatx4*)(p.out_f32 + at) = floatx4{z[0], z[1], z[2], z[3]};
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (i + e >= p.N || j >= p.K)
                continue;
            const size_t at = (size_t)(i + e) * p.K + j;
            if (p.out_bf16)
                p.out_bf16[at] = f32_to_bf16_rne(z[e]);
            else
                p.out_f32[at] = z[e];
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

// One float sample: the stream of the weights.  A workgroup takes 16 outputs, its
// eight waves a share of the reduction each, 64 bytes of every weight row to a
// step of the 16x16x64 instruction straight from memory (lane l: row l % 16,
// bytes 16 (l / 16) ..), and the shares are added in LDS.  The workgroup brings
// the sample to 8 bits itself while its first weights are on their way: 4096 x
// 9216 takes 11.4 us, a launch for the rounding and a tiled product 4.3 + 9.3.
constexpr int kOneWaves = 8, kOneThreads = 64 * kOneWaves;
constexpr int kOneRow = 16384;  // values of the sample, at most

template <typename T, int VEC>
__global__ void __launch_bounds__(kOneThreads)
ip8_one_kernel(const Ip8Params p, const T* __restrict__ x, int C)
{
    constexpr int U = 8;  // steps in flight
    __shared__ u32x4 xq[kOneRow / 16];
    __shared__ uint32_t top[kOneWaves];
    __shared__ int sum[kOneWaves][16];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int k0 = blockIdx.x * 16;
    const int steps = (int)(p.pitch / 64);
    const int t0 = steps * wave / kOneWaves, t1 = steps * (wave + 1) / kOneWaves;
    // rows past the last re-read it: their results are not stored
    const int8_t* w = p.w + (size_t)min(k0 + r, p.K - 1) * p.pitch + g * 16;
    intx4 acc = {0, 0, 0, 0}, wv[U];
    auto load = [&](int t) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            wv[u] = *(const intx4*)(w + min(t + u, steps - 1) * 64);
    };
    load(t0);
    constexpr int CH = kOneRow / (kOneThreads * 4);
    float y[CH][4];
    uint32_t m = 0;
#pragma unroll
    for (int h = 0; h < CH; ++h) {
        const int c = (h * kOneThreads + (int)threadIdx.x) * 4;
        load4<T, VEC>(x + c, C - c, y[h]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            m = max(m, __builtin_bit_cast(uint32_t, y[h][e]) & 0x7FFFFFFFu);
    }
    for (int off = 32; off > 0; off >>= 1)
        m = max(m, (uint32_t)__shfl_xor((int)m, off, 64));
    if (lane == 0)
        top[wave] = m;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kOneWaves; ++v)
        m = max(m, top[v]);
    const float xscale = row_scale(m);
#pragma unroll
    for (int h = 0; h < CH; ++h) {
        const int c = (h * kOneThreads + (int)threadIdx.x) * 4;
        if (c < (int)p.pitch)
            ((uint32_t*)xq)[c / 4] = round_row4(y[h], xscale);
    }
    __syncthreads();
    for (int t = t0; t < t1; t += U) {
        if (t > t0)
            load(t);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t + u >= t1)
                break;
            intx4 xv = {0, 0, 0, 0};
            if (r == 0)
                xv = __builtin_bit_cast(intx4, xq[(t + u) * 4 + g]);
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(xv, wv[u], acc, 0, 0, 0);
        }
    }
    if (g == 0)  // lane l < 16 holds the sample and output l
        sum[wave][r] = acc[0];
    __syncthreads();
    const int k = k0 + (int)threadIdx.x;
    if (threadIdx.x < 16 && k < p.K) {
        int s = 0;
#pragma unroll
        for (int v = 0; v < kOneWaves; ++v)
            s += sum[v][threadIdx.x];
        const float z = ip8_finish(s, xscale, p.ws[k], p.bias ? p.bias[k] : 0.f, p.relu);
        if (p.out_bf16)
            p.out_bf16[k] = f32_to_bf16_rne(z);
        else
            p.out_f32[k] = z;
    }
}

template <typename T>
hipError_t launch_ip8_one(const Ip8Params& p, const void* x, int C, hipStream_t s)
{
    const dim3 grid((unsigned)((p.K + 15) / 16)), threads(kOneThreads);
    if (C % 4 == 0)
        hipLaunchKernelGGL(HIP_KERNEL_NAME(ip8_one_kernel<T, 4>), grid, threads, 0, s, p,
                           (const T*)x, C);
    else
        hipLaunchKernelGGL(HIP_KERNEL_NAME(ip8_one_kernel<T, 1>), grid, threads, 0, s, p,
                           (const T*)x, C);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const void* x, int bf16, int64_t rows, int cols, int pitch,
                                int8_t* q, float* scale, hipStream_t s)
{
    // a launch holds fewer than 2^32 threads: 2^21 rows at a time
    constexpr int64_t kRows = 1 << 21;
    for (int64_t r = 0; r < rows; r += kRows) {
        const int64_t n = std::min(kRows, rows - r);
        int8_t* to = q + r * pitch;
        if (bf16) {
            const uint16_t* p = (const uint16_t*)x + r * cols;
            if (cols % 4 == 0)
                quantize_rows<uint16_t, 4>(p, n, cols, pitch, to, scale + r, s);
            else
                quantize_rows<uint16_t, 1>(p, n, cols, pitch, to, scale + r, s);
        } else {
            const float* p = (const float*)x + r * cols;
            if (cols % 4 == 0)
                quantize_rows<float, 4>(p, n, cols, pitch, to, scale + r, s);
            else
                quantize_rows<float, 1>(p, n, cols, pitch, to, scale + r, s);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
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
    if (a.bottom_type != kIp8BottomInt8 && a.N == 1 && a.pitch <= kOneRow)
        return a.bottom_type == kIp8BottomBf16 ? launch_ip8_one<uint16_t>(p, a.bottom, a.C, s)
                                               : launch_ip8_one<float>(p, a.bottom, a.C, s);
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
    // The tile by the model of its time.  Samples in 8 bits, bf16 top, measured /
    // modelled, us:
    //        20 x 9216 x 4096  64 x 4096 x 4096  1024 x 4096 x 4096  4096 x 4096 x 4096  8192 x 9216 x 4096
    //   32       9.6 / 11         6.8 / 7.1
    //   64        15 / 19         8.1 / 11            30 / 34            108 / 123           466 / 535
    //   128       45 / 62          18 / 34            29 / 34             78 / 89            298 / 358
    //   256       83 / 160         44 / 84            51 / 84             67 / 84            259 / 297
    auto tiles = [&](int64_t side) { return (a.N + side - 1) / side * ((a.K + side - 1) / side); };
    const int64_t lines = a.pitch / 128;
    const double t32 = TileTime{3.9, 0.10, 0.18}.of(tiles(32), lines);
    const double t64 = TileTime{5.0, 0.19, 0.23}.of(tiles(64), lines);
    const double t128 = TileTime{12.0, 0.70, 0.60}.of(tiles(128), lines);
    const double t256 = TileTime{23.0, 1.90, 1.90}.of(tiles(256), lines);
    const double least = std::min(std::min(t32, t64), std::min(t128, t256));
    if (t256 <= least)
        return launch_ip8_tile<Ip8Tile256>(p, s);
    if (t128 <= least)
        return launch_ip8_tile<Ip8Tile128>(p, s);
    if (t32 < t64)
        return launch_ip8_tile<Ip8Tile32>(p, s);
    return launch_ip8_tile<Ip8Tile64>(p, s);
}

}  // namespace caffe_hip
