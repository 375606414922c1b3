// muon.hip -- the Newton-Schulz orthogonalisation of weight matrices and the
// parameter update that steps along its result.
//
// Mathematics.  For G (m x n, m <= n; a taller matrix is taken transposed)
//   X_0 = G / (||G||_F + eps),   X <- (a I + b A + c A^2) X,  A = X X^T
// keeps the singular vectors of G and maps each singular value s by
// s q(s^2), q(t) = a + b t + c t^2.  Every factor on the left is a polynomial
// of the same m x m matrix, so a segment of L steps needs the wide matrix
// only at its ends: with R = X X^T,
//   Q = a I + b R + c R R,  T = Q R,  R <- T Q,  P <- Q P     (L times)
// and then X <- P X.  All of these are symmetric and commute, so one half of
// each is computed and mirrored.  Per segment 3 m^2 n + (4 L - 3) m^3
// operations against L (3 m^2 n + m^3) for the steps one by one.
//
// Segments are short because the Gram matrix holds the squares of the
// singular values: a rounding error of R grows by q(0)^2 per step in the
// directions whose values are still small.  The first segment, where the
// trace of R is 1, ends before max|q|^(2 (L - 1)) passes 2^8 (three steps of
// the usual quintic), a later one, where R has the singular values near 1 of
// many directions, before it passes 2^4 (two).  Errors of the iteration in
// float arithmetic, 1000 x 1024, relative 2-norm: five steps 1.6e-6 step by
// step, 2.5e-5 in one segment, 4.6e-6 as 3 + 2; six steps 2.3e-6, 1.1e-4,
// 2.0e-5 as 3 + 3 and 3.7e-6 as 2 + 2 + 2.
//
// Precision.  The products run on the half-precision matrix instructions with
// float accumulators, each operand as the sum of two half terms (22 bits; the
// low term is a multiple of 2^-24 at the least, so the sum has an absolute
// error of 2^-25 on the operand's scale).  The scales are powers of two from
// bounds on the iterates: t in [0, 1] at the start, t q(t)^2 after a step, so
// no element can leave the half type's range, whatever the matrix.  Three
// products (high high, high low, low high) give the accuracy of a float
// product: the missing low low term is 2^-22 of it.
#include <algorithm>
#include <type_traits>

#include "ns_device.h"

namespace caffe_hip {

namespace {

// --------------------------------------------------------------- first pass
constexpr int kNormBlocks = 1024;  // partial sums of one matrix, at most

// The momentum update and each block's part of ||u||^2, in double (squares of
// floats neither overflow nor vanish there).  Bound by HBM.
template <int VEC>
__global__ void __launch_bounds__(256)
ns_norm_kernel(const NsInput in, double* __restrict__ part)
{
    const int64_t base = (int64_t)blockIdx.y * in.count;
    double s = 0.0;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * VEC; i < in.count;
         i += (int64_t)gridDim.x * 256 * VEC) {
        float u[VEC];
        load_u<VEC>(in, base + i, true, u);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            s += (double)u[e] * (double)u[e];
    }
    s = block_sum<4>(s);
    if (threadIdx.x == 0)
        part[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
}

// u / norm as pair matrices in both orders: rows along u's columns (Nl) and
// columns along u's rows (Tl), through a 64 x 64 tile in LDS.
struct NsStage {
    NsInput in;
    const double* part;
    int parts;
    double eps;
    int rows, cols;
    char *Nl, *Tl;
    size_t n_pitch, t_pitch, n_batch, t_batch;  // bytes
    float scale;
};

template <int VEC>
__global__ void __launch_bounds__(256)
ns_stage_kernel(const NsStage p)
{
    __shared__ float tile[64][65];
    const int b = blockIdx.z;
    const double inv = inv_norm<4>(p.part + (size_t)b * p.parts, p.parts, p.eps) * p.scale;
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    const int64_t base = (int64_t)b * p.in.count;
    const int nk = (int)(p.n_pitch / 4), tk = (int)(p.t_pitch / 4);  // padded reduction lengths
    const int c4 = (threadIdx.x & 15) * 4, rt = threadIdx.x >> 4;
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int r = r0 + rt + 16 * it, c = c0 + c4;
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        if (r < p.rows) {
            const int64_t at = base + (int64_t)r * p.cols + c;
            if constexpr (VEC == 4) {
                if (c < p.cols)
                    load_u<4>(p.in, at, false, x);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < p.cols) {
                        float y[1];
                        load_u<1>(p.in, at + e, false, y);
                        x[e] = y[0];
                    }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = (float)((double)x[e] * inv);
            if (c < nk)
                store_pair4(p.Nl + b * p.n_batch, pair_off(p.n_pitch, r, c), x);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            tile[rt + 16 * it][c4 + e] = x[e];
    }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int c = c0 + rt + 16 * it, r = r0 + c4;
        if (c < p.cols && r < tk) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = tile[c4 + e][rt + 16 * it];
            store_pair4(p.Tl + b * p.t_batch, pair_off(p.t_pitch, c, r), x);
        }
    }
}

// ----------------------------------------------------------------- products
enum NsEpi {
    kEpiSym = 0,   // D = A B, symmetric, mirrored
    kEpiQ = 1,     // D = a I + b R + c A B, symmetric, mirrored
    kEpiPart = 2,  // part[split] = A B over a share of the reduction
    kEpiX = 3,     // D = A B and its transpose D2
    // the result, or the weights' step, four neighbours of the output to a lane
    // where its rows allow it, else one
    kEpiOut4 = 4,
    kEpiOut1 = 5,
    kEpiStep4 = 6,
    kEpiStep1 = 7
};

struct NsGemm {
    const char *A[2], *B[2];  // two products of the same shape in one launch
    char* D[2];
    char* D2;
    const char* R;
    size_t a_batch, b_batch, d_batch, d2_batch, r_batch;
    uint32_t a_pitch, b_pitch, d_pitch, d2_pitch, r_pitch;
    int M, N, stages, splits, jobs, batch;
    float mul;     // accumulator -> the value on D's scale (kEpiQ, outputs: the value itself)
    float mul2;    // ... of the second product
    float a, b, c; // kEpiQ: b on R's scale
    float d_scale; // kEpiQ: value -> D's scale
    // outputs
    float* out_f32;
    uint16_t* out_bf16;
    float* w;
    const float* lr_dev;
    float lr, decay, step_scale;
    int transposed;  // out is N x M
    float* part;     // kEpiPart: [batch][split][M][N]
};

// Tiles of one product in bands of four tile rows, columns outside, rows
// inside: what runs at the same time shares its operand rows in L2.  Below
// the diagonal only, with SYM.
template <bool SYM>
__device__ __forceinline__ void tile_at(int t, int mt, int nt, int& I, int& J)
{
    constexpr int GB = 4;
    if constexpr (!SYM) {
        const int band = t / (GB * nt);
        const int h = min(GB, mt - band * GB);
        const int r = t - band * GB * nt;
        J = r / h;
        I = band * GB + r % h;
    } else {
        // rows before row i hold i (i + 1) / 2 tiles
        int band = 0, left = t;
        for (;;) {
            const int i0 = band * GB, h = min(GB, mt - i0);
            const int cnt = h * i0 + h * (h + 1) / 2;
            if (left < cnt || i0 + h >= mt)
                break;
            left -= cnt;
            ++band;
        }
        const int i0 = band * GB, h = min(GB, mt - i0);
        if (left < h * (i0 + 1)) {
            J = left / h;
            I = i0 + left % h;
        } else {
            left -= h * (i0 + 1);
            J = i0 + 1;
            while (left >= i0 + h - J) {
                left -= i0 + h - J;
                ++J;
            }
            I = J + left;
        }
    }
}

// 32 x 32 by four waves that share the reduction, 64 x 64 and 128 x 128 by 2 x 2
// waves, all with accumulators for the low terms; 192 x 192 by four waves and
// 256 x 192 by eight, whose accumulators fill the registers.
typedef TileNT<OpPairLine, 2, 2, 1, 1, 5, true> Tile64;
typedef TileShared<OpPairLine, 4, true> Tile32;
typedef TileNT<OpPair, 2, 2, 2, 2, 2, true> Tile128;
typedef TileNT<OpPair, 2, 2, 3, 3, 3, false> Tile192;
typedef TileNT<OpPair, 4, 2, 2, 3, 2, false> Tile256;

template <class Tile, int EPI>
__global__ void __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd)
ns_gemm_kernel(const NsGemm p)
{
    constexpr bool SYM = EPI == kEpiSym || EPI == kEpiQ || EPI == kEpiPart;
    static_assert(!SYM || Tile::TM == Tile::TN, "mirrored tiles are square");
    const int mt = (p.M + Tile::TM - 1) / Tile::TM;
    const int nt = (p.N + Tile::TN - 1) / Tile::TN;
    const int per = SYM ? mt * (mt + 1) / 2 : mt * nt;
    // consecutive tiles on one XCD (workgroups go round the eight)
    const int chunk = gridDim.x >> 3;
    int t = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
    if (t >= per * p.jobs * p.splits * p.batch)
        return;
    int I, J;
    tile_at<SYM>(t % per, mt, nt, I, J);
    t /= per;
    const int split = t % p.splits;
    t /= p.splits;
    const int job = t % p.jobs, b = t / p.jobs;
    const int m0 = I * Tile::TM, n0 = J * Tile::TN;
    const char* A = p.A[job] + b * p.a_batch + (size_t)m0 * p.a_pitch;
    const char* B = p.B[job] + b * p.b_batch + (size_t)n0 * p.b_pitch;
    const int s0 = (int)((int64_t)p.stages * split / p.splits);
    const int s1 = (int)((int64_t)p.stages * (split + 1) / p.splits);
    // kEpiQ: a block of R, in each()'s order; a tile of one block has it on its
    // way during the product
    constexpr bool PRE = EPI == kEpiQ && Tile::kMI * Tile::kNI == 1;
    u32x2 pre[EPI == kEpiQ ? 8 : 1];
    auto load_r = [&](int q, int i, int j) {
        const char* r = p.R + b * p.r_batch +
                        pair_off(p.r_pitch, min(j, p.M - 1), min(i, (int)(p.r_pitch / 4) - 4));
        pre[2 * q] = *(const u32x2*)r;
        pre[2 * q + 1] = *(const u32x2*)(r + 64);
    };
    if constexpr (PRE)
        Tile::positions([&](int q, int di, int dj) { load_r(q, m0 + di, n0 + dj); });
    typename Tile::acc_t acc[Tile::kMI][Tile::kNI];
    Tile::run(A, (uint32_t)min(Tile::TM, p.M - m0) * p.a_pitch, p.a_pitch, B,
              (uint32_t)min(Tile::TN, p.N - n0) * p.b_pitch, p.b_pitch, s0, s1 - s0, acc);

    const int lt = threadIdx.x & 3;
    if constexpr (EPI == kEpiSym || EPI == kEpiQ) {
        char* D = p.D[job] + b * p.d_batch;
        const int kp = (int)(p.d_pitch / 4);
        const bool mirror = I != J;
        const float mul = job ? p.mul2 : p.mul;
        auto load = [&](int q, int di, int dj) {
            if constexpr (EPI == kEpiQ && !PRE)
                load_r(q, m0 + di, n0 + dj);
        };
        Tile::each(acc, load, [&](int q, int di, int dj, float(&v)[4]) {
            const int i = m0 + di, j = n0 + dj;
            if constexpr (EPI == kEpiQ) {
                const halfx4 h = __builtin_bit_cast(halfx4, pre[2 * q]);
                const halfx4 l = __builtin_bit_cast(halfx4, pre[2 * q + 1]);
                const bool in = j < p.M && i < kp;
                float r[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    r[e] = in ? (float)h[e] + (float)l[e] : 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = ((i + e == j && j < p.M ? p.a : 0.f) + p.b * r[e] +
                            p.c * (v[e] * p.mul)) * p.d_scale;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] *= mul;
            }
            if (mirror && j < p.M && i < kp)
                store_pair4(D, pair_off(p.d_pitch, j, i), v);
            quad_transpose(v);
            if (i + lt < p.M && j - lt < kp)
                store_pair4(D, pair_off(p.d_pitch, i + lt, j - lt), v);
        });
    } else if constexpr (EPI == kEpiPart) {
        float* D = p.part + ((size_t)b * p.splits + split) * p.M * p.N;
        Tile::each(acc, [&](int di, int dj, float(&v)[4]) {
            const int i = m0 + di, j = n0 + dj;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < p.M && j < p.N)
                    D[(size_t)(i + e) * p.N + j] = v[e];
        });
    } else if constexpr (EPI == kEpiX) {
        char *D = p.D[0] + b * p.d_batch, *D2 = p.D2 + b * p.d2_batch;
        const int kp = (int)(p.d_pitch / 4), kp2 = (int)(p.d2_pitch / 4);
        Tile::each(acc, [&](int di, int dj, float(&v)[4]) {
            const int i = m0 + di, j = n0 + dj;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] *= p.mul;
            if (j < p.N && i < kp2)
                store_pair4(D2, pair_off(p.d2_pitch, j, i), v);
            quad_transpose(v);
            if (i + lt < p.M && j - lt < kp)
                store_pair4(D, pair_off(p.d_pitch, i + lt, j - lt), v);
        });
    } else {
        // offsets from the tile's first output fit 32 bits: 256 rows of 2^20
        const int64_t at0 = (int64_t)b * p.M * p.N + (p.transposed ? (int64_t)n0 * p.M + m0
                                                                   : (int64_t)m0 * p.N + n0);
        constexpr bool STEP = EPI == kEpiStep4 || EPI == kEpiStep1;
        constexpr bool VEC = EPI == kEpiOut4 || EPI == kEpiStep4;
        float lr = 0.f;
        if constexpr (STEP)
            lr = p.lr_dev ? *p.lr_dev : p.lr;
        const uint32_t esize = !STEP && p.out_bf16 ? 2 : 4;
        char* out = STEP ? (char*)p.w : (p.out_bf16 ? (char*)p.out_bf16 : (char*)p.out_f32);
        const __amdgpu_buffer_rsrc_t ro = make_rsrc(out + at0 * esize, 0x7FFFFFFFu);
        auto off = [&](int di, int dj) -> uint32_t {
            const uint32_t e = p.transposed ? (uint32_t)dj * p.M + di : (uint32_t)di * p.N + dj;
            return m0 + di < p.M && n0 + dj < p.N ? e * esize : kOob;
        };
        const int shift = VEC && !p.transposed ? lt : 0;  // of the transposed quad
        // the weights of a block are on their way before the first is written
        floatx4 w[4];
        auto load = [&](int q, int di, int dj) {
            if constexpr (STEP && VEC)
                w[q] = __builtin_bit_cast(floatx4, buf_ld_b128(ro, off(di + shift, dj - shift)));
            else if constexpr (STEP)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w[q][e] = buf_ld_f32(ro, off(di + e, dj));
        };
        Tile::each(acc, load, [&](int q, int di, int dj, float(&v)[4]) {
            if (VEC && !p.transposed)
                quad_transpose(v);
            float o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[e] = v[e] * p.mul;
                if constexpr (STEP)
                    o[e] = w[q][e] - lr * (p.step_scale * o[e] + p.decay * w[q][e]);
            }
            if constexpr (VEC) {
                const uint32_t at = off(di + shift, dj - shift);
                if (!STEP && p.out_bf16)
                    __builtin_amdgcn_raw_buffer_store_b64(
                        u32x2{f32x2_to_bf16x2_rne(o[0], o[1]), f32x2_to_bf16x2_rne(o[2], o[3])},
                        ro, at, 0, 0);
                else
                    buf_st_b128(o, ro, at);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t at = off(di + e, dj);
                    if (!STEP && p.out_bf16)
                        __builtin_amdgcn_raw_buffer_store_b16(f32_to_bf16_rne(o[e]), ro, at, 0, 0);
                    else
                        buf_st_f32(o[e], ro, at);
                }
            }
        });
    }
}

// R = sum of the partial products, in order, as a mirrored pair matrix: a
// workgroup takes a 32 x 32 block at or below the diagonal (within the tiles of
// 64 that the parts hold), four loads of each thread in flight, and writes it
// and, through LDS, its mirror.
__global__ void __launch_bounds__(256)
ns_reduce_kernel(const float* __restrict__ part, int splits, int m, char* __restrict__ D,
                 size_t pitch, size_t d_batch, float mul)
{
    __shared__ float tile[32][33];
    int I = (int)((sqrtf(8.f * blockIdx.x + 1.f) - 1.f) * 0.5f);
    I += ((I + 1) * (I + 2) / 2 <= (int)blockIdx.x);  // (a root rounded down)
    I -= (I * (I + 1) / 2 > (int)blockIdx.x);         // (or up)
    const int J = (int)blockIdx.x - I * (I + 1) / 2;
    const int b = blockIdx.y, r = threadIdx.x >> 3, c = (threadIdx.x & 7) * 4;
    const int i = 32 * I + r, j = 32 * J + c;
    const size_t size = (size_t)m * m;
    const float* P = part + (size_t)b * splits * size;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (i < m) {
        if (m % 4 == 0) {
            if (j < m) {
                const float* p = P + (size_t)i * m + j;
                for (int s = 0; s < splits; s += 4) {
                    floatx4 x[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        x[q] = s + q < splits ? *(const floatx4*)(p + (s + q) * size)
                                              : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            v[e] += x[q][e];
                }
            }
        } else {
            for (int s = 0; s < splits; s += 4) {
                float x[4][4];
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[q][e] = s + q < splits && j + e < m
                                      ? P[(s + q) * size + (size_t)i * m + j + e] : 0.f;
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] += x[q][e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] *= mul;
        tile[r][c + e] = v[e];
    }
    const int kp = (int)(pitch / 4);
    if (i < m && j < kp)
        store_pair4(D + b * d_batch, pair_off(pitch, i, j), v);
    if (I == J)
        return;
    __syncthreads();
    const int mi = 32 * J + r, mk = 32 * I + c;  // row and columns of the mirror
    if (mi < m && mk < kp) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = tile[c + e][r];
        store_pair4(D + b * d_batch, pair_off(pitch, mi, mk), v);
    }
}

// --------------------------------------------------------------------- host
template <class Tile, int EPI>
int64_t tile_count(const NsGemm& p)
{
    constexpr bool SYM = EPI == kEpiSym || EPI == kEpiQ || EPI == kEpiPart;
    const int64_t mt = (p.M + Tile::TM - 1) / Tile::TM, nt = (p.N + Tile::TN - 1) / Tile::TN;
    return (SYM ? mt * (mt + 1) / 2 : mt * nt) * p.jobs * p.splits * p.batch;
}

template <class Tile, int EPI>
hipError_t launch_tile(const NsGemm& p, hipStream_t s)
{
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ns_gemm_kernel<Tile, EPI>),
                       dim3((unsigned)((tile_count<Tile, EPI>(p) + 7) / 8 * 8)),
                       dim3(Tile::kThreads), 0, s, p);
    return hipGetLastError();
}

// Fitted to 140 x 140 .. 4096 x 9216; us measured / modelled, symmetric products
// of m = 200 .. 4096 and the full one of 4096 x 9216 x 4096:
//          200       512       700       1280      1800      2560      3000       4096       x 9216
//   32   5.1 / 5.3 6.5 / 6.5 8.0 / 7.4  30 / 30   63 / 68
//   64   6.3 / 6.3 9.0 / 8.9  11 / 11   16 / 16   33 / 35   93 / 91   129 / 131  255 / 315  1090 / 1250
//   128             20 / 20             40 / 42   51 / 57   80 / 78   126 / 130  240 / 260   790 / 766
//   192             33 / 33             56 / 64   73 / 86  101 / 116  125 / 134  185 / 178   900 / 844
//   256 x 192 (full products only)                                                           755 / 745
constexpr TileTime kTime32 = {4.3, 0.14, 0.16}, kTime64 = {4.3, 0.29, 0.27},
                   kTime128 = {6.0, 0.90, 0.66}, kTime192 = {12.0, 1.30, 1.30},
                   kTime256 = {15.0, 1.90, 1.90};

// The tile with the least time by the model.
template <int EPI>
hipError_t launch_gemm(const NsGemm& p, hipStream_t s)
{
    const double t32 = kTime32.of(tile_count<Tile32, EPI>(p), p.stages);
    const double t64 = kTime64.of(tile_count<Tile64, EPI>(p), p.stages);
    const double t128 = kTime128.of(tile_count<Tile128, EPI>(p), p.stages);
    const double t192 = kTime192.of(tile_count<Tile192, EPI>(p), p.stages);
    double least = std::min(std::min(t32, t64), std::min(t128, t192));
    if constexpr (EPI >= kEpiX) {
        const double t256 = kTime256.of(tile_count<Tile256, EPI>(p), p.stages);
        if (t256 < least)
            return launch_tile<Tile256, EPI>(p, s);
    }
    if (t192 <= least)
        return launch_tile<Tile192, EPI>(p, s);
    if (t128 <= least)
        return launch_tile<Tile128, EPI>(p, s);
    if (t64 <= least)
        return launch_tile<Tile64, EPI>(p, s);
    return launch_tile<Tile32, EPI>(p, s);
}

}  // namespace

int ns_exponent(double bound)
{
    int e;
    frexp(bound, &e);
    return 14 - e;
}

// The ranges of t q(t)^2 and q(t) over t in [0, top]: their extremes lie at
// the ends or where a derivative vanishes.
static void ns_ranges(double a, double b, double c, double top, double* qmax, double* tmax)
{
    auto q = [&](double t) { return a + b * t + c * t * t; };
    double at[5] = {0.0, top, 0.0, 0.0, 0.0};
    int n = 2;
    if (c != 0.0)
        at[n++] = -b / (2 * c);
    // d/dt t q^2 = q (q + 2 t q'):  a + 3 b t + 5 c t^2 = 0 (q = 0 gives the minimum)
    // with the root that does not cancel formed by the quadratic formula and the
    // other from the product of both, a / (5 c): right for c of any size, also 0
    const double d = 9 * b * b - 20 * a * c;
    if (d >= 0) {
        const double w = -0.5 * (3 * b + copysign(sqrt(d), b));
        if (c != 0.0)
            at[n++] = w / (5 * c);
        if (w != 0.0)
            at[n++] = a / w;
    }
    *qmax = *tmax = 0.0;
    for (int i = 0; i < n; ++i)
        if (at[i] >= 0.0 && at[i] <= top) {
            *qmax = std::max(*qmax, fabs(q(at[i])));
            *tmax = std::max(*tmax, at[i] * q(at[i]) * q(at[i]));
        }
}

bool ns_plan(int batch, int rows, int cols, int steps, float a, float b, float c, NsPlan* q)
{
    *q = NsPlan{};
    q->batch = batch;
    q->rows = rows;
    q->cols = cols;
    q->tall = rows > cols;
    q->m = std::min(rows, cols);
    q->n = std::max(rows, cols);
    q->steps = steps;
    // ranges of every step
    double top = 1.0;
    q->bound[0] = 1.0;
    double qall = 0.0;
    for (int k = 0; k < steps; ++k) {
        double qmax, tmax;
        ns_ranges(a, b, c, top, &qmax, &tmax);
        if (!(tmax <= kNsMaxRange) || !(qmax <= kNsMaxRange))
            return false;
        q->qmax[k] = std::max(qmax, 1e-3);
        q->bound[k + 1] = top = std::max(tmax, 1e-3);
        qall = std::max(qall, q->qmax[k]);
    }
    // the longest first segment, and the longest later one
    int first = steps, later = steps;
    if (qall > 1.0) {
        // (as doubles: for qall next to 1 the quotients pass every int)
        const double per = 2.0 * log(qall);
        first = (int)std::min((double)steps, 1 + floor(log(256.0) / per + 1e-9));
        later = (int)std::min((double)steps, 1 + floor(log(16.0) / per + 1e-9));
    }
    q->segments = 1 + (steps - first + later - 1) / later;
    int left = steps;
    for (int i = q->segments - 1; i > 0; --i) {
        q->length[i] = std::min(later, left / (i + 1));
        left -= q->length[i];
    }
    q->length[0] = left;
    for (int i = 0, k = 0; i < q->segments; ++i) {
        double pb = 1.0;
        for (int l = 0; l < q->length[i]; ++l, ++k)
            // (the scale 2^-e of a product, e <= 109, and of X in it are floats)
            q->pmax[k] = pb = std::max(pb * q->qmax[k], 0x1p-96);
    }
    const size_t align = 255;
    const size_t mp = (size_t)((q->m + 31) / 32) * 128, np = (size_t)((q->n + 31) / 32) * 128;
    q->m_pitch = mp;
    q->n_pitch = np;
    q->mm_bytes = ((size_t)q->m * mp + align) & ~align;
    q->xr_bytes = ((size_t)q->m * np + align) & ~align;
    q->xt_bytes = ((size_t)q->n * mp + align) & ~align;
    // The Gram product of a short wide matrix has few tiles of long sums.  Its
    // reduction is split until tiles of 64 fill the 256 compute units, parts of
    // at least four lines each, where that and the launch that adds the parts
    // (3.5 us) take less time than the whole in one launch.
    const int64_t lines = (int64_t)(np / 128);
    auto tiles = [&](int64_t side) {
        const int64_t t = (q->m + side - 1) / side;
        return t * (t + 1) / 2 * batch;
    };
    q->splits = 1;
    if (batch > 0) {
        const int64_t s = std::min(256 / tiles(64), lines / 4);
        if (s > 1 && kTime64.of(s * tiles(64), (lines + s - 1) / s) + 3.5 <
                         std::min(kTime32.of(tiles(32), lines), kTime64.of(tiles(64), lines)))
            q->splits = (int)s;
    }
    q->norm_blocks = (int)std::min<int64_t>(kNormBlocks,
                                            ((int64_t)rows * cols + 4095) / 4096);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off += (bytes + align) & ~align;
        return at;
    };
    q->off_part = take((size_t)batch * q->norm_blocks * sizeof(double));
    q->small = q->m <= kNsSmall;
    if (q->small) {
        ns_small_sizes(q->m, q->n, q);
        q->off_split = take(batch * q->part_bytes);
        q->off_mm[0] = take(batch * q->img_bytes);
        q->off_xt[0] = take(q->segments > 1 ? batch * q->xs_bytes : 0);
        q->ws_bytes = off;
        return true;
    }
    q->off_split = take(q->splits > 1 ? (size_t)batch * q->splits * q->m * q->m * 4 : 0);
    q->off_xr = take(batch * q->xr_bytes);
    q->off_xt[0] = take(batch * q->xt_bytes);
    q->off_xt[1] = q->segments > 1 ? take(batch * q->xt_bytes) : 0;
    for (int i = 0; i < 5; ++i)
        q->off_mm[i] = take(batch * q->mm_bytes);
    q->ws_bytes = off;
    return true;
}

hipError_t launch_newton_schulz(const NsPlan& q, const NsArgs& x, char* ws, hipStream_t s)
{
    if (q.batch == 0)
        return hipSuccess;
    const int64_t count = (int64_t)q.rows * q.cols;
    NsInput in{};
    in.g = x.g;
    in.v = x.v;
    in.mu = x.momentum;
    in.nesterov = x.nesterov;
    in.bf16 = x.bf16;
    in.count = count;
    if (q.small && q.solo)
        return launch_ns_small(q, in, x, ws, s);
    double* part = (double*)(ws + q.off_part);
    const dim3 ng((unsigned)q.norm_blocks, (unsigned)q.batch);
    if (count % 4 == 0)
        hipLaunchKernelGGL(ns_norm_kernel<4>, ng, dim3(256), 0, s, in, part);
    else
        hipLaunchKernelGGL(ns_norm_kernel<1>, ng, dim3(256), 0, s, in, part);
    if (q.small)
        return launch_ns_small(q, in, x, ws, s);

    char *xr = ws + q.off_xr, *xt = ws + q.off_xt[0], *xt2 = ws + q.off_xt[1];
    int ex = ns_exponent(1.0);
    NsStage st{};
    st.in = in;
    st.part = part;
    st.parts = q.norm_blocks;
    st.eps = x.eps;
    st.rows = q.rows;
    st.cols = q.cols;
    st.Nl = q.tall ? xt : xr;
    st.Tl = q.tall ? xr : xt;
    st.n_pitch = q.tall ? q.m_pitch : q.n_pitch;
    st.t_pitch = q.tall ? q.n_pitch : q.m_pitch;
    st.n_batch = q.tall ? q.xt_bytes : q.xr_bytes;
    st.t_batch = q.tall ? q.xr_bytes : q.xt_bytes;
    st.scale = ldexpf(1.f, ex);
    const dim3 sg((unsigned)((q.cols + 63) / 64), (unsigned)((q.rows + 63) / 64),
                  (unsigned)q.batch);
    if (q.cols % 4 == 0)
        hipLaunchKernelGGL(ns_stage_kernel<4>, sg, dim3(256), 0, s, st);
    else
        hipLaunchKernelGGL(ns_stage_kernel<1>, sg, dim3(256), 0, s, st);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;

    auto square = [&](char* A, char* B, char* D) {
        NsGemm p{};
        p.A[0] = A;
        p.B[0] = B;
        p.D[0] = D;
        p.a_batch = p.b_batch = p.d_batch = p.r_batch = q.mm_bytes;
        p.a_pitch = p.b_pitch = p.d_pitch = p.r_pitch = (uint32_t)q.m_pitch;
        p.M = p.N = q.m;
        p.stages = (int)(q.m_pitch / 128);
        p.splits = p.jobs = 1;
        p.batch = q.batch;
        return p;
    };
    char* R = ws + q.off_mm[0];
    char* T = ws + q.off_mm[1];
    char* Qm = ws + q.off_mm[2];
    int k = 0;
    for (int seg = 0; seg < q.segments; ++seg) {
        const int L = q.length[seg];
        // R = X X^T
        int er = ns_exponent(q.bound[k]);
        {
            NsGemm p{};
            p.A[0] = p.B[0] = xr;
            p.D[0] = R;
            p.a_batch = p.b_batch = q.xr_bytes;
            p.d_batch = q.mm_bytes;
            p.a_pitch = p.b_pitch = (uint32_t)q.n_pitch;
            p.d_pitch = (uint32_t)q.m_pitch;
            p.M = p.N = q.m;
            p.stages = (int)(q.n_pitch / 128);
            p.splits = q.splits;
            p.jobs = 1;
            p.batch = q.batch;
            p.mul = ldexpf(1.f, er - 2 * ex);
            if (q.splits > 1) {
                p.part = (float*)(ws + q.off_split);
                e = launch_tile<Tile64, kEpiPart>(p, s);
                if (e != hipSuccess)
                    return e;
                const unsigned blocks = (unsigned)((q.m + 31) / 32);
                hipLaunchKernelGGL(ns_reduce_kernel,
                                   dim3(blocks * (blocks + 1) / 2, (unsigned)q.batch), dim3(256),
                                   0, s, p.part, q.splits, q.m, R, q.m_pitch, q.mm_bytes, p.mul);
                e = hipGetLastError();
            } else {
                e = launch_gemm<kEpiSym>(p, s);
            }
            if (e != hipSuccess)
                return e;
        }
        char* P = nullptr;
        int ep = 0;
        for (int l = 0; l < L; ++l, ++k) {
            // Q = a I + b R + c R R; the segment's first is its P as well
            char* spare = ws + q.off_mm[P == ws + q.off_mm[3] ? 4 : 3];
            char* Q = P ? Qm : spare;
            const int eq = ns_exponent(q.qmax[k]);
            NsGemm p = square(R, R, Q);
            p.R = R;
            p.mul = ldexpf(1.f, -2 * er);
            p.a = x.a;
            p.b = ldexpf(x.b, -er);
            p.c = x.c;
            p.d_scale = ldexpf(1.f, eq);
            if ((e = launch_gemm<kEpiQ>(p, s)) != hipSuccess)
                return e;
            const bool more = l + 1 < L;
            const int et = ns_exponent(q.qmax[k] * q.bound[k]);
            const int ep2 = ns_exponent(q.pmax[k]);
            char* P2 = spare;
            // T = Q R and P = Q P, neither of which waits for the other
            p = square(Q, R, T);
            p.mul = ldexpf(1.f, et - eq - er);
            if (P) {
                const int j = more ? 1 : 0;
                p.A[j] = Q;
                p.B[j] = P;
                p.D[j] = P2;
                (j ? p.mul2 : p.mul) = ldexpf(1.f, ep2 - eq - ep);
                p.jobs = j + 1;
            }
            if (more || P)
                if ((e = launch_gemm<kEpiSym>(p, s)) != hipSuccess)
                    return e;
            if (more) {
                er = ns_exponent(q.bound[k + 1]);
                p = square(T, Q, R);
                p.mul = ldexpf(1.f, er - et - eq);
                if ((e = launch_gemm<kEpiSym>(p, s)) != hipSuccess)
                    return e;
            }
            P = P2;
            ep = P == Q ? eq : ep2;
        }
        // X = P X
        NsGemm p{};
        p.A[0] = P;
        p.B[0] = xt;
        p.a_batch = q.mm_bytes;
        p.b_batch = q.xt_bytes;
        p.a_pitch = p.b_pitch = (uint32_t)q.m_pitch;
        p.M = q.m;
        p.N = q.n;
        p.stages = (int)(q.m_pitch / 128);
        p.splits = p.jobs = 1;
        p.batch = q.batch;
        if (seg + 1 < q.segments) {
            const int ex2 = ns_exponent(sqrt(q.bound[k]));
            p.D[0] = xr;
            p.D2 = xt2;
            p.d_batch = q.xr_bytes;
            p.d2_batch = q.xt_bytes;
            p.d_pitch = (uint32_t)q.n_pitch;
            p.d2_pitch = (uint32_t)q.m_pitch;
            p.mul = ldexpf(1.f, ex2 - ep - ex);
            ex = ex2;
            std::swap(xt, xt2);
            e = launch_gemm<kEpiX>(p, s);
        } else {
            p.mul = ldexpf(1.f, -ep - ex);
            p.out_f32 = (float*)x.out;
            p.out_bf16 = x.bf16 ? (uint16_t*)x.out : nullptr;
            p.w = x.w;
            p.lr = x.lr;
            p.lr_dev = x.lr_dev;
            p.decay = x.decay;
            p.step_scale = x.step_scale;
            p.transposed = q.tall;
            const bool four = (q.tall ? q.m : q.n) % 4 == 0;
            if (x.w)
                e = four ? launch_gemm<kEpiStep4>(p, s) : launch_gemm<kEpiStep1>(p, s);
            else
                e = four ? launch_gemm<kEpiOut4>(p, s) : launch_gemm<kEpiOut1>(p, s);
        }
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace caffe_hip
