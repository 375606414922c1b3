// muon_small.hip -- the Newton-Schulz iteration of matrices with a side of at
// most 128 (muon.hip holds the mathematics and the segments).
//
// With m <= 128 every m x m matrix of a segment fits one workgroup: the
// wave w of eight holds rows 16 w .. 16 w + 15 of each (its panel) in
// registers, and only the left factors of the products, R and Q, are in LDS.
// A panel is held transposed, in the layout that the 16x16x32 instruction
// leaves its results in (lane l: column l % 16 of the panel's transpose, rows
// 16 I + 4 (l / 16) + 0..3): the same instruction takes it as its right operand
// when the left operand's reduction index is permuted alike, which LDS rows
// are (image below), so no product moves a panel between lanes.
//
// The wide ends of a segment -- the Gram matrix X X^T and P X -- go over
// column slabs of X: eight waves take 16 columns each, in the same layout.
// A long X gives each slab a workgroup and the segment's m x m part a launch of
// one workgroup between them; a short one (NsPlan::solo) runs everything in
// one launch.  Bound by latency: 50 x 500 reads 100 KB and computes 10 MFLOP.
#include <algorithm>

#include "ns_device.h"

namespace caffe_hip {

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kChunk = 16 * kWaves;        // columns at a time
constexpr int kChunkPitch = kChunk * 4 + 16;

// LDS image of an m x m pair matrix: rows MT lines of 128 bytes and 16 bytes
// apart from a multiple (16 rows then start in different banks).  Of the 32
// reduction elements of a line, k = 16 h + 4 g + e is at place 8 g + 4 h + e.
template <int MT>
struct Small {
    static constexpr int LD = 32 * MT;     // padded side
    static constexpr int T16 = 2 * MT;     // 16-blocks of a side
    static constexpr int kPitch = MT * 128 + 16;
    static constexpr int kImage = LD * kPitch;
    static constexpr int kTiles = MT * (MT + 1) / 2;      // 32 x 32 below the diagonal
    static constexpr int kSplit = MT == 1 ? 8 : (MT == 2 ? 2 : 1);  // waves to a tile
    static constexpr int kOwn = (kTiles * kSplit + kWaves - 1) / kWaves;
    static constexpr int kShares = kSplit > 1 ? kWaves * 16 * 64 * 4 : 0;
    static constexpr int kChunkBytes = LD * kChunkPitch > kShares ? LD * kChunkPitch : kShares;
    static constexpr int kLds = kImage + (kImage > kChunkBytes ? kImage : kChunkBytes);
    typedef float Panel[T16][4];

    static __device__ __forceinline__ void store_panel(char* img, int row, const Panel& d,
                                                       float scale)
    {
        const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int I = 0; I < T16; ++I) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = d[I][e] * scale;
            store_pair4(img, (size_t)row * kPitch + (I >> 1) * 128 + g * 16 + (I & 1) * 8, v);
        }
    }

    // y = mul * (img d^T)^T, both factors as pairs, d's on its scale; y may be d
    static __device__ __forceinline__ void product(const char* img, const Panel& d, float scale,
                                                   float mul, Panel& y)
    {
        const int lane = threadIdx.x & 63;
        halfx8 bh[MT], bl[MT];
#pragma unroll
        for (int s = 0; s < MT; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = d[2 * s + (e >> 2)][e & 3] * scale;
                bh[s][e] = (_Float16)x;
                bl[s][e] = (_Float16)(x - (float)bh[s][e]);
            }
        const char* p = img + (size_t)(lane & 15) * kPitch + (lane >> 4) * 16;
#pragma unroll
        for (int I = 0; I < T16; ++I) {
            floatx4 hi = {0.f, 0.f, 0.f, 0.f}, lo = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < MT; ++s) {
                const halfx8 ah = *(const halfx8*)(p + I * 16 * kPitch + s * 128);
                const halfx8 al = *(const halfx8*)(p + I * 16 * kPitch + s * 128 + 64);
                hi = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bh[s], hi, 0, 0, 0);
                lo = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bl[s], lo, 0, 0, 0);
                lo = __builtin_amdgcn_mfma_f32_16x16x32_f16(al, bh[s], lo, 0, 0, 0);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                y[I][q] = (hi[q] + lo[q]) * mul;
            if (MT > 2 && I & 1)  // (all reads at once would not fit the registers)
                __builtin_amdgcn_sched_barrier(0);
        }
    }
};

__device__ __forceinline__ float pow2(int e) { return ldexpf(1.f, e); }

// A lane's elements (i0 + 4 g, j) of matrix b of a batch, i0 the same on all
// lanes: byte offset at(i0) (out of range outside the matrix) + step i0.  A
// matrix has at most 128 * 2^20 elements, so offsets fit 32 bits.
struct Columns {
    __amdgpu_buffer_rsrc_t r;
    uint32_t v0, step;
    int left;  // rows from this lane's first
    __device__ __forceinline__ Columns(const NsSmall& p, const void* base, uint32_t esize, int b,
                                       int j)
        : r(make_rsrc((const char*)base + (int64_t)b * p.in.count * esize,
                      (uint32_t)p.in.count * esize))
    {
        const int g4 = ((threadIdx.x & 63) >> 4) * 4;
        v0 = (p.tall ? (uint32_t)j * p.m + g4 : (uint32_t)g4 * p.n + j) * esize;
        step = (p.tall ? 1 : p.n) * esize;
        left = j < p.n ? p.m - g4 : 0;
    }
    __device__ __forceinline__ uint32_t at(int i0) const { return i0 < left ? v0 : kOob; }
};

// Columns of X in the panels' layout: d[I][q] = X[16 I + 4 g + q][j] / norm.
template <int MT, int VEC>
__device__ __forceinline__ void load_columns(const NsSmall& p, int b, int j, double inv, bool from_u,
                                             typename Small<MT>::Panel& d)
{
    const int g = (threadIdx.x & 63) >> 4;
    constexpr int T16 = Small<MT>::T16;
    if (!from_u) {
        const float* x = p.xs + ((size_t)b * p.n_pad + j) * Small<MT>::LD + 4 * g;
#pragma unroll
        for (int I = 0; I < T16; ++I) {
            const floatx4 v = *(const floatx4*)(x + 16 * I);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                d[I][q] = v[q];
        }
        return;
    }
    // all loads of an input go out before the first is used
    auto fetch = [&](const void* u, uint32_t esize, typename Small<MT>::Panel& x) {
        const Columns c(p, u, esize, b, j);
#pragma unroll
        for (int I = 0; I < T16; ++I) {
            if constexpr (VEC == 4) {  // tall, m % 4 == 0
                if (esize == 2) {
                    const u16x4 y = __builtin_bit_cast(
                        u16x4, __builtin_amdgcn_raw_buffer_load_b64(c.r, c.at(16 * I), 16 * I * 2, 0));
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        x[I][q] = bf16_to_f32(y[q]);
                } else {
                    const floatx4 y = __builtin_bit_cast(
                        floatx4, __builtin_amdgcn_raw_buffer_load_b128(c.r, c.at(16 * I), 16 * I * 4, 0));
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        x[I][q] = y[q];
                }
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = 16 * I + q;
                    if (esize == 2)
                        x[I][q] = bf16_to_f32(__builtin_amdgcn_raw_buffer_load_b16(
                            c.r, c.at(i), c.step * i, 0));
                    else
                        x[I][q] = __builtin_bit_cast(
                            float, __builtin_amdgcn_raw_buffer_load_b32(c.r, c.at(i), c.step * i, 0));
                }
            }
        }
    };
    if (p.in.bf16)
        fetch(p.in.g, 2, d);
    else
        fetch(p.in.g, 4, d);
    if (p.in.v) {
        typename Small<MT>::Panel h;
        fetch(p.in.v, 4, h);
#pragma unroll
        for (int I = 0; I < T16; ++I)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                d[I][q] = p.in.nesterov ? d[I][q] + p.in.mu * h[I][q] : h[I][q];
    }
#pragma unroll
    for (int I = 0; I < T16; ++I)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            d[I][q] = (float)((double)d[I][q] * inv);
}

enum { kGram = 0, kApplyGram = 1, kApplyOut = 2 };

// Column chunks c0 .. c1 - 1 of X: with kApply* X <- P X, then the chunks'
// part of X X^T (part number slab_no), or the result.  P's image is
// in LDS already where p_img is null.
template <int MT, int VEC, int MODE>
__device__ __forceinline__ void slab(const NsSmall& p, const NsOut& o, int b, int c0, int c1,
                                     int slab_no, double inv, bool from_u, int ex, int ep, int ex2,
                                     const char* p_img, char* lds)
{
    typedef Small<MT> S;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4;
    char *P = lds, *C = lds + S::kImage;
    if (MODE != kGram && p_img) {
        for (int i = threadIdx.x * 16; i < S::kImage; i += kThreads * 16)
            *(u32x4*)(P + i) = *(const u32x4*)(p_img + i);
        __syncthreads();
    }
    floatx16 hi[S::kOwn], lo[S::kOwn];
#pragma unroll
    for (int o2 = 0; o2 < S::kOwn; ++o2)
        hi[o2] = lo[o2] = floatx16{};
    float lr = 0.f;
    if (MODE == kApplyOut && o.w)
        lr = o.lr_dev ? *o.lr_dev : o.lr;
    for (int c = c0; c < c1; ++c) {
        const int j = c * kChunk + wave * 16 + (lane & 15);
        typename S::Panel d;
        load_columns<MT, VEC>(p, b, j, inv, from_u, d);
        if constexpr (MODE != kGram) {
            S::product(P, d, pow2(ex), pow2(-ep - ex), d);
            if constexpr (MODE == kApplyOut) {
                if (o.w) {
                    const Columns w(p, o.w, 4, b, j);
                    // two sixteens of rows at a time: their loads, then their stores
#pragma unroll
                    for (int I = 0; I < S::T16; I += 2) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int i = 16 * (I + e / 4) + e % 4;
                            x[e] = __builtin_bit_cast(
                                float, __builtin_amdgcn_raw_buffer_load_b32(w.r, w.at(i),
                                                                            w.step * i, 0));
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int i = 16 * (I + e / 4) + e % 4;
                            const float y =
                                x[e] - lr * (o.step_scale * d[I + e / 4][e % 4] + o.decay * x[e]);
                            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, y),
                                                                  w.r, w.at(i), w.step * i, 0);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    continue;
                }
                const Columns w(p, o.out_bf16 ? (const void*)o.out_bf16 : (const void*)o.out_f32,
                                o.out_bf16 ? 2 : 4, b, j);
#pragma unroll
                for (int I = 0; I < S::T16; ++I)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int i = 16 * I + q;
                        if (o.out_bf16)
                            __builtin_amdgcn_raw_buffer_store_b16(f32_to_bf16_rne(d[I][q]), w.r,
                                                                  w.at(i), w.step * i, 0);
                        else
                            __builtin_amdgcn_raw_buffer_store_b32(
                                __builtin_bit_cast(uint32_t, d[I][q]), w.r, w.at(i), w.step * i, 0);
                    }
                continue;
            }
            float* x = p.xs + ((size_t)b * p.n_pad + j) * S::LD + 4 * g;
#pragma unroll
            for (int I = 0; I < S::T16; ++I)
                *(floatx4*)(x + 16 * I) = floatx4{d[I][0], d[I][1], d[I][2], d[I][3]};
        }
        // rows of X along its columns, in LDS
        const float scale = pow2(MODE == kGram ? ex : ex2);
#pragma unroll
        for (int I = 0; I < S::T16; ++I) {
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                v[q] = d[I][q] * scale;
            quad_transpose(v);
            const int k = wave * 16 + (lane & 12);
            store_pair4(C, pair_off(kChunkPitch, 16 * I + 4 * g + (lane & 3), k), v);
        }
        __syncthreads();
#pragma unroll
        for (int o2 = 0; o2 < S::kOwn; ++o2) {
            const int unit = wave + kWaves * o2;
            if (unit < S::kTiles * S::kSplit) {
                const int tile = unit / S::kSplit, ks = unit % S::kSplit;
                const int I = tile >= 6 ? 3 : (tile >= 3 ? 2 : (tile >= 1 ? 1 : 0));
                const int J = tile - I * (I + 1) / 2;
                const char* ra = C + (size_t)(32 * I + (lane & 31)) * kChunkPitch + (lane >> 5) * 16;
                const char* rb = C + (size_t)(32 * J + (lane & 31)) * kChunkPitch + (lane >> 5) * 16;
#pragma unroll
                for (int s = 0; s < 8 / S::kSplit; ++s) {
                    const int k16 = ks * (8 / S::kSplit) + s;
                    const int off = (k16 >> 1) * 128 + (k16 & 1) * 32;
                    const halfx8 ah = *(const halfx8*)(ra + off), al = *(const halfx8*)(ra + off + 64);
                    const halfx8 bh = *(const halfx8*)(rb + off), bl = *(const halfx8*)(rb + off + 64);
                    hi[o2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bh, hi[o2], 0, 0, 0);
                    lo[o2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bl, lo[o2], 0, 0, 0);
                    lo[o2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, bh, lo[o2], 0, 0, 0);
                }
            }
        }
        __syncthreads();
    }
    if constexpr (MODE != kApplyOut) {
        const float mul = pow2(-2 * (MODE == kGram ? ex : ex2));
        if constexpr (S::kSplit > 1) {
            // the shares of a tile, added in order by the last one's wave
            float* share = (float*)C;
            const int tile = wave / S::kSplit, ks = wave % S::kSplit;
            if (tile < S::kTiles && ks + 1 < S::kSplit)
#pragma unroll
                for (int q = 0; q < 16; ++q)
                    share[(wave * 16 + q) * 64 + lane] = hi[0][q] + lo[0][q];
            __syncthreads();
            if (tile < S::kTiles && ks + 1 == S::kSplit)
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    float s = 0.f;
#pragma unroll
                    for (int w = 1; w < S::kSplit; ++w)
                        s += share[((wave - w) * 16 + q) * 64 + lane];
                    hi[0][q] += s;
                }
        }
#pragma unroll
        for (int o2 = 0; o2 < S::kOwn; ++o2) {
            const int unit = wave + kWaves * o2;
            if (unit < S::kTiles * S::kSplit && unit % S::kSplit + 1 == S::kSplit) {
                const int tile = unit / S::kSplit;
                const int I = tile >= 6 ? 3 : (tile >= 3 ? 2 : (tile >= 1 ? 1 : 0));
                const int J = tile - I * (I + 1) / 2;
                float* out = p.part + ((size_t)b * p.parts + slab_no) * S::LD * S::LD;
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const int i = 32 * I + 8 * (q >> 2) + 4 * (lane >> 5) + (q & 3);
                    out[i * S::LD + 32 * J + (lane & 31)] = (hi[o2][q] + lo[o2][q]) * mul;
                }
            }
        }
    }
}

// Steps k0 .. k0 + L - 1 on the m x m matrices: R from its parts, P's image to
// `out`.  Every wave takes the barriers, those with rows of R the work.
template <int MT>
__device__ __forceinline__ void segment(const NsSmall& p, const NsSteps& st, int b, int k0, int L,
                                        int parts, char* lds, char* out)
{
    typedef Small<MT> S;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, j = 16 * wave + (lane & 15);
    const bool live = 16 * wave < p.m;
    char *LR = lds, *LQ = lds + S::kImage;
    typename S::Panel R, Q, T, P;
    if (live) {
        const float* src = p.part + (size_t)b * p.parts * S::LD * S::LD;
#pragma unroll
        for (int I = 0; I < S::T16; ++I)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                R[I][e] = 0.f;
        for (int q = 0; q < parts; ++q) {
            const float* s = src + (size_t)q * S::LD * S::LD;
#pragma unroll
            for (int I = 0; I < S::T16; ++I) {
                const int i = 16 * I + 4 * g;
                if (I >= (wave & ~1)) {  // 32-block I / 2 of the rows at or below the panel's
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        R[I][e] += s[(i + e) * S::LD + j];
                } else {
                    const floatx4 x = *(const floatx4*)(s + j * S::LD + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        R[I][e] += x[e];
                }
            }
        }
    }
    for (int l = 0; l < L; ++l) {
        const int k = k0 + l;
        const int er = st.er[k], eq = st.eq[k], et = st.et[k];
        const bool more = l + 1 < L;
        // panels past m hold no rows: their lines of the images are never
        // multiplied with anything but zeros, and are zero themselves
        if (16 * wave < S::LD) {
            if (!live) {
#pragma unroll
                for (int I = 0; I < S::T16; ++I)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        R[I][e] = Q[I][e] = T[I][e] = P[I][e] = 0.f;
            }
            S::store_panel(LR, j, R, pow2(er));
        }
        __syncthreads();
        if (live) {
            S::product(LR, R, pow2(er), pow2(-2 * er), Q);
#pragma unroll
            for (int I = 0; I < S::T16; ++I)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    Q[I][e] = (16 * I + 4 * g + e == j && j < p.m ? st.a : 0.f) + st.b * R[I][e] +
                              st.c * Q[I][e];
            if (more)
                S::product(LR, Q, pow2(eq), pow2(-er - eq), T);
        }
        if (16 * wave < S::LD)
            S::store_panel(LQ, j, Q, pow2(eq));
        __syncthreads();
        if (live) {
            if (l) {
                const int ep = st.ep[k - 1];
                S::product(LQ, P, pow2(ep), pow2(-eq - ep), P);
            } else {
#pragma unroll
                for (int I = 0; I < S::T16; ++I)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        P[I][e] = Q[I][e];
            }
            if (more)
                S::product(LQ, T, pow2(et), pow2(-eq - et), R);
        }
        __syncthreads();
    }
    if (16 * wave < S::LD)
        S::store_panel(out, j, P, pow2(st.ep[k0 + L - 1]));
}

template <int MT, int VEC, int MODE>
__global__ void __launch_bounds__(kThreads)
ns_slab_kernel(const NsSmall p, const NsOut o, int from_u, int ex, int ep, int ex2)
{
    __shared__ __attribute__((aligned(16))) char lds[Small<MT>::kLds];
    const int b = blockIdx.y;
    const double inv =
        from_u ? inv_norm<kWaves>(p.norm + (size_t)b * p.norm_parts, p.norm_parts, p.eps) : 0.0;
    const int c0 = (int)((int64_t)p.chunks * blockIdx.x / gridDim.x);
    const int c1 = (int)((int64_t)p.chunks * (blockIdx.x + 1) / gridDim.x);
    slab<MT, VEC, MODE>(p, o, b, c0, c1, blockIdx.x, inv, from_u, ex, ep, ex2,
                        p.p_img + (size_t)b * Small<MT>::kImage, lds);
}

// The parts summed in order into the first: 64 elements to a workgroup, a
// fourth of the parts to each of its waves, eight loads in flight.
__global__ void __launch_bounds__(256)
ns_parts_kernel(float* part, int parts, int size)
{
    __shared__ float sum[4][64];
    float* p = part + (size_t)blockIdx.y * parts * size;
    const int i = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
    const int q0 = parts * w / 4, q1 = parts * (w + 1) / 4;
    float s = 0.f;
    for (int q = q0; q < q1; q += 8) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = q + e < q1 ? p[(size_t)(q + e) * size + i] : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            s += v[e];
    }
    sum[w][threadIdx.x & 63] = s;
    __syncthreads();
    if (w == 0)
        p[i] = (sum[0][threadIdx.x] + sum[1][threadIdx.x]) +
               (sum[2][threadIdx.x] + sum[3][threadIdx.x]);
}

template <int MT>
__global__ void __launch_bounds__(kThreads)
ns_segment_kernel(const NsSmall p, const NsSteps st, int k0, int L, int parts)
{
    __shared__ __attribute__((aligned(16))) char lds[Small<MT>::kLds];
    const int b = blockIdx.x;
    segment<MT>(p, st, b, k0, L, parts, lds, p.p_img + (size_t)b * Small<MT>::kImage);
}

// Everything in one launch, a workgroup to a matrix.
template <int MT, int VEC>
__global__ void __launch_bounds__(kThreads)
ns_solo_kernel(const NsSmall p, const NsSteps st, const NsOut o)
{
    typedef Small<MT> S;
    __shared__ __attribute__((aligned(16))) char lds[S::kLds];
    const int b = blockIdx.x;
    const int64_t base = (int64_t)b * p.in.count;
    double s = 0.0;
    constexpr int B = 16;  // loads in flight
    for (int64_t i0 = threadIdx.x; i0 < p.in.count; i0 += kThreads * B) {
        float u[B][1], v[B];
#pragma unroll
        for (int e = 0; e < B; ++e) {
            const int64_t i = i0 + e * kThreads;
            u[e][0] = v[e] = 0.f;
            if (i < p.in.count) {
                load_vec<1>(p.in, base + i, u[e]);
                if (p.in.v)
                    v[e] = p.in.v[base + i];
            }
        }
#pragma unroll
        for (int e = 0; e < B; ++e) {
            const int64_t i = i0 + e * kThreads;
            if (p.in.v) {
                v[e] = p.in.mu * v[e] + u[e][0];
                if (i < p.in.count)
                    p.in.v[base + i] = v[e];
                u[e][0] = p.in.nesterov ? u[e][0] + p.in.mu * v[e] : v[e];
            }
            s += (double)u[e][0] * (double)u[e][0];
        }
    }
    const double inv = inv_from(block_sum<kWaves>(s), p.eps);
    __syncthreads();
    slab<MT, VEC, kGram>(p, o, b, 0, p.chunks, 0, inv, true, st.ex[0], 0, 0, nullptr, lds);
    int k = 0;
    for (int seg = 0; seg < st.segments; ++seg) {
        const int L = st.length[seg];
        __syncthreads();
        segment<MT>(p, st, b, k, L, 1, lds, lds);
        k += L;
        __syncthreads();
        const int ep = st.ep[k - 1];
        if (seg + 1 < st.segments)
            slab<MT, VEC, kApplyGram>(p, o, b, 0, p.chunks, 0, inv, seg == 0, st.ex[seg], ep,
                                      st.ex[seg + 1], nullptr, lds);
        else
            slab<MT, VEC, kApplyOut>(p, o, b, 0, p.chunks, 0, inv, seg == 0, st.ex[seg], ep, 0,
                                     nullptr, lds);
    }
}

template <int MT, int VEC>
hipError_t launch(const NsPlan& q, const NsSmall& p, const NsSteps& st, const NsOut& o,
                  hipStream_t s)
{
    typedef Small<MT> S;
    const dim3 threads(kThreads);
    if (q.solo) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(ns_solo_kernel<MT, VEC>), dim3((unsigned)q.batch),
                           threads, 0, s, p, st, o);
        return hipGetLastError();
    }
    const dim3 slabs((unsigned)q.slabs, (unsigned)q.batch);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ns_slab_kernel<MT, VEC, kGram>), slabs, threads, 0, s, p, o,
                       1, st.ex[0], 0, 0);
    int k = 0;
    for (int seg = 0; seg < q.segments; ++seg) {
        const int L = q.length[seg];
        int parts = p.parts;
        // the one workgroup reads a part in a microsecond or two: beyond four, a
        // launch that sums them first costs less
        if (parts > 4) {
            hipLaunchKernelGGL(ns_parts_kernel,
                               dim3((unsigned)(S::LD * S::LD / 64), (unsigned)q.batch), dim3(256),
                               0, s, p.part, parts, S::LD * S::LD);
            parts = 1;
        }
        hipLaunchKernelGGL(HIP_KERNEL_NAME(ns_segment_kernel<MT>), dim3((unsigned)q.batch), threads,
                           0, s, p, st, k, L, parts);
        k += L;
        if (seg + 1 < q.segments)
            hipLaunchKernelGGL(HIP_KERNEL_NAME(ns_slab_kernel<MT, VEC, kApplyGram>), slabs, threads,
                               0, s, p, o, seg == 0, st.ex[seg], st.ep[k - 1], st.ex[seg + 1]);
        else
            hipLaunchKernelGGL(HIP_KERNEL_NAME(ns_slab_kernel<MT, VEC, kApplyOut>), slabs, threads,
                               0, s, p, o, seg == 0, st.ex[seg], st.ep[k - 1], 0);
    }
    return hipGetLastError();
}

}  // namespace

void ns_small_sizes(int m, int n, NsPlan* q)
{
    const int mt = (m + 31) / 32;
    q->chunks = (n + kChunk - 1) / kChunk;
    // everything in one launch against a launch per part, us: 32 x 300 25 / 35,
    // 64 x 128 30 / 40, 96 x 128 61 / 75, but 64 x 512 61 / 43, 128 x 512 181 / 94
    q->solo = q->chunks <= (mt == 1 ? 4 : 1);
    q->slabs = q->solo ? 1 : std::min(q->chunks, 64);
    q->parts = q->slabs;
    q->part_bytes = (size_t)q->parts * mt * mt * 4096;
    q->img_bytes = (size_t)32 * mt * (mt * 128 + 16);
    q->xs_bytes = (size_t)q->chunks * kChunk * mt * 128;
}

hipError_t launch_ns_small(const NsPlan& q, const NsInput& in, const NsArgs& x, char* ws,
                           hipStream_t s)
{
    NsSmall p{};
    p.in = in;
    p.norm = (const double*)(ws + q.off_part);
    p.norm_parts = q.norm_blocks;
    p.eps = x.eps;
    p.m = q.m;
    p.n = q.n;
    p.tall = q.tall;
    p.chunks = q.chunks;
    p.n_pad = q.chunks * kChunk;
    p.parts = q.parts;
    p.part = (float*)(ws + q.off_split);
    p.p_img = ws + q.off_mm[0];
    p.xs = (float*)(ws + q.off_xt[0]);
    NsSteps st{};
    st.a = x.a;
    st.b = x.b;
    st.c = x.c;
    st.segments = q.segments;
    st.ex[0] = (int8_t)ns_exponent(1.0);
    for (int seg = 0, k = 0; seg < q.segments; ++seg) {
        st.length[seg] = (int8_t)q.length[seg];
        for (int l = 0; l < q.length[seg]; ++l, ++k) {
            st.er[k] = (int8_t)ns_exponent(q.bound[k]);
            st.eq[k] = (int8_t)ns_exponent(q.qmax[k]);
            st.et[k] = (int8_t)ns_exponent(q.qmax[k] * q.bound[k]);
            st.ep[k] = (int8_t)ns_exponent(q.pmax[k]);
        }
        if (seg + 1 < q.segments)
            st.ex[seg + 1] = (int8_t)ns_exponent(sqrt(q.bound[k]));
    }
    NsOut o{};
    o.out_f32 = (float*)x.out;
    o.out_bf16 = x.bf16 ? (uint16_t*)x.out : nullptr;
    o.w = x.w;
    o.lr_dev = x.lr_dev;
    o.lr = x.lr;
    o.decay = x.decay;
    o.step_scale = x.step_scale;
    const bool vec = q.tall && q.m % 4 == 0;
    switch ((q.m + 31) / 32) {
    case 1:
        return vec ? launch<1, 4>(q, p, st, o, s) : launch<1, 1>(q, p, st, o, s);
    case 2:
        return vec ? launch<2, 4>(q, p, st, o, s) : launch<2, 1>(q, p, st, o, s);
    case 3:
        return vec ? launch<3, 4>(q, p, st, o, s) : launch<3, 1>(q, p, st, o, s);
    default:
        return vec ? launch<4, 4>(q, p, st, o, s) : launch<4, 1>(q, p, st, o, s);
    }
}

}  // namespace caffe_hip
