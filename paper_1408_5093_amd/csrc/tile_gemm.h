// tile_gemm.h -- the tile product that the dense operators share (the matrix
// products of muon.hip, the 8-bit inner product of int8.hip): a workgroup of
// four waves forms a TM x TN tile of A B^T from operands whose rows are runs
// of 128-byte lines along the reduction index.
//
// One stage is one line of every operand row.  A line holds eight 16-byte
// chunks, and lane l of a 32x32 instruction takes chunk 2j + l/32 of row
// l % 32 as its fragment j (j = 0..3).  What a line means is the operand
// type's (Op below); both operands use the same order, so the order of the
// reduction index inside a line does not matter to the product.
//
// Lines go global -> LDS by 16-byte DMA, eight rows per wave copy, chunk c of
// tile row r at slot c ^ line_swz(r): fragment reads of consecutive rows then
// spread over the banks.  NS buffers: the copies of stage t + NS - 1 go out
// among the instructions of stage t.
#pragma once

#include "device_common.h"

namespace caffe_hip {

typedef int32_t intx16 __attribute__((ext_vector_type(16)));
typedef int32_t intx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));

// Two-term half-precision operands: a line is 32 reduction elements, their
// high halves in chunks 0..3 (fragments 0, 1), their low halves in chunks
// 4..7 (fragments 2, 3).  x y = xh yh + xh yl + xl yh, the product of the low
// halves (2^-22 of it) left out.
struct OpPair {
    typedef floatx16 acc_t;
    static constexpr int kSteps = 2, kFrags = 2, kProds = 3;
    static constexpr int frag(int step, int f) { return step + 2 * f; }
    static constexpr int fa(int i) { return i == 2 ? 1 : 0; }
    static constexpr int fb(int i) { return i == 1 ? 1 : 0; }
    static __device__ __forceinline__ acc_t mma(u32x4 a, u32x4 b, acc_t c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a),
                                                      __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
    }
};

// 8-bit integers: a line is 128 reduction elements.
struct OpInt8 {
    typedef intx16 acc_t;
    static constexpr int kSteps = 4, kFrags = 1, kProds = 1;
    static constexpr int frag(int step, int) { return step; }
    static constexpr int fa(int) { return 0; }
    static constexpr int fb(int) { return 0; }
    static __device__ __forceinline__ acc_t mma(u32x4 a, u32x4 b, acc_t c)
    {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(intx4, a),
                                                     __builtin_bit_cast(intx4, b), c, 0, 0, 0);
    }
};

// Slot permutation of the 8 chunks of tile row r (bits 1..3 of r), the one
// that the bf16 convolutions' 128-byte rows use.
__device__ __forceinline__ int line_swz(int r)
{
    return ((((r >> 2) ^ (r >> 3)) & 1) << 2) | (r & 2) | ((r >> 3) & 1);
}

__device__ __forceinline__ void line_copy(__amdgpu_buffer_rsrc_t r, u32x4* dst, uint32_t voff,
                                          uint32_t soff)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)dst, 16, voff, soff, 0, 0);
}

// Barrier between stages: each wave has waited for its own copies of the
// stage it reads next, and has consumed its reads of the buffer that the next
// copies overwrite (__syncthreads would also wait for the copies in flight).
__device__ __forceinline__ void tile_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int N>
__device__ __forceinline__ void tile_wait()  // s_waitcnt vmcnt(N)
{
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (((N >> 4) & 3) << 14));
}

template <class Op, int MI, int NI, int NS>
struct TileNT {
    static constexpr int TM = 64 * MI, TN = 64 * NI;  // 2 x 2 waves of 32 MI x 32 NI
    static constexpr int kLdsBytes = (TM + TN) * 128 * NS;
    // workgroups that one compute unit's LDS holds, at most the four of a full
    // register file's halves
    static constexpr int kPerCu = 160 * 1024 / kLdsBytes > 4 ? 4 : 160 * 1024 / kLdsBytes;
    typedef typename Op::acc_t acc_t;

    // acc = A B^T over stages s0 .. s0 + nst - 1 (nst >= 1).  A points at the
    // tile's first row, a_bytes = rows in the tile * pitch (a row past it
    // reads as zeros), B likewise; TM * pitch < 2^31.
    static __device__ __forceinline__ void run(const void* A, uint32_t a_bytes, uint32_t a_pitch,
                                               const void* B, uint32_t b_bytes, uint32_t b_pitch,
                                               int s0, int nst, acc_t (&acc)[MI][NI])
    {
        constexpr int NA = 2 * MI, NB = 2 * NI;  // copies per wave and stage
        __shared__ u32x4 A0[TM * 8], A1[TM * 8], A2[NS > 2 ? TM * 8 : 1];
        __shared__ u32x4 B0[TN * 8], B1[TN * 8], B2[NS > 2 ? TN * 8 : 1];
        static_assert(NS == 2 || NS == 3, "buffers");

        const int tid = threadIdx.x;
        const int lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wm = wave & 1, wn = wave >> 1;
        const __amdgpu_buffer_rsrc_t ra = make_rsrc(A, a_bytes);
        const __amdgpu_buffer_rsrc_t rb = make_rsrc(B, b_bytes);

        // copy i = wave + 4 q moves tile rows 8 i .. 8 i + 7; of i, line_swz
        // sees only bit 3 of the row, the wave's parity
        const int cr = lane >> 3;
        const uint32_t ck = 16u * ((lane & 7) ^ line_swz(8 * wave + cr));
        uint32_t va[NA], vb[NB];
#pragma unroll
        for (int q = 0; q < NA; ++q)
            va[q] = (uint32_t)(8 * (wave + 4 * q) + cr) * a_pitch + ck;
#pragma unroll
        for (int q = 0; q < NB; ++q)
            vb[q] = (uint32_t)(8 * (wave + 4 * q) + cr) * b_pitch + ck;
#pragma unroll
        for (int q = 0; q < NA; ++q)
            va[q] = va[q] < a_bytes ? va[q] : kOob;
#pragma unroll
        for (int q = 0; q < NB; ++q)
            vb[q] = vb[q] < b_bytes ? vb[q] : kOob;

        constexpr int NC = NA + NB;
        constexpr int CPP = (NC + Op::kSteps - 1) / Op::kSteps;
        auto issue_part = [&](int t, u32x4* As, u32x4* Bs, int part) {
            const uint32_t soff = (uint32_t)(s0 + t) * 128u;
#pragma unroll
            for (int c = part * CPP; c < (part + 1) * CPP && c < NC; ++c) {
                if (c < NA)
                    line_copy(ra, &As[(wave + 4 * c) * 64], va[c], soff);
                else
                    line_copy(rb, &Bs[(wave + 4 * (c - NA)) * 64], vb[c - NA], soff);
            }
        };
        auto issue = [&](int t, u32x4* As, u32x4* Bs) {
#pragma unroll
            for (int part = 0; part < Op::kSteps; ++part)
                issue_part(t, As, Bs, part);
        };

        const int ra0 = wm * MI * 32 + (lane & 31);
        const int rb0 = wn * NI * 32 + (lane & 31);
        int fa[4], fb[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = 2 * j + (lane >> 5);
            fa[j] = (ra0 >> 3) * 64 + (ra0 & 7) * 8 + (c ^ line_swz(ra0));
            fb[j] = (rb0 >> 3) * 64 + (rb0 & 7) * 8 + (c ^ line_swz(rb0));
        }
        constexpr int FSTR = 4 * 64;  // next 32-row block
        acc_t low[MI][NI];  // the products with a low term

        auto compute = [&](const u32x4* As, const u32x4* Bs, auto&& after) {
            u32x4 xa[2][Op::kFrags][MI], xb[2][Op::kFrags][NI];
            auto read = [&](int step, int b) {
#pragma unroll
                for (int f = 0; f < Op::kFrags; ++f) {
#pragma unroll
                    for (int mi = 0; mi < MI; ++mi)
                        xa[b][f][mi] = As[fa[Op::frag(step, f)] + mi * FSTR];
#pragma unroll
                    for (int ni = 0; ni < NI; ++ni)
                        xb[b][f][ni] = Bs[fb[Op::frag(step, f)] + ni * FSTR];
                }
            };
            read(0, 0);
#pragma unroll
            for (int step = 0; step < Op::kSteps; ++step) {
                const int b = step & 1;
                if (step + 1 < Op::kSteps)
                    read(step + 1, b ^ 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < Op::kProds; ++i)
#pragma unroll
                    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                        for (int ni = 0; ni < NI; ++ni) {
                            acc_t& to = i ? low[mi][ni] : acc[mi][ni];
                            to = Op::mma(xa[b][Op::fa(i)][mi], xb[b][Op::fb(i)][ni], to);
                        }
                __builtin_amdgcn_sched_barrier(0);
                after(step);
                __builtin_amdgcn_sched_barrier(0);
            }
        };

#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni)
                acc[mi][ni] = low[mi][ni] = acc_t{};

        issue(0, A0, B0);
        if (NS > 2 && nst > 1)
            issue(1, A1, B1);
        for (int t0 = 0; t0 < nst; t0 += NS) {
#pragma unroll
            for (int h = 0; h < NS; ++h) {
                const int t = t0 + h;
                if (t >= nst)
                    break;
                u32x4* Ac = h == 0 ? A0 : (h == 1 ? A1 : A2);
                u32x4* Bc = h == 0 ? B0 : (h == 1 ? B1 : B2);
                const int hn = (h + NS - 1) % NS;
                u32x4* An = hn == 0 ? A0 : (hn == 1 ? A1 : A2);
                u32x4* Bn = hn == 0 ? B0 : (hn == 1 ? B1 : B2);
                if (NS > 2 && t + 1 < nst)
                    tile_wait<NA + NB>();
                else
                    tile_wait<0>();
                tile_barrier();
                const bool more = t + NS - 1 < nst;
                compute(Ac, Bc, [&](int part) {
                    if (more)
                        issue_part(t + NS - 1, An, Bn, part);
                });
            }
        }
        if constexpr (Op::kProds > 1) {
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int ni = 0; ni < NI; ++ni)
                    acc[mi][ni] += low[mi][ni];
        }
    }

    // f(i, j, v): v[0..3] are rows i .. i + 3 (i a multiple of 4) of column j
    // of the tile; lanes t = 0..3 of a quad hold columns j - t .. j - t + 3.
    template <class F>
    static __device__ __forceinline__ void each(const acc_t (&acc)[MI][NI], F&& f)
    {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = wave & 1, wn = wave >> 1;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    decltype(acc[0][0][0] + acc[0][0][0]) v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = acc[mi][ni][4 * q + e];
                    f((wm * MI + mi) * 32 + 8 * q + 4 * (lane >> 5),
                      (wn * NI + ni) * 32 + (lane & 31), v);
                }
    }
};

// 4 x 4 transpose inside each quad of lanes: in, lane t holds column j0 + t of
// rows i .. i + 3; out, lane t holds row i + t of columns j0 .. j0 + 3.
__device__ __forceinline__ void quad_transpose(float (&v)[4])
{
    const int t = threadIdx.x & 3;
    const bool odd = t & 1, hi = t & 2;
    auto swap = [](float x, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x),
                                                                  decltype(ctrl)::value, 0xF, 0xF,
                                                                  true));
    };
    constexpr std::integral_constant<int, 0xB1> x1{};  // lanes [1, 0, 3, 2]
    constexpr std::integral_constant<int, 0x4E> x2{};  // lanes [2, 3, 0, 1]
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
        const float r = swap(odd ? v[e] : v[e + 1], x1);
        v[e] = odd ? r : v[e];
        v[e + 1] = odd ? v[e + 1] : r;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const float r = swap(hi ? v[e] : v[e + 2], x2);
        v[e] = hi ? r : v[e];
        v[e + 2] = hi ? v[e + 2] : r;
    }
}

}  // namespace caffe_hip
