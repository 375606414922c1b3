// tile_gemm.h -- the tile product that the dense operators share (the matrix
// products of muon.hip, the 8-bit inner product of int8.hip): a workgroup
// forms a TM x TN tile of A B^T from operands whose rows are runs
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
// spread over the banks.  NS buffers; the instructions of a step carry the
// fragment reads of the next step and a share of the copies between them.
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
    typedef floatx4 acc4_t;
    static constexpr int kSteps = 2, kFrags = 2, kProds = 3;
    static constexpr int frag(int step, int f) { return step + 2 * f; }
    static constexpr int fa(int i) { return i == 2 ? 1 : 0; }
    static constexpr int fb(int i) { return i == 1 ? 1 : 0; }
    static constexpr bool low(int i) { return i % 3 != 0; }  // with a low term
    static __device__ __forceinline__ acc_t mma(u32x4 a, u32x4 b, acc_t c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a),
                                                      __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
    }
};

// The same with the whole line as one step: a small tile, with few
// instructions to a step, then has a whole stage's time for its fragment
// reads.
struct OpPairLine : OpPair {
    static constexpr int kSteps = 1, kFrags = 4, kProds = 6;
    static constexpr int frag(int, int f) { return f; }
    static constexpr int fa(int i) { return i % 3 == 2 ? i / 3 + 2 : i / 3; }
    static constexpr int fb(int i) { return i % 3 == 1 ? i / 3 + 2 : i / 3; }
};

// 8-bit integers: a line is 128 reduction elements.
struct OpInt8 {
    typedef intx16 acc_t;
    typedef intx4 acc4_t;
    static constexpr int kSteps = 4, kFrags = 1, kProds = 1;
    static constexpr int frag(int step, int) { return step; }
    static constexpr int fa(int) { return 0; }
    static constexpr int fb(int) { return 0; }
    static constexpr bool low(int) { return false; }
    static __device__ __forceinline__ acc_t mma(u32x4 a, u32x4 b, acc_t c)
    {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(intx4, a),
                                                     __builtin_bit_cast(intx4, b), c, 0, 0, 0);
    }
};

// ... the line in two steps, and in one (see OpPairLine)
struct OpInt8Half : OpInt8 {
    static constexpr int kSteps = 2, kFrags = 2, kProds = 2;
    static constexpr int frag(int step, int f) { return 2 * step + f; }
    static constexpr int fa(int i) { return i; }
    static constexpr int fb(int i) { return i; }
};
struct OpInt8Line : OpInt8 {
    static constexpr int kSteps = 1, kFrags = 4, kProds = 4;
    static constexpr int frag(int, int f) { return f; }
    static constexpr int fa(int i) { return i; }
    static constexpr int fb(int i) { return i; }
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

// s_waitcnt vmcnt(N) lgkmcnt(0): also this wave's LDS reads
template <int N>
__device__ __forceinline__ void tile_wait_lds()
{
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (((N >> 4) & 3) << 14));
}

// WM x WN waves of 32 MI x 32 NI each; LOW: products with a low term have
// accumulators of their own (kProds > 1), so that they do not round the sum.
// KW > 1: a wave forms the whole tile (WM = WN = 1) over every KW-th stage; its
// sum is the caller's to add to the others' (TileShared).
template <class Op, int WM, int WN, int MI, int NI, int NS, bool LOW, int KW = 1>
struct TileNT {
    static constexpr int NW = WM * WN;
    static_assert(KW == 1 || NW == 1, "one wave to a share of the reduction");
    static constexpr int TM = 32 * WM * MI, TN = 32 * WN * NI;
    static constexpr int kThreads = 64 * NW * KW;
    static constexpr int kMI = MI, kNI = NI;
    static constexpr int kLdsBytes = (TM + TN) * 128 * NS * KW;
    // workgroups that one compute unit's LDS holds, and with them the waves on
    // each of its four SIMDs: the register budget
    static constexpr int kPerCu = 160 * 1024 / kLdsBytes > 4 ? 4 : 160 * 1024 / kLdsBytes;
    static constexpr int kWavesPerSimd = kPerCu * NW * KW / 4;
    typedef typename Op::acc_t acc_t;

    // acc = A B^T over stages s0 .. s0 + all - 1 (all >= 1).  A points at the
    // tile's first row, a_bytes = rows in the tile * pitch (a row past it
    // reads as zeros), B likewise; TM * pitch < 2^31.
    static __device__ __forceinline__ void run(const void* A, uint32_t a_bytes, uint32_t a_pitch,
                                               const void* B, uint32_t b_bytes, uint32_t b_pitch,
                                               int s0, int all, acc_t (&acc)[MI][NI])
    {
        constexpr int NA = TM / 8 / NW, NB = TN / 8 / NW;  // copies per wave and stage
        static_assert(TM % (8 * NW) == 0 && TN % (8 * NW) == 0 && (NW == 1 || NW % 2 == 0),
                      "copy mapping");
        // one array per buffer, A's rows then B's: the compiler tells the copies
        // to one from the reads of another by the array (it follows eight)
        static_assert(NS >= 2 && NS <= 8, "buffers");
        constexpr int kBuf = (TM + TN) * 8;
        constexpr int kAll = kBuf * KW;
        __shared__ u32x4 L0[kAll], L1[kAll], L2[NS > 2 ? kAll : 1], L3[NS > 3 ? kAll : 1];
        __shared__ u32x4 L4[NS > 4 ? kAll : 1], L5[NS > 5 ? kAll : 1], L6[NS > 6 ? kAll : 1];
        __shared__ u32x4 L7[NS > 7 ? kAll : 1];

        const int lane = threadIdx.x & 63;
        const int wave_id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int kw = KW > 1 ? wave_id : 0;  // this wave's share of the stages
        const int wave = KW > 1 ? 0 : wave_id;
        const int wm = wave % WM, wn = wave / WM;
        const int nst = KW > 1 ? (all - kw + KW - 1) / KW : all;
        auto share = [&](u32x4* L, bool used) { return used ? L + kw * kBuf : L; };
        u32x4* const Lb[8] = {share(L0, true),   share(L1, true),   share(L2, NS > 2),
                              share(L3, NS > 3), share(L4, NS > 4), share(L5, NS > 5),
                              share(L6, NS > 6), share(L7, NS > 7)};

        // copy i = wave + NW q moves tile rows 8 i .. 8 i + 7; of i, line_swz
        // sees only bit 3 of the row, i's parity
        const int cr = lane >> 3;
        auto ck = [&](int q) {
            return 16u * ((lane & 7) ^ line_swz(8 * (NW == 1 ? q : wave) + cr));
        };
        uint32_t va[NA], vb[NB];
#pragma unroll
        for (int q = 0; q < NA; ++q)
            va[q] = (uint32_t)(8 * (wave + NW * q) + cr) * a_pitch + ck(q);
#pragma unroll
        for (int q = 0; q < NB; ++q)
            vb[q] = (uint32_t)(8 * (wave + NW * q) + cr) * b_pitch + ck(q);
#pragma unroll
        for (int q = 0; q < NA; ++q)
            va[q] = va[q] < a_bytes ? va[q] : kOob;
#pragma unroll
        for (int q = 0; q < NB; ++q)
            vb[q] = vb[q] < b_bytes ? vb[q] : kOob;

        // copy c of the wave's NC of stage t; past the last stage it lands zeros
        // and reads nothing, so that the number of copies in flight is known
        // everywhere (a copy in a branch made the compiler wait for all of them)
        constexpr int NC = NA + NB;
        auto copy = [&](int t, u32x4* L, int c) {
            const uint32_t soff = (uint32_t)(s0 + t * KW + kw) * 128u;
            if (c < NA)
                line_copy(make_rsrc(A, t < nst ? a_bytes : 0u), &L[(wave + NW * c) * 64], va[c],
                          soff);
            else
                line_copy(make_rsrc(B, t < nst ? b_bytes : 0u),
                          &L[TM * 8 + (wave + NW * (c - NA)) * 64], vb[c - NA], soff);
        };

        const int ra0 = wm * MI * 32 + (lane & 31);
        const int rb0 = wn * NI * 32 + (lane & 31);
        int fa[4], fb[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = 2 * j + (lane >> 5);
            fa[j] = (ra0 >> 3) * 64 + (ra0 & 7) * 8 + (c ^ line_swz(ra0));
            fb[j] = TM * 8 + (rb0 >> 3) * 64 + (rb0 & 7) * 8 + (c ^ line_swz(rb0));
        }
        constexpr int FSTR = 4 * 64;  // next 32-row block
        acc_t low[LOW ? MI : 1][LOW ? NI : 1];

        constexpr int S = Op::kSteps;
        constexpr int NR = Op::kFrags * (MI + NI);  // fragment reads of a step
        constexpr int NM = Op::kProds * MI * NI;    // instructions of a step
        // copies of a step: all at once where two buffers leave one stage's time
        constexpr int CPS = NS == 2 ? NC : (NC + S - 1) / S;
        u32x4 xa[2][Op::kFrags][MI], xb[2][Op::kFrags][NI];
        auto read = [&](const u32x4* L, int step, int r, int b) {
            const int f = r / (MI + NI), k = r % (MI + NI);
            if (k < MI)
                xa[b][f][k] = L[fa[Op::frag(step, f)] + k * FSTR];
            else
                xb[b][f][k - MI] = L[fb[Op::frag(step, f)] + (k - MI) * FSTR];
        };
        // The instructions of a step, with the next step's fragment reads
        // (from Lr) and a share of a stage's copies (part `part` of stage ct to
        // Lc) spread among them.
        auto run_step = [&](int b, int next, const u32x4* Lr, int ct, u32x4* Lc, int part) {
#pragma unroll
            for (int m = 0; m < NM; ++m) {
#pragma unroll
                for (int r = 0; r < NR; ++r)
                    if (r * (NM - NM / 4) / NR == m)
                        read(Lr, next, r, b ^ 1);
#pragma unroll
                for (int c = 0; c < CPS; ++c)
                    if (c * NM / CPS == m && part * CPS + c < NC)
                        copy(ct, Lc, part * CPS + c);
                __builtin_amdgcn_sched_barrier(0);
                const int i = m / (MI * NI), mi = m / NI % MI, ni = m % NI;
                acc_t& to = LOW && Op::low(i) ? low[LOW ? mi : 0][LOW ? ni : 0] : acc[mi][ni];
                to = Op::mma(xa[b][Op::fa(i)][mi], xb[b][Op::fb(i)][ni], to);
                __builtin_amdgcn_sched_barrier(0);
            }
        };

#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni)
                acc[mi][ni] = acc_t{};
        if constexpr (LOW) {
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int ni = 0; ni < NI; ++ni)
                    low[mi][ni] = acc_t{};
        }

        // Stage t + NS goes to stage t's buffer once every wave has read its
        // last fragments from it, before the last step of stage t: copies in
        // that step and (with more than two buffers) in the next stage's others.
        constexpr int P = NS - 1;  // (h + P) % NS: the buffer before h
#pragma unroll
        for (int t = 0; t < NS; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (t < P || CPS == NC || c < CPS)
                    copy(t, Lb[t], c);
        tile_wait<(NS - 2) * NC + CPS>();
        if constexpr (NW > 1)
            tile_barrier();
#pragma unroll
        for (int r = 0; r < NR; ++r)
            read(Lb[0], 0, r, 0);
        // whole turns of the buffers and of the two sets of fragments
        constexpr int U = NS * S % 2 ? 2 * NS : NS;
        for (int t0 = 0; t0 < nst; t0 += U) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int t = t0 + u, h = u % NS;
                if (t >= nst)
                    break;
                // the rest of stage t - 1 + NS
#pragma unroll
                for (int step = 0; step + 1 < S; ++step)
                    run_step((u * S + step) & 1, step + 1, Lb[h], t + P, Lb[(h + P) % NS],
                             step + 1);
                // stage t + 1 is there, stages t + 2 .. t + NS - 1 may be in flight
                tile_wait_lds<(NS - 2) * NC>();
                if constexpr (NW > 1)
                    tile_barrier();
                run_step((u * S + S - 1) & 1, 0, Lb[(h + 1) % NS], t + NS, Lb[h], 0);
            }
        }
        tile_wait<0>();  // no copy outlives the workgroup's LDS
        if constexpr (LOW) {
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int ni = 0; ni < NI; ++ni)
                    acc[mi][ni] += low[mi][ni];
        }
    }

    // use(q, i, j, v): v[0..3] are rows i .. i + 3 (i a multiple of 4) of column
    // j of the tile; lanes t = 0..3 of a quad hold columns j - t .. j - t + 3.
    // q = 0..3 of a 32 x 32 block follow one another, after load(q, i, j) of
    // all four.
    template <class L, class F>
    static __device__ __forceinline__ void each(const acc_t (&acc)[MI][NI], L&& load, F&& use)
    {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = wave % WM, wn = wave / WM;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                const int i = (wm * MI + mi) * 32 + 4 * (lane >> 5);
                const int j = (wn * NI + ni) * 32 + (lane & 31);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    load(q, i + 8 * q, j);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    decltype(acc[0][0][0] + acc[0][0][0]) v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = acc[mi][ni][4 * q + e];
                    use(q, i + 8 * q, j, v);
                }
                // (all blocks' addresses and loads at once would not fit)
                __builtin_amdgcn_sched_barrier(0);
            }
    }
    template <class F>
    static __device__ __forceinline__ void each(const acc_t (&acc)[MI][NI], F&& f)
    {
        each(acc, [](int, int, int) {},
             [&](int, int i, int j, auto& v) { f(i, j, v); });
    }
    // load(q, i, j) of a tile of one block to a wave, as each() calls it
    template <class L>
    static __device__ __forceinline__ void positions(L&& load)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            load(q, wave % WM * 32 + 4 * (lane >> 5) + 8 * q, wave / WM * 32 + (lane & 31));
    }
};

// A 32 x 32 tile whose reduction four waves share, a fourth of the lines each
// and no barriers between them; their sums are added in LDS in a fixed order,
// each wave left with eight rows.  For products with few tiles: a compute unit
// takes a line of a 64 x 64 tile's rows (16 KB) in 0.29 us or so, whatever the
// number of buffers, the order of reads and copies or the instructions between
// them, and four times as many units take a fourth each with half the bytes.
template <class Op, int NS, bool LOW>
struct TileShared {
    typedef TileNT<Op, 1, 1, 1, 1, NS, LOW, 4> Share;
    static constexpr int TM = 32, TN = 32, kThreads = 256, kMI = 1, kNI = 1;
    static constexpr int kWavesPerSimd = 1;
    typedef typename Op::acc4_t acc_t;

    static __device__ __forceinline__ void run(const void* A, uint32_t a_bytes, uint32_t a_pitch,
                                               const void* B, uint32_t b_bytes, uint32_t b_pitch,
                                               int s0, int all, acc_t (&acc)[1][1])
    {
        __shared__ acc_t part[4][4][64];
        typename Share::acc_t sum[1][1];
        Share::run(A, a_bytes, a_pitch, B, b_bytes, b_pitch, s0, all, sum);
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            part[wave][q][lane] = acc_t{sum[0][0][4 * q], sum[0][0][4 * q + 1],
                                        sum[0][0][4 * q + 2], sum[0][0][4 * q + 3]};
        __syncthreads();
        acc[0][0] = (part[0][wave][lane] + part[1][wave][lane]) +
                    (part[2][wave][lane] + part[3][wave][lane]);
    }
    template <class L>
    static __device__ __forceinline__ void positions(L&& load)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        load(0, 8 * wave + 4 * (lane >> 5), lane & 31);
    }
    template <class L, class F>
    static __device__ __forceinline__ void each(const acc_t (&acc)[1][1], L&& load, F&& use)
    {
        positions(load);
        positions([&](int q, int i, int j) {
            decltype(acc[0][0][0] + acc[0][0][0]) v[4] = {acc[0][0][0], acc[0][0][1],
                                                          acc[0][0][2], acc[0][0][3]};
            use(q, i, j, v);
        });
    }
    template <class F>
    static __device__ __forceinline__ void each(const acc_t (&acc)[1][1], F&& f)
    {
        each(acc, [](int, int, int) {}, [&](int, int i, int j, auto& v) { f(i, j, v); });
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
