// LDS-tiled MFMA GEMM for gfx950 (CDNA4):  C[M,N] = epilogue( sum_k A[m,k] * B[n,k] ).
//
// Both operands are K-contiguous ("NT"), which is exactly the operand shape of the gfx950
// 16x16 matrix instructions: every lane feeds 16 contiguous K-bytes of one row of A and of
// one row of B (v_mfma_i32_16x16x64_i8: 16 int8; v_mfma_f32_16x16x32_f16: 8 binary16).  The
// INT8 and FP16 kernels therefore move identical bytes and share one tiling:
//
//   * block tile BM x BN, K step of 128 bytes per row; WGM x WGN wavefronts, each owning a
//     (BM/WGM) x (BN/WGN) sub-tile as 16x16 accumulator fragments.  The large tile is
//     256x256 with 8 wavefronts (2 per SIMD, 128 accumulator registers each), so that one
//     wavefront's LDS reads and barrier waits hide behind the other's matrix instructions;
//   * global -> LDS with direct 16-byte loads (global_load_lds_dwordx4), bypassing the VGPRs;
//     LDS rows are 128 bytes.  The LDS of gfx950 serves a 16-byte read in groups of 16 lanes,
//     one 256-byte bank row per group, so the chunk position is XOR-swizzled with (row/2)%8
//     (applied on the global-address side of the direct load): the 16 lanes that read one
//     chunk index of 16 consecutive rows then touch 16 different 16-byte bank groups;
//   * two LDS stages: the next K step streams in while the current one feeds the matrix cores; a fragment of the next
//     64-byte K chunk is requested behind the last matrix instruction that reads its registers; one barrier per K step.
//     The 128x128 tile, while no compute unit gets a second workgroup, has three stages, or four and wavefronts of their
//     own for the loads (launch_traits);
//   * the dequantizer (scalar scales, per-column scale vector, per-column bias) runs on the
//     accumulator registers (the paper fuses dequantization at the same point: before the
//     accumulators are copied to shared memory); the B fragment is fed as the instruction's
//     first operand so that a lane holds four consecutive output columns per register quad,
//     which are packed, passed through the wavefront's private LDS slice and stored to C as
//     16-byte vectors along the rows;
//   * workgroup ids are remapped so that consecutive tiles stay on one XCD (ids are dealt
//     round-robin to the 8 XCDs, each with its own L2) and walk the tile grid in groups of
//     rows, which keeps the A and B panels of neighbouring tiles in that L2;
//   * split-K (for outputs with too few tiles to fill 256 CUs) writes raw partial
//     accumulators to a workspace; a second kernel adds them in a fixed order and applies
//     the epilogue, so results do not depend on scheduling.
#include "gemm_tile.h"

#include <cmath>

namespace qsync {

namespace {

constexpr int kPersistentLdsBytes = 159744;   // two 64 KB stages, hand-over area, column parameters

// (Two wavefronts a SIMD at least, i.e. at most 256 registers each: with more allowed the compiler keeps the accumulators in the other
// half of the register file, and moves the 64 tile's from there and back on every K tile.)
template <typename TR, int BM, int BN, int WGM, int WGN, int ST, int NL, bool SPLIT, bool CONV = false, bool TN = false>
__global__ __launch_bounds__(64 * (WGM * WGN + NL), 2) void gemm_nt_kernel(const GemmKernelArgs p)
{
    gemm_tile<TR, BM, BN, WGM, WGN, ST, NL, SPLIT, CONV, TN>(p, static_cast<int>(blockIdx.y * gridDim.x + blockIdx.x),
                                                         static_cast<int>(gridDim.y));
}

// Two independent GEMMs of one operand type in one launch, the first `na` workgroups on the first: the data and weight gradient
// of an operator.  Each of them alone leaves compute units idle unless its tiles happen to fill the chip, and pays its own
// launch, first-load latency and drain.
struct GemmPairArgs
{
    GemmKernelArgs g[2];
    int            na, total;      // workgroups of the first, of both; behind them those of the fold
    int            splits;         // K splits of the first (SPLITA)
    ColumnFoldArgs fold;
};
// (No loading wavefronts of their own here: with them 2048x1024x1024 int8 10.1 -> 10.4 us, 2056x1000x1032 binary16 24.8 -> 25.5.)
template <typename TR, int BM, int BN, int WGM, int WGN, int ST, bool TNA, bool SPLITA>
__global__ __launch_bounds__(64 * WGM * WGN, 2) void gemm_nt_pair_kernel(const GemmPairArgs p)
{
    const int blk = static_cast<int>(blockIdx.x);
    if(blk >= p.total)
    {
        extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
        fold_columns(p.fold, static_cast<uint32_t>(blk - p.total), reinterpret_cast<float*>(lds));
        return;
    }
    if constexpr(!TNA && !SPLITA)
        gemm_tile<TR, BM, BN, WGM, WGN, ST, 0, false, false, false>(p.g[blk < p.na ? 0 : 1], blk < p.na ? blk : blk - p.na, 1);
    else if constexpr(!TNA)
        gemm_tile<TR, BM, BN, WGM, WGN, ST, 0, true, false, false, true>(p.g[blk < p.na ? 0 : 1], blk < p.na ? blk : blk - p.na, blk < p.na ? p.splits : 1, blk < p.na);
    else if(blk < p.na)
        gemm_tile<TR, BM, BN, WGM, WGN, ST, 0, SPLITA, false, TNA>(p.g[0], blk, p.splits);
    else
        gemm_tile<TR, BM, BN, WGM, WGN, ST, 0, false, false, false>(p.g[1], blk - p.na, 1);
}

// ---------------------------------------------------------------------------------------------------------------
// Persistent variant of the 256x256 kernel for binary16 outputs whose M, N are multiples of 256 and whose operand
// rows are multiples of two K tiles.  One workgroup per compute unit walks its tiles; three things differ from
// gemm_nt_kernel:
//   * the wavefronts split the vector-memory roles.  Loads and stores of a wavefront share one in-flight counter
//     that retires in issue order, so a wavefront that has just stored its part of C cannot see a later load
//     land before those stores have reached the cache, microseconds later.  Wavefronts 0-3 (one per SIMD, the
//     upper half of the tile) therefore issue every direct global->LDS load and never store; wavefronts 4-7 (the
//     lower half) issue every store of C and never load.  The loaders pass their dequantized half through LDS;
//   * the next tile's first K tile is requested while the last K tile of the current one is still being
//     multiplied (its stage is free by then), the second one as soon as the storers have drained the hand-over
//     area (which is the other stage plus the spare LDS behind the stages); nobody waits for a store, so the
//     write-back of a tile overlaps the next tile's K loop;
//   * barriers are bare s_barrier instructions behind an LDS wait (the compiler's __syncthreads would wait for
//     every vector-memory operation of the wavefront, stores included), and every LDS access behind the first
//     store is written as an instruction for the same reason.
__device__ __forceinline__ void wait_lds_all() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); __builtin_amdgcn_sched_barrier(0); }
// LDS accesses as instructions; OFF is the instruction's immediate byte offset (16 bits)
template <int OFF> __device__ __forceinline__ void lds_write_b64(uint32_t addr, const v2u32& v)
{
    static_assert(OFF >= 0 && OFF < 65536, "immediate offset");
    asm volatile("ds_write_b64 %0, %1 offset:%2" ::"v"(addr), "v"(v), "n"(OFF) : "memory");
}
template <int OFF> __device__ __forceinline__ void lds_read_b128(v4u32& d, uint32_t addr)
{
    static_assert(OFF >= 0 && OFF < 65536, "immediate offset");
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(d) : "v"(addr), "n"(OFF) : "memory");
}
// bit patterns by value (a vector element is not an object a bit cast could be applied to directly)
template <typename T> __device__ __forceinline__ T word_as(uint32_t u);
template <> __device__ __forceinline__ int32_t word_as<int32_t>(uint32_t u) { return static_cast<int32_t>(u); }
template <> __device__ __forceinline__ float   word_as<float>(uint32_t u) { return __uint_as_float(u); }
__device__ __forceinline__ uint32_t as_word(int32_t v) { return static_cast<uint32_t>(v); }
__device__ __forceinline__ uint32_t as_word(float v) { return __float_as_uint(v); }

template <typename TR>
__global__ __launch_bounds__(512) void gemm_nt_persistent_kernel(const GemmKernelArgs p, const int total_tiles)
{
    typedef typename TR::accv_t accv_t;
    constexpr int BM = 256, BN = 256, WGN = 4, WTM = 128, WTN = 64, R = TR::kRows, FM = WTM / R, FN = WTN / R;
    static_assert(R == 16, "fragments of a wavefront");
    constexpr int STAGE_BYTES = (BM + BN) * kRowBytes;        // 64 KB
    constexpr int DPW         = 16;                           // direct loads per loader wavefront and K tile
    constexpr int PITCH       = WTN * 2 + 16;                 // padded row of 64 binary16 outputs in the hand-over area
    constexpr int L_STG       = WTM * PITCH;                  // a loader's whole sub-tile
    constexpr int S_STG       = 32 * PITCH;                   // a storer's private slice: 32 rows, two of fragments
    constexpr int STG_BASE    = STAGE_BYTES;                  // the hand-over area starts where stage 1 starts
    constexpr int S_BASE      = STG_BASE + 4 * L_STG;
    constexpr int COLP_BASE   = S_BASE + 4 * S_STG;           // [2][BN] floats: alpha * column scale, column bias
    static_assert(COLP_BASE + 2 * BN * 4 <= kPersistentLdsBytes, "LDS layout");

    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)lds));
    const int  tid = threadIdx.x, lane = tid % kWaveSize;
    const int  wave = __builtin_amdgcn_readfirstlane(tid / kWaveSize);
    const int  wm = wave / WGN, wn = wave % WGN;
    const bool loader = wave < 4;                              // uniform per wavefront
    const int  KT = static_cast<int>(p.Kb / kRowBytes);        // even, >= 2 (checked by the launcher)
    const int  G  = static_cast<int>(gridDim.x);

    // ---- loader set-up: wavefront l covers stage rows [128 l, 128 l + 128): l = 0, 1 rows of A, l = 2, 3 rows of B
    const int  lw   = wave & 3;
    const bool is_a = lw < 2;
    uint32_t   voff[DPW];
    {
        int imm[DPW];
        fill_dma_imms<DPW>(imm, std::make_integer_sequence<int, DPW>{});
#pragma unroll
        for(int d = 0; d < DPW; ++d)
        {
            const int srow  = (lw * DPW + d) * 8 + lane / 8;
            const int chunk = (lane % 8) ^ ((srow >> 1) & 7);
            const int lrow  = srow - (is_a ? 0 : BM);
            voff[d] = static_cast<uint32_t>(static_cast<int64_t>(lrow) * p.Kb + chunk * 16 + kDmaBias - imm[d]);
        }
    }
    auto panel_base = [&](int tm, int tn) -> const uint8_t* {
        const uint8_t* g = is_a ? p.A + static_cast<int64_t>(tm) * BM * p.Kb : p.B + static_cast<int64_t>(tn) * BN * p.Kb;
        const uint64_t bits = reinterpret_cast<uint64_t>(g) - kDmaBias;
        const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<uint32_t>(bits))));
        const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<uint32_t>(bits >> 32))));
        return reinterpret_cast<const uint8_t*>((static_cast<uint64_t>(hi) << 32) | static_cast<uint64_t>(lo));
    };
    auto dma = [&](int stage, const uint8_t* sbase, int kt) {
        const uint8_t* sb    = sbase + static_cast<int64_t>(kt) * kRowBytes;
        uint8_t*       lbase = lds + stage * STAGE_BYTES + lw * (DPW * 1024) + (dma_group<DPW>() / 2) * 1024;
        asm volatile("" : "+s"(sb));
        dma_sequence<DPW>(std::make_integer_sequence<int, DPW>{}, sb, voff, lbase);
    };
    auto park_column_parameters = [&](int tn) {               // threads 0..255 are exactly the loaders
        float alpha = 1.0f;
        if(p.s0) alpha *= *p.s0;
        if(p.s1) alpha *= *p.s1;
        const int64_t col = static_cast<int64_t>(tn) * BN + tid;
        const float   sc  = alpha * (p.col_scale ? p.col_scale[col] : 1.0f);
        const float   bi  = p.col_bias ? p.col_bias[col] : 0.0f;
        lds_write_b32(lds0 + COLP_BASE + tid * 4, __float_as_uint(sc));
        lds_write_b32(lds0 + COLP_BASE + (BN + tid) * 4, __float_as_uint(bi));
    };

    // ---- fragment reads (as in gemm_nt_kernel, but one set of registers for the columns too: there are none left for two)
    const int frag_row = lane % R, kq = lane / R;
    int       roff[2];
#pragma unroll
    for(int c = 0; c < 2; ++c) roff[c] = frag_row * kRowBytes + swizzle(frag_row, c * 4 + kq);
    const int a_base = (wm * WTM) * kRowBytes, b_base = BM * kRowBytes + (wn * WTN) * kRowBytes;
    v4i32     af[FM], bf[FN];
    auto      read_a = [&](auto ft, int stage, int c) {
        frag_read<decltype(ft)::value * R * kRowBytes>(af[decltype(ft)::value], lds0 + static_cast<uint32_t>(stage * STAGE_BYTES + a_base + roff[c]));
    };
    auto read_b = [&](auto ft, int stage, int c) {
        frag_read<decltype(ft)::value * R * kRowBytes>(bf[decltype(ft)::value], lds0 + static_cast<uint32_t>(stage * STAGE_BYTES + b_base + roff[c]));
    };
    accv_t acc[FM][FN];
    auto   mma = [&](auto ft) {
        constexpr int f = decltype(ft)::value;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for(int j = 0; j < FN; ++j) acc[f][j] = TR::mfma(bf[j], af[f], acc[f][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // the last row of a chunk, and the next chunk's columns behind it
    const std::integral_constant<int, FM - 1> last_row{};
    auto turn = [&](int stage, int c) {
        mma(last_row);
        static_for<FN>([&](auto j) { read_b(j, stage, c); });
        read_a(last_row, stage, c);
    };
    auto clear_acc = [&]() {
#pragma unroll
        for(int i = 0; i < FM; ++i)
#pragma unroll
            for(int j = 0; j < FN; ++j)
#pragma unroll
                for(int v = 0; v < 4; ++v) acc[i][j][v] = 0;
    };

    // ---- first tile: both stages requested, column parameters parked, first K tile awaited
    int lin = static_cast<int>(blockIdx.x);
    int split_unused, tm, tn;
    item_of_block(lin, p.tiles_m, p.tiles_n, 1, p.group_m, split_unused, tm, tn);
    const uint8_t* cur = panel_base(tm, tn);
    if(loader)
    {
        dma(0, cur, 0);
        dma(1, cur, 1);
        park_column_parameters(tn);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    wg_barrier();

    while(true)
    {
        __builtin_amdgcn_sched_barrier(0);     // the accumulators' live range starts here, not before the last tile's stores
        clear_acc();
        const int  nlin     = lin + G;
        const bool has_next = nlin < total_tiles;
        int        ntm = 0, ntn = 0;
        if(has_next) item_of_block(nlin, p.tiles_m, p.tiles_n, 1, p.group_m, split_unused, ntm, ntn);
        const uint8_t* nxt = has_next ? panel_base(ntm, ntn) : cur;

        // ---- K loop.  On entry K tile 0 is in stage 0 and published, K tile 1 is in flight towards stage 1.
        static_for<FN>([&](auto j) { read_b(j, 0, 0); });
        static_for<FM>([&](auto i) { read_a(i, 0, 0); });
        for(int kt = 0; kt < KT; ++kt)
        {
            const int stage = kt & 1;
            // chunk 0: younger than the fragment of row i are those of the FM - 1 other rows, less than the rows requested last
            // behind the columns
            static_for<FM - 1>([&](auto it) {
                if constexpr(decltype(it)::value == 0) wait_lds<1>();
                else                                   wait_lds<FM - 1>();
                mma(it);
                read_a(it, stage, 1);
            });
            wait_lds<FM - 1>();
            turn(stage, 1);
            static_for<FM / 2>([&](auto it) {
                wait_lds<1>();
                mma(it);
            });
            wait_lds<0>();
            const bool more = kt + 1 < KT;
            if(more)
            {
                // the loaders' K tile kt+1 has landed, everybody's reads of this stage have returned
                if(loader) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                wg_barrier();
                if(loader)
                {
                    if(kt + 2 < KT) dma(stage, cur, kt + 2);
                    else if(has_next) dma(stage, nxt, 0);        // kt + 2 == KT: stage 0, first K tile of the next tile
                }
            }
            // on the last K tile the reads below fetch chunk 0 of the current stage again: in bounds, unused
            const int nstage = more ? (stage ^ 1) : stage;
            static_for<FM / 2>([&](auto it) { read_a(it, nstage, 0); });
            static_for<FM / 2 - 1>([&](auto it) {
                const std::integral_constant<int, FM / 2 + decltype(it)::value> row{};
                mma(row);
                read_a(row, nstage, 0);
            });
            turn(nstage, 0);
        }
        wait_lds<0>();
#pragma unroll
        for(int f = 0; f < FM; ++f) asm volatile("" : "+v"(af[f]));
#pragma unroll
        for(int f = 0; f < FN; ++f) asm volatile("" : "+v"(bf[f]));

        // ---- epilogue.  Stage 1 (last K tile) is drained once everybody passes this barrier.
        wg_barrier();
        const int64_t m0 = static_cast<int64_t>(tm) * BM, n0 = static_cast<int64_t>(tn) * BN;
        // where this wavefront's dequantized rows go: a loader fills its whole 128-row region, a storer its
        // private 32-row slice, pass by pass (the storer's base steps back by one pass per pass, so that both
        // use the same immediates)
        const uint32_t my_stg  = lds0 + (loader ? STG_BASE + wave * L_STG : S_BASE + (wave - 4) * S_STG);
        const uint32_t wr_lane = my_stg + static_cast<uint32_t>(frag_row * PITCH + 8 * kq);
        const uint32_t cp_lane = lds0 + COLP_BASE + static_cast<uint32_t>((wn * WTN + 4 * kq) * 4);
        const int      lr8 = lane / 8, seg = lane % 8;
        const uint32_t rd_lane = static_cast<uint32_t>(lr8 * PITCH + seg * 16);
        const int64_t  wcol0 = n0 + wn * WTN;
        __half* const  cbase = static_cast<__half*>(p.C) + wcol0 + seg * 8;
        // alpha * column scale and bias of this lane's 4 x 4 columns, read once per tile
        v4u32 rs[FN], rb[FN];
        static_for<FN>([&](auto jt) {
            constexpr int j = decltype(jt)::value;
            lds_read_b128<j * R * 4>(rs[j], cp_lane);
            lds_read_b128<(BN + j * R) * 4>(rb[j], cp_lane);
        });
        wait_lds_all();
        static_for<WTM / 32>([&](auto it) {                     // 32 rows a pass
            constexpr int  i       = decltype(it)::value;
            const uint32_t wr_base = loader ? wr_lane : wr_lane - static_cast<uint32_t>(i * 32 * PITCH);
            static_for<32 / R>([&](auto ht) {
                constexpr int f = i * (32 / R) + decltype(ht)::value;
                static_for<FN>([&](auto jt) {
                    constexpr int j = decltype(jt)::value;
                    // the per-tile kernel's arithmetic: each value one fused multiply-add rounded once to binary16
                    auto pair = [&](int e) {
                        return fma_out_half2(static_cast<float>(acc[f][j][e]), __uint_as_float(rs[j][e]), __uint_as_float(rb[j][e]),
                                             static_cast<float>(acc[f][j][e + 1]), __uint_as_float(rs[j][e + 1]),
                                             __uint_as_float(rb[j][e + 1]));
                    };
                    const v2u32 packed = {pair(0), pair(2)};
                    lds_write_b64<f * R * PITCH + j * R * 2>(wr_base, packed);
                });
            });
            if(!loader)
            {   // the storer's own rows leave right away: written by this wavefront, read back transposed
                wait_lds_all();
                v4u32 val[4];
                static_for<4>([&](auto qt) { lds_read_b128<decltype(qt)::value * 8 * PITCH>(val[decltype(qt)::value], my_stg + rd_lane); });
                wait_lds_all();
#pragma unroll
                for(int q = 0; q < 4; ++q)
                {
                    const int64_t row = m0 + WTM + i * 32 + q * 8 + lr8;
                    __builtin_nontemporal_store(val[q], reinterpret_cast<v4u32*>(cbase + row * p.N));
                }
            }
        });
        wg_barrier();                                        // the loaders' rows are in the hand-over area
        // The storers take the partner's sub-tile (same columns, the upper half of the tile) out of the hand-over
        // area into registers, so that the area is free again after one more barrier and the loaders' request for
        // the next tile's second K tile enters the memory pipeline ahead of the stores that follow.
        // (The 64 registers are those of the accumulators, dead by now: a separate array would raise the kernel's
        // register demand and the compiler would spill the results of the LDS instructions before they arrive.)
        if(!loader)
        {
            const uint32_t src = lds0 + STG_BASE + static_cast<uint32_t>((wave - 4) * L_STG) + rd_lane;
            static_for<2>([&](auto bt) {                       // two batches: the LDS counter of a wavefront holds 15
                constexpr int b = decltype(bt)::value;
                v4u32 t[8];
                static_for<8>([&](auto rt) { lds_read_b128<(b * 8 + decltype(rt)::value) * 8 * PITCH>(t[decltype(rt)::value], src); });
                wait_lds_all();
                static_for<8>([&](auto rt) {
                    constexpr int r = b * 8 + decltype(rt)::value;
#pragma unroll
                    for(int e = 0; e < 4; ++e)
                        {
                        const uint32_t word = t[decltype(rt)::value][e];
                        acc[r / 4][r % 4][e] = word_as<typename TR::acc_t>(word);
                    }
                });
            });
        }
        if(loader && has_next)
        {
            park_column_parameters(ntn);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the next tile's first K tile has landed
        }
        wg_barrier();                                        // hand-over area drained, stage 0 and parameters published
        if(loader && has_next) dma(1, nxt, 1);
        if(!loader)
        {
#pragma unroll
            for(int r = 0; r < 16; ++r)
            {
                const int64_t row = m0 + r * 8 + lr8;
                v4u32         val;
#pragma unroll
                for(int e = 0; e < 4; ++e)
                {
                    const typename TR::acc_t a = acc[r / 4][r % 4][e];
                    val[e] = as_word(a);
                }
                __builtin_nontemporal_store(val, reinterpret_cast<v4u32*>(cbase + row * p.N));
            }
        }
        if(!has_next) break;
        lin = nlin; tm = ntm; tn = ntn; cur = nxt;
    }
}


// Adds the split-K partials in split order and applies the epilogue.
constexpr int kThreads = 256;   // split-K reduction

template <typename ACC, bool VEC4>
__global__ __launch_bounds__(kThreads) void splitk_reduce_kernel(const ACC* __restrict__ partial, int splits,
                                                                 int64_t M, int64_t N, void* C, int c_is_f16,
                                                                 const float* s0, const float* s1,
                                                                 const float* __restrict__ col_scale,
                                                                 const float* __restrict__ col_bias, int32_t* acc_dump,
                                                                 unsigned int* amax_bits, int8_t* codes,
                                                                 const float* code_inv_p, int code_qmax, const int blocks,
                                                                 const ColumnFoldArgs fold)
{
    if(static_cast<int>(blockIdx.x) >= blocks)      // workgroups behind the reduction's own: column sums of some other tensor
    {
        __shared__ float lds_f[kThreads];
        fold_columns(fold, blockIdx.x - blocks, lds_f);
        return;
    }
    const float code_inv = codes ? *code_inv_p : 0.0f;
    constexpr int V      = VEC4 ? 4 : 1;       // VEC4: N % 4 == 0 and 16-byte aligned buffers
    uint32_t      run    = 0u;                 // maximum of |C| as stored (fp32 bits), when amax_bits is given
    const uint32_t seen  = amax_bits ? __hip_atomic_load(amax_bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
    const int64_t n      = M * N;
    const int64_t stride = static_cast<int64_t>(blocks) * kThreads * V;
    float         alpha  = 1.0f;
    if(s0) alpha *= *s0;
    if(s1) alpha *= *s1;
    for(int64_t i = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * V; i < n; i += stride)
    {
        ACC acc[V];
#pragma unroll
        for(int e = 0; e < V; ++e) acc[e] = 0;
#pragma unroll 8                                  // eight independent partial loads in flight; the sum keeps its order
        for(int s = 0; s < splits; ++s)
        {
            ACC part[V];
            if(VEC4)
                *reinterpret_cast<uint4*>(part) = *reinterpret_cast<const uint4*>(partial + static_cast<int64_t>(s) * n + i);
            else
                part[0] = partial[static_cast<int64_t>(s) * n + i];
#pragma unroll
            for(int e = 0; e < V; ++e) acc[e] += part[e];
        }
        const int64_t col = i % N;
        float         y[V];
#pragma unroll
        for(int e = 0; e < V; ++e)
        {
            const float f = alpha * (col_scale ? col_scale[col + e] : 1.0f), b = col_bias ? col_bias[col + e] : 0.0f;
            const float a = static_cast<float>(acc[e]);
            y[e] = c_is_f16 ? __half2float(fma_out<__half>(a, f, b)) : fma_out<float>(a, f, b);      // the value as stored
        }
        if(amax_bits)
        {
#pragma unroll
            for(int e = 0; e < V; ++e)
            {
                const uint32_t u = __float_as_uint(y[e]) & 0x7FFFFFFFu;
                run = run > u ? run : u;
            }
        }
        if(codes)
        {   // codes of the values as stored (y holds the rounded value when the output is binary16)
            uint32_t cw = 0u;
#pragma unroll
            for(int e = 0; e < V; ++e)
                cw |= (static_cast<uint32_t>(quantize_code<kNearest>(y[e], code_inv, code_qmax, 0u)) & 0xFFu) << (8 * e);
            if(VEC4 && (reinterpret_cast<uintptr_t>(codes) & 3) == 0)
                *reinterpret_cast<uint32_t*>(codes + i) = cw;
            else
#pragma unroll
                for(int e = 0; e < V; ++e) codes[i + e] = static_cast<int8_t>((cw >> (8 * e)) & 0xFFu);
        }
        if(VEC4)
        {
            if(c_is_f16)
            {
                __half h[4];
#pragma unroll
                for(int e = 0; e < 4; ++e) h[e] = __float2half_rn(y[e]);      // exact: y is a binary16 value
                *reinterpret_cast<uint2*>(static_cast<__half*>(C) + i) = *reinterpret_cast<const uint2*>(h);
            }
            else
                *reinterpret_cast<uint4*>(static_cast<float*>(C) + i) = *reinterpret_cast<const uint4*>(y);
        }
        else if(c_is_f16)
            static_cast<__half*>(C)[i] = __float2half_rn(y[0]);
        else
            static_cast<float*>(C)[i] = y[0];
        if(acc_dump)
#pragma unroll
            for(int e = 0; e < V; ++e) acc_dump[i + e] = static_cast<int32_t>(acc[e]);
    }
    if(amax_bits)
    {   // one atomic maximum per workgroup
        __shared__ uint32_t slots[kThreads / 64];
#pragma unroll
        for(int off = 32; off >= 1; off >>= 1)
        {
            const uint32_t o = static_cast<uint32_t>(__shfl_xor(static_cast<int>(run), off));
            run = run > o ? run : o;
        }
        if(threadIdx.x % 64 == 0) slots[threadIdx.x / 64] = run;
        __syncthreads();
        if(threadIdx.x == 0)
        {
            uint32_t m = slots[0];
#pragma unroll
            for(int w = 1; w < kThreads / 64; ++w) m = m > slots[w] ? m : slots[w];
            if(m > seen) atomicMax(amax_bits, m);      // `seen` may be stale but never too large: skipping is safe
        }
    }
}

// 0: 256x256, 8 wavefronts (2x4, 128x64 each)   1: 128x128, 8 wavefronts (2x4, 64x32 each)
// 2: 64x64, 4 wavefronts (2x2, 32x32 each)
// (What follows was measured on 32x32 instructions.)
// (128x128 with four wavefronts of 64x64, one per SIMD, reads a third less LDS per operation but has nobody to issue
//  matrix instructions while it queues direct loads.  Four -> eight wavefronts: 4096x768x3072 int8 18.1 -> 16.2 us,
//  3072x768x4096 20.4 -> 18.2, 2056x1000x1032 binary16 14.0 -> 12.5, 64x128x128 4.7 -> 3.9.)
// (256x256 with 4 wavefronts of 128x128 -- a third fewer LDS fragment reads per matrix instruction, 256
//  accumulator registers per lane -- needs matrix instructions written as inline assembly on accumulator
//  registers, one loop body without branches around them, and fragment reads and direct loads placed one by one
//  between them; the compiler's own allocation keeps the accumulators in scratch memory.  Built that way it is
//  bit-identical and as fast as the 8-wavefront tile at 8192^3 but 7-14 % slower on 16384x4096x1024 and
//  16384x1024x4096, where its longer epilogue counts: not kept.)
constexpr TileShape kTiles[] = {{256, 256}, {128, 128}, {64, 64}};
constexpr int       kNumTiles = sizeof(kTiles) / sizeof(kTiles[0]);

// The dynamic-LDS attribute of a kernel is set once per device: flags indexed by the current device (a process
// that drives several GPUs sets it on each; beyond kMaxDevices it is set before every launch).
constexpr int kMaxDevices = 16;
inline int current_device_slot()
{
    int dev = 0;
    return (hipGetDevice(&dev) == hipSuccess && dev >= 0 && dev < kMaxDevices) ? dev : -1;
}

template <typename TR, int BM, int BN, int WGM, int WGN, int ST, int NL>
hipError_t launch_tile(const GemmKernelArgs& a, int splits, hipStream_t st, bool tn = false)
{
    constexpr size_t lds_bytes = ST * static_cast<size_t>(BM + BN) * kRowBytes + 2 * BN * sizeof(float) + 64;   // + amax slots
    auto go = [&](auto split, auto conv, auto rowmajor) {
        const auto  kernel = &gemm_nt_kernel<TR, BM, BN, WGM, WGN, ST, NL, decltype(split)::value, decltype(conv)::value, decltype(rowmajor)::value>;
        static bool attr_set[kMaxDevices] = {};   // per instantiation and device; benign if set twice
        const int   slot = current_device_slot();
        if(slot < 0 || !attr_set[slot])
        {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                     static_cast<int>(lds_bytes));
            if(e != hipSuccess) return e;
            if(slot >= 0) attr_set[slot] = true;
        }
        kernel<<<dim3(static_cast<unsigned>(a.tiles_m * a.tiles_n), static_cast<unsigned>(splits)), dim3(64 * (WGM * WGN + NL)), lds_bytes, st>>>(a);
        return hipGetLastError();
    };
    constexpr std::true_type  yes{};
    constexpr std::false_type no{};
    if constexpr(TR::kElemBytes <= 2 && NL == 0)
    {
        if(a.conv_H > 0 && tn) return splits > 1 ? go(yes, yes, yes) : go(no, yes, yes);
        if(a.conv_H > 0 && splits == 1) return go(no, yes, no);
    }
    if(a.conv_H > 0) return hipErrorInvalidValue;
    if constexpr(TR::kElemBytes <= 2)
        if(tn) return splits > 1 ? go(yes, no, yes) : go(no, no, yes);
    if(tn) return hipErrorInvalidValue;
    return splits > 1 ? go(yes, no, no) : go(no, no, no);
}

template <typename TR>
hipError_t launch_traits(int tile, const GemmKernelArgs& a, int splits, hipStream_t st, bool tn = false)
{
    // The 128x128 tile where every compute unit gets one workgroup at most (with a second one resident, two stages,
    // its K loop fills the gaps):
    //   four stages and four loading wavefronts, three stages -> this, us: 4096x768x3072 (192 workgroups) int8 16.4 -> 14.6,
    //   binary16 25.1 -> 22.6; 2048x2048x1536 int8 9.9 -> 9.3, 1024x512x2048 10.5 -> 9.6.
    //   Their start costs 0.3 us, a K tile less gains 0.05 to 0.12: 8 K tiles int8 7.33 -> 7.30, 6 lose (7.6 -> 7.8), 2 lose 5 %.
    //   Contiguous rows that straddle the 128-byte lines (two lines a piece) keep the loaders the bound: 4096x768x3088 int8 18.4 ->
    //   18.9.  A row-major stage row is 128 or 256 bytes of a longer operand row, for which that matters less: they take any row length.
    //   Whole lines 2048x1024x1024 12.8 -> 11.7, 4096x768x3072 int8 21.7 -> 18.8; others 1536x1344x1792 int8 11.1 -> 10.6, binary16
    //   1408x576x3640 17.1 -> 15.7, 1792x480x816 14.2 -> 13.8 (over 179 row-major products 0.83 to 1.04 of three stages, on average 0.96).
    //   The gathering loads of a convolution have too much arithmetic for four wavefronts (24.9 -> 28.2).
    //   three stages otherwise.  The rest was measured on 32x32 instructions.  Two -> three: 4096x768x3072 int8 18.5 -> 15.3 us,
    //   binary16 33.5 -> 26.4; 2048x2048x4096 (256) int8 25.8 -> 22.5; a short contraction gains nothing (4096x768x768 int8 6.8 -> 7.0).
    // Beyond 256 workgroups a third stage loses: 2176x2048x1024 (272) int8 10.9 -> 14.2, binary16 17.6 -> 21.8; 4096x2048x3072
    // (512) int8 29.9 -> 34.2, 4096x3072x768 (768) 15.5 -> 18.9.
    // The 64x64 tile gains nothing from 3, 4 or 8 stages (14.7 / 16.4 / 17.3 / 23.9 us on 2056x1000x1032 binary16), nor
    // from fragments read a whole K tile ahead (14.7).
    const int64_t workgroups = static_cast<int64_t>(a.tiles_m) * a.tiles_n * splits;
    switch(tile)
    {
    case 0: return launch_tile<TR, 256, 256, 2, 4, 2, 0>(a, splits, st, tn);
    case 1:
        if(workgroups > kNumCu) return launch_tile<TR, 128, 128, 2, 4, 2, 0>(a, splits, st, tn);
        return a.conv_H == 0 && a.remap_C == 0 && a.ktiles_per_split >= 8 && (tn || a.Kb % kRowBytes == 0)
                 ? launch_tile<TR, 128, 128, 2, 4, 4, 4>(a, splits, st, tn)
                 : launch_tile<TR, 128, 128, 2, 4, 3, 0>(a, splits, st, tn);
    default: return launch_tile<TR, 64, 64, 2, 2, 2, 0>(a, splits, st, tn);
    }
}

template <typename TR, int BM, int BN, int WGM, int WGN, int ST, bool TNA, bool SPLITA>
hipError_t launch_pair_tile(const GemmPairArgs& p, hipStream_t st)
{
    constexpr size_t lds_bytes = ST * static_cast<size_t>(BM + BN) * kRowBytes + 2 * BN * sizeof(float) + 64;
    const auto       kernel = &gemm_nt_pair_kernel<TR, BM, BN, WGM, WGN, ST, TNA, SPLITA>;
    static bool      attr_set[kMaxDevices] = {};      // per instantiation and device; benign if set twice
    const int        slot = current_device_slot();
    if(slot < 0 || !attr_set[slot])
    {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds_bytes));
        if(e != hipSuccess) return e;
        if(slot >= 0) attr_set[slot] = true;
    }
    kernel<<<dim3(static_cast<unsigned>(p.total + p.fold.blocks())), dim3(64 * WGM * WGN), lds_bytes, st>>>(p);
    return hipGetLastError();
}
template <typename TR, bool TNA, bool SPLITA>
hipError_t launch_pair_traits(int tile, const GemmPairArgs& p, hipStream_t st)
{
    if(tile == 1)
        return p.total <= kNumCu ? launch_pair_tile<TR, 128, 128, 2, 4, 3, TNA, SPLITA>(p, st)
                                 : launch_pair_tile<TR, 128, 128, 2, 4, 2, TNA, SPLITA>(p, st);
    return launch_pair_tile<TR, 64, 64, 2, 2, 2, TNA, SPLITA>(p, st);
}

// The persistent kernel serves full 256x256 tiles with binary16 output and nothing optional in the epilogue.
bool persistent_eligible(const GemmKernelArgs& a, int prec, int tile, int splits)
{
    return (prec == 8 || prec == 16) && tile == 0 && splits == 1 && a.c_is_f16 && !a.acc_dump && !a.amax_bits && !a.codes && a.conv_H == 0
        && a.remap_C == 0 && a.M % 256 == 0 && a.N % 256 == 0 && a.Kb % (2 * kRowBytes) == 0 && a.Kb >= 2 * kRowBytes
        && (reinterpret_cast<uintptr_t>(a.C) & 15) == 0;
}

template <typename TR> hipError_t launch_persistent(const GemmKernelArgs& a, hipStream_t st)
{
    static bool      attr_set[kMaxDevices] = {};      // per instantiation and device; benign if set twice
    const int        slot = current_device_slot();
    const void*      fn = reinterpret_cast<const void*>(&gemm_nt_persistent_kernel<TR>);
    if(slot < 0 || !attr_set[slot])
    {
        const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, kPersistentLdsBytes);
        if(e != hipSuccess) return e;
        if(slot >= 0) attr_set[slot] = true;
    }
    const int total = a.tiles_m * a.tiles_n;
    const int grid  = total < kNumCu ? total : kNumCu;
    gemm_nt_persistent_kernel<TR><<<dim3(static_cast<unsigned>(grid)), dim3(512), kPersistentLdsBytes, st>>>(a, total);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_f32(const GemmProblem& p, const GemmPlan& plan, void* workspace, hipStream_t stream);   // gemm_f32.hip

static thread_local int g_tile_override = -1;     // set by tests and tuning runs only; per calling thread
void set_gemm_tile_override(int tile) { g_tile_override = (tile >= 0 && tile < kNumTiles) ? tile : -1; }
bool gemm_tile_pinned() { return g_tile_override >= 0; }
static thread_local int g_persistent_mode = -1;   // 1: whenever eligible; anything else: never (the default, see launch_gemm)
void set_gemm_persistent_mode(int mode) { g_persistent_mode = (mode == 0 || mode == 1) ? mode : -1; }

// fp32 operands: 0 is 256x128 (gemm_f32.hip)
TileShape gemm_tile_shape(int prec, int tile) { return prec == 32 && tile == 0 ? TileShape{256, 128} : kTiles[tile]; }

// Model of a tile shape's time; the constants are explained in plan_gemm.
struct TileModel { double r1, rmax, ovh, cap; int occ; };
static constexpr TileModel kTileModel[kNumTiles] = {{14.0, 15.8, 7.5, 2280.0, 1}, {8.3, 9.0, 4.2, 1900.0, 2}, {3.55, 5.48, 3.2, 2060.0, 4}};
// fp32: an LDS stage of three bf16 parts leaves room for one workgroup of the larger tiles on a unit, three of the small one.  Fitted to
// 146 shapes of 64..16384 by 64..4096 by 64..8192, each tile with one and more K splits, replayed from a graph: the choice is 0.5 % behind
// the best on average, 18 % at most (3120x3508x72).
static constexpr TileModel kTileModelF32[kNumTiles] = {{37.3, 37.3, 8.4, 7520.0, 1}, {29.5, 29.5, 6.4, 6410.0, 1}, {14.9, 19.5, 5.1, 5400.0, 3}};
// Row-major (TN) operands: a K tile takes twice the LDS fragment reads, and a 64-wide tile of int8 operands
// loads 64-byte row pieces (binary16: 128 bytes, no penalty); fitted slow-down of the main loop per tile shape.
static double tn_factor(int tile, int prec, bool tn)
{
    const double rate[kNumTiles] = {0.94, 0.89, prec == 8 ? 0.74 : 0.97};
    return tn ? rate[tile] : 1.0;
}

GemmPlan plan_gemm(int prec, int64_t M, int64_t N, int64_t K, int force_tile, int force_splits, bool allow_split, bool tn)
{
    if(force_tile < 0 && g_tile_override >= 0)
    {   // a forced tile keeps the planner's split choice for that tile
        GemmPlan forced = plan_gemm(prec, M, N, K, g_tile_override, force_splits >= 1 ? force_splits : 0, allow_split, tn);
        return forced;
    }
    GemmPlan plan{1, 1, 0, 0.0};
    if(M <= 0 || N <= 0) return plan;
    const int64_t kb     = K * (prec == 8 ? 1 : (prec == 16 ? 2 : 4));
    // (the unit of fp32's constants: what a K tile of fp32 operands took on the fp32 instructions)
    const double  kwork  = prec == 32 ? 8.0 : 1.0;
    const int64_t ktiles = (kb + kRowBytes - 1) / kRowBytes;
    auto shape  = [&](int t) { return gemm_tile_shape(prec, t); };
    auto ntiles = [&](int t) { return ((M + shape(t).bm - 1) / shape(t).bm) * ((N + shape(t).bn - 1) / shape(t).bn); };
    // Plan = (tile, K splits) with the smallest estimated time.  The estimate is a small model fitted to gfx950
    // measurements of these tiles on 32x32 instructions (int8 and binary16, forward, row-major and transposed weight-gradient
    // forms: 54 operands x 3 tiles, replayed from a graph; rms error 11 %; fp32 operands have constants of their own).  It knows
    // nothing of the 128 tile's loading wavefronts.  The choice against the best of the three present tiles, over 465 shapes of 64..16384
    // by 64..4096 that are the tiles': forward 1.1 % behind on average with int8 and 1.7 % with binary16, row-major 0.6 % and 1.6 %,
    // as before (1.0 % and 1.6 %); more than 10 % in 18 of them, 35 % at most (row-major binary16 3328x528x2384, split on the 64 tile
    // where the 128 tile takes 22.9 us):
    //   a compute unit retires `r1` Mop/us per resident workgroup of a tile shape, up to `rmax` with `occ` of them
    //   sharing it; the chip as a whole retires at most `cap` Mop/us (256 busy units, at a lower clock and on
    //   shared caches, do not each reach `rmax`); every round of co-resident workgroups costs `ovh` us of launch, first-load latency
    //   and epilogue (the 256 tile's: fitted 6.9, raised to 7.5 for few K tiles: int8 9856 x 1920 x 176, fp32 output, 256
    //   tile 28.5 us, 128 tile 21.5; 49 of 6000 shapes drawn over the same range change, 18 % faster on average); split K adds its reduction pass.
    const double     cus = 256.0;
    const TileModel* models = prec == 32 ? kTileModelF32 : kTileModel;
    const int64_t    least = prec == 32 ? 4 : 8;      // K tiles of a split: one of fp32 operands is 0.5 us and more
    auto estimate = [&](int t, int64_t s) {
        const TileModel& m    = models[t];
        const double     tnf  = tn_factor(t, prec, tn);
        const double     wgs  = static_cast<double>(ntiles(t)) * static_cast<double>(s);
        const double     per  = std::ceil(wgs / cus);                                    // workgroups of the busiest unit
        const double     share = per < m.occ ? per : m.occ;                              // co-resident ones
        const double     rate = (m.r1 * share < m.rmax ? m.r1 * share : m.rmax) * tnf;
        const double     kt   = std::ceil(static_cast<double>(ktiles) / static_cast<double>(s));
        const double     mop  = 2.0 * shape(t).bm * shape(t).bn * kRowBytes * 1e-6 * kwork;    // per K tile (int8 ops)
        const double     unit = per * kt * mop / rate, chip = wgs * kt * mop / (m.cap * tnf);
        double           us   = (unit > chip ? unit : chip) + m.ovh * std::ceil(wgs / (cus * m.occ));
        // (the parts' way to memory and back; fp32's was fitted together with its other constants)
        if(s > 1) us += (prec == 32 ? 1.9 : 4.0) + (prec == 32 ? 2.7 : 1.0) * static_cast<double>(s + 1) * static_cast<double>(M) * static_cast<double>(N) * 4.0 / 6.24e6;
        return us;
    };
    // (fp32 up to kF32ShortK is latency and stores: the small tile, 2584x3144x4 14.7 us, 256 tile 20.4, 128 tile 19.7; 5960x1804x4 19.0, 23.7, 23.6)
    // Candidates: no split, and the split counts that fill the units once, twice or up to their co-residency.  Tiles are
    // visited from large to small and splits from few to many; a later candidate must win by 5 % (the larger tile
    // moves fewer bytes per operation, and estimates that close are inside the model's error) -- unless the
    // incumbent's tiles overhang the output by a quarter more than the candidate's: padding is where the model
    // errs in the larger tile's favour.
    int     tile = 0, splits = 1;
    double  best = -1.0, best_area = 0.0;
    for(int t = 0; t < kNumTiles; ++t)
    {
        if(force_tile >= 0 && force_tile < kNumTiles && t != force_tile) continue;
        if(force_tile < 0 && prec == 32 && K <= kF32ShortK && t + 1 < kNumTiles) continue;      // (below)
        int64_t cand[4] = {1, 1, 1, 1};
        int     ncand   = 1;
        if(allow_split && !(force_tile >= 0 && force_splits < 0))
            for(int f = 0; f < 3; ++f)
            {
                const int64_t fill = f == 0 ? 256 : (f == 1 ? 512 : 256 * models[t].occ);
                if(fill > 256 * models[t].occ) continue;
                int64_t       s    = fill / ntiles(t);
                if(s > ktiles / least) s = ktiles / least;
                if(s > 128) s = 128;
                if(s >= 2 && s != cand[ncand - 1]) cand[ncand++] = s;
            }
        const double area = static_cast<double>(ntiles(t)) * shape(t).bm * shape(t).bn;
        for(int c = 0; c < ncand; ++c)
        {
            const double us     = estimate(t, cand[c]);
            const double margin = best_area > 1.25 * area ? 1.0 : 0.95;
            if(best < 0.0 || us < margin * best) { best = us; best_area = area; tile = t; splits = static_cast<int>(cand[c]); }
        }
    }
    if(force_splits >= 1 && allow_split) splits = force_splits;
    if(splits > ktiles) splits = static_cast<int>(ktiles < 1 ? 1 : ktiles);
    plan.tile      = tile;
    plan.splits    = splits;
    plan.workspace = splits > 1 ? static_cast<size_t>(splits) * M * N * 4 : 0;
    plan.us        = estimate(tile, splits);
    return plan;
}

// Kernel arguments of a problem under a plan; hipErrorInvalidValue for operands the kernels cannot address.
static hipError_t kernel_args(const GemmProblem& p, const GemmPlan& plan, void* workspace, GemmKernelArgs& a)
{
    const int      esz = p.prec == 8 ? 1 : (p.prec == 16 ? 2 : 4);
    // lane offsets inside an operand panel are 32-bit: 255 rows of K bytes (plus the load immediates) must fit
    if(p.K > kGemmMaxRowBytes / esz) return hipErrorInvalidValue;
    a.A = static_cast<const uint8_t*>(p.A);
    a.B = static_cast<const uint8_t*>(p.B);
    a.M = p.M; a.N = p.N; a.Kb = p.K * esz;
    a.C = p.C; a.c_is_f16 = p.c_dtype == kF16;
    a.s0 = p.s0; a.s1 = p.s1; a.col_scale = p.col_scale; a.col_bias = p.col_bias;
    a.acc_dump = p.prec == 8 ? p.acc_dump : nullptr;
    a.partial  = workspace;
    a.conv_H = a.conv_W = a.conv_Cb = 0;
    a.remap_C = a.remap_shift = 0;
    if(p.tn)
    {   // A [K, M], B [K, N] row-major int8 or binary16: rows are contraction indices (128 bytes' worth per K tile),
        // 16-byte column chunks
        if((p.prec != 8 && p.prec != 16) || p.b_remap_C > 0
           || (p.M * esz) % 16 != 0 || (p.N * esz) % 16 != 0
           || p.M >= (int64_t(1) << 24) || p.N >= (int64_t(1) << 24)
           || ((reinterpret_cast<uintptr_t>(p.A) | reinterpret_cast<uintptr_t>(p.B)) & 15) != 0)
            return hipErrorInvalidValue;
    }
    a.amax_bits = plan.splits > 1 ? nullptr : p.out_amax_bits;      // with K splits the reduction pass takes the maximum
    a.codes     = plan.splits > 1 ? nullptr : static_cast<int8_t*>(p.out_codes);      // ... and writes the codes
    a.code_inv  = p.out_code_inv;
    a.code_qmax = p.out_code_qmax;
    if(p.b_remap_C > 0)
    {   // B is [3*remap_C, K] with a margin of |remap_shift| readable bytes in front of it and behind it
        if(p.conv_H > 0 || p.N != 9 * p.b_remap_C || p.b_remap_shift % 16 != 0 || p.b_remap_shift < 0
           || p.b_remap_shift > 1024 || 3 * p.b_remap_C * a.Kb >= (int64_t(1) << 32) - (1 << 20))
            return hipErrorInvalidValue;
        a.remap_C = static_cast<int>(p.b_remap_C); a.remap_shift = static_cast<int>(p.b_remap_shift);
    }
    if(p.conv_H > 0 && p.tn)
    {   // B is the NHWC tensor [K = images*H*W pixels, C]; the [pixels, 9*C] patch matrix is formed by the loads
        if(p.N != 9 * p.conv_C || p.K * p.conv_C * esz >= (int64_t(1) << 31) || p.conv_H > 65535 || p.conv_W > 65535
           || (p.conv_C * esz) % 16 != 0 || p.K % (static_cast<int64_t>(p.conv_H) * p.conv_W) != 0)
            return hipErrorInvalidValue;
        a.conv_H = p.conv_H; a.conv_W = p.conv_W; a.conv_Cb = static_cast<int>(p.conv_C * esz);
    }
    else if(p.conv_H > 0)
    {   // A is the NHWC tensor [M = images*H*W, C]; its 3x3 patch matrix [M, 9*C] is formed by the loads
        if(p.K != 9 * p.conv_C || plan.splits > 1 || p.M * p.conv_C * esz >= (int64_t(1) << 31)
           || p.conv_H > 65535 || p.conv_W > 65535 || (p.conv_C * esz) % 16 != 0
           || p.M % (static_cast<int64_t>(p.conv_H) * p.conv_W) != 0)
            return hipErrorInvalidValue;
        a.conv_H = p.conv_H; a.conv_W = p.conv_W; a.conv_Cb = static_cast<int>(p.conv_C * esz);
    }
    const int64_t ktiles = (a.Kb + kRowBytes - 1) / kRowBytes;
    int splits = plan.splits < 1 ? 1 : plan.splits;
    a.ktiles_per_split = static_cast<int>((ktiles + splits - 1) / splits);
    if(a.ktiles_per_split < 1) a.ktiles_per_split = 1;
    const TileShape ts = kTiles[plan.tile];
    a.tiles_m = static_cast<int>((p.M + ts.bm - 1) / ts.bm);
    a.tiles_n = static_cast<int>((p.N + ts.bn - 1) / ts.bn);
    a.group_m = kGroupM;      // (2, 4, 16 and 32 measured within noise of 8 on config 5's shapes, int8 and binary16)
    return hipSuccess;
}

// Second launch of a product in K splits: their sum and the epilogue.
static hipError_t reduce_splits(const GemmProblem& p, int splits, void* workspace, hipStream_t stream, ColumnFoldArgs* fold)
{
    const bool vec4 = p.N % 4 == 0 && ((reinterpret_cast<uintptr_t>(workspace) | reinterpret_cast<uintptr_t>(p.C)) & 15) == 0;
    int64_t    nb   = (p.M * p.N / (vec4 ? 4 : 1) + kThreads - 1) / kThreads;
    nb              = nb > 65536 ? 65536 : nb;
    if(p.out_amax_bits && nb > 1024) nb = 1024;    // at most one atomic per workgroup on one word: keep them few
    const ColumnFoldArgs beside = fold ? *fold : ColumnFoldArgs{};
    if(fold) *fold = ColumnFoldArgs{};
    auto reduce = [&](auto acc_tag, auto vec_tag, const void* ws, int32_t* dump) {
        typedef decltype(acc_tag) acc_t;
        splitk_reduce_kernel<acc_t, decltype(vec_tag)::value><<<dim3(nb + beside.blocks()), dim3(kThreads), 0, stream>>>(
            static_cast<const acc_t*>(ws), splits, p.M, p.N, p.C, p.c_dtype == kF16, p.s0, p.s1, p.col_scale, p.col_bias, dump,
            p.out_amax_bits, static_cast<int8_t*>(p.out_codes), p.out_code_inv, p.out_code_qmax, static_cast<int>(nb), beside);
    };
    if(p.prec == 8)
    {
        if(vec4) reduce(int32_t{}, std::true_type{}, workspace, p.acc_dump);
        else     reduce(int32_t{}, std::false_type{}, workspace, p.acc_dump);
    }
    else
    {
        if(vec4) reduce(float{}, std::true_type{}, workspace, nullptr);
        else     reduce(float{}, std::false_type{}, workspace, nullptr);
    }
    return hipGetLastError();
}

hipError_t launch_gemm(const GemmProblem& p, const GemmPlan& plan, void* workspace, hipStream_t stream, ColumnFoldArgs* fold)
{
    if(p.M <= 0 || p.N <= 0) return hipSuccess;
    if(p.prec == 32 && (p.conv_H > 0 || p.b_remap_C > 0)) return hipErrorInvalidValue;
    const int splits = plan.splits < 1 ? 1 : plan.splits;
    if(p.prec == 32)
    {
        const hipError_t e = launch_gemm_f32(p, plan, workspace, stream);
        return e != hipSuccess || splits == 1 ? e : reduce_splits(p, splits, workspace, stream, fold);
    }
    GemmKernelArgs   a;
    const hipError_t bad = kernel_args(p, plan, workspace, a);
    if(bad != hipSuccess) return bad;
    if(g_tile_override < 0 && g_persistent_mode != 1)
    {   // (whatever the plan holds: room for its K splits stays asked for, and unused here)
        bool             taken = false;
        const hipError_t e     = launch_gemm_rows(p, &taken, stream);
        if(taken || e != hipSuccess) return e;
    }
    if(p.conv_H > 0 && !p.tn)
    {
        bool             taken = false;
        const hipError_t e     = launch_conv3x3(p, g_tile_override, &taken, stream);
        if(taken || e != hipSuccess) return e;
    }
    if(p.conv_H > 0 && p.tn && splits > 1 && g_tile_override < 0)
    {
        hipError_t e   = hipSuccess;
        const int  own = launch_conv3x3_wgrad(p, splits, plan.us, workspace, stream, &e);
        if(own > 0) return e != hipSuccess ? e : reduce_splits(p, own, workspace, stream, fold);
    }
    // The persistent kernel is opt-in.  Its write-back of a tile overlaps the next tile's K loop, which on 32x32 instructions gained
    // 7-20 % launched alone and back to back; the present K loop leaves its wavefronts no registers for a second set of the columns'
    // fragments, and it loses there too: 16384x4096x1024 int8 75.1 us per tile, 80.5 persistent, binary16 124.4 and 127.1, 16384x1024x4096 53.0
    // and 53.5.  Inside an operator sequence its fixed tile assignment costs more: workgroups that start late, behind the tail of the
    // previous kernel, still walk their full share of tiles, while the per-tile grid is balanced by the hardware dispatcher.
    if(!p.tn && persistent_eligible(a, p.prec, plan.tile, splits)
       && g_persistent_mode == 1)
        return p.prec == 8 ? launch_persistent<I8Traits>(a, stream) : launch_persistent<F16Traits>(a, stream);
    hipError_t e = p.prec == 8 ? launch_traits<I8Traits>(plan.tile, a, splits, stream, p.tn)
                               : launch_traits<F16Traits>(plan.tile, a, splits, stream, p.tn);
    return e != hipSuccess || splits == 1 ? e : reduce_splits(p, splits, workspace, stream, fold);
}

// K tiles of a workgroup per round of 256 workgroups -> time of the compute unit that gets the first workgroup of every
// round (the hardware deals them out in order): `occ` workgroups share the unit's rate evenly, the next one starts when
// one ends.
static double unit_time(const TileModel& m, double mop, const double* rounds, int n)
{
    double left[8], us = 0.0;
    int    active = 0, next = 0;
    for(;;)
    {
        while(active < m.occ && next < n) left[active++] = rounds[next++];
        if(active == 0) return us;
        double shortest = left[0];
        for(int i = 1; i < active; ++i) shortest = left[i] < shortest ? left[i] : shortest;
        const double rate = m.r1 * active < m.rmax ? m.r1 * active : m.rmax;
        us += shortest * active * mop / rate;
        int kept = 0;
        for(int i = 0; i < active; ++i)
            if(left[i] > shortest) left[kept++] = left[i] - shortest;
        active = kept;
    }
}

// Tile on which two GEMMs share a launch (`a` first), or -1 when two launches are estimated to be about as fast: with more
// than sixteen rounds of workgroups each of them fills the chip by itself, and a long contraction unsplit beside short ones
// would outlast them.  Separate launches -> one, measured: int8 1808x1040x784 15.6 -> 12.2 us, 1024^3 10.7 -> 6.9, 512^3 6.8 -> 4.8,
// 4096x768x3072 31.5 -> 30.5; binary16 2056x1000x1032 31.0 -> 25.3, 4096x3072x768 50.3 -> 50.8 (4096x768x3072 and 4096x3072x768
// gained 5 and 9 us before the separate launches had loading wavefronts); not paired: 4096x768x768 binary16 26.1 (one launch
// 26.5), 3000x768x768 24.9 (25.1).
// How far the estimate reaches, over 146 backward passes (44 operators from 512^3 to 8192 x 1024^2, drawn evenly over the
// logarithm, both types, transposed copies and row-major, replayed from a graph; two launches against one on either tile), all on the
// tiles' form of 32x32 instructions: its rms error is 17 % for int8 and 27 % for binary16, where it is 14 % too long on average.  The choice costs 1.9 % on
// average against the best of the three and more than 10 % in ten cases (binary16 384x1744x1168 left apart, 19.5 us against
// 14.2, is the worst); it errs towards two launches: the 114 pairs run 1.48 times as fast as apart, the worst of them
// 2.4 % slower.
static double pair_us(const GemmProblem& a, const GemmProblem& b, int t, int splits)
{
    constexpr int kMaxRounds = 16;
    TileModel m = kTileModel[t];
    if(a.prec == 16) m.r1 *= t == 1 ? 0.83 : 0.6;       // a long binary16 contraction left over alone, fitted
    auto tiles  = [&](const GemmProblem& p) { return ((p.M + kTiles[t].bm - 1) / kTiles[t].bm) * ((p.N + kTiles[t].bn - 1) / kTiles[t].bn); };
    auto ktiles = [&](const GemmProblem& p, int s) { return std::ceil(std::ceil(static_cast<double>(p.K * (p.prec / 8)) / kRowBytes) / s) / tn_factor(t, p.prec, p.tn); };
    const int64_t wa = tiles(a) * splits, wgs = wa + tiles(b);
    if(wgs > kMaxRounds * kNumCu) return -1.0;
    const double ka = ktiles(a, splits), kb = ktiles(b, 1), mop = 2.0 * kTiles[t].bm * kTiles[t].bn * kRowBytes * 1e-6;
    double rounds[kMaxRounds];
    int    n = 0;
    for(int64_t at = 0; at < wgs; at += kNumCu) rounds[n++] = at < wa ? ka : kb;
    const double unit = unit_time(m, mop, rounds, n), chip = (wa * ka + (wgs - wa) * kb) * mop / m.cap;
    const double full = std::ceil(static_cast<double>(wgs) / (kNumCu * m.occ));      // rounds of co-resident workgroups
    const double us   = (unit > chip ? unit : chip) + m.ovh * (full > 1.0 ? full - 0.5 : full);
    return splits > 1 ? us + 4.0 + static_cast<double>(splits + 1) * static_cast<double>(a.M) * static_cast<double>(a.N) * 4.0 / 6.24e6 : us;
}
static int pair_tile(const GemmProblem& a, const GemmProblem& b, double separate_us)
{
    int    tile = -1;
    double best = 0.93 * separate_us;
    for(int t = 1; t < kNumTiles; ++t)
    {
        if(g_tile_override >= 0 && t != g_tile_override) continue;
        const double us = pair_us(a, b, t, 1);
        if(us >= 0.0 && us < (tile < 0 ? 1.0 : 0.95) * best) { best = us; tile = t; }      // (the smaller tile must win by 5 %)
    }
    return tile;
}
// Where the two would go apart, the first (the longer contraction) in K splits: the tile and the splits, up to as many, on which they share
// a launch all the same, with the sum of the splits behind it.  Few outputs over a long contraction leave units idle, and the parts of
// both together fill them: three launches become two.  Binary16 keeps the plan's splits, not fewer: a sum over a longer piece has more roundings
// (4096x768x3072 unsplit 59.8 -> 54.8 us, but the error of dW against 64 bits 2.4e-7 -> 4.1e-7); int8 sums are exact.  Backward passes of 64..16384 by
// 64..4096 (both types, both forms, replayed from a graph), apart -> this, us: binary16 6784x912x592 41.5 -> 31.2, 13536x1360x240 42.1 -> 37.6,
// 4224x312x160 13.5 -> 9.7, int8 15744x2288x112 32.2 -> 22.9, 14640x128x2608 54.9 -> 42.0; of 120 drawn 26 gain, 1.25 times on
// average.  The estimate does not know how the second's contraction drags on over the small tile: with
// more than 36 K tiles of it the pair may lose (binary16 3200x3656x128 30.7, 39.8 together), nor of gemm_rows_kernel
// (2112x1696x96 13.0, 20.0).
static GradientPair split_pair(const GemmProblem& a, const GemmPlan& plan_a, const GemmProblem& b, double separate_us)
{
    GradientPair pair;
    const int64_t kb = (b.K * (b.prec / 8) + kRowBytes - 1) / kRowBytes;
    if(plan_a.splits < 2 || kb > 36 || g_tile_override >= 0 || gemm_rows_takes(a) || gemm_rows_takes(b)) return pair;
    double best = separate_us;
    for(int t = 1; t < kNumTiles; ++t)
        for(int s = a.prec == 8 ? 1 : plan_a.splits; s <= plan_a.splits; ++s)
        {
            const double us = pair_us(a, b, t, s);
            if(us >= 0.0 && us < best) { best = us; pair = GradientPair{t, s}; }
        }
    return pair;
}

// The weight gradient lands in memory that the data gradient reads (a caller that stores dW over the transposed weights or
// over dY, say): fine in two launches, data gradient first, a race in one.
static bool dw_over_dx_operands(const GemmProblem& dx, const GemmProblem& dw)
{
    auto meets = [](const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
        return a && b && x < y + static_cast<uintptr_t>(b_bytes) && y < x + static_cast<uintptr_t>(a_bytes);
    };
    const int64_t esz = dx.prec / 8, out = dw.M * dw.N;
    auto written = [&](const void* p, int64_t bytes) {
        return meets(dw.C, out * (dw.c_dtype == kF16 ? 2 : 4), p, bytes) || meets(dw.acc_dump, out * 4, p, bytes);
    };
    return written(dx.A, dx.M * dx.K * esz) || written(dx.B, dx.N * dx.K * esz) || written(dx.s0, 4) || written(dx.s1, 4)
        || written(dx.col_scale, dx.N * 4);
}

static bool dw_is_first(const GemmProblem& dx, const GemmProblem& dw) { return dw.tn || dw.K >= dx.K; }      // the longer contraction, or the row-major one

GradientPair gradient_pair(const GemmProblem& dx, const GemmPlan& plan_dx, const GemmProblem& dw, const GemmPlan& plan_dw)
{
    auto plain = [](const GemmProblem& p) {
        return (p.prec == 8 || p.prec == 16) && p.M > 0 && p.N > 0 && p.K > 0 && p.conv_H == 0 && p.b_remap_C == 0
            && !p.out_amax_bits && !p.out_codes;
    };
    if(dx.prec != dw.prec || !plain(dx) || !plain(dw) || dx.tn || g_persistent_mode == 1 || dw_over_dx_operands(dx, dw)) return GradientPair{};
    // (The estimates are the tiles', also of a product that by itself would go to gemm_rows_kernel.  One shared launch -> that kernel for
    // what it takes, replayed from a graph: 64x128x128 int8 4.2 us, apart 6.3, 512^3 4.8 and 8.1, 128x1024x2048 8.2 and 8.8;
    // binary16 4.0 and 6.1, 5.8 and 9.1, but 128x1024x2048 11.0 and 9.7, 256x1024x1024 10.8 and 9.7: the worst of 32.)
    const double       us = plan_dx.us + plan_dw.us;
    const bool         dw_first = dw_is_first(dx, dw);
    const GemmProblem &a = dw_first ? dw : dx, &b = dw_first ? dx : dw;
    GradientPair       pair;
    pair.tile = pair_tile(a, b, us);
    return pair.tile >= 0 ? pair : split_pair(a, dw_first ? plan_dw : plan_dx, b, us);
}

hipError_t launch_gradient_pair(const GemmProblem& dx, void* ws_dx, const GemmProblem& dw, void* ws_dw, const GradientPair& pair, const ColumnFoldArgs& fold, hipStream_t stream)
{
    const bool         dw_first = dw_is_first(dx, dw);
    const GemmProblem &a = dw_first ? dw : dx, &b = dw_first ? dx : dw;
    void* const        workspace = dw_first ? ws_dw : ws_dx;
    GemmPairArgs       args;
    hipError_t         e = kernel_args(a, GemmPlan{pair.tile, pair.splits, 0, 0.0}, workspace, args.g[0]);
    if(e == hipSuccess) e = kernel_args(b, GemmPlan{pair.tile, 1, 0, 0.0}, nullptr, args.g[1]);
    if(e != hipSuccess) return e;
    args.splits = pair.splits;
    args.na     = args.g[0].tiles_m * args.g[0].tiles_n * pair.splits;
    args.total  = args.na + args.g[1].tiles_m * args.g[1].tiles_n;
    if(pair.splits == 1) args.fold = fold;
    auto go = [&](auto tn, auto split) {
        constexpr bool TNA = decltype(tn)::value, SPLITA = decltype(split)::value;
        return a.prec == 8 ? launch_pair_traits<I8Traits, TNA, SPLITA>(pair.tile, args, stream) : launch_pair_traits<F16Traits, TNA, SPLITA>(pair.tile, args, stream);
    };
    constexpr std::true_type  yes{};
    constexpr std::false_type no{};
    if(pair.splits == 1) return a.tn ? go(yes, no) : go(no, no);
    e = a.tn ? go(yes, yes) : go(no, yes);
    ColumnFoldArgs beside = fold;
    return e != hipSuccess ? e : reduce_splits(a, pair.splits, workspace, stream, &beside);
}

}  // namespace qsync
