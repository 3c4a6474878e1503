// 16 MF rows by 16 NF columns of an int8 or binary16 matrix product by one workgroup whose eight wavefronts share the contraction (gemm_rows.hip).
#pragma once
#include "gemm_device.h"

namespace qsync {

namespace {

constexpr int kRowsWaves = 8;
constexpr int rows_stages(int loads) { return loads > 4 ? 3 : 4; }             // turns in LDS: 144 KB of them at most
template <int MF, int NF> constexpr int kRowsLds = kRowsWaves * rows_stages(MF + NF) * (MF + NF) * 1024;
// MF, NF: fragments of 16 rows, of 16 columns.  The B fragment is the instruction's first operand, so a lane holds four consecutive columns
// (4 (lane / 16) ..) of output row lane % 16.
// TOKEN: scales of the rows and of the columns, outputs of fp32, binary16 or bfloat16 (c_is_f16 2).
template <typename TR, int MF, int NF, bool TOKEN = false>
__device__ __forceinline__ void gemm_rows_tile(const GemmKernelArgs& p, int64_t m0, int64_t n0)
{
    typedef typename TR::accv_t vec;
    constexpr int kLoads = MF + NF, kStages = rows_stages(kLoads), kTurn = kLoads * 1024;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int     lane = threadIdx.x % kWaveSize, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x / kWaveSize));
    uint8_t* const mine = lds + wave * (kStages * kTurn);

    // loads: four lanes read 64 consecutive bytes of a row (lanes on sixteen rows, as the operands want them, took four times as
    // long); the 16-byte chunks land XOR-swizzled so that sixteen rows of one chunk meet all banks
    const int      lrow = lane / 4, lchunk = ((lane % 4) ^ ((lane >> 4) & 3)) * 16;
    const uint8_t* src[kLoads];
#pragma unroll
    for(int f = 0; f < MF; ++f) src[f] = p.A + (m0 + f * 16 + lrow < p.M ? m0 + f * 16 + lrow : p.M - 1) * p.Kb;
#pragma unroll
    for(int j = 0; j < NF; ++j) src[MF + j] = p.B + (n0 + j * 16 + lrow < p.N ? n0 + j * 16 + lrow : p.N - 1) * p.Kb;
    // (rows and columns past the end: any valid one, never stored)
    const int all = static_cast<int>((p.Kb + 63) / 64), turns = all > wave ? (all - wave + kRowsWaves - 1) / kRowsWaves : 0;
    auto issue = [&](int t) {
        const int64_t k   = (static_cast<int64_t>(t) * kRowsWaves + wave) * 64 + lchunk;
        const bool    in  = k < p.Kb;                                        // (16-byte pieces: Kb is a multiple of 16)
        uint8_t*      dst = mine + t % kStages * kTurn;
        static_for<kLoads>([&](auto f) {
            constexpr int i = decltype(f)::value, IMM = i % 4 * 1024;
            const uint8_t* at = in ? src[i] + k : reinterpret_cast<const uint8_t*>(&g_zero_chunk);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(at - IMM),
                                             (__attribute__((address_space(3))) void*)(dst + i / 4 * 4096), 16, IMM, 0);
        });
    };
    vec acc[MF * NF];
#pragma unroll
    for(int f = 0; f < MF * NF; ++f) acc[f] = vec{0, 0, 0, 0};
    const int      row = lane % 16, quad = lane / 16;
    // (the epilogue's scales and biases are requested in front of everything)
    [[maybe_unused]] float row_scale = 0.0f, cs[4] = {}, cb[4] = {};
    if constexpr(TOKEN)
        if(wave < MF * NF)
        {
            const int64_t m = m0 + wave % MF * 16 + row, n = n0 + wave / MF * 16 + quad * 4;
            row_scale = p.row_scale[m < p.M ? m : p.M - 1];
#pragma unroll
            for(int e = 0; e < 4; ++e)
            {
                const int64_t c = n + e < p.N ? n + e : p.N - 1;
                cs[e] = p.col_scale[c];
                cb[e] = p.col_bias ? p.col_bias[c] : 0.0f;
            }
        }
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)mine));
    const uint32_t frag = static_cast<uint32_t>(row * 64 + ((quad ^ ((row >> 2) & 3)) * 16));
#pragma unroll
    for(int t = 0; t < kStages - 1; ++t)
        if(t < turns) issue(t);
    for(int t = 0; t < turns; ++t)
    {   // (every wavefront by itself: its loads, its slice of LDS)
        if(t + kStages - 1 < turns) issue(t + kStages - 1);
        wait_tiles<kLoads, kStages - 1>(turns - 1 - t);
        v4i32          op[kLoads];
        const uint32_t at = lds0 + static_cast<uint32_t>(t % kStages * kTurn) + frag;
        static_for<kLoads>([&](auto f) { frag_read<decltype(f)::value * 1024>(op[decltype(f)::value], at); });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for(int f = 0; f < MF; ++f)
#pragma unroll
            for(int j = 0; j < NF; ++j) acc[j * MF + f] = TR::mfma(op[MF + j], op[f], acc[j * MF + f]);
        __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();                                                        // (the sums take the place of the stages)
#pragma unroll
    for(int f = 0; f < MF * NF; ++f) *reinterpret_cast<vec*>(lds + ((wave * MF * NF + f) * 64 + lane) * 16) = acc[f];
    __syncthreads();
    if(wave >= MF * NF) return;
    vec sum = *reinterpret_cast<const vec*>(lds + (wave * 64 + lane) * 16);
#pragma unroll
    for(int w = 1; w < kRowsWaves; ++w) sum += *reinterpret_cast<const vec*>(lds + ((w * MF * NF + wave) * 64 + lane) * 16);

    const int64_t m = m0 + wave % MF * 16 + row, n = n0 + wave / MF * 16 + quad * 4;
    if(m >= p.M || n >= p.N) return;
    const float alpha = TOKEN ? row_scale : *(p.s0 ? p.s0 : &g_one) * *(p.s1 ? p.s1 : &g_one);
    float       fs[4], bs[4];
#pragma unroll
    for(int e = 0; e < 4; ++e)
    {
        if constexpr(TOKEN)
        {
            fs[e] = alpha * cs[e];
            bs[e] = cb[e];
            continue;
        }
        const int64_t c = n + e < p.N ? n + e : p.N - 1;
        fs[e] = p.col_scale ? alpha * p.col_scale[c] : alpha;
        bs[e] = p.col_bias ? p.col_bias[c] : 0.0f;
    }
    const int64_t at = m * p.N + n;
    const int     os = p.c_is_f16 ? 2 : 4;
    uint8_t* const dst = static_cast<uint8_t*>(p.C) + at * os;
    const bool    vector = p.N % 4 == 0 && (reinterpret_cast<uintptr_t>(p.C) & (4 * os - 1)) == 0;
    float v[4];
#pragma unroll
    for(int e = 0; e < 4; ++e) v[e] = static_cast<float>(sum[e]);
    if constexpr(TOKEN)
        if(p.c_is_f16 == 2)
        {
            for(int e = 0; e < 4 && n + e < p.N; ++e) reinterpret_cast<__bf16*>(dst)[e] = static_cast<__bf16>(fmaf(v[e], fs[e], bs[e]));
            return;
        }
    if(p.c_is_f16)
    {
        const uint2 h = make_uint2(fma_out_half2(v[0], fs[0], bs[0], v[1], fs[1], bs[1]), fma_out_half2(v[2], fs[2], bs[2], v[3], fs[3], bs[3]));
        if(vector) *reinterpret_cast<uint2*>(dst) = h;
        else
            for(int e = 0; e < 4 && n + e < p.N; ++e)
                reinterpret_cast<uint16_t*>(dst)[e] = static_cast<uint16_t>((e < 2 ? h.x : h.y) >> (16 * (e % 2)));
    }
    else
    {
        const float4 y = make_float4(fmaf(v[0], fs[0], bs[0]), fmaf(v[1], fs[1], bs[1]), fmaf(v[2], fs[2], bs[2]), fmaf(v[3], fs[3], bs[3]));
        const float  o[4] = {y.x, y.y, y.z, y.w};
        if(vector) *reinterpret_cast<float4*>(dst) = y;
        else
            for(int e = 0; e < 4 && n + e < p.N; ++e) reinterpret_cast<float*>(dst)[e] = o[e];
    }
}

}  // namespace

}  // namespace qsync
