// y = x w^T with a scale for each row of x and w, for the tokens of a handful of sequences: rows quantized and multiplied in one launch.
//
// Such a product reads its weights once and does nothing else to speak of, so what counts is the launch and how soon and how far ahead the
// weights are requested.  Every workgroup (16 columns) quantizes all the rows for itself, while the first of its weights are on their way: that
// reads x from L2 once a workgroup, 8 KB a token of 4096 binary16 values, and saves a launch and the round trip of the codes through memory.  The eight wavefronts then take
// the contraction in turns of 64 bytes, the weights through stages of their own (eight turns in flight, no barrier), the codes from LDS,
// and their sums meet in LDS.
#include "gemm_device.h"
#include "row_ops.h"
#include "token_ops.h"

namespace qsync {

namespace {

constexpr int kFewWaves = 8, kFewRows = 16, kFewHeld = 8;
constexpr int kFewLds = 96 * 1024;      // (at most 64 KB of stages, 16 KB of codes and their padding)
int64_t few_lds(int64_t rows, int64_t kb, int stages) { return kFewWaves * stages * 1024 + rows * (kb + 16); }

// What every workgroup quantizes for itself has to stay small, and the workgroups few enough to run at once.  One launch / two, us, binary16: 1 row
// 1024x4096 6.6 / 7.4, 4096x4096 8.2 / 8.3, 300x16384 9.8 / 13.0; 4 rows 4096x1024 5.5 / 7.3, 4096x4096 9.2 / 8.8; 16 rows 1024x1024 6.6 / 7.0, 1024x4096
// 11.1 / 7.0; 1 row 16384x1024 12.2 / 9.6.
constexpr int64_t kFewElements = 16384, kFewColumns = 4096;
// wavefronts that share a row: 1, 2, 4 or 8; and whether the longest row of any number of them fits the registers that hold it
__host__ __device__ constexpr int few_share(int rows) { return rows > 4 ? 1 : rows > 2 ? 2 : rows == 2 ? 4 : 8; }
constexpr bool few_held()
{
    for(int rows = 1; rows <= kFewRows; ++rows)
        if(kFewElements / rows / 8 > kFewHeld * few_share(rows) * kWaveSize) return false;
    return true;
}
static_assert(few_held(), "a row's vectors stay in registers between its maximum and its codes");

struct FewArgs
{
    const void*   x;
    const int8_t* w;
    const float * sw, *bias;
    void*         y;
    int64_t       K, ld, N;
    int           rows, ydt;
};

// STAGES: turns of a wavefront in flight, no more than there are (short contractions: more workgroups on a unit).
template <typename T, int STAGES> __global__ __launch_bounds__(64 * kFewWaves) void token_few_kernel(const FewArgs p)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    __shared__ uint32_t top[kFewWaves];
    __shared__ float    scales[kFewRows];
    const int     lane = threadIdx.x % kWaveSize, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x / kWaveSize));
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * 16, kb = code_pad(p.K);
    uint8_t* const mine = lds + wave * (STAGES * 1024);
    uint8_t* const codes = lds + kFewWaves * STAGES * 1024;
    const int      pitch = static_cast<int>(kb) + 16;      // (sixteen rows' chunks meet all banks)

    // Weights: four lanes read 64 consecutive bytes of a column's row; the 16-byte chunks land XOR-swizzled.
    const int      lrow = lane / 4, lchunk = ((lane % 4) ^ ((lane >> 4) & 3)) * 16;
    const uint8_t* src = reinterpret_cast<const uint8_t*>(p.w) + (n0 + lrow < p.N ? n0 + lrow : p.N - 1) * kb + lchunk;
    const int      all = static_cast<int>(kb / 64), turns = all > wave ? (all - wave + kFewWaves - 1) / kFewWaves : 0;
    auto issue = [&](int t) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + (static_cast<int64_t>(t) * kFewWaves + wave) * 64),
                                         (__attribute__((address_space(3))) void*)(mine + t % STAGES * 1024), 16, 0, 0);
    };
    // (the columns' scales and biases, by the wavefront that needs them: in front of everything, their latency is nobody's)
    float sb[4] = {}, bias[4] = {};
    if(wave == 0)
#pragma unroll
        for(int e = 0; e < 4; ++e)
        {
            const int64_t n = n0 + lane / 16 * 4 + e, c = n < p.N ? n : p.N - 1;
            sb[e]   = p.sw[c];
            bias[e] = p.bias ? p.bias[c] : 0.0f;
        }
    const int share = few_share(p.rows), at_once = kFewWaves / share, part = wave % share;
    const int groups = static_cast<int>(kb / 8), step = share * 64;
    Row8<T>   v[kFewHeld];
    bool      requested = false;
    for(int r0 = 0; r0 < p.rows; r0 += at_once)
    {
        const int r = r0 + wave / share;
        const T*  row = static_cast<const T*>(p.x) + (r < p.rows ? r : 0) * p.ld;
        auto      load = [&](int g, Row8<T>& d) {
            if(g * 8 + 8 <= p.K) d.load(row + g * 8);
            else
            {
                float e[8];
#pragma unroll
                for(int j = 0; j < 8; ++j) e[j] = g * 8 + j < p.K ? row_element(row + g * 8 + j) : 0.0f;
                d.encode(e);
            }
        };
        uint32_t m = 0u;
        auto     fold = [&](const Row8<T>& d) {
            float e[8];
            d.decode(e);
#pragma unroll
            for(int j = 0; j < 8; ++j) m = max(m, abs_bits(e[j]));
        };
        const int g0 = part * 64 + lane;
#pragma unroll
        for(int i = 0; i < kFewHeld; ++i)
            if(i * step < groups) load(g0 + i * step, v[i]);      // (the same for all lanes)
        if(!requested)      // (behind the first rows' loads: what waits for those does not wait for the weights)
        {
            for(int t = 0; t < STAGES && t < turns; ++t) issue(t);
            requested = true;
        }
#pragma unroll
        for(int i = 0; i < kFewHeld; ++i)
            if(i * step < groups) fold(v[i]);
#pragma unroll
        for(int off = 32; off >= 1; off >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), off)));
        if(share > 1)
        {
            if(lane == 0) top[wave] = m;
            wg_barrier();
            for(int i = 0; i < share; ++i) m = max(m, top[wave - part + i]);
        }
        const CodeScale cs = code_scale(m);
        if(r < p.rows)
        {
            if(part == 0 && lane == 0) scales[r] = cs.scale;
            auto put = [&](const Row8<T>& d, int g) {
                float e[8];
                d.decode(e);
                if(cs.inv == 0.0f)
#pragma unroll
                    for(int j = 0; j < 8; ++j) e[j] = 0.0f;
                uint32_t c[2];
                quantize_group<float, kNearest>(e, cs.inv, 127, make_uint4(0, 0, 0, 0), c);
                *reinterpret_cast<uint2*>(codes + r * pitch + g * 8) = make_uint2(c[0], c[1]);
            };
#pragma unroll
            for(int i = 0; i < kFewHeld; ++i)
                if(i * step < groups && g0 + i * step < groups) put(v[i], g0 + i * step);
        }
    }
    wg_barrier();

    const int      row = lane % 16, quad = lane / 16;
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)mine));
    const uint32_t code0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)codes))
                           + static_cast<uint32_t>((row < p.rows ? row : p.rows - 1) * pitch + quad * 16 + wave * 64);
    const uint32_t frag = lds0 + static_cast<uint32_t>(row * 64 + ((quad ^ ((row >> 2) & 3)) * 16));
    v4i32 acc = {0, 0, 0, 0};
    for(int t = 0; t < turns; ++t)
    {   // (every wavefront by itself: its loads, its slice of LDS)
        wait_tiles<1, STAGES - 1>(turns - 1 - t);
        v4i32 a, b;
        frag_read<0>(b, frag + static_cast<uint32_t>(t % STAGES * 1024));
        frag_read<0>(a, code0 + static_cast<uint32_t>(t * (kFewWaves * 64)));
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(a), "+v"(b)::"memory");
        __builtin_amdgcn_sched_barrier(0);
        if(t + STAGES < turns) issue(t + STAGES);      // (into the stage just read)
        acc = I8Traits::mfma(b, a, acc);
        __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();      // (the sums take the place of the stages)
    *reinterpret_cast<v4i32*>(lds + (wave * 64 + lane) * 16) = acc;
    __syncthreads();
    if(wave != 0 || row >= p.rows) return;
#pragma unroll
    for(int w = 1; w < kFewWaves; ++w) acc += *reinterpret_cast<const v4i32*>(lds + (w * 64 + lane) * 16);
    const float sa = scales[row];
#pragma unroll
    for(int e = 0; e < 4; ++e)
    {
        const int64_t n = n0 + quad * 4 + e;
        if(n >= p.N) continue;
        const float f = sa * sb[e], b = bias[e];
        if(p.ydt == kF16) static_cast<__half*>(p.y)[row * p.N + n] = fma_out<__half>(static_cast<float>(acc[e]), f, b);      // (the same bits as of the other products)
        else element_store(p.y, p.ydt, row * p.N + n, fmaf(static_cast<float>(acc[e]), f, b));
    }
}

template <typename T, int STAGES> hipError_t launch_stages(const FewArgs& a, hipStream_t st)
{
    static bool attr_set[16] = {};      // per instantiation and device; benign if set twice
    int         dev = 0;
    const bool  known = hipGetDevice(&dev) == hipSuccess && dev >= 0 && dev < 16;
    if(!known || !attr_set[dev])
    {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&token_few_kernel<T, STAGES>), hipFuncAttributeMaxDynamicSharedMemorySize, kFewLds);
        if(e != hipSuccess) return e;
        if(known) attr_set[dev] = true;
    }
    token_few_kernel<T, STAGES><<<static_cast<unsigned>((a.N + 15) / 16), 64 * kFewWaves, static_cast<size_t>(few_lds(a.rows, code_pad(a.K), STAGES)), st>>>(a);
    return hipGetLastError();
}
template <typename T> hipError_t launch_few(const FewArgs& a, hipStream_t st)
{
    const int64_t turns = (code_pad(a.K) / 64 + kFewWaves - 1) / kFewWaves;
    return turns <= 2 ? launch_stages<T, 2>(a, st) : turns <= 4 ? launch_stages<T, 4>(a, st) : launch_stages<T, 8>(a, st);
}

}  // namespace

hipError_t launch_token_few(const TokenMatrix& m, const TokenProduct& p, bool* taken, hipStream_t st)
{
    *taken = p.sets == 1 && !p.offsets && !m.source && p.rows <= kFewRows && p.K > 0 && p.rows * code_pad(p.K) <= kFewElements && p.N <= kFewColumns;
    if(!*taken) return hipSuccess;
    const FewArgs a{m.x, p.B, p.sb, p.bias, p.C, p.K, m.ld, p.N, static_cast<int>(p.rows), p.c_dtype};
    return m.dtype == kF16 ? launch_few<_Float16>(a, st) : m.dtype == kBF16 ? launch_few<__bf16>(a, st) : launch_few<float>(a, st);
}

}  // namespace qsync
