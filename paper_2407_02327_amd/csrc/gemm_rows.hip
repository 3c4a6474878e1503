// C[M,N] = epilogue( sum_k A[m,k] B[n,k] ), int8 and binary16, where 64 rows and 16 or 32 columns a workgroup are few enough
// workgroups for one on each unit: a handful of tokens, small operators.
//
// On the tiles of 64 columns and more such a product is a few dozen workgroups (or one K split each of them) that walk K one LDS
// stage and barrier after the other, 0.26 us per 128 bytes.  Here a workgroup's eight wavefronts take K in turns of 64 bytes,
// each through stages of its own with two or three turns in flight and no barrier, into the 16x16 matrix instructions; the
// eight sums meet in LDS once at the end.
#include "gemm_rows.h"
#include "token_ops.h"

namespace qsync {

namespace {

constexpr int64_t kRowsGroups = 256;                                        // one for each unit
// The dimension of more groups runs fastest and is padded to a multiple of the eight XCDs where that stays within one group for
// each unit: the workgroups that read one piece of the longer operand then share an L2.  4096x128 by 3072, int8: 11.5 -> 7.5 us.
template <int NF> __host__ __device__ constexpr bool rows_first(int64_t M, int64_t N) { return M > N * (4 / NF); }
template <typename TR, int MF, int NF, bool TOKEN = false>
__global__ __launch_bounds__(64 * kRowsWaves) void gemm_rows_kernel(const GemmKernelArgs p)
{
    const bool    tall = rows_first<NF>(p.M, p.N);
    const int64_t n0 = static_cast<int64_t>(tall ? blockIdx.y : blockIdx.x) * (16 * NF), m0 = static_cast<int64_t>(tall ? blockIdx.x : blockIdx.y) * 64;
    if(m0 >= p.M || n0 >= p.N) return;                                      // (padded to a multiple of the XCDs)
    gemm_rows_tile<TR, MF, NF, TOKEN>(p, m0, n0);
}

template <typename TR, int MF, int NF, bool TOKEN = false> hipError_t launch_fragments(const GemmKernelArgs& a, hipStream_t st)
{
    static_assert(MF * NF <= kRowsWaves, "a wavefront per fragment in the epilogue");
    constexpr int kLds = kRowsLds<MF, NF>;
    static bool   attr_set[16] = {};      // per instantiation and device; benign if set twice
    int           dev = 0;
    const bool    known = hipGetDevice(&dev) == hipSuccess && dev >= 0 && dev < 16;
    if(!known || !attr_set[dev])
    {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&gemm_rows_kernel<TR, MF, NF, TOKEN>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if(e != hipSuccess) return e;
        if(known) attr_set[dev] = true;
    }
    const int64_t m = (a.M + 63) / 64, n = (a.N + 16 * NF - 1) / (16 * NF), few = rows_first<NF>(a.M, a.N) ? n : m;
    int64_t       many = rows_first<NF>(a.M, a.N) ? m : n;
    if((many + 7) / 8 * 8 * few <= kRowsGroups) many = (many + 7) / 8 * 8;
    gemm_rows_kernel<TR, MF, NF, TOKEN><<<dim3(static_cast<unsigned>(many), static_cast<unsigned>(few)), dim3(64 * kRowsWaves), kLds, st>>>(a);
    return hipGetLastError();
}
template <typename TR, bool TOKEN = false> hipError_t launch_rows(const GemmKernelArgs& a, int columns, hipStream_t st)
{
    if(columns == 2) return launch_fragments<TR, 4, 2, TOKEN>(a, st);
    switch(a.M > 64 ? 4 : (a.M + 15) / 16)
    {
    case 1: return launch_fragments<TR, 1, 1, TOKEN>(a, st);
    case 2: return launch_fragments<TR, 2, 1, TOKEN>(a, st);
    case 3: return launch_fragments<TR, 3, 1, TOKEN>(a, st);
    default: return launch_fragments<TR, 4, 1, TOKEN>(a, st);
    }
}
// Fragments of columns a workgroup, 0: other tiles are faster.  A second workgroup on a unit waits for the first (its stages fill
// the LDS; at most 16 rows two fit), which loses at once: 64x16384x64 3.8 us on the tiles, 9.0 here.  Beyond 6 KB of contraction
// (8 KB up to 32 rows) K splits over workgroups win.  The better of the 128 and 64 tiles -> here, operands warm, binary16 outputs, us:
//   int8, 16 columns:  1x4096x1024 5.0 -> 3.3, 64x4096x4096 10.7 -> 8.5, 128x1024x2048 7.2 -> 4.7, 256x1024x4096 10.7 -> 6.9,
//                      512x512x4096 10.7 -> 7.1, 4096x64x3072 9.3 -> 6.0; 100x768x6144 9.7 -> 7.1 and 4096x64x64 3.6 -> 3.4 gain
//                      least, 100x768x8192 9.3 -> 8.7 and 65x1000x8192 9.0 -> 11.8 lie beyond
//   int8, 32 columns:  512x1024x2048 7.6 -> 5.7, 200x2000x4096 12.8 -> 7.9, 4096x128x3072 9.6 -> 7.2, 64x8192x6144 16.3 -> 13.9;
//                      512x1024x128 3.5 -> 3.9 is the loss at the short end (one K tile of the 64 tile: from 256 bytes on)
//   binary16, the same bytes: within 2 % of the int8 times.
// A product whose maximum, codes or accumulators are wanted too stays on the tiles, whose epilogue has them: with the maximum
// 64x128x128 int8 3.7 us (here, without it, 3.3), 45x4096x1024 5.6 (3.9), 512x1024x2048 7.9 (5.7); binary16 1.2 to 2.1 times.
int rows_columns(const GemmProblem& p)
{
    const int64_t bytes = p.K * (p.prec / 8), rows = (p.M + 63) / 64;
    if(bytes > (p.M <= 32 ? 8192 : 6144)) return 0;
    if(rows * ((p.N + 15) / 16) <= (p.M <= 16 ? 2 * kRowsGroups : kRowsGroups)) return 1;
    return bytes > 256 && rows * ((p.N + 31) / 32) <= kRowsGroups ? 2 : 0;
}

}  // namespace

static int token_rows_columns(const TokenProduct& p)
{
    GemmProblem shape{};
    shape.prec = 8; shape.M = p.rows; shape.N = p.N; shape.K = code_pad(p.K);
    return p.offsets || p.sets != 1 || p.K == 0 ? 0 : rows_columns(shape);
}
bool token_rows_takes(const TokenProduct& p) { return token_rows_columns(p) != 0; }

hipError_t launch_token_rows(const TokenProduct& p, bool* taken, hipStream_t st)
{
    const int columns = token_rows_columns(p);
    *taken = columns != 0;
    if(!*taken) return hipSuccess;
    GemmKernelArgs a{};
    a.A = reinterpret_cast<const uint8_t*>(p.A);
    a.B = reinterpret_cast<const uint8_t*>(p.B);
    a.M = p.rows; a.N = p.N; a.Kb = code_pad(p.K);
    a.C = p.C; a.c_is_f16 = p.c_dtype == kF16 ? 1 : p.c_dtype == kBF16 ? 2 : 0;
    a.row_scale = p.sa; a.col_scale = p.sb; a.col_bias = p.bias;
    return launch_rows<I8Traits, true>(a, columns, st);
}

bool gemm_rows_takes(const GemmProblem& p)
{
    if((p.prec != 8 && p.prec != 16) || p.tn || p.conv_H > 0 || p.b_remap_C > 0 || p.acc_dump || p.out_amax_bits || p.out_codes) return false;
    return rows_columns(p) != 0;
}

hipError_t launch_gemm_rows(const GemmProblem& p, bool* taken, hipStream_t st)
{
    *taken = gemm_rows_takes(p);
    if(!*taken) return hipSuccess;
    const int columns = rows_columns(p);
    GemmKernelArgs a{};
    a.A = static_cast<const uint8_t*>(p.A);
    a.B = static_cast<const uint8_t*>(p.B);
    a.M = p.M; a.N = p.N; a.Kb = p.K * (p.prec / 8);
    a.C = p.C; a.c_is_f16 = p.c_dtype == kF16;
    a.s0 = p.s0; a.s1 = p.s1; a.col_scale = p.col_scale; a.col_bias = p.col_bias;
    return p.prec == 8 ? launch_rows<I8Traits>(a, columns, st) : launch_rows<F16Traits>(a, columns, st);
}

}  // namespace qsync
