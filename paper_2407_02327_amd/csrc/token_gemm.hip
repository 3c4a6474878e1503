// Products of INT8 codes with a scale for each row of either operand, C[m,n] = acc * (sa[m] sb[n]) + bias[n], over sets of rows (one: a
// linear operator; many: the experts of a layer, each with its own B).  In the forward pass and the data gradient a set owns rows of A and
// C; in the weight gradient it owns a stretch of the contraction axis and a whole C.
//
// A workgroup's tile is a tile of one set's product, computed as any other product's (gemm_tile.h: direct loads to LDS, 16x16 matrix
// instructions), with the rows' scales beside the columns' in LDS for the epilogue.  The host knows how many tiles there may be at most, from the sizes; which there
// are is read from the offsets by the workgroups, and those behind the last one end at once.
#include "gemm_rows.h"
#include "gemm_tile.h"
#include "row_ops.h"
#include "token_ops.h"
#include <algorithm>

namespace qsync {

namespace {

// The set and tile of a workgroup; false: none.  Like item_of_block, an XCD takes a contiguous share of the tiles, a set's in groups of rows.
struct SetTile { int64_t set; SetRows rows; int tm, tn, quarter; };
__device__ __forceinline__ int64_t item_of_xcd(int64_t lin, int64_t total)
{
    const int64_t per = total / kNumXcd, rem = total % kNumXcd, xcd = lin % kNumXcd, loc = lin / kNumXcd;
    if(loc >= per + (xcd < rem ? 1 : 0)) return -1;
    return xcd * per + (xcd < rem ? xcd : rem) + loc;
}
__device__ __forceinline__ void tile_of(int64_t item, int tiles_m, int tiles_n, int group_m, SetTile& t)
{
    const int width = group_m * tiles_n, i = static_cast<int>(item), group = i / width, first = group * group_m;
    const int gsz = tiles_m - first < group_m ? tiles_m - first : group_m, in = i - group * width;
    t.tm = __builtin_amdgcn_readfirstlane(first + in % gsz);
    t.tn = __builtin_amdgcn_readfirstlane(in / gsz);
}
// Forward form.  `all` tiles of which the first `whole` stand for themselves; a last, incomplete round of the units (kRest tiles at most) goes
// in quarters, four times as many workgroups, where the kernel has them: 8 experts' 16384 rows by 1024 outputs, 4096 deep, are 272 tiles,
// 16 more than units.
constexpr int kRest = 64;
// (What stands in front of a workgroup's first load is paid once a tile.  The offsets are read once, a set a lane, and the set's rows come from that lane.)
__device__ __forceinline__ SetRows rows_of_lane(const SetRows& mine, int lane)
{
    return {static_cast<int64_t>(__builtin_amdgcn_readlane(static_cast<int>(mine.first), lane)), static_cast<int64_t>(__builtin_amdgcn_readlane(static_cast<int>(mine.len), lane))};
}
template <int BM, int BN, bool QUARTERS> __device__ __forceinline__ bool set_tile(const TokenProduct& p, uint32_t block, int group_m, SetTile& t)
{
    const int tiles_n = static_cast<int>((p.N + BN - 1) / BN), lane = threadIdx.x % kWaveSize;
    // lanes stand for sets, 64 at a time; `mine`, `tiles`, `upto`: of the 64 looked at last, tiles of the set and of those up to it
    SetRows mine{0, 0};
    int     tiles = 0, upto = 0;
    auto    look = [&](int64_t e0) {
        mine  = e0 + lane < p.sets ? set_rows(p.offsets, p.rows, p.sets, e0 + lane) : SetRows{0, 0};
        tiles = static_cast<int>((mine.len + BM - 1) / BM);
        upto  = tiles;
#pragma unroll
        for(int off = 1; off < kWaveSize; off <<= 1)
        {
            const int o = __shfl_up(upto, off);
            if(lane >= off) upto += o;
        }
        return __builtin_amdgcn_readlane(upto, kWaveSize - 1);
    };
    int tiles_m = 0;
    if(!p.offsets) tiles_m = static_cast<int>((p.rows + BM - 1) / BM);
    else
        for(int64_t e0 = 0; e0 < p.sets; e0 += kWaveSize) tiles_m += look(e0);
    const int64_t all = static_cast<int64_t>(tiles_m) * tiles_n;
    // (with three rounds and more the units do not end together, and a short last one is hidden)
    const int64_t rest = QUARTERS && all > kNumCu && all < 3 * kNumCu && all % kNumCu <= kRest ? all % kNumCu : 0, whole = all - rest;
    int64_t       item;
    t.quarter = -1;
    if(static_cast<int64_t>(block) < (whole + kNumXcd - 1) / kNumXcd * kNumXcd)
    {
        item = item_of_xcd(block, whole);
        if(item < 0) return false;
    }
    else
    {
        const int64_t q = static_cast<int64_t>(block) - (whole + kNumXcd - 1) / kNumXcd * kNumXcd;
        if(q >= 4 * rest) return false;
        item      = whole + q / 4;
        t.quarter = static_cast<int>(q % 4);
    }
    t.set  = 0;
    t.rows = SetRows{0, p.rows};
    if(!p.offsets)
    {
        tile_of(item, tiles_m, tiles_n, group_m, t);
        return true;
    }
    for(int64_t e0 = 0; e0 < p.sets; e0 += kWaveSize)
    {
        const int      sum = p.sets > kWaveSize ? look(e0) : tiles_m;
        const uint64_t behind = __ballot(static_cast<int64_t>(upto) * tiles_n > item);
        if(behind)
        {
            const int at = __builtin_ctzll(behind), n = __builtin_amdgcn_readlane(tiles, at);
            t.set  = e0 + at;
            t.rows = rows_of_lane(mine, at);
            tile_of(item - static_cast<int64_t>(__builtin_amdgcn_readlane(upto, at) - n) * tiles_n, n, tiles_n, group_m, t);
            return true;
        }
        item -= static_cast<int64_t>(sum) * tiles_n;
    }
    return false;
}
// Weight gradient: every set has the same tiles, but as long a contraction as it has rows.  An XCD takes a contiguous share of all tiles, or, with
// few sets of many tiles, an eighth of every set's, the longest sets first (16 sets of different size one after the other by XCD: half of the chip waits for the
// two longest, 16384 rows, 4096 x 1024 in 142 us, by eighths 124).  Eighths read every set's operands into all L2s, which costs where sets are alike or small.
// Share / eighths, bfloat16, us: 16384 rows, 1024 x 4096 4 sets 88 / 79, 8 98 / 70, 16 104 / 82, 23 118 / 100, 24 99 / 100, 32 125 / 119, 40 121 / 142, 64 168 / 215, 16 alike
// of 1024 x 2048 39 / 45; fewer tiles: 16384, 512 x 1024, 16 sets 19 / 22, 8192, 256 x 512, 8 sets 7.8 / 11.8, 4096, 128 x 256, 16 sets 4.3 / 5.2.  Over 213 draws of 2 to 64
// sets, 128 to 4096 either way, alike to very different: this rule is 1.3 % behind the faster one on average (28 % at most), up to 23 sets whatever their tiles
// 5.9 % (58 %), shares alone 3.0 % (a factor of 2), eighths alone 12.9 %.
__host__ __device__ constexpr bool by_eighths(bool offsets, int64_t sets, int64_t tiles, int BM)
{
    const int64_t least = BM == 256 ? 1 : BM == 128 ? 48 : 96, all = BM == 64 ? 2 * kNumCu : kNumCu;
    return offsets && sets <= 23 && tiles >= least && sets * tiles >= all;
}
template <int BM, int BN> __device__ __forceinline__ bool set_tile_wgrad(const TokenProduct& p, uint32_t block, int group_m, SetTile& t)
{
    const int tiles_m = static_cast<int>((p.M + BM - 1) / BM), tiles_n = static_cast<int>((p.N + BN - 1) / BN), tiles = tiles_m * tiles_n;
    t.quarter = -1;
    if(!by_eighths(p.offsets != nullptr, p.sets, tiles, BM))
    {
        const int64_t item = item_of_xcd(block, static_cast<int64_t>(tiles) * p.sets);
        if(item < 0) return false;
        t.set  = uniform64(item / tiles);
        t.rows = set_rows(p.offsets, p.rows, p.sets, t.set);
        tile_of(item - t.set * tiles, tiles_m, tiles_n, group_m, t);
        return true;
    }
    // Eight sets in a row give an XCD `tiles` tiles: of the q-th, per and one more where (xcd + q) % 8 < rem
    const int xcd = block % kNumXcd, loc = block / kNumXcd, per = tiles / kNumXcd, rem = tiles % kNumXcd;
    int       q = loc / tiles * kNumXcd, in = loc % tiles, first = 0;
    for(;; ++q)
    {
        const int turn = (xcd + q) % kNumXcd, n = per + (turn < rem ? 1 : 0);
        first = turn * per + (turn < rem ? turn : rem);
        if(in < n) break;
        in -= n;
    }
    if(q >= p.sets) return false;
    // the q-th by length; lanes stand for sets
    const int     lane = threadIdx.x % kWaveSize;
    const SetRows mine = lane < p.sets ? set_rows(p.offsets, p.rows, p.sets, lane) : SetRows{0, -1};
    const int     len = static_cast<int>(mine.len);
    int           rank = 0;
    for(int e = 0; e < p.sets; ++e)
    {
        const int other = __builtin_amdgcn_readlane(len, e);
        rank += other > len || (other == len && e < lane) ? 1 : 0;
    }
    const int at = __builtin_ctzll(__ballot(rank == q && lane < p.sets));
    t.set  = at;
    t.rows = rows_of_lane(mine, at);
    tile_of(first + in, tiles_m, tiles_n, group_m, t);
    return true;
}

// The contraction of one set's product in pieces (few tiles, long contractions): raw sums [splits][M][N], which a second launch adds up.
struct SplitArgs { void* partial; int splits, ktiles; };
template <int BM, int BN, int WGM, int WGN, int ST, bool WGRAD>
__global__ __launch_bounds__(64 * WGM * WGN, 2) void token_split_kernel(const TokenProduct p, const SplitArgs sp, int group_m)
{
    GemmKernelArgs a{};
    a.A = reinterpret_cast<const uint8_t*>(p.A);
    a.B = reinterpret_cast<const uint8_t*>(p.B);
    a.M = WGRAD ? p.M : p.rows;
    a.N = p.N;
    a.Kb = code_pad(WGRAD ? p.rows : p.K);
    a.partial = sp.partial;
    a.ktiles_per_split = sp.ktiles;
    a.tiles_m = static_cast<int>((a.M + BM - 1) / BM);
    a.tiles_n = static_cast<int>((a.N + BN - 1) / BN);
    int split, tm, tn;
    item_of_block(static_cast<int>(blockIdx.x), a.tiles_m, a.tiles_n, sp.splits, group_m, split, tm, tn);
    gemm_tile_at<I8Traits, BM, BN, WGM, WGN, ST, 0, true, false, false, false, true>(a, split, tm, tn);
}
// C from the pieces' sums: four consecutive columns a thread (VEC: N is a multiple of four) or one
template <bool VEC> __global__ __launch_bounds__(256) void token_reduce_kernel(const int32_t* partial, int splits, int64_t M, int64_t N, const float* sa, const float* sb, const float* bias, void* c, int cdt)
{
    constexpr int W = VEC ? 4 : 1;
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * W;
    if(i >= M * N) return;
    const int64_t m = i / N, n = i - m * N;
    int32_t       sum[W];
#pragma unroll
    for(int e = 0; e < W; ++e) sum[e] = 0;
    for(int s0 = 0; s0 < splits; s0 += 4)
    {
        int32_t o[4][W];
#pragma unroll
        for(int u = 0; u < 4; ++u)
        {
            const int32_t* at = partial + (s0 + u < splits ? s0 + u : s0) * M * N + i;
            if constexpr(VEC) *reinterpret_cast<int4*>(o[u]) = *reinterpret_cast<const int4*>(at);
            else o[u][0] = *at;
        }
#pragma unroll
        for(int u = 0; u < 4; ++u)
#pragma unroll
            for(int e = 0; e < W; ++e) sum[e] += s0 + u < splits ? o[u][e] : 0;
    }
    const float s = sa[m];
    float       f[W], b[W], v[W];
#pragma unroll
    for(int e = 0; e < W; ++e)
    {
        f[e] = s * sb[n + e];
        b[e] = bias ? bias[n + e] : 0.0f;
        v[e] = fmaf(static_cast<float>(sum[e]), f[e], b[e]);
    }
    if(cdt == kF16)
#pragma unroll
        for(int e = 0; e < W; ++e) static_cast<__half*>(c)[i + e] = fma_out<__half>(static_cast<float>(sum[e]), f[e], b[e]);
    else
#pragma unroll
        for(int e = 0; e < W; ++e) element_store(c, cdt, i + e, v[e]);
}

// A set's kernel arguments in the forward form
__device__ __forceinline__ GemmKernelArgs forward_args(const TokenProduct& p, int64_t set, const SetRows& s)
{
    GemmKernelArgs a{};
    a.N = p.N;
    a.c_is_f16 = p.c_dtype == kF16 ? 1 : p.c_dtype == kBF16 ? 2 : 0;
    a.Kb = code_pad(p.K);
    a.A = reinterpret_cast<const uint8_t*>(p.A) + s.first * a.Kb;
    a.B = reinterpret_cast<const uint8_t*>(p.B) + set * p.N * a.Kb;
    a.M = s.len;
    a.C = static_cast<uint8_t*>(p.C) + s.first * p.N * (p.c_dtype == kF32 ? 4 : 2);
    a.row_scale = a.Kb ? p.sa + s.first : nullptr;
    a.col_scale = a.Kb ? p.sb + set * p.N : nullptr;
    a.col_bias  = p.bias ? p.bias + set * p.N : nullptr;
    return a;
}
template <int BM, int BN, int WGM, int WGN, int ST, bool WGRAD>
__device__ __forceinline__ void product_body(const TokenProduct& p, uint32_t block, int group_m)
{
    constexpr bool QUARTERS = !WGRAD && BM == 256;
    SetTile        t;
    if constexpr(WGRAD)
    {
        if(!set_tile_wgrad<BM, BN>(p, block, group_m, t)) return;
    }
    else if(!set_tile<BM, BN, QUARTERS>(p, block, group_m, t)) return;
    const SetRows s{uniform64(t.rows.first), uniform64(t.rows.len)};
    GemmKernelArgs a;
    if constexpr(WGRAD)
    {
        const int64_t start = set_start(p.offsets, s, t.set);
        a = GemmKernelArgs{};
        a.N        = p.N;
        a.c_is_f16 = p.c_dtype == kF16 ? 1 : p.c_dtype == kBF16 ? 2 : 0;
        a.A = reinterpret_cast<const uint8_t*>(p.A) + start * p.M;
        a.B = reinterpret_cast<const uint8_t*>(p.B) + start * p.N;
        a.M = p.M;
        a.Kb = code_pad(s.len);
        a.C  = static_cast<uint8_t*>(p.C) + t.set * p.M * p.N * (p.c_dtype == kF32 ? 4 : 2);
        // (a set without rows has no scales worth the name: zeros)
        a.row_scale = s.len ? p.sa + t.set * p.M : nullptr;
        a.col_scale = s.len ? p.sb + t.set * p.N : nullptr;
    }
    else a = forward_args(p, t.set, s);
    if constexpr(QUARTERS)
        if(t.quarter >= 0)
        {
            const int tm = 2 * t.tm + t.quarter / 2, tn = 2 * t.tn + t.quarter % 2;
            if(tm * (BM / 2) < a.M && tn * (BN / 2) < a.N) gemm_tile_at<I8Traits, BM / 2, BN / 2, WGM, WGN, ST, 0, false, false, false, false, true>(a, 0, tm, tn);
            return;
        }
    gemm_tile_at<I8Traits, BM, BN, WGM, WGN, ST, 0, false, false, false, false, true>(a, 0, t.tm, t.tn);
}

template <int BM, int BN, int WGM, int WGN, int ST, bool WGRAD>
__global__ __launch_bounds__(64 * WGM * WGN, 2) void token_gemm_kernel(const TokenProduct p, int group_m)
{
    product_body<BM, BN, WGM, WGN, ST, WGRAD>(p, blockIdx.x, group_m);
}
// Sets of few rows whose 64 x 64 tiles leave units idle: a workgroup's wavefronts share the contraction.
template <int MF, int NF> __global__ __launch_bounds__(64 * kRowsWaves) void token_set_rows_kernel(const TokenProduct p)
{
    SetTile t;
    if(!set_tile<16 * MF, 16 * NF, false>(p, blockIdx.x, kGroupM, t)) return;
    const GemmKernelArgs a = forward_args(p, t.set, SetRows{uniform64(t.rows.first), uniform64(t.rows.len)});
    gemm_rows_tile<I8Traits, MF, NF, true>(a, static_cast<int64_t>(t.tm) * (16 * MF), static_cast<int64_t>(t.tn) * (16 * NF));
}
// Data and weight gradient side by side: each of them alone leaves units idle, and pays its own launch, first loads and drain.
template <int BM, int BN, int WGM, int WGN, int ST>
__global__ __launch_bounds__(64 * WGM * WGN, 2) void token_pair_kernel(const TokenProduct x, const TokenProduct w, uint32_t first, int group_x, int group_w)
{
    if(blockIdx.x < first) product_body<BM, BN, WGM, WGN, ST, false>(x, blockIdx.x, group_x);
    else                   product_body<BM, BN, WGM, WGN, ST, true>(w, blockIdx.x - first, group_w);
}

constexpr int kMaxDevices = 16;
template <typename F> hipError_t allow_lds(F kernel, int bytes, bool (&set)[kMaxDevices])      // (`set`: per instantiation and device; benign if set twice)
{
    int        dev = 0;
    const bool known = hipGetDevice(&dev) == hipSuccess && dev >= 0 && dev < kMaxDevices;
    if(known && set[dev]) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if(e == hipSuccess && known) set[dev] = true;
    return e;
}

// The tiles that there may be at most: each set may leave a part of one.  And the workgroups for them: the first tiles rounded up to the XCDs, a
// set's tiles shared out to eight of them, the last ones in quarters.
template <bool WGRAD> int64_t most_tiles(const TokenProduct& p, int BM, int BN)
{
    const int64_t tn = (p.N + BN - 1) / BN, tm = ((WGRAD ? p.M : p.rows) + BM - 1) / BM;
    return WGRAD ? tm * tn * p.sets : (p.offsets ? (tm + p.sets < p.rows ? tm + p.sets : p.rows) : tm) * tn;
}
template <bool WGRAD> int64_t blocks_of(const TokenProduct& p, int BM, int BN)
{
    const int64_t tiles = most_tiles<WGRAD>(p, BM, BN);
    if(!WGRAD) return tiles + kNumXcd + (BM == 256 ? 3 * kRest : 0);
    if(!by_eighths(p.offsets != nullptr, p.sets, tiles / p.sets, BM)) return (tiles + kNumXcd - 1) / kNumXcd * kNumXcd;
    const int64_t one = tiles / p.sets, left = p.sets % kNumXcd * (one / kNumXcd + 1);
    return kNumXcd * (p.sets / kNumXcd * one + (left < one ? left : one));
}
int wgrad_group(const TokenProduct& p, int BM, int BN) { return by_eighths(p.offsets != nullptr, p.sets, most_tiles<true>(p, BM, BN) / p.sets, BM) ? 4 : kGroupM; }

template <int BM, int BN, int WGM, int WGN, int ST, bool WGRAD> hipError_t launch_tiles(const TokenProduct& p, const SplitArgs& sp, hipStream_t st)
{
    constexpr int lds = ST * (BM + BN) * kRowBytes + kColumnBytes<BN> + BM * 4;
    const int64_t tiles = most_tiles<WGRAD>(p, BM, BN);
    static bool set[2][kMaxDevices] = {};
    if(sp.splits > 1)
    {
        const hipError_t e = allow_lds(&token_split_kernel<BM, BN, WGM, WGN, ST, WGRAD>, lds, set[0]);
        if(e != hipSuccess) return e;
        token_split_kernel<BM, BN, WGM, WGN, ST, WGRAD><<<static_cast<unsigned>(tiles * sp.splits), 64 * WGM * WGN, lds, st>>>(p, sp, kGroupM);
        return hipGetLastError();
    }
    const hipError_t e = allow_lds(&token_gemm_kernel<BM, BN, WGM, WGN, ST, WGRAD>, lds, set[1]);
    if(e != hipSuccess) return e;
    const int64_t blocks = blocks_of<WGRAD>(p, BM, BN);
    token_gemm_kernel<BM, BN, WGM, WGN, ST, WGRAD><<<static_cast<unsigned>(blocks), 64 * WGM * WGN, lds, st>>>(p, WGRAD ? wgrad_group(p, BM, BN) : kGroupM);
    return hipGetLastError();
}

// Tile and K splits: of one set, as of any other product of its size, the rows rounded up to a fragment's (so that few plans say what any number of
// rows may need); of several, without splits, no wider than their rows on average.
constexpr int64_t kPlanRows = 16;
GemmPlan product_plan(bool wgrad, int64_t rows, int64_t M, int64_t N, int64_t K, int64_t sets, bool offsets, int cdt)
{
    const int64_t share = (rows + sets - 1) / sets, k = code_pad(wgrad ? share : K);
    // Few K tiles and more outputs than a round of 256 tiles: two 128 tiles on a unit, of which one multiplies while the other stores (256 / 128 tile, us;
    // fp32: 8192x4096x128 42 / 28, 8192x3333x128 31 / 26, 16 sets of 1024x4096, 256 deep 73 / 59, 8 of 1024x2777, 384 deep 35 / 29, weight gradient
    // 8192x8192 of 128 78 / 52, of 4 sets 4096x4096 of 256 69 / 59; bfloat16: 16384x8192x128 76 / 70, 8192x4096x256 27 / 24, but 32768x4096x128 71 / 76; not: fp32 8192x4096x1024
    // 61 / 69, bfloat16 4096x4096x128 12 / 13, weight gradient of 32 sets 2048x2048 of 128 79 / 80).
    auto stores = [&](int64_t m) {
        const int64_t tiles = (m + 255) / 256 * ((N + 255) / 256);
        if(gemm_tile_pinned()) return false;
        return cdt == kF32 ? tiles > kNumCu && k <= (wgrad ? 256 : 384) : tiles >= 2 * kNumCu && k <= 256 && (!wgrad || !offsets);
    };
    if(!offsets)
    {
        const int64_t m = wgrad ? M : (rows + kPlanRows - 1) / kPlanRows * kPlanRows;
        GemmPlan      plan = plan_gemm(8, m, N, k, -1, -1, true);
        if(plan.tile == 0 && plan.splits == 1 && stores(m)) plan.tile = 1;
        // Operands beyond what the caches in front of the memory hold for them: the 256 tile, which reads half as much, in K splits instead of the
        // 128 tile without (weight gradients, 128 tile / 256 in pieces, us, operands from memory: 80 Mi 1024x4096 of 16384 rows 114 / 81, 64 Mi 2048x2048 of 16384
        // 111 / 78, 50 Mi 1024x4096 of 10240 73 / 62, 45 Mi of 9216 65 / 58; below, 40 Mi of 8192 57 / 55, 35 Mi of 7168 50 / 52, 32 Mi 2048x2048 of 8192 51 / 54, 24 Mi of 6144
        // 37 / 49; operands found in the caches: 80 Mi 80 / 75, 40 Mi 46 / 52)
        else if(!gemm_tile_pinned() && plan.tile == 1 && plan.splits == 1 && (m + N) * k >= (int64_t(44) << 20)) plan = plan_gemm(8, m, N, k, 0, 0, true);
        return plan;
    }
    const int64_t all = wgrad ? M * sets : rows;
    GemmPlan      plan = plan_gemm(8, all, N, k, -1, -1, false);
    const int64_t m = wgrad ? M : share;
    plan.tile = plan.tile == 0 && (m < 192 || stores(all)) ? 1 : plan.tile;
    plan.tile = plan.tile == 1 && m < 96 ? 2 : plan.tile;
    return plan;
}

// Workgroups (64 tiles of both gradients) up to which they share a launch; us, joined / apart: 300x200x100 of 3 sets 6.7 / 9.7, 2048x2048x1024 15.7 / 21.8,
// 1500x3000x700 18.9 / 29.8, 4000x1000x500 of 16 sets 25.0 / 32.9; 4096x1024x2048 (2576 workgroups) 34.4 / 32.6.
constexpr int64_t kPairBlocks = 8 * kNumCu, kPairBlocksSets = 16 * kNumCu;
template <int MF, int NF> hipError_t launch_set_rows(const TokenProduct& p, hipStream_t st)
{
    static bool      set[kMaxDevices] = {};
    const hipError_t e = allow_lds(&token_set_rows_kernel<MF, NF>, kRowsLds<MF, NF>, set);
    if(e != hipSuccess) return e;
    token_set_rows_kernel<MF, NF><<<static_cast<unsigned>(blocks_of<false>(p, 16 * MF, 16 * NF)), 64 * kRowsWaves, kRowsLds<MF, NF>, st>>>(p);
    return hipGetLastError();
}
// Row fragments of a workgroup (1: with one of columns, 4: with two), 0: the tiles are faster.  A 64 tile walks K alone, 0.45 us per 128 bytes, up to
// 512 of them at once; here a workgroup takes 0.37 us (0.95) for 512 bytes, with two of them on a unit (one).  us, bfloat16, tile / 1 / 4:
//   16 rows of 8 sets, 1024 x 4096 17.5 / 7.5 / 8.5; 128 of 8 17.7 / 11.0 / 10.6; 200 of 4, 256 x 8192 30.3 / 7.4 / 15.1; 2000 of 4, 200 x 4096 17.8 / 19.2 / 10.6;
//   64 of 16, 1024 x 1024 7.5 / 8.5 / 10.0; 256 of 8, 2048 x 2048 11.4 / 20.8 / 15.4; 512 of 8, 1024 x 4096 18.1 / 24.9 / 18.8.
int set_rows_fragments(const TokenProduct& p)
{
    if(!p.offsets || p.K == 0) return 0;
    const double kt = static_cast<double>(code_pad(p.K) / kRowBytes), sets = static_cast<double>(p.sets < p.rows ? p.sets : p.rows);
    auto         tiles = [&](int bm, int bn) { return std::max(static_cast<double>(p.rows) / bm + sets / 2, sets) * static_cast<double>((p.N + bn - 1) / bn); };
    const double tile = 2.0 + std::max(1.0, tiles(64, 64) / 512.0) * (1.5 + 0.45 * kt);
    const double one = 2.0 + std::max(1.0, tiles(16, 16) / 512.0) * (2.5 + 0.37 * kt / 4), four = 2.0 + std::max(1.0, tiles(64, 32) / 256.0) * (2.5 + 0.95 * kt / 4);
    return std::min(one, four) > 0.9 * tile ? 0 : one < four ? 1 : 4;
}

// The plan of a product, on a larger tile where its own has more threads than a grid counts (2^32).
template <bool WGRAD> bool countable(const TokenProduct& p, int tile)
{
    constexpr int side[3] = {256, 128, 64}, threads[3] = {512, 512, 256};
    return blocks_of<WGRAD>(p, side[tile], side[tile]) < (int64_t(1) << 32) / threads[tile];
}
template <bool WGRAD> GemmPlan countable_plan(const TokenProduct& p)
{
    GemmPlan plan = product_plan(WGRAD, p.rows, p.M, p.N, p.K, p.sets, p.offsets != nullptr, p.c_dtype);
    while(plan.tile > 0 && !countable<WGRAD>(p, plan.tile)) --plan.tile;
    return plan;
}

template <bool WGRAD> hipError_t launch_product(const TokenProduct& p, void* workspace, size_t workspace_bytes, hipStream_t st)
{
    const GemmPlan plan = countable_plan<WGRAD>(p);
    const int64_t  M = WGRAD ? p.M : p.rows, kt = code_pad(WGRAD ? p.rows : p.K) / kRowBytes;
    SplitArgs      sp{workspace, 1, 0};
    // (sums of integers: with less room there are fewer splits, and the same results)
    const size_t piece = static_cast<size_t>(M) * p.N * 4, room = workspace ? workspace_bytes / piece : 0;
    const int    splits = static_cast<int>(room < static_cast<size_t>(plan.splits) ? room : plan.splits);
    if(!p.offsets && splits > 1 && kt > 1)
    {
        sp.ktiles = static_cast<int>((kt + splits - 1) / splits);
        sp.splits = static_cast<int>((kt + sp.ktiles - 1) / sp.ktiles);
    }
    hipError_t e;
    switch(plan.tile)
    {
    case 0: e = launch_tiles<256, 256, 2, 4, 2, WGRAD>(p, sp, st); break;
    case 1: e = launch_tiles<128, 128, 2, 4, 2, WGRAD>(p, sp, st); break;
    default: e = launch_tiles<64, 64, 2, 2, 2, WGRAD>(p, sp, st);
    }
    if(e != hipSuccess || sp.splits == 1) return e;
    const int64_t  count = M * p.N, per = p.N % 4 == 0 ? 1024 : 256;
    const unsigned blocks = static_cast<unsigned>((count + per - 1) / per);
    const int32_t* partial = static_cast<const int32_t*>(workspace);
    if(p.N % 4 == 0) token_reduce_kernel<true><<<blocks, 256, 0, st>>>(partial, sp.splits, M, p.N, p.sa, p.sb, p.bias, p.C, p.c_dtype);
    else             token_reduce_kernel<false><<<blocks, 256, 0, st>>>(partial, sp.splits, M, p.N, p.sa, p.sb, p.bias, p.C, p.c_dtype);
    return hipGetLastError();
}

}  // namespace

// The largest need of any number of rows up to this one: fewer rows have fewer tiles, and those more splits.  (An operator of 8192 rows, 4096 outputs,
// 14336 deep, none of whose 8192 rows' tiles are split: with 64 rows and room for none 57 us, with room for their 8 splits 21; 400 rows 79, 55.)
size_t token_product_workspace_bytes(bool wgrad, int64_t rows, int64_t M, int64_t N, int64_t K, int64_t sets)
{
    if(sets != 1) return 0;
    // (the type moves tiles of unsplit products only)
    auto splits = [&](int64_t r) { return static_cast<size_t>(product_plan(wgrad, r, M, N, wgrad ? r : K, 1, false, kF32).splits); };
    // (Splits fill the units, with one workgroup of the 256 tile, two of the 128 or four of the 64 tile on each: none where an output has more than half as
    // many tiles as there are places, which is more than kNumCu / 2 of the 256 tile.)
    const int64_t tiles_n = (N + 255) / 256, tiles_m = kNumCu / 2 / tiles_n;
    if(wgrad)
    {
        if((M + 255) / 256 > tiles_m) return 0;
        size_t most = 1;
        for(int64_t r = kCodePad; r < rows + kCodePad; r += kCodePad) most = std::max(most, splits(r));      // (a plan knows the K tiles)
        return most > 1 ? most * M * N * 4 : 0;
    }
    const int64_t last = std::min(rows, tiles_m * 256);
    size_t        need = 0;      // rows times splits
    for(int64_t r = std::min(last, kPlanRows); r > 0; r = r < last ? std::min(last, r + kPlanRows) : 0)
    {
        const size_t s = splits(r);
        if(s > 1) need = std::max(need, s * r);
    }
    return need * N * 4;
}

bool token_product_countable(const TokenProduct& p, bool wgrad) { return wgrad ? countable<true>(p, 0) : countable<false>(p, 0); }

hipError_t launch_token_product(const TokenProduct& p, bool wgrad, void* workspace, size_t workspace_bytes, hipStream_t st)
{
    if(wgrad) return launch_product<true>(p, workspace, workspace_bytes, st);
    const int fragments = set_rows_fragments(p);
    if(fragments == 1) return launch_set_rows<1, 1>(p, st);
    if(fragments == 4) return launch_set_rows<4, 2>(p, st);
    bool             taken;
    const hipError_t e = launch_token_rows(p, &taken, st);
    return taken || e != hipSuccess ? e : launch_product<false>(p, workspace, workspace_bytes, st);
}

hipError_t launch_token_gradients(const TokenProduct& x, const TokenProduct& w, void* workspace, size_t workspace_bytes, hipStream_t st)
{
    const GemmPlan px = product_plan(false, x.rows, x.M, x.N, x.K, x.sets, x.offsets != nullptr, x.c_dtype), pw = product_plan(true, w.rows, w.M, w.N, w.K, w.sets, w.offsets != nullptr, w.c_dtype);
    const int64_t  first = (blocks_of<false>(x, 64, 64) + kNumXcd - 1) / kNumXcd * kNumXcd, all = first + blocks_of<true>(w, 64, 64);
    if(px.tile >= 1 && px.splits == 1 && pw.tile >= 1 && pw.splits == 1 && all <= (x.offsets ? kPairBlocksSets : kPairBlocks) && !token_rows_takes(x) && !set_rows_fragments(x))
    {
        constexpr int lds = 2 * (64 + 64) * kRowBytes + kColumnBytes<64> + 64 * 4;
        static bool   set[kMaxDevices] = {};
        const hipError_t e = allow_lds(&token_pair_kernel<64, 64, 2, 2, 2>, lds, set);
        if(e != hipSuccess) return e;
        token_pair_kernel<64, 64, 2, 2, 2><<<static_cast<unsigned>(all), 64 * 4, lds, st>>>(x, w, static_cast<uint32_t>(first), kGroupM, wgrad_group(w, 64, 64));
        return hipGetLastError();
    }
    const hipError_t e = launch_token_product(x, false, workspace, workspace_bytes, st);
    return e != hipSuccess ? e : launch_token_product(w, true, workspace, workspace_bytes, st);
}

}  // namespace qsync
