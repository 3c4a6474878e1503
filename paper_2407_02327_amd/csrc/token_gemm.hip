// Products of INT8 codes with a scale for each row of either operand, C[m,n] = acc * (sa[m] sb[n]) + bias[n], over sets of rows (one: a
// linear operator; many: the experts of a layer, each with its own B).  In the forward pass and the data gradient a set owns rows of A and
// C; in the weight gradient it owns a stretch of the contraction axis and a whole C.
//
// A workgroup's tile is a tile of one set's product, computed as any other product's (gemm_tile.h: direct loads to LDS, 16x16 matrix
// instructions), with the rows' scales beside the columns' in LDS for the epilogue.  The host knows how many tiles there may be at most, from the sizes; which there
// are is read from the offsets by the workgroups, and those behind the last one end at once.
#include "gemm_tile.h"
#include "row_ops.h"
#include "token_ops.h"

namespace qsync {

namespace {

// The set and tile of a workgroup; false: none.  Like item_of_block, an XCD takes a contiguous share of the tiles, a set's in groups of rows.
struct SetTile { int64_t set; int tm, tn; };
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
template <int BM, int BN, bool WGRAD> __device__ __forceinline__ bool set_tile(const TokenProduct& p, int group_m, SetTile& t)
{
    const int tiles_n = static_cast<int>((p.N + BN - 1) / BN);
    if(WGRAD || !p.offsets)
    {
        const int     tiles_m = static_cast<int>(((WGRAD ? p.M : p.rows) + BM - 1) / BM);
        const int64_t tiles = static_cast<int64_t>(tiles_m) * tiles_n, item = item_of_xcd(blockIdx.x, tiles * p.sets);
        if(item < 0) return false;
        t.set = uniform64(item / tiles);
        tile_of(item - t.set * tiles, tiles_m, tiles_n, group_m, t);
        return true;
    }
    // lanes stand for sets, 64 at a time
    const int lane = threadIdx.x % kWaveSize;
    auto      rows_of = [&](int64_t e) { return e < p.sets ? static_cast<int>((set_rows(p.offsets, p.rows, p.sets, e).len + BM - 1) / BM) : 0; };
    int       all = 0;
    for(int64_t e = lane; e < p.sets; e += kWaveSize) all += rows_of(e);
#pragma unroll
    for(int off = kWaveSize / 2; off > 0; off >>= 1) all += __shfl_xor(all, off);
    int64_t item = item_of_xcd(blockIdx.x, static_cast<int64_t>(all) * tiles_n);
    if(item < 0) return false;
    for(int64_t e0 = 0; e0 < p.sets; e0 += kWaveSize)
    {
        const int n = rows_of(e0 + lane);
        int       upto = n;
#pragma unroll
        for(int off = 1; off < kWaveSize; off <<= 1)
        {
            const int o = __shfl_up(upto, off);
            if(lane >= off) upto += o;
        }
        const uint64_t behind = __ballot(static_cast<int64_t>(upto) * tiles_n > item);
        if(behind)
        {
            const int first = __builtin_ctzll(behind), mine = __shfl(n, first);
            item -= static_cast<int64_t>(__shfl(upto, first) - mine) * tiles_n;
            t.set = uniform64(e0 + first);
            tile_of(item, mine, tiles_n, group_m, t);
            return true;
        }
        item -= static_cast<int64_t>(__shfl(upto, kWaveSize - 1)) * tiles_n;
    }
    return false;
}

template <int BM, int BN, int WGM, int WGN, int ST, bool WGRAD>
__global__ __launch_bounds__(64 * WGM * WGN, 2) void token_gemm_kernel(const TokenProduct p, int group_m)
{
    SetTile t;
    if(!set_tile<BM, BN, WGRAD>(p, group_m, t)) return;
    SetRows s = set_rows(p.offsets, p.rows, p.sets, t.set);
    s = {uniform64(s.first), uniform64(s.len)};
    GemmKernelArgs a{};
    const int64_t  os = p.c_dtype == kF32 ? 4 : 2;
    a.N        = p.N;
    a.c_is_f16 = p.c_dtype == kF16 ? 1 : p.c_dtype == kBF16 ? 2 : 0;
    if constexpr(WGRAD)
    {
        const int64_t start = set_start(p.offsets, s, t.set);
        a.A = reinterpret_cast<const uint8_t*>(p.A) + start * p.M;
        a.B = reinterpret_cast<const uint8_t*>(p.B) + start * p.N;
        a.M = p.M;
        a.Kb = code_pad(s.len);
        a.C  = static_cast<uint8_t*>(p.C) + t.set * p.M * p.N * os;
        // (a set without rows has no scales worth the name: zeros)
        a.row_scale = s.len ? p.sa + t.set * p.M : nullptr;
        a.col_scale = s.len ? p.sb + t.set * p.N : nullptr;
    }
    else
    {
        a.Kb = code_pad(p.K);
        a.A = reinterpret_cast<const uint8_t*>(p.A) + s.first * a.Kb;
        a.B = reinterpret_cast<const uint8_t*>(p.B) + t.set * p.N * a.Kb;
        a.M = s.len;
        a.C = static_cast<uint8_t*>(p.C) + s.first * p.N * os;
        a.row_scale = a.Kb ? p.sa + s.first : nullptr;
        a.col_scale = a.Kb ? p.sb + t.set * p.N : nullptr;
        a.col_bias  = p.bias ? p.bias + t.set * p.N : nullptr;
    }
    gemm_tile_at<I8Traits, BM, BN, WGM, WGN, ST, 0, false, false, false, false, true>(a, 0, t.tm, t.tn);
}

constexpr int kMaxDevices = 16;
template <int BM, int BN, int WGM, int WGN, int ST, bool WGRAD> hipError_t launch_tiles(const TokenProduct& p, hipStream_t st)
{
    constexpr int lds = ST * (BM + BN) * kRowBytes + kColumnBytes<BN> + BM * 4;
    const auto    kernel = &token_gemm_kernel<BM, BN, WGM, WGN, ST, WGRAD>;
    static bool   attr_set[kMaxDevices] = {};      // per instantiation and device; benign if set twice
    int           dev = 0;
    const bool    known = hipGetDevice(&dev) == hipSuccess && dev >= 0 && dev < kMaxDevices;
    if(!known || !attr_set[dev])
    {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if(e != hipSuccess) return e;
        if(known) attr_set[dev] = true;
    }
    const int64_t tn = (p.N + BN - 1) / BN, tm = ((WGRAD ? p.M : p.rows) + BM - 1) / BM;
    // (each set may leave a part of a tile)
    int64_t tiles = WGRAD ? tm * tn * p.sets : (p.offsets ? (tm + p.sets < p.rows ? tm + p.sets : p.rows) : tm) * tn;
    if(tiles >= int64_t(1) << 31) return hipErrorInvalidValue;
    kernel<<<static_cast<unsigned>(tiles), 64 * WGM * WGN, lds, st>>>(p, kGroupM);
    return hipGetLastError();
}

template <bool WGRAD> hipError_t launch_product(const TokenProduct& p, hipStream_t st)
{
    // The tile: as for a product without sets of the same size
    const int64_t  M = WGRAD ? p.M : (p.rows + p.sets - 1) / p.sets, K = WGRAD ? (p.rows + p.sets - 1) / p.sets : p.K;
    const GemmPlan plan = plan_gemm(8, M * p.sets, p.N, code_pad(K), -1, -1, false);
    const int      tile = plan.tile == 0 && M < 192 ? 1 : plan.tile == 1 && M < 96 ? 2 : plan.tile;
    switch(tile)
    {
    case 0: return launch_tiles<256, 256, 2, 4, 2, WGRAD>(p, st);
    case 1: return launch_tiles<128, 128, 2, 4, 2, WGRAD>(p, st);
    default: return launch_tiles<64, 64, 2, 2, 2, WGRAD>(p, st);
    }
}

}  // namespace

hipError_t launch_token_product(const TokenProduct& p, bool wgrad, hipStream_t st)
{
    if(wgrad) return launch_product<true>(p, st);
    bool             taken;
    const hipError_t e = launch_token_rows(p, &taken, st);
    return taken || e != hipSuccess ? e : launch_product<false>(p, st);
}

}  // namespace qsync
