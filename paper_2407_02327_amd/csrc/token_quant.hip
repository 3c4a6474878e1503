// INT8 codes with a scale for each row (token) of a matrix, for each column of each set of its rows, or both.
//
// Rows only (serving; the forward pass without a backward): a row stays in the registers of 64 or 256 threads between its maximum and
// its codes, so x is read once.  Both (training): the codes along the columns contract over the rows, in the weight gradient; a first pass leaves
// the maxima of rows and columns, a second reads x again and writes both sets of codes, the second one transposed through LDS.
#include "device_utils.h"
#include "row_ops.h"
#include "token_ops.h"

#include <type_traits>

namespace qsync {

namespace {

struct TokenSource      // where the matrix's rows come from
{
    const void*    x;
    int64_t        x_rows, cols, ld, rows;
    const int32_t* source;      // row r is x's row source[r] / group; nullptr: row r
    int            group;
};
// x's row of row r, or -1: there is none
__device__ __forceinline__ int64_t source_row(const TokenSource& s, int64_t r)
{
    if(!s.source) return r;
    const int32_t i = s.source[r];
    return i >= 0 && i / s.group < s.x_rows ? i / s.group : -1;
}

template <typename T> __device__ __forceinline__ void load8(const T* row, int64_t c, int64_t cols, Row8<T>& v)
{
    if(c + 8 <= cols) v.load(row + c);
    else
    {
        float e[8];
#pragma unroll
        for(int i = 0; i < 8; ++i) e[i] = c + i < cols ? row_element(row + c + i) : 0.0f;
        v.encode(e);
    }
}
// (bits of the largest magnitude: of the values as they are, NaN among them)
template <typename T> __device__ __forceinline__ uint32_t max8(const Row8<T>& v, uint32_t m)
{
    float e[8];
    v.decode(e);
#pragma unroll
    for(int i = 0; i < 8; ++i) m = max(m, abs_bits(e[i]));
    return m;
}
// Codes in as few vector operations as they take (with the general quantizer's,
// about twice as many, the vector unit is as busy as the memory).  A slice's own inverse keeps its products within 127 and a rounding:
//   nearest: adding 1.5 2^23 leaves the integer, to nearest even, in the low byte of the sum;
//   stochastic: floor(v) likewise, and 1 more where u < floor(fl(v - floor(v)) 2^16), the carry of that + 65535 - u into bit 16.  (The difference is
//   rounded to 32 bits, as the oracle's is: floor(v 2^16) would be four operations less, and another code for one negative v above -1/2 in 2^25.)
// The inverse of a slice that is not finite is 0, and the product by the rule that zero times anything is zero.
template <int RND, int J> __device__ __forceinline__ uint32_t code_word(float x, float inv, const uint32_t (&not_u)[4])
{
    float v;
    asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(v) : "v"(x), "v"(inv));
    if constexpr(RND == kStochastic)
    {
        v = __builtin_amdgcn_fmed3f(v, -127.0f, 127.0f);
        const float down = floorf(v), part = v - down;
        return add_half<1>(static_cast<int>(__float_as_uint(down + 12582912.0f)), add_half<J % 2>(static_cast<int>(static_cast<uint32_t>(part * 65536.0f)), not_u[J / 2]));
    }
    else return __float_as_uint(v + 12582912.0f);
}
__device__ __forceinline__ uint32_t pack_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_amdgcn_perm(b, a, 0x0C0C0400u) | __builtin_amdgcn_perm(d, c, 0x04000C0Cu);
}
template <int RND> __device__ __forceinline__ uint2 codes8(const float (&e)[8], float f, const uint32_t (&u)[4])
{
    return make_uint2(pack_codes(code_word<RND, 0>(e[0], f, u), code_word<RND, 1>(e[1], f, u), code_word<RND, 2>(e[2], f, u), code_word<RND, 3>(e[3], f, u)),
                      pack_codes(code_word<RND, 4>(e[4], f, u), code_word<RND, 5>(e[5], f, u), code_word<RND, 6>(e[6], f, u), code_word<RND, 7>(e[7], f, u)));
}
// the complements of the draws of a block of eight elements
template <int RND> __device__ __forceinline__ void draws8(uint64_t seed, uint64_t offset, int64_t group, uint32_t (&not_u)[4])
{
    if constexpr(RND == kStochastic)
    {
        const uint4 b = philox_group(seed, offset, static_cast<uint64_t>(group));
        not_u[0] = ~b.x; not_u[1] = ~b.y; not_u[2] = ~b.z; not_u[3] = ~b.w;
    }
}
__device__ __forceinline__ uint32_t wave_max(uint32_t m)
{
#pragma unroll
    for(int off = 32; off >= 1; off >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), off)));
    return m;
}

template <typename T, int RND, int THREADS, int V>
__global__ __launch_bounds__(256) void token_rows_kernel(TokenSource s, const int32_t* count, uint64_t seed, uint64_t offset, float* scale, int8_t* q)
{
    constexpr int kRows = 256 / THREADS;
    __shared__ uint32_t part[4];
    const int     t = threadIdx.x % THREADS;
    const int64_t r = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / THREADS;
    const int64_t rows = count ? min(s.rows, static_cast<int64_t>(*count)) : s.rows;
    if(r >= rows) return;      // (a whole workgroup, or whole wavefronts that meet no barrier)
    const int64_t from = source_row(s, r), groups = code_pad(s.cols) / 8, per_row = (s.cols + 7) / 8;
    const T*      row = static_cast<const T*>(s.x) + (from < 0 ? 0 : from) * s.ld;
    const int64_t cols = from < 0 ? 0 : s.cols;
    Row8<T>       v[V];
    uint32_t      m = from < 0 ? 0x7FC00000u : 0u;
#pragma unroll
    for(int i = 0; i < V; ++i)
    {
        load8(row, (i * THREADS + t) * 8, cols, v[i]);
        m = max8(v[i], m);
    }
    for(int64_t g = V * THREADS + t; g < groups; g += THREADS)
    {
        Row8<T> w;
        load8(row, g * 8, cols, w);
        m = max8(w, m);
    }
    m = wave_max(m);
    if constexpr(THREADS > 64)
    {
        if(threadIdx.x % 64 == 0) part[threadIdx.x / 64] = m;
        __syncthreads();
        m = max(max(part[0], part[1]), max(part[2], part[3]));
    }
    const CodeScale cs = code_scale(m);
    if(t == 0) scale[r] = cs.scale;
    int8_t* out = q + r * groups * 8;
    auto put = [&](const Row8<T>& w, int64_t g) {
        float    e[8];
        uint32_t u[4];
        w.decode(e);
        draws8<RND>(seed, offset, r * per_row + g, u);
        *reinterpret_cast<uint2*>(out + g * 8) = codes8<RND>(e, cs.inv, u);
    };
#pragma unroll
    for(int i = 0; i < V; ++i)
        if(i * THREADS + t < groups) put(v[i], i * THREADS + t);
    for(int64_t g = V * THREADS + t; g < groups; g += THREADS)
    {
        Row8<T> w;
        load8(row, g * 8, cols, w);
        put(w, g);
    }
}

template <typename T, int RND>
hipError_t launch_rows(const TokenSource& s, const int32_t* count, uint64_t seed, uint64_t offset, float* scale, int8_t* q, hipStream_t st)
{
    const int64_t groups = code_pad(s.cols) / 8;
    const dim3    few(static_cast<unsigned>((s.rows + 3) / 4)), one(static_cast<unsigned>(s.rows));
    if(groups <= 64) token_rows_kernel<T, RND, 64, 1><<<few, 256, 0, st>>>(s, count, seed, offset, scale, q);
    else if(groups <= 128) token_rows_kernel<T, RND, 64, 2><<<few, 256, 0, st>>>(s, count, seed, offset, scale, q);
    else if(groups <= 256) token_rows_kernel<T, RND, 256, 1><<<one, 256, 0, st>>>(s, count, seed, offset, scale, q);
    else if(groups <= 512) token_rows_kernel<T, RND, 256, 2><<<one, 256, 0, st>>>(s, count, seed, offset, scale, q);
    else token_rows_kernel<T, RND, 256, 4><<<one, 256, 0, st>>>(s, count, seed, offset, scale, q);
    return hipGetLastError();
}

// ---- rows and columns ------------------------------------------------------------------------------------------------------------
// The rows' axis is walked in chunks of 128 positions (see set_start): a chunk lies in one set.
struct Chunk { int64_t set, first, row0, start; int len; };      // (first: the set's first position / len: rows of the chunk, <= 0: none)
// (The set is the last one that starts at or before the chunk: each wavefront's lanes look at one each, 64 at a time.  A search by halves, a
// memory latency a step, took 6 of the 12 us of a launch over 37 sets.)
__device__ __forceinline__ Chunk chunk_rows(const int32_t* offsets, int64_t rows, int64_t sets, int64_t chunk)
{
    const int64_t p = chunk * kCodePad;
    int64_t       set = 0;
    if(!offsets) set = min(p / code_pad(rows / sets), sets - 1);
    else
        for(int64_t e0 = 0; e0 < sets; e0 += 64)
        {
            const int64_t e = e0 + threadIdx.x % 64;
            bool          from = false;
            if(e < sets)
            {
                int64_t a = offsets[e];
                a    = a < 0 ? 0 : a > rows ? rows : a;
                from = code_pad(a) + kCodePad * e <= p;
            }
            set += __popcll(__ballot(from));
        }
    if(offsets) set = max(static_cast<int64_t>(0), set - 1);
    const SetRows s = set_rows(offsets, rows, sets, set);
    const int64_t start = set_start(offsets, s, set), left = s.len - (p - start);
    return {set, start, s.first + (p - start), p - start, static_cast<int>(p < start || left < 0 ? 0 : left > kCodePad ? kCodePad : left)};
}

// First pass: maxima of 128 columns (eight a lane) over a chunk and of the chunk's rows over those columns.  Sixteen lanes stand side by side, so
// a workgroup has sixteen rows at a time and, with all eight of a lane's loads requested before the first is used, 32 to 64 KB in flight.
// With 512 columns, a row a wavefront and one load in flight a chunk took 30 us whatever its size.
// rowpart [column tiles][rows], colpart [chunks][cols]: maxima, sums
// A matrix of few such workgroups goes in quarters of a chunk (2187x1001 fp32 with sums, 144 of them: 8.5 -> 6.3 us).
constexpr int      kStatCols = 128, kStatRows = 32;
constexpr uint32_t kStatFew  = 1024;
__device__ __forceinline__ uint32_t max_of_16(uint32_t v)
{
    auto step = [&](auto ctrl) { v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), decltype(ctrl)::value, 0xF, 0xF, false))); };
    step(std::integral_constant<int, kRotate + 8>{});
    step(std::integral_constant<int, kRotate + 4>{});
    step(std::integral_constant<int, kRotate + 2>{});
    step(std::integral_constant<int, kRotate + 1>{});
    return v;
}
struct BothArgs      // one matrix's part in the three passes
{
    TokenSource    s;
    const int32_t* offsets;
    int64_t        sets;
    uint32_t       chunks, pieces, stat_tiles, code_tiles, scale_blocks, col_blocks;      // (pieces: of a chunk in the first pass; scale_blocks: of rows and columns, those of the columns first)
    uint32_t *     rowpart, *colmax;
    float *        colsum, *row_scale, *row_inv, *col_scale, *col_inv, *sum_out;
    int8_t *       q, *qT;
    __host__ __device__ uint32_t stat_blocks() const { return chunks * pieces * stat_tiles; }
};
template <bool SUM> struct StatsLds
{
    uint32_t lmax[4][kStatCols];
    float    lsum[SUM ? 4 : 1][SUM ? kStatCols : 1];
};
template <typename T, bool SUM, int R> __device__ __forceinline__ void stats_body(const BothArgs& p, uint32_t block, StatsLds<SUM>& lds)
{
    const TokenSource& s = p.s;
    const int32_t*     offsets = p.offsets;
    const int64_t      sets = p.sets;
    const uint32_t     tiles = p.stat_tiles;
    uint32_t *const    rowpart = p.rowpart, *const colmax = p.colmax;
    float* const       colsum = p.colsum;
    auto&              lmax = lds.lmax;
    [[maybe_unused]] auto& lsum = lds.lsum;
    const int     lane = threadIdx.x % 64, wave = threadIdx.x / 64, side = threadIdx.x % 16, down = threadIdx.x / 16;
    const uint32_t tile = block % tiles, piece = block / tiles;
    Chunk          c = chunk_rows(offsets, s.rows, sets, piece / (kCodePad / R));
    const int      skip = static_cast<int>(piece % (kCodePad / R)) * R;
    c.row0 += skip;
    c.len = min(c.len - skip, R);
    const int64_t col = static_cast<int64_t>(tile) * kStatCols + side * 8;
    if(c.len <= 0)
    {   // (a piece behind its chunk's rows is folded like the others)
        const int64_t at = static_cast<int64_t>(tile) * kStatCols + threadIdx.x;
        if(threadIdx.x < kStatCols && at < s.cols)
        {
            colmax[piece * s.cols + at] = 0u;
            if constexpr(SUM) colsum[piece * s.cols + at] = 0.0f;
        }
        return;
    }
    constexpr int N = R / 16;
    Row8<T>       v[N];
    bool          there[N];
#pragma unroll
    for(int i = 0; i < N; ++i)
    {
        const int64_t from = down + i * 16 < c.len ? source_row(s, c.row0 + down + i * 16) : 0;
        there[i] = from >= 0;
        load8(static_cast<const T*>(s.x) + (from < 0 ? 0 : from) * s.ld, col, from < 0 || down + i * 16 >= c.len ? 0 : s.cols, v[i]);
    }
    uint32_t m[8];
    float    sum[8];
#pragma unroll
    for(int j = 0; j < 8; ++j) { m[j] = 0u; sum[j] = 0.0f; }
#pragma unroll
    for(int i = 0; i < N; ++i)
    {
        float e[8];
        v[i].decode(e);
        uint32_t rm = 0u;
        if(!there[i])
#pragma unroll
            for(int j = 0; j < 8; ++j) e[j] = __uint_as_float(0x7FC00000u);
#pragma unroll
        for(int j = 0; j < 8; ++j)
        {
            const uint32_t a = abs_bits(e[j]);
            m[j] = max(m[j], a);
            rm   = max(rm, a);
            if constexpr(SUM) sum[j] += e[j];
        }
        rm = max_of_16(rm);
        if(side == 0 && down + i * 16 < c.len) rowpart[tile * s.rows + c.row0 + down + i * 16] = rm;
    }
#pragma unroll
    for(int j = 0; j < 8; ++j)
    {
#pragma unroll
        for(int off = 16; off < 64; off <<= 1)
        {
            m[j] = max(m[j], static_cast<uint32_t>(__shfl_xor(static_cast<int>(m[j]), off)));
            if constexpr(SUM) sum[j] += __shfl_xor(sum[j], off);
        }
        if(lane < 16)
        {
            lmax[wave][lane * 8 + j] = m[j];
            if constexpr(SUM) lsum[wave][lane * 8 + j] = sum[j];
        }
    }
    __syncthreads();
    const int     i  = threadIdx.x;
    const int64_t at = static_cast<int64_t>(tile) * kStatCols + i;
    if(i >= kStatCols || at >= s.cols) return;
    colmax[piece * s.cols + at] = max(max(lmax[0][i], lmax[1][i]), max(lmax[2][i], lmax[3][i]));
    if constexpr(SUM) colsum[piece * s.cols + at] = (lsum[0][i] + lsum[1][i]) + (lsum[2][i] + lsum[3][i]);
}

// R: rows of a workgroup, all of a chunk's or a quarter (BothArgs::pieces)
template <typename T, bool SUM, int R> __global__ __launch_bounds__(256) void token_stats_kernel(const BothArgs p)
{
    __shared__ StatsLds<SUM> lds;
    stats_body<T, SUM, R>(p, blockIdx.x, lds);
}
// of two matrices, `a` first
template <typename TA, typename TB, int R> __global__ __launch_bounds__(256) void token_stats_pair_kernel(const BothArgs a, const BothArgs b)
{
    __shared__ StatsLds<false> lds;
    const uint32_t n = a.stat_blocks();
    if(blockIdx.x < n) stats_body<TA, false, R>(a, blockIdx.x, lds);
    else               stats_body<TB, false, R>(b, blockIdx.x - n, lds);
}

// Scales and inverse scales of the rows (workgroups behind `col_blocks`) and of the sets' columns: sixteen threads fold a column's chunks,
// every sixteenth each, then their results in order (one thread a column took 35 us for 128 chunks).
template <bool SUM> __device__ __forceinline__ void scales_body(const BothArgs& p, uint32_t block, uint32_t (&lmax)[16][16], float (&lsum)[16][16])
{
    const int32_t* offsets = p.offsets;
    const int64_t  rows = p.s.rows, cols = p.s.cols, sets = p.sets, col_blocks = p.col_blocks;
    const int      col_tiles = static_cast<int>(p.stat_tiles);
    const uint32_t *rowpart = p.rowpart, *colmax = p.colmax;
    const float*    colsum = p.colsum;
    float *         row_scale = p.row_scale, *row_inv = p.row_inv, *col_scale = p.col_scale, *col_inv = p.col_inv, *sum_out = p.sum_out;
    if(block >= col_blocks)
    {
        const int64_t r = (static_cast<int64_t>(block) - col_blocks) * 256 + threadIdx.x;
        if(r >= rows || (offsets && r >= offsets[sets])) return;
        uint32_t m = 0u;
        for(int t0 = 0; t0 < col_tiles; t0 += 8)
        {
            uint32_t o[8];
#pragma unroll
            for(int u = 0; u < 8; ++u) o[u] = rowpart[(t0 + u < col_tiles ? t0 + u : 0) * rows + r];
#pragma unroll
            for(int u = 0; u < 8; ++u) m = max(m, o[u]);
        }
        const CodeScale cs = code_scale(m);
        row_scale[r] = cs.scale;
        row_inv[r]   = cs.inv;
        return;
    }
    const int     side = threadIdx.x % 16, part = threadIdx.x / 16;
    const int64_t tiles = (cols + 15) / 16, e = block / tiles, c = block % tiles * 16 + side, cc = c < cols ? c : cols - 1;
    const SetRows s = set_rows(offsets, rows, sets, e);
    const int64_t first = set_start(offsets, s, e) / kCodePad * p.pieces, end = first + code_pad(s.len) / kCodePad * p.pieces;
    uint32_t      m = 0u;
    float         sum = 0.0f;
    for(int64_t k0 = first + part; k0 < end; k0 += 64)
    {
        uint32_t o[4];
        float    f[4];
#pragma unroll
        for(int u = 0; u < 4; ++u)
        {
            const int64_t k = k0 + u * 16 < end ? k0 + u * 16 : k0;
            o[u] = colmax[k * cols + cc];
            if constexpr(SUM) f[u] = colsum[k * cols + cc];
        }
#pragma unroll
        for(int u = 0; u < 4; ++u)
        {
            m = max(m, o[u]);
            if constexpr(SUM) sum += k0 + u * 16 < end ? f[u] : 0.0f;
        }
    }
    lmax[part][side] = m;
    if constexpr(SUM) lsum[part][side] = sum;
    __syncthreads();
    if(part != 0 || c >= cols) return;
#pragma unroll
    for(int i = 1; i < 16; ++i)
    {
        m = max(m, lmax[i][side]);
        if constexpr(SUM) sum += lsum[i][side];
    }
    const CodeScale cs = code_scale(m);
    col_scale[e * cols + c] = cs.scale;
    col_inv[e * cols + c]   = cs.inv;
    if constexpr(SUM) sum_out[e * cols + c] = sum;
}

template <bool SUM> __global__ __launch_bounds__(256) void token_scales_kernel(const BothArgs p)
{
    __shared__ uint32_t lmax[16][16];
    __shared__ float    lsum[16][16];
    scales_body<SUM>(p, blockIdx.x, lmax, lsum);
}
__global__ __launch_bounds__(256) void token_scales_pair_kernel(const BothArgs a, const BothArgs b)
{
    __shared__ uint32_t lmax[16][16];
    __shared__ float    lsum[16][16];
    const bool first = blockIdx.x < a.scale_blocks;
    scales_body<false>(first ? a : b, first ? blockIdx.x : blockIdx.x - a.scale_blocks, lmax, lsum);
}

// (Both passes walk the matrix row after row, the second one from its end: what the first one read last still lies in front of the memory.)
// 128 positions x 64 columns a workgroup: a thread has four rows of eight columns, whose codes along the columns leave as words of four rows.
template <typename T, int RND> __device__ __forceinline__ void codes_body(const BothArgs& p, uint32_t back, uint64_t seed, uint64_t offset, uint32_t (&lds)[64 * 33])
{
    const TokenSource& s = p.s;
    const int32_t*     offsets = p.offsets;
    const int64_t      sets = p.sets;
    const float *      row_inv = p.row_inv, *col_inv = p.col_inv;
    int8_t *           q = p.q, *qT = p.qT;
    const uint32_t     tile = back % p.code_tiles;
    const Chunk        c = chunk_rows(offsets, s.rows, sets, back / p.code_tiles);
    if(c.len <= 0) return;
    const int     cg = threadIdx.x % 8, rq = threadIdx.x / 8;
    const int64_t col0 = static_cast<int64_t>(tile) * 64, col = col0 + cg * 8, per_row = (s.cols + 7) / 8, qcols = code_pad(s.cols);
    // (all loads before the first store, which might change what they read as far as the compiler knows)
    Row8<T> v[4];
    float   rf[4], ci[8];
#pragma unroll
    for(int i = 0; i < 4; ++i)
    {
        const bool    in = rq * 4 + i < c.len;
        const int64_t r = c.row0 + (in ? rq * 4 + i : 0), from = in ? source_row(s, r) : -1;
        load8(static_cast<const T*>(s.x) + (from < 0 ? 0 : from) * s.ld, col, from < 0 ? 0 : s.cols, v[i]);
        rf[i] = row_inv[r];
    }
#pragma unroll
    for(int j = 0; j < 8; ++j) ci[j] = col + j < s.cols ? col_inv[c.set * s.cols + col + j] : 0.0f;
    uint32_t k[4][8], w[8];
#pragma unroll
    for(int i = 0; i < 4; ++i)
    {
        const int64_t r = c.row0 + rq * 4 + i;
        float         e[8];
        uint32_t      u[4];
        v[i].decode(e);
        draws8<RND>(seed, offset, r * per_row + col / 8, u);
        if(rq * 4 + i < c.len) *reinterpret_cast<uint2*>(q + r * qcols + col) = codes8<RND>(e, rf[i], u);
        k[i][0] = code_word<RND, 0>(e[0], ci[0], u); k[i][1] = code_word<RND, 1>(e[1], ci[1], u);
        k[i][2] = code_word<RND, 2>(e[2], ci[2], u); k[i][3] = code_word<RND, 3>(e[3], ci[3], u);
        k[i][4] = code_word<RND, 4>(e[4], ci[4], u); k[i][5] = code_word<RND, 5>(e[5], ci[5], u);
        k[i][6] = code_word<RND, 6>(e[6], ci[6], u); k[i][7] = code_word<RND, 7>(e[7], ci[7], u);
    }
#pragma unroll
    for(int j = 0; j < 8; ++j) w[j] = pack_codes(k[0][j], k[1][j], k[2][j], k[3][j]);
#pragma unroll
    for(int j = 0; j < 8; ++j) lds[(cg * 8 + j) * 33 + rq] = w[j];
    __syncthreads();
    const SetRows set = set_rows(offsets, s.rows, sets, c.set);
    const int64_t ldt = code_pad(set.len);
    int8_t*       out = qT + c.first * s.cols + c.start;
#pragma unroll
    for(int k = 0; k < 2; ++k)
    {
        const int  i = threadIdx.x + k * 256, cc = i / 8, seg = i % 8;
        const uint32_t* at = lds + cc * 33 + seg * 4;
        if(col0 + cc < s.cols) *reinterpret_cast<uint4*>(out + (col0 + cc) * ldt + seg * 16) = make_uint4(at[0], at[1], at[2], at[3]);
    }
}

template <typename T, int RND> __global__ __launch_bounds__(256) void token_codes_kernel(const BothArgs p, uint64_t seed, uint64_t offset)
{
    __shared__ uint32_t lds[64 * 33];
    codes_body<T, RND>(p, gridDim.x - 1 - blockIdx.x, seed, offset, lds);
}
template <typename TA, typename TB> __global__ __launch_bounds__(256) void token_codes_pair_kernel(const BothArgs a, const BothArgs b)
{
    __shared__ uint32_t lds[64 * 33];
    const uint32_t      n = a.chunks * a.code_tiles, back = gridDim.x - 1 - blockIdx.x;
    if(back < n) codes_body<TA, kNearest>(a, back, 0, 0, lds);
    else         codes_body<TB, kNearest>(b, back - n, 0, 0, lds);
}

struct BothWorkspace { size_t rowpart, row_inv, col_inv, colmax, colsum, total; };
BothWorkspace both_workspace(int64_t rows, int64_t cols, int64_t sets, bool offsets)
{
    auto         up = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t chunks = static_cast<size_t>(code_positions(rows, sets, offsets) / kCodePad), tiles = static_cast<size_t>((cols + kStatCols - 1) / kStatCols);
    BothWorkspace w;
    w.rowpart = 0;
    w.row_inv = w.rowpart + up(tiles * rows * 4);
    w.col_inv = w.row_inv + up(static_cast<size_t>(rows) * 4);
    // (what is enough for some number of rows is enough for fewer: partial results of fewer chunks in more pieces)
    const size_t few = (kStatFew + tiles) / tiles * (kCodePad / kStatRows), parts = chunks * tiles < kStatFew ? chunks * (kCodePad / kStatRows) : chunks > few ? chunks : few;
    w.colmax  = w.col_inv + up(static_cast<size_t>(sets) * cols * 4);
    w.colsum  = w.colmax + up(parts * cols * 4);
    w.total   = w.colsum + up(parts * cols * 4);
    return w;
}

BothArgs both_args(const TokenMatrix& m, const TokenBoth& o)
{
    BothArgs             a{};
    const BothWorkspace  w = both_workspace(m.rows, m.cols, o.sets, o.offsets != nullptr);
    uint8_t* const       base = static_cast<uint8_t*>(o.workspace);
    a.s          = TokenSource{m.x, m.x_rows, m.cols, m.ld, m.rows, m.source, m.group};
    a.offsets    = o.offsets;
    a.sets       = o.sets;
    a.chunks     = static_cast<uint32_t>(code_positions(m.rows, o.sets, o.offsets != nullptr) / kCodePad);
    a.stat_tiles = static_cast<uint32_t>((m.cols + kStatCols - 1) / kStatCols);
    a.pieces     = a.chunks * a.stat_tiles < kStatFew ? kCodePad / kStatRows : 1;
    a.code_tiles = static_cast<uint32_t>(code_pad(m.cols) / 64);
    a.col_blocks = static_cast<uint32_t>(o.sets * ((m.cols + 15) / 16));
    a.scale_blocks = a.col_blocks + static_cast<uint32_t>((m.rows + 255) / 256);
    a.rowpart   = reinterpret_cast<uint32_t*>(base + w.rowpart);
    a.colmax    = reinterpret_cast<uint32_t*>(base + w.colmax);
    a.colsum    = reinterpret_cast<float*>(base + w.colsum);
    a.row_inv   = reinterpret_cast<float*>(base + w.row_inv);
    a.col_inv   = reinterpret_cast<float*>(base + w.col_inv);
    a.row_scale = o.row_scale;
    a.col_scale = o.col_scale;
    a.sum_out   = o.colsum;
    a.q         = o.q;
    a.qT        = o.qT;
    return a;
}
template <typename T, int RND> hipError_t launch_both(const BothArgs& a, uint64_t seed, uint64_t offset, hipStream_t st)
{
    const unsigned blocks = a.stat_blocks();
    if(a.sum_out)
    {
        if(a.pieces > 1) token_stats_kernel<T, true, kStatRows><<<blocks, 256, 0, st>>>(a);
        else             token_stats_kernel<T, true, kCodePad><<<blocks, 256, 0, st>>>(a);
        token_scales_kernel<true><<<a.scale_blocks, 256, 0, st>>>(a);
    }
    else
    {
        if(a.pieces > 1) token_stats_kernel<T, false, kStatRows><<<blocks, 256, 0, st>>>(a);
        else             token_stats_kernel<T, false, kCodePad><<<blocks, 256, 0, st>>>(a);
        token_scales_kernel<false><<<a.scale_blocks, 256, 0, st>>>(a);
    }
    token_codes_kernel<T, RND><<<a.chunks * a.code_tiles, 256, 0, st>>>(a, seed, offset);
    return hipGetLastError();
}
template <typename F> hipError_t with_type(int dtype, F&& f)
{
    return dtype == kF16 ? f(_Float16{}) : dtype == kBF16 ? f(__bf16{}) : f(float{});
}

}  // namespace

size_t token_both_workspace_bytes(int64_t rows, int64_t cols, int64_t sets, bool offsets) { return both_workspace(rows, cols, sets, offsets).total; }

hipError_t launch_token_quantize(const TokenMatrix& m, const int32_t* count, int rnd, uint64_t seed, uint64_t offset, float* scale, int8_t* q, hipStream_t st)
{
    const TokenSource s{m.x, m.x_rows, m.cols, m.ld, m.rows, m.source, m.group};
    return with_type(m.dtype, [&](auto tag) {
        typedef decltype(tag) T;
        if(rnd == kStochastic) return launch_rows<T, kStochastic>(s, count, seed, offset, scale, q, st);
        return launch_rows<T, kNearest>(s, count, seed, offset, scale, q, st);
    });
}

hipError_t launch_token_quantize_both(const TokenMatrix& m, const TokenBoth& o, int rnd, uint64_t seed, uint64_t offset, hipStream_t st)
{
    const BothArgs a = both_args(m, o);
    return with_type(m.dtype, [&](auto tag) {
        typedef decltype(tag) T;
        return rnd == kStochastic ? launch_both<T, kStochastic>(a, seed, offset, st) : launch_both<T, kNearest>(a, seed, offset, st);
    });
}

// Each pass of the two matrices in one launch.  (The launches of one beside the other's: what a small matrix's take is latency.)  One after the other where
// both together have more threads than a grid counts (2^32; the rest would not run, and no error would say so): columns' scales, 2^31 of one matrix at
// 2^27 columns of all the sets, and codes, 2^31 at 2^36 of them.
constexpr int64_t kGridBlocks = (int64_t(1) << 32) / 256;
hipError_t launch_token_quantize_pair(const TokenMatrix& m, const TokenBoth& o, const TokenMatrix& m2, const TokenBoth& o2, hipStream_t st)
{
    BothArgs a = both_args(m, o), b = both_args(m2, o2);
    auto     codes = [](const BothArgs& p) { return static_cast<int64_t>(p.chunks) * p.code_tiles; };
    if(static_cast<int64_t>(a.scale_blocks) + b.scale_blocks >= kGridBlocks || codes(a) + codes(b) >= kGridBlocks)
    {
        const hipError_t e = launch_token_quantize_both(m, o, kNearest, 0, 0, st);
        return e != hipSuccess ? e : launch_token_quantize_both(m2, o2, kNearest, 0, 0, st);
    }
    a.pieces = b.pieces = a.pieces > 1 && b.pieces > 1 ? a.pieces : 1;
    return with_type(m.dtype, [&](auto tag) {
        typedef decltype(tag) TA;
        return with_type(m2.dtype, [&](auto tag2) {
            typedef decltype(tag2) TB;
            if(a.pieces > 1) token_stats_pair_kernel<TA, TB, kStatRows><<<a.stat_blocks() + b.stat_blocks(), 256, 0, st>>>(a, b);
            else             token_stats_pair_kernel<TA, TB, kCodePad><<<a.stat_blocks() + b.stat_blocks(), 256, 0, st>>>(a, b);
            token_scales_pair_kernel<<<a.scale_blocks + b.scale_blocks, 256, 0, st>>>(a, b);
            token_codes_pair_kernel<TA, TB><<<a.chunks * a.code_tiles + b.chunks * b.code_tiles, 256, 0, st>>>(a, b);
            return hipGetLastError();
        });
    });
}

}  // namespace qsync
