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
    auto    put = [&](const Row8<T>& w, int64_t g) {
        float e[8];
        w.decode(e);
        if(cs.inv == 0.0f)
#pragma unroll
            for(int j = 0; j < 8; ++j) e[j] = 0.0f;
        uint4 blk = make_uint4(0, 0, 0, 0);
        if constexpr(RND == kStochastic) blk = philox_group(seed, offset, static_cast<uint64_t>(r * per_row + g));
        uint32_t c[2];
        quantize_group<float, RND>(e, cs.inv, 127, blk, c);
        *reinterpret_cast<uint2*>(out + g * 8) = make_uint2(c[0], c[1]);
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
constexpr int kStatCols = 128;
__device__ __forceinline__ uint32_t max_of_16(uint32_t v)
{
    auto step = [&](auto ctrl) { v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), decltype(ctrl)::value, 0xF, 0xF, false))); };
    step(std::integral_constant<int, kRotate + 8>{});
    step(std::integral_constant<int, kRotate + 4>{});
    step(std::integral_constant<int, kRotate + 2>{});
    step(std::integral_constant<int, kRotate + 1>{});
    return v;
}
template <typename T, bool SUM>
__global__ __launch_bounds__(256) void token_stats_kernel(TokenSource s, const int32_t* offsets, int64_t sets, uint32_t tiles, uint32_t* rowpart, uint32_t* colmax, float* colsum)
{
    __shared__ uint32_t lmax[4][kStatCols];
    __shared__ float    lsum[SUM ? 4 : 1][SUM ? kStatCols : 1];
    const int     lane = threadIdx.x % 64, wave = threadIdx.x / 64, side = threadIdx.x % 16, down = threadIdx.x / 16;
    const uint32_t tile = blockIdx.x % tiles, chunk = blockIdx.x / tiles;
    const Chunk    c = chunk_rows(offsets, s.rows, sets, chunk);
    if(c.len <= 0) return;
    const int64_t col = static_cast<int64_t>(tile) * kStatCols + side * 8;
    constexpr int N = kCodePad / 16;
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
    colmax[chunk * s.cols + at] = max(max(lmax[0][i], lmax[1][i]), max(lmax[2][i], lmax[3][i]));
    if constexpr(SUM) colsum[chunk * s.cols + at] = (lsum[0][i] + lsum[1][i]) + (lsum[2][i] + lsum[3][i]);
}

// Scales and inverse scales of the rows (workgroups behind `col_blocks`) and of the sets' columns: sixteen threads fold a column's chunks,
// every sixteenth each, then their results in order (one thread a column took 35 us for 128 chunks).
template <bool SUM>
__global__ __launch_bounds__(256) void token_scales_kernel(const int32_t* offsets, int64_t rows, int64_t cols, int64_t sets, int64_t col_blocks, int col_tiles, const uint32_t* rowpart,
                                                           const uint32_t* colmax, const float* colsum, float* row_scale, float* row_inv, float* col_scale, float* col_inv, float* sum_out)
{
    if(blockIdx.x >= col_blocks)
    {
        const int64_t r = (static_cast<int64_t>(blockIdx.x) - col_blocks) * 256 + threadIdx.x;
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
    __shared__ uint32_t lmax[16][16];
    __shared__ float    lsum[16][16];
    const int     side = threadIdx.x % 16, part = threadIdx.x / 16;
    const int64_t tiles = (cols + 15) / 16, e = blockIdx.x / tiles, c = blockIdx.x % tiles * 16 + side, cc = c < cols ? c : cols - 1;
    const SetRows s = set_rows(offsets, rows, sets, e);
    const int64_t first = set_start(offsets, s, e) / kCodePad, end = first + code_pad(s.len) / kCodePad;
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

// (Both passes walk the matrix row after row, the second one from its end: what the first one read last still lies in front of the memory.)
// 128 positions x 64 columns a workgroup: a thread has four rows of eight columns, whose codes along the columns leave as words of four rows.
template <typename T, int RND>
__global__ __launch_bounds__(256) void token_codes_kernel(TokenSource s, const int32_t* offsets, int64_t sets, uint32_t tiles, uint64_t seed, uint64_t offset,
                                                          const float* row_inv, const float* col_inv, int8_t* q, int8_t* qT)
{
    __shared__ uint32_t lds[64 * 33];
    const uint32_t back = gridDim.x - 1 - blockIdx.x, tile = back % tiles;
    const Chunk    c = chunk_rows(offsets, s.rows, sets, back / tiles);
    if(c.len <= 0) return;
    const int     cg = threadIdx.x % 8, rq = threadIdx.x / 8;
    const int64_t col0 = static_cast<int64_t>(tile) * 64, col = col0 + cg * 8, per_row = (s.cols + 7) / 8, qcols = code_pad(s.cols);
    float         ci[8];
#pragma unroll
    for(int j = 0; j < 8; ++j) ci[j] = col + j < s.cols ? col_inv[c.set * s.cols + col + j] : 0.0f;
    uint32_t w[8];
#pragma unroll
    for(int j = 0; j < 8; ++j) w[j] = 0u;
#pragma unroll
    for(int i = 0; i < 4; ++i)
    {
        if(rq * 4 + i >= c.len) break;
        const int64_t r = c.row0 + rq * 4 + i, from = source_row(s, r);
        Row8<T>       v;
        float         e[8];
        load8(static_cast<const T*>(s.x) + (from < 0 ? 0 : from) * s.ld, col, from < 0 ? 0 : s.cols, v);
        v.decode(e);
        uint4 blk = make_uint4(0, 0, 0, 0);
        if constexpr(RND == kStochastic) blk = philox_group(seed, offset, static_cast<uint64_t>(r * per_row + col / 8));
        uint32_t    b[2];
        const float ri = row_inv[r];
        float       er[8];
#pragma unroll
        for(int j = 0; j < 8; ++j)
        {
            er[j] = ri == 0.0f ? 0.0f : e[j];
            e[j]  = ci[j] == 0.0f ? 0.0f : e[j];
        }
        quantize_group<float, RND>(er, ri, 127, blk, b);
        *reinterpret_cast<uint2*>(q + r * qcols + col) = make_uint2(b[0], b[1]);
#pragma unroll
        for(int j = 0; j < 8; ++j)
            w[j] |= (static_cast<uint32_t>(quantize_code<RND>(e[j], ci[j], 127, philox_draw16(blk, j))) & 0xFFu) << (8 * i);
    }
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

struct BothWorkspace { size_t rowpart, row_inv, col_inv, colmax, colsum, total; };
BothWorkspace both_workspace(int64_t rows, int64_t cols, int64_t sets, bool offsets)
{
    auto         up = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t chunks = static_cast<size_t>(code_positions(rows, sets, offsets) / kCodePad), tiles = static_cast<size_t>((cols + kStatCols - 1) / kStatCols);
    BothWorkspace w;
    w.rowpart = 0;
    w.row_inv = w.rowpart + up(tiles * rows * 4);
    w.col_inv = w.row_inv + up(static_cast<size_t>(rows) * 4);
    w.colmax  = w.col_inv + up(static_cast<size_t>(sets) * cols * 4);
    w.colsum  = w.colmax + up(chunks * cols * 4);
    w.total   = w.colsum + up(chunks * cols * 4);
    return w;
}

template <typename T, int RND>
hipError_t launch_both(const TokenSource& s, int64_t sets, const int32_t* offsets, uint64_t seed, uint64_t offset, float* row_scale, int8_t* q, float* col_scale, int8_t* qT,
                       float* colsum, void* workspace, hipStream_t st)
{
    const BothWorkspace w = both_workspace(s.rows, s.cols, sets, offsets != nullptr);
    uint8_t* const      base = static_cast<uint8_t*>(workspace);
    uint32_t*           rowpart = reinterpret_cast<uint32_t*>(base + w.rowpart);
    uint32_t*           cm = reinterpret_cast<uint32_t*>(base + w.colmax);
    float *             ri = reinterpret_cast<float*>(base + w.row_inv), *ci = reinterpret_cast<float*>(base + w.col_inv), *sm = reinterpret_cast<float*>(base + w.colsum);
    const unsigned      chunks = static_cast<unsigned>(code_positions(s.rows, sets, offsets != nullptr) / kCodePad);
    const unsigned      tiles = static_cast<unsigned>((s.cols + kStatCols - 1) / kStatCols);
    if(colsum) token_stats_kernel<T, true><<<chunks * tiles, 256, 0, st>>>(s, offsets, sets, tiles, rowpart, cm, sm);
    else       token_stats_kernel<T, false><<<chunks * tiles, 256, 0, st>>>(s, offsets, sets, tiles, rowpart, cm, sm);
    const int64_t  col_blocks = sets * ((s.cols + 15) / 16);
    const unsigned blocks = static_cast<unsigned>(col_blocks + (s.rows + 255) / 256);
    if(colsum) token_scales_kernel<true><<<blocks, 256, 0, st>>>(offsets, s.rows, s.cols, sets, col_blocks, static_cast<int>(tiles), rowpart, cm, sm, row_scale, ri, col_scale, ci, colsum);
    else       token_scales_kernel<false><<<blocks, 256, 0, st>>>(offsets, s.rows, s.cols, sets, col_blocks, static_cast<int>(tiles), rowpart, cm, nullptr, row_scale, ri, col_scale, ci, nullptr);
    const unsigned wide = static_cast<unsigned>(code_pad(s.cols) / 64);
    token_codes_kernel<T, RND><<<chunks * wide, 256, 0, st>>>(s, offsets, sets, wide, seed, offset, ri, ci, q, qT);
    return hipGetLastError();
}

}  // namespace

size_t token_both_workspace_bytes(int64_t rows, int64_t cols, int64_t sets, bool offsets) { return both_workspace(rows, cols, sets, offsets).total; }

hipError_t launch_token_quantize(const TokenMatrix& m, const int32_t* count, int rnd, uint64_t seed, uint64_t offset, float* scale, int8_t* q, hipStream_t st)
{
    const TokenSource s{m.x, m.x_rows, m.cols, m.ld, m.rows, m.source, m.group};
    auto typed = [&](auto tag) {
        typedef decltype(tag) T;
        if(rnd == kStochastic) return launch_rows<T, kStochastic>(s, count, seed, offset, scale, q, st);
        return launch_rows<T, kNearest>(s, count, seed, offset, scale, q, st);
    };
    return m.dtype == kF16 ? typed(_Float16{}) : m.dtype == kBF16 ? typed(__bf16{}) : typed(float{});
}

hipError_t launch_token_quantize_both(const TokenMatrix& m, int64_t sets, const int32_t* offsets, int rnd, uint64_t seed, uint64_t offset, float* row_scale, int8_t* q,
                                      float* col_scale, int8_t* qT, float* colsum, void* workspace, hipStream_t st)
{
    const TokenSource s{m.x, m.x_rows, m.cols, m.ld, m.rows, m.source, m.group};
    auto typed = [&](auto tag) {
        typedef decltype(tag) T;
        if(rnd == kStochastic) return launch_both<T, kStochastic>(s, sets, offsets, seed, offset, row_scale, q, col_scale, qT, colsum, workspace, st);
        return launch_both<T, kNearest>(s, sets, offsets, seed, offset, row_scale, q, col_scale, qT, colsum, workspace, st);
    };
    return m.dtype == kF16 ? typed(_Float16{}) : m.dtype == kBF16 ? typed(__bf16{}) : typed(float{});
}

}  // namespace qsync
