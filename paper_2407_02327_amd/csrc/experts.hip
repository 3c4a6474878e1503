// Tokens sorted by the experts that a router gave them, their rows gathered, and the experts' rows combined again, with gradients.
#include "device_utils.h"
#include "row_ops.h"
#include "token_ops.h"

#include <type_traits>

namespace qsync {

namespace {

// ---- sort ------------------------------------------------------------------------------------------------------------------------
// Stable by expert: an entry's place is the number of entries of lower experts, plus those of its own in front of it.  A workgroup has a section
// of the entries, a wavefront a stretch of that.  Up to 2048 entries are one section and one launch; more are counted by a first launch
// (hist [sections][experts]), and each workgroup of the second adds up what lies in front of its own.  Entries of the same expert among a
// wavefront's 64 find each other by comparing the ids bit by bit.  One workgroup for everything took 81 us for 65536 entries.
constexpr int kSortWaves = 16, kSortThreads = 64 * kSortWaves, kSortSections = 256;
template <typename I> __device__ __forceinline__ int expert_of(const I* ids, int64_t i, int experts)
{
    const I v = ids[i];
    return v >= 0 && v < experts ? static_cast<int>(v) : -1;
}
__device__ __forceinline__ uint64_t same_expert(int e, bool valid, int bits)
{
    uint64_t m = __ballot(valid);
    for(int b = 0; b < bits; ++b)
    {
        const uint64_t one = __ballot((e >> b) & 1);
        m &= (e >> b) & 1 ? one : ~one;
    }
    return m;
}
template <typename I> __global__ __launch_bounds__(kSortThreads) void expert_count_kernel(const I* ids, int64_t n, int64_t section, int experts, int32_t* hist)
{
    extern __shared__ int32_t counts[];      // [experts]
    for(int i = threadIdx.x; i < experts; i += kSortThreads) counts[i] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * section, end = min(n, begin + section);
    for(int64_t i = begin + threadIdx.x; i < end; i += kSortThreads)
    {
        const int e = expert_of(ids, i, experts);
        if(e >= 0) atomicAdd(counts + e, 1);
    }
    __syncthreads();
    for(int i = threadIdx.x; i < experts; i += kSortThreads) hist[static_cast<int64_t>(blockIdx.x) * experts + i] = counts[i];
}

// `bits`: of experts - 1; hist nullptr: one section
template <typename I>
__global__ __launch_bounds__(kSortThreads) void expert_place_kernel(const I* ids, int64_t n, int64_t section, int experts, int bits, const int32_t* hist, int32_t* offsets, int32_t* source, int32_t* slot)
{
    extern __shared__ int32_t counts[];      // [wavefronts][experts], then running places
    __shared__ int32_t before[kSortThreads], whole[kSortThreads], carry[kSortWaves];
    const int     lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t first = blockIdx.x * section, last = min(n, first + section);
    const int64_t per = (section / kSortWaves + 63) / 64 * 64, begin = min(last, first + wave * per), end = min(last, begin + per);
    for(int i = threadIdx.x; i < kSortWaves * experts; i += kSortThreads) counts[i] = 0;
    __syncthreads();
    int32_t* mine = counts + wave * experts;
    for(int64_t i = begin + lane; i < end; i += 64)
    {
        const int e = expert_of(ids, i, experts);
        if(e >= 0) atomicAdd(mine + e, 1);
    }
    // Of each expert: its entries, and those in sections before this one.  1024 >> bits threads share an expert.
    const int e = threadIdx.x & ((1 << bits) - 1), part = threadIdx.x >> bits, parts = kSortThreads >> bits;
    int32_t   all = 0, ahead = 0;
    if(hist && e < experts)
        for(int b0 = part; b0 < static_cast<int>(gridDim.x); b0 += 4 * parts)
        {
            int32_t o[4];
#pragma unroll
            for(int u = 0; u < 4; ++u) o[u] = b0 + u * parts < static_cast<int>(gridDim.x) ? hist[static_cast<int64_t>(b0 + u * parts) * experts + e] : 0;
#pragma unroll
            for(int u = 0; u < 4; ++u)
            {
                all += o[u];
                ahead += b0 + u * parts < static_cast<int>(blockIdx.x) ? o[u] : 0;
            }
        }
    whole[threadIdx.x]  = all;
    before[threadIdx.x] = ahead;
    __syncthreads();
    if(part == 0 && e < experts)      // (the first 1 << bits threads)
    {
        if(hist)
            for(int i = 1; i < parts; ++i)
            {
                all += whole[(i << bits) + e];
                ahead += before[(i << bits) + e];
            }
        else
            for(int w = 0; w < kSortWaves; ++w) all += counts[w * experts + e];
    }
    else all = 0;
    int32_t scan = all;      // (of the experts up to this one)
#pragma unroll
    for(int off = 1; off < 64; off <<= 1)
    {
        const int32_t o = __shfl_up(scan, off);
        if(lane >= off) scan += o;
    }
    if(lane == 63) carry[wave] = scan;
    __syncthreads();
    for(int w = 0; w < wave; ++w) scan += carry[w];
    if(part == 0 && e < experts)
    {
        if(blockIdx.x == 0)
        {
            offsets[e] = scan - all;
            if(e == experts - 1) offsets[experts] = scan;
        }
        int32_t at = scan - all + ahead;
        for(int w = 0; w < kSortWaves; ++w)
        {
            const int32_t c = counts[w * experts + e];
            counts[w * experts + e] = at;
            at += c;
        }
    }
    __syncthreads();
    for(int64_t i = begin + lane; i - lane < end; i += 64)
    {
        const int      x = i < end ? expert_of(ids, i, experts) : -1;
        const uint64_t same = same_expert(x, x >= 0, bits);
        const int      rank = __popcll(same & ((1ull << lane) - 1));
        int32_t        place = -1;
        if(x >= 0)
        {
            place = mine[x] + rank;
            source[place] = static_cast<int32_t>(i);
        }
        if(i < end) slot[i] = place;
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        if(x >= 0 && rank == 0) mine[x] += static_cast<int32_t>(__popcll(same));
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    }
}

// ---- rows ------------------------------------------------------------------------------------------------------------------------
// A thread has V columns, 16 bytes of the input (in the backward pass eight, whatever the type: 3333x1001 fp32, three rows each, 19 us, by fours 2 more); a workgroup's 256 threads are 256 / side rows (or tokens) of
// `side` threads, as many as a row has vectors up to 256, and longer rows take several workgroups: whatever the shape, a thread does little, and
// a launch has as many threads as there is data.
// The last vector of a row that is no whole number of them starts V elements in front of the row's end: what two threads have in common they both
// leave, alike, and no thread walks single elements (rows of V elements and more; 3333 tokens of 1001 fp32, three rows each: gather 17.8 -> 15.3 us,
// combine 15.3 -> 14.1, backward 20.8 -> 19.4).
__device__ __forceinline__ int64_t vector_start(int64_t c, int64_t cols, int V) { return c + V > cols && cols >= V ? cols - V : c; }
struct RowGrid { int side_log2, blocks_x; };
RowGrid row_grid(int64_t cols, int V, int least)
{
    const int64_t vectors = (cols + V - 1) / V;
    int           log2 = least;
    while(log2 < 8 && (int64_t(1) << log2) < vectors) ++log2;
    return {log2, static_cast<int>((vectors + (1 << log2) - 1) >> log2)};
}
template <typename T, int V> struct RowPart
{
    static constexpr int N = RowType<T>::N;
    row_v4u32 w[V / N];
    __device__ __forceinline__ void load(const T* row, int64_t c, int64_t cols)      // zeros behind the last column
    {
        if(c + V <= cols)
#pragma unroll
            for(int i = 0; i < V / N; ++i) w[i] = row_load(row + c + i * N);
        else
        {
            float e[V];
#pragma unroll
            for(int i = 0; i < V; ++i) e[i] = c + i < cols ? row_element(row + c + i) : 0.0f;
            encode(e);
        }
    }
    __device__ __forceinline__ void decode(float (&v)[V]) const
    {
#pragma unroll
        for(int i = 0; i < V / N; ++i) row_decode<T>(w[i], v + i * N);
    }
    __device__ __forceinline__ void encode(const float (&v)[V])
    {
#pragma unroll
        for(int i = 0; i < V / N; ++i)
        {
            float e[N];
#pragma unroll
            for(int j = 0; j < N; ++j) e[j] = v[i * N + j];
            w[i] = RowType<T>::pack(e);
        }
    }
    __device__ __forceinline__ void store(T* p) const
    {
#pragma unroll
        for(int i = 0; i < V / N; ++i) row_store(p + i * N, w[i]);
    }
};
template <int V> __device__ __forceinline__ void store_part(void* base, int dtype, int64_t at, int64_t c, int64_t cols, float (&v)[V])
{
    if(c + V > cols)
    {
#pragma unroll
        for(int i = 0; i < V; ++i)
            if(c + i < cols) element_store(base, dtype, at + c + i, v[i]);
    }
    else if constexpr(V == 8) row8_store<false>(base, dtype, at + c, v);
    else                      vector_store<float, false>(base, dtype, at + c, v);
}

// rows[r] = x[source[r] / group]; a place outside of x: NaN.  A thread has U rows, their loads requested together (65536 rows of 1024 bfloat16: one
// 45 us, four 41).
template <typename T, int U>
__global__ __launch_bounds__(256) void expert_gather_kernel(const T* x, int64_t x_rows, int64_t cols, int64_t ld, const int32_t* source, int group, const int32_t* count, int64_t rows, T* y,
                                                            int side_log2)
{
    constexpr int V = RowType<T>::N;
    const int     side = threadIdx.x & ((1 << side_log2) - 1), at_once = 256 >> side_log2;
    const int64_t r0 = (static_cast<int64_t>(blockIdx.y) * gridDim.z + blockIdx.z) * at_once * U + (threadIdx.x >> side_log2);
    const int64_t c0 = ((static_cast<int64_t>(blockIdx.x) << side_log2) + side) * V, c = vector_start(c0, cols, V), n = min(rows, static_cast<int64_t>(*count));
    if(c0 >= cols) return;
    int32_t i[U];
    RowPart<T, V> v[U];
#pragma unroll
    for(int u = 0; u < U; ++u) i[u] = r0 + u * at_once < n ? source[r0 + u * at_once] : -1;
#pragma unroll
    for(int u = 0; u < U; ++u)
    {
        const bool ok = i[u] >= 0 && i[u] / group < x_rows;
        v[u].load(x + (ok ? i[u] / group : 0) * ld, c, ok ? cols : 0);
        if(!ok)
        {
            float e[V];
#pragma unroll
            for(int j = 0; j < V; ++j) e[j] = __uint_as_float(0x7FC00000u);
            v[u].encode(e);
        }
    }
#pragma unroll
    for(int u = 0; u < U; ++u)
    {
        const int64_t r = r0 + u * at_once;
        if(r >= n) break;
        T* out = y + r * cols;
        if(c + V <= cols) v[u].store(out + c);
        else
        {
            float e[V];
            v[u].decode(e);
#pragma unroll
            for(int j = 0; j < V; ++j)
                if(c + j < cols) out[c + j] = static_cast<T>(e[j]);
        }
    }
}

// (U rows requested at a time.)
template <typename T, int U>
__global__ __launch_bounds__(256) void expert_combine_kernel(const T* z, int64_t rows, int64_t cols, int64_t ld, const int32_t* slot, int64_t tokens, int group, const float* weight, void* y, int ydt,
                                                             int side_log2)
{
    constexpr int V = RowType<T>::N;
    const int     side = threadIdx.x & ((1 << side_log2) - 1);
    const int64_t t = static_cast<int64_t>(blockIdx.y) * gridDim.z * (256 >> side_log2) + blockIdx.z * (256 >> side_log2) + (threadIdx.x >> side_log2);
    const int64_t c0 = ((static_cast<int64_t>(blockIdx.x) << side_log2) + side) * V, c = vector_start(c0, cols, V);
    if(t >= tokens || c0 >= cols) return;
    float sum[V];
#pragma unroll
    for(int j = 0; j < V; ++j) sum[j] = 0.0f;
    for(int j0 = 0; j0 < group; j0 += U)
    {
        RowPart<T, V> v[U];
        float         w[U];
        bool          ok[U];
#pragma unroll
        for(int u = 0; u < U; ++u)
        {
            const int64_t at = t * group + (j0 + u < group ? j0 + u : j0);
            const int32_t r = slot[at];
            ok[u] = j0 + u < group && r >= 0 && r < rows;
            w[u]  = weight ? weight[at] : 1.0f;
            v[u].load(z + (ok[u] ? r : 0) * ld, c, ok[u] ? cols : 0);
        }
#pragma unroll
        for(int u = 0; u < U; ++u)
            if(ok[u])
            {
                float e[V];
                v[u].decode(e);
#pragma unroll
                for(int j = 0; j < V; ++j) sum[j] = fmaf(w[u], e[j], sum[j]);
            }
    }
    store_part<V>(y, ydt, t * cols, c, cols, sum);
}

// A token's gradient is read once for all its rows: `side` threads (64 at least, so that whole wavefronts share a token) walk its columns with
// four rows' vectors in flight, and leave the rows' gradients and their part of the products dy z, which meet by wavefronts and in LDS.
template <typename T, typename U, bool DOT, bool DZ>
__global__ __launch_bounds__(256) void expert_combine_bwd_kernel(const T* dy, int64_t tokens, int64_t cols, int64_t lddy, const U* z, int64_t rows, int64_t ldz, const int32_t* slot, int group,
                                                                 const float* weight, void* dz, int dzdt, float* dweight, int side_log2)
{
    constexpr int    V = 8;
    __shared__ float part[4][4];
    const int     threads = 1 << side_log2, side = threadIdx.x & (threads - 1), wave = threadIdx.x / 64;
    const int64_t t = (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * (256 >> side_log2) + (threadIdx.x >> side_log2);
    const bool    here = t < tokens;
    const int64_t tt = here ? t : 0;
    for(int j0 = 0; j0 < group; j0 += 4)
    {
        int64_t r[4];
        float   w[4], dot[4];
#pragma unroll
        for(int u = 0; u < 4; ++u)
        {
            const int64_t at = tt * group + (j0 + u < group ? j0 + u : j0);
            const int32_t i = slot[at];
            r[u]   = here && j0 + u < group && i >= 0 && i < rows ? i : -1;
            w[u]   = weight ? weight[at] : 1.0f;
            dot[u] = 0.0f;
        }
        for(int64_t c0 = side * V; c0 < cols; c0 += threads * V)
        {
            const int64_t c = vector_start(c0, cols, V);
            RowPart<T, V> g;
            RowPart<U, V> v[4];
            g.load(dy + tt * lddy, c, cols);
            if constexpr(DOT)
#pragma unroll
                for(int u = 0; u < 4; ++u) v[u].load(z + (r[u] < 0 ? 0 : r[u]) * ldz, c, r[u] < 0 ? 0 : cols);
            float d[V];
            g.decode(d);
#pragma unroll
            for(int u = 0; u < 4; ++u)
                if(r[u] >= 0)
                {
                    float e[V];
                    if constexpr(DOT)
                    {
                        v[u].decode(e);
#pragma unroll
                        for(int j = 0; j < V; ++j) dot[u] = c + j >= c0 && c + j < cols ? fmaf(d[j], e[j], dot[u]) : dot[u];
                    }
                    if constexpr(DZ)
                    {
#pragma unroll
                        for(int j = 0; j < V; ++j) e[j] = w[u] * d[j];
                        store_part<V>(dz, dzdt, r[u] * cols, c, cols, e);
                    }
                }
        }
        if constexpr(DOT)
        {
#pragma unroll
            for(int u = 0; u < 4; ++u) dot[u] = wave64_sum(dot[u]);
            if(side_log2 > 6)
            {
                if(threadIdx.x % 64 == 0)
#pragma unroll
                    for(int u = 0; u < 4; ++u) part[wave][u] = dot[u];
                __syncthreads();
#pragma unroll
                for(int u = 0; u < 4; ++u)
                {
                    dot[u] = part[wave & ~(threads / 64 - 1)][u];
                    for(int i = 1; i < threads / 64; ++i) dot[u] += part[(wave & ~(threads / 64 - 1)) + i][u];
                }
                __syncthreads();
            }
            if(side == 0 && here)
#pragma unroll
                for(int u = 0; u < 4; ++u)
                    if(j0 + u < group) dweight[t * group + j0 + u] = r[u] >= 0 ? dot[u] : 0.0f;
        }
    }
}

}  // namespace

static int64_t sort_section(int64_t n)
{
    if(n <= 2 * kSortThreads) return 2 * kSortThreads;
    return ((n + kSortSections - 1) / kSortSections + kSortThreads - 1) / kSortThreads * kSortThreads;
}
size_t expert_sort_workspace_bytes(int64_t n, int experts)
{
    // (what is enough for some number of entries is enough for fewer, though a longer section may be cut into fewer of them)
    const int64_t sections = (n + kSortThreads - 1) / kSortThreads;
    return n > sort_section(n) ? static_cast<size_t>(sections < kSortSections ? sections : kSortSections) * experts * 4 : 0;
}

hipError_t launch_expert_sort(const void* ids, bool wide, int64_t n, int experts, int32_t* offsets, int32_t* source, int32_t* slot, void* workspace, hipStream_t st)
{
    int bits = 0;
    while((1 << bits) < experts) ++bits;
    const int64_t  section = sort_section(n);
    const unsigned sections = static_cast<unsigned>(n > section ? (n + section - 1) / section : 1);
    const size_t   lds = static_cast<size_t>(experts) * 4;
    int32_t*       hist = sections > 1 ? static_cast<int32_t*>(workspace) : nullptr;
    auto typed = [&](auto tag) {
        typedef decltype(tag) I;
        if(hist) expert_count_kernel<I><<<sections, kSortThreads, lds, st>>>(static_cast<const I*>(ids), n, section, experts, hist);
        expert_place_kernel<I><<<sections, kSortThreads, kSortWaves * lds, st>>>(static_cast<const I*>(ids), n, section, experts, bits, hist, offsets, source, slot);
    };
    wide ? typed(int64_t{}) : typed(int32_t{});
    return hipGetLastError();
}

constexpr int64_t kManyRows = 4096;      // workgroups of one row a thread from which on a thread has four
// rows (of 256 >> side_log2 a workgroup) over the grid's y and z: neither may count more than 65535
dim3 rows_over_grid(const RowGrid& g, int64_t rows, int per_thread = 1)
{
    const int64_t each = static_cast<int64_t>(256 >> g.side_log2) * per_thread, blocks = (rows + each - 1) / each, z = blocks < 256 ? 1 : 256;
    return dim3(static_cast<unsigned>(g.blocks_x), static_cast<unsigned>((blocks + z - 1) / z), static_cast<unsigned>(z));
}

hipError_t launch_expert_gather(const void* x, int dtype, int64_t x_rows, int64_t cols, int64_t ld, const int32_t* source, int group, int64_t rows, const int32_t* count, void* y, hipStream_t st)
{
    const RowGrid g = row_grid(cols, dtype == kF32 ? 4 : 8, 3);
    auto typed = [&](auto tag) {
        typedef decltype(tag) T;
        if(rows * g.blocks_x >= kManyRows * (256 >> g.side_log2))
            expert_gather_kernel<T, 4><<<rows_over_grid(g, rows, 4), 256, 0, st>>>(static_cast<const T*>(x), x_rows, cols, ld, source, group, count, rows, static_cast<T*>(y), g.side_log2);
        else
            expert_gather_kernel<T, 1><<<rows_over_grid(g, rows), 256, 0, st>>>(static_cast<const T*>(x), x_rows, cols, ld, source, group, count, rows, static_cast<T*>(y), g.side_log2);
    };
    dtype == kF16 ? typed(_Float16{}) : dtype == kBF16 ? typed(__bf16{}) : typed(float{});
    return hipGetLastError();
}

hipError_t launch_expert_combine(const void* z, int zdt, int64_t rows, int64_t cols, int64_t ld, const int32_t* slot, int64_t tokens, int group, const float* weight, void* y, int ydt, hipStream_t st)
{
    const RowGrid g = row_grid(cols, zdt == kF32 ? 4 : 8, 3);
    auto typed = [&](auto tag) {
        typedef decltype(tag) T;
        // (8192 tokens of 1024 bfloat16, eight rows each: by fours 37.4 us, by eights 40.1; of 4096, two each: by fours 48.8, by twos 40.2)
        if(group > 2) expert_combine_kernel<T, 4><<<rows_over_grid(g, tokens), 256, 0, st>>>(static_cast<const T*>(z), rows, cols, ld, slot, tokens, group, weight, y, ydt, g.side_log2);
        else expert_combine_kernel<T, 2><<<rows_over_grid(g, tokens), 256, 0, st>>>(static_cast<const T*>(z), rows, cols, ld, slot, tokens, group, weight, y, ydt, g.side_log2);
    };
    zdt == kF16 ? typed(_Float16{}) : zdt == kBF16 ? typed(__bf16{}) : typed(float{});
    return hipGetLastError();
}

hipError_t launch_expert_combine_bwd(const void* dy, int dydt, int64_t tokens, int64_t cols, int64_t lddy, const void* z, int zdt, int64_t rows, int64_t ldz, const int32_t* slot, int group,
                                     const float* weight, void* dz, int dzdt, float* dweight, hipStream_t st)
{
    const int     side_log2 = row_grid(cols, 8, 6).side_log2;
    const int64_t blocks = (tokens + (256 >> side_log2) - 1) / (256 >> side_log2), x = blocks < 65536 ? blocks : 65536;
    const dim3    grid(static_cast<unsigned>(x), static_cast<unsigned>((blocks + x - 1) / x));
    auto typed = [&](auto tag, auto ztag) {
        typedef decltype(tag) T;
        typedef decltype(ztag) U;
        auto go = [&](auto dot, auto out) {
            expert_combine_bwd_kernel<T, U, decltype(dot)::value, decltype(out)::value><<<grid, 256, 0, st>>>(static_cast<const T*>(dy), tokens, cols, lddy, static_cast<const U*>(z), rows, ldz, slot,
                                                                                                            group, weight, dz, dzdt, dweight, side_log2);
        };
        constexpr std::true_type  yes{};
        constexpr std::false_type no{};
        if(dweight && dz) go(yes, yes);
        else if(dweight) go(yes, no);
        else go(no, yes);
    };
    auto with_z = [&](auto tag) { zdt == kF16 ? typed(tag, _Float16{}) : zdt == kBF16 ? typed(tag, __bf16{}) : typed(tag, float{}); };
    dydt == kF16 ? with_z(_Float16{}) : dydt == kBF16 ? with_z(__bf16{}) : with_z(float{});
    return hipGetLastError();
}

}  // namespace qsync
