// Tokens sorted by the experts that a router gave them, their rows gathered, and the experts' rows combined again, with gradients.
#include "device_utils.h"
#include "row_ops.h"
#include "token_ops.h"

namespace qsync {

namespace {

// ---- sort ------------------------------------------------------------------------------------------------------------------------
// Stable by expert: an entry's place is the number of entries of lower experts, plus those of its own in front of it.  One workgroup: each
// wavefront counts its stretch of the entries, the counts are added up over experts and wavefronts, and each wavefront walks its stretch
// again.  Entries of the same expert among 64 find each other by comparing the ids bit by bit.
constexpr int kSortWaves = 16;
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
template <typename I>
__global__ __launch_bounds__(64 * kSortWaves) void expert_sort_kernel(const I* ids, int64_t n, int experts, int bits, int32_t* offsets, int32_t* source, int32_t* slot)
{
    extern __shared__ int32_t counts[];      // [wavefronts][experts], then running places
    __shared__ int32_t carry[kSortWaves], total;
    const int     lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t per = ((n + kSortWaves - 1) / kSortWaves + 63) / 64 * 64, begin = min(n, wave * per), end = min(n, begin + per);
    for(int i = threadIdx.x; i < kSortWaves * experts; i += 64 * kSortWaves) counts[i] = 0;
    __syncthreads();
    int32_t* mine = counts + wave * experts;
    for(int64_t i = begin + lane; i - lane < end; i += 64)
    {
        const int e = i < end ? expert_of(ids, i, experts) : -1;
        if(e >= 0) atomicAdd(mine + e, 1);
    }
    __syncthreads();
    if(threadIdx.x == 0) total = 0;
    __syncthreads();
    for(int e0 = 0; e0 < experts; e0 += 64 * kSortWaves)
    {   // places of the experts, 1024 at a time; of an expert, those of its wavefronts
        const int e = e0 + threadIdx.x;
        int32_t   sum = 0;
        if(e < experts)
            for(int w = 0; w < kSortWaves; ++w) sum += counts[w * experts + e];
        int32_t scan = sum;
        for(int off = 1; off < 64; off <<= 1)
        {
            const int32_t o = __shfl_up(scan, off);
            if(lane >= off) scan += o;
        }
        if(lane == 63) carry[wave] = scan;
        __syncthreads();
        int32_t at = total + scan - sum;
        for(int w = 0; w < wave; ++w) at += carry[w];
        if(e < experts)
        {
            offsets[e] = at;
            for(int w = 0; w < kSortWaves; ++w)
            {
                const int32_t c = counts[w * experts + e];
                counts[w * experts + e] = at;
                at += c;
            }
        }
        __syncthreads();
        if(threadIdx.x == 64 * kSortWaves - 1) total = at;      // (experts past the last have no entries: at is the running total)
        __syncthreads();
    }
    if(threadIdx.x == 0) offsets[experts] = total;
    for(int64_t i = begin + lane; i - lane < end; i += 64)
    {
        const int      e = i < end ? expert_of(ids, i, experts) : -1;
        const uint64_t same = same_expert(e, e >= 0, bits);
        const int      ahead = __popcll(same & ((1ull << lane) - 1));
        int32_t        place = -1;
        if(e >= 0)
        {
            place = mine[e] + ahead;
            source[place] = static_cast<int32_t>(i);
        }
        if(i < end) slot[i] = place;
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        if(e >= 0 && ahead == 0) mine[e] += static_cast<int32_t>(__popcll(same));
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    }
}

// ---- rows ------------------------------------------------------------------------------------------------------------------------
// rows[r] = x[source[r] / group], a workgroup a row; a place outside of x: NaN
template <typename T>
__global__ __launch_bounds__(256) void expert_gather_kernel(const T* x, int64_t x_rows, int64_t cols, int64_t ld, const int32_t* source, int group, int64_t rows, const int32_t* count, T* y)
{
    const int64_t r = blockIdx.x;
    if(r >= *count) return;
    const int32_t i = source[r];
    const bool    ok = i >= 0 && i / group < x_rows;
    const T*      from = x + (ok ? i / group : 0) * ld;
    for(int64_t c = threadIdx.x; c < cols; c += 256) y[r * cols + c] = ok ? from[c] : static_cast<T>(__uint_as_float(0x7FC00000u));
}

template <typename T>
__global__ __launch_bounds__(256) void expert_combine_kernel(const T* z, int64_t rows, int64_t cols, int64_t ld, const int32_t* slot, int group, const float* weight, void* y, int ydt)
{
    const int64_t t = blockIdx.x;
    for(int64_t c = threadIdx.x; c < cols; c += 256)
    {
        float sum = 0.0f;
        for(int j = 0; j < group; ++j)
        {
            const int32_t r = slot[t * group + j];
            if(r < 0 || r >= rows) continue;
            sum = fmaf(weight ? weight[t * group + j] : 1.0f, row_element(z + r * ld + c), sum);
        }
        element_store(y, ydt, t * cols + c, sum);
    }
}

template <typename T, typename U>
__global__ __launch_bounds__(256) void expert_combine_bwd_kernel(const T* dy, int64_t cols, int64_t lddy, const U* z, int64_t rows, int64_t ldz, const int32_t* slot, int group, const float* weight,
                                                                 void* dz, int dzdt, float* dweight)
{
    __shared__ float lds[16];
    const int64_t t = blockIdx.x;
    for(int j = 0; j < group; ++j)
    {
        const int32_t r = slot[t * group + j];
        const bool    ok = r >= 0 && r < rows;
        float         dot = 0.0f;
        const float   w = weight ? weight[t * group + j] : 1.0f;
        if(ok)
            for(int64_t c = threadIdx.x; c < cols; c += 256)
            {
                const float g = row_element(dy + t * lddy + c);
                if(dweight) dot = fmaf(g, row_element(z + r * ldz + c), dot);
                if(dz) element_store(dz, dzdt, r * cols + c, w * g);
            }
        if(dweight)
        {
            dot = block_reduce_sum(dot, lds);
            if(threadIdx.x == 0) dweight[t * group + j] = dot;
            __syncthreads();
        }
    }
}

}  // namespace

size_t expert_sort_workspace_bytes(int64_t, int) { return 0; }

hipError_t launch_expert_sort(const void* ids, bool wide, int64_t n, int experts, int32_t* offsets, int32_t* source, int32_t* slot, void*, hipStream_t st)
{
    int bits = 0;
    while((1 << bits) < experts) ++bits;
    const size_t lds = static_cast<size_t>(kSortWaves) * experts * 4;
    if(wide) expert_sort_kernel<<<1, 64 * kSortWaves, lds, st>>>(static_cast<const int64_t*>(ids), n, experts, bits, offsets, source, slot);
    else     expert_sort_kernel<<<1, 64 * kSortWaves, lds, st>>>(static_cast<const int32_t*>(ids), n, experts, bits, offsets, source, slot);
    return hipGetLastError();
}

hipError_t launch_expert_gather(const void* x, int dtype, int64_t x_rows, int64_t cols, int64_t ld, const int32_t* source, int group, int64_t rows, const int32_t* count, void* y, hipStream_t st)
{
    auto typed = [&](auto tag) {
        typedef decltype(tag) T;
        expert_gather_kernel<T><<<static_cast<unsigned>(rows), 256, 0, st>>>(static_cast<const T*>(x), x_rows, cols, ld, source, group, rows, count, static_cast<T*>(y));
    };
    dtype == kF16 ? typed(_Float16{}) : dtype == kBF16 ? typed(__bf16{}) : typed(float{});
    return hipGetLastError();
}

hipError_t launch_expert_combine(const void* z, int zdt, int64_t rows, int64_t cols, int64_t ld, const int32_t* slot, int64_t tokens, int group, const float* weight, void* y, int ydt, hipStream_t st)
{
    auto typed = [&](auto tag) {
        typedef decltype(tag) T;
        expert_combine_kernel<T><<<static_cast<unsigned>(tokens), 256, 0, st>>>(static_cast<const T*>(z), rows, cols, ld, slot, group, weight, y, ydt);
    };
    zdt == kF16 ? typed(_Float16{}) : zdt == kBF16 ? typed(__bf16{}) : typed(float{});
    return hipGetLastError();
}

hipError_t launch_expert_combine_bwd(const void* dy, int dydt, int64_t tokens, int64_t cols, int64_t lddy, const void* z, int zdt, int64_t rows, int64_t ldz, const int32_t* slot, int group,
                                     const float* weight, void* dz, int dzdt, float* dweight, hipStream_t st)
{
    auto typed = [&](auto tag, auto ztag) {
        typedef decltype(tag) T;
        typedef decltype(ztag) U;
        expert_combine_bwd_kernel<T, U><<<static_cast<unsigned>(tokens), 256, 0, st>>>(static_cast<const T*>(dy), cols, lddy, static_cast<const U*>(z), rows, ldz, slot, group, weight, dz, dzdt, dweight);
    };
    auto with_z = [&](auto tag) { zdt == kF16 ? typed(tag, _Float16{}) : zdt == kBF16 ? typed(tag, __bf16{}) : typed(tag, float{}); };
    dydt == kF16 ? with_z(_Float16{}) : dydt == kBF16 ? with_z(__bf16{}) : with_z(float{});
    return hipGetLastError();
}

}  // namespace qsync
