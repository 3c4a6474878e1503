// What is done with the logits that a language model's head writes: log probabilities of given tokens with the entropy and the top
// alternatives of every position, the gradient of the first two, and distillation from a teacher's top logits with its gradient.
//
// With m = max_j z_j, d_j = scale (z_j - m), S = sum_j e^{d_j}:
//   log p_j = d_j - ln S      H = -sum_j p_j log p_j = ln S - (sum_j d_j e^{d_j}) / S
// so one pass over a row carries three numbers a lane, the maximum so far and the two sums relative to it, and joins the lanes' in a
// fixed order.  The exponential is that of two (v_exp_f32) with scale * log2(e) as the factor; the difference to the maximum is taken first,
// in fp32, so that a row whose logits all have one value -- the type's lowest included -- is the uniform distribution it stands for.
//   gradient of  g logp_token + h H:   scale (g (delta - p_j) - h p_j (log p_j + H))
//   distillation, q the teacher's probabilities on its k entries:   loss = sum_i q_i (log q_i - log p_{idx_i}),
//   gradient of  weight loss:          weight scale (p_j - q_j)
// All are bound by memory: a row of logits is read once, a gradient written once.  Vocabulary rows are long and few: where there are fewer rows
// than the device has room for, a row is cut into pieces whose results a second launch joins.
#include "device_utils.h"
#include "row_ops.h"

#include <cfloat>

namespace qsync {

namespace {

constexpr int   kRowThreads = 256;
constexpr int   kUnroll     = 4;          // vectors of a lane in flight: a chunk
constexpr int   kMaxChunks  = 16;         // chunks of a lane whose maxima the top search keeps in LDS
constexpr float kLn2 = 0.693147180559945309f, kLog2e = 1.44269504088896341f;
constexpr float kFar = -1.0e30f;          // stands for differences to the maximum that overflow: e^x is 0 there, and 0 * x is 0
constexpr int   kTopMost = kTopAlternatives;      // a sorted list is a value per lane
static_assert(kTopMost == kWaveSize && kTeacherEntries == kRowThreads, "a lane an alternative, a thread an entry");

template <typename T> constexpr int chunk_span() { return kRowThreads * RowType<T>::N * kUnroll; }      // elements of a workgroup's chunks

struct Moments
{
    float m, s, w;      // maximum, sum of 2^{k2 (z - m)}, sum of k2 (z - m) 2^{k2 (z - m)}
};

struct LogitsArgs
{
    const void* z;
    int64_t     rows, ld;
    int         cols;
    float       scale;
    int         pieces, piece;      // pieces of a row, elements of a piece
    const void* tokens;             // or nullptr
    int         wide;               // 64-bit tokens (indices)
    float *     logp, *entropy, *stats;
    int         top;
    float*      top_logp;
    int32_t*    top_index;
    float4*     part;               // [rows][pieces] moments
    uint64_t*   part_keys;          // [rows][pieces][top]
};

__device__ __forceinline__ int64_t index_at(const void* p, int wide, int64_t i)
{
    return wide ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
}

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// Joins the lanes' moments; the result in every lane.  `slots`: one per wavefront.
template <int WG> __device__ __forceinline__ Moments join_lanes(Moments a, float k2, float4* slots)
{
    const float m  = wave64_max(a.m);
    const float dm = fmaxf((a.m - m) * k2, kFar), f = exp2_fast(dm);
    a.w = wave64_sum((a.w + dm * a.s) * f);
    a.s = wave64_sum(a.s * f);
    if(threadIdx.x % kWaveSize == 0) slots[threadIdx.x / kWaveSize] = make_float4(m, a.s, a.w, 0.0f);
    __syncthreads();
    Moments r{slots[0].x, 0.0f, 0.0f};
#pragma unroll
    for(int i = 1; i < WG / kWaveSize; ++i) r.m = fmaxf(r.m, slots[i].x);
#pragma unroll
    for(int i = 0; i < WG / kWaveSize; ++i)
    {
        const float4 o = slots[i];
        const float  d = fmaxf((o.x - r.m) * k2, kFar), g = exp2_fast(d);
        r.s += o.y * g;
        r.w += (o.z + d * o.y) * g;
    }
    return r;
}

// The maximum that a top search keeps of a lane: value and the chunk it was first met in.
struct LaneBest
{
    float value = -INFINITY;
    int   chunk = -1;
};

// One pass over the elements [begin, end) of a row.
template <typename T, int WG, bool ENTROPY, bool TOP>
__device__ __forceinline__ Moments row_pass(const T* z, int begin, int end, float k2, float* chunk_max, LaneBest& best)
{
    constexpr int N = RowType<T>::N, SPAN = WG * N * kUnroll;
    const int     len = end - begin, chunks = (len + SPAN - 1) / SPAN;
    const T*      at  = z + begin + threadIdx.x * N;
    row_v4u32     next[kUnroll];
    auto          fetch = [&](int c) {
        const T* from = at + static_cast<int64_t>(c) * SPAN;
        if((c + 1) * static_cast<int64_t>(SPAN) <= len)
        {
#pragma unroll
            for(int u = 0; u < kUnroll; ++u) next[u] = row_load(from + u * WG * N);
            return;
        }
        const int left = len - c * SPAN - static_cast<int>(threadIdx.x) * N;
#pragma unroll
        for(int u = 0; u < kUnroll; ++u) next[u] = row_load_part(from + u * WG * N, left - u * WG * N, RowType<T>::kMinusInf);
    };
    Moments r{-FLT_MAX, 0.0f, 0.0f};
    if(chunks > 0) fetch(0);
    for(int c = 0; c < chunks; ++c)
    {
        float v[kUnroll * N];
#pragma unroll
        for(int u = 0; u < kUnroll; ++u) row_decode<T>(next[u], v + u * N);
        if(c + 1 < chunks) fetch(c + 1);
        float top = v[0];
#pragma unroll
        for(int i = 1; i < kUnroll * N; ++i) top = fmaxf(top, v[i]);
        if constexpr(TOP)
        {
            chunk_max[c * WG + threadIdx.x] = top;
            best.chunk = top > best.value ? c : best.chunk;
            best.value = top > best.value ? top : best.value;
        }
        const float m  = fmaxf(r.m, top);
        const float dm = fmaxf((r.m - m) * k2, kFar), f = exp2_fast(dm);
        if constexpr(ENTROPY) r.w = (r.w + dm * r.s) * f;
        r.s *= f;
        r.m = m;
#pragma unroll
        for(int i = 0; i < kUnroll * N; ++i)
        {
            const float d = (v[i] - m) * k2, e = exp2_fast(d);
            r.s += e;
            if constexpr(ENTROPY) r.w = fmaf(e, fmaxf(d, kFar), r.w);
        }
    }
    return r;
}

// ---- top alternatives -------------------------------------------------------------------------------------------------------
// A logit and its column as one whole number: larger is the larger value (-0 being +0), among equal ones the lower column.
__device__ __forceinline__ uint32_t ordered_bits(float v)
{
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint64_t rank_key(float v, uint32_t column)
{
    return static_cast<uint64_t>(ordered_bits(v)) << 32 | (0xFFFFFFFFu - column);
}
__device__ __forceinline__ float key_value(uint64_t key)
{
    const uint32_t o = static_cast<uint32_t>(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint32_t key_column(uint64_t key) { return 0xFFFFFFFFu - static_cast<uint32_t>(key); }

__device__ __forceinline__ uint64_t lane_xor(uint64_t v, int mask)
{
    const uint32_t lo = __shfl_xor(static_cast<uint32_t>(v), mask, kWaveSize), hi = __shfl_xor(static_cast<uint32_t>(v >> 32), mask, kWaveSize);
    return static_cast<uint64_t>(hi) << 32 | lo;
}
// The keys of a wavefront in descending order of the lanes: bitonic sort, and its last stage alone.
template <int SIZE> __device__ __forceinline__ void bitonic_stage(uint64_t& key)
{
    const int lane = threadIdx.x % kWaveSize;
#pragma unroll
    for(int j = SIZE / 2; j >= 1; j /= 2)
    {
        const uint64_t other   = lane_xor(key, j);
        const bool     larger  = ((lane & j) == 0) == ((lane & SIZE) == 0);
        key = (key > other) == larger ? key : other;
    }
}
__device__ __forceinline__ void sort_wave(uint64_t& key)
{
    bitonic_stage<2>(key);
    bitonic_stage<4>(key);
    bitonic_stage<8>(key);
    bitonic_stage<16>(key);
    bitonic_stage<32>(key);
    bitonic_stage<64>(key);
}
// The largest 64 of two descending lists; `reversed` is the other list read from its end.
__device__ __forceinline__ void merge_wave(uint64_t& key, uint64_t reversed)
{
    key = key > reversed ? key : reversed;
    bitonic_stage<64>(key);
}
__device__ __forceinline__ uint64_t lane_key(uint64_t v, int lane)
{
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(v)), lane);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(v >> 32)), lane);
    return static_cast<uint64_t>(hi) << 32 | lo;
}

// LDS of a top search, behind the chunk maxima.
struct TopShared
{
    uint64_t list[kRowThreads / kWaveSize][kTopMost];
    uint64_t gathered[kRowThreads / kWaveSize][2 * kTopMost];
    int      count;
};
constexpr size_t top_lds_bytes(int chunks)
{
    return sizeof(TopShared) + static_cast<size_t>(chunks) * kRowThreads * (sizeof(float) + sizeof(uint16_t));
}

// Joins the wavefronts' descending lists: every wavefront gets the largest 64.
__device__ __forceinline__ uint64_t join_lists(uint64_t key, TopShared& sh)
{
    const int lane = threadIdx.x % kWaveSize, wave = threadIdx.x / kWaveSize;
    sh.list[wave][lane] = key;
    __syncthreads();
    uint64_t all = sh.list[0][lane];
#pragma unroll
    for(int w = 1; w < kRowThreads / kWaveSize; ++w) merge_wave(all, sh.list[w][kWaveSize - 1 - lane]);
    return all;
}

// The `top` largest of [begin, end), descending over the lanes of every wavefront (0: fewer elements than that).
// The k-th largest of the lanes' maxima is a bound that at least k elements reach; a chunk whose maximum stays below it is not looked
// at again.  About k chunks (32 or 16 elements) remain of a row, and never more than the k best lanes have; they are read a second
// time, out of a cache, and what reaches the bound is sorted.  The work beside the pass does not depend on the order of the logits, and the
// order (value, then lower column) makes equal logits as good as different ones.
template <typename T>
__device__ __forceinline__ uint64_t row_top(const T* z, int begin, int end, int top, const LaneBest& best, const float* chunk_max,
                                            uint16_t* chosen, TopShared& sh)
{
    constexpr int N = RowType<T>::N, WG = kRowThreads, SPAN = WG * N * kUnroll;
    const int     tid = threadIdx.x, lane = tid % kWaveSize, wave = tid / kWaveSize;
    const int     first = begin + tid * N, chunks = (end - begin + SPAN - 1) / SPAN;
    // a lane's claim: an element of at least this value at this column or in front of it
    uint64_t claim = 0;
    if(best.chunk >= 0) claim = rank_key(best.value, first + best.chunk * SPAN + (kUnroll - 1) * WG * N + N - 1);
    else if(first < end) claim = rank_key(-INFINITY, first);
    if(tid == 0) sh.count = 0;
    sort_wave(claim);
    const uint64_t bound = lane_key(join_lists(claim, sh), top - 1);

    for(int c = 0; c < chunks; ++c)
        if(rank_key(chunk_max[c * WG + tid], first + c * SPAN) >= bound) chosen[atomicAdd(&sh.count, 1)] = static_cast<uint16_t>(c * WG + tid);
    __syncthreads();
    const int vectors = sh.count * kUnroll;
    uint64_t  list    = 0, limit = bound;
    uint64_t* mine    = sh.gathered[wave];
    int       held    = 0;
    auto      fold    = [&]() {
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        uint64_t key = lane < held ? mine[lane] : 0;
        const uint64_t rest = mine[kWaveSize + lane];
        sort_wave(key);
        const uint64_t reversed = static_cast<uint64_t>(__shfl(static_cast<uint32_t>(key >> 32), kWaveSize - 1 - lane, kWaveSize)) << 32
                                  | __shfl(static_cast<uint32_t>(key), kWaveSize - 1 - lane, kWaveSize);
        merge_wave(list, reversed);
        const uint64_t last = lane_key(list, top - 1);
        limit = last > limit ? last : limit;
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        mine[lane] = rest;
        held = held > kWaveSize ? held - kWaveSize : 0;
    };
    for(int i0 = wave * kWaveSize; i0 < vectors; i0 += WG)
    {
        const int i = i0 + lane;
        row_v4u32 w{};
        int       column = end;
        if(i < vectors)
        {
            const int id = chosen[i / kUnroll], c = id / WG, t = id % WG;
            column = begin + c * SPAN + (i % kUnroll) * WG * N + t * N;
            if(column < end) w = row_load_part(z + column, end - column, RowType<T>::kMinusInf);
        }
        float v[N];
        row_decode<T>(w, v);
#pragma unroll
        for(int e = 0; e < N; ++e)
        {
            const uint64_t key = rank_key(v[e], column + e);
            const bool     in  = column + e < end && key >= limit;
            const uint64_t who = __ballot(in);
            if(!who) continue;
            if(in) mine[held + __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(who >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(who), 0))] = key;
            held += __popcll(who);
            if(held >= kWaveSize) fold();
        }
    }
    if(held > 0) fold();
    return join_lists(list, sh);      // (every wavefront is past the lists' first use: a barrier lies between)
}

// ---- log probabilities --------------------------------------------------------------------------------------------------------
// What a row's moments give: written by the first wavefront, whose lanes hold the alternatives.
template <typename T>
__device__ __forceinline__ void write_logprobs(const LogitsArgs& p, int64_t row, const Moments& r, uint64_t key)
{
    const bool  empty = r.s == 0.0f;      // every logit is -inf
    const float ln_s  = empty ? -INFINITY : logf(r.s);
    const int   lane  = threadIdx.x;
    if(lane == 0)
    {
        if(p.logp)
        {
            const int64_t token = index_at(p.tokens, p.wide, row);
            float         v     = 0.0f;
            if(token >= p.cols) v = NAN;
            else if(token >= 0)
                v = empty ? -INFINITY : (row_element(static_cast<const T*>(p.z) + row * p.ld + token) - r.m) * p.scale - ln_s;
            p.logp[row] = v;
        }
        if(p.entropy)
        {
            const float h  = empty ? 0.0f : ln_s - kLn2 * (r.w / r.s);
            p.entropy[row] = h < 0.0f ? 0.0f : h;
        }
        if(p.stats)
        {
            p.stats[2 * row]     = r.m;
            p.stats[2 * row + 1] = ln_s;
        }
    }
    if(lane < p.top)
    {
        p.top_logp[row * p.top + lane]  = empty ? -INFINITY : (key_value(key) - r.m) * p.scale - ln_s;
        p.top_index[row * p.top + lane] = key ? static_cast<int32_t>(key_column(key)) : -1;
    }
}

// Item: a piece of a row.  One piece a row: the results; several: their moments and lists.
template <typename T, bool ENTROPY, bool TOP> __global__ __launch_bounds__(kRowThreads) void logprobs_kernel(const LogitsArgs p)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ float4 slots[kRowThreads / kWaveSize];
    TopShared&        sh        = *reinterpret_cast<TopShared*>(lds);
    float*            chunk_max = reinterpret_cast<float*>(lds + sizeof(TopShared));
    const float       k2        = p.scale * kLog2e;
    const int64_t     items     = p.rows * p.pieces;
    for(int64_t item = blockIdx.x; item < items; item += gridDim.x)
    {
        const int64_t row   = item / p.pieces;
        const int     begin = static_cast<int>(item - row * p.pieces) * p.piece;
        const int     end   = p.cols - begin < p.piece ? p.cols : begin + p.piece;
        const T*      z     = static_cast<const T*>(p.z) + row * p.ld;
        LaneBest      best;
        Moments       r     = row_pass<T, kRowThreads, ENTROPY, TOP>(z, begin, end, k2, chunk_max, best);
        uint64_t      key   = 0;
        r = join_lanes<kRowThreads>(r, k2, slots);
        if constexpr(TOP)
        {
            const int chunks = (p.piece + chunk_span<T>() - 1) / chunk_span<T>();
            key = row_top(z, begin, end, p.top, best, chunk_max, reinterpret_cast<uint16_t*>(chunk_max + chunks * kRowThreads), sh);
        }
        if(threadIdx.x < kWaveSize)
        {
            if(p.pieces == 1) write_logprobs<T>(p, row, r, key);
            else
            {
                if(threadIdx.x == 0) p.part[item] = make_float4(r.m, r.s, r.w, 0.0f);
                if(TOP && static_cast<int>(threadIdx.x) < p.top) p.part_keys[item * p.top + threadIdx.x] = key;
            }
        }
        __syncthreads();      // (the next item's sums and lists take the same LDS)
    }
}

// The moments of a row's pieces, joined.
template <int WG> __device__ __forceinline__ Moments join_pieces(const float4* part, int pieces, float k2, float4* slots)
{
    Moments r{-FLT_MAX, 0.0f, 0.0f};
    for(int i = threadIdx.x; i < pieces; i += WG)
    {
        const float4 o  = part[i];
        const float  m  = fmaxf(r.m, o.x), a = fmaxf((r.m - m) * k2, kFar), b = fmaxf((o.x - m) * k2, kFar);
        const float  fa = exp2_fast(a), fb = exp2_fast(b);
        r.w = (r.w + a * r.s) * fa + (o.z + b * o.y) * fb;
        r.s = r.s * fa + o.y * fb;
        r.m = m;
    }
    return join_lanes<WG>(r, k2, slots);
}

template <typename T> __global__ __launch_bounds__(kRowThreads) void logprobs_join_kernel(const LogitsArgs p)
{
    __shared__ float4    slots[kRowThreads / kWaveSize];
    __shared__ TopShared sh;
    const int            lane = threadIdx.x % kWaveSize, wave = threadIdx.x / kWaveSize;
    for(int64_t row = blockIdx.x; row < p.rows; row += gridDim.x)
    {
        const Moments r    = join_pieces<kRowThreads>(p.part + row * p.pieces, p.pieces, p.scale * kLog2e, slots);
        uint64_t      list = 0;
        if(p.top > 0)
        {
            for(int i = wave; i < p.pieces; i += kRowThreads / kWaveSize)
            {
                const int at = kWaveSize - 1 - lane;
                merge_wave(list, at < p.top ? p.part_keys[(row * p.pieces + i) * p.top + at] : 0);
            }
            list = join_lists(list, sh);
        }
        if(threadIdx.x < kWaveSize) write_logprobs<T>(p, row, r, list);
        __syncthreads();
    }
}

// ---- gradient of the log probabilities and the entropy ----------------------------------------------------------------------------
struct LogprobsGradArgs
{
    const void*  z;
    int64_t      rows, ld;
    int          cols;
    float        scale;
    int          pieces, piece;
    const void*  tokens;
    int          wide;
    const float *stats, *entropy, *dlogp, *dentropy;      // entropy and dentropy both or neither; dlogp or nullptr
    void*        dz;
    int          ddt;
};

// Walks over [begin, end) of a row in units of eight elements, two of them in flight a lane: body(column, values, valid).
template <typename T, int WG, typename F> __device__ __forceinline__ void row_units(const T* z, int begin, int end, F&& body)
{
    constexpr int U = 2, SPAN = WG * 8;
    int           c = begin + static_cast<int>(threadIdx.x) * 8;
    Row8<T>       next[U];
#pragma unroll
    for(int u = 0; u < U; ++u) next[u].load(z + c + u * SPAN, end - c - u * SPAN);
    for(; c < end; c += U * SPAN)
    {
        float v[U][8];
#pragma unroll
        for(int u = 0; u < U; ++u) next[u].decode(v[u]);
        if(c + U * SPAN < end)
        {
#pragma unroll
            for(int u = 0; u < U; ++u) next[u].load(z + c + (U + u) * SPAN, end - c - (U + u) * SPAN);
        }
#pragma unroll
        for(int u = 0; u < U; ++u)
            if(c + u * SPAN < end) body(c + u * SPAN, v[u], end - c - u * SPAN);
    }
}

__device__ __forceinline__ void store_zeros(void* dz, int ddt, int64_t row_at, int begin, int end, int threads)
{
    for(int c = begin + static_cast<int>(threadIdx.x) * 8; c < end; c += threads * 8)
    {
        float o[8] = {};
        row8_store<false>(dz, ddt, row_at + c, o, end - c);
    }
}

template <typename T, bool ENTROPY> __global__ __launch_bounds__(kRowThreads) void logprobs_grad_kernel(const LogprobsGradArgs p)
{
    const float   k2    = p.scale * kLog2e;
    const int64_t items = p.rows * p.pieces;
    for(int64_t item = blockIdx.x; item < items; item += gridDim.x)
    {
        const int64_t row    = item / p.pieces;
        const int     begin  = static_cast<int>(item - row * p.pieces) * p.piece;
        const int     end    = p.cols - begin < p.piece ? p.cols : begin + p.piece;
        const float   m      = p.stats[2 * row], ln_s = p.stats[2 * row + 1];
        const int64_t given  = p.dlogp ? index_at(p.tokens, p.wide, row) : -1;
        float         g      = given < 0 ? 0.0f : p.dlogp[row] * p.scale;
        float         h = 0.0f, entropy = 0.0f;
        if constexpr(ENTROPY)
        {
            h       = p.dentropy[row] * p.scale;
            entropy = p.entropy[row];
        }
        if(given >= p.cols) g = NAN;      // (no column of it: the row says so)
        const int64_t at = row * p.cols;
        if(ln_s == -INFINITY || (g == 0.0f && h == 0.0f))
        {
            store_zeros(p.dz, p.ddt, at, begin, end, kRowThreads);
            continue;
        }
        const int   token = given < p.cols ? static_cast<int>(given) : -1;
        const float l2 = ln_s * kLog2e;
        row_units<T, kRowThreads>(static_cast<const T*>(p.z) + row * p.ld, begin, end, [&](int c, float(&v)[8], int left) {
            float o[8];
#pragma unroll
            for(int e = 0; e < 8; ++e)
            {
                const float d = (v[e] - m) * k2 - l2, q = exp2_fast(d);      // log2 p and p
                o[e] = -(g * q);
                if constexpr(ENTROPY) o[e] = fmaf(-(h * q), fmaf(fmaxf(d, kFar), kLn2, entropy), o[e]);
            }
            if(static_cast<unsigned>(token - c) < 8u)
            {
#pragma unroll
                for(int e = 0; e < 8; ++e) o[e] += token - c == e ? g : 0.0f;
            }
            row8_store<false>(p.dz, p.ddt, at + c, o, left);
        });
    }
}

// ---- distillation ---------------------------------------------------------------------------------------------------------------
struct DistillArgs
{
    const void*  z;
    int64_t      rows, ld;
    int          cols;
    float        scale;
    int          pieces, piece;
    const void*  teacher;
    int          tdt;
    const void*  index;
    int          wide, k;
    const float* weight;      // or nullptr: 1
    float*       loss;
    void*        dz;          // or nullptr
    int          ddt;
    float4*      part;
};

constexpr int kEntries = kTeacherEntries;      // one a thread

struct EntriesShared
{
    int    column[kEntries];
    float  q[kEntries];
    float4 slots[16];
};

// A thread's entry of the teacher's.
struct Entry
{
    int   column = -1;
    float q = 0.0f, z = 0.0f;
    bool  any = false;      // (of the row) some entry has weight
    bool  bad = false;      // (of the row) a column beyond the vocabulary, or a NaN of the teacher's
};

template <int WG, bool MAX> __device__ __forceinline__ float block_all(float v, float* slots)
{
    v = MAX ? wave64_max(v) : wave64_sum(v);
    if(threadIdx.x % kWaveSize == 0) slots[threadIdx.x / kWaveSize] = v;
    __syncthreads();
    float t = slots[0];
#pragma unroll
    for(int w = 1; w < WG / kWaveSize; ++w) t = MAX ? fmaxf(t, slots[w]) : t + slots[w];
    return t;
}

// Loads the entries, the teacher's probabilities and the row's loss.
template <typename T, int WG>
__device__ __forceinline__ Entry row_entries(const DistillArgs& p, int64_t row, const Moments& r, float ln_s, EntriesShared& sh, float& loss)
{
    const int tid = threadIdx.x;
    Entry     e;
    float     t = -INFINITY, bad = 0.0f;
    if(tid < p.k)
    {
        const int64_t at = row * p.k + tid, column = index_at(p.index, p.wide, at);
        if(column >= p.cols) bad = 1.0f;
        else if(column >= 0)
        {
            e.column = static_cast<int>(column);
            t = p.tdt == kF32 ? row_element(static_cast<const float*>(p.teacher) + at)
                : p.tdt == kF16 ? row_element(static_cast<const _Float16*>(p.teacher) + at)
                                : row_element(static_cast<const __bf16*>(p.teacher) + at);
            e.z = row_element(static_cast<const T*>(p.z) + row * p.ld + e.column);
            if(t != t) bad = 1.0f;
        }
    }
    float*      slots = reinterpret_cast<float*>(sh.slots);
    const float top   = block_all<WG, true>(t, slots);
    e.bad = block_all<WG, true>(bad, slots + 16) > 0.0f;
    e.any = top > -INFINITY;
    const float mass  = e.any ? exp2_fast((t - top) * (p.scale * kLog2e)) : 0.0f;
    const float total = block_all<WG, false>(mass, slots + 32);
    float       part  = 0.0f;
    if(e.any && mass != 0.0f)
    {
        e.q = mass / total;
        // q (log q - log p), the logit's part by itself: a mask of the lowest value times the scale need not be a finite logarithm
        part = r.s == 0.0f ? INFINITY : e.q * ((t - top) * p.scale - logf(total) + ln_s) - (e.q * p.scale) * (e.z - r.m);
    }
    if(tid < p.k) { sh.column[tid] = e.column; sh.q[tid] = e.q; }
    loss = block_all<WG, false>(part, slots + 48);
    if(e.bad) loss = NAN;
    return e;
}

// The gradient of [begin, end): the student's probabilities, then, over them, the entries' columns less the teacher's.
template <typename T, int WG>
__device__ __forceinline__ void row_gradient(const DistillArgs& p, int64_t row, int begin, int end, const Moments& r, float ln_s, const Entry& e,
                                             const EntriesShared& sh)
{
    const float   weight = p.weight ? p.weight[row] : 1.0f;
    const int64_t at     = row * p.cols;
    float         g      = weight * p.scale;
    if(e.bad && weight != 0.0f) g = NAN;
    if(weight == 0.0f || r.s == 0.0f || !(e.any || e.bad))
    {
        store_zeros(p.dz, p.ddt, at, begin, end, WG);
        return;
    }
    const float k2 = p.scale * kLog2e, l2 = ln_s * kLog2e;
    row_units<T, WG>(static_cast<const T*>(p.z) + row * p.ld, begin, end, [&](int c, float(&v)[8], int left) {
        float o[8];
#pragma unroll
        for(int i = 0; i < 8; ++i) o[i] = g * exp2_fast((v[i] - r.m) * k2 - l2);
        row8_store<false>(p.dz, p.ddt, at + c, o, left);
    });
    __syncthreads();      // (behind the probabilities)
    if(static_cast<int>(threadIdx.x) < p.k && e.column >= begin && e.column < end)
    {
        float q = 0.0f;      // of all entries of this column
        for(int i = 0; i < p.k; ++i) q += sh.column[i] == e.column ? sh.q[i] : 0.0f;
        const float v = g * (exp2_fast((e.z - r.m) * k2 - l2) - q);
        if(p.ddt == kF16) static_cast<_Float16*>(p.dz)[at + e.column] = static_cast<_Float16>(v);
        else if(p.ddt == kBF16) static_cast<__bf16*>(p.dz)[at + e.column] = static_cast<__bf16>(v);
        else static_cast<float*>(p.dz)[at + e.column] = v;
    }
}

__device__ __forceinline__ float log_sum(const Moments& r) { return r.s == 0.0f ? -INFINITY : logf(r.s); }

// A row a workgroup: both passes, the second one out of a cache.
template <typename T, int WG> __global__ __launch_bounds__(WG) void distill_row_kernel(const DistillArgs p)
{
    __shared__ EntriesShared sh;
    __shared__ float4        slots[WG / kWaveSize];
    const float              k2 = p.scale * kLog2e;
    for(int64_t row = blockIdx.x; row < p.rows; row += gridDim.x)
    {
        LaneBest      none;
        const Moments r = join_lanes<WG>(row_pass<T, WG, false, false>(static_cast<const T*>(p.z) + row * p.ld, 0, p.cols, k2, nullptr, none), k2, slots);
        const float   ln_s = log_sum(r);
        float         loss;
        const Entry   e = row_entries<T, WG>(p, row, r, ln_s, sh, loss);
        if(threadIdx.x == 0) p.loss[row] = loss;
        if(p.dz) row_gradient<T, WG>(p, row, 0, p.cols, r, ln_s, e, sh);
        __syncthreads();
    }
}

// Few rows: the moments of the pieces ...
template <typename T> __global__ __launch_bounds__(kRowThreads) void distill_pieces_kernel(const DistillArgs p)
{
    __shared__ float4 slots[kRowThreads / kWaveSize];
    const float       k2    = p.scale * kLog2e;
    const int64_t     items = p.rows * p.pieces;
    for(int64_t item = blockIdx.x; item < items; item += gridDim.x)
    {
        const int64_t row   = item / p.pieces;
        const int     begin = static_cast<int>(item - row * p.pieces) * p.piece;
        const int     end   = p.cols - begin < p.piece ? p.cols : begin + p.piece;
        LaneBest      none;
        const Moments r = join_lanes<kRowThreads>(
            row_pass<T, kRowThreads, false, false>(static_cast<const T*>(p.z) + row * p.ld, begin, end, k2, nullptr, none), k2, slots);
        if(threadIdx.x == 0) p.part[item] = make_float4(r.m, r.s, r.w, 0.0f);
        __syncthreads();
    }
}
// ... then the loss (by a row's first workgroup) and the gradient of every piece; without a gradient a workgroup a row
template <typename T> __global__ __launch_bounds__(kRowThreads) void distill_join_kernel(const DistillArgs p)
{
    __shared__ EntriesShared sh;
    __shared__ float4        slots[kRowThreads / kWaveSize];
    const int64_t            items = p.dz ? p.rows * p.pieces : p.rows;
    for(int64_t item = blockIdx.x; item < items; item += gridDim.x)
    {
        const int64_t row  = p.dz ? item / p.pieces : item;
        const int     i    = p.dz ? static_cast<int>(item - row * p.pieces) : 0;
        const Moments r    = join_pieces<kRowThreads>(p.part + row * p.pieces, p.pieces, p.scale * kLog2e, slots);
        const float   ln_s = log_sum(r);
        float         loss;
        const Entry   e = row_entries<T, kRowThreads>(p, row, r, ln_s, sh, loss);
        if(p.loss && i == 0 && threadIdx.x == 0) p.loss[row] = loss;
        if(p.dz)
        {
            const int begin = i * p.piece, end = p.cols - begin < p.piece ? p.cols : begin + p.piece;
            row_gradient<T, kRowThreads>(p, row, begin, end, r, ln_s, e, sh);
        }
        __syncthreads();
    }
}

// ---- launches -------------------------------------------------------------------------------------------------------------------
constexpr int64_t kFill = 1024;           // workgroups that fill the device: four on every compute unit
constexpr int64_t kMostGroups = 1 << 22;  // of a launch; larger problems loop

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
int vector_elements(int dt) { return dt == kF32 ? 4 : 8; }

struct Split { int pieces, piece; };
// Pieces of a row: enough to fill the device, of one vector a thread at least, and of `most` elements at most.
Split split_rows(int64_t rows, int64_t cols, int64_t least, int64_t most)
{
    int64_t pieces = div_up(kFill, rows);
    if(pieces > div_up(cols, least)) pieces = div_up(cols, least);
    if(pieces < div_up(cols, most)) pieces = div_up(cols, most);
    if(pieces < 1) pieces = 1;
    int64_t piece = div_up(div_up(cols, pieces), least) * least;
    if(piece > most) piece = most;
    return Split{static_cast<int>(div_up(cols, piece)), static_cast<int>(piece)};
}
Split logprobs_split(int zdt, int64_t rows, int64_t cols, int top)
{
    const int64_t vector = static_cast<int64_t>(kRowThreads) * vector_elements(zdt);
    return split_rows(rows, cols, vector, top > 0 ? vector * kUnroll * kMaxChunks : kLogitsMaxCols);
}
// what `rows` rows or fewer are cut into at most
int64_t most_items(int zdt, int64_t rows, int64_t cols, int top)
{
    const int64_t vector = static_cast<int64_t>(kRowThreads) * vector_elements(zdt);
    const int64_t fill = kFill + rows, cap = rows * (top > 0 ? div_up(cols, vector * kUnroll * kMaxChunks) : div_up(cols, kLogitsMaxCols));
    return fill > cap ? fill : cap;
}
dim3 groups(int64_t items) { return dim3(static_cast<unsigned>(items < kMostGroups ? items : kMostGroups)); }

template <typename T> hipError_t logprobs_type(const LogitsArgs& a, hipStream_t st)
{
    const dim3   grid = groups(a.rows * a.pieces), block(kRowThreads);
    const size_t lds  = a.top > 0 ? top_lds_bytes((a.piece + chunk_span<T>() - 1) / chunk_span<T>()) : 0;
    if(a.top > 0)
    {
        if(a.entropy) logprobs_kernel<T, true, true><<<grid, block, lds, st>>>(a);
        else          logprobs_kernel<T, false, true><<<grid, block, lds, st>>>(a);
    }
    else
    {
        if(a.entropy) logprobs_kernel<T, true, false><<<grid, block, 0, st>>>(a);
        else          logprobs_kernel<T, false, false><<<grid, block, 0, st>>>(a);
    }
    hipError_t e = hipGetLastError();
    if(e != hipSuccess || a.pieces == 1) return e;
    logprobs_join_kernel<T><<<groups(a.rows), block, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T> hipError_t logprobs_grad_type(const LogprobsGradArgs& a, hipStream_t st)
{
    if(a.dentropy) logprobs_grad_kernel<T, true><<<groups(a.rows * a.pieces), dim3(kRowThreads), 0, st>>>(a);
    else           logprobs_grad_kernel<T, false><<<groups(a.rows * a.pieces), dim3(kRowThreads), 0, st>>>(a);
    return hipGetLastError();
}

template <typename T> hipError_t distill_type(const DistillArgs& a, hipStream_t st)
{
    if(a.pieces == 1)
    {
        distill_row_kernel<T, kRowThreads><<<groups(a.rows), dim3(kRowThreads), 0, st>>>(a);
        return hipGetLastError();
    }
    distill_pieces_kernel<T><<<groups(a.rows * a.pieces), dim3(kRowThreads), 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if(e != hipSuccess) return e;
    DistillArgs rest = a;
    if(a.dz && a.dz == a.z)
    {   // in place, a piece's gradient takes the place of logits that another workgroup's loss needs: the losses first
        rest.dz = nullptr;
        distill_join_kernel<T><<<groups(a.rows), dim3(kRowThreads), 0, st>>>(rest);
        e = hipGetLastError();
        if(e != hipSuccess) return e;
        rest.dz   = a.dz;
        rest.loss = nullptr;
    }
    distill_join_kernel<T><<<groups(a.dz ? a.rows * a.pieces : a.rows), dim3(kRowThreads), 0, st>>>(rest);
    return hipGetLastError();
}

template <typename F> hipError_t by_type(int dt, F&& f) { return dt == kF32 ? f(float{}) : dt == kF16 ? f(_Float16{}) : f(__bf16{}); }

}  // namespace

size_t token_logprobs_workspace_bytes(int zdt, int64_t rows, int64_t cols, int top)
{
    return static_cast<size_t>(most_items(zdt, rows, cols, top)) * (sizeof(float4) + static_cast<size_t>(top) * sizeof(uint64_t));
}

hipError_t launch_token_logprobs(const void* z, int zdt, int64_t rows, int64_t cols, int64_t ld, float scale, const void* tokens, bool wide,
                                 float* logp, float* entropy, float* stats, int top, float* top_logp, int32_t* top_index, void* workspace,
                                 hipStream_t st)
{
    const Split s = logprobs_split(zdt, rows, cols, top);
    LogitsArgs  a{};
    a.z = z; a.rows = rows; a.ld = ld; a.cols = static_cast<int>(cols); a.scale = scale;
    a.pieces = s.pieces; a.piece = s.piece;
    a.tokens = tokens; a.wide = wide; a.logp = logp; a.entropy = entropy; a.stats = stats;
    a.top = top; a.top_logp = top_logp; a.top_index = top_index;
    a.part = static_cast<float4*>(workspace);
    a.part_keys = reinterpret_cast<uint64_t*>(a.part + rows * s.pieces);
    return by_type(zdt, [&](auto tag) { return logprobs_type<decltype(tag)>(a, st); });
}

hipError_t launch_token_logprobs_bwd(const void* z, int zdt, int64_t rows, int64_t cols, int64_t ld, float scale, const void* tokens, bool wide,
                                     const float* stats, const float* entropy, const float* dlogp, const float* dentropy, void* dz, int ddt,
                                     hipStream_t st)
{
    const Split      s = split_rows(rows, cols, kRowThreads * 8, kRowThreads * 8 * 16);
    LogprobsGradArgs a{};
    a.z = z; a.rows = rows; a.ld = ld; a.cols = static_cast<int>(cols); a.scale = scale;
    a.pieces = s.pieces; a.piece = s.piece;
    a.tokens = tokens; a.wide = wide; a.stats = stats; a.entropy = entropy; a.dlogp = dlogp; a.dentropy = dentropy;
    a.dz = dz; a.ddt = ddt;
    return by_type(zdt, [&](auto tag) { return logprobs_grad_type<decltype(tag)>(a, st); });
}

size_t distill_topk_workspace_bytes(int zdt, int64_t rows, int64_t cols) { return static_cast<size_t>(most_items(zdt, rows, cols, 0)) * sizeof(float4); }

hipError_t launch_distill_topk(const void* z, int zdt, int64_t rows, int64_t cols, int64_t ld, float scale, const void* teacher, int tdt,
                               const void* index, bool wide, int k, const float* weight, float* loss, void* dz, int ddt, void* workspace,
                               hipStream_t st)
{
    const Split s = logprobs_split(zdt, rows, cols, 0);
    DistillArgs a{};
    a.z = z; a.rows = rows; a.ld = ld; a.cols = static_cast<int>(cols); a.scale = scale;
    a.pieces = s.pieces; a.piece = s.piece;
    a.teacher = teacher; a.tdt = tdt; a.index = index; a.wide = wide; a.k = k; a.weight = weight; a.loss = loss;
    a.dz = dz; a.ddt = ddt;
    a.part = static_cast<float4*>(workspace);
    return by_type(zdt, [&](auto tag) { return distill_type<decltype(tag)>(a, st); });
}

}  // namespace qsync
