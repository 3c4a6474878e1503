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

#include <algorithm>
#include <cfloat>
#include <type_traits>

namespace qsync {

namespace {

constexpr int   kRowThreads = 256;        // a row, or a piece of one
constexpr int   kUnroll     = 4;          // vectors of a lane in flight: a chunk
constexpr float kLn2 = 0.693147180559945309f, kLog2e = 1.44269504088896341f;
constexpr float kFar = -1.0e30f;          // stands for differences to the maximum that overflow: e^x is 0 there, and 0 * x is 0
// The fast form of a pass (row_pass) leaves the rounding of m k2 in its exponents, half a spacing of fp32 there: at most 64 below 2^31, and
// 2^64 times a row's 2^30 terms is still finite.  (Masks of -1e9 at a scale of 1 lie within; at 2^32 a row of one such value would be 0 or infinite.)
constexpr float kNearProduct = 2.0e9f;
constexpr int   kTopMost = kTopAlternatives;      // a sorted list is a value per lane
static_assert(kTopMost == kWaveSize, "an alternative per lane");

template <typename T> constexpr int chunk_span(int threads) { return threads * RowType<T>::N * kUnroll; }      // elements of a workgroup's chunks

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
    float       reach;              // see set_scale.  (It and k2 lie in gaps: eight bytes more put the grid's size, which stands behind
                                    // these, into a third line of memory, 4 x 131072 bfloat16 with 20 alternatives 12.0 -> 12.4 us.)
    float *     logp, *entropy, *stats;
    int         top;
    float       k2;
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

// Joins the lanes' moments; the result in every lane.  `slots`: one per wavefront.  FAR: what the references differ by is their difference
// times k2; otherwise the difference of their products, which is what a lane's own terms are relative to (row_pass), and at the end the
// rounding of the joined one's product is taken out of the sums.
template <int WG, bool FAR> __device__ __forceinline__ Moments join_lanes(Moments a, float k2, float4* slots)
{
    auto apart = [&](float x, float m) { return FAR ? fmaxf((x - m) * k2, kFar) : x * k2 - m * k2; };
    const float m  = wave64_max(a.m);
    const float dm = apart(a.m, m), f = exp2_fast(dm);
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
        const float  d = apart(o.x, r.m), g = exp2_fast(d);
        r.s += o.y * g;
        r.w += (o.z + d * o.y) * g;
    }
    if constexpr(!FAR)
    {
        const float d = -fmaf(r.m, k2, -(r.m * k2)), g = exp2_fast(d);
        r.w = (r.w + d * r.s) * g;
        r.s *= g;
    }
    return r;
}

// The maximum that a top search keeps of a lane: value and the chunk it was first met in.
struct LaneBest
{
    float value = -INFINITY;
    int   chunk = -1;
};

// A row's elements [begin, end): whole 16-byte lines of memory, taken as vectors, and the fewer than two lines' elements in front of and
// behind them, one each for the first threads ("edge").  A row of an odd number of elements is so read and written in whole lines: 2048 x
// 65535 bfloat16 63.0 -> 54.8 us, a distillation step over 4096 x 65535 363 -> 256.  ONCE: the loads are streamed, so that they leave the
// caches to what is read again -- the gradient, for one, by the head's backward pass (us: log probabilities of 2048 x 65536 bfloat16 55 ->
// 49, a distillation step over 1024 x 32768 binary16 41.3 -> 39.1, with the INT8 conversion of its gradient 74.5 -> 71.8).
template <typename T, bool ONCE> struct RowSpan
{
    const T* row;
    int      begin, end, body, vectors;      // body: column of the first vector
    __device__ RowSpan() {}
    __device__ RowSpan(const T* r, int b, int e) : row(r), begin(b), end(e)
    {
        constexpr int N    = RowType<T>::N;
        const int     past = static_cast<int>((reinterpret_cast<uintptr_t>(r + b) & 15u) / sizeof(T)), head = past ? N - past : 0;
        body    = b + (head < e - b ? head : e - b);
        vectors = (e - body) / N;
    }
    // the column of thread t's edge element, or -1
    __device__ int edge(int t) const
    {
        if(t < body - begin) return begin + t;
        const int behind = body + vectors * RowType<T>::N + t - (body - begin);
        return behind < end ? behind : -1;
    }
    template <int WG, int U = kUnroll> __device__ int chunks() const { return (vectors + WG * U - 1) / (WG * U); }
    // the number of vector u of chunk c of thread t, and a vector's column
    template <int WG, int U = kUnroll> static __device__ int vector(int c, int u, int t) { return (c * U + u) * WG + t; }
    // the vectors from number i on, without edges
    template <bool S> __device__ RowSpan<T, S> from(int i) const
    {
        RowSpan<T, S> s;
        s.row     = row;
        s.vectors = vectors > i ? vectors - i : 0;
        s.begin = s.body = column(i);
        s.end = s.body + s.vectors * RowType<T>::N;
        return s;
    }
    __device__ int column(int i) const { return body + i * RowType<T>::N; }
    // (a row's address in scalar registers and 32-bit offsets: a row of 2^30 fp32 elements ends below 2^32 bytes)
    __device__ __forceinline__ const T* at(int i) const
    {
        return reinterpret_cast<const T*>(reinterpret_cast<const uint8_t*>(row) + static_cast<uint32_t>(column(i)) * static_cast<uint32_t>(sizeof(T)));
    }
    __device__ __forceinline__ row_v4u32 load(int i) const { return row_load<ONCE>(at(i)); }
};

// One pass over a span.  FAR: the differences to the maximum are taken first, so that any finite logits do; otherwise z k2 less the rounded
// product m k2 is one operation, for rows whose maximum lies within `reach`.  A lane's reference does not go below -reach, whatever it has met:
// masked logits far below it are terms of 0 beside such a maximum, and so is what a lane that meets nothing else adds up.  The lanes'
// sums are relative to the product; join_lanes keeps to it.
template <typename T, int WG, int U, bool ENTROPY, bool TOP, bool FAR, bool ONCE>
__device__ __forceinline__ Moments row_pass(const RowSpan<T, ONCE>& z, float k2, float reach, float* chunk_max, LaneBest& best)
{
    constexpr int N = RowType<T>::N;
    const int     tid = threadIdx.x, chunks = z.template chunks<WG, U>();
    row_v4u32     next[U];
    auto          fetch = [&](int c) {
        if((c + 1) * U * WG <= z.vectors)
        {
#pragma unroll
            for(int u = 0; u < U; ++u) next[u] = z.load(z.template vector<WG, U>(c, u, tid));
            return;
        }
#pragma unroll
        for(int u = 0; u < U; ++u)
        {
            constexpr uint32_t absent = RowType<T>::kMinusInf;
            next[u] = row_v4u32{absent, absent, absent, absent};
            if(tid < z.vectors - z.template vector<WG, U>(c, u, 0)) next[u] = z.load(z.template vector<WG, U>(c, u, tid));
        }
    };
    const int edge = z.edge(tid);
    if(chunks > 0) fetch(0);
    Moments r{FAR ? -FLT_MAX : -reach, 0.0f, 0.0f};
    if(edge >= 0)
    {
        const float v = row_element(z.row + edge);
        r.m = fmaxf(r.m, v);
        const float d = FAR ? (v - r.m) * k2 : fmaf(v, k2, -(r.m * k2));      // (not 0: what the product lost by its rounding)
        r.s = exp2_fast(d);
        if constexpr(ENTROPY) r.w = r.s * fmaxf(d, kFar);
    }
    for(int c = 0; c < chunks; ++c)
    {
        float v[U * N];
#pragma unroll
        for(int u = 0; u < U; ++u) row_decode<T>(next[u], v + u * N);
        if(c + 1 < chunks) fetch(c + 1);
        float top = v[0];
#pragma unroll
        for(int i = 1; i < U * N; ++i) top = fmaxf(top, v[i]);
        if constexpr(TOP)
        {
            chunk_max[c * WG + tid] = top;
            best.chunk = top > best.value ? c : best.chunk;
            best.value = top > best.value ? top : best.value;
        }
        const float m  = fmaxf(r.m, top), mk = m * k2;
        const float dm = FAR ? fmaxf((r.m - m) * k2, kFar) : r.m * k2 - mk, f = exp2_fast(dm);
        if constexpr(ENTROPY) r.w = (r.w + dm * r.s) * f;
        r.s *= f;
        r.m = m;
#pragma unroll
        for(int i = 0; i < U * N; ++i)
        {
            const float d = FAR ? (v[i] - m) * k2 : fmaf(v[i], k2, -mk), e = exp2_fast(d);
            r.s += e;
            if constexpr(ENTROPY) r.w = fmaf(e, fmaxf(d, kFar), r.w);
        }
    }
    return r;
}

// The moments of a span, in every lane.
template <typename T, int WG, int U, bool ENTROPY, bool TOP, bool ONCE>
__device__ __forceinline__ Moments span_moments(const RowSpan<T, ONCE>& z, float k2, float reach, float* chunk_max, LaneBest& best, float4* slots)
{
    const Moments r = join_lanes<WG, false>(row_pass<T, WG, U, ENTROPY, TOP, false>(z, k2, reach, chunk_max, best), k2, slots);
    if(fabsf(r.m) < reach) return r;
    __syncthreads();      // (all lanes have read the slots)
    LaneBest none;
    return join_lanes<WG, true>(row_pass<T, WG, 1, ENTROPY, false, true>(z, k2, reach, nullptr, none), k2, slots);
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

// The value of the lane whose index differs in the bits of MASK, a power of two: on the data-parallel primitives and the row swaps,
// which answer in a few cycles where a permutation through LDS takes a hundred (2048 x 32768 binary16, 8 alternatives: 42.0 -> 38.6 us).
template <int MASK> __device__ __forceinline__ uint32_t lane_xor(uint32_t v)
{
    if constexpr(MASK == 1) return __builtin_amdgcn_update_dpp(v, v, 0xB1, 0xF, 0xF, false);             // quad_perm 1 0 3 2
    else if constexpr(MASK == 2) return __builtin_amdgcn_update_dpp(v, v, 0x4E, 0xF, 0xF, false);        // quad_perm 2 3 0 1
    else if constexpr(MASK == 4)
    {   // four lanes on (row_shl) into the quads of even number, four lanes back (row_shr) into the others
        const uint32_t r = __builtin_amdgcn_update_dpp(v, v, 0x104, 0xF, 0x5, false);
        return __builtin_amdgcn_update_dpp(r, v, 0x114, 0xF, 0xA, false);
    }
    else if constexpr(MASK == 8) return __builtin_amdgcn_update_dpp(v, v, kRotate + 8, 0xF, 0xF, false);
    else if constexpr(MASK == 16)
    {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    }
    else
    {
        static_assert(MASK == 32, "a power of two below 64");
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
}
template <int MASK> __device__ __forceinline__ uint64_t lane_xor(uint64_t v)
{
    return static_cast<uint64_t>(lane_xor<MASK>(static_cast<uint32_t>(v >> 32))) << 32 | lane_xor<MASK>(static_cast<uint32_t>(v));
}
// The keys of a wavefront in descending order of the lanes: bitonic sort, and its last stage alone.
template <int SIZE, int J = SIZE / 2> __device__ __forceinline__ void bitonic_stage(uint64_t& key)
{
    const int      lane   = threadIdx.x % kWaveSize;
    const uint64_t other  = lane_xor<J>(key);
    const bool     larger = ((lane & J) == 0) == ((lane & SIZE) == 0);
    key = (key > other) == larger ? key : other;
    if constexpr(J > 1) bitonic_stage<SIZE, J / 2>(key);
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

// LDS of a top search beside the chunk maxima.
constexpr int kGathered = 256;
struct TopShared
{
    uint64_t claim[kRowThreads];
    uint64_t list[4][kTopMost];
    uint64_t gathered[kGathered];
    uint64_t folding[4][2 * kTopMost];
    uint64_t bound;
    int      chosen, found;
};
// chunk maxima and the chosen chunks' numbers
constexpr size_t top_lds_bytes(int chunks) { return static_cast<size_t>(chunks) * kRowThreads * (sizeof(float) + sizeof(uint16_t)); }

// The first wavefront joins `lists` descending lists, its own and those of the next wavefronts.
__device__ __forceinline__ void join_lists(uint64_t& key, int lists, uint64_t (&list)[4][kTopMost])
{
    const int lane = threadIdx.x % kWaveSize, wave = threadIdx.x / kWaveSize;
    if(wave > 0 && wave < lists) list[wave][kWaveSize - 1 - lane] = key;
    __syncthreads();
    if(wave == 0)
        for(int w = 1; w < lists; ++w) merge_wave(key, list[w][lane]);
}

// The `top` largest of a span, descending over the lanes of the first wavefront (0: fewer elements than that).
// The k-th largest of the maxima of 64 or 256 groups of lanes is a bound that at least k elements reach; a chunk whose maximum stays
// below it is not looked at again.  About k chunks (32 or 16 elements) remain of a row, and never more than the k best groups
// have; they are read a second time, out of a cache, and what reaches the bound is sorted.  The work beside the pass hardly depends on
// the order of the logits, and the order (value, then lower column) makes equal logits as good as different ones.
template <typename T, bool ONCE>
__device__ __forceinline__ uint64_t row_top(const RowSpan<T, ONCE>& z, int top, const LaneBest& best, const float* chunk_max, uint16_t* chosen, TopShared& sh)
{
    constexpr int N = RowType<T>::N, WG = kRowThreads, WAVES = WG / kWaveSize;
    const int     tid = threadIdx.x, lane = tid % kWaveSize, wave = tid / kWaveSize, chunks = z.template chunks<WG>();
    // a lane's claim: an element of at least this value at this column or in front of it
    uint64_t claim = 0;
    if(best.chunk >= 0) claim = rank_key(best.value, z.column(z.template vector<WG>(best.chunk, kUnroll - 1, tid)) + N - 1);
    else if(tid < z.vectors) claim = rank_key(-INFINITY, z.column(tid));
    sh.claim[tid] = claim;
    if(tid == 0) sh.chosen = sh.found = 0;
    __syncthreads();
    const int lists = top <= kTopMost / 2 ? 1 : 4;      // groups of lanes, 64 or 256: the fewer, the more elements reach the bound
    if(wave < lists)
    {
        claim = 0;
        for(int w = wave; w < WAVES; w += lists)
        {
            const uint64_t other = sh.claim[w * kWaveSize + lane];
            claim = claim > other ? claim : other;
        }
        sort_wave(claim);
    }
    if(lists > 1) join_lists(claim, lists, sh.list);
    if(wave == 0) sh.bound = lane_key(claim, top - 1);
    __syncthreads();
    const uint64_t bound = sh.bound;

    for(int c = 0; c < chunks; ++c)
        if(rank_key(chunk_max[c * WG + tid], z.column(z.template vector<WG>(c, 0, tid))) >= bound)
            chosen[atomicAdd(&sh.chosen, 1)] = static_cast<uint16_t>(c * WG + tid);
    __syncthreads();
    const int vectors = sh.chosen * kUnroll;
    // body(key, reaches the bound, how many lanes in front do, how many do) for the elements of the chosen chunks, in wavefronts, of which
    // `of` share the vectors; the first one has the edges too
    auto chosen_keys = [&](int of, uint64_t& limit, auto&& body) {
        auto offer = [&](float v, int column, bool in) {
            const uint64_t key = rank_key(v, static_cast<uint32_t>(column));
            in = in && key >= limit;
            const uint64_t who = __ballot(in);
            if(who) body(key, in, __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(who >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(who), 0)),
                         __popcll(who));
        };
        if(wave == 0)
        {
            const int edge = z.edge(lane);
            offer(edge >= 0 ? row_element(z.row + edge) : 0.0f, edge, edge >= 0);
        }
        for(int i0 = wave * kWaveSize; i0 < vectors; i0 += of * kWaveSize)
        {
            const int i = i0 + lane;
            row_v4u32 w{};
            int       vector = z.vectors;
            if(i < vectors)
            {
                const int id = chosen[i / kUnroll];
                vector = z.template vector<WG>(id / WG, i % kUnroll, id % WG);
                if(vector < z.vectors) w = z.load(vector);
            }
            float v[N];
            row_decode<T>(w, v);
#pragma unroll
            for(int e = 0; e < N; ++e) offer(v[e], z.column(vector) + e, vector < z.vectors);
        }
    };
    uint64_t limit = bound, key = 0;
    chosen_keys(WAVES, limit, [&](uint64_t k, bool in, int place, int count) {
        int at = 0;
        if(lane == 0) at = atomicAdd(&sh.found, count);
        at = __builtin_amdgcn_readfirstlane(at) + place;
        if(in && at < kGathered) sh.gathered[at] = k;
    });
    __syncthreads();
    const int found = sh.found;
    if(found <= kGathered)
    {
        const int full = (found + kWaveSize - 1) / kWaveSize;
        if(wave < full)
        {
            const int i = wave * kWaveSize + lane;
            key = i < found ? sh.gathered[i] : 0;
            sort_wave(key);
        }
        if(full > 1) join_lists(key, full, sh.list);
        return key;
    }
    // more than there is room for (the best logits side by side): four wavefronts keep the largest 64 of theirs as they go
    if(wave < 4)
    {
        uint64_t* mine   = sh.folding[wave];
        int       held   = 0;
        bool      folded = false;
        auto      fold   = [&]() {
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
            uint64_t       next = lane < held ? mine[lane] : 0;
            const uint64_t rest = mine[kWaveSize + lane];
            sort_wave(next);
            if(folded)
            {
                mine[kWaveSize - 1 - lane] = next;
                __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
                merge_wave(key, mine[lane]);
                __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
            }
            else key = next;
            folded = true;
            const uint64_t last = lane_key(key, top - 1);
            limit = last > limit ? last : limit;
            mine[lane] = rest;
            held = held > kWaveSize ? held - kWaveSize : 0;
        };
        chosen_keys(4, limit, [&](uint64_t k, bool in, int place, int count) {
            if(in) mine[held + place] = k;
            held += count;
            if(held >= kWaveSize) fold();
        });
        if(held > 0) fold();
    }
    join_lists(key, 4, sh.list);
    return key;
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
// Bound by memory without alternatives (2048 x 65536 bfloat16 49 us, 5.4 TB/s) and with many (64 of 1024 x 131072 bfloat16 55 us, 4.9);
// rows of 64 KB in 16 bits are also bound by the vector unit, seven instructions a logit, one of them the exponential (four cycles' worth),
// and by the searches of the four workgroups on a compute unit, which end their rows together: 8 of 2048 x 32768 binary16 33 us, without
// them 27.
template <typename T, bool ENTROPY, bool TOP> __global__ __launch_bounds__(kRowThreads) void logprobs_kernel(const LogitsArgs p)
{
    constexpr int WG = kRowThreads;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ float4 slots[WG / kWaveSize];
    float*            chunk_max = reinterpret_cast<float*>(lds);
    float             k2        = p.k2;
    asm volatile("" : "+v"(k2));      // (in a vector register: scalar ones are short here, and are spilled)
    const int64_t     items     = p.rows * p.pieces;
    for(int64_t item = blockIdx.x; item < items; item += gridDim.x)
    {
        const int64_t    row   = item / p.pieces;
        const int        begin = static_cast<int>(item - row * p.pieces) * p.piece;
        const RowSpan<T, true> z(static_cast<const T*>(p.z) + row * p.ld, begin, p.cols - begin < p.piece ? p.cols : begin + p.piece);
        LaneBest         best;
        const Moments    r   = span_moments<T, WG, kUnroll, ENTROPY, TOP>(z, k2, p.reach, chunk_max, best, slots);
        uint64_t         key = 0;
        if constexpr(TOP)
        {
            __shared__ TopShared sh;
            key = row_top(z, p.top, best, chunk_max, reinterpret_cast<uint16_t*>(chunk_max + z.template chunks<WG>() * WG), sh);
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

// The moments of a row's pieces, joined, and their lists (the second launch: 4.9 us for 20 alternatives of 4 x 131072 bfloat16).
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
    return join_lanes<WG, true>(r, k2, slots);
}

template <typename T> __global__ __launch_bounds__(kRowThreads) void logprobs_join_kernel(const LogitsArgs p)
{
    __shared__ float4   slots[kRowThreads / kWaveSize];
    __shared__ uint64_t lists[4][kTopMost];
    const int           lane = threadIdx.x % kWaveSize, wave = threadIdx.x / kWaveSize;
    for(int64_t row = blockIdx.x; row < p.rows; row += gridDim.x)
    {
        const Moments r    = join_pieces<kRowThreads>(p.part + row * p.pieces, p.pieces, p.k2, slots);
        uint64_t      list = 0;
        if(p.top > 0)
        {
            constexpr int   WAVES = kRowThreads / kWaveSize, AHEAD = 4;      // lists of a wavefront under way
            const int       at    = kWaveSize - 1 - lane;
            const uint64_t* keys  = p.part_keys + row * p.pieces * p.top + at;
            for(int i = wave; i < p.pieces; i += AHEAD * WAVES)
            {
                uint64_t next[AHEAD];
#pragma unroll
                for(int a = 0; a < AHEAD; ++a)
                    next[a] = at < p.top && i + a * WAVES < p.pieces ? keys[static_cast<int64_t>(i + a * WAVES) * p.top] : 0;
#pragma unroll
                for(int a = 0; a < AHEAD; ++a)
                    if(i + a * WAVES < p.pieces) merge_wave(list, next[a]);
            }
            join_lists(list, p.pieces < WAVES ? p.pieces : WAVES, lists);
        }
        if(threadIdx.x < kWaveSize) write_logprobs<T>(p, row, r, list);
        __syncthreads();
    }
}

// ---- gradient of the log probabilities and the entropy ----------------------------------------------------------------------------
// Logits read again, gradient written: 2048 x 65536 bfloat16 108 us (5.0 TB/s).  Nothing of a row meets here, so pieces serve all sizes.
struct LogprobsGradArgs
{
    const void*  z;
    int64_t      rows, ld;
    int          cols;
    float        scale;
    int          pieces, piece;
    bool         streamed;          // stores of the gradient
    const void*  tokens;
    int          wide;
    float        k2;                // see set_scale
    const float *stats, *entropy, *dlogp, *dentropy;      // entropy and dentropy both or neither; dlogp or nullptr
    void*        dz;
    int          ddt;
};

// Walks over a span, 32 bytes of a lane in flight: body(column, values of a vector), edge(column, value).
template <typename T, int WG, bool ONCE, typename F, typename G> __device__ __forceinline__ void walk(const RowSpan<T, ONCE>& z, F&& body, G&& edge)
{
    constexpr int U = 2, N = RowType<T>::N;
    int           i = threadIdx.x;
    row_v4u32     next[U];
    auto          fetch = [&](int from) {
#pragma unroll
        for(int u = 0; u < U; ++u)
            if(from + u * WG < z.vectors) next[u] = z.load(from + u * WG);
    };
    fetch(i);
    const int e = z.edge(threadIdx.x);
    if(e >= 0) edge(e, row_element(z.row + e));
    for(; i < z.vectors; i += U * WG)
    {
        float v[U][N];
#pragma unroll
        for(int u = 0; u < U; ++u) row_decode<T>(next[u], v[u]);
        fetch(i + U * WG);
#pragma unroll
        for(int u = 0; u < U; ++u)
            if(i + u * WG < z.vectors) body(z.column(i + u * WG), v[u]);
    }
}
// The result of f for every element of a span, to a buffer of type dtype whose row begins at `at`.
template <typename T, int WG, bool STREAMED, bool ONCE, typename F> __device__ __forceinline__ void map_span(const RowSpan<T, ONCE>& z, void* out, int dtype, int64_t at, F&& f)
{
    constexpr int N = RowType<T>::N;
    walk<T, WG>(
        z,
        [&](int c, float(&v)[N]) {
            float o[N];
#pragma unroll
            for(int e = 0; e < N; ++e) o[e] = f(c + e, v[e]);
            vector_store<T, STREAMED>(out, dtype, at + c, o);
        },
        [&](int c, float v) { element_store(out, dtype, at + c, f(c, v)); });
}
template <typename T, int WG, bool STREAMED, bool ONCE> __device__ __forceinline__ void zero_span(const RowSpan<T, ONCE>& z, void* out, int dtype, int64_t at)
{
    const float o[RowType<T>::N] = {};
    for(int i = threadIdx.x; i < z.vectors; i += WG) vector_store<T, STREAMED>(out, dtype, at + z.column(i), o);
    const int e = z.edge(threadIdx.x);
    if(e >= 0) element_store(out, dtype, at + e, 0.0f);
}

template <typename T, bool ENTROPY, bool STREAMED> __global__ __launch_bounds__(kRowThreads) void logprobs_grad_kernel(const LogprobsGradArgs p)
{
    const float   k2    = p.k2;
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
        const int64_t    at = row * p.cols;
        const RowSpan<T, true> z(static_cast<const T*>(p.z) + row * p.ld, begin, end);
        if(ln_s == -INFINITY || (g == 0.0f && h == 0.0f))
        {
            zero_span<T, kRowThreads, STREAMED>(z, p.dz, p.ddt, at);
            continue;
        }
        const int   token = given < p.cols ? static_cast<int>(given) : -1;
        const float l2 = ln_s * kLog2e;
        map_span<T, kRowThreads, STREAMED>(z, p.dz, p.ddt, at, [&](int c, float v) {
            const float d = (v - m) * k2 - l2, q = exp2_fast(d);      // log2 p and p
            float       o = -(g * q);
            if constexpr(ENTROPY) o = fmaf(-(h * q), fmaf(fmaxf(d, kFar), kLn2, entropy), o);
            return c == token ? o + g : o;
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
    bool         streamed;          // stores of the gradient
    float        reach;             // see set_scale
    const void*  teacher;
    int          tdt;
    float        k2;
    const void*  index;
    int          wide, k;
    const float* weight;      // or nullptr: 1
    float*       loss;
    void*        dz;          // or nullptr
    int          ddt;
    float4*      part;
};

// The teacher's entries of a row, prepared by the first wavefront: in LDS, so that they take no registers beside a row's.
struct EntriesShared
{
    int   column[kTeacherEntries];      // -1: none
    float q[kTeacherEntries], log_q[kTeacherEntries], z[kTeacherEntries];
    int   any, bad;                     // some entry has weight; a column beyond the vocabulary, or a NaN of the teacher's
};
// The columns and the teacher's logits (in log_q) ...
__device__ __forceinline__ void entries_fetch(const DistillArgs& p, int64_t row, EntriesShared& sh)
{
    bool bad = false;
#pragma unroll 1
    for(int i = threadIdx.x; i < p.k; i += kWaveSize)
    {
        const int64_t e = row * p.k + i, c = index_at(p.index, p.wide, e);
        const float   t = p.tdt == kF32 ? row_element(static_cast<const float*>(p.teacher) + e)
                          : p.tdt == kF16 ? row_element(static_cast<const _Float16*>(p.teacher) + e)
                                          : row_element(static_cast<const __bf16*>(p.teacher) + e);
        const bool    in = c >= 0 && c < p.cols;
        bad |= c >= p.cols || (in && t != t);
        sh.column[i] = in ? static_cast<int>(c) : -1;
        sh.log_q[i]  = in ? t : -INFINITY;
    }
    const uint64_t spoilt = __ballot(bad);
    if(threadIdx.x == 0) sh.bad = spoilt != 0;
}
// ... then, behind the requests for the row itself, the student's logits and the teacher's probabilities.  (A lane reads what it wrote.)
template <typename T> __device__ __forceinline__ void entries_prepare(const DistillArgs& p, const T* row, EntriesShared& sh)
{
    float top = -INFINITY, total = 0.0f;
#pragma unroll 1
    for(int i = threadIdx.x; i < p.k; i += kWaveSize)
    {
        const int c = sh.column[i];
        sh.z[i] = c >= 0 ? row_element(row + c) : 0.0f;
        top     = fmaxf(top, sh.log_q[i]);
    }
    top = wave64_max(top);
    const bool any = top > -INFINITY;
#pragma unroll 1
    for(int i = threadIdx.x; i < p.k; i += kWaveSize)
    {
        const float q = any ? exp2_fast((sh.log_q[i] - top) * p.k2) : 0.0f;
        sh.q[i] = q;
        total += q;
    }
    total = wave64_sum(total);
    const float log_total = logf(total);
#pragma unroll 1
    for(int i = threadIdx.x; i < p.k; i += kWaveSize)
    {
        sh.q[i]     = any ? sh.q[i] / total : 0.0f;
        sh.log_q[i] = (sh.log_q[i] - top) * p.scale - log_total;
    }
    if(threadIdx.x == 0) sh.any = any;
}
// By the first wavefront: sum q (log q - log p), the logits' part by itself: a mask of the lowest value times the scale need not be a
// finite logarithm.
__device__ __forceinline__ float entries_loss(const DistillArgs& p, const Moments& r, float ln_s, const EntriesShared& sh)
{
    float sum = 0.0f;
    for(int i = threadIdx.x; i < p.k; i += kWaveSize)
    {
        const float q = sh.q[i];
        if(q != 0.0f) sum += r.s == 0.0f ? INFINITY : q * (sh.log_q[i] + ln_s) - (q * p.scale) * (sh.z[i] - r.m);
    }
    sum = wave64_sum(sum);
    return sh.bad ? NAN : sum;
}
// By the first wavefront, over the probabilities of [begin, end), which are written: the entries' columns less the teacher's.  mass(z) is
// weight scale p.
template <typename F>
__device__ __forceinline__ void entries_subtract(const DistillArgs& p, int64_t at, int begin, int end, float g, const EntriesShared& sh, F&& mass)
{
    for(int i = threadIdx.x; i < p.k; i += kWaveSize)
    {
        const int column = sh.column[i];
        if(column < begin || column >= end) continue;
        float of = 0.0f;      // of all entries of this column
        for(int j = 0; j < p.k; ++j) of += sh.column[j] == column ? sh.q[j] : 0.0f;
        const float v = mass(sh.z[i]) - g * of;
        element_store(p.dz, p.ddt, at + column, v);
    }
}

// weight scale of a row's gradient; 0 where the whole row's is 0 whatever its logits hold
__device__ __forceinline__ float row_factor(const DistillArgs& p, int64_t row, const Moments& r, const EntriesShared& sh)
{
    const float weight = p.weight ? p.weight[row] : 1.0f;
    if(weight == 0.0f || r.s == 0.0f || !(sh.any || sh.bad)) return 0.0f;
    return sh.bad ? NAN : weight * p.scale;
}

__device__ __forceinline__ float log_sum(const Moments& r) { return r.s == 0.0f ? -INFINITY : logf(r.s); }

// The gradient of a span from logits that are read again.
template <typename T, int WG, bool STREAMED, bool ONCE>
__device__ __forceinline__ void span_gradient(const DistillArgs& p, int64_t row, const RowSpan<T, ONCE>& z, const Moments& r, const EntriesShared& sh)
{
    const int64_t at = row * p.cols;
    const float   g  = row_factor(p, row, r, sh);
    if(g == 0.0f)
    {
        zero_span<T, WG, STREAMED>(z, p.dz, p.ddt, at);
        return;
    }
    const float k2 = p.k2, gs = g / r.s;
    auto        mass = [&](float v) { return gs * exp2_fast((v - r.m) * k2); };
    map_span<T, WG, STREAMED>(z, p.dz, p.ddt, at, [&](int, float v) { return mass(v); });
    __syncthreads();      // (behind the probabilities)
    if(threadIdx.x < kWaveSize) entries_subtract(p, at, z.begin, z.end, g, sh, mass);
}

// A row a workgroup, its logits in registers between the sums and the gradient: NV vectors of a thread, all under way at once.  What a
// longer row has beyond them is read twice, the second time out of a cache.
//   A step over 4096 x 65536 bfloat16 logits: 205 us, 5.2 TB/s of logits read once and gradient written once (under the profiler 217 to 223
//   on average, 208 the shortest); with all of a row read twice 272 (512 threads) and 309 (256), both before loads and stores were streamed and
//   this form took 230.
// (Four wavefronts of a SIMD leave 128 registers.  The scheduling barriers keep the phases from being unrolled into more values than
// that; the words are taken apart again in each phase, as fp32 values they would take twice the registers.)
template <typename T, int WG, int NV, bool REST, bool STREAMED> __global__ __launch_bounds__(WG, 4) void distill_held_kernel(const DistillArgs p)
{
    constexpr int            N = RowType<T>::N, WAVES = WG / kWaveSize;
    __shared__ EntriesShared sh;
    __shared__ float         largest[WAVES], sums[WAVES];
    __shared__ float4        slots[WAVES];
    const int                tid = threadIdx.x;
    const bool               first = tid < kWaveSize;
    float                    k2 = p.k2;
    // (In a vector register.  The six that binary16 saves otherwise let a third workgroup onto a unit: a step over 4096 x 32768 with one
    // entry 100 -> 105 us, with 64 of them 133 -> 129.)
    asm volatile("" : "+v"(k2));
    for(int64_t row = blockIdx.x; row < p.rows; row += gridDim.x)
    {
        const RowSpan<T, true> z(static_cast<const T*>(p.z) + row * p.ld, 0, p.cols);
        if(first) entries_fetch(p, row, sh);
        row_v4u32 w[NV];
        int       t = tid;
        asm volatile("" : "+v"(t));      // (offsets that hang on it are not kept from row to row)
#pragma unroll
        for(int u = 0; u < NV; ++u)
        {
            constexpr uint32_t absent = RowType<T>::kMinusInf;
            w[u] = row_v4u32{absent, absent, absent, absent};
            if(t < z.vectors - u * WG) w[u] = z.load(u * WG + t);
        }
        const int   edge    = z.edge(tid);
        const float at_edge = edge >= 0 ? row_element(z.row + edge) : -INFINITY;
        if(first) entries_prepare(p, z.row, sh);
        RowSpan<T, false> rest;      // (read again)
        LaneBest          none;
        Moments           r{-FLT_MAX, 0.0f, 0.0f};
        if constexpr(REST)
        {
            rest = z.template from<false>(WG * NV);
            r    = row_pass<T, WG, 2, false, false, false>(rest, k2, p.reach, nullptr, none);
        }
        const float rest_m = r.m;
        r.m = fmaxf(r.m, at_edge);
#pragma unroll
        for(int u = 0; u < NV; ++u)
        {
            float v[N];
            row_decode<T>(w[u], v);
#pragma unroll
            for(int i = 0; i < N; ++i) r.m = fmaxf(r.m, v[i]);
            __builtin_amdgcn_sched_barrier(0);
        }
        r.m = wave64_max(r.m);
        if(tid % kWaveSize == 0) largest[tid / kWaveSize] = r.m;
        __syncthreads();
#pragma unroll
        for(int i = 0; i < WAVES; ++i) r.m = fmaxf(r.m, largest[i]);
        // as in row_pass, one operation where the maximum allows it; the product's rounding is common to the sum and the probabilities,
        // and is taken out of the sum that the loss has
        const bool  near = fabsf(r.m) < p.reach;
        const float mk   = r.m * k2;
        auto        again = [&]() {
#pragma unroll
            for(int u = 0; u < NV; ++u) asm volatile("" : "+v"(w[u]));
            asm volatile("" : "+v"(t));
        };
        Moments exact;
        if(near)
        {
            if constexpr(REST) r.s *= exp2_fast(rest_m * k2 - mk);
            r.s += exp2_fast(fmaf(at_edge, k2, -mk));
            again();
#pragma unroll
            for(int u = 0; u < NV; ++u)
            {
                float v[N];
                row_decode<T>(w[u], v);
#pragma unroll
                for(int i = 0; i < N; ++i) r.s += exp2_fast(fmaf(v[i], k2, -mk));
                __builtin_amdgcn_sched_barrier(0);
            }
            r.s = wave64_sum(r.s);
            if(tid % kWaveSize == 0) sums[tid / kWaveSize] = r.s;
            __syncthreads();
            r.s = 0.0f;
#pragma unroll
            for(int i = 0; i < WAVES; ++i) r.s += sums[i];
            exact = r;
            exact.s *= exp2_fast(-fmaf(r.m, k2, -mk));
        }
        else exact = r = join_lanes<WG, true>(row_pass<T, WG, 1, false, false, true>(z, k2, p.reach, nullptr, none), k2, slots);
        if(first)
        {
            const float loss = entries_loss(p, exact, log_sum(exact), sh);
            if(tid == 0) p.loss[row] = loss;
        }
        const float g = row_factor(p, row, exact, sh);
        if(near && g != 0.0f && p.ddt == RowType<T>::kCode)
        {
            T* const    out  = static_cast<T*>(p.dz) + row * p.cols;
            const float gs   = g / r.s;
            auto        mass = [&](float v) { return gs * exp2_fast(fmaf(v, k2, -mk)); };
            again();
#pragma unroll
            for(int u = 0; u < NV; ++u)
            {
                float v[N];
                row_decode<T>(w[u], v);
#pragma unroll
                for(int i = 0; i < N; ++i) v[i] = mass(v[i]);
                if(t < z.vectors - u * WG)
                    row_store<STREAMED>(reinterpret_cast<T*>(reinterpret_cast<uint8_t*>(out) + static_cast<uint32_t>(z.column(u * WG + t)) * static_cast<uint32_t>(sizeof(T))),
                                        RowType<T>::pack(v));
                __builtin_amdgcn_sched_barrier(0);
            }
            if(edge >= 0) out[edge] = static_cast<T>(mass(at_edge));
            if constexpr(REST) map_span<T, WG, STREAMED>(z.template from<true>(WG * NV), p.dz, p.ddt, row * p.cols, [&](int, float v) { return mass(v); });
            __syncthreads();      // (behind the probabilities)
            if(first) entries_subtract(p, row * p.cols, 0, p.cols, g, sh, mass);
        }
        else span_gradient<T, WG, STREAMED>(p, row, z, exact, sh);      // (rows of zeros or of extreme logits, other types)
        __syncthreads();
    }
}

// The loss alone, a row a workgroup: 4096 x 32768 binary16 48 us (5.6 TB/s), 16 x 32768 5.3 a pass, launch included.
template <typename T> __global__ __launch_bounds__(kRowThreads) void distill_loss_kernel(const DistillArgs p)
{
    __shared__ EntriesShared sh;
    __shared__ float4        slots[kRowThreads / kWaveSize];
    const float              k2 = p.k2;
    for(int64_t row = blockIdx.x; row < p.rows; row += gridDim.x)
    {
        const RowSpan<T, true> z(static_cast<const T*>(p.z) + row * p.ld, 0, p.cols);
        if(threadIdx.x < kWaveSize)
        {
            entries_fetch(p, row, sh);
            entries_prepare(p, z.row, sh);
        }
        LaneBest      none;
        const Moments r = span_moments<T, kRowThreads, kUnroll, false, false>(z, k2, p.reach, nullptr, none, slots);
        if(threadIdx.x < kWaveSize)
        {
            const float loss = entries_loss(p, r, log_sum(r), sh);
            if(threadIdx.x == 0) p.loss[row] = loss;
        }
        __syncthreads();
    }
}

// Few long rows, which one compute unit each would take too long to read: the moments of the pieces (a step over 1 x 131072 bfloat16 11.4 us,
// by one workgroup 25) ...
template <typename T> __global__ __launch_bounds__(kRowThreads) void distill_pieces_kernel(const DistillArgs p)
{
    __shared__ float4 slots[kRowThreads / kWaveSize];
    const int64_t     items = p.rows * p.pieces;
    for(int64_t item = blockIdx.x; item < items; item += gridDim.x)
    {
        const int64_t    row   = item / p.pieces;
        const int        begin = static_cast<int>(item - row * p.pieces) * p.piece;
        const RowSpan<T, false> z(static_cast<const T*>(p.z) + row * p.ld, begin, p.cols - begin < p.piece ? p.cols : begin + p.piece);
        LaneBest         none;
        const Moments    r = span_moments<T, kRowThreads, kUnroll, false, false>(z, p.k2, p.reach, nullptr, none, slots);
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
        const int64_t row = p.dz ? item / p.pieces : item;
        const int     i   = p.dz ? static_cast<int>(item - row * p.pieces) : 0;
        const T*      z   = static_cast<const T*>(p.z) + row * p.ld;
        if(threadIdx.x < kWaveSize)
        {
            entries_fetch(p, row, sh);
            entries_prepare(p, z, sh);
        }
        const Moments r = join_pieces<kRowThreads>(p.part + row * p.pieces, p.pieces, p.k2, slots);
        if(p.loss && i == 0 && threadIdx.x < kWaveSize)
        {
            const float loss = entries_loss(p, r, log_sum(r), sh);
            if(threadIdx.x == 0) p.loss[row] = loss;
        }
        if(p.dz)
        {
            const int begin = i * p.piece;
            span_gradient<T, kRowThreads, false>(p, row, RowSpan<T, true>(z, begin, p.cols - begin < p.piece ? p.cols : begin + p.piece), r, sh);
        }
        __syncthreads();
    }
}

// ---- launches -------------------------------------------------------------------------------------------------------------------
constexpr int64_t kFill = 1024;           // workgroups that fill the device: four on every compute unit
constexpr int64_t kMostGroups = 1 << 22;  // of a launch; larger problems loop

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
// k2: scale log2(e), the largest number where that has none (0 of a difference must stay 0).  reach: |z| below which the fast form of a pass
// holds.  (Made on the host: beside its kernels' registers a division would cost two more.)
float exponent_scale(float scale) { return std::min(scale * kLog2e, FLT_MAX); }
template <typename A> void set_scale(A& a, float scale)
{
    a.scale = scale;
    a.k2    = exponent_scale(scale);
    a.reach = std::min(-kFar, kNearProduct / a.k2);
}
int vector_elements(int dt) { return dt == kF32 ? 4 : 8; }

struct Split { int pieces, piece; };
// Pieces of a row: enough to fill the device, multiples of `least` elements, and of `most` elements at most.
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
// A row a workgroup, or in pieces?  A compute unit takes in `unit` bytes of a row in a microsecond, however many threads ask for them, all of
// them together `device`; pieces cost a second launch and what it reads, `launch` microseconds.
struct RowRates { double unit, device, launch; };
//   log probabilities, 20 alternatives (the rates serve for none and for 64 as well, where they were not measured), us, a row a workgroup ->
//   in pieces: 1 x 131072 bfloat16 17.5 -> 11.9, 64 x 131072 18.3 -> 16.9, 128 x 131072 18.9 -> 19.2, 1 x 32768 9.4 -> 11.1,
//   333 x 50021 fp32 22.3 -> 28.7
constexpr RowRates kLogprobsRates = {27.0e3, 3.3e6, 3.5};
//   loss alone: 1 x 131072 bfloat16 10.4 -> 8.3, 64 x 131072 12.1 -> 9.8, 1 x 32768 5.8 -> 8.3
constexpr RowRates kLossRates = {45.0e3, 1.0e7, 3.0};
//   loss and gradient: 1 x 131072 bfloat16 25.5 -> 11.4, 64 x 131072 27.5 -> 19.3, 200 x 131072 37.4 -> 41.8, 1 x 32768 11.3 -> 11.4
constexpr RowRates kGradientRates = {14.0e3, 2.0e6, 5.0};
bool in_pieces(const RowRates& t, int zdt, int64_t rows, int64_t cols)
{
    const double bytes = static_cast<double>(cols) * (zdt == kF32 ? 4 : 2);
    return bytes / t.unit > t.launch + static_cast<double>(rows) * bytes / t.device;
}
// A top search keeps 6 bytes of LDS for every chunk of a thread: of 64 KB, beside its lists.
constexpr int64_t kMaxChunks = 24;
int64_t span_elements(int zdt) { return static_cast<int64_t>(kRowThreads) * vector_elements(zdt) * kUnroll; }
int64_t piece_most(int zdt, int top) { return top > 0 ? span_elements(zdt) * kMaxChunks : kLogitsMaxCols; }
Split whole_row(int64_t cols) { return Split{1, static_cast<int>(cols)}; }
Split logprobs_split(int zdt, int64_t rows, int64_t cols, int top)
{
    if(cols <= piece_most(zdt, top) && !in_pieces(kLogprobsRates, zdt, rows, cols)) return whole_row(cols);
    return split_rows(rows, cols, span_elements(zdt), piece_most(zdt, top));
}
// what `rows` rows or fewer are cut into at most
int64_t most_items(int zdt, int64_t rows, int64_t cols, int top)
{
    const int64_t fill = kFill + rows, cap = rows * div_up(cols, piece_most(zdt, top));
    return fill > cap ? fill : cap;
}
// Gradients that no cache (256 MB in front of the memory) holds until their reader comes are streamed.  us, ordinary -> streamed stores, a
// distillation step in binary16 with the INT8 conversion of the gradient behind it (alone): 4096 x 32768 235 -> 250 (132 -> 122),
// 6000 x 32768 376 -> 362 (186 -> 173), 4096 x 65536 479 -> 461 (234 -> 206).
bool streamed(int dt, int64_t rows, int64_t cols) { return rows * cols * (dt == kF32 ? 4 : 2) > (int64_t(320) << 20); }
// f(std::true_type or std::false_type)
template <typename F> void choose(bool v, F&& f)
{
    if(v) f(std::true_type{});
    else  f(std::false_type{});
}
dim3 groups(int64_t items) { return dim3(static_cast<unsigned>(items < kMostGroups ? items : kMostGroups)); }

template <typename T> hipError_t logprobs_type(const LogitsArgs& a, hipStream_t st)
{
    const dim3   grid = groups(a.rows * a.pieces), block(kRowThreads);
    const size_t lds  = a.top > 0 ? top_lds_bytes(static_cast<int>(div_up(a.piece, chunk_span<T>(kRowThreads)))) : 0;
    choose(a.entropy != nullptr, [&](auto entropy) {
        choose(a.top > 0, [&](auto top) {
            logprobs_kernel<T, decltype(entropy)::value, decltype(top)::value><<<grid, block, lds, st>>>(a);
        });
    });
    const hipError_t e = hipGetLastError();
    if(e != hipSuccess || a.pieces == 1) return e;
    logprobs_join_kernel<T><<<groups(a.rows), block, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T> hipError_t logprobs_grad_type(const LogprobsGradArgs& a, hipStream_t st)
{
    choose(a.dentropy != nullptr, [&](auto entropy) {
        choose(a.streamed, [&](auto through) {
            logprobs_grad_kernel<T, decltype(entropy)::value, decltype(through)::value><<<groups(a.rows * a.pieces), dim3(kRowThreads), 0, st>>>(a);
        });
    });
    return hipGetLastError();
}

template <typename T, int WG, int NV, bool REST = false> hipError_t distill_held(const DistillArgs& a, hipStream_t st)
{
    choose(a.streamed, [&](auto through) { distill_held_kernel<T, WG, NV, REST, decltype(through)::value><<<groups(a.rows), dim3(WG), 0, st>>>(a); });
    return hipGetLastError();
}
template <typename T> hipError_t distill_type(const DistillArgs& a, hipStream_t st)
{
    if(a.pieces == 1 && !a.dz)
    {
        distill_loss_kernel<T><<<groups(a.rows), dim3(kRowThreads), 0, st>>>(a);
        return hipGetLastError();
    }
    if(a.pieces == 1)
    {   // (the fewest registers that hold a row: 4096 x 32768 bfloat16 on 512 threads of 8 vectors 132 us, 256 of 16 141; 8192 x 8000 on 256
        // of 4 76)
        const int64_t vectors = a.cols / RowType<T>::N;
        if(vectors <= 256 * 4) return distill_held<T, 256, 4>(a, st);
        if(vectors <= 512 * 8) return distill_held<T, 512, 8>(a, st);
        return vectors <= 512 * 16 ? distill_held<T, 512, 16>(a, st) : distill_held<T, 512, 16, true>(a, st);
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
    a.z = z; a.rows = rows; a.ld = ld; a.cols = static_cast<int>(cols); set_scale(a, scale);
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
    a.z = z; a.rows = rows; a.ld = ld; a.cols = static_cast<int>(cols); a.scale = scale; a.k2 = exponent_scale(scale);
    a.pieces = s.pieces; a.piece = s.piece; a.streamed = streamed(ddt, rows, cols);
    a.tokens = tokens; a.wide = wide; a.stats = stats; a.entropy = entropy; a.dlogp = dlogp; a.dentropy = dentropy;
    a.dz = dz; a.ddt = ddt;
    return by_type(zdt, [&](auto tag) { return logprobs_grad_type<decltype(tag)>(a, st); });
}

size_t distill_topk_workspace_bytes(int zdt, int64_t rows, int64_t cols) { return static_cast<size_t>(most_items(zdt, rows, cols, 0)) * sizeof(float4); }

hipError_t launch_distill_topk(const void* z, int zdt, int64_t rows, int64_t cols, int64_t ld, float scale, const void* teacher, int tdt,
                               const void* index, bool wide, int k, const float* weight, float* loss, void* dz, int ddt, void* workspace,
                               hipStream_t st)
{
    const Split s = in_pieces(dz ? kGradientRates : kLossRates, zdt, rows, cols) ? split_rows(rows, cols, span_elements(zdt) / kUnroll, kLogitsMaxCols)
                                                                                 : whole_row(cols);
    DistillArgs a{};
    a.z = z; a.rows = rows; a.ld = ld; a.cols = static_cast<int>(cols); set_scale(a, scale);
    a.pieces = s.pieces; a.piece = s.piece; a.streamed = streamed(ddt, rows, cols);
    a.teacher = teacher; a.tdt = tdt; a.index = index; a.wide = wide; a.k = k; a.weight = weight; a.loss = loss;
    a.dz = dz; a.ddt = ddt;
    a.part = static_cast<float4*>(workspace);
    return by_type(zdt, [&](auto tag) { return distill_type<decltype(tag)>(a, st); });
}

}  // namespace qsync
