// Layer norm over the columns of a matrix, and its gradients.
//
//   mean = sum_c x / C      var = sum_c (x - mean)^2 / C      rstd = (var + eps)^(-1/2)      xh = (x - mean) rstd
//   y  = xh gamma + beta
//   dx = rstd (g - sum_c g / C - xh sum_c (g xh) / C),  g = dy gamma      dgamma = sum_r dy xh      dbeta = sum_r dy
//
// Both directions are bound by memory: x read and y written once, x and dy read and dx written once.  A row is held in the registers of
// its lanes (eight consecutive elements a unit, up to four units a lane) between its statistics and its result; workgroups walk over
// rows with the next row's loads under way, so that gamma and beta are fetched once per workgroup, not per row.  The variance is that
// of the differences to the mean, in fp32: sums of squares would cancel on rows whose mean is far from zero.  The parameters'
// gradients are sums over the rows: a workgroup keeps its rows' in registers and leaves one partial row each, which a second launch
// folds in a fixed order, so that results do not depend on scheduling.
#include "device_utils.h"
#include "row_ops.h"

namespace qsync {

namespace {

struct NormArgs
{
    const void*   x;
    const void*   dy;           // backward
    int64_t       rows, cols, ldx, lddy;
    const float*  gamma;        // or nullptr: 1
    const float*  beta;         // or nullptr: 0
    float         eps;
    void*         y;            // forward: y, backward: dx (or nullptr)
    int           ydt;
    float*        mean;         // forward: out or nullptr, backward: in
    float*        rstd;
    unsigned int* amax_bits;    // forward: or nullptr
    float*        partial;      // backward: [workgroups][2][cols] sums of dy xh and of dy, or nullptr
};

// The eight parameters of a unit, or `absent`.
__device__ __forceinline__ void load_params(const float* p, int64_t c, int64_t cols, float absent, float (&v)[8])
{
    if(!p)
    {
#pragma unroll
        for(int e = 0; e < 8; ++e) v[e] = absent;
        return;
    }
    Row8<float> r;
    r.load(p + c, cols - c);
    r.decode(v);
}

// Statistics of one row from per-wavefront sums: every wavefront hands in the sum and the squared differences to its own mean of the
// `n` elements that it holds; the parts are joined in order.  `slots`: a float4 per wavefront, two sets used in turn so that one
// barrier a row suffices.
template <int WAVES>
__device__ __forceinline__ void join_moments(float sum, float m2, float n, float cols, float4* slots, float& mean, float& var)
{
    if constexpr(WAVES == 1)
    {
        mean = sum / cols;
        var  = m2 / cols;
        return;
    }
    if(threadIdx.x % kWaveSize == 0) slots[threadIdx.x / kWaveSize] = make_float4(sum, m2, n, n > 0.0f ? sum / n : 0.0f);
    __syncthreads();
    float total = 0.0f;
#pragma unroll
    for(int w = 0; w < WAVES; ++w) total += slots[w].x;
    mean     = total / cols;
    float sq = 0.0f;
#pragma unroll
    for(int w = 0; w < WAVES; ++w)
    {
        const float4 s = slots[w];
        const float  d = s.w - mean;
        sq += s.y + s.z * d * d;
    }
    var = sq / cols;
}

template <int TPR> __device__ __forceinline__ float group_sum(float v) { return TPR == 16 ? row16_sum(v) : wave64_sum(v); }

// Largest |y| as stored, once per workgroup at most (`run`: this lane's).
__device__ __forceinline__ void publish_largest(float run, unsigned int* word, float* lds)
{
    run = block_reduce_max(run, lds);
    if(threadIdx.x != 0) return;
    const unsigned int bits = __float_as_uint(run);
    if(bits > __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(word, bits);
}

// TPR lanes a row, NU units of eight elements a lane; WG / TPR rows of a workgroup at a time.
template <typename T, int TPR, int NU, int WG>
__global__ __launch_bounds__(WG) void norm_forward_kernel(const NormArgs p)
{
    constexpr int WAVES = TPR > kWaveSize ? TPR / kWaveSize : 1, ROWS = WG / TPR;
    static_assert(TPR <= kWaveSize || TPR == WG, "rows of several wavefronts take the workgroup");
    __shared__ float4 slots[2][WG / kWaveSize];
    const int     lane = threadIdx.x % TPR;
    const int64_t step = static_cast<int64_t>(gridDim.x) * ROWS;
    const float   cols = static_cast<float>(p.cols);
    const T*      x    = static_cast<const T*>(p.x);

    float gamma[NU][8], beta[NU][8], held = 0.0f;
#pragma unroll
    for(int u = 0; u < NU; ++u)
    {
        const int64_t c = (static_cast<int64_t>(u) * TPR + lane) * 8;
        load_params(p.gamma, c, p.cols, 1.0f, gamma[u]);
        load_params(p.beta, c, p.cols, 0.0f, beta[u]);
        const int64_t left = p.cols - c;
        held += left <= 0 ? 0.0f : left >= 8 ? 8.0f : static_cast<float>(left);
    }
    const float n = group_sum<TPR>(held);      // elements of this wavefront (of these 16 lanes)

    int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
    Row8<T> next[NU];
    auto    fetch = [&](int64_t r) {
#pragma unroll
        for(int u = 0; u < NU; ++u)
        {
            const int64_t c = (static_cast<int64_t>(u) * TPR + lane) * 8;
            next[u].load(x + r * p.ldx + c, p.cols - c);
        }
    };
    if(row < p.rows) fetch(row);
    float run = 0.0f;
    for(int turn = 0; row < p.rows; row += step, turn ^= 1)
    {
        float v[NU][8];
        float sum = 0.0f;
#pragma unroll
        for(int u = 0; u < NU; ++u)
        {
            next[u].decode(v[u]);
#pragma unroll
            for(int e = 0; e < 8; ++e) sum += v[u][e];
        }
        if(row + step < p.rows) fetch(row + step);
        sum             = group_sum<TPR>(sum);
        const float own = n > 0.0f ? sum / n : 0.0f;
        float       m2  = 0.0f;
#pragma unroll
        for(int u = 0; u < NU; ++u)
        {
            const int64_t left = p.cols - (static_cast<int64_t>(u) * TPR + lane) * 8;
#pragma unroll
            for(int e = 0; e < 8; ++e)
            {
                const float d = e < left ? v[u][e] - own : 0.0f;
                m2            = fmaf(d, d, m2);
            }
        }
        m2 = group_sum<TPR>(m2);
        float mean, var;
        join_moments<WAVES>(sum, m2, n, cols, slots[turn], mean, var);
        const float rstd = 1.0f / sqrtf(var + p.eps);
        if(lane == 0)
        {
            if(p.mean) p.mean[row] = mean;
            if(p.rstd) p.rstd[row] = rstd;
        }
#pragma unroll
        for(int u = 0; u < NU; ++u)
        {
            const int64_t c = (static_cast<int64_t>(u) * TPR + lane) * 8;
            if(c >= p.cols) continue;
            float o[8];
#pragma unroll
            for(int e = 0; e < 8; ++e) o[e] = fmaf((v[u][e] - mean) * rstd, gamma[u][e], beta[u][e]);
            const int64_t left = p.cols - c;
            if(!p.amax_bits) row8_store<false>(p.y, p.ydt, row * p.cols + c, o, left);
            else
            {
                row8_store<true>(p.y, p.ydt, row * p.cols + c, o, left);
#pragma unroll
                for(int e = 0; e < 8; ++e) run = e < left ? fmaxf(run, fabsf(o[e])) : run;
            }
        }
    }
    if(p.amax_bits)
    {
        __syncthreads();
        publish_largest(run, p.amax_bits, reinterpret_cast<float*>(slots));
    }
}

// Sums over the workgroup of two values at once, in every lane.
template <int WG> __device__ __forceinline__ float2 block_sum2(float a, float b, float2* slots)
{
    a = wave64_sum(a);
    b = wave64_sum(b);
    if(threadIdx.x % kWaveSize == 0) slots[threadIdx.x / kWaveSize] = make_float2(a, b);
    __syncthreads();
    float2 t = slots[0];
#pragma unroll
    for(int w = 1; w < WG / kWaveSize; ++w) { t.x += slots[w].x; t.y += slots[w].y; }
    return t;
}

// Rows longer than the registers of a workgroup hold: read three times (the second and third time out of a cache).
template <typename T> __global__ __launch_bounds__(1024) void norm_forward_long_kernel(const NormArgs p)
{
    __shared__ float2 slots[3][16];
    const T*          x    = static_cast<const T*>(p.x);
    const float       cols = static_cast<float>(p.cols);
    float             run  = 0.0f;
    for(int64_t row = blockIdx.x; row < p.rows; row += gridDim.x)
    {
        const T* at = x + row * p.ldx;
        Row8<T>  r;
        float    v[8], sum = 0.0f, m2 = 0.0f;
        for(int64_t c = threadIdx.x * 8; c < p.cols; c += 8192)
        {
            r.load(at + c, p.cols - c);
            r.decode(v);
            sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
        const float mean = block_sum2<1024>(sum, 0.0f, slots[0]).x / cols;
        for(int64_t c = threadIdx.x * 8; c < p.cols; c += 8192)
        {
            r.load(at + c, p.cols - c);
            r.decode(v);
#pragma unroll
            for(int e = 0; e < 8; ++e)
            {
                const float d = c + e < p.cols ? v[e] - mean : 0.0f;
                m2            = fmaf(d, d, m2);
            }
        }
        const float var  = block_sum2<1024>(m2, 0.0f, slots[1]).x / cols;
        const float rstd = 1.0f / sqrtf(var + p.eps);
        if(threadIdx.x == 0)
        {
            if(p.mean) p.mean[row] = mean;
            if(p.rstd) p.rstd[row] = rstd;
        }
        for(int64_t c = threadIdx.x * 8; c < p.cols; c += 8192)
        {
            float g[8], b[8];
            r.load(at + c, p.cols - c);
            r.decode(v);
            load_params(p.gamma, c, p.cols, 1.0f, g);
            load_params(p.beta, c, p.cols, 0.0f, b);
#pragma unroll
            for(int e = 0; e < 8; ++e) v[e] = fmaf((v[e] - mean) * rstd, g[e], b[e]);
            row8_store<true>(p.y, p.ydt, row * p.cols + c, v, p.cols - c);
#pragma unroll
            for(int e = 0; e < 8; ++e) run = c + e < p.cols ? fmaxf(run, fabsf(v[e])) : run;
        }
    }
    if(p.amax_bits) publish_largest(run, p.amax_bits, reinterpret_cast<float*>(slots[2]));
}

// TD: dy, T: x.
template <typename TD, typename T, int TPR, int NU, int WG>
__global__ __launch_bounds__(WG) void norm_backward_kernel(const NormArgs p)
{
    constexpr int WAVES = TPR > kWaveSize ? TPR / kWaveSize : 1, ROWS = WG / TPR;
    static_assert(TPR <= kWaveSize || TPR == WG, "rows of several wavefronts take the workgroup");
    __shared__ float2 slots[2][WG / kWaveSize];
    const int     lane = threadIdx.x % TPR;
    const int64_t step = static_cast<int64_t>(gridDim.x) * ROWS;
    const float   cols = static_cast<float>(p.cols);
    const T*      x    = static_cast<const T*>(p.x);
    const TD*     dy   = static_cast<const TD*>(p.dy);

    float gamma[NU][8], sum_g[NU][8], sum_b[NU][8];
#pragma unroll
    for(int u = 0; u < NU; ++u)
    {
        load_params(p.gamma, (static_cast<int64_t>(u) * TPR + lane) * 8, p.cols, 1.0f, gamma[u]);
#pragma unroll
        for(int e = 0; e < 8; ++e) sum_g[u][e] = sum_b[u][e] = 0.0f;
    }
    int64_t  row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
    Row8<T>  next_x[NU];
    Row8<TD> next_dy[NU];
    float    next_mean = 0.0f, next_rstd = 0.0f;
    auto     fetch = [&](int64_t r) {
#pragma unroll
        for(int u = 0; u < NU; ++u)
        {
            const int64_t c = (static_cast<int64_t>(u) * TPR + lane) * 8;
            next_x[u].load(x + r * p.ldx + c, p.cols - c);
            next_dy[u].load(dy + r * p.lddy + c, p.cols - c);
        }
        next_mean = p.mean[r];
        next_rstd = p.rstd[r];
    };
    if(row < p.rows) fetch(row);
    for(int turn = 0; row < p.rows; row += step, turn ^= 1)
    {
        float       xh[NU][8], d[NU][8];
        const float mean = next_mean, rstd = next_rstd;
        float       s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for(int u = 0; u < NU; ++u)
        {
            next_x[u].decode(xh[u]);
            next_dy[u].decode(d[u]);      // (absent elements: 0, whatever their xh)
#pragma unroll
            for(int e = 0; e < 8; ++e)
            {
                xh[u][e] = (xh[u][e] - mean) * rstd;
                sum_g[u][e] = fmaf(d[u][e], xh[u][e], sum_g[u][e]);
                sum_b[u][e] += d[u][e];
                d[u][e] *= gamma[u][e];
                s1 += d[u][e];
                s2 = fmaf(d[u][e], xh[u][e], s2);
            }
        }
        if(row + step < p.rows) fetch(row + step);
        if(!p.y) continue;      // (the same for every lane)
        if constexpr(WAVES == 1)
        {
            s1 = group_sum<TPR>(s1);
            s2 = group_sum<TPR>(s2);
        }
        else
        {
            const float2 t = block_sum2<WG>(s1, s2, slots[turn]);
            s1 = t.x;
            s2 = t.y;
        }
        s1 /= cols;
        s2 /= cols;
#pragma unroll
        for(int u = 0; u < NU; ++u)
        {
            const int64_t c = (static_cast<int64_t>(u) * TPR + lane) * 8;
            if(c >= p.cols) continue;
            float o[8];
#pragma unroll
            for(int e = 0; e < 8; ++e) o[e] = rstd * (d[u][e] - s1 - xh[u][e] * s2);
            row8_store<false>(p.y, p.ydt, row * p.cols + c, o, p.cols - c);
        }
    }
    if(!p.partial) return;
    float* out = p.partial + static_cast<int64_t>(blockIdx.x) * 2 * p.cols;
    if constexpr(ROWS == 1)
    {
#pragma unroll
        for(int u = 0; u < NU; ++u)
        {
            const int64_t c = (static_cast<int64_t>(u) * TPR + lane) * 8;
            if(c >= p.cols) continue;
            row8_store<false>(out, kF32, c, sum_g[u], p.cols - c);
            row8_store<false>(out, kF32, p.cols + c, sum_b[u], p.cols - c);
        }
    }
    else
    {   // the groups' sums, added in order
        constexpr int     SPAN = TPR * NU * 8;
        __shared__ float4 sums[ROWS * SPAN / 4];
        float*            flat = reinterpret_cast<float*>(sums);
        const int         g    = threadIdx.x / TPR;
#pragma unroll
        for(int which = 0; which < 2; ++which)
        {
            if(which) __syncthreads();
#pragma unroll
            for(int u = 0; u < NU; ++u)
            {
                float(&s)[8] = which ? sum_b[u] : sum_g[u];
                float4* at   = sums + (g * SPAN + (u * TPR + lane) * 8) / 4;
                at[0] = make_float4(s[0], s[1], s[2], s[3]);
                at[1] = make_float4(s[4], s[5], s[6], s[7]);
            }
            __syncthreads();
            for(int c = threadIdx.x; c < p.cols; c += WG)
            {
                float t = 0.0f;
#pragma unroll
                for(int k = 0; k < ROWS; ++k) t += flat[k * SPAN + c];
                out[which * p.cols + c] = t;
            }
        }
    }
}

// Long rows: dx of a row by a workgroup, x and dy read twice.
template <typename TD, typename T> __global__ __launch_bounds__(1024) void norm_backward_long_kernel(const NormArgs p)
{
    __shared__ float2 slots[2][16];
    const float       cols = static_cast<float>(p.cols);
    int               turn = 0;
    for(int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1)
    {
        const T*    x    = static_cast<const T*>(p.x) + row * p.ldx;
        const TD*   dy   = static_cast<const TD*>(p.dy) + row * p.lddy;
        const float mean = p.mean[row], rstd = p.rstd[row];
        Row8<T>     rx;
        Row8<TD>    rd;
        float       xh[8], d[8], g[8], s1 = 0.0f, s2 = 0.0f;
        auto        fetch = [&](int64_t c) {
            rx.load(x + c, p.cols - c);
            rd.load(dy + c, p.cols - c);
            load_params(p.gamma, c, p.cols, 1.0f, g);
            rx.decode(xh);
            rd.decode(d);
#pragma unroll
            for(int e = 0; e < 8; ++e)
            {
                xh[e] = (xh[e] - mean) * rstd;
                d[e] *= g[e];
            }
        };
        for(int64_t c = threadIdx.x * 8; c < p.cols; c += 8192)
        {
            fetch(c);
#pragma unroll
            for(int e = 0; e < 8; ++e)
            {
                s1 += d[e];
                s2 = fmaf(d[e], xh[e], s2);
            }
        }
        const float2 t = block_sum2<1024>(s1, s2, slots[turn]);
        s1 = t.x / cols;
        s2 = t.y / cols;
        for(int64_t c = threadIdx.x * 8; c < p.cols; c += 8192)
        {
            fetch(c);
#pragma unroll
            for(int e = 0; e < 8; ++e) d[e] = rstd * (d[e] - s1 - xh[e] * s2);
            row8_store<false>(p.y, p.ydt, row * p.cols + c, d, p.cols - c);
        }
    }
}
// ... and the parameters' partial sums, a strip of 2048 columns over every gridDim.y-th row a workgroup
template <typename TD, typename T> __global__ __launch_bounds__(256) void norm_params_kernel(const NormArgs p)
{
    const int64_t c = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
    if(c >= p.cols) return;
    float sum_g[8] = {}, sum_b[8] = {};
    for(int64_t row = blockIdx.y; row < p.rows; row += gridDim.y)
    {
        Row8<T>  rx;
        Row8<TD> rd;
        rx.load(static_cast<const T*>(p.x) + row * p.ldx + c, p.cols - c);
        rd.load(static_cast<const TD*>(p.dy) + row * p.lddy + c, p.cols - c);
        const float mean = p.mean[row], rstd = p.rstd[row];
        float       xh[8], d[8];
        rx.decode(xh);
        rd.decode(d);
#pragma unroll
        for(int e = 0; e < 8; ++e)
        {
            sum_g[e] = fmaf(d[e], (xh[e] - mean) * rstd, sum_g[e]);
            sum_b[e] += d[e];
        }
    }
    float* out = p.partial + static_cast<int64_t>(blockIdx.y) * 2 * p.cols;
    row8_store<false>(out, kF32, c, sum_g, p.cols - c);
    row8_store<false>(out, kF32, p.cols + c, sum_b, p.cols - c);
}

// dgamma and dbeta from S partial rows [S][2][cols]
__global__ __launch_bounds__(256) void norm_fold_kernel(const float* partial, int S, int64_t cols, float* dgamma, float* dbeta)
{
    __shared__ float lds[256];
    const int        q = threadIdx.x / 16;
    const int64_t    c = static_cast<int64_t>(blockIdx.x) * 16 + threadIdx.x % 16;
    const float      t = fold_column<false>(partial, S, 2 * cols, c, q, lds);
    if(q != 0 || c >= 2 * cols) return;
    if(c < cols) { if(dgamma) dgamma[c] = t; }
    else if(dbeta) dbeta[c - cols] = t;
}

constexpr int64_t kNormMaxCols = 8192;       // columns of a row that is kept in registers by the backward pass
constexpr int64_t kNormGroups  = 1024;       // workgroups of a backward pass: partial rows of the parameters' gradients
constexpr int64_t kNormParamRows = 64;       // ... of rows that are longer

int64_t at_most(int64_t v, int64_t most) { return v < most ? v : most; }

template <typename T, int TPR, int NU, int WG> hipError_t forward_rows(const NormArgs& a, hipStream_t st)
{
    constexpr int rows = WG / TPR;
    norm_forward_kernel<T, TPR, NU, WG><<<dim3(static_cast<unsigned>(at_most((a.rows + rows - 1) / rows, 256 * (2048 / WG)))), dim3(WG), 0, st>>>(a);
    return hipGetLastError();
}
template <typename T> hipError_t forward_type(const NormArgs& a, hipStream_t st)
{
    if(a.cols <= 128) return forward_rows<T, 16, 1, 256>(a, st);
    if(a.cols <= 512) return forward_rows<T, 64, 1, 256>(a, st);
    if(a.cols <= 1024) return forward_rows<T, 64, 2, 256>(a, st);
    if(a.cols <= 2048) return forward_rows<T, 256, 1, 256>(a, st);
    if(a.cols <= 4096) return forward_rows<T, 256, 2, 256>(a, st);
    if(a.cols <= 8192) return forward_rows<T, 512, 2, 512>(a, st);
    if(a.cols <= 16384) return forward_rows<T, 512, 4, 512>(a, st);
    norm_forward_long_kernel<T><<<dim3(static_cast<unsigned>(at_most(a.rows, 512))), dim3(1024), 0, st>>>(a);
    return hipGetLastError();
}

template <typename TD, typename T, int TPR, int NU, int WG> hipError_t backward_rows(const NormArgs& a, int64_t groups, hipStream_t st)
{
    norm_backward_kernel<TD, T, TPR, NU, WG><<<dim3(static_cast<unsigned>(groups)), dim3(WG), 0, st>>>(a);
    return hipGetLastError();
}
// rows that a workgroup of the backward pass has at a time
int64_t backward_rows_of(int64_t cols) { return cols <= 128 ? 16 : cols <= 1024 ? 4 : 1; }
int64_t backward_groups(int64_t rows, int64_t cols)
{
    if(cols > kNormMaxCols) return at_most(rows, kNormParamRows);
    const int64_t at_once = backward_rows_of(cols);
    return at_most((rows + at_once - 1) / at_once, kNormGroups);
}
template <typename TD, typename T> hipError_t backward_types(const NormArgs& a, hipStream_t st)
{
    const int64_t groups = backward_groups(a.rows, a.cols);
    if(a.cols <= 128) return backward_rows<TD, T, 16, 1, 256>(a, groups, st);
    if(a.cols <= 512) return backward_rows<TD, T, 64, 1, 256>(a, groups, st);
    if(a.cols <= 1024) return backward_rows<TD, T, 64, 2, 256>(a, groups, st);
    if(a.cols <= 2048) return backward_rows<TD, T, 256, 1, 256>(a, groups, st);
    if(a.cols <= 4096) return backward_rows<TD, T, 256, 2, 256>(a, groups, st);
    if(a.cols <= kNormMaxCols) return backward_rows<TD, T, 512, 2, 512>(a, groups, st);
    // (the parameters' sums first: dx may take the place of dy or x)
    if(a.partial)
    {
        norm_params_kernel<TD, T><<<dim3(static_cast<unsigned>((a.cols + 2047) / 2048), static_cast<unsigned>(groups)), dim3(256), 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if(e != hipSuccess) return e;
    }
    if(a.y) norm_backward_long_kernel<TD, T><<<dim3(static_cast<unsigned>(at_most(a.rows, 512))), dim3(1024), 0, st>>>(a);
    return hipGetLastError();
}
template <typename TD> hipError_t backward_type(const NormArgs& a, int xdt, hipStream_t st)
{
    return xdt == kF32 ? backward_types<TD, float>(a, st) : xdt == kF16 ? backward_types<TD, _Float16>(a, st) : backward_types<TD, __bf16>(a, st);
}

}  // namespace

hipError_t launch_layernorm_fwd(const void* x, int xdt, int64_t rows, int64_t cols, int64_t ld, const float* gamma, const float* beta, float eps,
                                void* y, int ydt, float* mean, float* rstd, float* y_amax, hipStream_t st)
{
    NormArgs a{};
    a.x = x; a.rows = rows; a.cols = cols; a.ldx = ld; a.gamma = gamma; a.beta = beta; a.eps = eps;
    a.y = y; a.ydt = ydt; a.mean = mean; a.rstd = rstd;
    a.amax_bits = reinterpret_cast<unsigned int*>(y_amax);
    return xdt == kF32 ? forward_type<float>(a, st) : xdt == kF16 ? forward_type<_Float16>(a, st) : forward_type<__bf16>(a, st);
}

size_t layernorm_bwd_workspace_bytes(int64_t rows, int64_t cols)
{
    return static_cast<size_t>(backward_groups(rows, cols)) * 2 * static_cast<size_t>(cols) * sizeof(float);
}

hipError_t launch_layernorm_bwd(const void* dy, int dydt, int64_t lddy, const void* x, int xdt, int64_t rows, int64_t cols, int64_t ldx,
                                const float* gamma, const float* mean, const float* rstd, void* dx, int dxdt, float* dgamma, float* dbeta,
                                void* workspace, hipStream_t st)
{
    NormArgs a{};
    a.x = x; a.dy = dy; a.rows = rows; a.cols = cols; a.ldx = ldx; a.lddy = lddy; a.gamma = gamma;
    a.y = dx; a.ydt = dxdt;
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
    a.partial = dgamma || dbeta ? static_cast<float*>(workspace) : nullptr;
    const hipError_t e = dydt == kF32 ? backward_type<float>(a, xdt, st) : dydt == kF16 ? backward_type<_Float16>(a, xdt, st) : backward_type<__bf16>(a, xdt, st);
    if(e != hipSuccess || !a.partial) return e;
    norm_fold_kernel<<<dim3(static_cast<unsigned>((2 * cols + 15) / 16)), dim3(256), 0, st>>>(
        a.partial, static_cast<int>(backward_groups(rows, cols)), cols, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace qsync
