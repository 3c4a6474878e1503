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

// A row: cols / 8 units of eight elements, and the fewer than eight behind them, one each for the first lanes ("edge").
__device__ __forceinline__ int64_t units_of(int64_t cols) { return cols / 8; }
__device__ __forceinline__ int64_t edge_of(int64_t cols, int lane) { return lane < static_cast<int>(cols % 8) ? cols / 8 * 8 + lane : -1; }

// A lane behind the last unit loads that one again, and leaves it out of the sums: a branch around the loads of each unit and row made
// 16384 x 4096 bfloat16 59 us of 52.
__device__ __forceinline__ int64_t unit_or_last(int64_t unit, int64_t units) { return unit < units ? unit : units - 1; }

// The eight parameters of a unit, or `absent`.
__device__ __forceinline__ void load_params(const float* p, int64_t unit, int64_t units, float absent, float (&v)[8])
{
#pragma unroll
    for(int e = 0; e < 8; ++e) v[e] = absent;
    if(!p || unit >= units) return;
    Row8<float> r;
    r.load(p + unit * 8);
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

// TPR lanes a row, NU units of eight elements a lane; WG / TPR rows of a workgroup at a time.  Short rows take a wavefront, or a quarter of
// one, whose lanes exchange their sums without LDS; longer ones the workgroup, with one barrier.  Bound by memory: 16384 x 4096 bfloat16
// 50 us (5.3 TB/s of x and y), 16384 x 1024 binary16 15 (4.5); a single row of 4096 is 2.9 us of launch and two memory latencies.
template <typename T, int TPR, int NU, int WG>
__global__ __launch_bounds__(WG) void norm_forward_kernel(const NormArgs p)
{
    constexpr int WAVES = TPR > kWaveSize ? TPR / kWaveSize : 1, ROWS = WG / TPR;
    static_assert(TPR <= kWaveSize || TPR == WG, "rows of several wavefronts take the workgroup");
    __shared__ float4 slots[2][WG / kWaveSize];
    const int     lane = threadIdx.x % TPR;
    const int64_t step = static_cast<int64_t>(gridDim.x) * ROWS, units = units_of(p.cols), edge = edge_of(p.cols, lane);
    const float   cols = static_cast<float>(p.cols);
    const T*      x    = static_cast<const T*>(p.x);

    float gamma[NU][8], beta[NU][8], held = edge >= 0 ? 1.0f : 0.0f;
#pragma unroll
    for(int u = 0; u < NU; ++u)
    {
        load_params(p.gamma, u * TPR + lane, units, 1.0f, gamma[u]);
        load_params(p.beta, u * TPR + lane, units, 0.0f, beta[u]);
        held += u * TPR + lane < units ? 8.0f : 0.0f;
    }
    const float edge_gamma = edge >= 0 && p.gamma ? p.gamma[edge] : 1.0f, edge_beta = edge >= 0 && p.beta ? p.beta[edge] : 0.0f;
    const float n = group_sum<TPR>(held);      // elements of this wavefront (of these 16 lanes)

    int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
    Row8<T> next[NU] = {};      // (rows of fewer than eight elements have no unit: zeros)
    float   next_edge = 0.0f;
    auto    fetch = [&](int64_t r) {
        const T* at = x + r * p.ldx;
        if(units > 0)
        {
#pragma unroll
            for(int u = 0; u < NU; ++u) next[u].load(at + unit_or_last(u * TPR + lane, units) * 8);
        }
        if(edge >= 0) next_edge = row_element(at + edge);
    };
    if(row < p.rows) fetch(row);
    float run = 0.0f;
    for(int turn = 0; row < p.rows; row += step, turn ^= 1)
    {
        float       v[NU][8];
        const float ve  = next_edge;
        float       sum = ve;
#pragma unroll
        for(int u = 0; u < NU; ++u)
        {
            next[u].decode(v[u]);
#pragma unroll
            for(int e = 0; e < 8; ++e) sum += u * TPR + lane < units ? v[u][e] : 0.0f;
        }
        if(row + step < p.rows) fetch(row + step);
        sum             = group_sum<TPR>(sum);
        const float own = n > 0.0f ? sum / n : 0.0f;
        float       m2  = edge >= 0 ? (ve - own) * (ve - own) : 0.0f;
#pragma unroll
        for(int u = 0; u < NU; ++u)
#pragma unroll
            for(int e = 0; e < 8; ++e)
            {
                const float d = u * TPR + lane < units ? v[u][e] - own : 0.0f;
                m2            = fmaf(d, d, m2);
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
            const int64_t unit = u * TPR + lane;
            if(unit >= units) continue;
            float o[8];
#pragma unroll
            for(int e = 0; e < 8; ++e) o[e] = fmaf((v[u][e] - mean) * rstd, gamma[u][e], beta[u][e]);
            if(!p.amax_bits) row8_store<false>(p.y, p.ydt, row * p.cols + unit * 8, o);
            else
            {
                row8_store<true>(p.y, p.ydt, row * p.cols + unit * 8, o);
#pragma unroll
                for(int e = 0; e < 8; ++e) run = fmaxf(run, fabsf(o[e]));
            }
        }
        if(edge >= 0) run = fmaxf(run, fabsf(element_store(p.y, p.ydt, row * p.cols + edge, fmaf((ve - mean) * rstd, edge_gamma, edge_beta))));
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

// Every element of a row in turn: unit(number, column), then one(column) for the edge's.
template <int WG, typename F, typename G> __device__ __forceinline__ void each_of_row(int64_t cols, F&& unit, G&& one)
{
    for(int64_t u = threadIdx.x; u < units_of(cols); u += WG) unit(u * 8);
    const int64_t edge = edge_of(cols, threadIdx.x);
    if(edge >= 0) one(edge);
}

// Rows longer than the registers of a workgroup hold (16384 columns): read three times, the second and third time out of a cache.  200 x 20000
// fp32 11 us.
template <typename T> __global__ __launch_bounds__(1024) void norm_forward_long_kernel(const NormArgs p)
{
    __shared__ float2 slots[3][16];
    const float       cols = static_cast<float>(p.cols);
    float             run  = 0.0f;
    for(int64_t row = blockIdx.x; row < p.rows; row += gridDim.x)
    {
        const T* at = static_cast<const T*>(p.x) + row * p.ldx;
        float    v[8], sum = 0.0f, m2 = 0.0f;
        auto     fetch = [&](int64_t c) {
            Row8<T> r;
            r.load(at + c);
            r.decode(v);
        };
        each_of_row<1024>(
            p.cols,
            [&](int64_t c) {
                fetch(c);
                sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
            },
            [&](int64_t c) { sum += row_element(at + c); });
        const float mean = block_sum2<1024>(sum, 0.0f, slots[0]).x / cols;
        each_of_row<1024>(
            p.cols,
            [&](int64_t c) {
                fetch(c);
#pragma unroll
                for(int e = 0; e < 8; ++e)
                {
                    const float d = v[e] - mean;
                    m2            = fmaf(d, d, m2);
                }
            },
            [&](int64_t c) {
                const float d = row_element(at + c) - mean;
                m2            = fmaf(d, d, m2);
            });
        const float var  = block_sum2<1024>(m2, 0.0f, slots[1]).x / cols;
        const float rstd = 1.0f / sqrtf(var + p.eps);
        if(threadIdx.x == 0)
        {
            if(p.mean) p.mean[row] = mean;
            if(p.rstd) p.rstd[row] = rstd;
        }
        each_of_row<1024>(
            p.cols,
            [&](int64_t c) {
                float g[8], b[8];
                fetch(c);
                load_params(p.gamma, c / 8, units_of(p.cols), 1.0f, g);
                load_params(p.beta, c / 8, units_of(p.cols), 0.0f, b);
#pragma unroll
                for(int e = 0; e < 8; ++e) v[e] = fmaf((v[e] - mean) * rstd, g[e], b[e]);
                row8_store<true>(p.y, p.ydt, row * p.cols + c, v);
#pragma unroll
                for(int e = 0; e < 8; ++e) run = fmaxf(run, fabsf(v[e]));
            },
            [&](int64_t c) {
                const float o = fmaf((row_element(at + c) - mean) * rstd, p.gamma ? p.gamma[c] : 1.0f, p.beta ? p.beta[c] : 0.0f);
                run           = fmaxf(run, fabsf(element_store(p.y, p.ydt, row * p.cols + c, o)));
            });
    }
    if(p.amax_bits) publish_largest(run, p.amax_bits, reinterpret_cast<float*>(slots[2]));
}

// TD: dy, T: x.  One pass: the row's two sums (one barrier for both), dx from registers, and the parameters' sums, which a lane keeps for its
// columns over all rows of the workgroup -- 32 registers a unit, the reason for at most two.  16384 x 1024 binary16 19 us (5.3 TB/s of x, dy
// and dx) and 3.7 for the fold of 256 partial rows; 16384 x 4096 bfloat16 84 with it (4.8 TB/s).
template <typename TD, typename T, int TPR, int NU, int WG>
__global__ __launch_bounds__(WG) void norm_backward_kernel(const NormArgs p)
{
    constexpr int WAVES = TPR > kWaveSize ? TPR / kWaveSize : 1, ROWS = WG / TPR;
    static_assert(TPR <= kWaveSize || TPR == WG, "rows of several wavefronts take the workgroup");
    __shared__ float2 slots[2][WG / kWaveSize];
    const int     lane = threadIdx.x % TPR;
    const int64_t step = static_cast<int64_t>(gridDim.x) * ROWS, units = units_of(p.cols), edge = edge_of(p.cols, lane);
    const float   cols = static_cast<float>(p.cols);
    const T*      x    = static_cast<const T*>(p.x);
    const TD*     dy   = static_cast<const TD*>(p.dy);

    float gamma[NU][8], sum_g[NU][8], sum_b[NU][8], edge_g = 0.0f, edge_b = 0.0f;
#pragma unroll
    for(int u = 0; u < NU; ++u)
    {
        load_params(p.gamma, u * TPR + lane, units, 1.0f, gamma[u]);
#pragma unroll
        for(int e = 0; e < 8; ++e) sum_g[u][e] = sum_b[u][e] = 0.0f;
    }
    const float edge_gamma = edge >= 0 && p.gamma ? p.gamma[edge] : 1.0f;
    int64_t     row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
    Row8<T>     next_x[NU]  = {};
    Row8<TD>    next_dy[NU] = {};
    float       next_mean = 0.0f, next_rstd = 0.0f, next_edge_x = 0.0f, next_edge_dy = 0.0f;
    auto        fetch = [&](int64_t r) {
        const T*  at_x  = x + r * p.ldx;
        const TD* at_dy = dy + r * p.lddy;
        if(units > 0)
        {
#pragma unroll
            for(int u = 0; u < NU; ++u)
            {
                next_x[u].load(at_x + unit_or_last(u * TPR + lane, units) * 8);
                next_dy[u].load(at_dy + unit_or_last(u * TPR + lane, units) * 8);
            }
        }
        if(edge >= 0)
        {
            next_edge_x  = row_element(at_x + edge);
            next_edge_dy = row_element(at_dy + edge);
        }
        next_mean = p.mean[r];
        next_rstd = p.rstd[r];
    };
    if(row < p.rows) fetch(row);
    for(int turn = 0; row < p.rows; row += step, turn ^= 1)
    {
        float       xh[NU][8], d[NU][8];
        const float mean = next_mean, rstd = next_rstd;
        const float edge_xh = edge >= 0 ? (next_edge_x - mean) * rstd : 0.0f, edge_dy = next_edge_dy, edge_d = edge_dy * edge_gamma;
        float       s1 = edge_d, s2 = edge_d * edge_xh;
        edge_g = fmaf(edge_dy, edge_xh, edge_g);
        edge_b += edge_dy;
#pragma unroll
        for(int u = 0; u < NU; ++u)
        {
            next_x[u].decode(xh[u]);
            next_dy[u].decode(d[u]);
#pragma unroll
            for(int e = 0; e < 8; ++e)
            {
                d[u][e] = u * TPR + lane < units ? d[u][e] : 0.0f;
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
            const int64_t unit = u * TPR + lane;
            if(unit >= units) continue;
            float o[8];
#pragma unroll
            for(int e = 0; e < 8; ++e) o[e] = rstd * (d[u][e] - s1 - xh[u][e] * s2);
            row8_store<false>(p.y, p.ydt, row * p.cols + unit * 8, o);
        }
        if(edge >= 0) element_store(p.y, p.ydt, row * p.cols + edge, rstd * (edge_d - s1 - edge_xh * s2));
    }
    if(!p.partial) return;
    float* out = p.partial + static_cast<int64_t>(blockIdx.x) * 2 * p.cols;
    if constexpr(ROWS == 1)
    {
#pragma unroll
        for(int u = 0; u < NU; ++u)
        {
            const int64_t unit = u * TPR + lane;
            if(unit >= units) continue;
            row8_store<false>(out, kF32, unit * 8, sum_g[u]);
            row8_store<false>(out, kF32, p.cols + unit * 8, sum_b[u]);
        }
        if(edge >= 0)
        {
            out[edge]          = edge_g;
            out[p.cols + edge] = edge_b;
        }
    }
    else
    {   // the groups' sums, added in order
        constexpr int     SPAN = TPR * NU * 8 + 8;
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
                if(u * TPR + lane >= units) continue;
                at[0] = make_float4(s[0], s[1], s[2], s[3]);
                at[1] = make_float4(s[4], s[5], s[6], s[7]);
            }
            if(edge >= 0) flat[g * SPAN + edge] = which ? edge_b : edge_g;
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

// Long rows: dx of a row by a workgroup, x and dy read twice (and once more for the parameters): 4096 x 16384 bfloat16 165 us.
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
        float       xh[8], d[8], s1 = 0.0f, s2 = 0.0f;
        auto        fetch = [&](int64_t c) {
            Row8<T>  rx;
            Row8<TD> rd;
            float    g[8];
            rx.load(x + c);
            rd.load(dy + c);
            load_params(p.gamma, c / 8, units_of(p.cols), 1.0f, g);
            rx.decode(xh);
            rd.decode(d);
#pragma unroll
            for(int e = 0; e < 8; ++e)
            {
                xh[e] = (xh[e] - mean) * rstd;
                d[e] *= g[e];
            }
        };
        auto fetch_one = [&](int64_t c) {
            xh[0] = (row_element(x + c) - mean) * rstd;
            d[0]  = row_element(dy + c) * (p.gamma ? p.gamma[c] : 1.0f);
        };
        each_of_row<1024>(
            p.cols,
            [&](int64_t c) {
                fetch(c);
#pragma unroll
                for(int e = 0; e < 8; ++e)
                {
                    s1 += d[e];
                    s2 = fmaf(d[e], xh[e], s2);
                }
            },
            [&](int64_t c) {
                fetch_one(c);
                s1 += d[0];
                s2 = fmaf(d[0], xh[0], s2);
            });
        const float2 t = block_sum2<1024>(s1, s2, slots[turn]);
        s1 = t.x / cols;
        s2 = t.y / cols;
        each_of_row<1024>(
            p.cols,
            [&](int64_t c) {
                fetch(c);
#pragma unroll
                for(int e = 0; e < 8; ++e) d[e] = rstd * (d[e] - s1 - xh[e] * s2);
                row8_store<false>(p.y, p.ydt, row * p.cols + c, d);
            },
            [&](int64_t c) {
                fetch_one(c);
                element_store(p.y, p.ydt, row * p.cols + c, rstd * (d[0] - s1 - xh[0] * s2));
            });
    }
}
// ... and the parameters' partial sums, a strip of 2048 columns over every gridDim.y-th row a workgroup; the last one has the edge
template <typename TD, typename T> __global__ __launch_bounds__(256) void norm_params_kernel(const NormArgs p)
{
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, units = units_of(p.cols);
    const int64_t edge = blockIdx.x == gridDim.x - 1 ? edge_of(p.cols, threadIdx.x) : -1;
    if(unit >= units && edge < 0) return;
    float sum_g[8] = {}, sum_b[8] = {}, edge_g = 0.0f, edge_b = 0.0f;
    for(int64_t row = blockIdx.y; row < p.rows; row += gridDim.y)
    {
        const T*    x    = static_cast<const T*>(p.x) + row * p.ldx;
        const TD*   dy   = static_cast<const TD*>(p.dy) + row * p.lddy;
        const float mean = p.mean[row], rstd = p.rstd[row];
        if(unit < units)
        {
            Row8<T>  rx;
            Row8<TD> rd;
            float    xh[8], d[8];
            rx.load(x + unit * 8);
            rd.load(dy + unit * 8);
            rx.decode(xh);
            rd.decode(d);
#pragma unroll
            for(int e = 0; e < 8; ++e)
            {
                sum_g[e] = fmaf(d[e], (xh[e] - mean) * rstd, sum_g[e]);
                sum_b[e] += d[e];
            }
        }
        if(edge >= 0)
        {
            const float d = row_element(dy + edge);
            edge_g = fmaf(d, (row_element(x + edge) - mean) * rstd, edge_g);
            edge_b += d;
        }
    }
    float* out = p.partial + static_cast<int64_t>(blockIdx.y) * 2 * p.cols;
    if(unit < units)
    {
        row8_store<false>(out, kF32, unit * 8, sum_g);
        row8_store<false>(out, kF32, p.cols + unit * 8, sum_b);
    }
    if(edge >= 0)
    {
        out[edge]          = edge_g;
        out[p.cols + edge] = edge_b;
    }
}

// Workgroups of a launch: larger problems loop, or go on in the grid's next row.  A launch of 2^32 threads is refused, and one of a few more runs as those few alone.
constexpr int64_t kNormMostGroups = 1 << 22;

// dgamma and dbeta from S partial rows [S][2][cols]
__global__ __launch_bounds__(256) void norm_fold_kernel(const float* partial, int S, int64_t cols, float* dgamma, float* dbeta)
{
    __shared__ float lds[256];
    const int        q = threadIdx.x / 16;
    const int64_t    c = (static_cast<int64_t>(blockIdx.y) * kNormMostGroups + blockIdx.x) * 16 + threadIdx.x % 16;
    const float      t = fold_column<false>(partial, S, 2 * cols, c, q, lds);
    if(q != 0 || c >= 2 * cols) return;
    if(c < cols) { if(dgamma) dgamma[c] = t; }
    else if(dbeta) dbeta[c - cols] = t;
}

constexpr int64_t kNormMaxCols   = 8192;      // columns of a row that is kept in registers by the backward pass
constexpr int64_t kNormParamRows = 64;        // partial rows of the parameters' gradients of rows that are longer

int64_t at_most(int64_t v, int64_t most) { return v < most ? v : most; }
int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Workgroups for `turns` turns of one, all with the same number of turns (but the last): `most` of them, or as many as have `turns_each`.
int64_t even_groups(int64_t turns, int64_t most, int64_t turns_each)
{
    const int64_t each = at_most(div_up(turns, most), turns_each);
    return div_up(turns, each);
}

// Four turns of a workgroup (eight of the wide ones) repay its loads of gamma and beta; more of them, and the device runs out of step.  us
// at 1, 2, 4 and 8 turns: 16384 x 1024 binary16 17.4 17.1 15.7 16.9, 16384 x 2048 (4, 8, 16) 31.3 33.4 35.7, 4096 x 8192 (4, 8) 31.2 29.7.
template <typename T, int TPR, int NU, int WG> hipError_t forward_rows(const NormArgs& a, hipStream_t st)
{
    const int64_t turns = div_up(a.rows, WG / TPR), groups = even_groups(turns, WG == 256 ? 1024 : 512, WG == 256 ? 4 : 8);
    norm_forward_kernel<T, TPR, NU, WG><<<dim3(static_cast<unsigned>(at_most(groups, kNormMostGroups))), dim3(WG), 0, st>>>(a);
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

// How a row of the backward pass is divided, and the most workgroups: what registers let run at once, less where their partial rows --
// written, and read again by the fold -- would weigh.  us with 256, 512, 768 and 1024 of them: 16384 x 4096 bfloat16 90.7 83.7 90.0 98.9,
// 16384 x 2048 binary16 62.7 52.1 48.5 48.7, 4096 x 8192 48.4 58.1 66.8 77.5; 16384 x 1024 with eight rows at a time and 256 24.8, four and
// 512 26.2.  Where x and dy have 16 bits, a workgroup for every seven rows, and more of them where rows are not whole units of eight,
// whose loads and stores straddle lines: 7199 x 2443 bfloat16 61 -> 49, 16384 x 2501 binary16 102 -> 84, 7199 x 4096 bfloat16 47 -> 43.  With
// fp32 one for every twenty: seven make 4096 x 4095 50 of 45, and up to 768 of them 10000 x 3001 87 of 77.
struct BackwardShape { int64_t rows_at_once, most; };
BackwardShape backward_shape(int64_t cols, bool narrow)
{
    return cols <= 128 ? BackwardShape{16, 256} : cols <= 1024 ? BackwardShape{8, 256}
           : cols <= 2048 ? BackwardShape{1, 768} : cols <= 4096 ? BackwardShape{1, narrow && cols % 8 ? 768 : 512} : BackwardShape{1, 256};
}
int64_t backward_wanted(int64_t rows, bool narrow)
{
    const int64_t groups = rows / (narrow ? 7 : 20);
    return groups < 256 ? 256 : groups;
}
int64_t backward_groups(int64_t rows, int64_t cols, bool narrow)
{
    if(cols > kNormMaxCols) return at_most(rows, kNormParamRows);
    const BackwardShape s = backward_shape(cols, narrow);
    return even_groups(div_up(rows, s.rows_at_once), at_most(backward_wanted(rows, narrow), s.most), rows);
}
// No number of rows up to this one, whatever the types, has more workgroups (16-bit ones have the most; backward_groups itself falls where a turn more evens them out).
int64_t most_backward_groups(int64_t rows, int64_t cols)
{
    constexpr bool narrow = true;
    if(cols > kNormMaxCols) return at_most(rows, kNormParamRows);
    const BackwardShape s = backward_shape(cols, narrow);
    return at_most(div_up(rows, s.rows_at_once), at_most(backward_wanted(rows, narrow), s.most));
}
template <typename TD, typename T, int TPR, int NU, int WG> hipError_t backward_rows(const NormArgs& a, int64_t groups, hipStream_t st)
{
    norm_backward_kernel<TD, T, TPR, NU, WG><<<dim3(static_cast<unsigned>(groups)), dim3(WG), 0, st>>>(a);
    return hipGetLastError();
}
template <typename TD, typename T> hipError_t backward_types(const NormArgs& a, hipStream_t st)
{
    const int64_t groups = backward_groups(a.rows, a.cols, sizeof(TD) == 2 && sizeof(T) == 2);
    if(a.cols <= 128) return backward_rows<TD, T, 16, 1, 256>(a, groups, st);
    if(a.cols <= 512) return backward_rows<TD, T, 64, 1, 512>(a, groups, st);
    if(a.cols <= 1024) return backward_rows<TD, T, 64, 2, 512>(a, groups, st);
    if(a.cols <= 2048) return backward_rows<TD, T, 256, 1, 256>(a, groups, st);
    if(a.cols <= 4096) return backward_rows<TD, T, 256, 2, 256>(a, groups, st);
    if(a.cols <= kNormMaxCols) return backward_rows<TD, T, 512, 2, 512>(a, groups, st);
    // (the parameters' sums first: dx may take the place of dy or x)
    if(a.partial)
    {
        norm_params_kernel<TD, T><<<dim3(static_cast<unsigned>(div_up(a.cols / 8, 256)), static_cast<unsigned>(groups)), dim3(256), 0, st>>>(a);
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
    return static_cast<size_t>(most_backward_groups(rows, cols)) * 2 * static_cast<size_t>(cols) * sizeof(float);
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
    const int64_t groups = div_up(2 * cols, 16);
    norm_fold_kernel<<<dim3(static_cast<unsigned>(at_most(groups, kNormMostGroups)), static_cast<unsigned>(div_up(groups, kNormMostGroups))), dim3(256), 0, st>>>(
        a.partial, static_cast<int>(backward_groups(rows, cols, dydt != kF32 && xdt != kF32)), cols, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace qsync
