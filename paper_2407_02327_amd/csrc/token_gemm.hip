// Products of INT8 codes with a scale for each row of either operand, C[m,n] = acc * (sa[m] sb[n]) + bias[n], over sets of rows (one: a
// linear operator; many: the experts of a layer, each with its own B).  In the forward pass and the data gradient a set owns rows of A and
// C; in the weight gradient it owns a stretch of the contraction axis and a whole C.
//
// The plainest form: a wavefront for 16 x 16 outputs, operands straight from memory into the matrix instruction.
#include "gemm_device.h"
#include "row_ops.h"
#include "token_ops.h"

namespace qsync {

namespace {

struct ProductTile      // one workgroup's: pointers to its set
{
    const int8_t *A, *B;
    int64_t       rows, cols, kb, m0, n0, c_at;      // rows and columns of the set's C, bytes of the contraction; c_at: C's element (0, 0)
    const float * sa, *sb, *bias;
};

// Tile `index` of the sets' tiles of BM x BN, false: there are fewer.
template <int BM, int BN, bool WGRAD> __device__ __forceinline__ bool product_tile(const TokenProduct& p, int64_t index, ProductTile& t)
{
    const int64_t tn = (p.N + BN - 1) / BN;
    if constexpr(WGRAD)
    {
        const int64_t tm = (p.M + BM - 1) / BM, e = index / (tm * tn), in = index % (tm * tn);
        if(e >= p.sets) return false;
        const SetRows s = set_rows(p.offsets, p.rows, p.sets, e);
        const int64_t start = set_start(p.offsets, s, e);
        t = {p.A + start * p.M, p.B + start * p.N, p.M, p.N, code_pad(s.len), in / tn * BM, in % tn * BN, e * p.M * p.N, p.sa + e * p.M, p.sb + e * p.N, nullptr};
        return true;
    }
    else
    {
        for(int64_t e = 0; e < p.sets; ++e)
        {
            const SetRows s = set_rows(p.offsets, p.rows, p.sets, e);
            const int64_t n = (s.len + BM - 1) / BM * tn;
            if(index < n)
            {
                const int64_t kb = code_pad(p.K);
                t = {p.A + s.first * kb, p.B + e * p.N * kb, s.len, p.N, kb, index / tn * BM, index % tn * BN, s.first * p.N, p.sa + s.first, p.sb + e * p.N,
                     p.bias ? p.bias + e * p.N : nullptr};
                return true;
            }
            index -= n;
        }
        return false;
    }
}

template <bool WGRAD> __global__ __launch_bounds__(64) void token_product_kernel(TokenProduct p)
{
    ProductTile t;
    if(!product_tile<16, 16, WGRAD>(p, blockIdx.x, t)) return;
    const int     lane = threadIdx.x, row = lane % 16, quad = lane / 16;
    const int64_t am = min(t.m0 + row, t.rows - 1), bn = min(t.n0 + row, t.cols - 1);
    v4i32         acc = {0, 0, 0, 0};
    for(int64_t k = quad * 16; k < t.kb; k += 64)
    {
        const v4i32 a = *reinterpret_cast<const v4i32*>(t.A + am * t.kb + k), b = *reinterpret_cast<const v4i32*>(t.B + bn * t.kb + k);
        acc           = I8Traits::mfma(b, a, acc);
    }
    // a lane holds four consecutive columns of row lane % 16
    const int64_t m = t.m0 + row;
    if(m >= t.rows) return;
    for(int i = 0; i < 4; ++i)
    {
        const int64_t n = t.n0 + quad * 4 + i;
        if(n < t.cols) element_store(p.C, p.c_dtype, t.c_at + m * t.cols + n, t.kb ? fmaf(static_cast<float>(acc[i]), t.sa[m] * t.sb[n], t.bias ? t.bias[n] : 0.0f) : t.bias ? t.bias[n] : 0.0f);
    }
}

}  // namespace

hipError_t launch_token_product(const TokenProduct& p, bool wgrad, hipStream_t st)
{
    const int64_t tn = (p.N + 15) / 16;
    const int64_t tiles = wgrad ? (p.M + 15) / 16 * tn * p.sets : ((p.rows + 15) / 16 + (p.offsets ? p.sets : 0)) * tn;
    if(wgrad) token_product_kernel<true><<<static_cast<unsigned>(tiles), 64, 0, st>>>(p);
    else      token_product_kernel<false><<<static_cast<unsigned>(tiles), 64, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace qsync
