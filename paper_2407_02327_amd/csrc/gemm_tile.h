// One output tile of an int8 or binary16 matrix product on the matrix instructions: loads through LDS, K loop, hand-over to the epilogue.  The
// forms that gemm_mfma.hip and token_gemm.hip launch are described there.
#pragma once
#include "gemm_device.h"

namespace qsync {

namespace {

// Implicit patch matrix of a 3x3 / stride 1 / pad 1 convolution over an NHWC tensor: row m of A is
// output pixel m, its K axis runs (kh, kw, c).  A 16-byte chunk lies inside one tap because the
// pixel size is a multiple of 16 bytes, so the direct load of a lane either reads 16 bytes of the
// neighbouring pixel (same image, inside the border) or, for padding and for chunks past the end
// of K, 16 zero bytes from a constant block.
// Where a lane's two chunk positions (by parity of the load slot) stand on the K axis: the byte offset (less W + 1 pixels,
// modulo 2^32), the tap it lies in and the channel offset in that tap.  Requests go over consecutive K tiles, so the position is carried on instead of
// divided out of the tile index (a division per parity and tile, and border tests per load, made the gather's own
// arithmetic the bound of the K loop: four loads took about 130 vector instructions, now about 55).
struct ConvTap { uint32_t koff[2], tap[2], c0[2]; };

// `mask`: bit t says that tap t of the lane's output pixel lies inside the image; taps from 9 on (chunks past the end
// of K) have no bit.  `delta`: byte distance from the pixel to the chunk's source, modulo 2^32: their sum is the source's
// offset in the tensor, below 2^31 wherever the mask has the bit.  (Without the modulus, on a base W + 1 pixels in front
// of the tensor, the sum reaches 2 W + 1 pixels and left 32 bits for one row of nearly 2^31 bytes.)
template <int D, int DPW>
__device__ __forceinline__ void conv_issue(const uint8_t* a, const uint8_t* zero, uint32_t pix_off, uint32_t mask,
                                           const ConvTap& t, const uint32_t (&delta)[2], uint8_t* lds_mid)
{
    constexpr int IMM = dma_imm<D, DPW>();
    constexpr int par = D & 1;
    const uint8_t* src = ((mask >> t.tap[par]) & 1u) ? a + (pix_off + delta[par]) : zero;
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src - IMM),
                                     (__attribute__((address_space(3))) void*)(lds_mid + dma_lds_shift<D, DPW>()), 16, IMM, 0);
}

template <int DPW, int... Ds>
__device__ __forceinline__ void conv_sequence(std::integer_sequence<int, Ds...>, const uint8_t* a, const uint8_t* zero,
                                              const uint32_t (&pix_off)[DPW], const uint32_t (&mask)[DPW],
                                              const ConvTap& t, const uint32_t (&delta)[2], uint8_t* lds_mid)
{
    (conv_issue<Ds, DPW>(a, zero, pix_off[Ds], mask[Ds], t, delta, lds_mid), ...);
}

// TN form with the B operand gathered from an NHWC tensor (weight gradient of the 3x3 convolution): stage row r of
// K tile kt is pixel m = kt * KR + r, and a lane's 16-byte chunk lies in one tap (dh, dw) at channel offset c0, both
// fixed per load slot; what changes from K tile to K tile is the pixel, i.e. (h, w).  `delta` holds the slot's whole
// constant part ((dh W + dw) Cb + c0 + r Cb), modulo 2^32; `code`, low byte: (dh + 1) | (dw + 1) << 2 | valid << 4; `hw` = h << 16 | w of the
// pixel of the NEXT K tile to be requested and is advanced by KR pixels here (dr = KR % W, hq = (KR / W) % H).
template <int D, int DPW>
__device__ __forceinline__ void conv_tn_issue(const uint8_t* x, const uint8_t* zero, uint32_t pix_base, uint32_t delta, int code,
                                              uint32_t& hw, int H, int W, int dr, int hq, uint8_t* lds_mid)
{
    constexpr int IMM = dma_imm<D, DPW>();
    int        h = static_cast<int>(hw >> 16), w = static_cast<int>(hw & 0xffffu);
    const int  hh = h + (code & 3) - 1, ww = w + ((code >> 2) & 3) - 1;
    const bool inb = ((code >> 4) & 1) != 0 && static_cast<unsigned>(hh) < static_cast<unsigned>(H)
                     && static_cast<unsigned>(ww) < static_cast<unsigned>(W);
    const uint8_t* src = inb ? x + (pix_base + delta) : zero;       // (an offset in the tensor, below 2^31, wherever it is read)
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src - IMM),
                                     (__attribute__((address_space(3))) void*)(lds_mid + dma_lds_shift<D, DPW>()), 16, IMM, 0);
    w += dr;
    const int carry = w >= W ? 1 : 0;
    w -= carry ? W : 0;
    h += hq + carry;
    h -= h >= H ? H : 0;
    hw = (static_cast<uint32_t>(h) << 16) | static_cast<uint32_t>(w);
}

template <int DPW, int... Ds>
__device__ __forceinline__ void conv_tn_sequence(std::integer_sequence<int, Ds...>, const uint8_t* x, const uint8_t* zero,
                                                 uint32_t pix_base, const uint32_t (&delta)[DPW], const uint32_t (&codes)[(DPW + 3) / 4],
                                                 uint32_t (&hw)[DPW], int H, int W, int dr, int hq, uint8_t* lds_mid)
{
    (conv_tn_issue<Ds, DPW>(x, zero, pix_base, delta[Ds], static_cast<int>(codes[Ds / 4] >> (8 * (Ds % 4))), hw[Ds], H, W, dr, hq, lds_mid), ...);
}

// TN, last K tile with fewer contraction rows than a stage holds: rows from `rows` on are fetched from the tile's first
// row instead (and overwritten with zeros once landed).
template <int DPW, int RPS, int... Ds>
__device__ __forceinline__ void dma_sequence_short(std::integer_sequence<int, Ds...>, const uint8_t* sbase,
                                                   const uint32_t (&voff)[DPW], int row0, int rows, uint32_t row_bytes, uint8_t* lds_mid)
{
    (dma_issue<Ds, DPW>(sbase, voff[Ds] - (row0 + Ds * RPS >= rows ? static_cast<uint32_t>(row0 + Ds * RPS) * row_bytes : 0u), lds_mid), ...);
}

// TN (int8 and binary16): both operands are handed over with the contraction axis as their ROW axis, A [P, M] and
// B [P, N] row-major (C[m,n] = sum_p A[p,m] B[p,n]): the weight gradient dW = dY^T X straight from the row-major
// operands, no transposed copies.  A stage then holds 128 (int8) or 64 (binary16) contraction rows of each operand
// (rows of BM / BN elements), and the fragments come out of LDS through the transposing reads of gfx950
// (ds_read_b64_tr_b8 / _b16): sixteen lanes read 8 rows x 16 bytes (4 rows x 32 bytes) and receive, lane j, the
// eight (four) elements of column j -- consecutive contraction indices of one output row, which is what the
// matrix instruction wants; two reads make a lane's 16 operand bytes.  16-byte chunks are XOR-swizzled per row so
// that the lanes of one access pass touch all banks once.  Everything behind the fragments
// (matrix instructions, epilogue, split K) is shared with the NT form.  Kb is the contraction length P here.
// MIXED: whether the workgroup leaves raw sums (its problem is in K splits) is known at run time only (`raw`).
// TOKEN: scales of the rows, too (store_tile).
template <typename TR, int BM, int BN, int WGM, int WGN, int ST, int NL, bool SPLIT, bool CONV, bool TN, bool MIXED = false, bool TOKEN = false>
__device__ __forceinline__ void gemm_tile_at(const GemmKernelArgs& p, int split, int tm, int tn, bool raw = SPLIT)
{
    static_assert(!MIXED || SPLIT, "one body for both");
    constexpr bool WHOLE = !SPLIT || MIXED;      // the epilogue may be this workgroup's
    static_assert(!(SPLIT && CONV && !TN), "the implicit patch matrix of the forward is not combined with split K");
    static_assert(!TN || (TR::kElemBytes <= 2 && BM == BN && BM >= 64), "TN: int8 or binary16 operands, square tiles");
    constexpr bool CONVA  = CONV && !TN;       // NT form: the A operand is the implicit patch matrix (forward, data gradient)
    constexpr bool CONVTN = CONV && TN;        // TN form: the B operand is gathered from the NHWC tensor (weight gradient)
    constexpr int ESZ = TR::kElemBytes;
    typedef typename TR::accv_t accv_t;
    typedef typename TR::acc_t  acc_t;
    constexpr int kThreads = 64 * WGM * WGN;
    constexpr int WTM = BM / WGM, WTN = BN / WGN;   // wavefront sub-tile
    constexpr int R = TR::kRows, FM = WTM / R, FN = WTN / R;         // fragments per wavefront
    constexpr int CH = kRowBytes / (16 * (64 / R));                 // K chunks (16 bytes of each of 64 / R lanes) per K tile
    constexpr int STAGE_BYTES = (BM + BN) * kRowBytes;
    constexpr int WC = WGM * WGN, WL = NL > 0 ? NL : WC;            // wavefronts that compute, that load
    constexpr int DPW = (BM + BN) / 8 / WL;                         // direct-load instructions per loading wavefront per K tile
    static_assert(R == 16 && CH == 2 && WTM % R == 0 && WTN % R == 0 && FM >= FN && (FN == 2 || FN == 4), "fragments of a wavefront");
    static_assert((BM + BN) % (8 * WL) == 0 && BM % 16 == 0, "stage rows must split evenly over the wavefronts");

    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];

    const int64_t m0 = static_cast<int64_t>(tm) * BM, n0 = static_cast<int64_t>(tn) * BN;
    const int     tid = threadIdx.x, lane = tid % kWaveSize;
    const int     wave = __builtin_amdgcn_readfirstlane(tid / kWaveSize);     // wavefront index, held in an SGPR
    const int     wm = wave / WGN, wn = wave % WGN;
    const int     lwave = NL == 0 ? wave : wave >= WC ? wave - WC : 0;          // index among the loading wavefronts

    // K-tile indices are 32-bit so that the loop control stays on the scalar unit
    const int ktiles_all = static_cast<int>((p.Kb + kRowBytes - 1) / kRowBytes);
    const int tail_kt    = (p.Kb % kRowBytes) ? ktiles_all - 1 : -1;     // index of a partial last tile, if any
    int       kt_begin = 0, kt_end = ktiles_all;
    if(SPLIT)
    {
        kt_begin = split * p.ktiles_per_split;
        kt_end   = kt_begin + p.ktiles_per_split < ktiles_all ? kt_begin + p.ktiles_per_split : ktiles_all;
    }

    // Global -> LDS with direct loads (global_load_lds_dwordx4): the data never passes through
    // VGPRs and no LDS store instruction is issued.  One such instruction of a wavefront fills
    // 1 KB of LDS = 8 consecutive stage rows (A rows first, then B rows): lane l lands at row l/8,
    // chunk position l%8, so it fetches the logical chunk (l%8) ^ ((row/2)%8) of that row.
    // Rows beyond M (or N) are clamped to the last row: they only feed accumulators of outputs
    // that are never stored.  Chunks beyond the end of K (last, partial K tile only) are
    // fetched from the row's first chunk of that tile and overwritten with zeros once landed.
    // A wavefront's DPW instructions cover 8*DPW consecutive stage rows, all of A or all of B, so
    // its source is one uniform base pointer plus a 32-bit lane offset per instruction.
    constexpr bool kUniformSide = (BM / 8) % DPW == 0;
    static_assert(kUniformSide, "a wavefront must not straddle the A/B boundary of a stage");
    const bool     is_a      = lwave * DPW < BM / 8;
    // TN: the panel starts at the tile's first column of the operand (its rows are contraction indices)
    const uint8_t* gbase     = TN ? (is_a ? p.A + m0 * ESZ : (CONVTN ? p.B : p.B + n0 * ESZ))
                                  : (is_a ? p.A + m0 * p.Kb : ((!CONV && p.remap_C > 0) ? p.B : p.B + n0 * p.Kb));
    const int64_t  rows_left = is_a ? p.M - m0 : p.N - n0;           // >= 1
    uint32_t       voff[DPW];                                         // lane offset + kDmaBias - immediate
    uint32_t       hw[CONV ? DPW : 1];       // CONVTN: (h << 16) | w of the lane's pixels; CONVA: their taps inside the image
    uint32_t       tnc_code[CONVTN ? (DPW + 3) / 4 : 1] = {};      // CONVTN, B side (see conv_tn_issue), a byte per load; voff holds the deltas there
    int            gchunk[2];                                         // the swizzle term depends on d%2 only
    {
        int imm[DPW];
        fill_dma_imms<DPW>(imm, std::make_integer_sequence<int, DPW>{});
        if constexpr(TN)
        {   // instruction q of the stage fills LDS bytes [1024 q, 1024 q + 1024) of the A region (128 / ESZ rows of
            // BM elements), then of the B region; a lane's 16 bytes are chunk (position ^ swizzle(row)) of its row
            constexpr int RB = BM * ESZ;                                   // bytes per region row
            const int64_t ld    = (is_a ? p.M : p.N) * ESZ;                // operand row length in bytes
            const int64_t width = (is_a ? p.M - m0 : p.N - n0) * ESZ;      // valid bytes of this tile's columns (>= 16)
#pragma unroll
            for(int d = 0; d < DPW; ++d)
            {
                const int q     = lwave * DPW + d - (is_a ? 0 : BM / 8);
                const int o     = q * 1024 + lane * 16;
                const int row   = o / RB, pos = (o % RB) / 16;
                int       chunk = pos ^ tn_swizzle<ESZ, RB>(row);
                if constexpr(CONVTN)
                    if(!is_a)
                    {   // B side: column byte (n0 * ESZ + 16 chunk) of the implicit [pixels, 9 C] matrix = tap, channel offset
                        constexpr int KR = kRowBytes / ESZ;                       // pixels per K tile
                        const uint32_t colb  = static_cast<uint32_t>(n0) * ESZ + static_cast<uint32_t>(chunk) * 16u;      // (9 C < 2^24)
                        const bool     valid = colb < 9u * static_cast<uint32_t>(p.conv_Cb);      // tile columns past 9 C: zeros, never stored
                        const int      tap   = valid ? static_cast<int>(colb / static_cast<uint32_t>(p.conv_Cb)) : 0;
                        const int      c0    = valid ? static_cast<int>(colb) - tap * p.conv_Cb : 0;
                        const int     kh = (tap * 11) >> 5, kw = tap - 3 * kh;          // tap / 3 for tap < 12
                        voff[d]      = static_cast<uint32_t>(((kh - 1) * p.conv_W + (kw - 1)) * p.conv_Cb + c0 + row * p.conv_Cb);
                        tnc_code[d / 4] |= static_cast<uint32_t>(kh | (kw << 2) | (valid ? 16 : 0)) << (8 * (d % 4));
                        const uint32_t m  = static_cast<uint32_t>(kt_begin) * KR + static_cast<uint32_t>(row);
                        const uint32_t qq = m / static_cast<uint32_t>(p.conv_W);
                        hw[d]   = ((qq % static_cast<uint32_t>(p.conv_H)) << 16) | (m - qq * static_cast<uint32_t>(p.conv_W));
                        continue;
                    }
                if(static_cast<int64_t>(chunk) * 16 >= width) chunk = 0;    // columns past the matrix: any valid chunk, never stored
                voff[d] = static_cast<uint32_t>(static_cast<int64_t>(row) * ld + chunk * 16 + kDmaBias - imm[d]);
            }
            gchunk[0] = gchunk[1] = 0;
        }
        else
#pragma unroll
        for(int d = 0; d < DPW; ++d)
        {
            const int srow  = (lwave * DPW + d) * 8 + lane / 8;           // row inside the stage
            const int chunk = (lane % 8) ^ ((srow >> 1) & 7);             // BM % 16 == 0: same term for A and B rows
            int64_t   lrow  = srow - (is_a ? 0 : BM);
            if(lrow >= rows_left) lrow = rows_left - 1;
            voff[d] = static_cast<uint32_t>(lrow * p.Kb + chunk * 16 + kDmaBias - imm[d]);
            if constexpr(CONVA)
                if(is_a)
                {   // A side: voff holds the byte offset of output pixel m in the NHWC tensor instead
                    const uint32_t m = static_cast<uint32_t>(m0 + lrow), q = m / static_cast<uint32_t>(p.conv_W);
                    voff[d] = m * static_cast<uint32_t>(p.conv_Cb);
                    const uint32_t h = q % static_cast<uint32_t>(p.conv_H), w = m - q * static_cast<uint32_t>(p.conv_W);
                    const uint32_t row = (w > 0 ? 1u : 0u) | 2u | (w + 1 < static_cast<uint32_t>(p.conv_W) ? 4u : 0u);
                    hw[d] = (h > 0 ? row : 0u) | (row << 3) | (h + 1 < static_cast<uint32_t>(p.conv_H) ? row << 6 : 0u);
                }
            if(d < 2) gchunk[d] = chunk * 16;
        }
        if constexpr(!CONV && !TN)
            if(p.remap_C > 0 && !is_a)
            {   // offset from p.B itself (the base below is not advanced to this tile's rows); in a block of its own, so
                // that the ordinary kernel's first instructions are not spread over these divisions
#pragma unroll
                for(int d = 0; d < DPW; ++d)
                {
                    const int      lrow = (lwave * DPW + d) * 8 + lane / 8 - BM;
                    const uint32_t row  = static_cast<uint32_t>(n0 + (lrow < rows_left ? lrow : rows_left - 1));
                    const int      tap  = static_cast<int>(row / static_cast<uint32_t>(p.remap_C));
                    const int      c    = static_cast<int>(row) - tap * p.remap_C;
                    const int      kh = (tap * 11) >> 5, kw = tap - 3 * kh;      // tap / 3 for tap < 12
                    voff[d] = static_cast<uint32_t>(static_cast<int64_t>(kw * p.remap_C + c) * p.Kb + (kh - 1) * p.remap_shift
                                                    + gchunk[d & 1] + kDmaBias - imm[d]);
                }
            }
    }
    // the panel base as two scalar registers (the wavefront index is uniform, so is the choice of panel)
    const uint64_t gbits = reinterpret_cast<uint64_t>(gbase) - kDmaBias;
    const uint8_t* sbase0 = reinterpret_cast<const uint8_t*>(uniform64(static_cast<int64_t>(gbits)));
    // All DPW instructions of a wavefront share one LDS base (M0): instruction d reaches its 1 KB
    // slot through the instruction's immediate offset (d - DPW/2) KB.  Rewriting M0 between direct
    // loads would stall the wavefront until the previous load has left the issue queue
    // (measured: +20 % GEMM throughput without it).
    // CONVTN: pixels per K tile, and how far (h, w) of a stage row move from one K tile to the next
    constexpr int tnc_KR = kRowBytes / ESZ;
    const int     tnc_dr = CONVTN ? tnc_KR % p.conv_W : 0, tnc_hq = CONVTN ? (tnc_KR / p.conv_W) % p.conv_H : 0;
    // CONVA: the K axis position of the lane's two chunks, how it moves from one K tile to the next, and the extra distance
    // of a step in kh
    ConvTap        conv_t;
    const uint32_t conv_cb = CONVA ? static_cast<uint32_t>(p.conv_Cb) : 1u;
    const uint32_t conv_q = kRowBytes / conv_cb, conv_r = kRowBytes % conv_cb;
    const uint32_t conv_kh_step = CONVA ? static_cast<uint32_t>((p.conv_W - 3) * p.conv_Cb) : 0u;       // (modulo 2^32 for W < 3)
    if constexpr(CONVA)
#pragma unroll
        for(int par = 0; par < 2; ++par)
        {
            conv_t.koff[par] = static_cast<uint32_t>(gchunk[par]);
            conv_t.tap[par]  = conv_t.koff[par] / conv_cb;
            conv_t.c0[par]   = conv_t.koff[par] % conv_cb;
            conv_t.koff[par] -= (static_cast<uint32_t>(p.conv_W) + 1u) * conv_cb;
        }
    const int64_t tn_ld = TN ? uniform64(is_a ? p.M : p.N) : 0;      // operand row length in elements
    // TN: stage row of the lane in load slot 0, rows from slot to slot, and the contraction rows of a partial last K tile
    constexpr int tn_rps = TN ? 1024 / (BM * ESZ) : 0;
    auto          tn_first_row = [&]() { return ((lwave * DPW - (is_a ? 0 : BM / 8)) * 1024 + lane_again() * 16) / (BM * ESZ); };
    const int     tn_tail_rows = TN ? static_cast<int>(p.Kb % kRowBytes) / ESZ : 0;
    auto dma = [&](int stage, int kt) {
        const int64_t  kb    = static_cast<int64_t>(kt) * kRowBytes;
        uint8_t*       lbase = lds + stage * STAGE_BYTES + lwave * (DPW * 1024) + (dma_group<DPW>() / 2) * 1024;
        if constexpr(CONVTN)
            if(!is_a)
            {   // (requested for consecutive K tiles only, starting at kt_begin: hw is advanced by every call)
                if(kt == tail_kt)      // (the last request) stage rows without a pixel read zeros
                {
                    const int row0 = tn_first_row();
#pragma unroll
                    for(int d = 0; d < DPW; ++d)
                        if(row0 + d * tn_rps >= tn_tail_rows) tnc_code[d / 4] &= ~(0xFFu << (8 * (d % 4)));
                }
                conv_tn_sequence<DPW>(std::make_integer_sequence<int, DPW>{}, p.B, reinterpret_cast<const uint8_t*>(&g_zero_chunk),
                                      static_cast<uint32_t>(kt) * static_cast<uint32_t>(tnc_KR) * static_cast<uint32_t>(p.conv_Cb), voff, tnc_code, hw, p.conv_H, p.conv_W,
                                      tnc_dr, tnc_hq, lbase);
                return;
            }
        if constexpr(CONVA)
            if(is_a)
            {
                // (for consecutive K tiles, starting at 0)  Source of a chunk: pixel + (kh - 1) rows + (kw - 1) pixels + c0
                // = pixel - (W + 1) pixels + K offset + kh (W - 3) pixels, since the K offset = (3 kh + kw) pixels + c0;
                // koff carries the constant part.
                uint32_t delta[2];
#pragma unroll
                for(int par = 0; par < 2; ++par)
                    delta[par] = conv_t.koff[par] + (conv_t.tap[par] >= 3 ? conv_kh_step : 0u) + (conv_t.tap[par] >= 6 ? conv_kh_step : 0u);
                conv_sequence<DPW>(std::make_integer_sequence<int, DPW>{}, p.A, reinterpret_cast<const uint8_t*>(&g_zero_chunk),
                                   voff, hw, conv_t, delta, lbase);
#pragma unroll
                for(int par = 0; par < 2; ++par)
                {
                    conv_t.koff[par] += kRowBytes;
                    conv_t.tap[par]  += conv_q;
                    conv_t.c0[par]   += conv_r;
                    if(conv_t.c0[par] >= static_cast<uint32_t>(p.conv_Cb)) { conv_t.c0[par] -= static_cast<uint32_t>(p.conv_Cb); ++conv_t.tap[par]; }
                }
                return;
            }
        const uint8_t* sb    = TN ? sbase0 + kb * tn_ld : sbase0 + kb;      // TN: 128 operand rows further
        asm volatile("" : "+s"(sb));      // keep base + K offset a scalar pair: the lane offsets stay loop-invariant 32-bit values
        if(TN && kt == tail_kt)
            dma_sequence_short<DPW, tn_rps>(std::make_integer_sequence<int, DPW>{}, sb, voff, tn_first_row(), tn_tail_rows,
                                            static_cast<uint32_t>(tn_ld * ESZ), lbase);
        else if(!TN && kt == tail_kt)
            dma_sequence_tail<DPW>(std::make_integer_sequence<int, DPW>{}, sb, voff, gchunk, kb, p.Kb, lbase);
        else
            dma_sequence<DPW>(std::make_integer_sequence<int, DPW>{}, sb, voff, lbase);
    };
    // Waits for this wavefront's direct loads and for its outstanding fragment reads (the barrier hands the
    // stage they read to the next direct load, and the compiler does not see those reads), zero-fills its
    // out-of-K chunks, then joins the block.
    auto zero_tail = [&](int stage, int kt) {
        if((!CONVTN || is_a) && kt == tail_kt)
        {
            const int64_t kb   = static_cast<int64_t>(kt) * kRowBytes;
            const int     l    = lane_again(), row0 = TN ? ((lwave * DPW - (is_a ? 0 : BM / 8)) * 1024 + l * 16) / (BM * ESZ) : 0;
#pragma unroll
            for(int d = 0; d < DPW; ++d)
                if(TN ? row0 + d * tn_rps >= tn_tail_rows : kb + gchunk[d & 1] >= p.Kb)
                    *reinterpret_cast<uint4*>(lds + stage * STAGE_BYTES + (lwave * DPW + d) * 1024 + l * 16)
                        = make_uint4(0, 0, 0, 0);
        }
    };
    auto land = [&](int stage, int kt) {
        // direct loads retire in order: tile kt has landed when at most the loads of the tiles requested behind it
        // (up to ST - 2 of them; fewer at the end of K) are outstanding
        wait_tiles<DPW, ST - 2>(kt_end - 1 - kt);
        zero_tail(stage, kt);
        wg_barrier();
    };
    float*     colp  = reinterpret_cast<float*>(lds + ST * STAGE_BYTES);       // [2][BN]: scale, bias
    const bool any_k = kt_begin < kt_end;
    // Column parameters and as many K tiles as there are stages; the wait for tile 0 (up to ST - 1 tiles are requested behind it).
    // Nothing in front of the K loop waits for global memory except that wait (a load into a register here would make the
    // compiler drain the queue before its use).
    auto request_first = [&]() {
        if(WHOLE && lwave < BN / 64)
        {
            const int64_t c = n0 + lwave * 64 + lane, col = c < p.N ? c : p.N - 1;       // columns past N: any valid one, never stored
            if(p.col_scale) column_param_issue(p.col_scale + col, lds + ST * STAGE_BYTES + lwave * 256);
            if(p.col_bias) column_param_issue(p.col_bias + col, lds + ST * STAGE_BYTES + BN * 4 + lwave * 256);
        }
        if constexpr(TOKEN)
            if(lwave < BM / 64)
            {
                const int64_t r = m0 + lwave * 64 + lane, row = r < p.M ? r : p.M - 1;
                if(p.row_scale) column_param_issue(p.row_scale + row, lds + ST * STAGE_BYTES + kColumnBytes<BN> + lwave * 256);
            }
#pragma unroll
        for(int t = 0; t < ST; ++t)
            if(kt_begin + t < kt_end) dma(t, kt_begin + t);
    };
    auto await_first = [&]() {
        wait_tiles<DPW, ST - 1>(kt_end - 1 - kt_begin);
        zero_tail(0, kt_begin);
        wg_barrier();
    };
    // Loading wavefronts of their own (NL): they meet the others at every K tile's barrier and do nothing but request, wait and
    // clear.  A direct load occupies the compute unit's vector-memory path for 16 clocks, the 32 of a 128 tile's K tile for
    // 512, and a wavefront whose loads queue there issues nothing else; with two computing wavefronts a SIMD that was twice
    // what their instructions and LDS reads took.
    if constexpr(NL > 0)
        if(wave >= WC)
        {
            request_first();
            if(!any_k)
            {
                wait_direct_loads<0>();              // the column parameters
                return;
            }
            await_first();
            int stage = 0;
            for(int kt = kt_begin; kt + 1 < kt_end; ++kt)
            {
                const int next = stage + 1 < ST ? stage + 1 : 0;
                land(next, kt + 1);
                if(kt + ST < kt_end) dma(stage, kt + ST);
                stage = next;
            }
            return;
        }

    accv_t acc[FM][FN];
#pragma unroll
    for(int i = 0; i < FM; ++i)
#pragma unroll
        for(int j = 0; j < FN; ++j)
#pragma unroll
            for(int v = 0; v < 4; ++v) acc[i][j][v] = 0;

    // Fragment reads: lane -> row lane%16 of a fragment, 16-byte chunk 4*c + lane/16 of the stage row.  The swizzle term
    // (row/2)%8 is the same for every fragment of a lane because fragments start at multiples of 16.
    const int frag_row = lane % R, kq = lane / R;
    int       roff[CH];
#pragma unroll
    for(int c = 0; c < CH; ++c) roff[c] = frag_row * kRowBytes + swizzle(frag_row, c * (8 / CH) + kq);
    const int a_base = (wm * WTM) * kRowBytes, b_base = BM * kRowBytes + (wn * WTN) * kRowBytes;

    // The fragment reads are written as instructions with hand-placed waits.  The compiler's own wait
    // insertion treats a direct global->LDS load as an access that may return through either counter, and
    // while one is in flight (always, here) every wait it places on an LDS read becomes "all LDS reads
    // done", including the reads just issued for a later chunk: the wavefront would then sit out a full LDS
    // latency twice per K tile.  LDS reads of a wavefront return in order, so "at most n outstanding" says which have arrived.
    constexpr bool ROLL = FM > 4;                    // one set of registers for the rows' fragments (below)
    v4i32          af[ROLL ? 1 : 2][FM], bf[2][FN];
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)lds));
    // TN: lane (q = lane/16, s = lane%16) receives row s of a fragment.
    // int8: it supplies the 8-byte half s%2 of chunk (first chunk of the sub-tile + f) of contraction row
    // 64 c + 16 q + 8 r + s/2 (r = 0, 1: the two reads of a fragment) and receives contraction indices
    // 64 c + 16 q + 8 r + 0..7.  binary16: the 8-byte half s%2 of chunk (first chunk + 2f + (s%4)/2) of
    // contraction row 32 c + 8 q + 4 r + s/4; it receives contraction indices 32 c + 8 q + 4 r + 0..3.
    // A sub-tile's first chunk is a multiple of its fragments' chunks, so every fragment lies at one lane's address with a
    // wavefront-uniform chunk XORed in, which leaves stage bases (multiples of 1024) alone: one register for all of them.
    uint32_t       tn_lane = 0u;
    const uint32_t tn_a = static_cast<uint32_t>(wm * WTM * ESZ), tn_b = static_cast<uint32_t>(wn * WTN * ESZ);
    if constexpr(TN)
    {
        constexpr int RB = BM * ESZ;
        static_assert((WTM / 16) % FM == 0 && (WTN / 16) % FN == 0 && RB <= 1024, "fragments by XOR");
        const int s16 = lane & 15;
        const int prow = ESZ == 1 ? 16 * kq + s16 / 2 : 8 * kq + s16 / 4;       // + c and r steps through the immediate
        const int lch  = ESZ == 1 ? 0 : (s16 & 3) / 2;                           // chunk inside the fragment's columns
        tn_lane = static_cast<uint32_t>(prow * RB + ((lch ^ tn_swizzle<ESZ, RB>(prow)) * 16) + 8 * (s16 & 1));
    }
    // fragment f of chunk c of the stage at LDS address sb
    auto read_tn = [&](v4i32& d, uint32_t addr, auto ct) {
        constexpr int c = decltype(ct)::value;
        v2u32 lo, hi;
        frag_read_tr<ESZ, c * 64 * BM>(lo, addr);
        frag_read_tr<ESZ, c * 64 * BM + 8 * BM>(hi, addr);
        d = v4i32{static_cast<int>(lo.x), static_cast<int>(lo.y), static_cast<int>(hi.x), static_cast<int>(hi.y)};
    };
    auto read_a = [&](auto ft, auto ct, uint32_t sb) {
        constexpr int f = decltype(ft)::value, c = decltype(ct)::value;
        if constexpr(TN) read_tn(af[ROLL ? 0 : c][f], (sb + tn_lane) ^ (tn_a + static_cast<uint32_t>(f * ESZ * 16)), ct);
        else             frag_read<f * R * kRowBytes>(af[ROLL ? 0 : c][f], sb + static_cast<uint32_t>(a_base + roff[c]));
    };
    auto read_b = [&](auto ft, auto ct, uint32_t sb) {
        constexpr int f = decltype(ft)::value, c = decltype(ct)::value;
        if constexpr(TN) read_tn(bf[c][f], (sb + 128 * BM + tn_lane) ^ (tn_b + static_cast<uint32_t>(f * ESZ * 16)), ct);
        else             frag_read<f * R * kRowBytes>(bf[c][f], sb + static_cast<uint32_t>(b_base + roff[c]));
    };
    constexpr int kPer = TN ? 2 : 1;                 // LDS instructions per fragment
    // row fragment f of chunk c: FN matrix instructions; every other row walks its columns backwards, so that the B operand
    // stays from one row to the next (instructions on the same operands draw less power: +2 % of the rate above)
    auto mma = [&](auto ft, auto ct) {
        constexpr int f = decltype(ft)::value, c = decltype(ct)::value;
        __builtin_amdgcn_sched_barrier(0);           // fences: the matrix instructions stay behind the wait in front of them
#pragma unroll
        for(int jj = 0; jj < FN; ++jj)
        {
            const int j = f % 2 ? FN - 1 - jj : jj;
            acc[f][j]   = TR::mfma(bf[c][j], af[ROLL ? 0 : c][f], acc[f][j]);
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    // K pipeline.  A tile has two 64-byte K chunks.
    // Wavefronts of few fragments hold those of both chunks: behind the matrix instructions of chunk 0 the wavefront joins the
    // barrier that publishes the next stage (every wavefront's reads of the current one have returned by then), requests the
    // direct load of the tile after next into the stage just drained (some wavefronts: later in the tile, see below), reads
    // chunk 0 of the next tile, issues chunk 1, whose operands are already in registers, and reads chunk 1 of the next tile: barrier release, LDS latency and a whole K tile of memory latency hide behind matrix work.
    // With four rows (128 tile) the reads go out between the rows' instructions, and the load behind row 0: 4096x768x3072 in three
    // stages int8 16.4 -> 15.7 us, binary16 28.0 -> 26.4, against all of them at the chunk's end; the 64 tile, of which a unit holds
    // several, gains nothing from that (its convolution's weight gradient 32.2 -> 33.2).
    // The 256 tile's wavefronts have no registers for both chunks.  A row's fragment is used by FN instructions in a row and
    // never again, so its registers are requested anew, for the next chunk, right behind them; the columns'
    // fragments, which every row uses, have two sets, and those of the next chunk are requested behind the first rows.  In chunk 1 no
    // row in front of the middle requests anything: there the barrier and the load's request follow, then the next tile's columns
    // and first rows, and the other rows go on as before.
    // 32x32 instructions with four 32-byte chunks and two sets of fragments -> this, values N(0,1), side by side, us: 16384x1024x4096
    // int8 59.1 -> 53.0, binary16 112 -> 101, 16384x4096x1024 79.4 -> 75.1 and 132 -> 124; 8192^3 2.55 -> 2.84 POP/s and 1.28 -> 1.42
    // PFLOP/s; on zeros, i.e. at the full clock, within 2 % of the same times.  The smaller tiles are not bound by power, and gain
    // little: 128 tile, 4096x3072x768 int8 14.9 -> 15.3, binary16 24.5 -> 24.8 (256 tile 15.8 -> 15.6, 23.0 -> 22.1); 64 tile, 2048x2048x1024
    // binary16 14.4 -> 14.1, 1808x1040x784 int8 7.42 -> 7.37, 64x64x6144 in splits 8.69 -> 8.67.
    // The column scales and biases of this tile are fetched by direct loads as well, in front of the first K tile, and
    // wait in LDS behind the stages for the epilogue.
    // The direct loads of a K tile are not requested by all wavefronts at once.  A compute unit takes such an
    // instruction (1 KB) at about 64 bytes per clock, and a wavefront issues nothing else while its loads
    // queue up: with every wavefront requesting right behind the barrier, both wavefronts of every SIMD sit
    // in that queue together and the matrix pipeline idles until the unit has taken all (BM + BN) / 8 of them.
    // The upper half of the wavefronts (the second wavefront of each SIMD) therefore requests later, among the instructions of
    // chunk 1: while one wavefront of a SIMD queues loads, its sibling issues matrix instructions (launched alone: 4-10 % fewer
    // cycles per launch on the 256 and 128 tiles, int8 and binary16).  256 tile: behind the last row.  128 tile: behind the third of
    // four rows; behind the last, binary16 256x1408x768 backward 14.1 -> 14.5 us, weight gradient of a convolution 200->168 over
    // 18x47x53 83.3 -> 85.0.
    // The 64 tile has no second wavefront on a SIMD, and a K tile of its own is over in less than a load takes: a request that goes
    // out at the chunk's end holds up the next barrier.  All of its wavefronts request right behind the barrier, at the end of
    // the tile -> this, us: row-major binary16 10368x168x1568 27.4 -> 23.5, 12416x3240x192 47.1 -> 41.1, int8 2560x96x1296 9.78 ->
    // 8.60.  Operand rows that straddle the 128-byte lines double the queue (binary16 960x1024x1808 16.6 -> 17.8 with all of them
    // at once): there the upper half requests behind the first of two rows.
    const bool late_loader = wave >= WC / 2 && (FM > 2 || (!TN && p.Kb % kRowBytes != 0));
    // (scalar loads: in front of the first direct load, used by the epilogue)
    const float scale0 = *(WHOLE && p.s0 ? p.s0 : &g_one), scale1 = *(WHOLE && p.s1 ? p.s1 : &g_one);
    const float code_inv = *(WHOLE && p.codes ? p.code_inv : &g_one);
    if constexpr(NL == 0) request_first();
    // (What the K loop starts from is formed while the first loads are in flight, not behind the wait for them: 4096x3072x768 on the
    // 128 tile int8 15.3 -> 14.8 us)
    if constexpr(FM > 2 && ESZ <= 2)
    {
#pragma unroll
        for(int i = 0; i < FM; ++i)
#pragma unroll
            for(int j = 0; j < FN; ++j) asm volatile("" : "+v"(acc[i][j]));
        if constexpr(TN) asm volatile("" : "+v"(tn_lane));
        else             asm volatile("" : "+v"(roff[0]), "+v"(roff[1]));
    }
    if(any_k)
    {
        if constexpr(NL == 0) await_first();
        else                  wg_barrier();
        constexpr int H = FM / 2;
        const std::integral_constant<int, 0> c0{};
        const std::integral_constant<int, 1> c1{};
        auto read_chunk = [&](auto ct, uint32_t sb) {
            static_for<FN>([&](auto j) { read_b(j, ct, sb); });
            static_for<FM>([&](auto i) { read_a(i, ct, sb); });
        };
        // Both chunks held, four rows: the other chunk's columns and first row go out behind row 0, its other rows behind row 1.
        auto requested   = [](int i) constexpr { return i == 0 ? 0 : i == 1 ? FN + 1 : FN + FM; };      // in front of row i
        auto read_behind = [&](auto it, auto ct, uint32_t sb) {
            constexpr int i = decltype(it)::value;
            if constexpr(i == 0)
            {
                static_for<FN>([&](auto j) { read_b(j, ct, sb); });
                read_a(std::integral_constant<int, 0>{}, ct, sb);
            }
            if constexpr(i == 1)
                static_for<FM - 1>([&](auto r) { read_a(std::integral_constant<int, decltype(r)::value + 1>{}, ct, sb); });
        };
        read_chunk(c0, lds0);
        if constexpr(FM == 2) read_chunk(c1, lds0);
        int stage = 0;
        for(int kt = kt_begin; kt < kt_end; ++kt)
        {
            const bool     more = kt + 1 < kt_end;
            const int      next = stage + 1 < ST ? stage + 1 : 0;
            const uint32_t sb   = lds0 + static_cast<uint32_t>(stage * STAGE_BYTES);
            // without a next tile the reads behind the barrier fetch the current stage again: in bounds, unused
            const uint32_t nb      = lds0 + static_cast<uint32_t>((more ? next : stage) * STAGE_BYTES);
            const bool     request = NL == 0 && kt + ST < kt_end;
            if constexpr(ROLL)
            {
                static_for<FM>([&](auto it) {
                    // Younger than this row's fragment: those of the FM - 1 other rows and of min(2 i, FN) columns (and younger
                    // than the last column's, at row 0: FM - 1 rows)
                    constexpr int i = decltype(it)::value;
                    wait_lds<kPer * (FM - 1 + (2 * i < FN ? 2 * i : FN))>();
                    mma(it, c0);
                    if constexpr(2 * i < FN)
                    {
                        read_b(std::integral_constant<int, 2 * i>{}, c1, sb);
                        read_b(std::integral_constant<int, 2 * i + 1>{}, c1, sb);
                    }
                    read_a(it, c1, sb);
                });
                static_for<H>([&](auto it) {
                    wait_lds<kPer * (FM - 1 - decltype(it)::value)>();
                    mma(it, c1);
                });
            }
            else if constexpr(FM == 2)
            {
                wait_lds<kPer * (FM + FN)>();
                static_for<FM>([&](auto it) { mma(it, c0); });
            }
            else
                static_for<FM>([&](auto it) {
                    constexpr int i = decltype(it)::value;
                    wait_lds<kPer * (FM - 1 - i + requested(i))>();
                    mma(it, c0);
                    read_behind(it, c1, sb);
                });
            wait_lds<0>();
            if(more)
            {
                if constexpr(NL > 0) wg_barrier();
                else                 land(next, kt + 1);
            }
            if((ROLL || FM == 2) && request && !late_loader) dma(stage, kt + ST);
            if constexpr(ROLL)
            {
                static_for<FN>([&](auto j) { read_b(j, c0, nb); });
                static_for<H>([&](auto i) { read_a(i, c0, nb); });
                static_for<FM - H>([&](auto it) {
                    const std::integral_constant<int, H + decltype(it)::value> row{};
                    mma(row, c1);
                    read_a(row, c0, nb);
                });
            }
            else if constexpr(FM == 2)
            {
                read_chunk(c0, nb);
                mma(c0, c1);
                if(request && late_loader) dma(stage, kt + ST);
                mma(c1, c1);
                read_chunk(c1, nb);
            }
            else
                static_for<FM>([&](auto it) {
                    mma(it, c1);
                    read_behind(it, c0, nb);
                    if constexpr(decltype(it)::value == 0)
                        if(request && !late_loader) dma(stage, kt + ST);
                    if constexpr(decltype(it)::value == 2)
                        if(request && late_loader) dma(stage, kt + ST);
                });
            if(ROLL && request && late_loader) dma(stage, kt + ST);
            stage = next;
        }
    }
    // The unused reads of the last trip land before their registers are reused: naming the registers behind the wait
    // keeps the compiler from handing them out in front of it.
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if(any_k)
    {
#pragma unroll
        for(int f = 0; f < FM; ++f) asm volatile("" : "+v"(af[0][f]), "+v"(af[ROLL ? 0 : 1][f]));
#pragma unroll
        for(int f = 0; f < FN; ++f) asm volatile("" : "+v"(bf[0][f]), "+v"(bf[1][f]));
    }
    else if(NL == 0)
        wait_direct_loads<0>();                  // the column parameters
    const float    alpha     = scale0 * scale1;
    // (by the wavefront that publishes: loads of the word stand in line with the atomics on it, and with some hundred workgroups that end
    // together the line is what they wait for.  Every wavefront -> one, int8 912x3008x752 28.5 -> 20.4 us, 12896x576x368 24.4 -> 17.3)
    const uint32_t amax_seen = (WHOLE && p.amax_bits && wave == 0) ? __hip_atomic_load(p.amax_bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;

    constexpr int STG = 2 * STAGE_BYTES / (WGM * WGN);
    if(MIXED ? raw : SPLIT) store_tile<TR, BM, BN, WGM, WGN, STG, true, TOKEN>(p, acc, lds, colp, m0, n0, split, alpha, code_inv, amax_seen);
    else if constexpr(WHOLE) store_tile<TR, BM, BN, WGM, WGN, STG, false, TOKEN>(p, acc, lds, colp, m0, n0, split, alpha, code_inv, amax_seen);
}

// `lin` is the workgroup's index among the `splits` x tiles workgroups of the problem.
template <typename TR, int BM, int BN, int WGM, int WGN, int ST, int NL, bool SPLIT, bool CONV, bool TN, bool MIXED = false>
__device__ __forceinline__ void gemm_tile(const GemmKernelArgs& p, int lin, int splits, bool raw = SPLIT)
{
    int split, tm, tn;
    item_of_block(lin, p.tiles_m, p.tiles_n, SPLIT ? splits : 1, p.group_m, split, tm, tn);
    gemm_tile_at<TR, BM, BN, WGM, WGN, ST, NL, SPLIT, CONV, TN, MIXED>(p, split, tm, tn, raw);
}

}  // namespace

}  // namespace qsync
