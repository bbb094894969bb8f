// Softmax cross entropy of rows against a large set of classes, and its
// gradients, without the logits:
//
//   z_iv = h_i . w_v,  lse_i = log sum_v exp z_iv,  loss_i = lse_i - z_i,y(i)
//   p_iv = exp(z_iv - lse_i) - [v = y(i)]
//   dh_i = (1/N) sum_v p_iv w_v,   dw_v = (1/N) sum_i p_iv h_i
//
// The classes are taken in pieces.  A first pass over the pieces multiplies and
// keeps, per row and tile of classes, the largest logit and the sum of
// exponentials (the logits stay in registers); one launch joins them to lse, which
// is kept as two numbers, the largest logit and the log of the sum: their sum in
// fp32 would be off by a step of the logits' size, and every p of the row by as
// much of itself (900 equal logits of -1e30: p = 1 instead of 1 / 900).  A
// second pass multiplies a piece again, writes its p, in the matrix cores' 16-bit
// type, to a buffer the size of a piece, and two products take the piece's dw and
// its part of dh from that buffer.
//
// Operands are packed first: chunk-major, 16-byte chunks of 8 consecutive
// columns, the chunks of one column group side by side for all rows
// (x[c / 8][row][c % 8]), padded with zeros to whole tiles.  This one layout
// serves as an operand whose columns are summed over (a fragment is 8 columns of
// a row: one chunk) and as one whose rows are (the transposing LDS reads
// of gfx950 take 4 rows of 16 columns); copies to LDS are contiguous and need
// no bounds.  fp32 operands are packed as three bf16 planes and multiplied with
// the six part products of bf16split.hpp; bf16 ones as they are.
//
// The products are one tile function: M (MFMA rows) is the class of the logits and
// the feature of the gradients, N (MFMA columns) the row of h, or the class for dw.
// Narrow bf16 rows have a logit kernel of their own (k_xent_strip), few rows
// two, for the statistics and for the gradients (k_xent_score, k_xent_few).
//
// Operations: 2 m V d for each of the two logit passes, dh and dw: 8 m V d, where
// kept logits would take 6.  8,192 x 65,536 x 1,024 bf16: 4.05 to 4.35 ms on one card and another, 1,010 to
// 1,085 TFLOP/s of the 1,307 that a library product of 8,192^3 reaches; 4,093 x 169,000 x 256 bf16 1.51 to 1.58 ms
// (895 to 940); 1,024 x 169,000 x 256 fp32 2.02 to 2.15 ms (990 to 1,050 of bf16 part products).
#include <algorithm>
#include <cmath>

#include "bf16split.hpp"
#include "common.hpp"
#include "dma.hpp"

namespace gnnav {

namespace {

typedef float f32x16x __attribute__((ext_vector_type(16)));
typedef float f32x4x __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4x __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2x __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kPiece = 256;    // pieces of the classes are multiples of this, a whole number of any product's tiles
constexpr float kLog2e = 1.44269504088896340736f;
// exp2(x log2e - r log2e) as one multiply-add errs by the rounding of r log2e: below this 2^-17.5 of the result at most
// (with the log of a sum of up to 2^31 beside r).  Past it the difference is taken first, by each row for itself: what
// other rows hold changes no bit of a row's.
constexpr float kFmaRange = 128.f;

// Two values rounded to bf16, nearest even.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// Two groups of 4 values (as bf16 pairs) of a lane, of its row's classes c .. c + 3 and c + 8 .. c + 11, with those of
// lane ^ 32, c + 4 .. and c + 12 ..: the chunk of 8 from c for the lower lanes, from c + 8 for the upper ones.
__device__ __forceinline__ u32x4x join_chunk(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
    const auto lo = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
    return u32x4x{lo[0], hi[0], lo[1], hi[1]};
}

// What a row does: counted rows carry their largest logit and the log of their sum, the others 0 and +inf (a sum of at
// most 2^31 ones has no such log).
__device__ __forceinline__ bool row_counts(float2 lse) { return lse.y < INFINITY || lse.y != lse.y; }

}  // namespace

// ------------------------------------------------------------------ packing
// rows x d (row-major, 16-byte aligned rows) -> PL planes of chunks
// [chunk][R rows], zeros past rows and d, and in rows whose label is `ignore` or
// outside [0, n_classes) (labels nullable).  One workgroup: 64 rows x 64 columns
// through LDS.  A launch takes two matrices (the first has `blocks` workgroups of rows).
// Bound by memory: 4,096 + 84,736 bf16 rows of 256 columns 18 us, 5.0 TB/s.
struct PackArgs {
    const void *src;
    int64_t ld, rows, R;
    const int32_t *labels;
    u32x4x *out;
};
template <bool BF>
__global__ void __launch_bounds__(256) k_xent_pack(const PackArgs first, const PackArgs second, int32_t blocks, int64_t d,
                                                   int32_t ignore, int64_t n_classes, int64_t chunks) {
    const bool one = (int32_t)blockIdx.x < blocks;
    const void *__restrict__ src = one ? first.src : second.src;
    const int64_t ld = one ? first.ld : second.ld, rows = one ? first.rows : second.rows, R = one ? first.R : second.R;
    const int32_t *__restrict__ labels = one ? first.labels : second.labels;
    u32x4x *__restrict__ out = one ? first.out : second.out;
    constexpr int PL = BF ? 1 : 3;
    __shared__ u32x4x tile[PL][8][65];
    const int tid = threadIdx.x;
    const int64_t r0 = (int64_t)(blockIdx.x - (one ? 0 : blocks)) * 64, c0 = (int64_t)blockIdx.y * 8;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int lr = tid / 8 + 32 * k, lc = tid % 8;
        const int64_t r = r0 + lr, col = (c0 + lc) * 8;
        bool live = r < rows && col < d;
        if (live && labels) {
            const int32_t y = labels[r];
            live = y != ignore && y >= 0 && y < n_classes;
        }
        if constexpr (BF) {
            u32x4x x = {0, 0, 0, 0};
            if (live) {
                x = *(const u32x4x *)((const uint16_t *)src + r * ld + col);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (col + 2 * q + 1 >= d) x[q] &= 0xffffu;
                    if (col + 2 * q >= d) x[q] = 0;
                }
            }
            tile[0][lc][lr] = x;
        } else {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.f;
            if (live) {
                const float *p = (const float *)src + r * ld + col;
                const f32x4x a = *(const f32x4x *)p;
                f32x4x b = {0.f, 0.f, 0.f, 0.f};
                if (col + 4 < d) b = *(const f32x4x *)(p + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = col + e < d ? a[e] : 0.f;
                    x[4 + e] = col + 4 + e < d ? b[e] : 0.f;
                }
            }
            bf16x8 p1, p2, p3;
            split3(x, p1, p2, p3);
            tile[0][lc][lr] = __builtin_bit_cast(u32x4x, p1);
            tile[PL - 2][lc][lr] = __builtin_bit_cast(u32x4x, p2);
            tile[PL - 1][lc][lr] = __builtin_bit_cast(u32x4x, p3);
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2 * PL; ++k) {
        const int lc = (tid / 64) + 4 * (k & 1), lr = tid % 64, p = k >> 1;
        if (c0 + lc < chunks && r0 + lr < R) out[(p * chunks + c0 + lc) * R + r0 + lr] = tile[p][lc][lr];
    }
}

// ------------------------------------------------------------------ products
enum { kStats, kProb, kDh, kDw };

struct XentArgs {
    const u32x4x *A, *B;       // packed operands
    int64_t a_rows, b_rows;    // rows of their chunks
    int64_t a_plane, b_plane;  // chunks of a plane
    int64_t k;                 // summed length, a multiple of the step
    int32_t m_tiles, n_tiles, splits;
    int32_t split_steps;       // kDh: steps of one split; k_xent_strip: tiles of a strip
    // kStats, kProb
    int64_t v0, n_classes;     // first class of the piece, classes in all
    int64_t rows;              // packed rows of h
    const int32_t *labels;
    int64_t m;                 // rows of h
    float2 *stats;             // [1 + tile or strip of the piece's classes][rows]; the first: of earlier pieces (k_xent_score: nullable)
    float *label_logit;        // [rows]
    const float2 *lse;         // [rows]: the largest logit, the log of the sum of exponentials less it
    u32x4x *p;                 // planes [class chunk][rows]
    int64_t p_plane;
    // kDh
    f32x4x *part;
    int64_t split_stride;      // float4s of a split's parts
    bool first;
    // kDw
    void *dw;
    int64_t ld_dw, d;
    float *inv_count;
    bool dw_bf16;
    // the mean loss, taken by a workgroup of its own of the first kProb launch (-1: none)
    int32_t loss_block;
    const float *losses;
    int32_t ignore;
    float *loss;
    // few rows: the logits of four classes at a time, [class / 4][few] (nullable)
    f32x4x *z;
    int32_t few;               // rows of z, a power of two of at most 64
};

// Wave grid WGM x WGN, each wavefront WMF x WNF MFMA blocks of 32 x 32; BK summed
// elements per stage, ST stages in LDS.
template <int PL, int WMF, int WNF, int WGM, int WGN>
struct Tile {
    static constexpr int BK = PL == 1 ? 32 : 16;
    static constexpr int NW = WGM * WGN, BM = 32 * WMF * WGM, BN = 32 * WNF * WGN;
    static constexpr int APC = BM * BK / 8, BPC = BN * BK / 8;   // chunks of a plane of a stage
    static constexpr int STAGE = PL * (APC + BPC);
    static constexpr int ST = 3, LDS = ST * STAGE;   // stages
    static_assert(APC % 64 == 0 && BPC % 64 == 0, "whole wavefront copies");
};

// Tile of workgroup `id` of those of one product.  Workgroups go to the eight
// XCDs in turn; each XCD gets a contiguous run of the tiles, in groups of
// kGroup along M, so that the tiles it works on together share operands in its L2.
constexpr int kGroup = 8;
__device__ __forceinline__ bool tile_of(const XentArgs &a, int32_t id, int32_t &split, int32_t &mt, int32_t &nt) {
    const int32_t plane = a.m_tiles * a.n_tiles, total = plane * a.splits;
    const int32_t per = total / 8, extra = total % 8, x = id & 7, k = id >> 3;
    if (k >= per + (x < extra ? 1 : 0)) return false;
    const int32_t lin = x * per + std::min(x, extra) + k;
    split = lin / plane;
    const int32_t t = lin - split * plane, g = t / (kGroup * a.n_tiles), r = t - g * (kGroup * a.n_tiles);
    const int32_t wide = std::min(kGroup, a.m_tiles - g * kGroup);
    nt = r / wide;
    mt = g * kGroup + r - nt * wide;
    return true;
}

// Block (i, j), register r of a lane of a product: M index 32 i + 8 (r / 4) + 4 (lane / 32) + r % 4, N index 32 j + lane % 32.

// Less the lane's 4 (lane / 32): the same for every lane, so that what is compared with it is kept per lane and not these.
__device__ __forceinline__ constexpr int place(int i, int r) { return 32 * i + 8 * (r / 4) + r % 4; }

// The place of a row's label among the 32 WMF classes from mw of the piece on, below -4 if it is none of them.
template <int WMF>
__device__ __forceinline__ int label_place(const XentArgs &a, int64_t n, int64_t mw, int h) {
    const int64_t y = (n < a.m ? a.labels[n] : -1) - (a.v0 + mw);
    return y >= 0 && y < 32 * WMF ? (int)y - 4 * h : -64;
}

// The place past the last class, of 32 WMF ones from mw of the piece on.
template <int WMF>
__device__ __forceinline__ int live_classes(const XentArgs &a, int64_t mw, int h) {
    return (int)std::max<int64_t>(std::min<int64_t>(a.n_classes - a.v0 - mw, 32 * WMF), 0) - 4 * h;
}

// Largest logit and sum of exponentials of the workgroup's classes, for each of its rows.
template <int PL, int WMF, int WNF, int WGM, int WGN>
__device__ __forceinline__ void stats_of(const XentArgs &a, f32x16x (&acc)[WMF][WNF], int64_t mt, int64_t n0, float2 *red) {
    constexpr int BM = 32 * WMF * WGM, BN = 32 * WNF * WGN;
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wid / WGN, wn = wid % WGN, h = lane >> 5, lr = lane & 31;
    const int64_t m0 = mt * BM, mw = m0 + wm * (32 * WMF), nw = n0 + wn * (32 * WNF);
    const bool tail = a.v0 + m0 + BM > a.n_classes;
    const int live = live_classes<WMF>(a, mw, h);
    float2 mine[WNF];
#pragma unroll
    for (int j = 0; j < WNF; ++j) {
        const int64_t n = nw + 32 * j + lr;
        const int y = label_place<WMF>(a, n, mw, h);
        if (tail)
#pragma unroll
            for (int i = 0; i < WMF; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (place(i, r) >= live) acc[i][j][r] = -INFINITY;
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < WMF; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, acc[i][j][r]);
        if (y > -64) {
#pragma unroll
            for (int i = 0; i < WMF; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (y == place(i, r)) a.label_logit[n] = acc[i][j][r];
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
        // a row whose classes here are all -inf has the sum 0: any finite reference does
        const float ref = mx == -INFINITY ? 0.f : mx;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < WMF; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                // (the difference first: of huge logits a product's rounding alone would overflow)
                if constexpr (PL == 1) s += __builtin_amdgcn_exp2f((acc[i][j][r] - ref) * kLog2e);
                else s += expf(acc[i][j][r] - ref);
            }
        s += __shfl_xor(s, 32, kWave);
        mine[j] = make_float2(mx, s);
    }
#pragma unroll
    for (int j = 0; j < WNF; ++j)
        if (h == 0) red[wm * BN + wn * (32 * WNF) + 32 * j + lr] = mine[j];
    __syncthreads();
    for (int c = tid; c < BN; c += 64 * WGM * WGN) {
        float mx = red[c].x;
#pragma unroll
        for (int w = 1; w < WGM; ++w) mx = fmaxf(mx, red[w * BN + c].x);
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < WGM; ++w) {
            const float2 o = red[w * BN + c];
            s += o.x == -INFINITY ? o.y : o.y * expf(o.x - mx);
        }
        a.stats[(1 + mt) * a.rows + n0 + c] = make_float2(mx, s);
    }
}

// One tile of a product, from packed operands by way of LDS, and what becomes of it.  Bound by the matrix cores at the clock
// that their power leaves (the same launch on zeros is 1.3 times as fast; 1.4 to 2.0 GHz by the counters, where the
// kernels that wait for memory run at 2.4): 128 x 128 x 1,024 logit tiles 1,035 TFLOP/s, 256 x 256 gradient tiles 1,100 to
// 1,120 of 1,024 columns and 880 to 1,020 of 256, a library product of the larger shapes 1,150 to 1,300.  Fragments that
// are read and copies that are issued in one burst behind the barrier: 10% slower; higher priority for the
// products, a fourth stage, 128 x 128 blocks per wavefront, groups of 4 or 16 tiles: nothing or slower.
// AT, BT: the operand's rows are summed over.
template <int PL, int WMF, int WNF, int WGM, int WGN, bool AT, bool BT, int EPI>
__device__ __forceinline__ void xent_tile(const XentArgs &a, int32_t id, u32x4x *S, float2 *red) {
    using C = Tile<PL, WMF, WNF, WGM, WGN>;
    constexpr int BK = C::BK, ST = C::ST, NW = C::NW, BM = C::BM, BN = C::BN, APC = C::APC, BPC = C::BPC;
    constexpr int STAGE = C::STAGE, INSTR = STAGE / 64, IN = (INSTR + NW - 1) / NW;
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wid / WGN, wn = wid % WGN, h = lane >> 5, lr = lane & 31;
    int32_t split, mt, nt;
    if (!tile_of(a, id, split, mt, nt)) return;
    const int64_t m0 = (int64_t)mt * BM, n0 = (int64_t)nt * BN;
    const int32_t all_steps = (int32_t)(a.k / BK);
    int32_t s0 = 0, T = all_steps;
    if constexpr (EPI == kDh) {
        s0 = split * a.split_steps;
        T = std::min(a.split_steps, all_steps - s0);
    }

    // this wavefront's copies of a stage: source of the next step, its advance
    const char *src[IN];
    int64_t inc[IN];
    int dst[IN];
#pragma unroll
    for (int u = 0; u < IN; ++u) {
        const int q = std::min(wid * IN + u, INSTR - 1);   // the last wavefront may repeat the last copy
        const int slot = q * 64;
        const bool isB = slot >= PL * APC;
        const int rel = slot - (isB ? PL * APC : 0), pc = isB ? BPC : APC;
        const int plane = rel / pc, s = rel % pc + lane;
        const u32x4x *base = (isB ? a.B + plane * a.b_plane : a.A + plane * a.a_plane);
        const int64_t R = isB ? a.b_rows : a.a_rows, x0 = isB ? n0 : m0;
        const bool tr = isB ? BT : AT;
        if (tr) {
            const int mc = s / BK, kk = (s % BK) ^ ((mc & 3) * 4);
            src[u] = (const char *)(base + (x0 / 8 + mc) * R + (int64_t)s0 * BK + kk);
            inc[u] = (int64_t)BK * 16;
        } else {
            const int tile = isB ? BN : BM, c = s / tile, r = s % tile;
            src[u] = (const char *)(base + ((int64_t)s0 * (BK / 8) + c) * R + x0 + r);
            inc[u] = (int64_t)(BK / 8) * R * 16;
        }
        dst[u] = slot;
    }
    auto issue = [&](int stage, int u) {
        dma16(src[u], &S[stage * STAGE + dst[u]]);
        src[u] += inc[u];
    };

    f32x16x acc[WMF][WNF];
#pragma unroll
    for (int i = 0; i < WMF; ++i)
#pragma unroll
        for (int j = 0; j < WNF; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    // lane parts of the fragments' LDS addresses
    const int tr_mc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), tr_k = 8 * h + ((lane & 15) >> 2);
    const int tr_swz = tr_mc * 4;   // of the lane's chunk, its number mod 4: 32 lanes read from 256 bytes of distinct banks
    auto frag = [&](const u32x4x *plane, auto tr_, int tile, int x, int kk) -> bf16x8 {
        if constexpr (decltype(tr_)::value) {
            typedef __attribute__((address_space(3))) s16x4 lds4;
            const char *p0 = (const char *)(plane + (x / 8 + tr_mc) * BK + ((kk * 16 + tr_k) ^ tr_swz)) + 8 * (lane & 1);
            const char *p1 = (const char *)(plane + (x / 8 + tr_mc) * BK + ((kk * 16 + tr_k + 4) ^ tr_swz)) + 8 * (lane & 1);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)p0);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)p1);
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(bf16x8, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
        } else {
            return __builtin_bit_cast(bf16x8, plane[(2 * kk + h) * tile + x + lr]);
        }
    };
    struct Frags {
        bf16x8 a[WMF][PL], b[WNF][PL];
    };
    // fragment k of a step: B's, then A's, as the products need them
    constexpr int NF = (WMF + WNF) * PL;
    auto read = [&](Frags &f, int stage, int kk, int k) {
        const u32x4x *sa = &S[stage * STAGE], *sb = sa + PL * APC;
        const int x = k / PL, p = k % PL;
        if (x < WNF) f.b[x][p] = frag(sb + p * BPC, std::integral_constant<bool, BT>(), BN, wn * (32 * WNF) + 32 * x, kk);
        else f.a[x - WNF][p] = frag(sa + p * APC, std::integral_constant<bool, AT>(), BM, wm * (32 * WMF) + 32 * (x - WNF), kk);
    };
    // The products of one fragment set.  Between them go, one at a time, the reads of the next set (first half) and
    // copies [c0, c1) of a stage to come (second half): in one burst behind the barrier they queue
    // up, and the wavefront's products wait with them.  Past the last stage the reads are idle ones.
    auto multiply = [&](const Frags &f, Frags &nxt, int from, int kk, bool more, int into, auto c0_, auto c1_) {
        constexpr int SLOTS = WMF * WNF, HALF = (SLOTS + 1) / 2, C0 = decltype(c0_)::value, C1 = decltype(c1_)::value;
        constexpr int REST = SLOTS > HALF ? SLOTS - HALF : 1, CUT = SLOTS > HALF ? HALF : 0;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            const int i = k / WNF, j = k % WNF;
            if constexpr (PL == 1)
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[i][0], f.b[j][0], acc[i][j], 0, 0, 0);
            else
                acc[i][j] = mfma_split6(f.a[i][0], f.a[i][PL - 2], f.a[i][PL - 1], f.b[j][0], f.b[j][PL - 2],
                                        f.b[j][PL - 1], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
            if (k < HALF)
#pragma unroll
                for (int q = NF * k / HALF; q < NF * (k + 1) / HALF; ++q) read(nxt, from, kk, q);
            if (k >= CUT && more)
#pragma unroll
                for (int q = C0 + (C1 - C0) * (k - CUT) / REST; q < C0 + (C1 - C0) * (k - CUT + 1) / REST; ++q) issue(into, q);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Makes stage t readable: its copies are done, everywhere; those of the stage after it may not be.
    auto advance = [&](int32_t t) {
        if (t + 1 < T) wait_vm<IN *(ST - 2)>();
        else wait_vm<0>();
        lds_barrier();
    };
    static_assert(ST == 3 && (BK == 16 || BK == 32), "loop below");
    auto next = [](int stage) { return stage + 1 == ST ? 0 : stage + 1; };
    // One fragment set is multiplied while the next one is read, across the barrier between two stages.  Once
    // stage t is readable, stage t + ST - 1 is copied into the one read before it, over the products up to the next barrier.
    constexpr int FIRST = BK == 32 ? IN / 2 : IN;   // copies before a stage's second fragment set is read
    constexpr std::integral_constant<int, 0> kBegin{};
    constexpr std::integral_constant<int, FIRST> kMiddle{};
    constexpr std::integral_constant<int, IN> kEnd{};
    Frags f0, f1;
    int ready = 0, fill = BK == 32 ? ST - 1 : 0;
    if (T > 0) {
#pragma unroll
        for (int k = 0; k < ST - 1; ++k)
            if (k < T)
#pragma unroll
                for (int u = 0; u < IN; ++u) issue(k, u);
        advance(0);
        if (ST - 1 < T)
#pragma unroll
            for (int u = 0; u < FIRST; ++u) issue(ST - 1, u);
#pragma unroll
        for (int q = 0; q < NF; ++q) read(f0, 0, 0, q);
    }
    for (int32_t t = 0; t < T;) {
        if constexpr (BK == 32) {
            multiply(f0, f1, ready, 1, t + ST - 1 < T, fill, kMiddle, kEnd);
            fill = next(fill);
            ready = next(ready);
            if (++t < T) advance(t);
            multiply(f1, f0, ready, 0, t + ST - 1 < T, fill, kBegin, kMiddle);
        } else {
            ready = next(ready);
            if (++t < T) advance(t);
            multiply(f0, f1, ready, 0, t + ST - 1 < T, fill, kBegin, kEnd);
            fill = next(fill);
            if (t >= T) break;
            ready = next(ready);
            if (++t < T) advance(t);
            multiply(f1, f0, ready, 0, t + ST - 1 < T, fill, kBegin, kEnd);
            fill = next(fill);
        }
    }

    const int64_t mw = m0 + wm * (32 * WMF), nw = n0 + wn * (32 * WNF);
    if constexpr (EPI == kStats) {
        stats_of<PL, WMF, WNF, WGM, WGN>(a, acc, mt, n0, red);
    } else if constexpr (EPI == kProb) {
        const bool tail = a.v0 + m0 + BM > a.n_classes;
        const int live = live_classes<WMF>(a, mw, h);
#pragma unroll
        for (int j = 0; j < WNF; ++j) {
            const int64_t n = nw + 32 * j + lr;
            const float2 lse = a.lse[n];
            const float shift = -lse.y * kLog2e;
            const int y = label_place<WMF>(a, n, mw, h);
#pragma unroll
            for (int i = 0; i < WMF; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    if constexpr (PL == 1) acc[i][j][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][r] - lse.x, kLog2e, shift));
                    else acc[i][j][r] = expf((acc[i][j][r] - lse.x) - lse.y);
                }
            if (__any(y > -64) || tail) {   // labels here, or classes that are none
#pragma unroll
                for (int i = 0; i < WMF; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        if (y == place(i, r)) acc[i][j][r] -= 1.f;
                        if (place(i, r) >= live) acc[i][j][r] = 0.f;
                    }
            }
            // a row that does not count was packed as zeros: its logits are NaN where w is infinite, and so would its p be
            const bool out = lse.y == INFINITY;
            if (__any(out))
#pragma unroll
                for (int i = 0; i < WMF; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] = out ? 0.f : acc[i][j][r];
#pragma unroll
            for (int i = 0; i < WMF; ++i) {
#pragma unroll
                for (int pl = 0; pl < PL; ++pl)
#pragma unroll
                    for (int g = 0; g < 4; g += 2) {
                        uint32_t w[2][2];
#pragma unroll
                        for (int x = 0; x < 2; ++x)
#pragma unroll
                            for (int y2 = 0; y2 < 2; ++y2) {
                                const float f0 = acc[i][j][4 * (g + x) + 2 * y2], f1 = acc[i][j][4 * (g + x) + 2 * y2 + 1];
                                if constexpr (PL == 1) {
                                    // rounded to the operands' type: at most 2^-8 of each p, as the rounding
                                    // of the gradients themselves costs
                                    w[x][y2] = bf16_pair(f0, f1);
                                } else {
                                    uint16_t q0[3], q1[3];
                                    split3_bits(f0, q0[0], q0[1], q0[2]);
                                    split3_bits(f1, q1[0], q1[1], q1[2]);
                                    w[x][y2] = (uint32_t)q0[pl] | ((uint32_t)q1[pl] << 16);
                                }
                            }
                        const int64_t chunk = (mw + 32 * i) / 8 + g + h;
                        a.p[pl * a.p_plane + chunk * a.rows + n] = join_chunk(w[0][0], w[0][1], w[1][0], w[1][1]);
                    }
            }
        }
    } else if constexpr (EPI == kDh) {
        f32x4x *to = a.part + split * a.split_stride +
                     ((int64_t)(nt * a.m_tiles + mt) * NW + wid) * (WMF * WNF * 4 * 64) + lane;
#pragma unroll
        for (int i = 0; i < WMF; ++i)
#pragma unroll
            for (int j = 0; j < WNF; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    f32x4x *at = to + ((i * WNF + j) * 4 + g) * 64;
                    f32x4x v = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                    if (!a.first) v += *at;
                    *at = v;
                }
    } else {
        const float inv = a.inv_count[0];
#pragma unroll
        for (int j = 0; j < WNF; ++j) {
            const int64_t v = a.v0 + nw + 32 * j + lr;
            if (v >= a.n_classes) continue;
#pragma unroll
            for (int i = 0; i < WMF; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int64_t c = mw + 32 * i + 8 * g + 4 * h;
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = c + e < a.d ? acc[i][j][4 * g + e] * inv : 0.f;
                    if (a.dw_bf16) {
                        if (c < (a.d + 7) / 8 * 8)
                            *(u32x2x *)((uint16_t *)a.dw + v * a.ld_dw + c) =
                                u32x2x{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
                    } else if (c < (a.d + 3) / 4 * 4) {
                        *(f32x4x *)((float *)a.dw + v * a.ld_dw + c) = f32x4x{x[0], x[1], x[2], x[3]};
                    }
                }
        }
    }
}

// The mean over the rows that count, in 64 bits and a fixed order, and its weight.  Run by one workgroup.
template <int THREADS>
__device__ __forceinline__ void xent_loss(const float *losses, int64_t m, const int32_t *labels, int32_t ignore,
                                          float *loss, float *inv_count) {
    __shared__ double part[THREADS / kWave];
    __shared__ int32_t count[THREADS / kWave];
    double s = 0.0;
    int32_t k = 0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < m; i += THREADS) {
        s += (double)losses[i];
        k += labels[i] != ignore;
    }
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) {
        s += __shfl_xor(s, o, kWave);
        k += __shfl_xor(k, o, kWave);
    }
    if (lane_id() == 0) {
        part[threadIdx.x / kWave] = s;
        count[threadIdx.x / kWave] = k;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < THREADS / kWave; ++w) {
            s += part[w];
            k += count[w];
        }
        loss[0] = k > 0 ? (float)(s / (double)k) : 0.f;
        inv_count[0] = k > 0 ? (float)(1.0 / (double)k) : 0.f;
    }
}

template <int PL, int WMF, int WNF, int WGM, int WGN, int EPI>
__global__ void __launch_bounds__(64 * WGM * WGN, 2) k_xent_logits(const XentArgs a) {
    using C = Tile<PL, WMF, WNF, WGM, WGN>;
    __shared__ u32x4x S[C::LDS];
    __shared__ float2 red[EPI == kStats ? WGM * C::BN : 1];
    if (EPI == kProb && (int32_t)blockIdx.x == a.loss_block) {
        xent_loss<64 * WGM * WGN>(a.losses, a.m, a.labels, a.ignore, a.loss, a.inv_count);
        return;
    }
    xent_tile<PL, WMF, WNF, WGM, WGN, false, false, EPI>(a, blockIdx.x, S, red);
}

// The logits of bf16 rows of at most 256 columns.  The tiles above copy 128 KB to LDS per 128 x 128 of them, and
// those copies' rate (2.8 GB in 230 us below, some 25 bytes a clock and unit) is their bound at so few columns: here a wavefront keeps its 32 WNF
// rows of h in registers for good (KS steps of 16 columns) and only the classes stream through LDS, 64 at a
// time, two buffers and one barrier a tile.  A workgroup's four wavefronts hold 128 WNF rows and take a strip
// of the piece's classes; two workgroups a unit, so that one's exponentials run beside the other's products.
// A lane's running maximum and sum stay in registers over the strip.  4,096 x 84,736 x 256: statistics 230 us
// with the tiles above, 157 to 186 so (955 to 1,130 TFLOP/s); probabilities 345, and 212 to 230 (the 694 MB of p go out at
// 3.0 to 3.3 TB/s).
constexpr int kStrip = 64;   // classes of a tile
// Tiles of a strip, at most: the running sums round once a tile, 384 2^-24 of a sum in a strip.
constexpr int64_t kStripTiles = 384;

template <int KS, int WNF, int EPI>
__global__ void __launch_bounds__(256, 2) k_xent_strip(const XentArgs a) {
    constexpr int TILE = 2 * KS * kStrip;            // chunks
    constexpr int IN = 2 * KS / 4;                   // copies of a wavefront per tile
    static_assert(KS % 2 == 0, "whole copies");
    __shared__ u32x4x S[2 * TILE];
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, lr = lane & 31;
    if (EPI == kProb && (int32_t)blockIdx.x == a.loss_block) {
        xent_loss<256>(a.losses, a.m, a.labels, a.ignore, a.loss, a.inv_count);
        return;
    }
    int32_t split, rb, strip;   // row blocks along M, strips along N
    if (!tile_of(a, blockIdx.x, split, rb, strip)) return;
    const int32_t all = (int32_t)(a.a_rows / kStrip), t0 = strip * a.split_steps, T = std::min(a.split_steps, all - t0);
    const int64_t n0 = (int64_t)rb * (128 * WNF) + wid * (32 * WNF);

    const char *src = (const char *)(a.A + (int64_t)(IN * wid) * a.a_rows + (int64_t)t0 * kStrip + lane);
    auto issue = [&](int buf, int u) { dma16(src + (int64_t)u * a.a_rows * 16, &S[buf * TILE + (IN * wid + u) * kStrip]); };
    if (T > 0)
#pragma unroll
        for (int u = 0; u < IN; ++u) issue(0, u);
    src += kStrip * 16;
    bf16x8 b[KS][WNF];
    float2 lse[WNF];
    float mx[WNF], sum[WNF];
    int32_t y[WNF];   // the label's place in the piece (negative or past it: elsewhere)
#pragma unroll
    for (int j = 0; j < WNF; ++j) {
        const int64_t n = n0 + 32 * j + lr;
#pragma unroll
        for (int k = 0; k < KS; ++k) b[k][j] = __builtin_bit_cast(bf16x8, a.B[(2 * k + h) * a.b_rows + n]);
        y[j] = n < a.m && a.labels[n] >= 0 ? a.labels[n] - (int32_t)a.v0 : -1;
        lse[j] = EPI == kProb ? a.lse[n] : make_float2(0.f, 0.f);
        mx[j] = -INFINITY;
        sum[j] = 0.f;
    }
    for (int32_t t = 0; t < T; ++t) {
        const u32x4x *tile = &S[(t & 1) * TILE];
        // this tile's copies are done; the stores of the tile before it (the newest of all) may not be
        if (EPI == kProb && t > 0) wait_vm<4 * WNF>();
        else wait_vm<0>();
        lds_barrier();
        const bool more = t + 1 < T;
        f32x16x acc[2][WNF];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < WNF; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
        bf16x8 f[2][2];
        auto read = [&](int k) {
#pragma unroll
            for (int i = 0; i < 2; ++i) f[k & 1][i] = __builtin_bit_cast(bf16x8, tile[(2 * k + h) * kStrip + 32 * i + lr]);
        };
        read(0);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            if (k + 1 < KS) read(k + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < WNF; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[k & 1][i], b[k][j], acc[i][j], 0, 0, 0);
            if (more)
#pragma unroll
                for (int u = IN * k / KS; u < IN * (k + 1) / KS; ++u) issue((t + 1) & 1, u);
            __builtin_amdgcn_sched_barrier(0);
        }
        src += kStrip * 16;
        const int64_t m0 = (int64_t)(t0 + t) * kStrip;                        // the tile's first class in the piece
        const bool tail = a.v0 + m0 + kStrip > a.n_classes;
        const int live = (int)std::max<int64_t>(std::min<int64_t>(a.n_classes - a.v0 - m0, kStrip), 0) - 4 * h;   // classes that are any
#pragma unroll
        for (int j = 0; j < WNF; ++j) {
            const int64_t n = n0 + 32 * j + lr;
            const uint32_t off = (uint32_t)y[j] - (uint32_t)m0;
            const int at = off < (uint32_t)kStrip ? (int)off - 4 * h : -64;   // (less 4 h, as the places below)
            if constexpr (EPI == kStats) {
                if (tail)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (place(i, r) >= live) acc[i][j][r] = -INFINITY;
                if (__any(at > -64))
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (at == place(i, r)) a.label_logit[n] = acc[i][j][r];
                float top = mx[j];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) top = fmaxf(top, acc[i][j][r]);
                const float ref = top == -INFINITY ? 0.f : top;
                float part[2] = {0.f, 0.f};
                const bool far = !(fabsf(ref) < kFmaRange);
                const float shift = -ref * kLog2e;
                if (__any(far)) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const float x = acc[i][j][r];
                            part[i] += __builtin_amdgcn_exp2f(far ? (x - ref) * kLog2e : __builtin_fmaf(x, kLog2e, shift));
                        }
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            part[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][r], kLog2e, shift));
                }
                // (a tile's 32 terms to each other first: one rounding of the running sum a tile)
                sum[j] = __builtin_fmaf(sum[j], __builtin_amdgcn_exp2f((mx[j] - ref) * kLog2e), part[0] + part[1]);
                mx[j] = top;
            } else {
                const bool far = !(fabsf(lse[j].x) < kFmaRange);
                const float sum2 = -lse[j].y * kLog2e, shift = __builtin_fmaf(-lse[j].x, kLog2e, sum2);
                if (__any(far)) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const float x = acc[i][j][r];
                            acc[i][j][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(far ? x - lse[j].x : x, kLog2e, far ? sum2 : shift));
                        }
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[i][j][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][r], kLog2e, shift));
                }
                if (__any(at > -64) || tail) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            if (at == place(i, r)) acc[i][j][r] -= 1.f;
                            if (place(i, r) >= live) acc[i][j][r] = 0.f;
                        }
                }
                const bool out = lse[j].y == INFINITY;   // (as in the tiles above)
                if (__any(out))
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[i][j][r] = out ? 0.f : acc[i][j][r];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int g = 0; g < 4; g += 2) {
                        const f32x16x &p = acc[i][j];
                        a.p[(m0 / 8 + 4 * i + g + h) * a.rows + n] =
                            join_chunk(bf16_pair(p[4 * g], p[4 * g + 1]), bf16_pair(p[4 * g + 2], p[4 * g + 3]),
                                       bf16_pair(p[4 * g + 4], p[4 * g + 5]), bf16_pair(p[4 * g + 6], p[4 * g + 7]));
                    }
            }
        }
    }
    if constexpr (EPI == kStats) {
#pragma unroll
        for (int j = 0; j < WNF; ++j) {
            const float om = __shfl_xor(mx[j], 32, kWave), os = __shfl_xor(sum[j], 32, kWave);
            const float top = fmaxf(mx[j], om), ref = top == -INFINITY ? 0.f : top;
            // (a lane whose logits are all -inf has the sum 0, or NaN, with no reference)
            const float s = (mx[j] == -INFINITY ? sum[j] : sum[j] * expf(mx[j] - ref)) + (om == -INFINITY ? os : os * expf(om - ref));
            if (h == 0) a.stats[((int64_t)1 + strip) * a.rows + n0 + 32 * j + lr] = make_float2(top, s);
        }
    }
}

// The statistics for at most 32 NR rows: bound by reading w once, so w and h are read as they lie (row-major, into the
// fragments), without the packing that the tiles above need.  A wavefront takes F x 32 classes: two blocks where its rows
// are short (30 x 200,000 x 64 bf16 24 -> 18 us), else one, so that there are more of them (1 x 169,000 x 256 31 -> 27;
// with the columns dealt to the four wavefronts of a workgroup 32).  169,000 x 256 bf16, one row: 19 us, 4.6 TB/s.
template <int PL>
__device__ __forceinline__ f32x16x product(const bf16x8 (&p)[PL], const bf16x8 (&q)[PL], f32x16x c) {
    if constexpr (PL == 1) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(p[0], q[0], c, 0, 0, 0);
    else return mfma_split6(p[0], p[PL - 2], p[PL - 1], q[0], q[PL - 2], q[PL - 1], c);
}

template <int PL, int NR, int F, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) k_xent_score(const XentArgs a, const void *__restrict__ W, int64_t ld_w,
                                                    const void *__restrict__ H, int64_t ld_h, int32_t ignore,
                                                    int32_t d) {
    constexpr int X = PL == 1 ? 1 : 2;                 // 16-byte units of 8 columns
    constexpr int U = 4;                 // steps of 16 columns in flight
    constexpr int TILE = 32 * F * WAVES;   // classes of a workgroup
    __shared__ float2 red[WAVES * 32 * NR];
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, lr = lane & 31;
    const int elt = PL == 1 ? 2 : 4;
    const char *src[F + NR];   // this lane's rows of w, and of h
#pragma unroll
    for (int f = 0; f < F; ++f) {
        const int64_t v = std::min<int64_t>(a.v0 + (int64_t)blockIdx.x * TILE + 32 * (F * wid + f) + lr, a.n_classes - 1);
        src[f] = (const char *)W + v * ld_w * elt;
    }
    bool live[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j) {
        const int n = 32 * j + lr;
        const int32_t y = n < a.m ? a.labels[n] : -1;
        live[j] = n < a.m && y != ignore && y >= 0 && y < a.n_classes;
        src[F + j] = (const char *)H + (live[j] ? n : 0) * ld_h * elt;
    }
    f32x16x acc[F][NR];
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int j = 0; j < NR; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[f][j][r] = 0.f;
    // 16 columns a step, 8 of them this lane's; past the end they count as zeros
    for (int32_t k0 = 0; k0 < d; k0 += 16 * U) {
        u32x4x x[U][F + NR][X];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int f = 0; f < F + NR; ++f)
#pragma unroll
                for (int q = 0; q < X; ++q) {
                    const int32_t k = k0 + 16 * u + 8 * h + q * 4;
                    x[u][f][q] = u32x4x{0, 0, 0, 0};
                    if (k < d && (f < F || live[f < F ? 0 : f - F])) x[u][f][q] = *(const u32x4x *)(src[f] + k * elt);
                }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t left = d - (k0 + 16 * u + 8 * h);
            bf16x8 p[F + NR][PL];
            if (left < 8)
#pragma unroll
                for (int f = 0; f < F + NR; ++f)
#pragma unroll
                    for (int q = 0; q < 4 * X; ++q) {
                        const uint32_t unit = x[u][f][q / 4][q % 4];
                        if constexpr (PL == 1) x[u][f][0][q] = 2 * q >= left ? 0u : 2 * q + 1 >= left ? unit & 0xffffu : unit;
                        else x[u][f][q / 4][q % 4] = q >= left ? 0u : unit;
                    }
#pragma unroll
            for (int f = 0; f < F + NR; ++f) {
                if constexpr (PL == 1) {
                    p[f][0] = __builtin_bit_cast(bf16x8, x[u][f][0]);
                } else {
                    float z[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = __uint_as_float(x[u][f][e / 4 * (X - 1)][e % 4]);
                    split3(z, p[f][0], p[f][PL - 2], p[f][PL - 1]);
                }
            }
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int j = 0; j < NR; ++j) acc[f][j] = product<PL>(p[f], p[F + j], acc[f][j]);
        }
    }
    if (a.z)
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int j = 0; j < NR; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    if (32 * j + lr < a.few)
                        a.z[((int64_t)blockIdx.x * (TILE / 4) + 8 * (F * wid + f) + 2 * g + h) * a.few + 32 * j + lr] =
                            f32x4x{acc[f][j][4 * g], acc[f][j][4 * g + 1], acc[f][j][4 * g + 2], acc[f][j][4 * g + 3]};
    if (a.stats) stats_of<PL, F, NR, WAVES, 1>(a, acc, blockIdx.x, 0, red);
}

// The gradients of at most 32 NR rows: bound by reading w and writing dw once, so they too take w and h as they lie, and the
// logits that the statistics kept (4 bytes a class and row, where a second product would read all of w again).
// A workgroup takes CW columns of every splits-th block of CB classes: w's block goes through LDS, where both its
// classes (dh) and, of p, the rows (dw) can be summed over; the next block's loads are in flight meanwhile.  One row x
// 169,000 x 256 bf16, in all: 61 us, through packed operands and the tiles 126; 4 x 39,124 x 373 fp32 138 -> 58, 64 x
// 1,000,000 x 128 bf16 486 -> 348, 57 x 25,820 x 602 fp32 157 -> 104.  Blocks
// of 128 classes need more registers than three workgroups leave (2 x 244,200 x 100 bf16 36 us against 20).
// p of bf16 rows is multiplied in two parts, its rounded value and the rest, 2^-16 of it off at most: sums of so few
// rows would show one rounding.  The second product costs little beside the loads: 1 x 169,000 x 256 60.1 -> 60.8 us, 64 x
// 1,000,000 x 128 346 -> 349, 57 x 137,653 x 200 83.6 -> 86.5.
constexpr int kFewClasses = 64;

template <int PL>
__device__ __forceinline__ f32x16x product_p(const bf16x8 (&x)[PL], const bf16x8 (&p)[PL == 1 ? 2 : PL], f32x16x c) {
    if constexpr (PL == 1)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[0], p[0], __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[0], p[1], c, 0, 0, 0),
                                                       0, 0, 0);
    else return product<PL>(x, p, c);
}

template <int PL, int NR, int CW, int CB>
__global__ void __launch_bounds__(256, NR == 1 ? 3 : 2) k_xent_few(const XentArgs a, const void *__restrict__ W, int64_t ld_w,
                                                     const void *__restrict__ H, int64_t ld_h, int32_t blocks,
                                                     float *__restrict__ part, int64_t width) {
    constexpr int FB = CW / 32, HALVES = 4 / FB;       // wavefronts along the columns, along the classes
    constexpr int C8 = CW / 8, UW = CB * C8 / 256, X = PL == 1 ? 1 : 2, RB = 32 * NR, ZN = CB / 4 * RB / 256;
    constexpr int PP = PL == 1 ? 2 : PL;               // parts of p
    __shared__ u32x4x sw[PL][C8 * CB], sp[PP][CB / 8 * RB], sh[PL][C8 * RB];
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, lr = lane & 31;
    const int fb = wid % FB, half = wid / FB, elt = PL == 1 ? 2 : 4;
    const int64_t c0 = (int64_t)blockIdx.y * CW;
    const bool want_dh = part != nullptr, want_dw = a.dw != nullptr;
    // 8 columns from `col` on as the matrix cores take them, zeros past d
    auto fetch = [&](u32x4x (&x)[X], const void *base, int64_t row, int64_t ld, int64_t col, bool live) {
#pragma unroll
        for (int q = 0; q < X; ++q) {
            x[q] = u32x4x{0, 0, 0, 0};
            if (live && col + 4 * q < a.d) x[q] = *(const u32x4x *)((const char *)base + (row * ld + col + 4 * q) * elt);
        }
    };
    auto put = [&](u32x4x (&x)[X], int64_t col, u32x4x *to, int plane) {
        if constexpr (PL == 1) {
            if (col + 8 > a.d)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (col + 2 * q + 1 >= a.d) x[0][q] &= 0xffffu;
                    if (col + 2 * q >= a.d) x[0][q] = 0;
                }
            to[0] = x[0];
        } else {
            float v[8];
            bf16x8 p[3];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = col + e < a.d ? __uint_as_float(x[e / 4 * (X - 1)][e % 4]) : 0.f;
            split3(v, p[0], p[1], p[2]);
#pragma unroll
            for (int pl = 0; pl < PL; ++pl) to[pl * plane] = __builtin_bit_cast(u32x4x, p[pl]);
        }
    };
    for (int q = tid; q < C8 * RB; q += 256) {
        const int lc = q % C8, r = q / C8;
        const int32_t y = r < a.m ? a.labels[r] : -1;
        u32x4x x[X];
        fetch(x, H, r, ld_h, c0 + 8 * lc, r < a.m && y != a.ignore && y >= 0 && y < a.n_classes);
        put(x, c0 + 8 * lc, &sh[0][lc * RB + (r ^ ((lc & 3) * 4))], C8 * RB);
    }
    for (int q = tid; q < PP * (CB / 8) * RB; q += 256) (&sp[0][0])[q] = u32x4x{0, 0, 0, 0};
    // p of four classes of a row, per thread and entry: the row is the same for all of a thread's entries
    const int quads = CB / 4 * a.few, row = tid & (a.few - 1), log = __builtin_ctz(a.few);
    const float2 lse = row < a.m ? a.lse[row] : make_float2(0.f, INFINITY);
    const int32_t label = row < a.m ? a.labels[row] : -1;
    u32x4x x[UW][X];
    f32x4x z[ZN];
    auto load = [&](int32_t b) {
        if (want_dh)
#pragma unroll
            for (int u = 0; u < UW; ++u) {
                const int q = tid + 256 * u;
                const int64_t v = a.v0 + (int64_t)b * CB + q / C8;
                fetch(x[u], W, v, ld_w, c0 + 8 * (q % C8), v < a.n_classes);
            }
#pragma unroll
        for (int u = 0; u < ZN; ++u)
            if (tid + 256 * u < quads) z[u] = a.z[(int64_t)b * quads + tid + 256 * u];
    };
    const int tr_mc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), tr_k = 8 * h + ((lane & 15) >> 2), tr_swz = tr_mc * 4;
    auto across = [&](const u32x4x *plane, auto rows_, int x0, int kk) -> bf16x8 {   // 16 rows of 32 columns from x0 on
        constexpr int R = decltype(rows_)::value;
        typedef __attribute__((address_space(3))) s16x4 lds4;
        const char *p0 = (const char *)(plane + (x0 / 8 + tr_mc) * R + ((kk * 16 + tr_k) ^ tr_swz)) + 8 * (lane & 1);
        const char *p1 = (const char *)(plane + (x0 / 8 + tr_mc) * R + ((kk * 16 + tr_k + 4) ^ tr_swz)) + 8 * (lane & 1);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)p0);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)p1);
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        return __builtin_bit_cast(bf16x8, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    };
    f32x16x dh[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) dh[j][r] = 0.f;
    const float inv = want_dw ? a.inv_count[0] : 0.f;
    if ((int32_t)blockIdx.x < blocks) load(blockIdx.x);
    __syncthreads();
    bf16x8 fh[2 * NR][PL];
#pragma unroll
    for (int kk = 0; kk < 2 * NR; ++kk)
#pragma unroll
        for (int pl = 0; pl < PL; ++pl) fh[kk][pl] = across(sh[pl], std::integral_constant<int, RB>(), 32 * fb, kk);
    for (int32_t b = blockIdx.x; b < blocks; b += gridDim.x) {
        if (want_dh)
#pragma unroll
            for (int u = 0; u < UW; ++u) {
                const int q = tid + 256 * u, lc = q % C8, r = q / C8;
                put(x[u], c0 + 8 * lc, &sw[0][lc * CB + (r ^ ((lc & 3) * 4))], C8 * CB);
            }
#pragma unroll
        for (int u = 0; u < ZN; ++u) {
            const int q = tid + 256 * u;
            if (q >= quads) break;
            const int c4 = q >> log;
            const int64_t v = a.v0 + (int64_t)b * CB + 4 * c4;
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (PL == 1) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[u][e] - lse.x, kLog2e, -lse.y * kLog2e));
                else p[e] = expf((z[u][e] - lse.x) - lse.y);
                if (label == v + e) p[e] -= 1.f;
                if (lse.y == INFINITY || v + e >= a.n_classes) p[e] = 0.f;
            }
            const int at = c4 / 2 * RB + (row ^ ((c4 / 2 & 3) * 4));
            if constexpr (PL == 1) {   // the value rounded, and what that leaves
#pragma unroll
                for (int pl = 0; pl < PP; ++pl) {
                    const u32x2x w = {bf16_pair(p[0], p[1]), bf16_pair(p[2], p[3])};
                    ((u32x2x *)&sp[pl][at])[c4 & 1] = w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] -= __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
                }
            } else {
                uint16_t s[4][3];
#pragma unroll
                for (int e = 0; e < 4; ++e) split3_bits(p[e], s[e][0], s[e][1], s[e][2]);
#pragma unroll
                for (int pl = 0; pl < PL; ++pl)
                    ((u32x2x *)&sp[pl][at])[c4 & 1] =
                        u32x2x{(uint32_t)s[0][pl] | ((uint32_t)s[1][pl] << 16), (uint32_t)s[2][pl] | ((uint32_t)s[3][pl] << 16)};
            }
        }
        __syncthreads();
        if (b + (int32_t)gridDim.x < blocks) load(b + gridDim.x);
        if (want_dh)
#pragma unroll
            for (int k = 0; k < CB / 16 / HALVES; ++k) {
                const int kk = half * (CB / 16 / HALVES) + k, c8 = 2 * kk + h;
                bf16x8 f[PL], g[PP];
#pragma unroll
                for (int pl = 0; pl < PL; ++pl) f[pl] = across(sw[pl], std::integral_constant<int, CB>(), 32 * fb, kk);
#pragma unroll
                for (int j = 0; j < NR; ++j) {
#pragma unroll
                    for (int pl = 0; pl < PP; ++pl)
                        g[pl] = __builtin_bit_cast(bf16x8, sp[pl][c8 * RB + ((32 * j + lr) ^ ((c8 & 3) * 4))]);
                    dh[j] = product_p<PL>(f, g, dh[j]);
                }
            }
        if (want_dw)
#pragma unroll
            for (int k = 0; k < CB / 32 / HALVES; ++k) {
                const int cb = half * (CB / 32 / HALVES) + k;
                f32x16x acc;
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[r] = 0.f;
#pragma unroll
                for (int kk = 0; kk < 2 * NR; ++kk) {
                    bf16x8 g[PP];
#pragma unroll
                    for (int pl = 0; pl < PP; ++pl) g[pl] = across(sp[pl], std::integral_constant<int, RB>(), 32 * cb, kk);
                    acc = product_p<PL>(fh[kk], g, acc);
                }
                const int64_t v = a.v0 + (int64_t)b * CB + 32 * cb + lr, c = c0 + 32 * fb;
                if constexpr (PL == 1) {
#pragma unroll
                    for (int g = 0; g < 4; g += 2) {
                        float o[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = c + 8 * (g + e / 4) + 4 * h + e % 4 < a.d ? acc[4 * g + e] * inv : 0.f;
                        const u32x4x w = join_chunk(bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3]), bf16_pair(o[4], o[5]), bf16_pair(o[6], o[7]));
                        if (v < a.n_classes && c + 8 * (g + h) < a.d) *(u32x4x *)((uint16_t *)a.dw + v * a.ld_dw + c + 8 * (g + h)) = w;
                    }
                } else {
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        f32x4x o;
                        const int64_t at = c + 8 * g + 4 * h;
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = at + e < a.d ? acc[4 * g + e] * inv : 0.f;
                        if (v < a.n_classes && at < a.d) *(f32x4x *)((float *)a.dw + v * a.ld_dw + at) = o;
                    }
                }
            }
        __syncthreads();
    }
    if (want_dh)
#pragma unroll
        for (int j = 0; j < NR; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (32 * j + lr < a.few) {
                    f32x4x *at = (f32x4x *)(part + (((int64_t)blockIdx.x * HALVES + half) * a.few + 32 * j + lr) * width + c0 +
                                            32 * fb + 8 * g + 4 * h);
                    f32x4x v = {dh[j][4 * g], dh[j][4 * g + 1], dh[j][4 * g + 2], dh[j][4 * g + 3]};
                    if (!a.first) v += *at;
                    *at = v;
                }
}

// dh of few rows from its parts: 8 units of four columns a workgroup, the parts dealt to 32 threads of each.
__global__ void __launch_bounds__(256) k_xent_few_dh(const f32x4x *__restrict__ part, int32_t parts, int32_t few,
                                                     int64_t width, int64_t d, const float2 *__restrict__ lse,
                                                     const float *__restrict__ inv_count, void *__restrict__ dh, int64_t ld,
                                                     bool bf16) {
    __shared__ f32x4x sums[4][8];
    const int tid = threadIdx.x, unit = tid & 7;
    const int64_t c = ((int64_t)blockIdx.x * 8 + unit) * 4, n = blockIdx.y, units = width / 4;
    f32x4x v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int32_t s = tid >> 3; s < parts; s += 32) v += part[((int64_t)s * few + n) * units + c / 4];
#pragma unroll
    for (int o = 8; o < kWave; o <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], o, kWave);
    if ((tid & 63) < 8) sums[tid / 64][unit] = v;
    __syncthreads();
    if (tid >= 8 || c >= (bf16 ? (d + 7) / 8 * 8 : (d + 3) / 4 * 4)) return;
    v = (sums[0][unit] + sums[1][unit]) + (sums[2][unit] + sums[3][unit]);
    const bool counts = row_counts(lse[n]);
    const float inv = inv_count[0];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = counts && c + e < d ? v[e] * inv : 0.f;
    if (bf16) *(u32x2x *)((uint16_t *)dh + n * ld + c) = u32x2x{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    else *(f32x4x *)((float *)dh + n * ld + c) = v;
}

// A piece's dh and dw in one launch: the workgroups of dh (the first `dh_ids`), then those of dw, fill
// the units together.  Both take the same tiles.
template <int PL, int WMF, int WNF, int WGM, int WGN>
__global__ void __launch_bounds__(64 * WGM * WGN, 2) k_xent_grads(const XentArgs w, const XentArgs h, int32_t dh_ids) {
    __shared__ u32x4x S[Tile<PL, WMF, WNF, WGM, WGN>::LDS];
    if ((int32_t)blockIdx.x < dh_ids) xent_tile<PL, WMF, WNF, WGM, WGN, true, false, kDh>(h, blockIdx.x, S, nullptr);
    else xent_tile<PL, WMF, WNF, WGM, WGN, true, true, kDw>(w, blockIdx.x - dh_ids, S, nullptr);
}

// ------------------------------------------------------------- rows and loss
// Joins a row's entries [from, tiles]: before the last piece to entry 0 (kFold), then to lse (0 and +inf for a row that
// does not count) and the row's loss.  ROWS rows a workgroup, the entries dealt to SLICES threads of each.
// kLoss: there is one workgroup, which takes the mean too.
enum { kFold, kLse, kLoss };
template <int ROWS, int SLICES, int MODE>
__global__ void __launch_bounds__(ROWS * SLICES) k_xent_rows(float2 *stats, int64_t from, int64_t tiles, int64_t rows,
                                                             int64_t m, const int32_t *__restrict__ labels,
                                                             int32_t ignore, int64_t n_classes,
                                                             const float *__restrict__ label_logit,
                                                             float2 *__restrict__ lse, float *losses,
                                                             float *__restrict__ row_loss, float *loss,
                                                             float *inv_count) {
    __shared__ float2 part[SLICES][ROWS];
    const int tid = threadIdx.x, c = tid % ROWS, k = tid / ROWS;
    const int64_t n = (int64_t)blockIdx.x * ROWS + c;
    float mx = -INFINITY, s = 0.f;
    // (a tile whose logits are all -inf has the sum 0, or NaN, with no reference)
    auto join = [&](const float2 *o, int count) {
        float top = mx;
        for (int q = 0; q < count; ++q) top = fmaxf(top, o[q].x);
        const float ref = top == -INFINITY ? 0.f : top;
        s *= expf(mx - ref);
        for (int q = 0; q < count; ++q) s += o[q].x == -INFINITY ? o[q].y : o[q].y * expf(o[q].x - ref);
        mx = top;
    };
    int64_t t = from + k;
    for (; t + 7 * SLICES <= tiles; t += 8 * SLICES) {
        float2 o[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) o[q] = stats[(t + q * SLICES) * rows + n];
        join(o, 8);
    }
    for (; t <= tiles; t += SLICES) {
        const float2 o = stats[t * rows + n];
        join(&o, 1);
    }
    part[k][c] = make_float2(mx, s);
    __syncthreads();
    for (int w = SLICES / 2; w > 0; w >>= 1) {
        if (k < w) {
            join(&part[k + w][c], 1);
            part[k][c] = make_float2(mx, s);
        }
        __syncthreads();
    }
    if constexpr (MODE == kFold) {   // (every entry has been read)
        if (k == 0) stats[n] = make_float2(mx, s);
        return;
    }
    if (k == 0) {
        const int32_t y = n < m ? labels[n] : ignore;
        const bool out = n >= m || y == ignore, bad = !out && (y < 0 || y >= n_classes);
        lse[n] = out || bad ? make_float2(0.f, INFINITY) : make_float2(mx, logf(s));
        const float one = out ? 0.f : bad ? NAN : logf(s) + (mx - label_logit[n]);
        losses[n] = one;
        if (row_loss && n < m) row_loss[n] = one;
    }
    if constexpr (MODE == kLoss) {
        __syncthreads();
        xent_loss<ROWS * SLICES>(losses, m, labels, ignore, loss, inv_count);
    }
}

__global__ void __launch_bounds__(1024) k_xent_loss(const float *__restrict__ losses, int64_t m,
                                                    const int32_t *__restrict__ labels, int32_t ignore,
                                                    float *__restrict__ loss, float *__restrict__ inv_count) {
    xent_loss<1024>(losses, m, labels, ignore, loss, inv_count);
}

// dh from the splits' parts, in the order the products kept them in (each lane's registers side by side, so that
// parts are written, added to and read in whole lines).
// SLICES > 1: a workgroup has 256 / SLICES units and deals the splits to as many threads of each (few units: 57 x 137,653 x
// 200 bf16 8 -> 5 us).
template <int WMF, int WNF, int WGM, int WGN, int SLICES>
__global__ void __launch_bounds__(256) k_xent_dh(const f32x4x *__restrict__ part, int64_t total, int32_t splits,
                                                 int64_t split_stride, int32_t m_tiles, int64_t m, int64_t d,
                                                 const float2 *__restrict__ lse, const float *__restrict__ inv_count,
                                                 void *__restrict__ dh, int64_t ld, bool bf16) {
    constexpr int UNITS = 256 / SLICES;
    __shared__ f32x4x sums[SLICES][UNITS];
    const float inv = inv_count[0];
    const int64_t stride = (int64_t)gridDim.x * UNITS;
    const int unit = threadIdx.x % UNITS, slice = threadIdx.x / UNITS;
    for (int64_t base = (int64_t)blockIdx.x * UNITS; base < total; base += stride) {
        const int64_t at = base + unit;
        int64_t x = at;
        const int lane = x & 63;
        x >>= 6;
        const int g = x & 3;
        x >>= 2;
        const int j = x % WNF;
        x /= WNF;
        const int i = x % WMF;
        x /= WMF;
        const int wid = x % (WGM * WGN);
        x /= WGM * WGN;
        const int64_t c = (x % m_tiles) * (32 * WMF * WGM) + (wid / WGN) * (32 * WMF) + 32 * i + 8 * g + 4 * (lane >> 5);
        const int64_t n = (x / m_tiles) * (32 * WNF * WGN) + (wid % WGN) * (32 * WNF) + 32 * j + (lane & 31);
        const int64_t width = bf16 ? (d + 7) / 8 * 8 : (d + 3) / 4 * 4;
        const bool live = at < total && n < m && c < width;
        f32x4x v = {0.f, 0.f, 0.f, 0.f};
        if (live && row_counts(lse[n]))
#pragma unroll 8
            for (int32_t s = slice; s < splits; s += SLICES) v += part[s * split_stride + at];
        if constexpr (SLICES > 1) {
            sums[slice][unit] = v;
            __syncthreads();
            if (slice == 0)
#pragma unroll
                for (int k = 1; k < SLICES; ++k) v += sums[k][unit];
            __syncthreads();
            if (slice > 0) continue;
        }
        if (!live) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = c + e < d ? v[e] * inv : 0.f;
        if (bf16)
            *(u32x2x *)((uint16_t *)dh + n * ld + c) = u32x2x{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
        else
            *(f32x4x *)((float *)dh + n * ld + c) = v;
    }
}

// ------------------------------------------------------------------ the plan
namespace {

constexpr int64_t kPBytes = int64_t(1) << 30;     // p of a piece, at most (or one tile of classes)
// Kept logits of few rows, at most: past it (32 rows of 262,144 classes) the gradients score a piece again, which reads
// w a third time.
constexpr int64_t kFewBytes = int64_t(32) << 20;
constexpr int64_t kFewMore = int64_t(1) << 20;   // classes for which 33 to 64 rows count as few, at most (256 MiB of logits)
constexpr int64_t kLogits = int64_t(1) << 32;     // logits of a piece whose p is not kept, at most: its statistics are a 64th of their size
constexpr int64_t kWBytes = int64_t(896) << 20;   // packed weights, at most (or one tile): of all pieces, else of one

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct XentPlan {
    int pl;                         // planes
    int64_t rows, bk;               // packed rows of h, summed elements per step
    int64_t dw_rows;                // rows that dw sums over: whole steps of those that there are (150 x 30,000 x 256 fp32 131 -> 112 us)
    int64_t ln, rn;                 // rows of a logit tile, of a dh tile (and classes of a dw tile)
    int64_t bm, width, chunks;      // features of a gradient tile, packed columns, their chunks
    int32_t strips, strip_tiles;    // k_xent_strip: strips of a piece, their tiles (0: the other kernels)
    int64_t piece, vt;              // classes of a piece, of a logit tile
    int32_t few;                    // rows of the kept logits, of the kernels for at most 64 rows (0: the other kernels)
    int32_t few_tile;               // k_xent_score: classes of a workgroup
    int32_t few_splits;             // k_xent_few: workgroups along the classes of a piece
    bool whole;                     // the packed weights of all pieces are kept between the passes
    int32_t splits, split_steps;    // of dh's sum over a piece
    size_t z, h, w, p, part, stats, label_logit, lse, losses, inv, total;

    // In how many parts dh's sum over a piece is taken: `tiles` workgroups of `steps` steps each are cut into so many,
    // and `dw` workgroups of `dw_steps` follow them on the device's places.  The makespan of that, and the time of
    // moving a part's sums (`part_bytes`), decide: 4,093 x 169,000 x 256 bf16 takes 16 tiles of 2,646 steps and 331 of
    // 128 on 256 places, 420 us a piece in 16 parts.
    int32_t dh_splits(int64_t tiles, int64_t steps, int64_t dw, int64_t dw_steps, int64_t part_bytes) const {
        const int64_t places = rn == 256 ? 256 : 512;   // a 256 x 256 tile has a unit to itself
        // seconds of a step of one workgroup at the rate that the products reach
        const double step = 2.0 * bm * rn * bk * (pl == 3 ? 6 : 1) * places / 1.1e15;
        double best = 0;
        int32_t best_s = 0;
        for (int64_t s = 1; s <= 128 && s <= std::max<int64_t>(1, steps / 8); s += s < 16 ? 1 : s < 32 ? 2 : 8) {
            const int64_t len = (steps + s - 1) / s, jobs = tiles * s, full = jobs / places, late = jobs % places;
            // `late` places are free after full + 1 jobs, the others after full
            auto done = [&](int64_t t) {
                const int64_t x = t - full * len, y = x - len;
                return (places - late) * (x > 0 ? x / dw_steps : 0) + late * (y > 0 ? y / dw_steps : 0);
            };
            int64_t end = full * len + (late ? len : 0);
            if (dw > 0) {
                int64_t k = dw / places;   // rounds of dw on the earlier places at least, on the later ones one fewer
                k = std::max<int64_t>(0, k - (len + dw_steps - 1) / dw_steps - 1);
                int64_t t = full * len + k * dw_steps, u = full * len + len + std::max<int64_t>(0, k - len / dw_steps - 1) * dw_steps;
                while (done(t) < dw) t += dw_steps;
                while (done(u) < dw) u += dw_steps;
                end = std::max(end, std::min(t, u));
            }
            const double cost = end * step + (double)s * part_bytes / 4e12;
            if (best_s == 0 || cost < best) {
                best = cost;
                best_s = (int32_t)s;
            }
        }
        return best_s;
    }

    // Columns and classes of a block of k_xent_few: 256 bytes of a row, half where that is all.
    static int few_columns(int64_t d, bool bf16) { return bf16 && d > 64 ? 128 : 64; }
    

    void few_plan(int64_t n_classes, int64_t d, bool bf16, bool grads, bool dh) {
        const int64_t all = up(n_classes, kPiece), cw = few_columns(d, bf16);
        width = up(d, cw);
        // one workgroup of 8 wavefronts to 256 classes, of 4 to 128 where those are too few for the device (17 x 30,000 x 1,024
        // bf16 66 -> 57 us in all)
        few_tile = d > 64 && all / 256 < 512 ? 128 : 256;
        piece = few > 32 ? all : std::min(all, std::max<int64_t>(kPiece, kFewBytes / (few * 4) / kPiece * kPiece));
        const int64_t pieces = (all + piece - 1) / piece;
        piece = up((all + pieces - 1) / pieces, kPiece);
        const int64_t blocks = piece / kFewClasses;
        // two workgroups a unit (three: 32 x 169,000 x 256 fp32 167 -> 172 us, 1 row 121 -> 126), of as many blocks each
        const int64_t most = std::max<int64_t>(1, 512 / (width / cw)), each = (blocks + most - 1) / most;
        few_splits = (int32_t)((blocks + each - 1) / each);
        size_t at = 0;
        auto take = [&](int64_t bytes) {
            const size_t here = at;
            at += (size_t)up(bytes, 256);
            return here;
        };
        z = take(grads ? piece * few * 4 : 0);
        part = take(dh ? few_splits * (128 / cw) * few * width * 4 : 0);
        stats = take((1 + all / few_tile) * rows * 8);
        label_logit = take(rows * 4);
        lse = take(rows * 8);
        losses = take(rows * 4);
        inv = take(4);
        total = at;
    }

    XentPlan(int64_t m, int64_t n_classes, int64_t d, bool bf16, bool grads, bool dh) {
        pl = bf16 ? 1 : 3;
        bk = bf16 ? 32 : 16;
        // Gradient tiles of 256 x 256 where the columns fill them: 4,093 x 169,000 x 256 bf16 2,093 us in all (256 x 128: 2,178,
        // 128 x 128: 2,303), 8,192 x 65,536 x 1,024 4,105 (4,200, 4,435), and where dw has some half a round of them:
        // 1,000 x 40,000 x 256 (157) 120 us, 128 x 128 126; 1,000 x 20,000 (79) 93 and 86.
        const bool big = bf16 && m > 128 && d > 128 && up(d, 256) * 10 <= up(d, 128) * 11 &&
                         up(d, 256) / 256 * (up(n_classes, 256) / 256) >= 128;
        few = 0;
        if (m <= 32 || (m <= 64 && n_classes <= kFewMore))
            for (few = 1; few < m;) few *= 2;
        ln = few > 32 ? 64 : few > 0 ? 32 : 128;
        rn = big ? 256 : ln;
        // 64 features where d has no more, and where dw, whose sum is not cut, has too few tiles of 128: 3,590 x 6,349 x 128
        // fp32 (50) 264 -> 221 us, 8,000 x 5,000 x 128 bf16 (40) 145 -> 135; 2,000 x 6,000 x 602 fp32 (235) 345, 372 with 64
        bm = big ? 256 : (d <= 64 || up(d, 128) / 128 * (up(n_classes, 128) / 128) < 128) && rn == 128 ? 64 : 128;
        if (bf16 && few == 0 && d <= 256) ln = m > 128 ? 256 : 128;   // held in registers
        rows = up(std::max<int64_t>(m, 1), grads ? std::max(rn, ln) : ln);
        dw_rows = up(std::max<int64_t>(m, 1), bk);
        width = up(d, grads ? bm : 64);
        if (bf16 && few == 0 && d > 128 && d <= 256) width = 256;
        if (bf16 && few == 0 && d > 64 && d <= 128) width = 128;
        if (few > 0) {
            few_plan(n_classes, d, bf16, grads, dh);
            return;
        }
        chunks = width / 8;
        const int64_t all = up(n_classes, kPiece);
        piece = std::max<int64_t>(kPiece, kWBytes / (width * 2 * pl) / kPiece * kPiece);
        const int64_t most = grads ? kPBytes / (2 * pl) : kLogits;
        piece = std::min(piece, std::max<int64_t>(kPiece, most / rows / kPiece * kPiece));
        piece = std::min(piece, all);
        const int64_t pieces = (all + piece - 1) / piece;
        piece = up((all + pieces - 1) / pieces, kPiece);   // equal ones
        // fp32 with fewer 128 x 128 tiles than places for them: 64 x 64 (256 x 10,000 x 64 47 -> 41 us, 128 x 5,000 x 256 59 ->
        // 44; bf16 tiles are too short for it to matter)
        vt = !bf16 && piece / 128 * (rows / 128) < 512 ? 64 : 128;
        strips = strip_tiles = 0;
        if (bf16 && d <= 256) {   // two workgroups a unit
            const int64_t t = piece / kStrip, round = std::max<int64_t>(1, 512 / (rows / ln));
            const int64_t s = std::min(t, (t + round * kStripTiles - 1) / (round * kStripTiles) * round);
            strip_tiles = (int32_t)((t + s - 1) / s);
            strips = (int32_t)((t + strip_tiles - 1) / strip_tiles);
        }
        splits = 1;
        split_steps = 0;
        if (dh) {
            const int64_t steps = piece / bk, dw = width / bm * (piece / rn);
            // (dw with the steps of all packed rows: the ones that it leaves out about pay for its stores; 520 x 50,000 x 512
            // bf16 195 us so, 203 with its own)
            splits = dh_splits(width / bm * (rows / rn), steps, dw, rows / bk, rows * width * 4 * (pieces + 1));
            split_steps = (int32_t)((steps + splits - 1) / splits);
            splits = (int32_t)((steps + split_steps - 1) / split_steps);
        }
        size_t at = 0;
        auto take = [&](int64_t bytes) {
            const size_t here = at;
            at += (size_t)up(bytes, 256);
            return here;
        };
        h = take(rows * width * 2 * pl);
        whole = all * width * 2 * pl <= kWBytes;
        w = take((whole ? all : piece) * width * 2 * pl);
        p = take(grads ? rows * piece * 2 * pl : 0);
        part = take(dh ? splits * rows * width * 4 : 0);
        stats = take((1 + (strips > 0 ? strips : piece / vt)) * rows * 8);
        label_logit = take(rows * 4);
        lse = take(rows * 8);
        losses = take(rows * 4);
        inv = take(4);
        total = at;
    }
};

unsigned ids_of(const XentArgs &a) {   // workgroups of a product, whole rounds over the XCDs
    return (unsigned)up((int64_t)a.m_tiles * a.n_tiles * a.splits, 8);
}

// Logit tiles: 128 classes x 128 rows.  256 x 128 and, in 8 wavefronts, 256 x 256 tiles move less to LDS
// but have fewer workgroups on a unit to fill each other's gaps (4,093 x 169,000 x 256 bf16: both
// passes 609 us, 128 x 128 595; x 1,024 columns 2,118 and 2,145; fp32 1,024 rows 1,342 and 1,256).
template <int PL, int EPI>
void run_logits(XentArgs &a, const XentPlan &plan, int64_t d, int64_t vdim, bool with_loss, const char *label,
                hipStream_t s) {
    const int64_t ln = plan.ln;
    if constexpr (PL == 1)
        if (plan.strips > 0) {
            a.m_tiles = (int32_t)(a.rows / ln);
            a.n_tiles = plan.strips;
            a.splits = 1;
            a.split_steps = plan.strip_tiles;
            KernelTimer t(label, s);
            a.loss_block = with_loss ? (int32_t)ids_of(a) : -1;
            const unsigned grid = ids_of(a) + (with_loss ? 1 : 0);
#define GNNAV_L(KS)                                                                                                   \
    do {                                                                                                              \
        if (ln == 256) hipLaunchKernelGGL((k_xent_strip<KS, 2, EPI>), dim3(grid), dim3(256), 0, s, a);                \
        else hipLaunchKernelGGL((k_xent_strip<KS, 1, EPI>), dim3(grid), dim3(256), 0, s, a);                          \
    } while (0)
            if (d <= 64) GNNAV_L(4);
            else if (d <= 128) GNNAV_L(8);
            else GNNAV_L(16);
#undef GNNAV_L
            return;
        }
    const bool small = PL == 3 && plan.vt == 64;
    a.m_tiles = (int32_t)(vdim / plan.vt);
    // (64 rows past the last one are not written, nor does a result read them)
    a.n_tiles = (int32_t)(small ? up(std::max<int64_t>(a.m, 1), 64) / 64 : a.rows / ln);
    a.splits = 1;
    a.loss_block = with_loss ? (int32_t)ids_of(a) : -1;
    const unsigned grid = ids_of(a) + (with_loss ? 1 : 0);
    KernelTimer t(label, s);
    if constexpr (PL == 3)
        if (small) {
            hipLaunchKernelGGL((k_xent_logits<PL, 1, 1, 2, 2, EPI>), dim3(grid), dim3(256), 0, s, a);
            return;
        }
    hipLaunchKernelGGL((k_xent_logits<PL, 2, 2, 2, 2, EPI>), dim3(grid), dim3(256), 0, s, a);
}

// Gradient tiles: bm features x rn classes for dw, x rn rows for dh.  Either product may be absent (no tiles).
template <int PL>
void run_grads(const XentArgs &w, const XentArgs &h, int64_t bm, int64_t rn, hipStream_t s) {
    KernelTimer t("xent_grads", s);
    const unsigned nw = w.m_tiles > 0 ? ids_of(w) : 0, nh = h.m_tiles > 0 ? ids_of(h) : 0;
#define GNNAV_L(WMF, WNF, WGM, WGN)                                                                                   \
    hipLaunchKernelGGL((k_xent_grads<PL, WMF, WNF, WGM, WGN>), dim3(nw + nh), dim3(64 * WGM * WGN), 0, s, w, h, (int32_t)nh)
    if (rn == 256) {
        if constexpr (PL == 1) GNNAV_L(4, 2, 2, 4);
    } else if (bm == 128) {
        GNNAV_L(2, 2, 2, 2);
    } else {
        GNNAV_L(1, 2, 2, 2);
    }
#undef GNNAV_L
}

template <int PL, int NR>
void xent_few(const XentPlan &p, const LinearXentArgs &x, hipStream_t s) {
    constexpr bool BF = PL == 1;
    char *ws = (char *)x.workspace;
    float2 *lse = (float2 *)(ws + p.lse);
    float *inv = (float *)(ws + p.inv), *losses = (float *)(ws + p.losses);
    XentArgs a = {};
    a.n_classes = x.n_classes;
    a.rows = p.rows;
    a.labels = x.labels;
    a.m = x.m;
    a.d = x.d;
    a.stats = (float2 *)(ws + p.stats);
    a.label_logit = (float *)(ws + p.label_logit);
    a.lse = lse;
    a.inv_count = inv;
    a.ignore = x.ignore;
    a.few = p.few;
    a.dw = x.dw;
    a.ld_dw = x.ld_dw;
    f32x4x *z = (f32x4x *)(ws + p.z);
    const bool grads = x.dh || x.dw;
    const int64_t all = up(x.n_classes, kPiece), entries = all / p.few_tile;
    const bool one = p.piece == all;   // otherwise the gradients score each piece again
    auto score = [&](int64_t classes) {
        KernelTimer t("xent_stats", s);
#define GNNAV_L(F, WAVES)                                                                                                \
    hipLaunchKernelGGL((k_xent_score<PL, NR, F, WAVES>), dim3((unsigned)(classes / p.few_tile)), dim3(64 * WAVES), 0, s, a,  \
                       x.w, x.ld_w, x.h, x.ld_h, x.ignore, (int32_t)x.d)
        if (x.d <= 64) GNNAV_L(2, 4);
        else if (p.few_tile == 128) GNNAV_L(1, 4);
        else GNNAV_L(1, 8);
#undef GNNAV_L
    };
    a.z = grads && one ? z : nullptr;
    score(all);
    {
        KernelTimer t("xent_rows", s);
#define GNNAV_L(ROWS)                                                                                                    \
    hipLaunchKernelGGL((k_xent_rows<ROWS, 1024 / (ROWS), kLoss>), dim3(1), dim3(1024), 0, s, a.stats, (int64_t)1, entries, p.rows, \
                       x.m, x.labels, x.ignore, x.n_classes, a.label_logit, lse, losses, x.row_loss, x.loss, inv)
        if (NR == 1 && p.few <= 4) GNNAV_L(4);
        else GNNAV_L(32 * NR);
#undef GNNAV_L
    }
    if (!grads) {
        GNNAV_HIP(hipGetLastError());
        return;
    }
    float *part = x.dh ? (float *)(ws + p.part) : nullptr;
    const int cw = p.few_columns(x.d, BF);
    a.z = z;
    a.stats = nullptr;
    for (int64_t v0 = 0; v0 < all; v0 += p.piece) {
        const int64_t vp = std::min(p.piece, all - v0);
        a.v0 = v0;
        a.first = v0 == 0;
        if (!one) score(vp);
        KernelTimer t("xent_grads", s);
        const dim3 grid((unsigned)p.few_splits, (unsigned)(p.width / cw));
        const int32_t blocks = (int32_t)(vp / kFewClasses);
        if constexpr (BF)
            if (cw == 128)
                hipLaunchKernelGGL((k_xent_few<PL, NR, 128, kFewClasses>), grid, dim3(256), 0, s, a, x.w, x.ld_w, x.h, x.ld_h, blocks, part, p.width);
        if (cw == 64)
            hipLaunchKernelGGL((k_xent_few<PL, NR, 64, kFewClasses>), grid, dim3(256), 0, s, a, x.w, x.ld_w, x.h, x.ld_h, blocks, part, p.width);
    }
    if (x.dh && x.m > 0) {
        KernelTimer t("xent_dh_join", s);
        hipLaunchKernelGGL(k_xent_few_dh, dim3((unsigned)(p.width / 32), (unsigned)x.m), dim3(256), 0, s, (const f32x4x *)part,
                           p.few_splits * (128 / cw), p.few, p.width, x.d, lse, inv, x.dh, x.ld_dh, BF);
    }
    GNNAV_HIP(hipGetLastError());
}

template <int PL>
void xent(const XentPlan &p, const LinearXentArgs &x, hipStream_t s) {
    if (p.few > 32) return xent_few<PL, 2>(p, x, s);
    if (p.few > 0) return xent_few<PL, 1>(p, x, s);
    constexpr bool BF = PL == 1;
    char *ws = (char *)x.workspace;
    u32x4x *H = (u32x4x *)(ws + p.h), *W = (u32x4x *)(ws + p.w), *Pb = (u32x4x *)(ws + p.p);
    float2 *lse = (float2 *)(ws + p.lse);
    float *inv = (float *)(ws + p.inv), *losses = (float *)(ws + p.losses);
    const int64_t esize = BF ? 2 : 4, k1 = up(x.d, p.bk);
    // h, with the first piece of w that is packed
    bool h_packed = false;
    auto weights = [&](int64_t v0) { return W + (p.whole ? v0 * p.chunks * PL : 0); };
    auto pack_w = [&](int64_t v0, int64_t vp) {
        KernelTimer t("xent_pack", s);
        const PackArgs rows = {x.h, x.ld_h, x.m, p.rows, x.labels, H};
        const PackArgs classes = {(const char *)x.w + v0 * x.ld_w * esize, x.ld_w, std::min(vp, x.n_classes - v0), vp, nullptr, weights(v0)};
        const unsigned blocks = h_packed ? 0 : (unsigned)((p.rows + 63) / 64);
        hipLaunchKernelGGL(k_xent_pack<BF>, dim3(blocks + (unsigned)(vp / 64), (unsigned)((p.chunks + 7) / 8)), dim3(256),
                           0, s, rows, classes, (int32_t)blocks, x.d, x.ignore, x.n_classes, p.chunks);
        h_packed = true;
    };
    XentArgs a = {};
    a.n_classes = x.n_classes;
    a.rows = p.rows;
    a.labels = x.labels;
    a.m = x.m;
    a.stats = (float2 *)(ws + p.stats);
    a.label_logit = (float *)(ws + p.label_logit);
    a.lse = lse;
    a.inv_count = inv;
    a.losses = losses;
    a.ignore = x.ignore;
    a.loss = x.loss;
    a.loss_block = -1;
    auto logits = [&](int64_t v0, int64_t vp) {
        a.v0 = v0;
        a.A = weights(v0);
        a.a_rows = vp;
        a.a_plane = p.chunks * vp;
        a.B = H;
        a.b_rows = p.rows;
        a.b_plane = p.chunks * p.rows;
        a.k = k1;
    };
    const int64_t all = up(x.n_classes, kPiece);
    bool several = false;  // entry 0 of the statistics holds earlier pieces'
    int64_t entries = 0;   // of the piece
    for (int64_t v0 = 0; v0 < all; v0 += p.piece) {
        const int64_t vp = std::min(p.piece, all - v0);
        if (v0 > 0) {
            KernelTimer t("xent_rows", s);
            hipLaunchKernelGGL((k_xent_rows<16, 16, kFold>), dim3((unsigned)(p.rows / 16)), dim3(256), 0, s, a.stats,
                               several ? 0 : 1, entries, p.rows, x.m, x.labels, x.ignore, x.n_classes, a.label_logit,
                               lse, losses, nullptr, nullptr, nullptr);
            several = true;
        }
        pack_w(v0, vp);
        logits(v0, vp);
        run_logits<PL, kStats>(a, p, x.d, vp, false, "xent_stats", s);
        entries = p.strips > 0 ? p.strips : vp / p.vt;
    }
    {
        KernelTimer t("xent_rows", s);
        const int64_t from = several ? 0 : 1;
        hipLaunchKernelGGL((k_xent_rows<16, 16, kLse>), dim3((unsigned)(p.rows / 16)), dim3(256), 0, s, a.stats, from,
                           entries, p.rows, x.m, x.labels, x.ignore, x.n_classes, a.label_logit, lse, losses, x.row_loss,
                           nullptr, nullptr);
        if (!(x.dh || x.dw))   // otherwise it rides with the first probabilities
            hipLaunchKernelGGL(k_xent_loss, dim3(1), dim3(1024), 0, s, losses, x.m, x.labels, x.ignore, x.loss, inv);
    }
    if (x.dh || x.dw) {
        for (int64_t v0 = 0; v0 < all; v0 += p.piece) {
            const int64_t vp = std::min(p.piece, all - v0);
            if (!p.whole && p.piece < all) pack_w(v0, vp);   // otherwise the first pass packed it
            logits(v0, vp);
            a.p = Pb;
            a.p_plane = vp / 8 * p.rows;
            run_logits<PL, kProb>(a, p, x.d, vp, v0 == 0, "xent_prob", s);
            XentArgs w = a, h = a;
            w.B = h.B = Pb;
            w.b_rows = h.b_rows = p.rows;
            w.b_plane = h.b_plane = a.p_plane;
            w.A = H;
            w.a_rows = p.rows;
            w.a_plane = p.chunks * p.rows;
            w.k = p.dw_rows;
            w.dw = x.dw;
            w.ld_dw = x.ld_dw;
            w.d = x.d;
            w.dw_bf16 = BF;
            w.m_tiles = x.dw ? (int32_t)(p.width / p.bm) : 0;
            w.n_tiles = (int32_t)(vp / std::max<int64_t>(p.rn, 128));
            h.k = vp;
            h.part = (f32x4x *)(ws + p.part);
            h.split_stride = p.rows * p.width / 4;
            h.split_steps = p.split_steps;
            h.splits = p.splits;
            h.first = v0 == 0;
            h.m_tiles = x.dh ? (int32_t)(p.width / p.bm) : 0;
            h.n_tiles = (int32_t)(p.rows / p.rn);
            run_grads<PL>(w, h, p.bm, p.rn, s);
        }
        if (x.dh) {
            KernelTimer t("xent_dh_join", s);
            const int64_t total = p.rows * p.width / 4;
            const f32x4x *part = (const f32x4x *)(ws + p.part);
            const int32_t mt = (int32_t)(p.width / p.bm);
            const bool slices = total < 256 * 256;   // fewer workgroups than compute units
            const unsigned grid = grid_for(total, slices ? 32 : 256, 4096);
#define GNNAV_L(A, B, C, D)                                                                                               \
    do {                                                                                                                  \
        if (slices)                                                                                                       \
            hipLaunchKernelGGL((k_xent_dh<A, B, C, D, 8>), dim3(grid), dim3(256), 0, s, part, total, p.splits, total, mt, \
                               x.m, x.d, lse, inv, x.dh, x.ld_dh, BF);                                                    \
        else                                                                                                              \
            hipLaunchKernelGGL((k_xent_dh<A, B, C, D, 1>), dim3(grid), dim3(256), 0, s, part, total, p.splits, total, mt, \
                               x.m, x.d, lse, inv, x.dh, x.ld_dh, BF);                                                    \
    } while (0)
            if (p.rn == 256) GNNAV_L(4, 2, 2, 4);
            else if (p.bm == 128) GNNAV_L(2, 2, 2, 2);
            else GNNAV_L(1, 2, 2, 2);
#undef GNNAV_L
        }
    }
    GNNAV_HIP(hipGetLastError());
}

}  // namespace

size_t linear_xent_workspace(int64_t m, int64_t n_classes, int64_t d, bool bf16, bool grads) {
    return XentPlan(m, n_classes, d, bf16, grads, grads).total;
}

void launch_linear_xent(const LinearXentArgs &x, hipStream_t s) {
    const XentPlan p(x.m, x.n_classes, x.d, x.bf16, x.dh || x.dw, x.dh != nullptr);
    if (x.bf16) xent<1>(p, x, s);
    else xent<3>(p, x, s);
}

}  // namespace gnnav
