// Gated feed-forward blocks and their backward pass:
//
//   a = x Wg,  b = x Wu,  h = act(a) * b,  y = h Wd
//   dh = dy Wd^T,  da = dh * b * act'(a),  db = dh * act(a)
//   dx = da Wg^T + db Wu^T,  dWg = x^T da,  dWu = x^T db,  dWd = h^T dy
//
// Every product is one tile function on the matrix cores.  Its operands lie in memory as 16-byte chunks of 8
// consecutive columns at any distance from row to row and from chunk to chunk: bf16 matrices as the caller has them
// (row after row), and what the kernels write themselves (h, da, db) or pack chunk-major, [chunk][row], which
// stores and reads whole lines.  An operand's columns are summed over (a fragment is a chunk of a row) or its rows are
// (gfx950's transposing LDS reads take 4 rows of 16 columns).  Copies go to LDS asynchronously; past the end of a sum
// they read zeros, past the last row or chunk of an output the last one again.
//
// fp32 operands are split into three bf16 planes and multiplied with the six part products of bf16split.hpp.
//
// Rounding: a and b stay in fp32 (bf16 ones would cost da and db a second rounding of the results' own size): fp32 keeps them
// for the backward pass, bf16 multiplies x with Wg and Wu again in the tiles of dh, which is less time than 16 bytes an entry
// until d is some 900 and more past that (137 of 756 GFLOP at 8,192 x 1,024 x 4,096 x 1,024), and five times less memory at any d.  h, da
// and db are rounded once to the operands' type for the products that read them, or to two bf16 parts where a product's
// output has few entries.
#include <algorithm>
#include <cmath>

#include "bf16split.hpp"
#include "common.hpp"
#include "dma.hpp"
#include "gated_plan.hpp"
#include "lanes.hpp"

namespace gnnav {

namespace {

typedef float f32x16x __attribute__((ext_vector_type(16)));
typedef float f32x4x __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4x __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2x __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// Two groups of 4 values (as bf16 pairs) of a lane, of its row's columns c .. c + 3 and c + 8 .. c + 11, with those of
// lane ^ 32, c + 4 .. and c + 12 ..: the chunk of 8 from c for the lower lanes, from c + 8 for the upper ones.
__device__ __forceinline__ u32x4x join_chunk(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
    const auto lo = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
    return u32x4x{lo[0], hi[0], lo[1], hi[1]};
}

// act(a) and act'(a).  EXACT: fp32's functions; otherwise the hardware's exp2 and reciprocal, within 2^-21 of the value
// for |a| of a few tens (past them the results are 0 or a itself).
template <int ACT, bool EXACT>
__device__ __forceinline__ void activate(float a, float &value, float &slope) {
    if constexpr (ACT == GNNAV_ACT_SILU) {
        const float g = EXACT ? 1.f / (1.f + expf(-a))
                              : __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(a * -1.44269504088896340736f));
        value = a * g;
        slope = g + value * (1.f - g);
    } else if constexpr (ACT == GNNAV_ACT_GELU) {
        const float g = 0.5f * erfcf(a * -0.70710678118654752440f);
        value = a * g;
        slope = g + a * (0.39894228040143267794f * expf(-0.5f * a * a));
    } else {
        value = a > 0.f ? a : (a == a ? 0.f : a);
        slope = a > 0.f ? 1.f : 0.f;
    }
}

// The three bf16 parts of fp32 values, each rounded to nearest (bf16split.hpp's are cut): the second is then below 2^-9 of the
// value and the third below 2^-18, and what six products leave out below 2^-26 of theirs.  A value that would round to
// infinity is cut.
__device__ __forceinline__ void parts_of(float x0, float x1, uint32_t (&q)[3]) {
    q[0] = bf16_pair(x0, x1);
    const uint32_t u0 = __float_as_uint(x0), u1 = __float_as_uint(x1);
    if ((u0 & 0x7fffffffu) >= 0x7f7f8000u) q[0] = (q[0] & 0xffff0000u) | (u0 >> 16);
    if ((u1 & 0x7fffffffu) >= 0x7f7f8000u) q[0] = (q[0] & 0xffffu) | (u1 & 0xffff0000u);
    const float r0 = x0 - __uint_as_float(q[0] << 16), r1 = x1 - __uint_as_float(q[0] & 0xffff0000u);
    q[1] = bf16_pair(r0, r1);
    q[2] = bf16_pair(r0 - __uint_as_float(q[1] << 16), r1 - __uint_as_float(q[1] & 0xffff0000u));
}

// What copies read past the end of a sum.
__device__ const u32x4x kZeros = {0, 0, 0, 0};

// ------------------------------------------------------------------ packing
// rows x cols (row-major, 16-byte aligned rows) -> PL planes of chunks [chunk][row], zeros past the columns.
// One workgroup: 64 rows x 64 columns through LDS.  A launch takes up to five matrices.  Bound by memory and, where the matrices are
// small, by the launch: 12.8 million fp32 of four matrices 23 us, 5.6 TB/s; 100,000 x 100 30 us, 3.3 TB/s; a small one 5 us.
struct PackJob {
    const void *src;
    int64_t ld;
    int32_t rows, cols, col_tiles, end;   // end: workgroups of the jobs so far
    u32x4x *out;
};
// Norms of x's rows, times `scale`, and of wg's columns (`blocks` workgroups: `row_blocks`, and one for 16 columns).
struct NormJob {
    const float *x, *wg;
    int64_t ld_x, ld_wg, m;
    int32_t d, f, row_blocks, blocks;
    float scale, *rows, *columns;
};
struct PackJobs {
    PackJob job[5];
    NormJob norms;
};
// Sums in 64 bits, in which any fp32 entry's square is a number.  Rows of up to 256 columns take 16 lanes, longer ones a wavefront;
// 16 threads share a column.
__device__ __forceinline__ void norms_of(const NormJob &a, double *part) {   // part: 16 x 16 sums in LDS
    const int tid = threadIdx.x;
    if ((int32_t)blockIdx.x < a.row_blocks) {
        const int lanes = a.d <= 256 ? 16 : 64, at = tid % lanes, each = 256 / lanes;
        for (int64_t first = (int64_t)blockIdx.x * each; first < a.m; first += (int64_t)a.row_blocks * each) {
            const int64_t r = first + tid / lanes;
            double sum = 0;
            if (r < a.m) {
#pragma unroll 4
                for (int32_t c = at * 4; c < a.d; c += lanes * 4) {
                    const f32x4x v = *(const f32x4x *)(a.x + r * a.ld_x + c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const double w = c + e < a.d ? v[e] : 0.f;
                        sum = fma(w, w, sum);
                    }
                }
            }
#pragma unroll
            for (int q = 8; q > 0; q /= 2) sum += __shfl_xor(sum, q);
            if (lanes == 64) {
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
            }
            if (at == 0 && r < a.m) a.rows[r] = (float)(sqrt(sum) * a.scale);
        }
        return;
    }
    const int at = tid % 16, from = tid / 16;
    const int32_t c = ((int32_t)blockIdx.x - a.row_blocks) * 16 + at;
    double sum = 0;
    if (c < a.f) {
#pragma unroll 8
        for (int32_t r = from; r < a.d; r += 16) {
            const double v = a.wg[r * a.ld_wg + c];
            sum = fma(v, v, sum);
        }
    }
    part[from * 16 + at] = sum;
    __syncthreads();
    if (from == 0 && c < a.f) {
#pragma unroll
        for (int q = 1; q < 16; ++q) sum += part[q * 16 + at];
        a.columns[c] = (float)sqrt(sum);
    }
}
template <bool BF>
__global__ void __launch_bounds__(256) k_gated_pack(const PackJobs jobs) {
    constexpr int PL = BF ? 1 : 3;
    __shared__ u32x4x tile[PL][8][65];
    if constexpr (!BF)
        if ((int32_t)blockIdx.x < jobs.norms.blocks) return norms_of(jobs.norms, (double *)tile);
    const int32_t id = (int32_t)blockIdx.x - (BF ? 0 : jobs.norms.blocks);
    int32_t k = 0, base = 0;
    while (id >= jobs.job[k].end) base = jobs.job[k++].end;
    const PackJob &a = jobs.job[k];
    const int32_t t = id - base, rows = a.rows, d = a.cols, chunks = (d + 7) / 8;
    const int tid = threadIdx.x;
    const int64_t r0 = (int64_t)(t / a.col_tiles) * 64;
    const int32_t c0 = (t % a.col_tiles) * 8;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int lr = tid / 8 + 32 * q, lc = tid % 8;
        const int64_t r = r0 + lr;
        const int32_t col = (c0 + lc) * 8;
        const bool live = r < rows && col < d;
        if constexpr (BF) {
            u32x4x x = {0, 0, 0, 0};
            if (live) {
                x = *(const u32x4x *)((const uint16_t *)a.src + r * a.ld + col);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (col + 2 * e + 1 >= d) x[e] &= 0xffffu;
                    if (col + 2 * e >= d) x[e] = 0;
                }
            }
            tile[0][lc][lr] = x;
        } else {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.f;
            if (live) {
                const float *p = (const float *)a.src + r * a.ld + col;
                const f32x4x lo = *(const f32x4x *)p;
                f32x4x hi = {0.f, 0.f, 0.f, 0.f};
                if (col + 4 < d) hi = *(const f32x4x *)(p + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = col + e < d ? lo[e] : 0.f;
                    x[4 + e] = col + 4 + e < d ? hi[e] : 0.f;
                }
            }
            u32x4x part[3];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t q[3];
                parts_of(x[2 * e], x[2 * e + 1], q);
#pragma unroll
                for (int i = 0; i < 3; ++i) part[i][e] = q[i];
            }
#pragma unroll
            for (int i = 0; i < PL; ++i) tile[i][lc][lr] = part[i];
        }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2 * PL; ++q) {
        const int lc = (tid / 64) + 4 * (q & 1), lr = tid % 64, p = q >> 1;
        if (c0 + lc < chunks && r0 + lr < rows) a.out[((int64_t)p * chunks + c0 + lc) * rows + r0 + lr] = tile[p][lc][lr];
    }
}

// ------------------------------------------------------------------ products
// out[n][m] = sum over k of A(m, k) B(n, k).  The tile's M index is the output's column, N its row: a lane then holds four
// consecutive columns of a row.
// (no arrays: what is indexed at run time would be copied to memory)
struct Operand {
    const char *p0, *p1, *p2, *p3;   // matrices side by side along M (both projections: two), or one after the other along the sum
    int64_t row0, row1;          // bytes from a row to the next, of either side (one after the other along the sum: row0)
    int64_t chunk, plane;        // from a chunk, from a plane
    int32_t rows, chunks;        // what there is of each
};
// A sum: `segments` matrices one after the other, of `steps` steps each; the last step of each takes `tail` of its BK.
struct Sum {
    Operand A, B;
    int32_t segments, steps, tail;
};

struct Product {
    Sum s;
    int32_t m_tiles, n_tiles, splits, split_steps;
    int32_t n;                   // rows of the output
    // h, da and db: columns, 4-float groups [group][row] of a and b (nullable for h), chunks of h, or of da and db
    int32_t f;
    f32x4x *a, *b;
    u32x4x *h;
    const float *x, *wg;         // fp32's ReLU that keeps a: the operands of a, their strides and columns, the norms of x's rows,
    const float *row_norms, *column_norms;   // times what a norm's part may be off by, and of wg's columns
    int64_t ld_x, ld_wg;
    int32_t d;
    int64_t h_plane, second;     // chunks of a plane; from da to db
    int64_t low;                 // bf16: from the values to their second parts (0: none are kept)
    u32x4x *h2;                  // da and db, bf16: h in two parts (nullable)
    int64_t h2_low;
    // y and the gradients: columns of one output, where the second one starts (INT_MAX: there is none)
    int32_t cols, half;
    void *out[2];
    int64_t ld[2];
    bool bf16;
    f32x4x *part;                // splits > 1: the tiles' sums, split after split
    int64_t split_stride;        // float4s
};

// Wave grid WGM x WGN, each wavefront WMF x WNF MFMA blocks of 32 x 32; BK summed elements per stage, ST stages in LDS (small
// tiles, whose steps are shorter than a copy's way, take more).
template <int PL, int WMF, int WNF, int WGM, int WGN, int ST_ = 3>
struct Tile {
    static constexpr int BK = PL == 1 ? 32 : 16;
    static constexpr int NW = WGM * WGN, BM = 32 * WMF * WGM, BN = 32 * WNF * WGN;
    static constexpr int APC = BM * BK / 8, BPC = BN * BK / 8;   // chunks of a plane of a stage
    static constexpr int STAGE = PL * (APC + BPC);
    static constexpr int ST = ST_, LDS = ST * STAGE;
    static_assert(APC % 64 == 0 && BPC % 64 == 0, "whole wavefront copies");
};

// Tile of workgroup `id` of those of one product.  Workgroups go to the eight XCDs in turn; each XCD gets a contiguous run
// of the tiles, in groups of kGroup along M, so that the tiles it works on together share operands in its L2.
constexpr int kGroup = 8;
__device__ __forceinline__ bool tile_of(const Product &a, int32_t id, int32_t &split, int32_t &mt, int32_t &nt) {
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

// Four consecutive columns from c of row n: rounded to the type, zeros from the last column to the next 16-byte boundary.
__device__ __forceinline__ void store4(const Product &a, int64_t n, int32_t c, const f32x4x &v) {
    const int32_t which = c >= a.half ? 1 : 0;
    void *out = a.out[which];
    c -= which ? a.half : 0;
    if (n >= a.n || c >= (a.bf16 ? (a.cols + 7) / 8 * 8 : (a.cols + 3) / 4 * 4) || !out) return;
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = c + e < a.cols ? v[e] : 0.f;
    if (a.bf16) *(u32x2x *)((uint16_t *)out + n * a.ld[which] + c) = u32x2x{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
    else *(f32x4x *)((float *)out + n * a.ld[which] + c) = f32x4x{x[0], x[1], x[2], x[3]};
}

// 16 values of a lane (four groups of 4 columns, c + 8 g + 4 h) of row n as chunks of the operands' type.
template <int PL>
__device__ __forceinline__ void store_chunks(u32x4x *to, int64_t plane, int64_t rows, int32_t chunk, int32_t chunks, int64_t n,
                                             int h, const float (&x)[16]) {
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
        uint32_t w[2][2][3];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float f0 = x[4 * (g + i) + 2 * j], f1 = x[4 * (g + i) + 2 * j + 1];
                if constexpr (PL == 1) w[i][j][0] = bf16_pair(f0, f1);
                else parts_of(f0, f1, w[i][j]);
            }
#pragma unroll
        for (int pl = 0; pl < PL; ++pl) {
            const u32x4x v = join_chunk(w[0][0][pl], w[0][1][pl], w[1][0][pl], w[1][1][pl]);
            if (n < rows && chunk + g + h < chunks) to[pl * plane + (int64_t)(chunk + g + h) * rows + n] = v;
        }
    }
}

// ... and what bf16 leaves of the values, in bf16.
__device__ __forceinline__ void store_low(u32x4x *to, int64_t rows, int32_t chunk, int32_t chunks, int64_t n, int h, const float (&x)[16]) {
    float low[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        // (an infinite value leaves nothing)
        const float high = bf16_to_f32(bf16_rne(x[e]));
        low[e] = fabsf(high) < INFINITY ? x[e] - high : 0.f;
    }
    store_chunks<1>(to, 0, rows, chunk, chunks, n, h, low);
}

// A wavefront's copies of a sum's stages to LDS.  DUAL: A's two matrices side by side.  AT, BT: the operand's rows are summed
// over.  In LDS an operand whose columns are summed over lies row by row, its BK / 8 chunks exchanged by the row (16 rows read
// 256 bytes of distinct banks); one whose rows are lies in blocks of 8 of them, chunk by chunk, the two halves of a block
// exchanged by the chunk (32 lanes of a transposing read take 256 bytes of distinct banks).  Both copy whole runs from
// row-major and from chunk-major memory.  STRIDE: chunks from a stage to the next.
template <int PL_, int WMF_, int WNF_, int WGM_, int WGN_, int ST_, bool AT_, bool BT_, bool DUAL_, int STRIDE_ = Tile<PL_, WMF_, WNF_, WGM_, WGN_>::STAGE>
struct Feed {
    using C = Tile<PL_, WMF_, WNF_, WGM_, WGN_, ST_>;
    static constexpr int PL = PL_, WMF = WMF_, WNF = WNF_, WGM = WGM_, WGN = WGN_, STRIDE = STRIDE_;
    static constexpr bool AT = AT_, BT = BT_, DUAL = DUAL_;
    static constexpr int BK = C::BK, CK = BK / 8, APC = C::APC, BPC = C::BPC, BN = C::BN, INSTR = C::STAGE / 64, IN = (INSTR + C::NW - 1) / C::NW;
    static constexpr int AM = DUAL ? C::BM / 2 : C::BM, WA = DUAL ? WMF / 2 : WMF;   // columns of one matrix in the tile, blocks of a wavefront
    static_assert(!DUAL || WMF % 2 == 0, "both projections in one tile");
    int64_t m0, n0;
    const char *src[IN];   // source of the next step
    int64_t inc[IN];       // its advance
    int dst[IN];           // place in the stage
    uint32_t in_tail;      // whether the lane's is part of a last step
    int32_t segment, local;
    bool tail;             // of the step that is copied: it is such a one

    __device__ __forceinline__ int slot(int u) const {   // (the last wavefront may repeat the last copy)
        return std::min((int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * IN + u, INSTR - 1) * 64;
    }
    __device__ __forceinline__ void aim(const Sum &a, int32_t step) {
        // (every field is read, then chosen among: a choice of addresses would put the arguments into memory)
        const char *const a0 = a.A.p0, *const a1 = a.A.p1, *const a2 = a.A.p2, *const a3 = a.A.p3;
        const char *const b0 = a.B.p0, *const b1 = a.B.p1, *const b2 = a.B.p2, *const b3 = a.B.p3;
        const int64_t a_row0 = a.A.row0, a_row1 = a.A.row1, b_row = a.B.row0, a_chunk = a.A.chunk, b_chunk = a.B.chunk, a_plane = a.A.plane, b_plane = a.B.plane;
        const int32_t a_rows = a.A.rows, b_rows = a.B.rows, a_chunks = a.A.chunks, b_chunks = a.B.chunks;
        const char *const a_at = segment < 2 ? (segment < 1 ? a0 : a1) : (segment < 3 ? a2 : a3), *const b_at = segment < 2 ? (segment < 1 ? b0 : b1) : (segment < 3 ? b2 : b3);
        in_tail = 0;
#pragma unroll
        for (int u = 0; u < IN; ++u) {
            const int at = dst[u] = slot(u);
            const bool isB = at >= PL * APC;
            const int rel = at - (isB ? PL * APC : 0), pc = isB ? BPC : APC;
            const int plane = rel / pc;
            int s = rel % pc + (threadIdx.x & 63);
            bool side = false;   // the second of two matrices side by side
            if (DUAL && !isB) {
                side = rel % pc >= APC / 2;
                s -= side ? APC / 2 : 0;
            }
            const int64_t x0 = isB ? n0 : m0;
            const char *base = isB ? b_at + plane * b_plane : (DUAL ? (side ? a1 : a0) : a_at) + plane * a_plane;
            const int64_t row = isB ? b_row : DUAL && side ? a_row1 : a_row0, chunk = isB ? b_chunk : a_chunk;
            const int32_t rows = isB ? b_rows : a_rows, chunks = isB ? b_chunks : a_chunks;
            int k;
            if (isB ? BT : AT) {
                const int mcs = (isB ? BN : AM) / 8, mc = (s / 8) % mcs;
                k = s / (8 * mcs) * 8 + ((s % 8) ^ ((mc & 2) * 2));
                src[u] = base + ((int64_t)step * BK + k) * row + std::min<int64_t>(x0 / 8 + mc, chunks - 1) * chunk;
                inc[u] = BK * row;
            } else {
                const int r = s / CK, c = (s % CK) ^ (CK == 4 ? (r >> 2) & 3 : (r >> 3) & 1);
                k = c * 8;
                src[u] = base + std::min<int64_t>(x0 + r, rows - 1) * row + ((int64_t)step * CK + c) * chunk;
                inc[u] = CK * chunk;
            }
            in_tail |= (uint32_t)(k < a.tail) << u;
        }
    }
    // from step s0 on of the tile at m0, n0
    __device__ __forceinline__ void start(const Sum &a, int64_t m, int64_t n, int32_t s0) {
        m0 = m;
        n0 = n;
        segment = s0 / std::max(a.steps, 1);
        local = s0 - segment * a.steps;
        aim(a, local);
    }
    // before the copies of the next step: the next matrices, which lie as the ones before them, or the end of a sum
    __device__ __forceinline__ void prepare(const Sum &a) {
        if (local == a.steps) {
            local = 0;
            const char *const a0 = a.A.p0, *const a1 = a.A.p1, *const a2 = a.A.p2, *const a3 = a.A.p3;
            const char *const b0 = a.B.p0, *const b1 = a.B.p1, *const b2 = a.B.p2, *const b3 = a.B.p3;
            const int64_t a_on = segment < 1 ? a1 - a0 : segment < 2 ? a2 - a1 : a3 - a2, b_on = segment < 1 ? b1 - b0 : segment < 2 ? b2 - b1 : b3 - b2;
#pragma unroll
            for (int u = 0; u < IN; ++u) src[u] += (dst[u] >= PL * APC ? b_on : a_on) - a.steps * inc[u];
            ++segment;
        }
        tail = ++local == a.steps && a.tail < BK;
    }
    __device__ __forceinline__ void issue(u32x4x *S, int stage, int u) {
        const char *from = src[u];
        if (tail) from = in_tail >> u & 1 ? from : (const char *)&kZeros;
        dma16(from, &S[stage * STRIDE + dst[u]]);
        src[u] += inc[u];
    }
};

// The sum that follows one: its first two stages are copied over the end of the one before it.
template <class F>
struct Next {
    static constexpr int IN = F::IN;
    int64_t m0, n0;
    int32_t stages;   // 2, 1 where it has no more, 0 where nothing follows
};
struct Nothing {
    static constexpr int IN = 0;
    static constexpr int32_t stages = 0;
};

// The sum of one tile, T steps of `feed`, from operands in memory by way of LDS.  `ready`: the stage that holds its first step, and
// after it the next sum's; `primed`: stages that are on their way; stored: stores may have been issued behind their copies.
template <class F, class N, class G>
__device__ __forceinline__ void tile_sum(F &feed, const Sum &sum, int32_t T, u32x4x *S, f32x16x (&acc)[F::WMF][F::WNF], int &ready, int primed, bool stored, const N &follow,
                                         G &after, const Sum &after_sum) {
    constexpr int PL = F::PL, WMF = F::WMF, WNF = F::WNF, WGN = F::WGN, BK = F::BK, CK = F::CK, APC = F::APC, BPC = F::BPC, BN = F::BN;
    constexpr int AM = F::AM, WA = F::WA, IN = F::IN, NIN = N::IN, ST = F::C::ST;
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wid / WGN, wn = wid % WGN, h = lane >> 5, lr = lane & 31;
    // stage i of this sum, or i - T of the next one
    enum { kIdle, kOwn, kNext };
    auto whose = [&](int32_t i) __attribute__((always_inline)) { return i < T ? kOwn : i - T < follow.stages ? kNext : kIdle; };
    auto prepare = [&](int32_t i) __attribute__((always_inline)) {
        if (i < T) {
            feed.prepare(sum);
        } else if constexpr (NIN > 0) {
            if (i - T < follow.stages) {
                if (i == T) after.start(after_sum, follow.m0, follow.n0, 0);
                after.prepare(after_sum);
            }
        }
    };
    auto issue = [&](int mode, int stage, int u, bool last) __attribute__((always_inline)) {
        if (NIN == 0 || mode == kOwn) feed.issue(S, stage, u);
        if constexpr (NIN > 0) {
            if (mode == kNext) {
                if (u < NIN) after.issue(S, stage, u);
                if (last)
#pragma unroll
                    for (int more = IN; more < NIN; ++more) after.issue(S, stage, more);
            }
        }
        (void)last;
    };
    auto issue_all = [&](int32_t i, int stage, int from, int to) __attribute__((always_inline)) {
        const int mode = whose(i);
        if (mode != kIdle)
#pragma unroll
            for (int u = from; u < to; ++u) issue(mode, stage, u, u == IN - 1);
    };

#pragma unroll
    for (int i = 0; i < WMF; ++i)
#pragma unroll
        for (int j = 0; j < WNF; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    // lane parts of the transposing reads: chunk among 4, row among 4 (the swizzle is that of the chunk)
    const int tr_mc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    const int tr_at = tr_mc * 8 + (((lane & 15) >> 2) ^ ((tr_mc & 2) * 2));
    const int n_swz = CK == 4 ? (lr >> 2) & 3 : (lr >> 3) & 1;
    auto frag = [&](const u32x4x *plane, auto tr_, int tile, int x, int kk) __attribute__((always_inline)) -> bf16x8 {
        if constexpr (decltype(tr_)::value) {
            typedef __attribute__((address_space(3))) s16x4 lds4;
            const u32x4x *p = plane + ((2 * kk + h) * (tile / 8) + x / 8) * 8;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)((const char *)(p + tr_at) + 8 * (lane & 1)));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)((const char *)(p + (tr_at ^ 4)) + 8 * (lane & 1)));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(bf16x8, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
        } else {
            return __builtin_bit_cast(bf16x8, plane[(x + lr) * CK + ((2 * kk + h) ^ n_swz)]);
        }
    };
    struct Frags {
        bf16x8 a[WMF][PL], b[WNF][PL];
    };
    // fragment k of a step: B's, then A's, as the products need them
    constexpr int NF = (WMF + WNF) * PL;
    auto read = [&](Frags &f, int stage, int kk, int k) __attribute__((always_inline)) {
        const u32x4x *sa = &S[stage * F::STRIDE], *sb = sa + PL * APC;
        const int x = k / PL, p = k % PL;
        if (x < WNF) {
            f.b[x][p] = frag(sb + p * BPC, std::integral_constant<bool, F::BT>(), BN, wn * (32 * WNF) + 32 * x, kk);
        } else {
            const int i = x - WNF, matrix = i / WA;
            f.a[i][p] = frag(sa + p * APC + matrix * (APC / 2), std::integral_constant<bool, F::AT>(), AM, wm * (32 * WA) + 32 * (i % WA), kk);
        }
    };
    // The products of one fragment set.  Between them go, one at a time, the reads of the next set (first half) and
    // copies [c0, c1) of a stage to come (second half): in one burst behind the barrier they queue
    // up, and the wavefront's products wait with them.  Past the last stage the reads are idle ones.
    auto multiply = [&](const Frags &f, Frags &nxt, int from, int kk, int mode, int into, auto c0_, auto c1_) __attribute__((always_inline)) {
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
            if (k >= CUT && mode != kIdle)
#pragma unroll
                for (int q = C0 + (C1 - C0) * (k - CUT) / REST; q < C0 + (C1 - C0) * (k - CUT + 1) / REST; ++q) issue(mode, into, q, q == IN - 1);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Makes stage t readable: its copies are done, everywhere; those of the stage after it may not be.
    auto advance = [&](int32_t t) __attribute__((always_inline)) {
        if constexpr (ST == 3) {
            const int then = whose(t + 1);
            if (then == kOwn) wait_vm<IN>();
            else if (NIN > 0 && then == kNext) wait_vm<NIN>();
            else wait_vm<0>();
        } else {
            const int32_t behind = T - 1 - t;   // stages that may be on their way
            if (behind >= ST - 2) wait_vm<IN *(ST - 2)>();
            else if (ST > 5 && behind == 3) wait_vm<IN * 3>();
            else if (ST > 4 && behind == 2) wait_vm<IN * 2>();
            else if (behind == 1) wait_vm<IN>();
            else wait_vm<0>();
        }
        lds_barrier();
    };
    static_assert(ST >= 3 && ST <= 6 && (ST == 3 || NIN == 0) && IN * (ST - 2) < 64 && (BK == 16 || BK == 32), "the waits and the loop below");
    auto next = [](int stage) { return stage + 1 == ST ? 0 : stage + 1; };
    // One fragment set is multiplied while the next one is read, across the barrier between two stages.  Once
    // stage t is readable, stage t + ST - 1 is copied into the one read before it, over the products up to the next barrier.
    constexpr int FIRST = BK == 32 ? IN / 2 : IN;   // copies before a stage's second fragment set is read
    constexpr std::integral_constant<int, 0> kBegin{};
    constexpr std::integral_constant<int, FIRST> kMiddle{};
    constexpr std::integral_constant<int, IN> kEnd{};
    Frags f0, f1;
    int fill = ready;
    if (T > 0) {
#pragma unroll
        for (int k = 0; k < ST - 1; ++k) {
            if (k >= primed) {
                prepare(k);
                issue_all(k, fill, 0, IN);
            }
            fill = next(fill);
        }
        if (primed > 0 && stored) {
            wait_vm<0>();
            lds_barrier();
        } else {
            advance(0);
        }
        prepare(ST - 1);
        issue_all(ST - 1, fill, 0, FIRST);
        if constexpr (BK == 16) fill = next(fill);
#pragma unroll
        for (int q = 0; q < NF; ++q) read(f0, ready, 0, q);
    }
    // (while every copy is this sum's own, without asking)
    auto round = [&](int32_t &t, auto own_) __attribute__((always_inline)) {
        constexpr bool OWN = decltype(own_)::value;
        auto mode = [&](int32_t i) __attribute__((always_inline)) -> int { return OWN ? (int)kOwn : (int)whose(i); };
        auto go_on = [&](int32_t to) __attribute__((always_inline)) {
            if constexpr (OWN) {
                wait_vm<IN *(ST - 2)>();
                lds_barrier();
                feed.prepare(sum);
            } else if (to < T) {
                advance(to);
                prepare(to + ST - 1);
            }
        };
        if constexpr (BK == 32) {
            multiply(f0, f1, ready, 1, mode(t + ST - 1), fill, kMiddle, kEnd);
            fill = next(fill);
            ready = next(ready);
            go_on(++t);
            multiply(f1, f0, ready, 0, OWN || t < T ? mode(t + ST - 1) : kIdle, fill, kBegin, kMiddle);
        } else {
            ready = next(ready);
            go_on(++t);
            multiply(f0, f1, ready, 0, OWN || t < T ? mode(t + ST - 1) : kIdle, fill, kBegin, kEnd);
            fill = next(fill);
            if (!OWN && t >= T) return;
            ready = next(ready);
            go_on(++t);
            multiply(f1, f0, ready, 0, OWN || t < T ? mode(t + ST - 1) : kIdle, fill, kBegin, kEnd);
            fill = next(fill);
        }
    };
    int32_t t = 0;
    while (t + (BK == 32 ? ST : ST + 1) < T) round(t, std::true_type());
    while (t < T) round(t, std::false_type());
}

// ReLU's slope jumps at 0: where the rounding of a sum in fp32 decides which side a is on, da is 0 instead of a whole term, or the
// other way round.  Values below sure_below |x's row| |wg's column| are summed again in 64 bits by the whole wavefront.  A sum's terms
// are together at most that product of norms, its running sum at most half of it where they cancel in the worst order, and
// each of some 6 d / 16 additions rounds it by a part of 2^-24: errors grow with sqrt(d).  Measured over 2 million
// entries each, in sqrt(d) 2^-24 of the norms: terms that rise to their largest sum and fall again 0.10 as a spread, 0.6 at the
// most at 40 columns, 0.08 and 0.4 at 1,024; in random order some 0.25 2^-24 at any d, 4 2^-24 at the most.
// Random entries are summed again at d x 5 10^-8 of them, and at d x 5 10^-5 where features lie 1,000 spreads from zero and columns sum
// to nothing.  A 3,000 x 1,024 x 2,048 block's h takes 153 us (SiLU's 138) and its packing 3 more; with features 10, 100 and 1,000
// spreads from zero 183, 340 and 1,490.  Without it 1 of 5.6 million signs of a random 1,362 x 333 x 4,096 block is wrong, which
// is 6e-4 of dWg's norm, and 1 in 100 of a 33 x 4,096 x 64 one whose terms cancel.
constexpr float sure_below(float root_d) { return std::max(root_d, 8.f) * 0x1p-24f; }
template <int WA, int WNF>
__device__ __forceinline__ void sure_signs(const Product &a, int32_t c0, int64_t n, int j, int h, f32x16x (&acc)[2 * WA][WNF]) {
    const float row = n < a.n ? a.row_norms[n] : 0.f;
#pragma unroll
    for (int i = 0; i < WA; ++i) {
        uint32_t near = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int32_t c = c0 + 32 * i + 8 * g + 4 * h;
            f32x4x column = {0.f, 0.f, 0.f, 0.f};
            if (c < a.f) column = *(const f32x4x *)(a.column_norms + c);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                near |= (uint32_t)(c + e < a.f && fabsf(acc[i][j][4 * g + e]) < row * column[e]) << (4 * g + e);
        }
        uint64_t lanes;
        while ((lanes = __ballot(near != 0)) != 0) {
            const int from = __builtin_ctzll(lanes), r = __builtin_ctz(__builtin_amdgcn_readlane(near, from));
            const int64_t row = n - (threadIdx.x & 31) + (from & 31);
            const float *const x = a.x + row * a.ld_x, *const w = a.wg + c0 + 32 * i + 8 * (r / 4) + 4 * (from >> 5) + r % 4;
            double sum = 0;
            for (int32_t k = threadIdx.x & 63; k < a.d; k += 64) sum = fma((double)x[k], (double)w[k * a.ld_wg], sum);
#pragma unroll
            for (int q = 32; q > 0; q /= 2) sum += __shfl_xor(sum, q);
            const bool mine = (int)(threadIdx.x & 63) == from;
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = mine && q == r ? (float)sum : acc[i][j][q];
            near &= mine ? near - 1 : ~0u;
        }
    }
}

// h = act(x Wg) * (x Wu) for one tile from both sums, kept for the product with Wd, and a and b where they are kept.  WA: blocks
// of a wavefront along f.
template <int PL, int WA, int WNF, int WGM, int WGN, int ACT>
__device__ __forceinline__ void gate_store(const Product &a, int64_t m0, int64_t n0, f32x16x (&acc)[2 * WA][WNF]) {
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, lr = lane & 31;
    const int32_t mw = (int32_t)m0 + wid / WGN * (32 * WA);
    const int64_t nw = n0 + wid % WGN * (32 * WNF);
    const int32_t chunks = (a.f + 7) / 8;
    const bool whole = m0 + 32 * WA * WGM <= a.f;   // no column past the last
#pragma unroll
    for (int j = 0; j < WNF; ++j) {
        const int64_t n = nw + 32 * j + lr;
        if constexpr (PL == 3 && ACT == GNNAV_ACT_RELU)
            if (a.a) sure_signs<WA, WNF>(a, mw, n, j, h, acc);
#pragma unroll
        for (int i = 0; i < WA; ++i) {
            float x[16];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int32_t c = mw + 32 * i + 8 * g + 4 * h;
                if (PL == 3 && a.a && n < a.n && c < chunks * 8) {
                    f32x4x va, vb;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        va[e] = acc[i][j][4 * g + e];
                        vb[e] = acc[i + WA][j][4 * g + e];
                    }
                    a.a[(int64_t)(c / 4) * a.n + n] = va;
                    a.b[(int64_t)(c / 4) * a.n + n] = vb;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float value, slope;
                    activate<ACT, PL == 3>(acc[i][j][4 * g + e], value, slope);
                    x[4 * g + e] = value * acc[i + WA][j][4 * g + e];
                }
            }
            if (!whole)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (mw + 32 * i + 8 * (r / 4) + 4 * h + r % 4 >= a.f) x[r] = 0.f;
            store_chunks<PL>(a.h, a.h_plane, a.n, (mw + 32 * i) / 8, chunks, n, h, x);
            if (PL == 1 && a.low) store_low(a.h + a.low, a.n, (mw + 32 * i) / 8, chunks, n, h, x);
        }
    }
}

// da and db of one tile from dh = dy Wd^T; a and b are read (fp32) or were multiplied again (bf16).
template <int PL, int WA, int WNF, int WGM, int WGN, int ACT>
__device__ __forceinline__ void dgate_store(const Product &a, int64_t m0, int64_t n0, const f32x16x (&ab)[PL == 1 ? 2 * WA : 1][PL == 1 ? WNF : 1],
                                            const f32x16x (&acc)[WA][WNF]) {
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, lr = lane & 31;
    const int32_t mw = (int32_t)m0 + wid / WGN * (32 * WA);
    const int64_t nw = n0 + wid % WGN * (32 * WNF);
    const int32_t chunks = (a.f + 7) / 8;
    const bool whole = m0 + 32 * WA * WGM <= a.f;
#pragma unroll
    for (int j = 0; j < WNF; ++j) {
        const int64_t n = nw + 32 * j + lr;
#pragma unroll
        for (int i = 0; i < WA; ++i) {
            float x[16], z[16], v[16];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int32_t c = mw + 32 * i + 8 * g + 4 * h;
                f32x4x va = {0.f, 0.f, 0.f, 0.f}, vb = va;
                if constexpr (PL == 1) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        va[e] = ab[i][j][4 * g + e];
                        vb[e] = ab[i + WA][j][4 * g + e];
                    }
                } else if (n < a.n && c < chunks * 8) {
                    va = a.a[(int64_t)(c / 4) * a.n + n];
                    vb = a.b[(int64_t)(c / 4) * a.n + n];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float value, slope;
                    activate<ACT, PL == 3>(va[e], value, slope);
                    const float dh = acc[i][j][4 * g + e];
                    x[4 * g + e] = dh * vb[e] * slope;
                    z[4 * g + e] = dh * value;
                    v[4 * g + e] = value * vb[e];
                }
            }
            if (!whole)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (mw + 32 * i + 8 * (r / 4) + 4 * h + r % 4 >= a.f) x[r] = z[r] = v[r] = 0.f;
            const int32_t chunk = (mw + 32 * i) / 8;
            store_chunks<PL>(a.h, a.h_plane, a.n, chunk, chunks, n, h, x);
            store_chunks<PL>(a.h + a.second, a.h_plane, a.n, chunk, chunks, n, h, z);
            if (PL == 1 && a.low) {
                store_low(a.h + a.low, a.n, chunk, chunks, n, h, x);
                store_low(a.h + a.second + a.low, a.n, chunk, chunks, n, h, z);
            }
            if (PL == 1 && a.h2) {
                store_chunks<1>(a.h2, 0, a.n, chunk, chunks, n, h, v);
                store_low(a.h2 + a.h2_low, a.n, chunk, chunks, n, h, v);
            }
        }
    }
}

// Tile `id` of a product that goes to the caller, or to parts.
template <int PL, int WMF, int WNF, int WGM, int WGN, int ST, bool AT, bool BT>
__device__ __forceinline__ void out_tile(const Product &a, int32_t id, u32x4x *S) {
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, lr = lane & 31;
    int32_t split, mt, nt;
    if (!tile_of(a, id, split, mt, nt)) return;
    const int64_t m0 = (int64_t)mt * (32 * WMF * WGM), n0 = (int64_t)nt * (32 * WNF * WGN);
    const int32_t s0 = split * a.split_steps, T = std::max(0, std::min(a.split_steps, a.s.segments * a.s.steps - s0));
    f32x16x acc[WMF][WNF];
    Feed<PL, WMF, WNF, WGM, WGN, ST, AT, BT, false> feed;
    int ready = 0;
    Nothing nothing;
    if (T > 0) feed.start(a.s, m0, n0, s0);
    tile_sum(feed, a.s, T, S, acc, ready, 0, false, nothing, feed, a.s);
    const int64_t mw = m0 + wid / WGN * (32 * WMF), nw = n0 + wid % WGN * (32 * WNF);
    f32x4x *part = a.part;
    if (part) part += split * a.split_stride + ((int64_t)(nt * a.m_tiles + mt) * (WGM * WGN) + wid) * (WMF * WNF * 4 * 64) + lane;
#pragma unroll
    for (int j = 0; j < WNF; ++j)
#pragma unroll
        for (int i = 0; i < WMF; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4x v = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                if (part) part[((i * WNF + j) * 4 + g) * 64] = v;
                else store4(a, nw + 32 * j + lr, (int32_t)(mw + 32 * i + 8 * g + 4 * h), v);
            }
}

// A workgroup takes tile after tile, the next one's first copies under way while one's results are formed and stored.
// (Tiles of more than three stages are for launches that have one a workgroup.)  8,192 x 1,024 x 4,096 bf16: 137 to 163 us, 840 to 1,000
// TFLOP/s, bound by the matrix cores' power; 65,537 x 256 x 1,024: 110 to 130 us (110 and 117 with a tile a workgroup on one
// card), bound by a tile's ends, its sum having eight steps; 99,603 x 128 x 512: 66 to 69 us (73), four steps and SiLU; with
// GELU, in fp32's accuracy, the block's two launches take 149 us instead of 88.
template <int PL, int WMF, int WNF, int WGM, int WGN, int ST, int ACT>
__global__ void __launch_bounds__(64 * WGM * WGN, 2) k_gated_gate(const Product a, int32_t ids) {
    constexpr int WA = WMF / 2;
    constexpr int64_t AM = 32 * WA * WGM, BN = 32 * WNF * WGN;
    __shared__ u32x4x S[Tile<PL, WMF, WNF, WGM, WGN, ST>::LDS];
    int32_t split, mt, nt, id = blockIdx.x;
    if (!tile_of(a, id, split, mt, nt)) return;
    using F = Feed<PL, WMF, WNF, WGM, WGN, ST, true, false, true>;
    F feed;
    feed.start(a.s, mt * AM, nt * BN, 0);
    f32x16x acc[WMF][WNF];
    int ready = 0, primed = 0;
    if constexpr (ST > 3) {
        const Nothing nothing;
        tile_sum(feed, a.s, a.s.steps, S, acc, ready, 0, false, nothing, feed, a.s);
        gate_store<PL, WA, WNF, WGM, WGN, ACT>(a, mt * AM, nt * BN, acc);
    } else {
        while (true) {
            int32_t m2 = 0, n2 = 0;
            id += gridDim.x;
            const bool more = id < ids && tile_of(a, id, split, m2, n2);
            const Next<F> next = {m2 * AM, n2 * BN, more ? std::min(a.s.steps, 2) : 0};
            tile_sum(feed, a.s, a.s.steps, S, acc, ready, primed, true, next, feed, a.s);
            gate_store<PL, WA, WNF, WGM, WGN, ACT>(a, mt * AM, nt * BN, acc);
            if (!more) break;
            primed = next.stages;
            mt = m2;
            nt = n2;
        }
    }
}
// 8,192 x 4,096 x 1,024 bf16: 105 to 134 us, 510 to 650 TFLOP/s: 256 tiles, one a unit, which leaves a step's latencies open; in tiles of 256 x 256
// two splits' parts would take as long.  99,603 x 512 x 64: 26 us, 4.4 TB/s.
template <int PL, int WMF, int WNF, int WGM, int WGN, int ST>
__global__ void __launch_bounds__(64 * WGM * WGN, 2) k_gated_down(const Product a) {
    __shared__ u32x4x S[Tile<PL, WMF, WNF, WGM, WGN, ST>::LDS];
    out_tile<PL, WMF, WNF, WGM, WGN, ST, true, false>(a, blockIdx.x, S);
}
// fp32 takes tile after tile too; bf16, whose three sums leave no registers for the next tile's copies, one: the copies of dh's sum
// follow those of a and b.  8,192 x 1,024 x 4,096 x 1,024 bf16: 221 to 264 us, 780 to 930 TFLOP/s; 65,537 x 256 x 1,024 x 256: 196 to 222, its
// stores 1.4 TB/s beside eight and sixteen steps.
template <int PL, int WA, int WNF, int WGM, int WGN, int ST, int ACT>
__global__ void __launch_bounds__(64 * WGM * WGN, 2) k_gated_dgate(const Product a, const Sum again, int32_t ids) {
    constexpr int64_t AM = 32 * WA * WGM, BN = 32 * WNF * WGN;
    using C = Tile<PL, PL == 1 ? 2 * WA : WA, WNF, WGM, WGN, ST>;
    __shared__ u32x4x S[C::LDS];
    int32_t split, mt, nt, id = blockIdx.x;
    if (!tile_of(a, id, split, mt, nt)) return;
    using F = Feed<PL, WA, WNF, WGM, WGN, ST, false, false, false, C::STAGE>;
    F feed;
    f32x16x ab[PL == 1 ? 2 * WA : 1][PL == 1 ? WNF : 1], acc[WA][WNF];
    int ready = 0, primed = 0;
    const Nothing nothing;
    if constexpr (PL == 1) {
        using A = Feed<PL, 2 * WA, WNF, WGM, WGN, ST, true, false, true>;
        A first;
        first.start(again, mt * AM, nt * BN, 0);
        if constexpr (ST == 3) {
            const Next<F> dh = {mt * AM, nt * BN, std::min(a.s.steps, 2)};
            tile_sum(first, again, again.steps, S, ab, ready, 0, false, dh, feed, a.s);
            primed = dh.stages;
        } else {
            tile_sum(first, again, again.steps, S, ab, ready, 0, false, nothing, first, again);
            lds_barrier();   // (the last fragments are read)
            feed.start(a.s, mt * AM, nt * BN, 0);
        }
        tile_sum(feed, a.s, a.s.steps, S, acc, ready, primed, false, nothing, feed, a.s);
        dgate_store<PL, WA, WNF, WGM, WGN, ACT>(a, mt * AM, nt * BN, ab, acc);
    } else if constexpr (ST > 3) {
        feed.start(a.s, mt * AM, nt * BN, 0);
        tile_sum(feed, a.s, a.s.steps, S, acc, ready, 0, false, nothing, feed, a.s);
        dgate_store<PL, WA, WNF, WGM, WGN, ACT>(a, mt * AM, nt * BN, ab, acc);
    } else {
        feed.start(a.s, mt * AM, nt * BN, 0);
        while (true) {
            int32_t m2 = 0, n2 = 0;
            id += gridDim.x;
            const bool more = id < ids && tile_of(a, id, split, m2, n2);
            const Next<F> next = {m2 * AM, n2 * BN, more ? std::min(a.s.steps, 2) : 0};
            tile_sum(feed, a.s, a.s.steps, S, acc, ready, primed, true, next, feed, a.s);
            primed = next.stages;
            dgate_store<PL, WA, WNF, WGM, WGN, ACT>(a, mt * AM, nt * BN, ab, acc);
            if (!more) break;
            mt = m2;
            nt = n2;
        }
    }
}
// dx and the weights' gradients in one launch (8,192 x 1,024 x 4,096 x 1,024 bf16: 307 to 352 us, 980 to 1,120 TFLOP/s; 65,537 x 256 x
// 1,024 x 256: 218 to 233 us, 880 to 940 TFLOP/s and 4 TB/s): workgroups below `w_at` take dx's tiles, below `d_at` those of dWg and dWu.
template <int PL, int WMF, int WNF, int WGM, int WGN, int ST>
__global__ void __launch_bounds__(64 * WGM * WGN, 2) k_gated_grads(const Product x, const Product w, const Product d, int32_t w_at,
                                                                   int32_t d_at) {
    __shared__ u32x4x S[Tile<PL, WMF, WNF, WGM, WGN, ST>::LDS];
    const int32_t id = blockIdx.x;
    if (id < w_at) out_tile<PL, WMF, WNF, WGM, WGN, ST, false, false>(x, id, S);
    else if (id < d_at) out_tile<PL, WMF, WNF, WGM, WGN, ST, true, true>(w, id - w_at, S);
    else out_tile<PL, WMF, WNF, WGM, WGN, ST, true, true>(d, id - d_at, S);
}

// The sum of the splits' parts, in their order.  A launch takes up to three products.
struct JoinJobs {
    Product p[3];
    int64_t end[3];   // float4s of the products so far
};
template <int WMF, int WNF, int WGM, int WGN>
__global__ void __launch_bounds__(256) k_gated_join(const JoinJobs jobs) {
    constexpr int NW = WGM * WGN, BM = 32 * WMF * WGM, BN = 32 * WNF * WGN;
    // 256 threads take a block of 32 x 32: 8 consecutive ones four columns each of one row
    const int row = threadIdx.x / 8, group = threadIdx.x % 8;
    for (int64_t at = (int64_t)blockIdx.x * 256; at < jobs.end[2]; at += (int64_t)gridDim.x * 256) {
        const int k = at < jobs.end[0] ? 0 : at < jobs.end[1] ? 1 : 2;
        const Product &a = jobs.p[k];
        int64_t r = at - (k ? jobs.end[k - 1] : 0);
        const f32x4x *part = a.part + r + group * 32 + row;   // (register group g, half h of the lanes: 64 g + 32 h)
        f32x4x v = {0.f, 0.f, 0.f, 0.f};
        int32_t s = 0;
        for (; s + 8 <= a.splits; s += 8) {
            f32x4x x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = part[(s + i) * a.split_stride];
#pragma unroll
            for (int i = 0; i < 8; ++i) v += x[i];
        }
        for (; s < a.splits; ++s) v += part[s * a.split_stride];
        r >>= 8;
        const int fj = (int)(r % WNF), fi = (int)(r / WNF % WMF);
        r /= WNF * WMF;
        const int wid = (int)(r % NW);
        r /= NW;
        const int32_t mt = (int32_t)(r % a.m_tiles), nt = (int32_t)(r / a.m_tiles);
        store4(a, (int64_t)nt * BN + wid % WGN * (32 * WNF) + 32 * fj + row, mt * BM + wid / WGN * (32 * WMF) + 32 * fi + 4 * group, v);
    }
}

// ------------------------------------------------------------------ few rows
// At most 8 rows, nothing kept: the weights are read once as they lie and multiplied in fp32; h stays in fp32.  A workgroup
// takes 32 columns, its lanes 16 bytes of a row each, the wavefronts different rows; the sums over the rows are joined in
// registers and then in LDS.  Two launches: h, from both projections (MATS = 2), and y.
// 1 x 1,024 x 4,096 x 1,024 bf16: 12 us over the same weights again, 19 over four sets of them in turn, 30 over 24 sets, which no cache
// holds (24, 24 and 26 with the tiles); the weights' way at 4.72 TB/s is 5.3.  The columns / 32 workgroups, 128 and 32 here, leave most of
// the 256 units idle, and a round of 1,024 summed rows is not on its way while the one before it is multiplied.
struct FewArgs {
    const void *x;             // rows that are multiplied: of the operands' type, or h in fp32
    int64_t ld_x;
    const void *w, *w2;
    int64_t ld_w, ld_w2;
    int32_t m, k, cols;
    float *h;                  // [m][cols]
    void *y;
    int64_t ld_y;
};
constexpr int kFewColumns = 32, kFewChunk = 1024;   // summed rows that are staged at a time

template <bool BF, bool XF, int MR, int MATS, int ACT>
__global__ void __launch_bounds__(MATS == 2 ? 512 : 1024) k_gated_few(const FewArgs a) {
    constexpr int NW = MATS == 2 ? 8 : 16, PER = BF ? 8 : 4, CL = kFewColumns / PER, RW = 64 / CL, ROUND = NW * RW, ROUNDS = kFewChunk / ROUND;
    __shared__ float X[MR][kFewChunk];
    __shared__ float red[NW][MATS][MR][kFewColumns];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, cl = lane % CL, rl = lane / CL;
    // workgroups go to the eight XCDs in turn: each takes neighbouring columns, whose lines its L2 shares
    const int groups = gridDim.x, per = groups / 8, extra = groups % 8, xcd = blockIdx.x % 8;
    const int group = xcd * per + std::min(xcd, extra) + blockIdx.x / 8;
    const int32_t c = group * kFewColumns + cl * PER;
    const bool here = c < a.cols;
    float acc[MATS][MR][PER];
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int r = 0; r < MR; ++r)
#pragma unroll
            for (int e = 0; e < PER; ++e) acc[q][r][e] = 0.f;
    for (int32_t k0 = 0; k0 < a.k; k0 += kFewChunk) {
        u32x4x w[MATS][ROUNDS];
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            const int64_t k = k0 + i * ROUND + wid * RW + rl;
#pragma unroll
            for (int q = 0; q < MATS; ++q) {
                w[q][i] = u32x4x{0, 0, 0, 0};
                if (here && k < a.k) {
                    const char *at = (const char *)(q ? a.w2 : a.w) + (k * (q ? a.ld_w2 : a.ld_w) + c) * (BF ? 2 : 4);
                    w[q][i] = *(const u32x4x *)at;
                }
            }
        }
        if (k0 > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < MR; ++r)
            for (int i = tid; i < kFewChunk; i += 64 * NW) {
                float v = 0.f;
                if (r < a.m && k0 + i < a.k) {
                    if constexpr (XF) v = ((const float *)a.x)[r * a.ld_x + k0 + i];
                    else v = bf16_to_f32(((const uint16_t *)a.x)[r * a.ld_x + k0 + i]);
                }
                X[r][i] = v;
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            const int at = i * ROUND + wid * RW + rl;
            if (k0 + at >= a.k) continue;   // (past the end the staged zeros would meet what is not the weights')
#pragma unroll
            for (int q = 0; q < MATS; ++q) {
                float v[PER];
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    if constexpr (BF) v[e] = __uint_as_float(e & 1 ? w[q][i][e / 2] & 0xffff0000u : w[q][i][e / 2] << 16);
                    else v[e] = __uint_as_float(w[q][i][e]);
                }
#pragma unroll
                for (int r = 0; r < MR; ++r)
#pragma unroll
                    for (int e = 0; e < PER; ++e) acc[q][r][e] = __builtin_fmaf(v[e], X[r][at], acc[q][r][e]);
            }
        }
    }
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int r = 0; r < MR; ++r)
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                float v = acc[q][r][e];
                auto f = [](uint32_t u) { return __uint_as_float(u); };
                if constexpr (CL <= 4) v += f(lane_xor<4>(__float_as_uint(v)));
                v += f(lane_xor<8>(__float_as_uint(v)));
                const LanePair p = lane_pair<16>(__float_as_uint(v));
                v = f(p.low) + f(p.high);
                const LanePair z = lane_pair<32>(__float_as_uint(v));
                v = f(z.low) + f(z.high);
                if (rl == 0) red[wid][q][r][cl * PER + e] = v;
            }
    __syncthreads();
    for (int i = tid; i < MR * kFewColumns; i += 64 * NW) {
        const int r = i / kFewColumns, at = i % kFewColumns;
        const int64_t col = (int64_t)group * kFewColumns + at;
        if (r >= a.m) break;
        float v[MATS];
#pragma unroll
        for (int q = 0; q < MATS; ++q) {
            v[q] = red[0][q][r][at];
#pragma unroll
            for (int w = 1; w < NW; ++w) v[q] += red[w][q][r][at];
        }
        if constexpr (MATS == 2) {
            float value, slope;
            activate<ACT, true>(v[0], value, slope);
            if (col < a.cols) a.h[r * (int64_t)a.cols + col] = value * v[MATS - 1];
        } else if (col < (a.cols + 16 / (BF ? 2 : 4) - 1) / (16 / (BF ? 2 : 4)) * (16 / (BF ? 2 : 4))) {
            const float out = col < a.cols ? v[0] : 0.f;   // (zeros to the next 16-byte boundary)
            if constexpr (BF) ((uint16_t *)a.y)[r * a.ld_y + col] = bf16_rne(out);
            else ((float *)a.y)[r * a.ld_y + col] = out;
        }
    }
}

// ------------------------------------------------------------------ host
unsigned ids_of(const Product &a) {   // workgroups of a product, whole rounds over the XCDs
    return (unsigned)up((int64_t)a.m_tiles * a.n_tiles * a.splits, 8);
}

// rows x cols of the caller's, as it lies or packed at `at`
Operand operand(const void *p, int64_t ld, int64_t rows, int64_t cols, const char *packed_at) {
    Operand o = {};
    o.rows = (int32_t)rows;
    o.chunks = (int32_t)(up(cols, 8) / 8);
    o.chunk = packed_at ? rows * 16 : 16;
    o.plane = packed_at ? o.chunk * o.chunks : 0;
    o.p0 = o.p1 = o.p2 = o.p3 = packed_at ? packed_at : (const char *)p;
    o.row0 = o.row1 = packed_at ? 16 : ld * 2;
    return o;
}
// ... and a second matrix of the same sizes (and so on, in turn)
void second(Operand &o, const void *p, int64_t ld, const char *packed_at) {
    o.p1 = o.p3 = packed_at ? packed_at : (const char *)p;
    o.row1 = packed_at ? 16 : ld * 2;
}

void sum_over(Sum &p, int64_t k, int bk, int32_t segments) {
    p.segments = segments;
    p.steps = (int32_t)((k + bk - 1) / bk);
    p.tail = (int32_t)(k - (int64_t)(p.steps - 1) * bk);
}
void cut(Product &p, int32_t splits) {
    p.splits = splits;
    p.split_steps = (int32_t)((p.s.segments * (int64_t)p.s.steps + splits - 1) / splits);
}
void tiles_of(Product &p, int64_t rows, int64_t cols, const Shape &e) {
    p.n = (int32_t)rows;
    p.n_tiles = (int32_t)(up(rows, e.bn) / e.bn);
    p.m_tiles = (int32_t)(up(cols, e.bm) / e.bm);
}
void writes(Product &p, void *out, int64_t ld, int64_t cols, bool bf16) {
    p.out[0] = out;
    p.out[1] = nullptr;
    p.half = INT_MAX;
    p.ld[0] = p.ld[1] = ld;
    p.cols = (int32_t)cols;
    p.bf16 = bf16;
}
void parts_at(Product &p, char *at, const Shape &e) {
    p.split_stride = (int64_t)p.n_tiles * p.m_tiles * e.bn * e.bm / 4;
    p.part = p.splits > 1 ? (f32x4x *)at : nullptr;
}

struct Packer {
    PackJobs jobs = {};
    int n = 0;
    int32_t blocks = 0;
    void add(const void *src, int64_t ld, int64_t rows, int64_t cols, char *out) {
        if (rows == 0) return;
        PackJob &j = jobs.job[n++];
        j.src = src;
        j.ld = ld;
        j.rows = (int32_t)rows;
        j.cols = (int32_t)cols;
        j.col_tiles = (int32_t)(up(cols, 64) / 64);
        blocks += (int32_t)(up(rows, 64) / 64 * j.col_tiles);
        j.end = blocks;
        j.out = (u32x4x *)out;
    }
    void add_norms(const GatedArgs &x, float scale, float *rows, float *columns) {
        const int32_t row_blocks = (int32_t)grid_for(x.m, x.d <= 256 ? 16 : 4, 4096);
        jobs.norms = {(const float *)x.x, (const float *)x.wg, x.ld_x, x.ld_wg, x.m, (int32_t)x.d, (int32_t)x.f, row_blocks,
                      row_blocks + (int32_t)(up(x.f, 16) / 16), scale, rows, columns};
    }
    void run(bool bf16, hipStream_t s) {
        if (blocks == 0) return;
        KernelTimer t("gated_pack", s);
        if (bf16) hipLaunchKernelGGL(k_gated_pack<true>, dim3((unsigned)blocks), dim3(256), 0, s, jobs);
        else hipLaunchKernelGGL(k_gated_pack<false>, dim3((unsigned)(blocks + jobs.norms.blocks)), dim3(256), 0, s, jobs);
    }
};

#define GNNAV_TILES(PL, WHICH, L)                           \
    do {                                                    \
        if constexpr (PL == 1) {                            \
            if (WHICH == kLarge) L(1, 4, 2, 2, 4, 3);       \
            else if (WHICH == kWide) L(1, 2, 2, 2, 4, 3);   \
            else if (WHICH == kMedium) L(1, 1, 2, 2, 2, 4); \
            else L(1, 2, 1, 1, 2, 6);                       \
        } else {                                            \
            if (WHICH == kWide) L(3, 2, 2, 2, 2, 3);        \
            else if (WHICH == kMedium) L(3, 1, 2, 2, 2, 4); \
            else L(3, 2, 1, 1, 2, 6);                       \
        }                                                   \
    } while (0)

// Workgroups of a launch that takes tile after tile: `each` a unit, whole rounds over the XCDs.
unsigned places_of(const Product &a, int each, hipStream_t s) {
    return std::min<unsigned>(ids_of(a), (unsigned)up((int64_t)stream_units(s) * each, 8));
}
template <int PL, int ACT>
void run_gate(const Product &p, int which, hipStream_t s) {
    KernelTimer t("gated_gate", s);
#define GNNAV_L(A, B, C, D, ST, EACH)                                                                                   \
    hipLaunchKernelGGL((k_gated_gate<PL, A, B, C, D, ST, ACT>), dim3(ST == 3 ? places_of(p, EACH, s) : ids_of(p)), dim3(64 * C * D), 0, s, p, \
                       (int32_t)ids_of(p))
    if constexpr (PL == 1) {
        if (which == kLarge) GNNAV_L(4, 2, 2, 4, 3, 1);
        else if (which == kMedium) GNNAV_L(2, 2, 2, 2, 3, 3);
        else GNNAV_L(2, 1, 1, 2, 6, 0);
    } else {
        if (which == kWide) GNNAV_L(2, 2, 2, 2, 3, 2);
        else GNNAV_L(2, 1, 1, 2, 6, 0);
    }
#undef GNNAV_L
}
template <int PL, int ACT>
void run_dgate(const Product &p, const Sum &again, int which, hipStream_t s) {
    KernelTimer t("gated_dgate", s);
#define GNNAV_L(A, B, C, D, ST)                                                                                         \
    hipLaunchKernelGGL((k_gated_dgate<PL, A, B, C, D, ST, ACT>), dim3(PL == 1 || ST > 3 ? ids_of(p) : places_of(p, 2, s)), dim3(64 * C * D), 0, s, p, \
                       again, (int32_t)ids_of(p))
    if constexpr (PL == 1) {
        if (which == kLarge) GNNAV_L(2, 2, 2, 4, 3);
        else if (which == kMedium) GNNAV_L(1, 2, 2, 2, 3);
        else GNNAV_L(1, 1, 2, 2, 6);
    } else {
        if (which == kWide) GNNAV_L(2, 2, 2, 2, 3);
        else GNNAV_L(1, 1, 2, 2, 6);
    }
#undef GNNAV_L
}
template <int PL>
void run_join(const Product &p, const Product &q, const Product &r, int tile, hipStream_t s) {
    JoinJobs j = {{p, q, r}, {}};
    int64_t at = 0;
    for (int k = 0; k < 3; ++k) j.end[k] = at += j.p[k].part ? j.p[k].split_stride : 0;
    if (at == 0) return;
    KernelTimer t("gated_join", s);
    const unsigned grid = grid_for(at, 256, 4096);
#define GNNAV_L(P, A, B, C, D, ST) hipLaunchKernelGGL((k_gated_join<A, B, C, D>), dim3(grid), dim3(256), 0, s, j)
    GNNAV_TILES(PL, tile, GNNAV_L);
#undef GNNAV_L
}
template <int PL>
void run_down(const Product &p, int tile, hipStream_t s) {
    {
        KernelTimer t("gated_down", s);
#define GNNAV_L(P, A, B, C, D, ST) hipLaunchKernelGGL((k_gated_down<P, A, B, C, D, ST>), dim3(ids_of(p)), dim3(64 * C * D), 0, s, p)
        GNNAV_TILES(PL, tile, GNNAV_L);
#undef GNNAV_L
    }
    run_join<PL>(p, Product{}, Product{}, tile, s);
}
template <int PL>
void run_grads(const Product &x, const Product &w, const Product &d, int tile, hipStream_t s) {
    const unsigned nx = x.m_tiles > 0 ? ids_of(x) : 0, nw = w.m_tiles > 0 ? ids_of(w) : 0, nd = d.m_tiles > 0 ? ids_of(d) : 0;
    if (nx + nw + nd == 0) return;
    {
        KernelTimer t("gated_grads", s);
#define GNNAV_L(P, A, B, C, D, ST)                                                                                    \
    hipLaunchKernelGGL((k_gated_grads<P, A, B, C, D, ST>), dim3(nx + nw + nd), dim3(64 * C * D), 0, s, x, w, d, (int32_t)nx, \
                       (int32_t)(nx + nw))
        GNNAV_TILES(PL, tile, GNNAV_L);
#undef GNNAV_L
    }
    run_join<PL>(x, w, d, tile, s);
}

// where a, b (fp32) and h lie in what is kept for the backward pass
struct Saved {
    f32x4x *a = nullptr, *b = nullptr;
    u32x4x *h;
    Saved(void *p, int64_t m, int64_t f, bool bf16) {
        const int64_t fp = up(f, 8);
        if (!bf16 && p) {
            a = (f32x4x *)p;
            b = a + fp / 4 * m;
        }
        h = bf16 ? (u32x4x *)p : (u32x4x *)((char *)p + fp * m * 8);
    }
};

// Few rows that keep nothing; longer sums than these would have too few workgroups for themselves.  x 1,024 x 4,096 x 1,024 in
// bf16 over the same weights again: 1 row 12 us, 4 23, 8 37, in tiles 24; over four sets of weights in turn 19, 28 for 4 rows, in tiles
// 24; over 24 sets 30 and 38, in tiles 26.  In fp32, whose tiles need the weights in planes: 22, 28, 37 and 64 in tiles; 33, 39, 47
// and 71 over 24 sets.
bool few_rows(const GatedArgs &x) { return x.m <= (x.bf16 ? 4 : kFewRows) && !x.saved && x.d <= 16384 && x.f <= 16384; }

template <int PL, int MR, int ACT>
void forward_few(const GatedArgs &x, hipStream_t s) {
    constexpr bool BF = PL == 1;
    float *h = (float *)x.workspace;
    {
        KernelTimer t("gated_few", s);
        const FewArgs a = {x.x, x.ld_x, x.wg, x.wu, x.ld_wg, x.ld_wu, (int32_t)x.m, (int32_t)x.d, (int32_t)x.f, h, nullptr, 0};
        hipLaunchKernelGGL((k_gated_few<BF, !BF, MR, 2, ACT>), dim3((unsigned)(up(x.f, kFewColumns) / kFewColumns)), dim3(512), 0, s, a);
    }
    {
        KernelTimer t("gated_few_down", s);
        const FewArgs a = {h, x.f, x.wd, nullptr, x.ld_wd, 0, (int32_t)x.m, (int32_t)x.f, (int32_t)x.d_out, nullptr, x.y, x.ld_y};
        hipLaunchKernelGGL((k_gated_few<BF, true, MR, 1, 0>), dim3((unsigned)(up(x.d_out, kFewColumns) / kFewColumns)), dim3(1024), 0, s, a);
    }
    GNNAV_HIP(hipGetLastError());
}

template <int PL, int ACT>
void forward(const GatedArgs &x, hipStream_t s) {
    if (few_rows(x)) {
        if (x.m == 1) return forward_few<PL, 1, ACT>(x, s);
        if (x.m == 2) return forward_few<PL, 2, ACT>(x, s);
        if (x.m <= 4) return forward_few<PL, 4, ACT>(x, s);
        if constexpr (PL == 3) return forward_few<PL, kFewRows, ACT>(x, s);
    }
    const Plan p(x, false);
    char *ws = (char *)x.workspace;
    auto at = [&](bool packed, size_t offset) { return packed ? ws + offset : nullptr; };
    Packer pack;
    if (p.pack_x) pack.add(x.x, x.ld_x, x.m, x.d, ws + p.x);
    if (p.pack_w) {
        pack.add(x.wg, x.ld_wg, x.d, x.f, ws + p.wg);
        pack.add(x.wu, x.ld_wu, x.d, x.f, ws + p.wu);
    }
    if (p.pack_wd) pack.add(x.wd, x.ld_wd, x.f, x.d_out, ws + p.wd);
    float *const row_norms = (float *)(ws + p.row_norms), *const column_norms = (float *)(ws + p.column_norms);
    if (PL == 3 && ACT == GNNAV_ACT_RELU && x.saved) pack.add_norms(x, sure_below(std::sqrt((float)x.d)), row_norms, column_norms);
    pack.run(x.bf16, s);
    const Saved saved(x.saved, x.m, x.f, x.bf16);
    u32x4x *h = x.saved ? saved.h : (u32x4x *)(ws + p.h);
    const int64_t plane = p.fp() / 8 * x.m;   // chunks of h

    Product g = {};
    g.s.A = operand(x.wg, x.ld_wg, x.d, x.f, at(p.pack_w, p.wg));
    second(g.s.A, x.wu, x.ld_wu, at(p.pack_w, p.wu));
    g.s.B = operand(x.x, x.ld_x, x.m, x.d, at(p.pack_x, p.x));
    sum_over(g.s, x.d, p.bk, 1);
    cut(g, 1);
    tiles_of(g, x.m, x.f, (PL == 1 ? kGateBf16 : kGateF32)[p.gate]);
    g.f = (int32_t)x.f;
    g.a = saved.a;
    g.b = saved.b;
    g.x = (const float *)x.x;
    g.wg = (const float *)x.wg;
    g.ld_x = x.ld_x;
    g.ld_wg = x.ld_wg;
    g.d = (int32_t)x.d;
    g.row_norms = row_norms;
    g.column_norms = column_norms;
    g.h = h;
    g.h_plane = plane;
    // (second parts always go to the workspace, behind the place that h has there)
    u32x4x *low = (u32x4x *)(ws + p.h) + plane;
    g.low = p.low_y ? low - h : 0;
    run_gate<PL, ACT>(g, p.gate, s);

    Product y = {};
    y.s.A = operand(x.wd, x.ld_wd, x.f, x.d_out, at(p.pack_wd, p.wd));
    y.s.B = operand(nullptr, 0, x.m, x.f, (const char *)h);
    y.s.B.p1 = (const char *)low;
    sum_over(y.s, x.f, p.bk, p.low_y ? 2 : 1);
    cut(y, p.down_splits);
    tiles_of(y, x.m, x.d_out, p.out(p.down));
    writes(y, x.y, x.ld_y, x.d_out, x.bf16);
    parts_at(y, ws + p.part, p.out(p.down));
    run_down<PL>(y, p.down, s);
    GNNAV_HIP(hipGetLastError());
}

template <int PL, int ACT>
void backward(const GatedArgs &x, hipStream_t s) {
    const Plan p(x, true);
    char *ws = (char *)x.workspace;
    auto at = [&](bool packed, size_t offset) { return packed ? ws + offset : nullptr; };
    const bool dgate = x.m > 0 && (x.dx || x.dwg || x.dwu || (x.dwd && p.low_dd));
    Packer pack;
    if (p.pack_x && (x.dwg || x.dwu || (PL == 1 && dgate))) pack.add(x.x, x.ld_x, x.m, x.d, ws + p.x);
    if (p.pack_w && x.dx) {
        pack.add(x.wg, x.ld_wg, x.d, x.f, ws + p.wg);
        pack.add(x.wu, x.ld_wu, x.d, x.f, ws + p.wu);
    }
    if (p.pack_wd && dgate) pack.add(x.wd, x.ld_wd, x.f, x.d_out, ws + p.wd);
    if (p.pack_dy) pack.add(x.dy, x.ld_dy, x.m, x.d_out, ws + p.dy);
    if (x.m > 0) pack.run(x.bf16, s);
    const Saved saved(x.saved, x.m, x.f, x.bf16);
    u32x4x *D = (u32x4x *)(ws + p.D), *h = (u32x4x *)(ws + p.h);
    const int64_t fp = p.fp(), plane = fp / 8 * x.m;   // chunks of da, of db, of h
    const Shape &e = p.out(p.grads);
    const Operand wg = operand(x.wg, x.ld_wg, x.d, x.f, at(p.pack_w, p.wg)), rows = operand(x.x, x.ld_x, x.m, x.d, at(p.pack_x, p.x)),
                  dy = operand(x.dy, x.ld_dy, x.m, x.d_out, at(p.pack_dy, p.dy));

    if (dgate) {
        Product g = {};
        g.s.A = operand(x.wd, x.ld_wd, x.f, x.d_out, at(p.pack_wd, p.wd));
        g.s.B = dy;
        sum_over(g.s, x.d_out, p.bk, 1);
        cut(g, 1);
        tiles_of(g, x.m, x.f, (PL == 1 ? kDgateBf16 : kDgateF32)[p.dgate]);
        g.f = (int32_t)x.f;
        g.a = saved.a;
        g.b = saved.b;
        g.h = D;
        g.h_plane = 2 * plane;
        g.second = plane;
        g.low = p.low_dx || p.low_dw ? 2 * plane : 0;
        g.h2 = p.low_dd ? h : nullptr;
        g.h2_low = plane;
        Sum again = {};   // (the weights' rows are summed over: as they lie)
        again.A = operand(x.wg, x.ld_wg, x.d, x.f, nullptr);
        second(again.A, x.wu, x.ld_wu, nullptr);
        again.B = rows;
        sum_over(again, x.d, p.bk, 1);
        run_dgate<PL, ACT>(g, again, p.dgate, s);
    }

    Product dx = {}, w = {}, d = {};
    if (x.dx && x.m > 0) {
        dx.s.A = wg;
        second(dx.s.A, x.wu, x.ld_wu, at(p.pack_w, p.wu));
        dx.s.B = operand(nullptr, 0, x.m, x.f, (const char *)D);
        dx.s.B.p1 += plane * 16;   // da, db, their second parts
        dx.s.B.p2 += 2 * plane * 16;
        dx.s.B.p3 += 3 * plane * 16;
        dx.s.B.plane = 2 * plane * 16;
        sum_over(dx.s, fp, p.bk, p.low_dx ? 4 : 2);
        cut(dx, p.dx_splits);
        tiles_of(dx, x.m, x.d, e);
        writes(dx, x.dx, x.ld_dx, x.d, x.bf16);
        parts_at(dx, ws + p.part, e);
    }
    if (x.dwg || x.dwu) {
        w.s.A = operand(nullptr, 0, x.m, 2 * fp, (const char *)D);
        w.s.A.p1 += 2 * plane * 16;
        w.s.B = rows;
        sum_over(w.s, x.m, p.bk, p.low_dw ? 2 : 1);
        cut(w, p.dw_splits);
        tiles_of(w, x.d, 2 * fp, e);
        writes(w, x.dwg, x.ld_dwg, x.f, x.bf16);
        w.out[1] = x.dwu;
        w.ld[1] = x.ld_dwu;
        w.half = (int32_t)fp;
        parts_at(w, ws + p.part2, e);
    }
    if (x.dwd) {
        d.s.A = dy;
        d.s.B = operand(nullptr, 0, x.m, x.f, (const char *)(p.low_dd ? h : saved.h));
        d.s.B.p1 = (const char *)(h + plane);
        sum_over(d.s, x.m, p.bk, p.low_dd ? 2 : 1);
        cut(d, p.dd_splits);
        tiles_of(d, x.f, x.d_out, e);
        writes(d, x.dwd, x.ld_dwd, x.d_out, x.bf16);
        parts_at(d, ws + p.part3, e);
    }
    run_grads<PL>(dx, w, d, p.grads, s);
    GNNAV_HIP(hipGetLastError());
}

template <int PL>
void by_act(const GatedArgs &x, bool back, hipStream_t s) {
    switch (x.act) {
    case GNNAV_ACT_SILU: return back ? backward<PL, GNNAV_ACT_SILU>(x, s) : forward<PL, GNNAV_ACT_SILU>(x, s);
    case GNNAV_ACT_GELU: return back ? backward<PL, GNNAV_ACT_GELU>(x, s) : forward<PL, GNNAV_ACT_GELU>(x, s);
    default: return back ? backward<PL, GNNAV_ACT_RELU>(x, s) : forward<PL, GNNAV_ACT_RELU>(x, s);
    }
}

}  // namespace

size_t gated_workspace(const GatedArgs &a, bool backward) { return Plan(a, backward).total; }
size_t gated_saved(int64_t m, int64_t f, bool bf16) { return (size_t)(m * up(f, 8) * (bf16 ? 2 : 14)); }

void launch_gated(const GatedArgs &x, bool backward, hipStream_t s) {
    if (x.m == 0 && !backward) return;
    if (x.bf16) by_act<1>(x, backward, s);
    else by_act<3>(x, backward, s);
}

}  // namespace gnnav
