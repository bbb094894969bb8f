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
// Rounding: a and b stay in fp32, also where they are kept for the backward pass (bf16 ones would cost da and db a second
// rounding of the results' own size); h, da and db are rounded once to the operands' type for the products that read them.
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

// Two values rounded to bf16, nearest even.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

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

// What copies read past the end of a sum.
__device__ const u32x4x kZeros = {0, 0, 0, 0};

// ------------------------------------------------------------------ packing
// rows x cols (row-major, 16-byte aligned rows) -> PL planes of chunks [chunk][row], zeros past the columns.
// One workgroup: 64 rows x 64 columns through LDS.  A launch takes up to five matrices.
struct PackJob {
    const void *src;
    int64_t ld;
    int32_t rows, cols, col_tiles, end;   // end: workgroups of the jobs so far
    u32x4x *out;
};
struct PackJobs {
    PackJob job[5];
};
template <bool BF>
__global__ void __launch_bounds__(256) k_gated_pack(const PackJobs jobs) {
    int32_t k = 0, base = 0;
    while ((int32_t)blockIdx.x >= jobs.job[k].end) base = jobs.job[k++].end;
    const PackJob &a = jobs.job[k];
    const int32_t t = (int32_t)blockIdx.x - base, rows = a.rows, d = a.cols, chunks = (d + 7) / 8;
    constexpr int PL = BF ? 1 : 3;
    __shared__ u32x4x tile[PL][8][65];
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
            bf16x8 p1, p2, p3;
            split3(x, p1, p2, p3);
            tile[0][lc][lr] = __builtin_bit_cast(u32x4x, p1);
            tile[PL - 2][lc][lr] = __builtin_bit_cast(u32x4x, p2);
            tile[PL - 1][lc][lr] = __builtin_bit_cast(u32x4x, p3);
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
struct Operand {
    const char *p[2];            // two matrices: side by side along M (kGate), or one after the other along the sum
    int64_t row[2];              // bytes from a row of each to the next
    int64_t chunk, plane;        // from a chunk, from a plane
    int32_t rows, chunks;        // what there is of each
};

enum { kGate, kDgate, kOut };

struct Product {
    Operand A, B;
    int32_t m_tiles, n_tiles, splits, split_steps;
    int32_t segments, steps;     // matrices one after the other; steps of each
    int32_t tail;                // what the last step of a segment sums over (its BK where that is whole)
    int32_t n;                   // rows of the output
    // kGate, kDgate: columns, 4-float groups [group][row] of a and b (kGate: nullable), chunks of h, or of da and db
    int32_t f;
    f32x4x *a, *b;
    u32x4x *h;
    int64_t h_plane, second;     // chunks of a plane; from da to db
    // kOut: columns of one output, where the second one starts (INT_MAX: there is none)
    int32_t cols, half;
    void *out[2];
    int64_t ld[2];
    bool bf16;
    f32x4x *part;                // splits > 1: the tiles' sums, split after split
    int64_t split_stride;        // float4s
};

// Wave grid WGM x WGN, each wavefront WMF x WNF MFMA blocks of 32 x 32; BK summed elements per stage, three stages in LDS.
template <int PL, int WMF, int WNF, int WGM, int WGN>
struct Tile {
    static constexpr int BK = PL == 1 ? 32 : 16;
    static constexpr int NW = WGM * WGN, BM = 32 * WMF * WGM, BN = 32 * WNF * WGN;
    static constexpr int APC = BM * BK / 8, BPC = BN * BK / 8;   // chunks of a plane of a stage
    static constexpr int STAGE = PL * (APC + BPC);
    static constexpr int ST = 3, LDS = ST * STAGE;
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
__device__ __forceinline__ void store_chunks(u32x4x *to, int64_t plane, int64_t rows, int64_t chunk, int64_t chunks, int64_t n,
                                             int h, const float (&x)[16]) {
#pragma unroll
    for (int pl = 0; pl < PL; ++pl)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            uint32_t w[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float f0 = x[4 * (g + i) + 2 * j], f1 = x[4 * (g + i) + 2 * j + 1];
                    if constexpr (PL == 1) {
                        w[i][j] = bf16_pair(f0, f1);
                    } else {
                        uint16_t q0[3], q1[3];
                        split3_bits(f0, q0[0], q0[1], q0[2]);
                        split3_bits(f1, q1[0], q1[1], q1[2]);
                        w[i][j] = (uint32_t)q0[pl] | ((uint32_t)q1[pl] << 16);
                    }
                }
            const u32x4x v = join_chunk(w[0][0], w[0][1], w[1][0], w[1][1]);
            if (n < rows && chunk + g + h < chunks) to[pl * plane + (chunk + g + h) * rows + n] = v;
        }
}

// One tile of a product, from operands in memory by way of LDS, and what becomes of it.
// AT, BT: the operand's rows are summed over.  In LDS an operand whose columns are summed over lies row by row, its BK / 8
// chunks exchanged by the row (16 rows read 256 bytes of distinct banks); one whose rows are lies in blocks of 8 of them,
// chunk by chunk, the two halves of a block exchanged by the chunk (32 lanes of a transposing read take 256 bytes of distinct
// banks).  Both copy whole runs from row-major and from chunk-major memory.
template <int PL, int WMF, int WNF, int WGM, int WGN, bool AT, bool BT, int EPI, int ACT>
__device__ __forceinline__ void gated_tile(const Product &a, int32_t id, u32x4x *S) {
    using C = Tile<PL, WMF, WNF, WGM, WGN>;
    constexpr int BK = C::BK, ST = C::ST, NW = C::NW, BM = C::BM, BN = C::BN, APC = C::APC, BPC = C::BPC;
    constexpr int STAGE = C::STAGE, INSTR = STAGE / 64, IN = (INSTR + NW - 1) / NW, CK = BK / 8;
    constexpr bool DUAL = EPI == kGate;
    static_assert(!DUAL || (AT && WMF % 2 == 0), "both projections in one tile");
    constexpr int AM = DUAL ? BM / 2 : BM, WA = DUAL ? WMF / 2 : WMF;   // columns of one matrix in the tile, blocks of a wavefront
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wid / WGN, wn = wid % WGN, h = lane >> 5, lr = lane & 31;
    int32_t split, mt, nt;
    if (!tile_of(a, id, split, mt, nt)) return;
    const int64_t m0 = (int64_t)mt * AM, n0 = (int64_t)nt * BN;
    const int32_t all = a.segments * a.steps, s0 = EPI == kOut ? split * a.split_steps : 0;
    const int32_t T = EPI == kOut ? std::max(0, std::min(a.split_steps, all - s0)) : all;

    // This wavefront's copies of a stage: source of the next step, its advance, whether the lane's is part of a last step.
    const char *src[IN];
    int64_t inc[IN];
    int dst[IN];
    uint32_t in_tail = 0;
    auto aim = [&](int32_t segment, int32_t step) {
#pragma unroll
        for (int u = 0; u < IN; ++u) {
            const int q = std::min(wid * IN + u, INSTR - 1);   // the last wavefront may repeat the last copy
            const int slot = q * 64;
            const bool isB = slot >= PL * APC;
            const int rel = slot - (isB ? PL * APC : 0), pc = isB ? BPC : APC;
            const int plane = rel / pc;
            int s = rel % pc + lane;
            const Operand &o = isB ? a.B : a.A;
            int32_t matrix = segment;
            if (DUAL && !isB) {
                matrix = s / (APC / 2);
                s -= matrix * (APC / 2);
            }
            const int64_t x0 = isB ? n0 : m0;
            const char *base = o.p[matrix] + plane * o.plane;
            const int64_t row = o.row[matrix];
            int k;
            if (isB ? BT : AT) {
                const int mcs = (isB ? BN : AM) / 8, mc = (s / 8) % mcs;
                k = s / (8 * mcs) * 8 + ((s % 8) ^ ((mc & 2) * 2));
                src[u] = base + ((int64_t)step * BK + k) * row + std::min<int64_t>(x0 / 8 + mc, o.chunks - 1) * o.chunk;
                inc[u] = BK * row;
            } else {
                const int r = s / CK, c = (s % CK) ^ (CK == 4 ? (r >> 2) & 3 : (r >> 3) & 1);
                k = c * 8;
                src[u] = base + std::min<int64_t>(x0 + r, o.rows - 1) * row + ((int64_t)step * CK + c) * o.chunk;
                inc[u] = CK * o.chunk;
            }
            dst[u] = slot;
            in_tail = (in_tail & ~(1u << u)) | (uint32_t)(k < a.tail) << u;
        }
    };
    auto issue = [&](int stage, int u) {
        dma16(src[u], &S[stage * STAGE + dst[u]]);
        src[u] += inc[u];
    };
    int32_t segment = s0 / std::max(a.steps, 1), local = s0 - segment * a.steps;   // of the step that is copied next
    // before the copies of the next step: the second matrices, or the end of a sum
    auto prepare = [&]() {
        if (local == a.steps) {
            local = 0;
            aim(++segment, 0);
        }
        if (++local == a.steps && a.tail < BK) {
#pragma unroll
            for (int u = 0; u < IN; ++u)
                if (!(in_tail >> u & 1)) src[u] = (const char *)&kZeros;
        }
    };

    f32x16x acc[WMF][WNF];
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
    auto frag = [&](const u32x4x *plane, auto tr_, int tile, int x, int kk) -> bf16x8 {
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
    auto read = [&](Frags &f, int stage, int kk, int k) {
        const u32x4x *sa = &S[stage * STAGE], *sb = sa + PL * APC;
        const int x = k / PL, p = k % PL;
        if (x < WNF) {
            f.b[x][p] = frag(sb + p * BPC, std::integral_constant<bool, BT>(), BN, wn * (32 * WNF) + 32 * x, kk);
        } else {
            const int i = x - WNF, matrix = i / WA;
            f.a[i][p] = frag(sa + p * APC + matrix * (APC / 2), std::integral_constant<bool, AT>(), AM, wm * (32 * WA) + 32 * (i % WA), kk);
        }
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
        aim(segment, local);
#pragma unroll
        for (int k = 0; k < ST - 1; ++k)
            if (k < T) {
                prepare();
#pragma unroll
                for (int u = 0; u < IN; ++u) issue(k, u);
            }
        advance(0);
        if (ST - 1 < T) {
            prepare();
#pragma unroll
            for (int u = 0; u < FIRST; ++u) issue(ST - 1, u);
        }
#pragma unroll
        for (int q = 0; q < NF; ++q) read(f0, 0, 0, q);
    }
    for (int32_t t = 0; t < T;) {
        if constexpr (BK == 32) {
            multiply(f0, f1, ready, 1, t + ST - 1 < T, fill, kMiddle, kEnd);
            fill = next(fill);
            ready = next(ready);
            if (++t < T) advance(t);
            if (t + ST - 1 < T) prepare();
            multiply(f1, f0, ready, 0, t + ST - 1 < T, fill, kBegin, kMiddle);
        } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                // (its copies of the first stages were issued above: ST - 1 whole ones and this one)
                ready = next(ready);
                if (++t < T) advance(t);
                if (t + ST - 1 < T) prepare();
                if (half == 0) multiply(f0, f1, ready, 0, t + ST - 1 < T, fill, kBegin, kEnd);
                else multiply(f1, f0, ready, 0, t + ST - 1 < T, fill, kBegin, kEnd);
                fill = next(fill);
                if (t >= T) break;
            }
        }
    }

    const int64_t mw = m0 + wm * (32 * WA), nw = n0 + wn * (32 * WNF);
    if constexpr (EPI == kGate || EPI == kDgate) {
        const int32_t chunks = (a.f + 7) / 8;
#pragma unroll
        for (int j = 0; j < WNF; ++j) {
            const int64_t n = nw + 32 * j + lr;
#pragma unroll
            for (int i = 0; i < WA; ++i) {
                float x[16], z[16];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int64_t c = mw + 32 * i + 8 * g + 4 * h;
                    const bool here = n < a.n && c < chunks * 8;
                    f32x4x va = {0.f, 0.f, 0.f, 0.f}, vb = va;
                    if constexpr (EPI == kGate) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            va[e] = acc[i][j][4 * g + e];
                            vb[e] = acc[i + WA][j][4 * g + e];
                        }
                        if (here && a.a) {
                            a.a[c / 4 * a.n + n] = va;
                            a.b[c / 4 * a.n + n] = vb;
                        }
                    } else if (here) {
                        va = a.a[c / 4 * a.n + n];
                        vb = a.b[c / 4 * a.n + n];
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float value, slope;
                        activate<ACT, PL == 3>(va[e], value, slope);
                        const bool live = c + e < a.f;
                        if constexpr (EPI == kGate) {
                            x[4 * g + e] = live ? value * vb[e] : 0.f;
                        } else {
                            x[4 * g + e] = live ? acc[i][j][4 * g + e] * vb[e] * slope : 0.f;
                            z[4 * g + e] = live ? acc[i][j][4 * g + e] * value : 0.f;
                        }
                    }
                }
                store_chunks<PL>(a.h, a.h_plane, a.n, (mw + 32 * i) / 8, chunks, n, h, x);
                if constexpr (EPI == kDgate) store_chunks<PL>(a.h + a.second, a.h_plane, a.n, (mw + 32 * i) / 8, chunks, n, h, z);
            }
        }
    } else {
        f32x4x *part = a.part;
        if (part) part += split * a.split_stride + ((int64_t)(nt * a.m_tiles + mt) * NW + wid) * (WMF * WNF * 4 * 64) + lane;
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
}

template <int PL, int WMF, int WNF, int WGM, int WGN, int ACT>
__global__ void __launch_bounds__(64 * WGM * WGN, 2) k_gated_gate(const Product a) {
    __shared__ u32x4x S[Tile<PL, WMF, WNF, WGM, WGN>::LDS];
    gated_tile<PL, WMF, WNF, WGM, WGN, true, false, kGate, ACT>(a, blockIdx.x, S);
}
template <int PL, int WMF, int WNF, int WGM, int WGN>
__global__ void __launch_bounds__(64 * WGM * WGN, 2) k_gated_down(const Product a) {
    __shared__ u32x4x S[Tile<PL, WMF, WNF, WGM, WGN>::LDS];
    gated_tile<PL, WMF, WNF, WGM, WGN, true, false, kOut, 0>(a, blockIdx.x, S);
}
template <int PL, int WMF, int WNF, int WGM, int WGN, int ACT>
__global__ void __launch_bounds__(64 * WGM * WGN, 2) k_gated_dgate(const Product a) {
    __shared__ u32x4x S[Tile<PL, WMF, WNF, WGM, WGN>::LDS];
    gated_tile<PL, WMF, WNF, WGM, WGN, false, false, kDgate, ACT>(a, blockIdx.x, S);
}
// dx and the weights' gradients in one launch: workgroups below `w_at` take dx's tiles, below `d_at` those of dWg and dWu.
template <int PL, int WMF, int WNF, int WGM, int WGN>
__global__ void __launch_bounds__(64 * WGM * WGN, 2) k_gated_grads(const Product x, const Product w, const Product d, int32_t w_at,
                                                                   int32_t d_at) {
    __shared__ u32x4x S[Tile<PL, WMF, WNF, WGM, WGN>::LDS];
    const int32_t id = blockIdx.x;
    if (id < w_at) gated_tile<PL, WMF, WNF, WGM, WGN, false, false, kOut, 0>(x, id, S);
    else if (id < d_at) gated_tile<PL, WMF, WNF, WGM, WGN, true, true, kOut, 0>(w, id - w_at, S);
    else gated_tile<PL, WMF, WNF, WGM, WGN, true, true, kOut, 0>(d, id - d_at, S);
}

// The sum of the splits' parts, in their order.  A launch takes up to three products.
struct JoinJobs {
    Product p[3];
    int64_t end[3];   // float4s of the products so far
};
template <int WMF, int WNF, int WGM, int WGN>
__global__ void __launch_bounds__(256) k_gated_join(const JoinJobs jobs) {
    constexpr int NW = WGM * WGN, BM = 32 * WMF * WGM, BN = 32 * WNF * WGN;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < jobs.end[2]; at += (int64_t)gridDim.x * 256) {
        const int k = at < jobs.end[0] ? 0 : at < jobs.end[1] ? 1 : 2;
        const Product &a = jobs.p[k];
        const int64_t i = at - (k ? jobs.end[k - 1] : 0);
        f32x4x v = a.part[i];
        for (int32_t s = 1; s < a.splits; ++s) v += a.part[s * a.split_stride + i];
        const int lane = (int)(i & 63);
        int64_t r = i >> 6;
        const int g = (int)(r & 3);
        r >>= 2;
        const int fj = (int)(r % WNF), fi = (int)(r / WNF % WMF);
        r /= WNF * WMF;
        const int wid = (int)(r % NW);
        r /= NW;
        const int32_t mt = (int32_t)(r % a.m_tiles), nt = (int32_t)(r / a.m_tiles);
        store4(a, (int64_t)nt * BN + wid % WGN * (32 * WNF) + 32 * fj + (lane & 31),
               mt * BM + wid / WGN * (32 * WMF) + 32 * fi + 8 * g + 4 * (lane >> 5), v);
    }
}

// ------------------------------------------------------------------ host
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

enum { kTile64, kTile128, kTile256 };

// Tile of the launches over m rows and these columns: the largest that gives every compute unit something to do.
int tile_for(int64_t rows, int64_t cols, bool bf16) {
    if (bf16 && up(rows, 256) / 256 * (up(cols, 256) / 256) >= 192) return kTile256;
    return up(rows, 128) / 128 * (up(cols, 128) / 128) >= 192 ? kTile128 : kTile64;
}
int64_t edge_of(int tile) { return tile == kTile256 ? 256 : tile == kTile128 ? 128 : 64; }

// Splits of a sum of `steps` steps whose product has `tiles` tiles: two workgroups a unit, 8 steps each at least.
int32_t splits_for(int64_t tiles, int64_t steps) {
    const int64_t want = std::max<int64_t>(1, 512 / std::max<int64_t>(tiles, 1));
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>({want, steps / 8, 64}));
}

unsigned ids_of(const Product &a) {   // workgroups of a product, whole rounds over the XCDs
    return (unsigned)up((int64_t)a.m_tiles * a.n_tiles * a.splits, 8);
}

// Where everything lies in the workspace, and how the products are cut.
struct Plan {
    int64_t m, d, f, o;
    int pl, bk;
    bool bf16, pack_x, pack_w, pack_wd, pack_dy;
    int gate, down, dgate, grads;
    int32_t down_splits = 1, dx_splits = 1, dw_splits = 1, dd_splits = 1;
    size_t x = 0, wg = 0, wu = 0, wd = 0, dy = 0, h = 0, D = 0, part = 0, part2 = 0, part3 = 0, total = 0;
    int64_t fp() const { return up(f, 8); }
    size_t take(int64_t bytes) {
        const size_t here = total;
        total += (size_t)up(bytes, 256);
        return here;
    }
    size_t packed(int64_t rows, int64_t cols) { return take(rows * up(cols, 8) * 2 * pl); }
    static int64_t parts(int64_t rows, int64_t cols, int64_t edge, int32_t splits) {
        return splits > 1 ? splits * up(rows, edge) * up(cols, edge) * 4 : 0;
    }
    Plan(const GatedArgs &a, bool backward) : m(a.m), d(a.d), f(a.f), o(a.d_out), bf16(a.bf16) {
        pl = bf16 ? 1 : 3;
        bk = bf16 ? 32 : 16;
        // (where the columns are summed over, the last chunk has to end in zeros)
        pack_x = !bf16 || (!backward && d % 8);
        pack_wd = !bf16 || (backward && o % 8);
        pack_dy = !bf16 || o % 8;
        pack_w = !bf16 || (backward && f % 8);
        if (pack_x) x = packed(m, d);
        if (pack_w) {
            wg = packed(d, f);
            wu = packed(d, f);
        }
        if (pack_wd) wd = packed(f, o);
        if (!backward) {
            h = take(fp() * m * 2 * pl);
            gate = tile_for(m, 2 * f, bf16);
            down = tile_for(m, o, bf16);
            const int64_t e = edge_of(down), steps = (f + bk - 1) / bk;
            down_splits = cut(splits_for(up(m, e) / e * (up(o, e) / e), steps), steps);
            part = take(parts(m, o, e, down_splits));
        } else {
            if (pack_dy) dy = packed(m, o);
            D = take(2 * fp() * m * 2 * pl);
            dgate = tile_for(m, f, bf16);
            grads = std::min(tile_for(m + d, 2 * f, bf16), tile_for(std::max(m, d), std::max(d, f), bf16));
            const int64_t e = edge_of(grads), ks = (fp() + bk - 1) / bk * 2, ms = (m + bk - 1) / bk;
            const int64_t tx = up(m, e) / e * (up(d, e) / e), tw = up(d, e) / e * (up(2 * fp(), e) / e), td = up(f, e) / e * (up(o, e) / e);
            dx_splits = cut(splits_for(tx, ks), ks);
            dw_splits = cut(splits_for(tw, ms), ms);
            dd_splits = cut(splits_for(td, ms), ms);
            part = take(parts(m, d, e, dx_splits));
            part2 = take(parts(d, 2 * fp(), e, dw_splits));
            part3 = take(parts(f, o, e, dd_splits));
        }
    }
    static int32_t cut(int32_t splits, int64_t steps) {   // without empty ones
        const int64_t each = std::max<int64_t>(1, (steps + splits - 1) / splits);
        return (int32_t)std::max<int64_t>(1, (steps + each - 1) / each);
    }
};

// rows x cols of the caller's, as it lies or packed at `at`
Operand operand(const void *p, int64_t ld, int64_t rows, int64_t cols, const char *packed_at) {
    Operand o = {};
    o.rows = (int32_t)rows;
    o.chunks = (int32_t)(up(cols, 8) / 8);
    if (packed_at) {
        o.p[0] = o.p[1] = packed_at;
        o.row[0] = o.row[1] = 16;
        o.chunk = rows * 16;
        o.plane = o.chunk * o.chunks;
    } else {
        o.p[0] = o.p[1] = (const char *)p;
        o.row[0] = o.row[1] = ld * 2;
        o.chunk = 16;
        o.plane = 0;
    }
    return o;
}

// ... and a second matrix of the same sizes
void second(Operand &o, const void *p, int64_t ld, const char *packed_at) {
    o.p[1] = packed_at ? packed_at : (const char *)p;
    o.row[1] = packed_at ? 16 : ld * 2;
}

void sum_over(Product &p, int64_t k, int bk, int32_t segments, int32_t splits) {
    p.segments = segments;
    p.steps = (int32_t)((k + bk - 1) / bk);
    p.tail = (int32_t)(k - (int64_t)(p.steps - 1) * bk);
    p.splits = splits;
    p.split_steps = (int32_t)((segments * (int64_t)p.steps + splits - 1) / splits);
}
void tiles_of(Product &p, int64_t rows, int64_t cols, int64_t bn, int64_t bm) {
    p.n = (int32_t)rows;
    p.n_tiles = (int32_t)(up(rows, bn) / bn);
    p.m_tiles = (int32_t)(up(cols, bm) / bm);
}
void writes(Product &p, void *out, int64_t ld, int64_t cols, bool bf16) {
    p.out[0] = out;
    p.out[1] = nullptr;
    p.half = INT_MAX;
    p.ld[0] = p.ld[1] = ld;
    p.cols = (int32_t)cols;
    p.bf16 = bf16;
}
void parts_at(Product &p, char *at, int64_t edge) {
    p.split_stride = (int64_t)p.n_tiles * p.m_tiles * edge * edge / 4;
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
    void run(bool bf16, hipStream_t s) {
        if (blocks == 0) return;
        KernelTimer t("gated_pack", s);
        if (bf16) hipLaunchKernelGGL(k_gated_pack<true>, dim3((unsigned)blocks), dim3(256), 0, s, jobs);
        else hipLaunchKernelGGL(k_gated_pack<false>, dim3((unsigned)blocks), dim3(256), 0, s, jobs);
    }
};

#define GNNAV_TILES(PL, TILE, L)                       \
    do {                                               \
        if (PL == 1 && TILE == kTile256) L(1, 4, 2, 2, 4); \
        else if (TILE >= kTile128) L(PL, 2, 2, 2, 2);  \
        else L(PL, 2, 1, 1, 2);                        \
    } while (0)

template <int PL, int ACT>
void run_gate(const Product &p, int tile, hipStream_t s) {
    KernelTimer t("gated_gate", s);
#define GNNAV_L(P, A, B, C, D) hipLaunchKernelGGL((k_gated_gate<P, A, B, C, D, ACT>), dim3(ids_of(p)), dim3(64 * C * D), 0, s, p)
    GNNAV_TILES(PL, tile, GNNAV_L);
#undef GNNAV_L
}
template <int PL, int ACT>
void run_dgate(const Product &p, int tile, hipStream_t s) {
    KernelTimer t("gated_dgate", s);
#define GNNAV_L(P, A, B, C, D) hipLaunchKernelGGL((k_gated_dgate<P, A, B, C, D, ACT>), dim3(ids_of(p)), dim3(64 * C * D), 0, s, p)
    GNNAV_TILES(PL, tile, GNNAV_L);
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
#define GNNAV_L(P, A, B, C, D) hipLaunchKernelGGL((k_gated_join<A, B, C, D>), dim3(grid), dim3(256), 0, s, j)
    GNNAV_TILES(PL, tile, GNNAV_L);
#undef GNNAV_L
}
template <int PL>
void run_down(const Product &p, int tile, hipStream_t s) {
    {
        KernelTimer t("gated_down", s);
#define GNNAV_L(P, A, B, C, D) hipLaunchKernelGGL((k_gated_down<P, A, B, C, D>), dim3(ids_of(p)), dim3(64 * C * D), 0, s, p)
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
#define GNNAV_L(P, A, B, C, D)                                                                                        \
    hipLaunchKernelGGL((k_gated_grads<P, A, B, C, D>), dim3(nx + nw + nd), dim3(64 * C * D), 0, s, x, w, d, (int32_t)nx, \
                       (int32_t)(nx + nw))
        GNNAV_TILES(PL, tile, GNNAV_L);
#undef GNNAV_L
    }
    run_join<PL>(x, w, d, tile, s);
}

// where a, b and h lie in what is kept for the backward pass
struct Saved {
    f32x4x *a, *b;
    u32x4x *h;
    Saved(void *p, int64_t m, int64_t f) {
        const int64_t fp = up(f, 8);
        a = (f32x4x *)p;
        b = a + fp / 4 * m;
        h = (u32x4x *)(b + fp / 4 * m);
    }
};

template <int PL, int ACT>
void forward(const GatedArgs &x, hipStream_t s) {
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
    pack.run(x.bf16, s);
    const Saved saved(x.saved, x.m, x.f);
    u32x4x *h = x.saved ? saved.h : (u32x4x *)(ws + p.h);
    const int64_t fp = p.fp();

    Product g = {};
    g.A = operand(x.wg, x.ld_wg, x.d, x.f, at(p.pack_w, p.wg));
    second(g.A, x.wu, x.ld_wu, at(p.pack_w, p.wu));
    g.B = operand(x.x, x.ld_x, x.m, x.d, at(p.pack_x, p.x));
    sum_over(g, x.d, p.bk, 1, 1);
    const int64_t e = edge_of(p.gate);
    tiles_of(g, x.m, x.f, e, e / 2);
    g.f = (int32_t)x.f;
    g.a = x.saved ? saved.a : nullptr;
    g.b = x.saved ? saved.b : nullptr;
    g.h = h;
    g.h_plane = fp / 8 * x.m;
    run_gate<PL, ACT>(g, p.gate, s);

    Product y = {};
    y.A = operand(x.wd, x.ld_wd, x.f, x.d_out, at(p.pack_wd, p.wd));
    y.B = operand(nullptr, 0, x.m, x.f, (const char *)h);
    sum_over(y, x.f, p.bk, 1, p.down_splits);
    tiles_of(y, x.m, x.d_out, edge_of(p.down), edge_of(p.down));
    writes(y, x.y, x.ld_y, x.d_out, x.bf16);
    parts_at(y, ws + p.part, edge_of(p.down));
    run_down<PL>(y, p.down, s);
    GNNAV_HIP(hipGetLastError());
}

template <int PL, int ACT>
void backward(const GatedArgs &x, hipStream_t s) {
    const Plan p(x, true);
    char *ws = (char *)x.workspace;
    auto at = [&](bool packed, size_t offset) { return packed ? ws + offset : nullptr; };
    Packer pack;
    if (p.pack_x && (x.dwg || x.dwu)) pack.add(x.x, x.ld_x, x.m, x.d, ws + p.x);
    if (p.pack_w && x.dx) {
        pack.add(x.wg, x.ld_wg, x.d, x.f, ws + p.wg);
        pack.add(x.wu, x.ld_wu, x.d, x.f, ws + p.wu);
    }
    if (p.pack_wd) pack.add(x.wd, x.ld_wd, x.f, x.d_out, ws + p.wd);
    if (p.pack_dy) pack.add(x.dy, x.ld_dy, x.m, x.d_out, ws + p.dy);
    if (x.m > 0) pack.run(x.bf16, s);
    const Saved saved(const_cast<void *>(x.saved), x.m, x.f);
    u32x4x *D = (u32x4x *)(ws + p.D);
    const int64_t fp = p.fp(), e = edge_of(p.grads);

    if (x.m > 0 && (x.dx || x.dwg || x.dwu)) {
        Product g = {};
        g.A = operand(x.wd, x.ld_wd, x.f, x.d_out, at(p.pack_wd, p.wd));
        g.B = operand(x.dy, x.ld_dy, x.m, x.d_out, at(p.pack_dy, p.dy));
        sum_over(g, x.d_out, p.bk, 1, 1);
        tiles_of(g, x.m, x.f, edge_of(p.dgate), edge_of(p.dgate));
        g.f = (int32_t)x.f;
        g.a = saved.a;
        g.b = saved.b;
        g.h = D;
        g.h_plane = 2 * fp / 8 * x.m;
        g.second = fp / 8 * x.m;
        run_dgate<PL, ACT>(g, p.dgate, s);
    }

    Product dx = {}, w = {}, d = {};
    if (x.dx && x.m > 0) {
        dx.A = operand(x.wg, x.ld_wg, x.d, x.f, at(p.pack_w, p.wg));
        second(dx.A, x.wu, x.ld_wu, at(p.pack_w, p.wu));
        dx.B = operand(nullptr, 0, x.m, x.f, (const char *)D);
        dx.B.p[1] += fp / 8 * x.m * 16;
        dx.B.plane *= 2;
        sum_over(dx, fp, p.bk, 2, p.dx_splits);
        tiles_of(dx, x.m, x.d, e, e);
        writes(dx, x.dx, x.ld_dx, x.d, x.bf16);
        parts_at(dx, ws + p.part, e);
    }
    if (x.dwg || x.dwu) {
        w.A = operand(nullptr, 0, x.m, 2 * fp, (const char *)D);
        w.B = operand(x.x, x.ld_x, x.m, x.d, at(p.pack_x, p.x));
        sum_over(w, x.m, p.bk, 1, p.dw_splits);
        tiles_of(w, x.d, 2 * fp, e, e);
        writes(w, x.dwg, x.ld_dwg, x.f, x.bf16);
        w.out[1] = x.dwu;
        w.ld[1] = x.ld_dwu;
        w.half = (int32_t)fp;
        parts_at(w, ws + p.part2, e);
    }
    if (x.dwd) {
        d.A = operand(x.dy, x.ld_dy, x.m, x.d_out, at(p.pack_dy, p.dy));
        d.B = operand(nullptr, 0, x.m, x.f, (const char *)saved.h);
        sum_over(d, x.m, p.bk, 1, p.dd_splits);
        tiles_of(d, x.f, x.d_out, e, e);
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
size_t gated_saved(int64_t m, int64_t f, bool bf16) { return (size_t)(m * up(f, 8) * (8 + (bf16 ? 2 : 6))); }

void launch_gated(const GatedArgs &x, bool backward, hipStream_t s) {
    if (x.m == 0 && !backward) return;
    if (x.bf16) by_act<1>(x, backward, s);
    else by_act<3>(x, backward, s);
}

}  // namespace gnnav
