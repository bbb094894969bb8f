// Lookup in a trained table and its gradient.
//
//   lookup     out[i] = scale * table[ids[i]]: one lane group per row, 16-byte
//              units, several rows in flight
//   gradient   dtable[v] = scale * sum of dout[i] over the i with ids[i] = v, in
//              fp32.  The (id, position) pairs are sorted by id with a stable
//              radix sort, so equal ids lie side by side in order of position;
//              the sorted list is cut into stretches of equal length, each
//              summed by one lane group, and an id's part sums of several
//              stretches are joined in order afterwards.  Every lane group
//              reads the same number of rows however popular an id is, and
//              there are no floating-point atomics, so the bits are the same
//              on every run (the stretches' length goes by the size of the list,
//              and so does the order of the sums).  Rows of ids that do not occur are filled with
//              zeros by the same launch.  A few ids need no sort: each
//              position looks for its id among the others itself, and a popular
//              id's rows are added up by one workgroup.
#include <algorithm>
#include <type_traits>

#include "common.hpp"

namespace gnnav {

namespace {

typedef float f32x4e __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4e __attribute__((ext_vector_type(4)));

// A 16-byte unit of a row as fp32 values: 4 of fp32, 8 of bf16.
template <bool BF>
struct Unit {
    static constexpr int N = BF ? 8 : 4;
    float v[N];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = 0.f;
    }
    __device__ __forceinline__ void from(u32x4e u) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (BF) {
                v[2 * q] = __uint_as_float(u[q] << 16);
                v[2 * q + 1] = __uint_as_float(u[q] & 0xffff0000u);
            } else {
                v[q] = __uint_as_float(u[q]);
            }
        }
    }
    __device__ __forceinline__ void add(u32x4e u) {
        Unit x;
        x.from(u);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] += x.v[e];
    }
    // rounded once to the row's type; zeros from column d on (first: the unit's first column)
    __device__ __forceinline__ u32x4e to(int64_t first, int64_t d) const {
        u32x4e u;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (BF) {
                const uint32_t lo = first + 2 * q < d ? bf16_rne(v[2 * q]) : 0u;
                const uint32_t hi = first + 2 * q + 1 < d ? bf16_rne(v[2 * q + 1]) : 0u;
                u[q] = lo | (hi << 16);
            } else {
                u[q] = first + q < d ? __float_as_uint(v[q]) : 0u;
            }
        }
        return u;
    }
};

// Results larger than this are stored past the caches, which the tables and gradients being read then have for
// themselves (smaller ones stay there for what reads them next): 800,000 rows of 256 bytes 89.3 us, 84.2 so; the gradient
// of 524,288 skewed ids x 256 bf16 148.7 and 145.5, of 260,003 x 602 fp32 326.4 and 317.3; 67 MB of rows 31.7 and 26.1.
// A kernel has one kind of store: of two in the branches of an `if` the compiler makes one, of the ordinary kind.
constexpr int64_t kStreamBytes = int64_t(64) << 20;
template <bool STREAMED>
__device__ __forceinline__ void store(u32x4e *to, u32x4e v) {
    if constexpr (STREAMED) __builtin_nontemporal_store(v, to);
    else *to = v;
}

// launch(g, bf16, streamed) with the last two as constants
template <class F, class GV>
void by_type(F &&launch, GV g, bool bf16, bool streamed) {
    const std::true_type yes{};
    const std::false_type no{};
    if (bf16) streamed ? launch(g, yes, yes) : launch(g, yes, no);
    else streamed ? launch(g, no, yes) : launch(g, no, no);
}

int lane_group(int64_t units) {   // lanes per row: the power of two that covers it, at most a wavefront
    int g = 1;
    while (g < units && g < kWave) g <<= 1;
    return g;
}

}  // namespace

// ---------------------------------------------------------------- lookup
// G lanes per row, R rows of a lane group in flight: their units are loaded
// before any is stored; longer rows loop over slabs of G units.  Bound by HBM: 800,000 random rows of
// 256 bytes 84 us, 4.9 TB/s; few rows by the launch.
template <int G, int R, bool BF, bool STREAMED>
__global__ void __launch_bounds__(256) k_embedding(const u32x4e *__restrict__ table, int64_t n_rows, int64_t ld16,
                                                   int32_t units, int64_t d, const int32_t *__restrict__ ids,
                                                   const int32_t *__restrict__ n_dev, int64_t n, float scale,
                                                   u32x4e *__restrict__ out, int64_t out_ld16) {
    constexpr int RPW = kWave / G;
    const int lane = lane_id(), sub = lane / G, c0 = lane % G;
    if (n_dev) n = std::min<int64_t>(n, std::max<int32_t>(*n_dev, 0));
    const int64_t groups = ((int64_t)gridDim.x * blockDim.x) / kWave * RPW;
    const int64_t first = (((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / kWave) * RPW + sub;
    for (int64_t i0 = first; i0 < n; i0 += R * groups) {
        int32_t id[R];
#pragma unroll
        for (int r = 0; r < R; ++r) id[r] = i0 + r * groups < n ? ids[i0 + r * groups] : -1;
        for (int32_t c = c0; c < units; c += G) {
            u32x4e x[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                x[r] = u32x4e{0, 0, 0, 0};
                if (id[r] >= 0 && id[r] < n_rows) x[r] = table[(int64_t)id[r] * ld16 + c];
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (i0 + r * groups >= n) continue;
                Unit<BF> v;
                v.from(x[r]);
#pragma unroll
                for (int e = 0; e < Unit<BF>::N; ++e) v.v[e] *= scale;
                if (id[r] < 0 || id[r] >= n_rows) v.zero();
                store<STREAMED>(&out[(i0 + r * groups) * out_ld16 + c], v.to((int64_t)c * Unit<BF>::N, d));
            }
        }
    }
}

void launch_embedding(const void *table, int64_t n_rows, int64_t ld_bytes, int64_t d, bool bf16, const int32_t *ids,
                      const int32_t *n_dev, int64_t n, float scale, void *out, int64_t out_ld_bytes, hipStream_t s) {
    if (n <= 0) return;
    const int32_t units = (int32_t)((d * (bf16 ? 2 : 4) + 15) / 16);
    const int g = lane_group(units);
    KernelTimer t("embedding", s);
    const unsigned grid = grid_for(n, 256 / g * 4, 4096);
    const bool streamed = n * units * 16 > kStreamBytes;
    auto launch = [&](auto g_, auto bf_, auto st_) {
        hipLaunchKernelGGL((k_embedding<decltype(g_)::value, 4, decltype(bf_)::value, decltype(st_)::value>), dim3(grid), dim3(256),
                           0, s, (const u32x4e *)table, n_rows, ld_bytes / 16, units, d, ids, n_dev, n, scale, (u32x4e *)out,
                           out_ld_bytes / 16);
    };
#define GNNAV_L(GV)                                                                                                 \
    case GV: by_type(launch, std::integral_constant<int, GV>{}, bf16, streamed); break
    switch (g) {
        GNNAV_L(1);
        GNNAV_L(2);
        GNNAV_L(4);
        GNNAV_L(8);
        GNNAV_L(16);
        GNNAV_L(32);
        GNNAV_L(64);
        default: fail(GNNAV_E_INVALID, "bad row width");
    }
#undef GNNAV_L
    GNNAV_HIP(hipGetLastError());
}

// ------------------------------------------------- gradient: few positions
// One workgroup per position: it lists the positions of its id, in order, and
// leaves if one of them lies before it; otherwise its lane groups add up the
// rows in turn and their sums are joined in a fixed order.  Workgroups past the
// positions fill the rows of ids that do not occur (one stretch of rows each,
// the ids that occur in it marked in LDS).  One launch: 2,509 ids of a table of 10,000 x 64 fp32 rows 9 us, where
// the sort below would be six launches.
constexpr int64_t kFewIds = 4096;
constexpr int kZeroRows = 64;      // rows of the table per zero-filling workgroup at least
constexpr int kMarkWords = 1024;   // marks of at most 32,768 rows

template <int G, bool BF>
__global__ void __launch_bounds__(256) k_embedding_grad_few(const u32x4e *__restrict__ dout, int64_t ld16,
                                                            int32_t units, int64_t d, const int32_t *__restrict__ ids,
                                                            const int32_t *__restrict__ n_dev, int32_t n, float scale,
                                                            bool accumulate, u32x4e *__restrict__ dtable,
                                                            int64_t n_rows, int64_t table_ld16, int32_t positions,
                                                            int32_t zero_rows) {
    constexpr int RPW = kWave / G, PAR = 4 * RPW, N = Unit<BF>::N;
    __shared__ union {
        struct {
            uint16_t list[kFewIds];
            int32_t counts[4];
        } p;
        uint32_t marks[kMarkWords];
    } sh;
    __shared__ float part[4][kWave][N];
    const int tid = threadIdx.x, lane = lane_id(), wid = tid / kWave;
    if (n_dev) n = std::min(n, std::max(*n_dev, 0));
    if ((int32_t)blockIdx.x >= positions) {
        const int64_t lo = (int64_t)(blockIdx.x - positions) * zero_rows;
        const int64_t hi = std::min<int64_t>(lo + zero_rows, n_rows);
        for (int32_t w = tid; w < (zero_rows + 31) / 32; w += 256) sh.marks[w] = 0;
        __syncthreads();
        for (int32_t i = tid; i < n; i += 256) {
            const int64_t v = ids[i];
            if (v >= lo && v < hi) atomicOr(&sh.marks[(v - lo) >> 5], 1u << ((v - lo) & 31));
        }
        __syncthreads();
        for (int64_t r = lo + wid * RPW + lane / G; r < hi; r += 4 * RPW) {
            if ((sh.marks[(r - lo) >> 5] >> ((r - lo) & 31)) & 1) continue;
            for (int32_t c = lane % G; c < units; c += G) dtable[r * table_ld16 + c] = u32x4e{0, 0, 0, 0};
        }
        return;
    }
    const int32_t p = blockIdx.x;
    if (p >= n) return;
    const int32_t id = ids[p];
    if (id < 0 || id >= n_rows) return;
    // positions of the id: each wavefront looks through a quarter of the list
    constexpr int PER = kFewIds / 4 / kWave;
    int32_t seen[PER];
    const int32_t b = wid * (kFewIds / 4);
#pragma unroll
    for (int k = 0; k < PER; ++k) seen[k] = b + k * kWave + lane < n ? ids[b + k * kWave + lane] : -1;
    int32_t mine = 0;
    bool earlier = false;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const bool hit = seen[k] == id;
        earlier = earlier || (hit && b + k * kWave + lane < p);
        mine += __popcll(__ballot(hit));
    }
    if (lane == 0) sh.p.counts[wid] = mine;
    if (__syncthreads_or(earlier)) return;
    int32_t at = 0, total = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        at += w < wid ? sh.p.counts[w] : 0;
        total += sh.p.counts[w];
    }
    auto put = [&](Unit<BF> &sum, int32_t c) {
        Unit<BF> old;
        u32x4e *to = dtable + (int64_t)id * table_ld16 + c;
        old.zero();
        if (accumulate) old.from(*to);
#pragma unroll
        for (int q = 0; q < N; ++q) sum.v[q] = old.v[q] + scale * sum.v[q];
        *to = sum.to((int64_t)c * N, d);
    };
    if (total == 1) {   // most ids of a frontier
        for (int32_t c = tid; c < units; c += 256) {
            Unit<BF> x;
            x.from(dout[(int64_t)p * ld16 + c]);
            put(x, c);
        }
        return;
    }
    if (mine > 0)
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const bool hit = seen[k] == id;
            const uint64_t m = __ballot(hit);
            if (hit) sh.p.list[at + __popcll(m & ((1ull << lane) - 1ull))] = (uint16_t)(b + k * kWave + lane);
            at += __popcll(m);
        }
    __syncthreads();
    const int sub = wid * RPW + lane / G;
    for (int32_t slab = 0; slab < units; slab += G) {
        const int32_t c = slab + lane % G;
        Unit<BF> acc;
        acc.zero();
        if (c < units) {
            int32_t k = sub;
            for (; k + 3 * PAR < total; k += 4 * PAR) {
                u32x4e x[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) x[q] = dout[(int64_t)sh.p.list[k + q * PAR] * ld16 + c];
#pragma unroll
                for (int q = 0; q < 4; ++q) acc.add(x[q]);
            }
            for (; k < total; k += PAR) acc.add(dout[(int64_t)sh.p.list[k] * ld16 + c]);
        }
#pragma unroll
        for (int o = G; o < kWave; o <<= 1)
#pragma unroll
            for (int q = 0; q < N; ++q) acc.v[q] += __shfl_xor(acc.v[q], o, kWave);
        __syncthreads();
#pragma unroll
        for (int q = 0; q < N; ++q) part[wid][lane][q] = acc.v[q];
        __syncthreads();
        if (wid == 0 && lane < G && c < units) {
#pragma unroll
            for (int q = 0; q < N; ++q)
                acc.v[q] = (part[0][lane][q] + part[1][lane][q]) + (part[2][lane][q] + part[3][lane][q]);
            put(acc, c);
        }
    }
}

// ------------------------------------------------------- gradient: the sort
// Stable radix sort of (id, position), digits of at most 10 bits, least
// significant first.  A tile is a number of rounds of 4,096 pairs (one round up to
// a million); there are at most kIdTiles tiles, so every scatter workgroup adds up all tiles' digit counts by
// itself: a pass is two launches.  (Counting the next pass's digits from the scatter, with global additions, is one
// launch less, but popular ids meet at a few counters: 55 us where the two launches take 25.)  Ids outside [0, n_rows) become n_rows and sort to the end.
namespace {

constexpr int kIdThreads = 1024;
constexpr int kIdWaves = kIdThreads / kWave;
constexpr int kIdIters = 4;
constexpr int64_t kIdRound = kIdThreads * kIdIters;
constexpr int64_t kIdTiles = 256;
constexpr int kMaxBits = 10;

struct IdSortPlan {
    int passes, bits, rounds;
    int64_t tiles;
    IdSortPlan(int64_t n, int64_t n_rows) {
        int all = 1;
        while (all < 32 && (int64_t(1) << all) <= n_rows) ++all;   // values 0 .. n_rows
        passes = (all + kMaxBits - 1) / kMaxBits;
        bits = std::max(2, (all + passes - 1) / passes);
        rounds = (int)std::max<int64_t>(1, (n + kIdTiles * kIdRound - 1) / (kIdTiles * kIdRound));
        tiles = std::max<int64_t>(1, (n + kIdRound * rounds - 1) / (kIdRound * rounds));
    }
    int64_t digits() const { return int64_t(1) << bits; }
};

__device__ __forceinline__ uint32_t sort_key(int32_t id, int64_t n_rows) {
    return id < 0 || id >= n_rows ? (uint32_t)n_rows : (uint32_t)id;
}

}  // namespace

// Digit counts of a pass; in the first one (ids as given), workgroups past the tiles clear the flags.
template <bool FIRST>
__global__ void __launch_bounds__(kIdThreads) k_id_count(const void *__restrict__ in,
                                                         const int32_t *__restrict__ n_dev, int64_t n, int64_t n_rows,
                                                         int shift, int bits, int rounds, int32_t *__restrict__ hist,
                                                         int64_t tiles, uint32_t *__restrict__ flags,
                                                         int64_t flag_words) {
    __shared__ int32_t h[1 << kMaxBits];
    if (n_dev) n = std::min<int64_t>(n, std::max<int32_t>(*n_dev, 0));
    const int64_t digits = int64_t(1) << bits;
    if (blockIdx.x < tiles) {
        h[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll 8
        for (int it = 0; it < kIdIters * rounds; ++it) {
            const int64_t e = ((int64_t)blockIdx.x * kIdIters * rounds + it) * kIdThreads + threadIdx.x;
            if (e >= n) continue;
            const uint32_t key = FIRST ? sort_key(((const int32_t *)in)[e], n_rows) : (uint32_t)((const int2 *)in)[e].x;
            atomicAdd(&h[(key >> shift) & (digits - 1)], 1);
        }
        __syncthreads();
        if (threadIdx.x < digits) hist[blockIdx.x * digits + threadIdx.x] = h[threadIdx.x];
        return;
    }
    const int64_t stride = (int64_t)(gridDim.x - tiles) * kIdThreads;
    for (int64_t i = (int64_t)(blockIdx.x - tiles) * kIdThreads + threadIdx.x; i < flag_words; i += stride) flags[i] = 0;
}

// flags (first pass only, nullable): a byte per row of the table, set where its id occurs.
template <bool FIRST>
__global__ void __launch_bounds__(kIdThreads) k_id_scatter(const void *__restrict__ in,
                                                           const int32_t *__restrict__ n_dev, int64_t n,
                                                           int64_t n_rows, int shift, int bits, int rounds,
                                                           const int32_t *__restrict__ hist, int64_t tiles,
                                                           int2 *__restrict__ out,
                                                           uint8_t *__restrict__ flags) {
    __shared__ int32_t run[1 << kMaxBits];
    __shared__ __align__(16) int32_t cnt[kIdWaves][1 << kMaxBits];
    __shared__ int32_t scratch[kIdWaves];
    if (n_dev) n = std::min<int64_t>(n, std::max<int32_t>(*n_dev, 0));
    const int64_t base = (int64_t)blockIdx.x * kIdRound * rounds;
    if (base >= n) return;
    const int lane = lane_id(), wid = threadIdx.x / kWave, digits = 1 << bits;
    // a digit's count in all tiles and in those before this one: four digits a thread, the tiles dealt to the threads that
    // share them
    int32_t all = 0, before = 0;
    {
        typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
        const int quads = digits / 4, quad = threadIdx.x & (quads - 1), first = threadIdx.x / quads, step = kIdThreads / quads;
        i32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
#pragma unroll 16
        for (int t = first; t < (int)tiles; t += step) {
            const i32x4 c = ((const i32x4 *)hist)[t * quads + quad];
            a += c;
            if (t < (int)blockIdx.x) b += c;
        }
        int32_t *sum = &cnt[0][0];   // [step][digits] twice, 4 * kIdThreads each
        ((i32x4 *)sum)[threadIdx.x] = a;
        ((i32x4 *)sum)[kIdThreads + threadIdx.x] = b;
        __syncthreads();
        for (int q = 0; q < step && (int)threadIdx.x < digits; ++q) {
            all += sum[q * digits + threadIdx.x];
            before += sum[4 * kIdThreads + q * digits + threadIdx.x];
        }
        __syncthreads();
        if ((int)threadIdx.x < digits)
#pragma unroll
            for (int w = 0; w < kIdWaves; ++w) cnt[w][threadIdx.x] = 0;
    }
    int32_t total;
    const int32_t off = block_exclusive_sum<int32_t, kIdThreads>(all, scratch, total) + before;
    if ((int)threadIdx.x < digits) run[threadIdx.x] = off;
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1ull;
    for (int r = 0; r < rounds; ++r) {
        const int64_t at = base + (int64_t)r * kIdRound;
        if (at >= n) break;
        // a wavefront's run of the round: each pair's place among the wavefront's of its digit
        uint32_t key[kIdIters];
        int32_t val[kIdIters], place[kIdIters];
#pragma unroll
        for (int it = 0; it < kIdIters; ++it) {
            const int64_t e = at + (wid * kIdIters + it) * kWave + lane;
            key[it] = 0;
            val[it] = (int32_t)e;
            if (e < n) {
                if constexpr (FIRST) {
                    key[it] = sort_key(((const int32_t *)in)[e], n_rows);
                } else {
                    const int2 p = ((const int2 *)in)[e];
                    key[it] = (uint32_t)p.x;
                    val[it] = p.y;
                }
            }
        }
#pragma unroll
        for (int it = 0; it < kIdIters; ++it) {
            const bool valid = at + (wid * kIdIters + it) * kWave + lane < n;
            if (FIRST && flags && valid && key[it] < (uint32_t)n_rows) flags[key[it]] = 1;
            const int dg = (int)(key[it] >> shift) & (digits - 1);
            uint64_t m = __ballot(valid);
            for (int bit = 0; bit < bits; ++bit) {
                const uint64_t ones = __ballot((dg >> bit) & 1);
                m &= ((dg >> bit) & 1) ? ones : ~ones;
            }
            const int rank = __popcll(m & below);
            const int32_t earlier = valid ? cnt[wid][dg] : 0;
            if (valid && rank == 0) cnt[wid][dg] = earlier + __popcll(m);
            place[it] = earlier + rank;
        }
        __syncthreads();
        if ((int)threadIdx.x < digits) {   // exclusive sums over the wavefronts, from the digit's place
            int32_t to = run[threadIdx.x];
#pragma unroll
            for (int w = 0; w < kIdWaves; ++w) {
                const int32_t c = cnt[w][threadIdx.x];
                cnt[w][threadIdx.x] = to;
                to += c;
            }
            run[threadIdx.x] = to;
        }
        __syncthreads();
#pragma unroll
        for (int it = 0; it < kIdIters; ++it)
            if (at + (wid * kIdIters + it) * kWave + lane < n) {
                const int32_t pos = cnt[wid][(key[it] >> shift) & (digits - 1)] + place[it];
                out[pos] = make_int2((int32_t)key[it], val[it]);
            }
        __syncthreads();
        if ((int)threadIdx.x < digits)
#pragma unroll
            for (int w = 0; w < kIdWaves; ++w) cnt[w][threadIdx.x] = 0;
        __syncthreads();
    }
}

// ------------------------------------------------ gradient: stretches of ids
// A lane group takes a stretch of sorted pairs and adds up the rows of equal ids.
// An id that lies inside the stretch is written at once; the part of one that
// began earlier goes to part[2 * stretch], of one that begins here and goes on to
// part[2 * stretch + 1].  Workgroups past the stretches fill the rows of ids that
// do not occur.  Q units of a row per lane, wider rows in slabs (blockIdx.y).  Bound by HBM: 260,003 rows of
// 602 fp32 into 233,000, 273 us, 4.6 TB/s by the counters; 524,288 skewed ones of 256 bf16 79 us, 4.7 TB/s.  Stretches of 32 ids join
// more parts (skewed 151 -> 158 us in all), of 128 leave units idle (168).  Where stretches of 64 are fewer than
// kFullWaves wavefronts their loads are too few to hide each other: they are halved, to 8 at the least (7,124 ids of
// 272 bf16 73 -> 37 us in all, 43,847 skewed ones of 100 83 -> 51; kFullWaves of 4,096: 218,815 skewed ones of 584 fp32
// 158 -> 172).
constexpr int kStretch = 64, kShortStretch = 8, kFullWaves = 1024;

namespace {
int stretch_of(int64_t n, int32_t units) {
    const int64_t per = kWave / lane_group(units);
    int len = kStretch;
    while (len > kShortStretch && (n + len * per - 1) / (len * per) < kFullWaves) len /= 2;
    return len;
}
}  // namespace

template <int G, int Q, bool BF, bool STREAMED>
__global__ void __launch_bounds__(256) k_embedding_grad(const u32x4e *__restrict__ dout, int64_t ld16, int32_t units,
                                                        int64_t d, const int2 *__restrict__ pairs,
                                                        const int32_t *__restrict__ n_dev, int64_t n, float scale,
                                                        bool accumulate, u32x4e *__restrict__ dtable, int64_t n_rows,
                                                        int64_t table_ld16, float *__restrict__ part,
                                                        const uint8_t *__restrict__ flags, int64_t blocks,
                                                        int32_t stretch) {
    constexpr int RPW = kWave / G, N = Unit<BF>::N;
    const int lane = lane_id(), sub = lane / G, cl = lane % G;
    if (n_dev) n = std::min<int64_t>(n, std::max<int32_t>(*n_dev, 0));
    const int32_t c0 = (int32_t)blockIdx.y * (G * Q) + cl;
    if ((int64_t)blockIdx.x >= blocks) {
        const int64_t waves = (int64_t)(gridDim.x - blocks) * 4;
        const int64_t w0 = (int64_t)(blockIdx.x - blocks) * 4 + threadIdx.x / kWave;
        for (int64_t r0 = w0 * kWave; r0 < n_rows; r0 += waves * kWave) {
            const bool mine = r0 + lane < n_rows && flags[r0 + lane] == 0;
            uint64_t m = __ballot(mine);
            while (m) {   // RPW rows at a time
                uint64_t left = m;
                int row = -1;
#pragma unroll
                for (int k = 0; k < RPW; ++k) {
                    const int at = left ? __builtin_ctzll(left) : -1;
                    if (k == sub) row = at;
                    left = left ? left & (left - 1) : 0;
                }
                m = left;
                if (row >= 0)
#pragma unroll
                    for (int q = 0; q < Q; ++q)
                        if (c0 + q * G < units) store<STREAMED>(&dtable[(r0 + row) * table_ld16 + c0 + q * G], u32x4e{0, 0, 0, 0});
            }
        }
        return;
    }
    const int64_t st = ((int64_t)blockIdx.x * 4 + threadIdx.x / kWave) * RPW + sub;
    const int64_t b = st * stretch, e = std::min<int64_t>(b + stretch, n);
    const int64_t padded = (int64_t)units * N;
    const int32_t before = b > 0 && b < n ? pairs[b - 1].x : -1, after = e < n && b < n ? pairs[e].x : -1;
    Unit<BF> acc[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) acc[q].zero();
    auto flush = [&](int32_t id, bool began, bool ended) {
        if (id >= n_rows) return;
        if (began && ended) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int32_t c = c0 + q * G;
                if (c >= units) continue;
                u32x4e *to = dtable + (int64_t)id * table_ld16 + c;
                Unit<BF> o;
                o.zero();
                if (accumulate) o.from(*to);
#pragma unroll
                for (int x = 0; x < N; ++x) o.v[x] += scale * acc[q].v[x];
                store<STREAMED>(to, o.to((int64_t)c * N, d));
            }
        } else {
            float *to = part + (2 * st + (began ? 1 : 0)) * padded;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int32_t c = c0 + q * G;
                if (c >= units) continue;
#pragma unroll
                for (int x = 0; x < N; x += 4)
                    *(f32x4e *)(to + (int64_t)c * N + x) = f32x4e{acc[q].v[x], acc[q].v[x + 1], acc[q].v[x + 2], acc[q].v[x + 3]};
            }
        }
    };
    constexpr int U = Q == 1 ? 8 : 4;   // rows in flight; their ids are read one round ahead
    int32_t cur = b < n ? pairs[b].x : -1;
    bool began = b < n && cur != before;
    int32_t key[U], row[U];
    auto ids = [&](int i0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t p = b + i0 + u;
            const int2 pair = p < e ? pairs[p] : make_int2(-1, 0);
            key[u] = pair.x;
            row[u] = pair.y;
        }
    };
    ids(0);
    // the loop's trip count is the same for all lane groups of a wavefront
    for (int i0 = 0; i0 < stretch; i0 += U) {
        u32x4e x[U][Q];
        int32_t now[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            now[u] = key[u];
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                x[u][q] = u32x4e{0, 0, 0, 0};
                if (key[u] >= 0 && key[u] < n_rows && c0 + q * G < units) x[u][q] = dout[(int64_t)row[u] * ld16 + c0 + q * G];
            }
        }
        if (i0 + U < stretch) ids(i0 + U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (now[u] < 0) continue;
            if (now[u] != cur) {
                flush(cur, began, true);
                cur = now[u];
                began = true;
#pragma unroll
                for (int q = 0; q < Q; ++q) acc[q].zero();
            }
#pragma unroll
            for (int q = 0; q < Q; ++q) acc[q].add(x[u][q]);
        }
    }
    if (b < n) flush(cur, began, cur != after);
}

// Joins the parts of ids that span stretches: the part of the stretch where such
// an id begins and those of the stretches up to its last one, in order.  A
// wavefront takes a stretch; what goes on over more than kJoinLong others is left
// to the whole workgroup, an eighth of the parts per wavefront.
constexpr int kJoinWaves = 8, kJoinLong = 16;

template <bool BF>
__global__ void __launch_bounds__(64 * kJoinWaves) k_embedding_grad_join(const int2 *__restrict__ pairs,
                                                                         const int32_t *__restrict__ n_dev, int64_t n,
                                                                         int32_t units, int64_t d, float scale,
                                                                         bool accumulate, u32x4e *__restrict__ dtable,
                                                                         int64_t n_rows, int64_t table_ld16,
                                                                         const float *__restrict__ part,
                                                                         int32_t stretch) {
    constexpr int N = Unit<BF>::N;
    __shared__ float sums[kJoinWaves][kWave][N];
    __shared__ int32_t s_rest[kJoinWaves];
    if (n_dev) n = std::min<int64_t>(n, std::max<int32_t>(*n_dev, 0));
    const int lane = lane_id(), wid = threadIdx.x / kWave;
    const int64_t padded = (int64_t)units * N;
    // parts [k0, k1) of those after stretch st, unit c; the stretch's own first if `first`
    auto add = [&](float (&acc)[N], int64_t st, int64_t k0, int64_t k1, int32_t c, bool first) {
        const float *at = part + (int64_t)c * N;
#pragma unroll
        for (int x = 0; x < N; ++x) acc[x] = first ? at[(2 * st + 1) * padded + x] : 0.f;
        int64_t k = k0;
        for (; k + 4 <= k1; k += 4) {   // four at a time, so that thousands of parts round a quarter as often
            f32x4e v[4][N / 4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int x = 0; x < N / 4; ++x) v[u][x] = *(const f32x4e *)(at + 2 * (st + 1 + k + u) * padded + 4 * x);
#pragma unroll
            for (int x = 0; x < N; ++x)
                acc[x] += (v[0][x / 4][x % 4] + v[1][x / 4][x % 4]) + (v[2][x / 4][x % 4] + v[3][x / 4][x % 4]);
        }
        for (; k < k1; ++k)
#pragma unroll
            for (int x = 0; x < N; ++x) acc[x] += at[2 * (st + 1 + k) * padded + x];
    };
    auto put = [&](const float (&acc)[N], int32_t id, int32_t c) {
        u32x4e *to = dtable + (int64_t)id * table_ld16 + c;
        Unit<BF> o;
        o.zero();
        if (accumulate) o.from(*to);
#pragma unroll
        for (int x = 0; x < N; ++x) o.v[x] += scale * acc[x];
        *to = o.to((int64_t)c * N, d);
    };
    for (int64_t base = (int64_t)blockIdx.x * kJoinWaves; (base + 1) * stretch < n; base += (int64_t)gridDim.x * kJoinWaves) {
        const int64_t st = base + wid, b = st * stretch, e = b + stretch;
        int32_t rest = 0;   // stretches after this one that the id goes on in
        if (e < n) {
            const int32_t id = pairs[e - 1].x;
            const bool begins = !(pairs[b].x == id && b > 0 && pairs[b - 1].x == id);
            if (id < n_rows && begins && pairs[e].x == id)
                for (;;) {
                    const int64_t p = (st + 1 + rest + lane) * stretch;
                    const uint64_t on = __ballot(p < n && pairs[p < n ? p : n - 1].x == id);
                    if (on != ~0ull) {
                        rest += __builtin_ctzll(~on);
                        break;
                    }
                    rest += kWave;
                }
        }
        if (lane == 0) s_rest[wid] = rest > kJoinLong ? rest : 0;
        if (rest > 0 && rest <= kJoinLong)
            for (int32_t c = lane; c < units; c += kWave) {
                float acc[N];
                add(acc, st, 0, rest, c, true);
                put(acc, pairs[e - 1].x, c);
            }
        __syncthreads();
        for (int w = 0; w < kJoinWaves; ++w) {
            const int32_t all = s_rest[w];
            if (all == 0) continue;
            const int64_t from = base + w, share = (all + kJoinWaves - 1) / kJoinWaves;
            const int64_t k0 = std::min<int64_t>(wid * share, all), k1 = std::min<int64_t>(k0 + share, all);
            for (int32_t slab = 0; slab < units; slab += kWave) {
                const int32_t c = slab + lane;
                float acc[N];
                if (c < units) {
                    add(acc, from, k0, k1, c, wid == 0);
#pragma unroll
                    for (int x = 0; x < N; ++x) sums[wid][lane][x] = acc[x];
                }
                __syncthreads();
                if (wid == 0 && c < units) {
                    for (int v = 1; v < kJoinWaves; ++v)
#pragma unroll
                        for (int x = 0; x < N; ++x) acc[x] += sums[v][lane][x];
                    put(acc, pairs[(from + 1) * stretch - 1].x, c);
                }
                __syncthreads();
            }
        }
        __syncthreads();
    }
}

namespace {
// Workspace of the gradient: two lists of (id, position), the digit counts of a
// pass, a byte per table row, the part sums.
struct GradWorkspace {
    size_t pairs[2], hist, flags, part, total;
    GradWorkspace(int64_t n, int64_t n_rows, int64_t d, bool bf16) {
        const IdSortPlan p(n, n_rows);
        const int64_t units = (d * (bf16 ? 2 : 4) + 15) / 16, padded = units * (bf16 ? 8 : 4);
        const int64_t stretch = stretch_of(n, (int32_t)units);
        size_t at = 0;
        auto take = [&](size_t bytes) {
            const size_t here = at;
            at += (bytes + 255) / 256 * 256;
            return here;
        };
        for (int k = 0; k < 2; ++k) pairs[k] = take((size_t)n * 8);
        hist = take((size_t)(p.tiles * p.digits()) * 4);
        flags = take((size_t)n_rows);
        part = take((size_t)(2 * ((n + stretch - 1) / stretch) * padded) * 4);
        total = at;
    }
};
}  // namespace

size_t embedding_backward_workspace(int64_t n, int64_t n_rows, int64_t d, bool bf16) {
    return n <= kFewIds ? 0 : GradWorkspace(n, n_rows, d, bf16).total;
}

void launch_embedding_backward(const void *dout, int64_t ld_bytes, const int32_t *ids, const int32_t *n_dev,
                               int64_t n, int64_t d, bool bf16, float scale, bool accumulate, void *dtable,
                               int64_t n_rows, int64_t table_ld_bytes, void *ws, hipStream_t s) {
    if (n_rows <= 0 || (n <= 0 && accumulate)) return;
    const int32_t units = (int32_t)((d * (bf16 ? 2 : 4) + 15) / 16);
    const int g = lane_group(units);
    const u32x4e *in = (const u32x4e *)dout;
    u32x4e *out = (u32x4e *)dtable;
    const int64_t ld16 = ld_bytes / 16, tld16 = table_ld_bytes / 16;
    if (n <= kFewIds) {
        KernelTimer t("embedding_grad_few", s);
        int64_t zero_rows = (n_rows + 511) / 512;   // two workgroups per compute unit fill zeros
        zero_rows = std::max<int64_t>(kZeroRows, std::min<int64_t>(zero_rows, kMarkWords * 32));
        const int64_t zeros = accumulate ? 0 : (n_rows + zero_rows - 1) / zero_rows;
#define GNNAV_L(GV)                                                                                                   \
    case GV:                                                                                                          \
        if (bf16)                                                                                                     \
            hipLaunchKernelGGL((k_embedding_grad_few<GV, true>), dim3((unsigned)(n + zeros)), dim3(256), 0, s, in,    \
                               ld16, units, d, ids, n_dev, (int32_t)n, scale, accumulate, out, n_rows, tld16,         \
                               (int32_t)n, (int32_t)zero_rows);                                                       \
        else                                                                                                          \
            hipLaunchKernelGGL((k_embedding_grad_few<GV, false>), dim3((unsigned)(n + zeros)), dim3(256), 0, s, in,   \
                               ld16, units, d, ids, n_dev, (int32_t)n, scale, accumulate, out, n_rows, tld16,         \
                               (int32_t)n, (int32_t)zero_rows);                                                       \
        break
        switch (g) {
            GNNAV_L(1);
            GNNAV_L(2);
            GNNAV_L(4);
            GNNAV_L(8);
            GNNAV_L(16);
            GNNAV_L(32);
            default: GNNAV_L(64);
        }
#undef GNNAV_L
        GNNAV_HIP(hipGetLastError());
        return;
    }
    const GradWorkspace w(n, n_rows, d, bf16);
    const IdSortPlan p(n, n_rows);
    char *base = (char *)ws;
    auto i32 = [&](size_t at) { return (int32_t *)(base + at); };
    int32_t *hist = i32(w.hist);
    uint8_t *flags = accumulate ? nullptr : (uint8_t *)(base + w.flags);
    const void *in_ids = ids;   // the list to sort, then what the last pass wrote
    {
        KernelTimer t("embedding_sort", s);
        const int64_t words = accumulate ? 0 : (n_rows + 3) / 4;
        for (int k = 0; k < p.passes; ++k) {
            int2 *to = (int2 *)(base + w.pairs[k & 1]);
            const int shift = k * p.bits;
            if (k == 0) {
                hipLaunchKernelGGL(k_id_count<true>, dim3((unsigned)p.tiles + (words ? grid_for(words, kIdThreads, 256) : 0)),
                                   dim3(kIdThreads), 0, s, in_ids, n_dev, n, n_rows, shift, p.bits, p.rounds, hist, p.tiles,
                                   (uint32_t *)flags, words);
                hipLaunchKernelGGL(k_id_scatter<true>, dim3((unsigned)p.tiles), dim3(kIdThreads), 0, s, in_ids, n_dev,
                                   n, n_rows, shift, p.bits, p.rounds, hist, p.tiles, to, flags);
            } else {
                hipLaunchKernelGGL(k_id_count<false>, dim3((unsigned)p.tiles), dim3(kIdThreads), 0, s, in_ids, n_dev, n,
                                   n_rows, shift, p.bits, p.rounds, hist, p.tiles, nullptr, 0);
                hipLaunchKernelGGL(k_id_scatter<false>, dim3((unsigned)p.tiles), dim3(kIdThreads), 0, s, in_ids, n_dev,
                                   n, n_rows, shift, p.bits, p.rounds, hist, p.tiles, to, nullptr);
            }
            in_ids = to;
        }
    }
    float *part = (float *)(base + w.part);
    const int2 *pairs = (const int2 *)in_ids;
    const int32_t stretch = stretch_of(n, units);
    {
        KernelTimer t("embedding_grad", s);
        const int64_t stretches = (n + stretch - 1) / stretch;
        const int64_t blocks = (stretches + 4 * (kWave / g) - 1) / (4 * (kWave / g));
        const unsigned zeros = accumulate ? 0u : grid_for(n_rows, 256, 1024);
        const bool streamed = n_rows * units * 16 > kStreamBytes;
        const unsigned slabs = (unsigned)((units + 3 * kWave - 1) / (3 * kWave));
        const int q = (int)((units + g * slabs - 1) / (g * slabs));
        auto launch = [&](auto gq_, auto bf_, auto st_) {
            constexpr int GV = decltype(gq_)::value / 4, QV = decltype(gq_)::value % 4;
            hipLaunchKernelGGL((k_embedding_grad<GV, QV, decltype(bf_)::value, decltype(st_)::value>),
                               dim3((unsigned)blocks + zeros, slabs), dim3(256), 0, s, in, ld16, units, d, pairs, n_dev, n, scale,
                               accumulate, out, n_rows, tld16, part, flags, blocks, stretch);
        };
#define GNNAV_L(GV, QV) by_type(launch, std::integral_constant<int, 4 * GV + QV>{}, bf16, streamed)
        switch (g) {
            case 1: GNNAV_L(1, 1); break;
            case 2: GNNAV_L(2, 1); break;
            case 4: GNNAV_L(4, 1); break;
            case 8: GNNAV_L(8, 1); break;
            case 16: GNNAV_L(16, 1); break;
            case 32: GNNAV_L(32, 1); break;
            default:
                if (q == 1) GNNAV_L(64, 1);
                else if (q == 2) GNNAV_L(64, 2);
                else GNNAV_L(64, 3);
        }
#undef GNNAV_L
        GNNAV_HIP(hipGetLastError());
    }
    {
        KernelTimer t("embedding_grad_join", s);
        const unsigned grid = grid_for((n + stretch - 1) / stretch, kJoinWaves, 2048);
        if (bf16)
            hipLaunchKernelGGL(k_embedding_grad_join<true>, dim3(grid), dim3(64 * kJoinWaves), 0, s, pairs, n_dev, n, units, d,
                               scale, accumulate, out, n_rows, tld16, part, stretch);
        else
            hipLaunchKernelGGL(k_embedding_grad_join<false>, dim3(grid), dim3(64 * kJoinWaves), 0, s, pairs, n_dev, n, units, d,
                               scale, accumulate, out, n_rows, tld16, part, stretch);
    }
    GNNAV_HIP(hipGetLastError());
}

}  // namespace gnnav
