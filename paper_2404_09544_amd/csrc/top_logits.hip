// The k largest logits of each row, in falling order, ties to the lowest class.
//
// A logit and its class are one 64-bit number, the logit's order above the class' complement: no two are equal, and
// the largest numbers are the answer.  Three kernels:
//
//   k_top_strip  a wavefront walks a row, or a strip of it, in order and keeps its k largest sorted over its lanes.  What is
//                above the k-th of them goes to a buffer in LDS; a full buffer is sorted over the lanes and joined to the
//                list (the larger of a falling and a rising list, place by place, is a bitonic one).  The k-th largest of the
//                lanes' largest of the first logits is where it starts from: k logits are not below it.  On random logits
//                some k log(n / k) of n are ever appended, so a logit costs a comparison and the row is read once; of a
//                rising row all are, and every block is sorted: 1,024 x 169,000 fp32, k = 32, 989 us instead of 142 (bf16 742 and
//                88), one such row, in strips, 22 instead of 16.
//   k_top_join   joins the strips' lists where long rows of few are cut.
//   k_top_rows   many short rows and small k: a lane a row, its list in registers.
#include <algorithm>

#include "common.hpp"
#include "lanes.hpp"

namespace gnnav {

namespace {

typedef uint32_t u32x4x __attribute__((ext_vector_type(4)));

// A logit's place in the order: -inf lowest, both zeros equal, NaN above +inf.  Never 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t u = __float_as_uint(x + 0.f);   // -0 becomes 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t order) {
    return __uint_as_float(order & 0x80000000u ? (order == 0xffffffffu ? 0x7fc00000u : order & 0x7fffffffu) : ~order);
}

// The lanes of register r that keep the larger number of their pair in one step of a bitonic network over places
// r * 64 + lane: falling where (place & block) == 0, rising elsewhere, and the other way round if `rising`.
constexpr uint64_t larger_lanes(int r, int stride, int block, bool rising) {
    uint64_t m = 0;
    for (int l = 0; l < 64; ++l) {
        const bool down = (((r * 64 + l) & block) == 0) != rising, low = (l & stride) == 0;
        if (down == low) m |= 1ull << l;
    }
    return m;
}

template <int KR, int STRIDE, int BLOCK, bool RISING>
__device__ __forceinline__ void exchange(uint64_t (&x)[KR]) {
    if constexpr (STRIDE >= 64) {
#pragma unroll
        for (int r = 0; r < KR; ++r) {
            constexpr int RS = STRIDE / 64;
            if (r & RS) continue;
            const bool down = (((r * 64) & BLOCK) == 0) != RISING;
            const uint64_t a = x[r], b = x[(r | RS) & (KR - 1)];
            const bool swap = down ? a < b : a > b;
            x[r] = swap ? b : a;
            x[(r | RS) & (KR - 1)] = swap ? a : b;
        }
    } else {
        auto one = [&](auto r_) {
            constexpr int r = decltype(r_)::value;
            constexpr uint64_t keep = larger_lanes(r, STRIDE, BLOCK, RISING);
            const uint32_t lo = (uint32_t)x[r], hi = (uint32_t)(x[r] >> 32);
            uint64_t a, b;
            if constexpr (STRIDE >= 16) {
                const LanePair l = lane_pair<STRIDE>(lo), h = lane_pair<STRIDE>(hi);
                a = (uint64_t)h.low << 32 | l.low;
                b = (uint64_t)h.high << 32 | l.high;
            } else {
                a = x[r];
                b = (uint64_t)lane_xor<STRIDE>(hi) << 32 | lane_xor<STRIDE>(lo);
            }
            x[r] = __builtin_amdgcn_inverse_ballot_w64(__builtin_amdgcn_ballot_w64(a < b) ^ ~keep) ? b : a;
        };
        one(std::integral_constant<int, 0>());
        if constexpr (KR > 1) one(std::integral_constant<int, 1>());
        if constexpr (KR > 2) {
            one(std::integral_constant<int, 2>());
            one(std::integral_constant<int, 3>());
        }
    }
}
template <int KR, int STRIDE, int BLOCK, bool RISING>
__device__ __forceinline__ void strides(uint64_t (&x)[KR]) {
    exchange<KR, STRIDE, BLOCK, RISING>(x);
    if constexpr (STRIDE > 1) strides<KR, STRIDE / 2, BLOCK, RISING>(x);
}
// 64 KR numbers, place r * 64 + lane, in falling or rising order.
template <int KR, bool RISING, int BLOCK = 2>
__device__ __forceinline__ void sort(uint64_t (&x)[KR]) {
    constexpr int N = 64 * KR;
    strides<KR, BLOCK / 2, BLOCK == N ? 0 : BLOCK, RISING>(x);
    if constexpr (BLOCK < N) sort<KR, RISING, BLOCK * 2>(x);
}
// A falling list and a rising one: the 64 KR largest of both, falling.
template <int KR>
__device__ __forceinline__ void merge(uint64_t (&best)[KR], const uint64_t (&rising)[KR]) {
#pragma unroll
    for (int r = 0; r < KR; ++r) best[r] = best[r] < rising[r] ? rising[r] : best[r];
    strides<KR, 32 * KR, 0, false>(best);
}

// The number at place i, in every lane (i the same in all).
template <int KR>
__device__ __forceinline__ uint64_t number_at(const uint64_t (&x)[KR], int i) {
    uint32_t lo = 0, hi = 0;
#pragma unroll
    for (int r = 0; r < KR; ++r)
        if (r == i / 64) {
            lo = __builtin_amdgcn_readlane((uint32_t)x[r], i % 64);
            hi = __builtin_amdgcn_readlane((uint32_t)(x[r] >> 32), i % 64);
        }
    return (uint64_t)hi << 32 | lo;
}

// A wavefront's walk: its list and the buffer of what is above `least`, at most the order of the list's k-th number.  What
// comes later in the row and is not above it has no place: of equal logits the earlier class goes first.
template <int KR>
struct Walk {
    uint64_t best[KR];
    uint64_t *buffer;   // LDS: a vector's logits of all lanes behind 64 KR numbers
    int count = 0, k;
    uint32_t least = 0;
    float bar;          // the logit above `least`, NaN while everything is
    __device__ __forceinline__ Walk(uint64_t *b, int kk) : buffer(b), k(kk) {
#pragma unroll
        for (int r = 0; r < KR; ++r) best[r] = 0;
        set(0);
    }
    __device__ __forceinline__ void set(uint32_t order) {
        least = order;
        bar = logit_of(order + 1);   // (of 0 and 1: NaN)
    }
    // each lane's logits from class `at` on whose bit is set in `bits`
    template <bool BF>
    __device__ __forceinline__ void offer(const u32x4x &v, uint32_t at, uint32_t bits) {
        while (__any(bits != 0)) {
            const int e = __ffs((int)bits) - 1, w = BF ? e >> 1 : e;
            const uint32_t word = w < 2 ? (w < 1 ? v[0] : v[1]) : (w < 3 ? v[2] : v[3]);
            const uint32_t order = order_of(__uint_as_float(BF ? (e & 1 ? word & 0xffff0000u : word << 16) : word));
            const bool take = bits != 0 && order > least;
            const uint64_t mask = __ballot(take);
            const int place = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, count));
            if (take) buffer[place] = (uint64_t)order << 32 | ~(at + e);
            count += __popcll(mask);
            bits &= bits - 1;
        }
    }
    // joins whole batches of the buffer, or all of it
    __device__ __forceinline__ void settle(bool all) {
        if (count < 64 * KR && !(all && count > 0)) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        while (count >= 64 * KR || (all && count > 0)) {
            const int n = std::min(count, 64 * KR), from = count - n;
            uint64_t fresh[KR];
#pragma unroll
            for (int r = 0; r < KR; ++r) {
                const int i = r * 64 + lane_id();
                fresh[r] = i < n ? buffer[from + i] : 0;
            }
            sort<KR, true>(fresh);
            merge<KR>(best, fresh);
            count = from;
        }
        set(std::max(least, (uint32_t)(number_at<KR>(best, k - 1) >> 32)));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
};

struct TopArgs {
    const void *logits;
    int64_t ld, m, n_classes, width;
    int32_t strips, k;
    float *values;
    int32_t *ids;
    uint64_t *lists;   // [row][strip][k]
};

template <int KR>
__device__ __forceinline__ void write_top(const TopArgs &a, int64_t row, const uint64_t (&best)[KR]) {
#pragma unroll
    for (int r = 0; r < KR; ++r) {
        const int i = r * 64 + lane_id();
        if (i < a.k) {
            a.values[row * a.k + i] = best[r] ? logit_of((uint32_t)(best[r] >> 32)) : -INFINITY;
            a.ids[row * a.k + i] = best[r] ? (int32_t)~(uint32_t)best[r] : -1;
        }
    }
}

}  // namespace

// A wavefront takes columns [strip * width, ...) of a row; four of them a workgroup.  One strip: the answer; else the
// strips' lists.
constexpr int kVectors = 4;   // 16-byte loads of a lane in flight
template <bool BF, int KR>
__global__ void __launch_bounds__(256) k_top_strip(const TopArgs a) {
    constexpr int PER = BF ? 8 : 4, BLOCK = 64 * PER, ELT = BF ? 2 : 4, G = KR == 1 ? 2 : 4;
    __shared__ uint64_t buffers[4][64 * KR + BLOCK];
    const int wid = threadIdx.x / 64, lane = lane_id();
    for (int64_t task = (int64_t)blockIdx.x * 4 + wid; task < a.m * a.strips; task += (int64_t)gridDim.x * 4) {
        const int64_t row = task / a.strips, strip = task % a.strips;
        const int64_t begin = strip * a.width, end = std::min(a.n_classes, begin + a.width);
        const char *src = (const char *)a.logits + row * a.ld * ELT;
        Walk<KR> walk(buffers[wid], a.k);
        for (int64_t c = begin; c < end; c += kVectors * BLOCK) {
            u32x4x v[kVectors];
#pragma unroll
            for (int u = 0; u < kVectors; ++u) {
                const int64_t at = c + u * BLOCK + lane * PER;
                v[u] = u32x4x{0, 0, 0, 0};
                if (at < end) v[u] = *(const u32x4x *)(src + at * ELT);
            }
            if (c == begin && end - c > 64 * G) {
                // each lane's largest, in G groups of its logits (NaN, which is larger, apart): the k-th of all is not above
                // the k-th logit
                constexpr int EACH = kVectors * PER / G;
                uint64_t group[G];
                const bool tail = c + kVectors * BLOCK > end;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    float top = -INFINITY;
#pragma unroll
                    for (int i = g * EACH; i < (g + 1) * EACH; ++i)
                        if (!tail || c + i / PER * BLOCK + lane * PER + i % PER < end) top = fmaxf(top, element<BF>(v[i / PER], i % PER));
                    group[g] = (uint64_t)order_of(top) << 32;
                }
                sort<G, false>(group);
                const uint32_t kth = (uint32_t)(number_at<G>(group, a.k - 1) >> 32);
                walk.set(kth - 1);
            }
#pragma unroll
            for (int u = 0; u < kVectors; ++u) {
                const int64_t from = c + u * BLOCK;
                if (from >= end) break;
                uint64_t some[PER], any = 0;
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    some[e] = __ballot(!(element<BF>(v[u], e) < walk.bar));
                    any |= some[e];
                }
                if (any == 0) continue;
                uint32_t bits = 0;
#pragma unroll
                for (int e = 0; e < PER; ++e) bits |= __builtin_amdgcn_inverse_ballot_w64(some[e]) ? 1u << e : 0u;
                const int64_t left = end - (from + lane * PER);
                if (left < PER) bits &= left > 0 ? (1u << left) - 1 : 0u;
                walk.template offer<BF>(v[u], (uint32_t)(from + lane * PER), bits);
                walk.settle(false);
            }
        }
        walk.settle(true);
        if (a.strips == 1) {
            write_top<KR>(a, row, walk.best);
        } else {
#pragma unroll
            for (int r = 0; r < KR; ++r) {
                const int i = r * 64 + lane;
                if (i < a.k) a.lists[task * a.k + i] = walk.best[r];
            }
        }
    }
}

// The strips' lists of a row, by W wavefronts: each merges every W-th list, then they merge each other's by way of LDS.
template <int KR, int W>
__global__ void __launch_bounds__(W == 1 ? 256 : 64 * W) k_top_join(const TopArgs a) {
    __shared__ uint64_t half[W == 1 ? 1 : W / 2][64 * KR];
    constexpr int ROWS = W == 1 ? 4 : 1, N = 64 * KR;
    const int wid = threadIdx.x / 64, lane = lane_id(), part = W == 1 ? 0 : wid;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + (W == 1 ? wid : 0); row < a.m; row += (int64_t)gridDim.x * ROWS) {
        uint64_t best[KR];
#pragma unroll
        for (int r = 0; r < KR; ++r) best[r] = 0;
        for (int32_t s = part; s < a.strips; s += W) {
            uint64_t list[KR];
#pragma unroll
            for (int r = 0; r < KR; ++r) {
                const int i = N - 1 - (r * 64 + lane);
                list[r] = i < a.k ? a.lists[(row * a.strips + s) * a.k + i] : 0;
            }
            merge<KR>(best, list);
        }
        if constexpr (W > 1) {
#pragma unroll
            for (int w = W / 2; w > 0; w /= 2) {
                if (wid >= w && wid < 2 * w)
#pragma unroll
                    for (int r = 0; r < KR; ++r) half[wid - w][r * 64 + lane] = best[r];
                __syncthreads();
                if (wid < w) {
                    uint64_t list[KR];
#pragma unroll
                    for (int r = 0; r < KR; ++r) list[r] = half[wid][N - 1 - (r * 64 + lane)];
                    merge<KR>(best, list);
                }
                __syncthreads();
            }
        }
        if (wid == 0 || W == 1) write_top<KR>(a, row, best);
    }
}

// Rows of at most 64 KR classes: all of a row sorted over the lanes, four rows a workgroup.
template <bool BF, int KR>
__global__ void __launch_bounds__(256) k_top_short(const TopArgs a) {
    const int wid = threadIdx.x / 64, lane = lane_id();
    for (int64_t row = (int64_t)blockIdx.x * 4 + wid; row < a.m; row += (int64_t)gridDim.x * 4) {
        uint64_t x[KR];
#pragma unroll
        for (int r = 0; r < KR; ++r) {
            const int c = r * 64 + lane;
            x[r] = 0;
            if (c < a.n_classes) {
                float z;
                if constexpr (BF) z = bf16_to_f32(((const uint16_t *)a.logits)[row * a.ld + c]);
                else z = ((const float *)a.logits)[row * a.ld + c];
                x[r] = (uint64_t)order_of(z) << 32 | ~(uint32_t)c;
            }
        }
        sort<KR, false>(x);
        write_top<KR>(a, row, x);
#pragma unroll
        for (int i = KR * 64 + lane; i < a.k; i += 64) {   // (more places than numbers)
            a.values[row * a.k + i] = -INFINITY;
            a.ids[row * a.k + i] = -1;
        }
    }
}

// Rows of few classes, a lane each: its K largest in registers, falling.  A new logit goes to its place by medians: place j
// takes the middle of its own, its neighbour's and the new one.
template <bool BF, int K>
__global__ void __launch_bounds__(256) k_top_rows(const TopArgs a) {
    constexpr int PER = BF ? 8 : 4, ELT = BF ? 2 : 4;
    for (int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x; row < a.m; row += (int64_t)gridDim.x * 256) {
        const char *src = (const char *)a.logits + row * a.ld * ELT;
        uint32_t order[K];
        int32_t cls[K];
#pragma unroll
        for (int j = 0; j < K; ++j) {
            order[j] = 0;
            cls[j] = -1;
        }
        for (int32_t c = 0; c < (int32_t)a.n_classes; c += PER) {
            const u32x4x v = *(const u32x4x *)(src + (int64_t)c * ELT);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const uint32_t x = c + e < (int32_t)a.n_classes ? order_of(element<BF>(v, e)) : 0;
                bool above = x > order[K - 1];
#pragma unroll
                for (int j = K - 1; j > 0; --j) {
                    const bool next = x > order[j - 1];
                    cls[j] = next ? cls[j - 1] : above ? c + e : cls[j];
                    order[j] = next ? order[j - 1] : above ? x : order[j];
                    above = next;
                }
                cls[0] = above ? c + e : cls[0];
                order[0] = above ? x : order[0];
            }
        }
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (j < a.k) {
                a.values[row * a.k + j] = cls[j] >= 0 ? logit_of(order[j]) : -INFINITY;
                a.ids[row * a.k + j] = cls[j];
            }
    }
}

namespace {
// Strips of a row: 4,096 wavefronts (1,024 x 169,000 bf16, k = 32: 93 us; 2,048 115, 8,192 101, with more starts), 1,024 logits
// each at least (1 x 169,000 fp32, k = 64: 16.5 us; 2,048 17.9, 512 16.3).
void cut(int64_t m, int64_t n_classes, int64_t &width, int32_t &strips) {
    const int64_t want = std::max<int64_t>(1, 4096 / std::max<int64_t>(m, 1));
    int64_t n = std::max<int64_t>(1, std::min<int64_t>(want, n_classes / 1024));
    width = ((n_classes + n - 1) / n + 511) / 512 * 512;
    strips = (int32_t)((n_classes + width - 1) / width);
}
}  // namespace

size_t top_logits_workspace(int64_t m, int64_t n_classes, int64_t k) {
    int64_t width;
    int32_t strips;
    cut(m, n_classes, width, strips);
    return strips > 1 ? (size_t)(m * strips * k * 8) : 0;
}

void launch_top_logits(const void *logits, int64_t ld, int64_t m, int64_t n_classes, bool bf16, int32_t k, float *values,
                       int32_t *ids, void *ws, hipStream_t s) {
    TopArgs a = {logits, ld, m, n_classes, 0, 0, k, values, ids, (uint64_t *)ws};
    cut(m, n_classes, a.width, a.strips);
    // A lane a row: its time is a lane's, some classes x places x 17 ns, until there are rows enough; a wavefront a row takes m x
    // 0.26 ns (up to 64 classes), 0.57 (128), 1.1.  fp32: 100,000 x 41, k = 8: 15 us, 26 by wavefronts, k = 16: 32, 26; x 100,
    // k = 16: 51, 57; x 250, k = 8: 60, 112; 20,000 x 41, k = 8: 12, 7; x 250, k = 8: 45, 25
    const int64_t places = k <= 4 ? 4 : k <= 8 ? 8 : 16, rows = n_classes <= 64 ? 128 : n_classes <= 128 ? 64 : 32;
    if (k <= (n_classes <= 64 ? 8 : 16) && n_classes <= 256 && n_classes * places * rows <= m) {
        KernelTimer t("top_rows", s);
        const dim3 grid(grid_for(m, 256, 1 << 20));
#define GNNAV_L(K)                                                                                 \
    do {                                                                                           \
        if (bf16) hipLaunchKernelGGL((k_top_rows<true, K>), grid, dim3(256), 0, s, a);             \
        else hipLaunchKernelGGL((k_top_rows<false, K>), grid, dim3(256), 0, s, a);                 \
    } while (0)
        if (k <= 4) GNNAV_L(4);
        else if (k <= 8) GNNAV_L(8);
        else GNNAV_L(16);
#undef GNNAV_L
        GNNAV_HIP(hipGetLastError());
        return;
    }
    // whole rows sorted: 100,000 x 41 fp32, k = 17: 26 us, 74 by the walk; x 100: 57, 90
    if (n_classes <= 128) {
        KernelTimer t("top_short", s);
        const dim3 grid(grid_for(m, 4, 1 << 20));
#define GNNAV_L(KR)                                                                                \
    do {                                                                                           \
        if (bf16) hipLaunchKernelGGL((k_top_short<true, KR>), grid, dim3(256), 0, s, a);           \
        else hipLaunchKernelGGL((k_top_short<false, KR>), grid, dim3(256), 0, s, a);               \
    } while (0)
        if (n_classes <= 64) GNNAV_L(1);
        else GNNAV_L(2);
#undef GNNAV_L
        GNNAV_HIP(hipGetLastError());
        return;
    }
#define GNNAV_L(KR)                                                                                                      \
    do {                                                                                                                 \
        {                                                                                                                \
            KernelTimer t("top_strip", s);                                                                               \
            const dim3 grid(grid_for(m * a.strips, 4, 1 << 20));                                                         \
            if (bf16) hipLaunchKernelGGL((k_top_strip<true, KR>), grid, dim3(256), 0, s, a);                             \
            else hipLaunchKernelGGL((k_top_strip<false, KR>), grid, dim3(256), 0, s, a);                                 \
        }                                                                                                                \
        if (a.strips > 1) {                                                                                              \
            KernelTimer t("top_join", s);                                                                                \
            if (a.strips > 16) hipLaunchKernelGGL((k_top_join<KR, 16>), dim3(grid_for(m, 1, 1 << 20)), dim3(1024), 0, s, a); \
            else hipLaunchKernelGGL((k_top_join<KR, 1>), dim3(grid_for(m, 4, 1 << 20)), dim3(256), 0, s, a);             \
        }                                                                                                                \
    } while (0)
    if (k <= 64) GNNAV_L(1);
    else if (k <= 128) GNNAV_L(2);
    else GNNAV_L(4);
#undef GNNAV_L
    GNNAV_HIP(hipGetLastError());
}

}  // namespace gnnav
