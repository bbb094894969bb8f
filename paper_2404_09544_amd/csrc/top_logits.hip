// The k largest logits of each row, in falling order, ties to the lowest class.
//
// A logit and its class are one 64-bit number, the logit's order above the class' complement: no two are equal, and
// the largest numbers are the answer.  A wavefront walks its part of a row in order and keeps its k largest sorted over its
// lanes.  What is above the k-th of them is appended to a buffer in LDS; a full buffer is sorted over the lanes and joined
// to the list (the larger of a falling and a rising list, place by place, is a bitonic one).  On random logits
// k log(n / k) of n are ever appended, so a logit costs a comparison, and the row is read once.  Long rows of few are cut into
// strips, whose lists a second launch joins in the same way.
#include <algorithm>

#include "common.hpp"

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

__device__ __forceinline__ uint64_t from_lane(uint64_t x, int lane) {
    const uint32_t lo = __shfl((int)(uint32_t)x, lane, kWave), hi = __shfl((int)(uint32_t)(x >> 32), lane, kWave);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t from_xor(uint64_t x, int mask) {
    const uint32_t lo = __shfl_xor((int)(uint32_t)x, mask, kWave), hi = __shfl_xor((int)(uint32_t)(x >> 32), mask, kWave);
    return (uint64_t)hi << 32 | lo;
}

// 64 KR numbers of a wavefront, number r * 64 + lane in register r.  One step of a bitonic network: places i and i ^ stride are
// put in order, falling where (i & block) == 0 and not `rising`, rising elsewhere.
template <int KR>
__device__ __forceinline__ void exchange(uint64_t (&x)[KR], int stride, int block, bool rising) {
    const int lane = lane_id();
    if (stride >= kWave) {
        const int rs = stride / kWave;
#pragma unroll
        for (int r = 0; r < KR; ++r) {
            if (r & rs) continue;
            const bool down = (((r * kWave) & block) == 0) != rising;
            const uint64_t a = x[r], b = x[(r | rs) & (KR - 1)];
            const bool swap = down ? a < b : a > b;
            x[r] = swap ? b : a;
            x[(r | rs) & (KR - 1)] = swap ? a : b;
        }
    } else {
#pragma unroll
        for (int r = 0; r < KR; ++r) {
            const int i = r * kWave + lane;
            const uint64_t other = from_xor(x[r], stride);
            const bool down = ((i & block) == 0) != rising, low = (lane & stride) == 0;
            x[r] = (down == low) == (x[r] < other) ? other : x[r];
        }
    }
}

// The wavefront's list `best` (falling) and `fresh` (in any order): the 64 KR largest of both, falling.
template <int KR>
__device__ __forceinline__ void absorb(uint64_t (&best)[KR], uint64_t (&fresh)[KR]) {
    constexpr int N = kWave * KR;
#pragma unroll
    for (int block = 2; block <= N; block *= 2)
#pragma unroll
        for (int stride = block / 2; stride > 0; stride /= 2) exchange<KR>(fresh, stride, block == N ? 0 : block, true);
#pragma unroll
    for (int r = 0; r < KR; ++r) best[r] = best[r] < fresh[r] ? fresh[r] : best[r];
#pragma unroll
    for (int stride = N / 2; stride > 0; stride /= 2) exchange<KR>(best, stride, 0, false);
}

// A wavefront's walk: its list and the buffer of what is above the list's k-th number.
template <int KR, int BLOCK>
struct Walk {
    uint64_t best[KR];
    uint64_t *buffer;   // LDS, 64 KR + BLOCK numbers
    int count = 0, k;
    uint32_t least = 0;   // order of the k-th number; what is not above it comes later in the row and has no place
    __device__ __forceinline__ Walk(uint64_t *b, int kk) : buffer(b), k(kk) {
#pragma unroll
        for (int r = 0; r < KR; ++r) best[r] = 0;
    }
    __device__ __forceinline__ void offer(uint32_t order, uint64_t number, bool live) {
        const bool take = live && order > least;
        const uint64_t mask = __ballot(take);
        if (mask == 0) return;
        if (take) buffer[count + __popcll(mask & ((1ull << lane_id()) - 1))] = number;
        count += __popcll(mask);
    }
    // joins whole batches of the buffer, or all of it
    __device__ __forceinline__ void settle(bool all) {
        if (count < kWave * KR && !(all && count > 0)) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        while (count >= kWave * KR || (all && count > 0)) {
            const int n = std::min(count, kWave * KR), from = count - n;
            uint64_t fresh[KR];
#pragma unroll
            for (int r = 0; r < KR; ++r) {
                const int i = r * kWave + lane_id();
                fresh[r] = i < n ? buffer[from + i] : 0;
            }
            absorb<KR>(best, fresh);
            count = from;
        }
        uint64_t kth = 0;
#pragma unroll
        for (int r = 0; r < KR; ++r)
            if (r == (k - 1) / kWave) kth = from_lane(best[r], (k - 1) % kWave);
        least = (uint32_t)(kth >> 32);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
};

}  // namespace

// A wavefront takes columns [strip * width, ...) of a row; four of them a workgroup.  One strip: the answer; else the
// strips' lists.
struct TopArgs {
    const void *logits;
    int64_t ld, m, n_classes, width;
    int32_t strips, k;
    float *values;
    int32_t *ids;
    uint64_t *lists;   // [row][strip][k]
};

namespace {
template <int KR>
__device__ __forceinline__ void write_top(const TopArgs &a, int64_t row, const uint64_t (&best)[KR]) {
#pragma unroll
    for (int r = 0; r < KR; ++r) {
        const int i = r * kWave + lane_id();
        if (i < a.k) {
            a.values[row * a.k + i] = best[r] ? logit_of((uint32_t)(best[r] >> 32)) : -INFINITY;
            a.ids[row * a.k + i] = best[r] ? (int32_t)~(uint32_t)best[r] : -1;
        }
    }
}
}  // namespace

template <bool BF, int KR>
__global__ void __launch_bounds__(256) k_top_strip(const TopArgs a) {
    constexpr int PER = BF ? 8 : 4, BLOCK = kWave * PER;
    __shared__ uint64_t buffers[4][kWave * KR + BLOCK];
    const int wid = threadIdx.x / kWave, lane = lane_id();
    for (int64_t task = (int64_t)blockIdx.x * 4 + wid; task < a.m * a.strips; task += (int64_t)gridDim.x * 4) {
    const int64_t row = task / a.strips, strip = task % a.strips;
    const int64_t begin = strip * a.width, end = std::min(a.n_classes, begin + a.width);
    const char *src = (const char *)a.logits + row * a.ld * (BF ? 2 : 4);
    Walk<KR, BLOCK> walk(buffers[wid], a.k);
    for (int64_t c = begin; c < end; c += BLOCK) {
        const int64_t at = c + lane * PER;
        u32x4x v = {0, 0, 0, 0};
        if (at < end) v = *(const u32x4x *)(src + at * (BF ? 2 : 4));
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            float x;
            if constexpr (BF) x = __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
            else x = __uint_as_float(v[e]);
            const uint32_t order = order_of(x);
            walk.offer(order, (uint64_t)order << 32 | (uint32_t)~(uint32_t)(at + e), at + e < end);
        }
        walk.settle(c + BLOCK >= end);
    }
    if (a.strips == 1) {
        write_top<KR>(a, row, walk.best);
    } else {
#pragma unroll
        for (int r = 0; r < KR; ++r) {
            const int i = r * kWave + lane;
            if (i < a.k) a.lists[task * a.k + i] = walk.best[r];
        }
    }
    }
}

// The strips' lists of a row, a wavefront each.
template <int KR>
__global__ void __launch_bounds__(256) k_top_join(const TopArgs a) {
    __shared__ uint64_t buffers[4][kWave * KR + kWave];
    const int wid = threadIdx.x / kWave, lane = lane_id();
    const int64_t n = (int64_t)a.strips * a.k;
    for (int64_t row = (int64_t)blockIdx.x * 4 + wid; row < a.m; row += (int64_t)gridDim.x * 4) {
    Walk<KR, kWave> walk(buffers[wid], a.k);
    for (int64_t c = 0; c < n; c += kWave) {
        const uint64_t x = c + lane < n ? a.lists[row * n + c + lane] : 0;
        walk.offer((uint32_t)(x >> 32), x, x != 0);   // (equal logits come in the order of their classes here too)
        walk.settle(c + kWave >= n);
    }
    write_top<KR>(a, row, walk.best);
    }
}

namespace {
// Strips of a row: enough wavefronts to fill the device, 2,048 logits each at least.
void cut(int64_t m, int64_t n_classes, int64_t &width, int32_t &strips) {
    const int64_t want = std::max<int64_t>(1, 4096 / std::max<int64_t>(m, 1));
    int64_t n = std::max<int64_t>(1, std::min<int64_t>(want, n_classes / 2048));
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
            hipLaunchKernelGGL((k_top_join<KR>), dim3(grid_for(m, 4, 1 << 20)), dim3(256), 0, s, a);                     \
        }                                                                                                                \
    } while (0)
    if (k <= 64) GNNAV_L(1);
    else if (k <= 128) GNNAV_L(2);
    else GNNAV_L(4);
#undef GNNAV_L
    GNNAV_HIP(hipGetLastError());
}

}  // namespace gnnav
