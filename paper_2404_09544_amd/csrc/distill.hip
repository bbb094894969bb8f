// Distillation: the student's logits against the k logits that a teacher kept of each row, with the labels' cross entropy
// beside it, and the gradient.  For row i, M its largest logit, over the entries j that are there
//
//   q_j = softmax_j(t_j / T),  s(T) = sum_v exp((z_v - M) / T),  p_v(T) = exp((z_v - M) / T) / s(T)
//   kd_i = T^2 sum_j q_j (log q_j - (z_j - M) / T + log s(T)),   ce_i = log s(1) - (z_y - M)
//   dz_v = alpha T / A (p_v(T) - sum_{j: id_j = v} q_j) + (1 - alpha) / B (p_v(1) - [v = y_i])
//
// A the rows with entries, B those with a label that counts.  Bound by memory: a row is read once, into the registers of a
// team of 16 lanes to four wavefronts, and its gradient written from them: 4,093 x 10,000 bf16 64 us, of which reading and writing
// at 4.72 TB/s is 35; the exponentials (one a logit and pass at least) and the four barriers of a row take the rest.  Rows of
// more classes are cut into strips, whose sums take a launch of their own; the gradient's starts with the last rows, which
// the memory-side cache still holds: 1,024 x 169,000 fp32 385 us (293), 392 in the same order.  Groups of rows by turns, small enough
// for that cache, are slower (a launch's end each), and so are teams of 512 and 1,024 threads, which spill.
#include <algorithm>
#include <cmath>

#include "common.hpp"
#include "lanes.hpp"

namespace gnnav {

namespace {

typedef uint32_t u32x4x __attribute__((ext_vector_type(4)));
constexpr double kLog2e = 1.44269504088896340736;
constexpr int kParts = 1024;   // counts of rows, at most
constexpr int kSplitVectors = 4;   // 16-byte vectors of a thread in a strip
constexpr int kBlocks = 2048;      // workgroups that take whole rows, at most

struct Args {
    DistillArgs x;
    int2 *counts;        // [parts]: rows with entries, with labels
    int32_t parts;       // 0: every workgroup counts for itself
    double2 *losses;     // [n_losses]: sums of both parts of the loss
    int32_t n_losses;
    int64_t first;       // strips > 0: first row of the launch
    float scale, inv_t;  // log2(e) times what the logits are divided by (1 / T, or 1 where there is no teacher's part); 1 / T
    int32_t strips, width;
    float4 *sums;        // strips > 0: [m][strips] largest logit, sums at T and at 1
    float *own;          // ... and [m][k + 1] logits of the entries' classes and of the label
};

__device__ __forceinline__ bool entry_there(int32_t id, float t) { return id >= 0 && t != -INFINITY; }

template <bool BF>
__device__ __forceinline__ float logit(const char *row, int64_t c) {
    if constexpr (BF) return bf16_to_f32(((const uint16_t *)row)[c]);
    else return ((const float *)row)[c];
}

// 16 bytes of a row from class c on, -inf past the last class.
template <bool BF>
__device__ __forceinline__ u32x4x load(const char *row, int64_t c, int64_t end) {
    constexpr int PER = BF ? 8 : 4;
    constexpr uint32_t NONE = BF ? 0xff80ff80u : 0xff800000u;
    u32x4x v = {NONE, NONE, NONE, NONE};
    if (c < end) v = *(const u32x4x *)(row + c * (BF ? 2 : 4));
    if (c < end && c + PER > end)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (BF) {
                if (c + 2 * e + 1 >= end) v[e] = (v[e] & 0xffffu) | (NONE & 0xffff0000u);
                if (c + 2 * e >= end) v[e] = NONE;
            } else if (c + e >= end) {
                v[e] = NONE;
            }
        }
    return v;
}

// What the T threads of a row's team have in common.  Round r of its reductions has a place of its own in LDS, so that one
// barrier does for each.
template <int T>
struct Team {
    static constexpr int W = T > 64 ? T / 64 : 1;
    float (*scratch)[W];   // [places][W]
    __device__ __forceinline__ void sync() const {
        if constexpr (T > 64) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    template <bool MAX>
    __device__ __forceinline__ float within(float x, int place) const {
        x = lanes_reduce<(T < 64 ? T : 64), MAX>(x);
        if constexpr (T > 64)
            if (lane_id() == 0) scratch[place][threadIdx.x / 64] = x;
        return x;
    }
    template <bool MAX>
    __device__ __forceinline__ float across(float x, int place) const {
        if constexpr (T > 64) {
            x = scratch[place][0];
#pragma unroll
            for (int w = 1; w < W; ++w) x = MAX ? fmaxf(x, scratch[place][w]) : x + scratch[place][w];
        }
        return x;
    }
};

// Rows with entries and rows with labels that count, of those that this thread looks at: most rows show by their first entry.
__device__ __forceinline__ int2 count_rows(const DistillArgs &x, int64_t first, int64_t step) {
    int32_t n = 0, l = 0;
#pragma unroll 4
    for (int64_t i = first; i < x.m; i += step) {
        bool any = x.k > 0 && entry_there(x.ids[i * x.k], x.teacher[i * x.k]);
        if (!any)
            for (int32_t j = 1; j < x.k && !any; ++j) any = entry_there(x.ids[i * x.k + j], x.teacher[i * x.k + j]);
        n += any;
        if (x.labels) l += x.labels[i] != x.ignore;
    }
    return make_int2(n, l);
}
// ... and their sum over a workgroup of NT threads, in every thread; s: LDS.
template <int NT>
__device__ __forceinline__ int2 sum_counts(int2 c, int2 *s) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        c.x += __shfl_xor(c.x, o, 64);
        c.y += __shfl_xor(c.y, o, 64);
    }
    if (lane_id() == 0) s[threadIdx.x / 64] = c;
    __syncthreads();
    c = s[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) {
        c.x += s[w].x;
        c.y += s[w].y;
    }
    return c;
}

// A running largest logit, the sums of exponentials less it.
struct Sums {
    float top = -INFINITY, st = 0.f, s1 = 0.f;
};
__device__ __forceinline__ float exp_of(float x, float scale) { return __builtin_amdgcn_exp2f(x * scale); }

// Whether the exponentials at 1 are needed beside those at T, and how they are had: from those at T = 2 or 4 by one or two
// products.  The argument's rounding counts as much either way; exp2's own (2^-23) counts T times, and the products round
// log2(T) times: at T = 4 within 2^-20 of the value.  4,093 x 10,000 bf16 at T = 4: 64 us, 67 with two.
enum { kOne, kBoth, kSquare, kFourth };
template <int WAY>
__device__ __forceinline__ float exp_at_one(float x, float at_t) {
    if constexpr (WAY == kSquare) return at_t * at_t;
    else if constexpr (WAY == kFourth) return (at_t * at_t) * (at_t * at_t);
    else return exp_of(x, (float)kLog2e);
}

}  // namespace

// Rows with entries and rows with labels that count, by parts: 16 lanes a row.
__global__ void __launch_bounds__(256) k_distill_count(const Args a) {
    __shared__ int2 s[4];
    const DistillArgs &x = a.x;
    const int lane = threadIdx.x % 16, shift = lane_id() & 48;
    int32_t n = 0, l = 0;
    for (int64_t first = (int64_t)blockIdx.x * 16; first < x.m; first += (int64_t)gridDim.x * 16) {
        const int64_t i = first + threadIdx.x / 16;
        bool any = false;
        for (int32_t j = lane; i < x.m && j < x.k; j += 16) any |= entry_there(x.ids[i * x.k + j], x.teacher[i * x.k + j]);
        const bool row = (__ballot(any) >> shift & 0xffff) != 0;
        if (lane == 0 && i < x.m) {
            n += row;
            if (x.labels) l += x.labels[i] != x.ignore;
        }
    }
    const int2 c = sum_counts<256>(make_int2(n, l), s);
    if (threadIdx.x == 0) a.counts[blockIdx.x] = c;
}

// The losses' means, in 64 bits and a fixed order.
__global__ void __launch_bounds__(256) k_distill_mean(const Args a) {
    const DistillArgs &x = a.x;
    __shared__ double sd[4][2];
    __shared__ int2 si[4];
    double kd = 0.0, ce = 0.0;
#pragma unroll 8
    for (int32_t i = threadIdx.x; i < a.n_losses; i += 256) {
        const double2 p = a.losses[i];
        kd += p.x;
        ce += p.y;
    }
    int2 c = make_int2(0, 0);
    for (int32_t i = threadIdx.x; i < std::max(a.parts, 1); i += 256) {
        const int2 p = a.counts[i];
        c.x += p.x;
        c.y += p.y;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        kd += __shfl_xor(kd, o, 64);
        ce += __shfl_xor(ce, o, 64);
    }
    if (lane_id() == 0) {
        sd[threadIdx.x / 64][0] = kd;
        sd[threadIdx.x / 64][1] = ce;
    }
    c = sum_counts<256>(c, si);
    if (threadIdx.x == 0) {
        for (int w = 1; w < 4; ++w) {
            kd += sd[w][0];
            ce += sd[w][1];
        }
        kd = c.x ? kd / (double)c.x : 0.0;
        ce = c.y ? ce / (double)c.y : 0.0;
        const double first = x.alpha > 0.f ? (double)x.alpha * kd : 0.0, second = x.alpha < 1.f ? (1.0 - (double)x.alpha) * ce : 0.0;
        x.loss[0] = (float)(first + second);
        x.loss[1] = (float)kd;
        x.loss[2] = (float)ce;
    }
}

// The sums of one strip of a row, and the logits that are needed by themselves (the gradient may take their place).
template <bool BF, int BOTH>
__global__ void __launch_bounds__(256) k_distill_sums(const Args a) {
    constexpr int PER = BF ? 8 : 4;
    __shared__ float scratch[3][4];
    const DistillArgs &x = a.x;
    const Team<256> team = {scratch};
    const int tid = threadIdx.x;
    const int64_t row = a.first + blockIdx.y, begin = (int64_t)blockIdx.x * a.width, end = std::min(x.n_classes, begin + a.width);
    const char *src = (const char *)x.logits + row * x.ld * (BF ? 2 : 4);
    u32x4x v[kSplitVectors];
#pragma unroll
    for (int i = 0; i < kSplitVectors; ++i) v[i] = load<BF>(src, begin + (i * 256 + tid) * PER, end);
    Sums s;
#pragma unroll
    for (int i = 0; i < kSplitVectors; ++i)
#pragma unroll
        for (int e = 0; e < PER; ++e) s.top = fmaxf(s.top, element<BF>(v[i], e));
    const float ref = s.top == -INFINITY ? 0.f : s.top;
#pragma unroll
    for (int i = 0; i < kSplitVectors; ++i)
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const float z = element<BF>(v[i], e) - ref, p = exp_of(z, a.scale);
            s.st += p;
            if constexpr (BOTH) s.s1 += exp_at_one<BOTH>(z, p);
        }
    const float top = team.across<true>((team.within<true>(s.top, 0), team.sync(), 0.f), 0);
    const float ft = s.top == -INFINITY ? 1.f : exp_of(s.top - top, a.scale), f1 = s.top == -INFINITY ? 1.f : exp_of(s.top - top, (float)kLog2e);
    team.within<false>(s.st * ft, 1);
    if constexpr (BOTH) team.within<false>(s.s1 * f1, 2);
    team.sync();
    if (tid == 0) {
        const float st = team.across<false>(0.f, 1);
        a.sums[row * a.strips + blockIdx.x] = make_float4(top, st, BOTH ? team.across<false>(0.f, 2) : st, 0.f);
    }
    for (int32_t j = tid; j <= x.k; j += 256) {
        const int32_t id = j < x.k ? (x.alpha > 0.f ? x.ids[row * x.k + j] : -1) : x.labels ? x.labels[row] : -1;
        if (id >= begin && id < end) a.own[row * (x.k + 1) + j] = logit<BF>(src, id);
    }
}

// One row, by the team of T threads that calls it.  VEC: 16-byte loads (otherwise a class a lane); NV of them a thread stay
// in registers.  SPLIT: the sums are there, and strip `strip` of the gradient is written.
template <bool BF, int T, int NV, bool VEC, int BOTH, bool SPLIT>
__device__ __forceinline__ void distill_row(const Args &a, int64_t row, int32_t strip, bool live, int2 counted_rows, const Team<T> &team, int32_t *ids,
                                            float *share, double2 &loss) {
    constexpr int PER = !VEC ? 1 : BF ? 8 : 4, ELT = BF ? 2 : 4;
    constexpr bool EXPS = VEC && !BF && !BOTH && !SPLIT;   // the kept logits give way to their exponentials
    const DistillArgs &x = a.x;
    const int tid = threadIdx.x % T;
    const int64_t C = x.n_classes, begin = SPLIT ? (int64_t)strip * a.width : 0, end = SPLIT ? std::min(C, begin + a.width) : C;
    const char *src = (const char *)x.logits + row * x.ld * ELT;
    char *out = x.dlogits ? (char *)x.dlogits + row * x.ld_d * ELT : nullptr;

    // the row, and what there is to do
    u32x4x keep[VEC ? NV : 1];
    float one[VEC ? 1 : NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int64_t c = begin + (int64_t)(v * T + tid) * PER;
        if constexpr (VEC) keep[v] = live ? load<BF>(src, c, end) : u32x4x{0, 0, 0, 0};
        else one[v] = live && c < C ? logit<BF>(src, c) : -INFINITY;
    }
    int32_t id = -1;
    float t = -INFINITY;
    if (live && x.alpha > 0.f && tid < x.k) {
        id = x.ids[row * x.k + tid];
        t = x.teacher[row * x.k + tid];
        if (!entry_there(id, t)) id = -1;
    }
    if (tid < (x.k + 3) / 4 * 4) ids[tid] = id;
    const int32_t y = live && x.labels ? x.labels[row] : x.ignore;
    const bool counts = live && x.labels && y != x.ignore, off = counts && (y < 0 || y >= C);

    // largest logit, largest of the teacher's, whether there are entries and wrong ones
    Sums s;
    float kept = 0.f;   // what the kept exponentials are less
    if constexpr (SPLIT) {
        for (int i = tid; i < a.strips; i += T) s.top = fmaxf(s.top, a.sums[row * a.strips + i].x);
    } else {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if ((int64_t)v * T * PER >= C) break;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                if constexpr (VEC) s.top = fmaxf(s.top, element<BF>(keep[v], e));
                else s.top = fmaxf(s.top, one[v]);
            }
        }
        const float ref = s.top == -INFINITY ? 0.f : s.top;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if ((int64_t)v * T * PER >= C) break;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                float z;
                if constexpr (VEC) z = element<BF>(keep[v], e);
                else z = one[v];
                const float p = exp_of(z - ref, a.scale);
                s.st += p;
                if constexpr (BOTH) s.s1 += exp_at_one<BOTH>(z - ref, p);
                if constexpr (EXPS) keep[v][e] = __float_as_uint(p);
            }
        }
        kept = ref;
    }
    float top = team.template within<true>(s.top, 0), most = team.template within<true>(id >= 0 ? t : -INFINITY, 1);
    float has_f = team.template within<true>(id >= 0 ? 1.f : 0.f, 2), wrong_f = team.template within<true>(id >= C ? 1.f : 0.f, 3);
    float listed_f = team.template within<true>(id >= 0 && id == y ? 1.f : 0.f, 8);
    team.sync();
    top = team.template across<true>(top, 0);
    most = team.template across<true>(most, 1);
    const bool has = team.template across<true>(has_f, 2) > 0.f, wrong = team.template across<true>(wrong_f, 3) > 0.f;
    const bool listed = team.template across<true>(listed_f, 8) > 0.f;   // whether the label is an entry's class
    const bool do_kd = has && !wrong, do_ce = counts && !off, some = do_kd || do_ce;

    // sums of exponentials (a thread without logits has no part)
    float st, s1;
    if constexpr (SPLIT) {
        st = s1 = 0.f;
        for (int i = tid; i < a.strips; i += T) {
            const float4 p = a.sums[row * a.strips + i];
            st += p.x == -INFINITY ? p.y : p.y * exp_of(p.x - top, a.scale);
            if constexpr (BOTH) s1 += p.x == -INFINITY ? p.z : p.z * exp_of(p.x - top, (float)kLog2e);
        }
    } else {
        st = s.top == -INFINITY ? s.st : s.st * exp_of(s.top - top, a.scale);
        s1 = 0.f;
        if constexpr (BOTH) s1 = s.top == -INFINITY ? s.s1 : s.s1 * exp_of(s.top - top, (float)kLog2e);
    }
    const float u = id >= 0 ? (t - most) * a.inv_t : 0.f, w = id >= 0 ? expf(u) : 0.f;
    st = team.template within<false>(st, 4);
    if constexpr (BOTH) s1 = team.template within<false>(s1, 5);
    float sum = team.template within<false>(w, 6);
    float zj = 0.f, zy = 0.f;   // every logit that is needed by itself is read before the gradient may take its place
    if (do_kd && id >= 0) zj = SPLIT ? a.own[row * (x.k + 1) + tid] : logit<BF>(src, id);
    if (do_ce) zy = SPLIT ? a.own[row * (x.k + 1) + x.k] : logit<BF>(src, y);
    team.sync();
    st = team.template across<false>(st, 4);
    s1 = BOTH ? team.template across<false>(s1, 5) : st;
    sum = team.template across<false>(sum, 6);
    const float nan = __builtin_nanf("");
    const bool none = top == -INFINITY;   // a row of -inf alone has no distribution
    const float q = do_kd ? w / sum : 0.f;
    // an entry whose q is zero has no part, whatever the student's logit
    const float term = q == 0.f ? 0.f : q * ((u - logf(sum)) - ((zj - top) * a.inv_t - logf(st)));
    float kd = team.template within<false>(term, 7);
    if (tid < x.k) share[tid] = q;
    asm volatile("" ::"v"(zj), "v"(zy));   // (both have arrived when the row is written)
    team.sync();
    kd = team.template across<false>(kd, 7) * (x.temperature * x.temperature);
    if (!live) return;
    if (strip == 0 && tid == 0) {
        kd = has && wrong ? nan : !do_kd ? 0.f : none ? nan : kd;
        const float ce = off ? nan : !do_ce ? 0.f : none ? nan : logf(s1) - (zy - top);
        loss.x += (double)kd;
        loss.y += (double)ce;
        if (x.row_loss) x.row_loss[row] = (x.alpha > 0.f ? x.alpha * kd : 0.f) + (x.alpha < 1.f ? (1.f - x.alpha) * ce : 0.f);
    }
    if (!out) return;

    // the gradient: coefficients of the exponentials at T and at 1
    const float wk = do_kd ? (float)((double)x.alpha * x.temperature / counted_rows.x) : 0.f;
    const float wc = do_ce ? (float)((1.0 - (double)x.alpha) / counted_rows.y) : 0.f;
    const float ct = do_kd ? (none ? nan : wk / st) : 0.f, c1 = do_ce ? (none ? nan : wc / s1) : 0.f;
    const float ref = some ? top : 0.f;
    auto grad = [&](float z) {
        const float p = exp_of(z - ref, a.scale);
        if constexpr (BOTH) return ct * p + c1 * exp_at_one<BOTH>(z - ref, p);
        else return (ct + c1) * p;
    };
    auto write = [&](const u32x4x &v, int64_t c, auto exps_, float factor) {   // of logits, or of their exponentials
        float g[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if constexpr (decltype(exps_)::value) g[e] = factor * element<BF>(v, e);
            else g[e] = grad(element<BF>(v, e));
        }
        if (c + PER > C)
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (c + e >= C) g[e] = 0.f;
        u32x4x o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (BF) o[e] = bf16_pair(g[2 * e % PER], g[(2 * e + 1) % PER]);
            else o[e] = __float_as_uint(g[e % PER]);
        }
        *(u32x4x *)(out + c * ELT) = o;
    };
    auto put = [&](int64_t c, float g) {
        if constexpr (BF) ((uint16_t *)out)[c] = bf16_rne(g);
        else ((float *)out)[c] = g;
    };
    const u32x4x zeros = {0, 0, 0, 0};
    // (a row that does not count may hold what makes the exponential infinite; a thread of -inf alone kept zeros, with no scale of
    // their own)
    const float down = s.top == -INFINITY ? 0.f : exp_of(kept - ref, a.scale);
    const float factor = EXPS && some ? (ct + c1) * down : 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int64_t c = begin + (int64_t)(v * T + tid) * PER;
        if (begin + (int64_t)v * T * PER >= end) break;
        if constexpr (VEC) {
            if (c < end) write(some ? keep[v] : zeros, c, std::integral_constant<bool, EXPS>(), factor);
        } else if (c < (C * ELT + 15) / 16 * 16 / ELT) {
            put(c, c < C ? grad(some ? one[v] : 0.f) : 0.f);
        }
    }
    // the classes that have a share of the target, once each, over what was written
    team.sync();
    if (do_kd && id >= begin && id < end) {
        bool twice = false;
        for (int32_t j = 0; j < x.k; j += 4) {
            const int4 other = *(const int4 *)(ids + j);
            twice = twice || (other.x == id && j != tid) || (other.y == id && j + 1 != tid) || (other.z == id && j + 2 != tid) ||
                    (other.w == id && j + 3 != tid);
        }
        float all = q;
        bool first = true;
        if (twice) {
            all = 0.f;
            for (int32_t j = 0; j < x.k; ++j)
                if (ids[j] == id) {
                    first = first && j >= tid;
                    all += share[j];
                }
        }
        if (first) put(id, grad(zj) - wk * all - (do_ce && id == y ? wc : 0.f));
    }
    if (do_ce && tid == 0 && y >= begin && y < end && !(do_kd && listed)) put(y, grad(zy) - wc);
}

template <bool BF, int T, int NV, bool VEC, int BOTH, bool SPLIT>
__global__ void __launch_bounds__(256) k_distill_row(const Args a) {
    constexpr int NT = 256, ROWS = NT / T, ENTRIES = T;
    __shared__ float scratch[9][Team<T>::W];
    __shared__ __align__(16) int32_t ids[ROWS][ENTRIES];
    __shared__ float share[ROWS][ENTRIES];
    __shared__ int2 counts[NT / 64];
    int2 c = make_int2(0, 0);
    if (a.parts == 0) c = count_rows(a.x, threadIdx.x, NT);
    else
        for (int32_t i = threadIdx.x; i < a.parts; i += NT) {
            const int2 p = a.counts[i];
            c.x += p.x;
            c.y += p.y;
        }
    c = sum_counts<NT>(c, counts);
    if (a.parts == 0 && threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) a.counts[0] = c;   // for the means
    const Team<T> team = {scratch};
    const int at = threadIdx.x / T;
    double2 loss = make_double2(0.0, 0.0);
    if constexpr (SPLIT) {
        // (the last rows first: the memory-side cache still holds them from the sums' launch)
        const int64_t row = a.first + (gridDim.y - 1 - blockIdx.y);
        distill_row<BF, T, NV, VEC, BOTH, SPLIT>(a, row, blockIdx.x, true, c, team, ids[0], share[0], loss);
        if (threadIdx.x == 0 && blockIdx.x == 0) a.losses[row] = loss;
    } else {
        // (whole teams of a wavefront past the last row go along with the others)
        for (int64_t row = (int64_t)blockIdx.x * ROWS; row < a.x.m; row += (int64_t)gridDim.x * ROWS) {
            distill_row<BF, T, NV, VEC, BOTH, SPLIT>(a, std::min(row + at, a.x.m - 1), 0, row + at < a.x.m, c, team, ids[at], share[at], loss);
            team.sync();   // (the next row takes the same LDS)
        }
        __shared__ double2 losses[ROWS];
        if (threadIdx.x % T == 0) losses[at] = loss;
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int r = 1; r < ROWS; ++r) {
                loss.x += losses[r].x;
                loss.y += losses[r].y;
            }
            a.losses[blockIdx.x] = loss;
        }
    }
}

namespace {
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Strips of a row: 0 where a row is taken whole, as long as four wavefronts hold it.  1,024 x 8,192 fp32: 31 us, in strips 36;
// 4,093 x 16,000 bf16: 84 and 90; 64 x 16,000 as much.
int32_t strips_for(int64_t n_classes, bool bf16) {
    const int64_t per = bf16 ? 8 : 4, width = 256 * kSplitVectors * per;
    return n_classes > 2048 * per ? (int32_t)((n_classes + width - 1) / width) : 0;
}

struct Plan {
    int32_t strips, n_losses;
    size_t losses, sums, own, total;
    Plan(int64_t m, int64_t n_classes, int64_t k, bool bf16) {
        strips = strips_for(n_classes, bf16);
        n_losses = strips > 0 ? (int32_t)m : (int32_t)std::min<int64_t>(m, kBlocks);
        size_t at = kParts * sizeof(int2);
        auto take = [&](int64_t bytes) {
            const size_t here = at;
            at += (size_t)up(bytes, 256);
            return here;
        };
        losses = take((int64_t)n_losses * 16);
        sums = take(m * strips * 16);
        own = take(strips > 0 ? m * (k + 1) * 4 : 0);
        total = at;
    }
};

template <bool BF, int BOTH>
void rows(Args &a, hipStream_t s) {
    const int64_t m = a.x.m, C = a.x.n_classes, k = a.x.alpha > 0.f ? a.x.k : 0;
    constexpr int PER = BF ? 8 : 4;
    if (a.strips > 0) {
        for (int64_t first = 0; first < m; first += 65535) {
            Args g = a;
            g.first = first;
            const dim3 grid((unsigned)a.strips, (unsigned)std::min<int64_t>(65535, m - first));
            {
                KernelTimer t("distill_sums", s);
                hipLaunchKernelGGL((k_distill_sums<BF, BOTH>), grid, dim3(256), 0, s, g);
            }
            KernelTimer t("distill_row", s);
            hipLaunchKernelGGL((k_distill_row<BF, 256, kSplitVectors, true, BOTH, true>), grid, dim3(256), 0, s, g);
        }
        return;
    }
    KernelTimer t("distill_row", s);
#define GNNAV_L(T, NV, VEC)                                                                                                \
    do {                                                                                                                   \
        a.n_losses = (int32_t)grid_for(m, 256 / T, kBlocks);                                                               \
        hipLaunchKernelGGL((k_distill_row<BF, T, NV, VEC, BOTH, false>), dim3((unsigned)a.n_losses), dim3(256), 0, s, a);  \
    } while (0)
    // The smallest team that holds the row and its entries.  99,603 x 41 fp32, k = 8: 16 lanes 39 us, 32 60, 64 104, 256 350; 20,000 x
    // 100, k = 16: 32 lanes 23, 64 30, 256 80; 20,000 x 1,000: 64 lanes 55, 256 110; 4,093 x 4,000 bf16: 33 and 40; 500 x 2,000: as much.
    if (C <= 64 && k <= 16) GNNAV_L(16, 4, false);
    else if (C <= 128 && k <= 32) GNNAV_L(32, 4, false);
    else if (C <= 64 * PER && k <= 64) GNNAV_L(64, 1, true);
    else if (C <= 128 * PER && k <= 64) GNNAV_L(64, 2, true);
    else if (C <= 256 * PER && k <= 64) GNNAV_L(64, 4, true);
    else if (C <= 512 * PER && k <= 64) GNNAV_L(64, 8, true);
    else if (C <= 512 * PER) GNNAV_L(256, 2, true);
    else if (C <= 1024 * PER) GNNAV_L(256, 4, true);
    else GNNAV_L(256, 8, true);
#undef GNNAV_L
}
template <bool BF>
void by_way(Args &a, int way, hipStream_t s) {
    switch (way) {
    case kOne: return rows<BF, kOne>(a, s);
    case kSquare: return rows<BF, kSquare>(a, s);
    case kFourth: return rows<BF, kFourth>(a, s);
    default: return rows<BF, kBoth>(a, s);
    }
}
}  // namespace

size_t distill_workspace(int64_t m, int64_t n_classes, int64_t k, bool bf16) { return Plan(m, n_classes, k, bf16).total; }

void launch_distill(const DistillArgs &x, hipStream_t s) {
    Args a = {};
    a.x = x;
    if (x.alpha == 0.f) a.x.k = 0;
    const Plan p(x.m, x.n_classes, x.k, x.bf16);
    char *ws = (char *)x.workspace;
    a.counts = (int2 *)ws;
    a.losses = (double2 *)(ws + p.losses);
    a.n_losses = p.n_losses;
    a.sums = (float4 *)(ws + p.sums);
    a.own = (float *)(ws + p.own);
    a.inv_t = 1.f / x.temperature;
    a.scale = (float)(x.alpha > 0.f ? kLog2e / x.temperature : kLog2e);
    a.strips = p.strips;
    a.width = 256 * kSplitVectors * (x.bf16 ? 8 : 4);
    a.parts = x.m <= 1024 && a.x.k <= 16 ? 0 : (int32_t)grid_for(x.m, 16, kParts);
    if (a.parts > 0) {
        KernelTimer t("distill_count", s);
        hipLaunchKernelGGL(k_distill_count, dim3((unsigned)a.parts), dim3(256), 0, s, a);
    }
    if (x.m > 0) {
        const bool both = x.alpha > 0.f && x.labels && x.temperature != 1.f;
        const int way = !both ? kOne : x.temperature == 2.f ? kSquare : x.temperature == 4.f ? kFourth : kBoth;
        if (x.bf16) by_way<true>(a, way, s);
        else by_way<false>(a, way, s);
    }
    {
        KernelTimer t("distill_mean", s);
        hipLaunchKernelGGL(k_distill_mean, dim3(1), dim3(256), 0, s, a);
    }
    GNNAV_HIP(hipGetLastError());
}

}  // namespace gnnav
