// Distillation: the student's logits against the k logits that a teacher kept of each row, with the labels' cross entropy
// beside it, and the gradient.  For row i, M its largest logit, over the entries j that are there
//
//   q_j = softmax_j(t_j / T),  s(T) = sum_v exp((z_v - M) / T),  p_v(T) = exp((z_v - M) / T) / s(T)
//   kd_i = T^2 sum_j q_j (log q_j - (z_j - M) / T + log s(T)),   ce_i = log s(1) - (z_y - M)
//   dz_v = alpha T / A (p_v(T) - sum_{j: id_j = v} q_j) + (1 - alpha) / B (p_v(1) - [v = y_i])
//
// A the rows with entries, B those with a label that counts.  Bound by memory: the logits are read once where a row's fit the
// registers, and the gradient written once.
#include <algorithm>
#include <cmath>

#include "common.hpp"

namespace gnnav {

namespace {

typedef uint32_t u32x4x __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2x __attribute__((ext_vector_type(2)));
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kParts = 256;   // counts of rows, at most
constexpr int kMost = 256;    // entries of a row, at most

struct Args {
    DistillArgs x;
    int2 *counts;        // [parts]: rows with entries, with labels
    int32_t parts;
    float *kd, *ce;      // [m]
};

// exp(x c): fp32 logits by expf, bf16 ones, whose own rounding is coarser, by the hardware's exp2
template <bool BF>
__device__ __forceinline__ float exp_of(float x, float inv_t) {
    if constexpr (BF) return __builtin_amdgcn_exp2f(x * (inv_t * kLog2e));
    else return expf(x * inv_t);
}

__device__ __forceinline__ bool entry_there(int32_t id, float t) { return id >= 0 && t != -INFINITY; }

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// Max, or sum, over a workgroup of NT threads; scratch: NT / 64 values of LDS.
template <int NT, bool MAX>
__device__ __forceinline__ float reduce(float x, float *scratch) {
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const float y = __shfl_xor(x, o, kWave);
        x = MAX ? fmaxf(x, y) : x + y;
    }
    if (NT == kWave) return x;
    if (lane_id() == 0) scratch[threadIdx.x / kWave] = x;
    __syncthreads();
    x = scratch[0];
#pragma unroll
    for (int w = 1; w < NT / kWave; ++w) x = MAX ? fmaxf(x, scratch[w]) : x + scratch[w];
    __syncthreads();
    return x;
}

}  // namespace

// Rows with entries and rows with labels that count, by parts.
__global__ void __launch_bounds__(256) k_distill_count(const Args a) {
    const DistillArgs &x = a.x;
    int32_t n = 0, l = 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < x.m; i += (int64_t)gridDim.x * 256) {
        if (x.alpha > 0.f) {
            bool any = false;
            for (int32_t j = 0; j < x.k && !any; ++j) any = entry_there(x.ids[i * x.k + j], x.teacher[i * x.k + j]);
            n += any;
        }
        if (x.labels) l += x.labels[i] != x.ignore;
    }
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        n += __shfl_xor(n, o, kWave);
        l += __shfl_xor(l, o, kWave);
    }
    __shared__ int2 s[4];
    if (lane_id() == 0) s[threadIdx.x / kWave] = make_int2(n, l);
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 4; ++w) {
            n += s[w].x;
            l += s[w].y;
        }
        a.counts[blockIdx.x] = make_int2(n, l);
    }
}

// The losses' means, in 64 bits and a fixed order.
__global__ void __launch_bounds__(1024) k_distill_mean(const Args a) {
    const DistillArgs &x = a.x;
    double kd = 0.0, ce = 0.0;
    int64_t n = 0, l = 0;
    for (int64_t i = threadIdx.x; i < x.m; i += 1024) {
        kd += (double)a.kd[i];
        ce += (double)a.ce[i];
    }
    if ((int)threadIdx.x < a.parts) {
        n = a.counts[threadIdx.x].x;
        l = a.counts[threadIdx.x].y;
    }
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        kd += __shfl_xor(kd, o, kWave);
        ce += __shfl_xor(ce, o, kWave);
        n += __shfl_xor(n, o, kWave);
        l += __shfl_xor(l, o, kWave);
    }
    __shared__ double sd[16][2];
    __shared__ int64_t si[16][2];
    if (lane_id() == 0) {
        sd[threadIdx.x / kWave][0] = kd;
        sd[threadIdx.x / kWave][1] = ce;
        si[threadIdx.x / kWave][0] = n;
        si[threadIdx.x / kWave][1] = l;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) {
            kd += sd[w][0];
            ce += sd[w][1];
            n += si[w][0];
            l += si[w][1];
        }
        kd = n ? kd / (double)n : 0.0;
        ce = l ? ce / (double)l : 0.0;
        const double first = x.alpha > 0.f ? (double)x.alpha * kd : 0.0, second = x.alpha < 1.f ? (1.0 - (double)x.alpha) * ce : 0.0;
        x.loss[0] = (float)(first + second);
        x.loss[1] = (float)kd;
        x.loss[2] = (float)ce;
    }
}

namespace {

template <bool BF>
__device__ __forceinline__ float element(const u32x4x &v, int e) {
    if constexpr (BF) return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
    else return __uint_as_float(v[e]);
}

// A running largest logit and the sums of exponentials less it.
struct Sums {
    float top = -INFINITY, st = 0.f, s1 = 0.f;
};

template <bool BF>
__device__ __forceinline__ void add(Sums &s, const float *z, int n, float inv_t, bool both) {
    float mx = s.top;
#pragma unroll
    for (int e = 0; e < n; ++e) mx = fmaxf(mx, z[e]);
    if (mx > s.top) {
        s.st *= exp_of<BF>(s.top - mx, inv_t);
        if (both) s.s1 *= exp_of<BF>(s.top - mx, 1.f);
        s.top = mx;
    }
    const float ref = s.top == -INFINITY ? 0.f : s.top;
#pragma unroll
    for (int e = 0; e < n; ++e) {
        s.st += exp_of<BF>(z[e] - ref, inv_t);
        if (both) s.s1 += exp_of<BF>(z[e] - ref, 1.f);
    }
}

}  // namespace

// One row a workgroup of NT threads.  Its first NV vectors of 16 bytes a thread stay in registers; what is beyond them
// is read again for the gradient.
template <bool BF, int NT, int NV>
__device__ __forceinline__ void distill_row(const Args &a, int64_t row) {
    constexpr int PER = BF ? 8 : 4;
    const DistillArgs &x = a.x;
    __shared__ float scratch[NT / kWave];
    __shared__ int32_t ids[kMost];
    __shared__ float share[kMost];
    __shared__ int32_t flags[4];
    const int tid = threadIdx.x;
    const int32_t C = (int32_t)x.n_classes;
    const char *src = (const char *)x.logits + row * x.ld * (BF ? 2 : 4);

    // what there is to do (the row before may still be looked up in ids and share)
    __syncthreads();
    if (tid < 4) flags[tid] = 0;
    __syncthreads();
    int32_t id = -1;
    float t = -INFINITY;
    if (x.alpha > 0.f && tid < x.k) {
        id = x.ids[row * x.k + tid];
        t = x.teacher[row * x.k + tid];
        if (!entry_there(id, t)) id = -1;
        ids[tid] = id;
        if (id >= 0) flags[0] = 1;
        if (id >= C) flags[1] = 1;
    }
    if (tid < kWave) {
        int32_t n = 0, l = 0;
        for (int i = tid; i < a.parts; i += kWave) {
            n += a.counts[i].x;
            l += a.counts[i].y;
        }
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            n += __shfl_xor(n, o, kWave);
            l += __shfl_xor(l, o, kWave);
        }
        if (tid == 0) {
            flags[2] = n;
            flags[3] = l;
        }
    }
    __syncthreads();
    const bool has = flags[0], wrong = flags[1];
    const int32_t y = x.labels ? x.labels[row] : x.ignore;
    const bool counted = x.labels && y != x.ignore, off = counted && (y < 0 || y >= C);
    const bool do_kd = has && !wrong, do_ce = counted && !off;
    const float wk = do_kd ? (float)((double)x.alpha * x.temperature / flags[2]) : 0.f;
    const float wc = do_ce ? (float)((1.0 - (double)x.alpha) / flags[3]) : 0.f;
    const bool both = do_ce && !(do_kd && x.temperature == 1.f);
    const float inv_t = 1.f / x.temperature;

    u32x4x keep[NV];
    float top = 0.f, rt = 0.f, r1 = 0.f, kd = 0.f, ce = 0.f, zj = 0.f, zy = 0.f, q = 0.f;
    if (do_kd || do_ce) {
        Sums s;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int32_t c = (v * NT + tid) * PER;
            keep[v] = u32x4x{0, 0, 0, 0};
            if (c < C) keep[v] = *(const u32x4x *)(src + (int64_t)c * (BF ? 2 : 4));
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int32_t c = (v * NT + tid) * PER;
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (c + e < C) s.top = fmaxf(s.top, element<BF>(keep[v], e));
        }
        const float ref = s.top == -INFINITY ? 0.f : s.top;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int32_t c = (v * NT + tid) * PER;
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (c + e < C) {
                    s.st += exp_of<BF>(element<BF>(keep[v], e) - ref, inv_t);
                    if (both) s.s1 += exp_of<BF>(element<BF>(keep[v], e) - ref, 1.f);
                }
        }
        for (int64_t c = (int64_t)(NV * NT + tid) * PER; c < C; c += NT * PER) {
            const u32x4x v = *(const u32x4x *)(src + c * (BF ? 2 : 4));
            float z[PER];
#pragma unroll
            for (int e = 0; e < PER; ++e) z[e] = c + e < C ? element<BF>(v, e) : -INFINITY;
            add<BF>(s, z, PER, inv_t, both);
        }
        top = reduce<NT, true>(s.top, scratch);
        // (a thread without logits has no part; a row of -inf alone has no distribution)
        const float st = reduce<NT, false>(s.top == -INFINITY ? s.st : s.st * exp_of<BF>(s.top - top, inv_t), scratch);
        float s1 = st;
        if (both) s1 = reduce<NT, false>(s.top == -INFINITY ? s.s1 : s.s1 * exp_of<BF>(s.top - top, 1.f), scratch);
        const float nan = __builtin_nanf("");
        rt = top == -INFINITY ? nan : 1.f / st;
        r1 = top == -INFINITY ? nan : 1.f / s1;
        if (do_kd) {
            const float most = reduce<NT, true>(t, scratch);
            const float u = id >= 0 ? (t - most) * inv_t : 0.f, w = id >= 0 ? expf(u) : 0.f;
            const float sum = reduce<NT, false>(w, scratch);
            q = w / sum;
            if (id >= 0) {
                if constexpr (BF) zj = bf16_to_f32(((const uint16_t *)src)[id]);
                else zj = ((const float *)src)[id];
            }
            // an entry whose q is zero has no part, whatever the student's logit
            const float term = q == 0.f ? 0.f : q * ((u - logf(sum)) - ((zj - top) * inv_t - logf(st)));
            kd = reduce<NT, false>(term, scratch) * (x.temperature * x.temperature);
            if (top == -INFINITY) kd = nan;
            if (tid < x.k) share[tid] = q;
        }
        if (do_ce) {
            if constexpr (BF) zy = bf16_to_f32(((const uint16_t *)src)[y]);
            else zy = ((const float *)src)[y];
            ce = top == -INFINITY ? nan : logf(s1) - (zy - top);
        }
        // every logit that is needed by itself has been read: the gradient may take the logits' place
        __syncthreads();
    }
    if (tid == 0) {
        const float nan = __builtin_nanf("");
        if (has && wrong) kd = nan;
        if (off) ce = nan;
        a.kd[row] = kd;
        a.ce[row] = ce;
        if (x.row_loss) x.row_loss[row] = (x.alpha > 0.f ? x.alpha * kd : 0.f) + (x.alpha < 1.f ? (1.f - x.alpha) * ce : 0.f);
    }
    if (!x.dlogits) return;

    char *out = (char *)x.dlogits + row * x.ld_d * (BF ? 2 : 4);
    auto grad = [&](float z) {
        float g = 0.f;
        if (do_kd) g = wk * (exp_of<BF>(z - top, inv_t) * rt);
        if (do_ce) g += wc * ((both ? exp_of<BF>(z - top, 1.f) : exp_of<BF>(z - top, inv_t)) * r1);
        return g;
    };
    auto write = [&](const u32x4x &v, int64_t c) {
        float g[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) g[e] = c + e < C ? grad(element<BF>(v, e)) : 0.f;
        u32x4x o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (BF) o[e] = bf16_pair(g[2 * e], g[2 * e + 1]);
            else o[e] = __float_as_uint(g[e]);
        }
        *(u32x4x *)(out + c * (BF ? 2 : 4)) = o;
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int64_t c = (int64_t)(v * NT + tid) * PER;
        if (c < C) write(keep[v], c);
    }
    for (int64_t c = (int64_t)(NV * NT + tid) * PER; c < C; c += NT * PER) {
        u32x4x v = {0, 0, 0, 0};
        if (do_kd || do_ce) v = *(const u32x4x *)(src + c * (BF ? 2 : 4));
        write(v, c);
    }
    if (!do_kd && !do_ce) return;
    // the classes that have a share of the target, once each, over what was written
    __syncthreads();
    auto put = [&](int32_t c, float g) {
        if constexpr (BF) ((uint16_t *)out)[c] = bf16_rne(g);
        else ((float *)out)[c] = g;
    };
    if (do_kd && id >= 0) {
        float sum = 0.f;
        bool first = true;
        for (int32_t j = 0; j < x.k; ++j)
            if (ids[j] == id) {
                first = first && j >= tid;
                sum += share[j];
            }
        if (first) {
            float g = wk * (exp_of<BF>(zj - top, inv_t) * rt - sum);
            if (do_ce) g += wc * ((both ? exp_of<BF>(zj - top, 1.f) : exp_of<BF>(zj - top, inv_t)) * r1 - (id == y ? 1.f : 0.f));
            put(id, g);
        }
    }
    if (do_ce && tid == 0) {
        bool listed = false;
        if (do_kd)
            for (int32_t j = 0; j < x.k; ++j) listed = listed || ids[j] == y;
        if (!listed) {
            float g = wc * ((both ? exp_of<BF>(zy - top, 1.f) : exp_of<BF>(zy - top, inv_t)) * r1 - 1.f);
            if (do_kd) g += wk * (exp_of<BF>(zy - top, inv_t) * rt);
            put(y, g);
        }
    }
}

template <bool BF, int NT, int NV>
__global__ void __launch_bounds__(NT) k_distill_row(const Args a) {
    for (int64_t row = blockIdx.x; row < a.x.m; row += gridDim.x) distill_row<BF, NT, NV>(a, row);
}

namespace {
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
}  // namespace

size_t distill_workspace(int64_t m) { return (size_t)(kParts * 8 + 2 * up(m * 4, 256)); }

void launch_distill(const DistillArgs &x, hipStream_t s) {
    Args a = {};
    a.x = x;
    char *ws = (char *)x.workspace;
    a.counts = (int2 *)ws;
    a.parts = (int32_t)grid_for(x.m, 256, kParts);
    a.kd = (float *)(ws + kParts * 8);
    a.ce = a.kd + up(x.m * 4, 256) / 4;
    {
        KernelTimer t("distill_count", s);
        hipLaunchKernelGGL(k_distill_count, dim3((unsigned)a.parts), dim3(256), 0, s, a);
    }
    if (x.m > 0) {
        KernelTimer t("distill_row", s);
        if (x.bf16) hipLaunchKernelGGL((k_distill_row<true, 256, 4>), dim3(grid_for(x.m, 1, 1 << 20)), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_distill_row<false, 256, 4>), dim3(grid_for(x.m, 1, 1 << 20)), dim3(256), 0, s, a);
    }
    {
        KernelTimer t("distill_mean", s);
        hipLaunchKernelGGL(k_distill_mean, dim3(1), dim3(1024), 0, s, a);
    }
    GNNAV_HIP(hipGetLastError());
}

}  // namespace gnnav
