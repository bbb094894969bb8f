// The global norm of many tensors, clipping by it, and the SGD step of clipped
// gradients.
//
//   norm = sqrt(sum of squares over all tensors), c = min(1, max_norm / norm)
//   clip: out = c * g      step: w = w - lr * c * g
//
// Squares are summed in 64 bits: fp32 squares leave their range at 2^64, and
// the adds are free beside the loads.  A first launch writes one part sum per
// workgroup, the second adds the parts up in every workgroup, in one fixed
// order, and goes over the tensors again, last element first: what the first
// pass read last is still in the last-level cache.  The tensors' table travels
// as a kernel argument, kClipTensors tensors a launch.
//
// Bound by HBM, read twice and written once: 400 million bf16 gradients 2.4 GB in
// 471 us, 5.1 TB/s; two small tensors by their two launches, 9 us.
#include <algorithm>

#include "common.hpp"

namespace gnnav {

namespace {

typedef float f32x4p __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4p __attribute__((ext_vector_type(4)));

constexpr int kClipTensors = 96;       // of a launch: the table stays below 4 KB of arguments
constexpr int64_t kClipChunk = 16384;  // elements a workgroup takes at a time
constexpr int64_t kClipParts = 4096;   // part sums, at most (or one per launch)
// Results larger than this are stored past the caches, which then hold more of the gradients for the second
// pass: 400 million bf16 gradients, three sets of buffers in turn, 502 us, 471 so; 84 million 100.5 and 85.0.  (A kernel has
// one kind of store: of two in the branches of an `if` the compiler makes one, of the ordinary kind.)
constexpr int64_t kStreamBytes = int64_t(128) << 20;

struct ClipTable {
    const void *g[kClipTensors];
    void *out[kClipTensors];
    int64_t count[kClipTensors];
    int32_t first[kClipTensors + 1];   // first chunk of each tensor
    int32_t n;
};
static_assert(sizeof(ClipTable) <= 2704, "kernel arguments");

enum { kNorm, kClip, kStep };

template <class T>
__device__ __forceinline__ float to_f32(T x) {
    if constexpr (sizeof(T) == 2) return bf16_to_f32(x);
    else return x;
}
template <class T>
__device__ __forceinline__ T from_f32(float x) {
    if constexpr (sizeof(T) == 2) return bf16_rne(x);
    else return x;
}

__device__ __forceinline__ double block_sum(double x, double *scratch) {   // 256 threads; the sum, in every thread
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
    if (lane_id() == 0) scratch[threadIdx.x / kWave] = x;
    __syncthreads();
    x = (scratch[0] + scratch[1]) + (scratch[2] + scratch[3]);
    __syncthreads();
    return x;
}

}  // namespace

// The part sums, added up by every workgroup that needs them in the same order.
__device__ __forceinline__ double norm_of(const double *parts, int32_t n_parts, double *scratch) {
    double x = 0.0;
    for (int32_t i = threadIdx.x; i < n_parts; i += 256) x += parts[i];
    return sqrt(block_sum(x, scratch));
}

// OP kNorm: one part sum per workgroup to parts[blockIdx.x].  kClip, kStep: the second pass.
template <class T, int OP, bool STREAMED>
__global__ void __launch_bounds__(256) k_clip(const ClipTable t, double *__restrict__ parts, int32_t n_parts,
                                              double max_norm, float lr, float *__restrict__ norm, bool in_place) {
    constexpr int N = 16 / sizeof(T);
    __shared__ double scratch[4];
    const int tid = threadIdx.x;
    float factor = 1.f;
    if constexpr (OP != kNorm) {
        const double x = norm_of(parts, n_parts, scratch);
        if (norm && blockIdx.x == 0 && tid == 0) norm[0] = (float)x;
        const float c = x <= max_norm ? 1.f : (float)(max_norm / x);
        factor = OP == kStep ? lr * c : c;
        if (OP == kClip && in_place && c == 1.f) return;
    }
    double sum = 0.0;
    const int32_t chunks = t.first[t.n];
    for (int32_t i = blockIdx.x; i < chunks; i += gridDim.x) {
        const int32_t chunk = OP == kNorm ? i : chunks - 1 - i;
        int lo = 0, hi = t.n - 1;
        while (lo < hi) {   // the tensor that holds the chunk
            const int mid = (lo + hi + 1) >> 1;
            if (t.first[mid] <= chunk) lo = mid;
            else hi = mid - 1;
        }
        const int64_t at = (int64_t)(chunk - t.first[lo]) * kClipChunk;
        const int32_t len = (int32_t)std::min<int64_t>(kClipChunk, t.count[lo] - at);
        const T *g = (const T *)t.g[lo] + at;
        T *out = OP == kNorm ? nullptr : (T *)t.out[lo] + at;
        const uint32_t off = (uint32_t)((uintptr_t)g & 15u);
        // 16-byte units where both tensors lie alike; the elements before the first and behind the last one by one
        const bool alike = OP == kNorm || off == (uint32_t)((uintptr_t)out & 15u);
        const int32_t head = alike ? std::min<int32_t>(len, off ? (int32_t)((16u - off) / sizeof(T)) : 0) : len;
        const int32_t units = (len - head) / N;
        auto one = [&](int32_t e) {
            const float x = to_f32<T>(g[e]);
            if constexpr (OP == kNorm) sum += (double)x * (double)x;
            else if constexpr (OP == kClip) out[e] = from_f32<T>(factor * x);
            else out[e] = from_f32<T>(to_f32<T>(out[e]) - factor * x);
        };
        for (int32_t e = tid; e < head; e += 256) one(e);
        for (int32_t e = head + units * N + tid; e < len; e += 256) one(e);
        const u32x4p *gv = (const u32x4p *)(g + head);
        u32x4p *ov = (u32x4p *)(out + (OP == kNorm ? 0 : head));
        auto value = [](const u32x4p &u, int e) {
            if constexpr (N == 4) return __uint_as_float(u[e]);
            else return __uint_as_float(e & 1 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16);
        };
        auto unit = [&](int32_t u, u32x4p x, u32x4p w) {
            if constexpr (OP == kNorm) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const double y = value(x, e);
                    sum += y * y;
                }
            } else {
                float y[N];
#pragma unroll
                for (int e = 0; e < N; ++e) y[e] = OP == kClip ? factor * value(x, e) : value(w, e) - factor * value(x, e);
                u32x4p r;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if constexpr (N == 4) r[q] = __float_as_uint(y[q]);
                    else r[q] = (uint32_t)bf16_rne(y[2 * q]) | ((uint32_t)bf16_rne(y[2 * q + 1]) << 16);
                }
                if constexpr (STREAMED) __builtin_nontemporal_store(r, &ov[u]);
                else ov[u] = r;
            }
        };
        constexpr int F = 4;   // units of a thread in flight
        int32_t u = tid;
        for (; u + (F - 1) * 256 < units; u += F * 256) {
            u32x4p x[F], w[F];
#pragma unroll
            for (int f = 0; f < F; ++f) {
                x[f] = gv[u + f * 256];
                w[f] = OP == kStep ? ov[u + f * 256] : x[f];
            }
#pragma unroll
            for (int f = 0; f < F; ++f) unit(u + f * 256, x[f], w[f]);
        }
        for (; u < units; u += 256) unit(u, gv[u], OP == kStep ? ov[u] : gv[u]);
    }
    if constexpr (OP == kNorm) {
        sum = block_sum(sum, scratch);
        if (tid == 0) parts[blockIdx.x] = sum;
    }
}

__global__ void __launch_bounds__(256) k_norm(const double *__restrict__ parts, int32_t n_parts,
                                              float *__restrict__ norm) {
    __shared__ double scratch[4];
    const double x = norm_of(parts, n_parts, scratch);
    if (threadIdx.x == 0) norm[0] = (float)x;
}

namespace {
int64_t clip_launches(int64_t n_tensors) { return std::max<int64_t>(1, (n_tensors + kClipTensors - 1) / kClipTensors); }
int64_t chunks_of(int64_t count) { return (count + kClipChunk - 1) / kClipChunk; }
}  // namespace

size_t clip_workspace(int64_t n_tensors) {
    return (size_t)std::max<int64_t>(kClipParts, clip_launches(n_tensors)) * sizeof(double);
}

// out nullptr: the norm only.  step: out holds weights, which take -lr * c * g.
void launch_clip(int32_t n_tensors, const void *const *grads, const int64_t *counts, bool bf16, double max_norm,
                 void *const *out, bool step, float lr, float *norm, void *ws, hipStream_t s) {
    double *parts = (double *)ws;
    const int64_t launches = clip_launches(n_tensors);
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(1024, kClipParts / launches));
    int32_t n_parts = 0;
    bool in_place = out && !step;
    int64_t elements = 0;
    for (int32_t k = 0; k < n_tensors; ++k) elements += counts[k];
    const bool streamed = elements * (bf16 ? 2 : 4) > kStreamBytes;
    auto each = [&](bool backwards, auto &&f) {
        for (int64_t i = 0; i < launches; ++i) {
            const int64_t l = backwards ? launches - 1 - i : i;
            ClipTable t = {};
            const int32_t b = (int32_t)(l * kClipTensors);
            t.n = std::min<int32_t>(kClipTensors, n_tensors - b);
            int64_t chunk = 0;
            for (int32_t k = 0; k < t.n; ++k) {
                t.g[k] = grads[b + k];
                t.out[k] = out ? out[b + k] : nullptr;
                t.count[k] = counts[b + k];
                t.first[k] = (int32_t)chunk;
                chunk += chunks_of(counts[b + k]);
                if (counts[b + k] > 0 && t.g[k] != t.out[k]) in_place = false;
            }
            if (chunk > INT32_MAX) fail(GNNAV_E_CAPACITY, "too many elements");
            t.first[t.n] = (int32_t)chunk;
            f(t, chunk);
        }
    };
    each(false, [&](const ClipTable &t, int64_t chunks) {
        if (chunks == 0) return;
        KernelTimer timer("grad_norm", s);
        const unsigned grid = (unsigned)std::min<int64_t>(chunks, most);
        if (bf16)
            hipLaunchKernelGGL((k_clip<uint16_t, kNorm, false>), dim3(grid), dim3(256), 0, s, t, parts + n_parts, 0, 0.0, 0.f,
                               nullptr, false);
        else
            hipLaunchKernelGGL((k_clip<float, kNorm, false>), dim3(grid), dim3(256), 0, s, t, parts + n_parts, 0, 0.0, 0.f,
                               nullptr, false);
        n_parts += (int32_t)grid;
    });
    if (!out || n_parts == 0) {
        KernelTimer timer("grad_norm", s);
        hipLaunchKernelGGL(k_norm, dim3(1), dim3(256), 0, s, parts, n_parts, norm);
    } else {
        each(true, [&](const ClipTable &t, int64_t chunks) {
            if (chunks == 0) return;
            KernelTimer timer(step ? "sgd_clip_step" : "clip_grads", s);
            const unsigned grid = (unsigned)std::min<int64_t>(chunks, 1024);
#define GNNAV_L(T, OP)                                                                                                \
    do {                                                                                                              \
        if (streamed)                                                                                                 \
            hipLaunchKernelGGL((k_clip<T, OP, true>), dim3(grid), dim3(256), 0, s, t, parts, n_parts, max_norm, lr,   \
                               norm, in_place);                                                                       \
        else                                                                                                          \
            hipLaunchKernelGGL((k_clip<T, OP, false>), dim3(grid), dim3(256), 0, s, t, parts, n_parts, max_norm, lr,  \
                               norm, in_place);                                                                       \
    } while (0)
            if (step) {
                if (bf16) GNNAV_L(uint16_t, kStep);
                else GNNAV_L(float, kStep);
            } else {
                if (bf16) GNNAV_L(uint16_t, kClip);
                else GNNAV_L(float, kClip);
            }
#undef GNNAV_L
        });
    }
    GNNAV_HIP(hipGetLastError());
}

}  // namespace gnnav
