// Kernels of the exchange of answers (see include/d2mhe.h): row statistics of logits, the largest logits of a
// row, log-probabilities at given classes, distillation loss and gradient.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "../../include/d2mhe.h"

namespace d2 {
namespace answers {

constexpr uint32_t MAX_TOP = D2MHE_MAX_TOP;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

struct Rows {
    const void *z;
    uint64_t stride;
    uint32_t rows, classes;
};

struct Answers {
    const int32_t *index;
    const float *sum, *weight;
    uint32_t k;
    float inv_members, inv_t;
};

__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(_Float16 x) { return (float)x; }
__device__ inline float to_float(__bf16 x) { return (float)x; }

__device__ inline float neg_inf() { return -__builtin_inff(); }

// ---- reductions over a workgroup of 256 ------------------------------------------------------------------

struct Max {
    static __device__ float of(float a, float b) { return fmaxf(a, b); }
};
struct Add {
    static __device__ float of(float a, float b) { return a + b; }
};

// every thread gets the result; `buf` is 4 floats of LDS that nothing else uses until the next barrier
template <class Op> __device__ inline float block_reduce(float v, float *buf)
{
    for (int d = 32; d; d >>= 1) v = Op::of(v, __shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    return Op::of(Op::of(buf[0], buf[1]), Op::of(buf[2], buf[3]));
}

// Maximum m and S = sum exp((z - m) / T) of a row.  (z - m) is rounded before the product with 1 / T, so that a row of the
// type's lowest value gives S = classes and not inf - inf; a row of -inf gives S = 0.
struct Stats {
    float m, s;
};

template <class T> __device__ inline Stats row_stats(const T *z, uint32_t n, float scale, float *buf)
{
    float m = neg_inf();
    for (uint32_t v = threadIdx.x; v < n; v += 256) m = fmaxf(m, to_float(z[v]));
    m = block_reduce<Max>(m, buf);
    const float base = m == neg_inf() ? 0.0f : m;
    float s = 0;
    for (uint32_t v = threadIdx.x; v < n; v += 256) s += __builtin_amdgcn_exp2f((to_float(z[v]) - base) * scale);
    return {m, block_reduce<Add>(s, buf)};
}

// ---- log-probabilities at given classes ------------------------------------------------------------------

template <class T>
__global__ void __launch_bounds__(256) k_logprobs_at(Rows in, const int32_t *index, uint32_t k, float *out)
{
    __shared__ float buf[4];
    for (uint64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
        const T *z = (const T *)in.z + r * in.stride;
        const Stats st = row_stats(z, in.classes, LOG2E, buf);
        const float log_s = __logf(st.s);
        for (uint32_t j = threadIdx.x; j < k; j += 256) {
            const int32_t v = index[r * k + j];
            float lp = 0;
            if ((uint32_t)v < in.classes) {
                const float x = to_float(z[v]);
                lp = x == neg_inf() && st.s == st.s ? neg_inf() : (x - st.m) - log_s;
            }
            out[r * k + j] = lp;
        }
    }
}

// ---- the k largest logits --------------------------------------------------------------------------------

// Order of the floats as whole numbers (-0 as +0); 0 for what is never chosen: NaN and -inf.
__device__ inline uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    if (!(x > neg_inf())) return 0;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ inline float value_of(uint32_t order)
{
    return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order);
}

// order and position in one key: of equal values the lower class is the larger key; no two keys of a row are alike
__device__ inline uint64_t key_of(float x, uint32_t v) { return (uint64_t)order_of(x) << 32 | (0xffffffffu - v); }

// The k-th largest key digit by digit from the top: the counts of the next eight bits among the keys that agree with the
// digits chosen so far.
template <class T>
__global__ void __launch_bounds__(256) k_top(Rows in, uint32_t k, int32_t *index, float *out)
{
    __shared__ float buf[4];
    __shared__ uint32_t count[256], found;
    __shared__ uint64_t least, best[MAX_TOP];
    __shared__ uint32_t need, done;
    for (uint64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
        const T *z = (const T *)in.z + r * in.stride;
        const Stats st = row_stats(z, in.classes, LOG2E, buf);
        const float log_s = __logf(st.s);
        __syncthreads();
        if (threadIdx.x == 0) {
            least = 0;
            need = k;
            done = found = 0;
        }
        for (int shift = 56; shift >= 0; shift -= 8) {
            count[threadIdx.x] = 0;
            __syncthreads();
            if (done) break;
            const uint64_t prefix = least;
            for (uint32_t v = threadIdx.x; v < in.classes; v += 256) {
                const uint64_t key = key_of(to_float(z[v]), v);
                if ((key >> 32) && (shift == 56 || (key >> (shift + 8)) == (prefix >> (shift + 8))))
                    atomicAdd(&count[(key >> shift) & 255], 1u);
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                int d = 255;
                uint32_t left = need;
                while (d > 0 && count[d] < left) left -= count[d--];
                least = prefix | (uint64_t)d << shift;
                done = count[d] <= left;
                need = left;
            }
            __syncthreads();
        }
        __syncthreads();
        for (uint32_t v = threadIdx.x; v < in.classes; v += 256) {
            const uint64_t key = key_of(to_float(z[v]), v);
            if ((key >> 32) && key >= least) best[atomicAdd(&found, 1u)] = key;
        }
        __syncthreads();
        const uint32_t n = found;
        if (threadIdx.x < k) {
            if (threadIdx.x < n) {
                const uint64_t key = best[threadIdx.x];
                uint32_t rank = 0;
                for (uint32_t j = 0; j < n; ++j) rank += best[j] > key;
                index[r * k + rank] = (int32_t)(0xffffffffu - (uint32_t)key);
                out[r * k + rank] = (value_of((uint32_t)(key >> 32)) - st.m) - log_s;
            } else {
                index[r * k + threadIdx.x] = -1;
                out[r * k + threadIdx.x] = 0;
            }
        }
        __syncthreads();
    }
}

// ---- distillation ----------------------------------------------------------------------------------------

// Slot j of a row belongs to thread j (k <= 256 = threads).
struct Slot {
    int32_t v;      // class, or -1: empty
    float t, p;     // log p and p
};

// softmax over the filled slots; false: the row has none (the whole workgroup gets the same answer)
__device__ inline bool teacher_slot(const Answers &a, uint64_t r, uint32_t classes, Slot &slot, float *buf)
{
    slot.v = -1;
    slot.t = neg_inf();
    if (threadIdx.x < a.k) {
        const int32_t v = a.index[r * a.k + threadIdx.x];
        const float t = a.sum[r * a.k + threadIdx.x];
        if ((uint32_t)v < classes && t != neg_inf()) {
            slot.v = v;
            slot.t = t * a.inv_members * a.inv_t;
        }
    }
    const bool some = __syncthreads_or(slot.v >= 0);
    const float m = block_reduce<Max>(slot.t, buf);
    slot.t -= m;
    slot.p = slot.v >= 0 ? __builtin_amdgcn_exp2f(slot.t * LOG2E) : 0.0f;
    const float s = block_reduce<Add>(slot.p, buf);
    slot.t -= __logf(s);
    slot.p /= s;
    return some;
}

// Gradient at the teacher's classes, over the dense part that the workgroup has stored: the p of all slots of a class are
// added up in slot order by each of them, so that a class given twice is stored twice with the same value.
template <class T>
__device__ inline void store_slots(T *grad, const Slot &slot, float student, float g, uint32_t k, int32_t *vs, float *ps)
{
    __syncthreads();
    vs[threadIdx.x] = slot.v;
    ps[threadIdx.x] = slot.p;
    __syncthreads();
    if (slot.v >= 0) {
        float p = 0;
        for (uint32_t j = 0; j < k; ++j) p += vs[j] == slot.v ? ps[j] : 0.0f;
        grad[slot.v] = (T)((student - p) * g);
    }
}

template <class T>
__global__ void __launch_bounds__(256) k_distill(Rows in, Answers a, float *loss, float *lse, T *grad, uint64_t grad_stride)
{
    __shared__ float buf[4], ps[MAX_TOP];
    __shared__ int32_t vs[MAX_TOP];
    const float scale = a.inv_t * LOG2E;
    for (uint64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
        const T *z = (const T *)in.z + r * in.stride;
        T *out = grad ? grad + r * grad_stride : nullptr;
        const float w = a.weight ? a.weight[r] : 1.0f;
        Slot slot;
        bool live = w != 0.0f && teacher_slot(a, r, in.classes, slot, buf);
        Stats st = {0, 0};
        if (live) st = row_stats(z, in.classes, scale, buf);
        const bool none = live && st.m == neg_inf() && st.s == 0.0f;     // all logits -inf
        live = live && !none;
        if (!live) {
            if (threadIdx.x == 0) {
                loss[r] = 0;
                lse[r] = none ? neg_inf() : 0.0f;
            }
            if (out)
                for (uint32_t v = threadIdx.x; v < in.classes; v += 256) out[v] = (T)0.0f;
            continue;
        }
        const float log_s = __logf(st.s), inv_s = 1.0f / st.s;
        float x = 0, part = 0;
        if (slot.v >= 0) {
            x = to_float(z[slot.v]) - st.m;
            part = slot.p > 0 || slot.p != slot.p ? slot.p * (slot.t - (x * a.inv_t - log_s)) : 0.0f;
        }
        part = block_reduce<Add>(part, buf);
        if (threadIdx.x == 0) {
            loss[r] = w * part;
            lse[r] = st.m * a.inv_t + log_s;
        }
        if (!out) continue;
        const float g = w * a.inv_t;
        for (uint32_t v = threadIdx.x; v < in.classes; v += 256)
            out[v] = (T)(__builtin_amdgcn_exp2f((to_float(z[v]) - st.m) * scale) * inv_s * g);
        store_slots(out, slot, __builtin_amdgcn_exp2f(x * scale) * inv_s, g, a.k, vs, ps);
    }
}

template <class T>
__global__ void __launch_bounds__(256) k_distill_backward(Rows in, Answers a, const float *lse, T *grad, uint64_t grad_stride)
{
    __shared__ float buf[4], ps[MAX_TOP];
    __shared__ int32_t vs[MAX_TOP];
    for (uint64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
        const T *z = (const T *)in.z + r * in.stride;
        T *out = grad + r * grad_stride;
        const float w = a.weight ? a.weight[r] : 1.0f, l = lse[r];
        Slot slot;
        const bool live = w != 0.0f && l != neg_inf() && teacher_slot(a, r, in.classes, slot, buf);
        if (!live) {
            for (uint32_t v = threadIdx.x; v < in.classes; v += 256) out[v] = (T)0.0f;
            continue;
        }
        const float g = w * a.inv_t;
        // z / T is not rounded before lse is taken off
        auto student = [&](float x) { return __builtin_amdgcn_exp2f(__builtin_fmaf(x, a.inv_t, -l) * LOG2E); };
        for (uint32_t v = threadIdx.x; v < in.classes; v += 256) out[v] = (T)(student(to_float(z[v])) * g);
        const float p = slot.v >= 0 ? student(to_float(z[slot.v])) : 0.0f;
        store_slots(out, slot, p, g, a.k, vs, ps);
    }
}

}  // namespace answers
}  // namespace d2
