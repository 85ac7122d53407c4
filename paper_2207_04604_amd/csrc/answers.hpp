// Kernels of the exchange of answers (see include/d2mhe.h): row statistics of logits, the largest logits of a
// row, log-probabilities at given classes, distillation loss and gradient.
//
// All of them stream: a row of V logits is read once (and its gradient written once), with one exp2 per logit for the
// statistics and one more for the gradient.  Vector instructions a logit, by counters: log-probabilities of 32768 classes 9, loss of
// 50001 10, top classes of 131072 11 and of 100 71, step of 131072 13 and of 32768 17, gradient alone of 1000 and of 65537 21: the
// slots' part of the last is as large as the row's.  What bounds long rows is memory (a device copy moves 4.9 TB/s here), short rows
// the instructions around a row.  Rows therefore stay in registers between the passes, and 16 to 1024 threads share one: as many
// as hold it.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../../include/d2mhe.h"

namespace d2 {
namespace answers {

constexpr uint32_t MAX_TOP = D2MHE_MAX_TOP;
constexpr float LOG2E = 1.44269504088896340736f;

struct Rows {
    const void *z;
    uint64_t stride;
    uint32_t first, rows, classes;      // the launch's rows: first .. rows - 1
};

struct Answers {
    const int32_t *index;
    const float *sum, *weight;
    uint32_t k;
    float share, inv_t;                 // a sum's factor to s / T: 1 / (members * T); 1 / T
};

__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(_Float16 x) { return (float)x; }
__device__ inline float to_float(__bf16 x) { return (float)x; }

__device__ inline float neg_inf() { return -__builtin_inff(); }

// ---- 16 bytes of logits -----------------------------------------------------------------------------------

typedef uint32_t Word4 __attribute__((ext_vector_type(4), may_alias));
// any alignment of an element: the machine takes 16-byte accesses at odd addresses
typedef Word4 Word4Any __attribute__((aligned(2), may_alias));

template <class T> struct Pack;                 // E elements in 16 bytes
template <> struct Pack<float> {
    static constexpr int E = 4;
    static __device__ void open(Word4 w, float *x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
    }
    static __device__ Word4 close(const float *x)
    {
        Word4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
        return w;
    }
    static constexpr uint32_t NONE = 0xff800000u;                // -inf
};
template <> struct Pack<__bf16> {
    static constexpr int E = 8;
    static __device__ void open(Word4 w, float *x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ Word4 close(const float *x)
    {
        typedef __bf16 Two __attribute__((ext_vector_type(2)));
        Word4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Two t = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, t);
        }
        return w;
    }
    static constexpr uint32_t NONE = 0xff80ff80u;
};
template <> struct Pack<_Float16> {
    static constexpr int E = 8;
    typedef _Float16 Two __attribute__((ext_vector_type(2)));
    static __device__ void open(Word4 w, float *x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t pair = w[i];          // a bit cast of w[i] itself reads element 0
            const Two t = __builtin_bit_cast(Two, pair);
            x[2 * i] = (float)t.x;
            x[2 * i + 1] = (float)t.y;
        }
    }
    static __device__ Word4 close(const float *x)
    {
        Word4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Two t = {(_Float16)x[2 * i], (_Float16)x[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, t);
        }
        return w;
    }
    static constexpr uint32_t NONE = 0xfc00fc00u;
};

// fmaxf without the quieting of signalling NaNs that it costs on values that come straight from memory: where one of them is a
// signalling NaN, the others may get lost
__device__ inline float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// ---- a row and the NT threads that work on it -------------------------------------------------------------

struct Max {
    static __device__ float of(float a, float b) { return fmaxf(a, b); }
};
struct Add {
    static __device__ float of(float a, float b) { return a + b; }
    static __device__ uint32_t of(uint32_t a, uint32_t b) { return a + b; }
};

struct Min {
    static __device__ uint32_t of(uint32_t a, uint32_t b) { return a < b ? a : b; }
};

template <int ROR, class V> __device__ inline V rotated(V v)            // lane l of 16: what lane l - ROR holds
{
    if constexpr (sizeof(V) == 8) {
        return (V)rotated<ROR>((uint32_t)(v >> 32)) << 32 | rotated<ROR>((uint32_t)v);
    } else {
        const int i = __builtin_bit_cast(int, v);
        return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(i, i, 0x120 + ROR, 0xf, 0xf, false));
    }
}

// how many of the 16 lanes that turn with a lane hold more than it
template <int R = 15, class V> __device__ inline uint32_t larger_of_16(V v)
{
    if constexpr (R == 0) return 0;
    else return larger_of_16<R - 1>(v) + (rotated<R>(v) > v);
}

// lane l of 16: the sum of what the lanes before it hold
__device__ inline uint32_t before_in_16(uint32_t v)
{
    uint32_t s = v;
    s += __builtin_amdgcn_update_dpp(0, s, 0x111, 0xf, 0xf, true);          // from the lane before, 0 in the first
    s += __builtin_amdgcn_update_dpp(0, s, 0x112, 0xf, 0xf, true);
    s += __builtin_amdgcn_update_dpp(0, s, 0x114, 0xf, 0xf, true);
    s += __builtin_amdgcn_update_dpp(0, s, 0x118, 0xf, 0xf, true);
    return s - v;
}

// Op over the W neighbouring lanes of a lane, in all of them and to the same bits: rotations within 16 lanes, then exchanges
// of halves (register moves, where a shuffle goes through LDS).
template <class Op, int W, class V> __device__ inline V across(V v)
{
    if (W >= 2) v = Op::of(v, rotated<W >= 16 ? 8 : W >= 8 ? 4 : W >= 4 ? 2 : 1>(v));
    if (W >= 4) v = Op::of(v, rotated<W >= 16 ? 4 : W >= 8 ? 2 : 1>(v));
    if (W >= 8) v = Op::of(v, rotated<W >= 16 ? 2 : 1>(v));
    if (W >= 16) v = Op::of(v, rotated<1>(v));
    if (W >= 32) {
        const uint32_t i = __builtin_bit_cast(uint32_t, v);
        const auto halves = __builtin_amdgcn_permlane16_swap(i, i, false, false);
        const uint32_t x = halves[0], y = halves[1];
        v = Op::of(__builtin_bit_cast(V, x), __builtin_bit_cast(V, y));
    }
    if (W >= 64) {
        const uint32_t i = __builtin_bit_cast(uint32_t, v);
        const auto halves = __builtin_amdgcn_permlane32_swap(i, i, false, false);
        const uint32_t x = halves[0], y = halves[1];
        v = Op::of(__builtin_bit_cast(V, x), __builtin_bit_cast(V, y));
    }
    return v;
}

// Maximum m and s = sum exp2((x - m) * scale) of some elements.  (x - m) is rounded before the product, so that elements of
// the type's lowest value give their number and not inf - inf; elements of -inf give m = -inf, s = 0.
struct Stats {
    float m, s;

    // s as seen from another maximum
    __device__ float at(float top, float scale) const { return s == 0.0f ? 0.0f : s * __builtin_amdgcn_exp2f((m - top) * scale); }
    // of the W neighbouring lanes
    template <int W> __device__ Stats together(float scale) const
    {
        const float top = across<Max, W>(m);
        return {top, across<Add, W>(at(top, scale))};
    }
};

// A workgroup has 256 threads or NT, whichever is more; groups of up to a wavefront never meet a barrier.
template <int NT> struct Group {
    static constexpr int SIZE = NT < 256 ? 256 : NT, ROWS = SIZE / NT, WAVES = NT < 64 ? 1 : NT / 64, LANES = NT < 64 ? NT : 64;
    static constexpr int TOP = NT < 64 ? 64 : MAX_TOP, SLOTS = NT < TOP ? TOP / NT : 1;     // slots of a row, of a thread

    static __device__ uint32_t thread() { return threadIdx.x % NT; }
    static __device__ uint32_t row_in_group() { return threadIdx.x / NT; }
    static __device__ uint32_t wave() { return NT > 64 ? threadIdx.x >> 6 : 0; }
    static __device__ void sync()
    {
        if (NT > 64) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    // Statistics of a wavefront's lanes to those of the group, over a barrier between the two calls.
    static __device__ void put(Stats v, Stats *buf)
    {
        if (NT > 64 && (threadIdx.x & 63) == 0) buf[wave()] = v;
    }
    static __device__ Stats get(Stats v, const Stats *buf, float scale)
    {
        if (NT <= 64) return v;
        return buf[threadIdx.x % WAVES].template together<WAVES>(scale);
    }
};

constexpr float FAR = 4194304.0f;       // from here on x * scale has no bits to spare next to the whole numbers

// The elements of a row: full 16-byte words from the first aligned address on, word c of the row with thread c % NT; the
// words 0 .. NV * NT - 1 stay in registers, any others are read again by every pass.  What lies before and behind the
// full words (at most 2 (E - 1) elements) goes one to a thread: `edge`, -inf where a thread has none.
template <class T, int NT, int NV> struct Row {
    using P = Pack<T>;
    using G = Group<NT>;
    static constexpr int E = P::E;
    const T *z;
    const Word4 *words;
    uint32_t head, n, at;           // elements before the words; words; position of the edge element (none: 0xffffffff)
    float edge;
    Word4 held[NV];

    // `first`, `count`: the words to take of the row, with the edges if the first is among them
    __device__ void place(const T *row, uint32_t classes, uint32_t first = 0, uint32_t count = 0xffffffffu)
    {
        const uint32_t t = G::thread();
        z = row;
        const uint32_t skip = (uint32_t)(-(uintptr_t)row & 15) / sizeof(T);
        head = skip < classes ? skip : classes;
        n = (classes - head) / E;
        const uint32_t tail = (classes - head) % E;
        at = t < head ? t : t >= NT - tail ? classes - NT + t : 0xffffffffu;
        if (first) at = 0xffffffffu;
        head += first * E;
        words = (const Word4 *)(row + head);
        n = n > first ? n - first : 0;
        n = n < count ? n : count;
    }
    __device__ void load()
    {
        const uint32_t t = G::thread();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            held[i] = Word4{P::NONE, P::NONE, P::NONE, P::NONE};
            if ((uint32_t)i * NT < n) {
                const uint32_t c = i * NT + t;
                if (c < n) held[i] = words[c];
            }
        }
        edge = at != 0xffffffffu ? to_float(z[at]) : neg_inf();
    }
    // The words as they are, not as what an earlier pass made of them: the compiler would keep the opened elements of all
    // words for the next pass, twice the registers of the words themselves.
    __device__ Word4 fresh(int i)
    {
        asm("" : "+v"(held[i]));
        return held[i];
    }
    // f(16 bytes): the words of this thread; words past the end hold -inf
    template <class F> __device__ void each(F f)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((uint32_t)i * NT < n) f(fresh(i));
        for (uint32_t c = NV * NT + G::thread(); c < n; c += NT) f(words[c]);
    }
    // f(16 bytes, position of their first element): the words of this thread that the row has
    template <class F> __device__ void each_at(F f)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((uint32_t)i * NT < n) {
                const uint32_t c = i * NT + G::thread();
                if (c < n) f(fresh(i), head + c * E);
            }
        for (uint32_t c = NV * NT + G::thread(); c < n; c += NT) f(words[c], head + c * E);
    }
    // the same from memory, in a loop: for what hardly ever runs
    template <class F> __device__ void again_at(F f) const
    {
#pragma unroll 1
        for (uint32_t c = G::thread(); c < n; c += NT) f(words[c], head + c * E);
    }
    // f(element, its position), from memory
    template <class F> __device__ void elements_again(F f) const
    {
        again_at([&](Word4 w, uint32_t v) {
            float x[E];
            P::open(w, x);
#pragma unroll
            for (int i = 0; i < E; ++i) f(x[i], v + i);
        });
        if (at != 0xffffffffu) f(edge, at);
    }
    // Statistics of a wavefront's elements, and `mine`: the maximum of this thread's.
    // One pass, while the words arrive: exp2 of x * scale less a whole number next to the maximum of the first words, which
    // costs one rounding and needs no maximum of the row.  Where the true maximum turns out to be far from it, or far from 0,
    // the sum is made again.
    __device__ Stats stats(float scale, float &mine)
    {
        float m = edge;
        if (NV > 1) {
            float x[E];
            P::open(held[0], x);
#pragma unroll
            for (int i = 0; i < E; i += 2) m = max3(m, x[i], x[i + 1]);
            m = across<Max, G::LANES>(m);
        } else {
            each([&](Word4 w) {
                float x[E];
                P::open(w, x);
#pragma unroll
                for (int i = 0; i < E; i += 2) m = max3(m, x[i], x[i + 1]);
            });
            mine = m;
            m = across<Max, G::LANES>(m);
        }
        const float first = m * scale, base = fabsf(first) < FAR ? __builtin_rintf(first) : 0.0f;
        float s = __builtin_amdgcn_exp2f(__builtin_fmaf(edge, scale, -base)), most = edge;
        each([&](Word4 w) {
            float x[E], part = 0;
            P::open(w, x);
            if (NV > 1)
#pragma unroll
                for (int i = 0; i < E; i += 2) most = max3(most, x[i], x[i + 1]);
#pragma unroll
            for (int i = 0; i < E; ++i) part += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], scale, -base));
            s += part;
        });
        if (NV > 1) {
            mine = most;
            m = across<Max, G::LANES>(most);
        }
        const float top = m * scale;
        if (fabsf(top) < FAR && fabsf(top - base) <= 64) {
            s *= __builtin_amdgcn_exp2f(__builtin_fmaf(-m, scale, base));
        } else if (m != neg_inf()) {
            s = __builtin_amdgcn_exp2f((edge - m) * scale);
            again_at([&](Word4 w, uint32_t) {
                float x[E];
                P::open(w, x);
#pragma unroll
                for (int i = 0; i < E; ++i) s += __builtin_amdgcn_exp2f((x[i] - m) * scale);
            });
        }
        return {m, across<Add, G::LANES>(s)};
    }
    // grad = f * exp2((x - m) * scale), rounded to nearest once, here; exp2 of the machine is 0 below 2^-126
    __device__ void store(T *out, float m, float scale, float f)
    {
        const float top = m * scale;
        if (fabsf(top) < FAR) {
            const float base = __builtin_rintf(top), g = f * __builtin_amdgcn_exp2f(__builtin_fmaf(-m, scale, base));
            each_at([&](Word4 w, uint32_t v) {
                float x[E];
                P::open(w, x);
#pragma unroll
                for (int i = 0; i < E; ++i) x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], scale, -base)) * g;
                *(Word4Any *)(out + v) = P::close(x);
            });
        } else {
            again_at([&](Word4 w, uint32_t v) {
                float x[E];
                P::open(w, x);
#pragma unroll
                for (int i = 0; i < E; ++i) x[i] = __builtin_amdgcn_exp2f((x[i] - m) * scale) * f;
                *(Word4Any *)(out + v) = P::close(x);
            });
        }
        if (at != 0xffffffffu) out[at] = (T)(__builtin_amdgcn_exp2f((edge - m) * scale) * f);
    }
    __device__ void clear(T *out)
    {
        for (uint32_t c = G::thread(); c < n; c += NT) *(Word4Any *)(out + head + c * E) = Word4{0, 0, 0, 0};
        if (at != 0xffffffffu) out[at] = (T)0.0f;
    }
};

// ---- log-probabilities at given classes ------------------------------------------------------------------

// Bound by reading: 2048 x 32768 in bf16 25.6 us, 5.3 TB/s.
template <class T, int NT, int NV>
__global__ void __launch_bounds__(Group<NT>::SIZE) k_logprobs_at(Rows in, const int32_t *index, uint32_t k, float *out)
{
    using G = Group<NT>;
    __shared__ Stats buf[G::WAVES];
    const uint64_t r = in.first + (uint64_t)blockIdx.x * G::ROWS + G::row_in_group();
    if (r >= in.rows) return;                       // NT > 64: the whole workgroup
    int32_t at[G::SLOTS];
#pragma unroll
    for (int i = 0; i < G::SLOTS; ++i) {
        const uint32_t j = i * NT + G::thread();
        at[i] = j < k ? index[r * k + j] : -1;
    }
    Row<T, NT, NV> row;
    row.place((const T *)in.z + r * in.stride, in.classes);
    row.load();
    float x[G::SLOTS], mine;
#pragma unroll
    for (int i = 0; i < G::SLOTS; ++i) x[i] = (uint32_t)at[i] < in.classes ? to_float(row.z[at[i]]) : 0.0f;
    Stats st = row.stats(LOG2E, mine);
    G::put(st, buf);
    G::sync();
    st = G::get(st, buf, LOG2E);
    const float log_s = __logf(st.s);
#pragma unroll
    for (int i = 0; i < G::SLOTS; ++i) {
        const uint32_t j = i * NT + G::thread();
        float lp = 0;
        if ((uint32_t)at[i] < in.classes) lp = x[i] == neg_inf() && st.s == st.s ? neg_inf() : (x[i] - st.m) - log_s;
        if (j < k) out[r * k + j] = lp;
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

// Order and position in one key: of equal values the lower class is the larger key, no two keys of a row are alike, and 0 is
// less than any.  Short rows of 16-bit types have room for both in 32 bits.
template <class T, class Key> struct Keys {
    static __device__ Key of(float x, uint32_t v) { return (Key)order_of(x) << 32 | (0xffffffffu - v); }
    static __device__ float value(Key k) { return value_of((uint32_t)(k >> 32)); }
    static __device__ int32_t position(Key k) { return (int32_t)(0xffffffffu - (uint32_t)k); }
};
template <class T> struct Keys<T, uint32_t> {
    static __device__ uint32_t of(float x, uint32_t v)
    {
        const uint32_t h = __builtin_bit_cast(uint16_t, (T)(x + 0.0f));
        return (h & 0x8000u ? ~h & 0xffffu : h | 0x8000u) << 16 | (0xffffu - v);
    }
    static __device__ float value(uint32_t k)
    {
        const uint32_t o = k >> 16;
        return to_float(__builtin_bit_cast(T, (uint16_t)(o & 0x8000u ? o & 0x7fffu : ~o)));
    }
    static __device__ int32_t position(uint32_t k) { return (int32_t)(0xffffu - (k & 0xffffu)); }
};

// A number t that at least `count` of the keys reach, and none but equal ones more, among the keys of the group's lanes of a
// wavefront (N keys to a lane); 0 if there are not as many keys above 0.  Bit by bit from the top, of the given leading bits:
// the bits below are 0, also where those of a negative value are ones.
template <int NT, int BITS, int N> __device__ inline uint32_t nth_largest(const uint32_t *keys, uint32_t count)
{
    uint32_t t = 0;
#pragma unroll 1
    for (uint32_t bit = 0x80000000u; bit >= (1u << (32 - BITS)) && bit; bit >>= 1) {
        uint32_t above = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool yes = keys[i] >= (t | bit);
            above += NT >= 64 ? (uint32_t)__popcll(__ballot(yes)) : yes;
        }
        if (NT < 64) above = across<Add, Group<NT>::LANES>(above);
        if (above >= count) t |= bit;
        if (above == count) break;
    }
    return t;
}

// bits of order_of that tell the values of a type apart
template <class T> struct OrderBits { static constexpr int N = 32; };
template <> struct OrderBits<__bf16> { static constexpr int N = 16; };
template <> struct OrderBits<_Float16> { static constexpr int N = 19; };

constexpr uint32_t CANDIDATES = 1024;

// The keys of a row's elements that equal `value`, from the lowest position on, to best[have] and on until there are k; returns
// how many there are then.  One turn of the threads after the other, the elements before the words first and those behind
// them last: most rows of many equal values end with the first words.
template <class T, int NT, class R, class Key> __device__ uint32_t equal_in_order(const R &row, float value, uint32_t have, uint32_t k, Key *best)
{
    using P = Pack<T>;
    __shared__ uint32_t totals[Group<NT>::WAVES];
    const uint32_t turns = (row.n + NT - 1) / NT;
#pragma unroll 1
    for (uint32_t turn = 0; turn < turns + 2 && have < k; ++turn) {
        float x[P::E];
        uint32_t at = 0, equal = 0;
#pragma unroll
        for (int e = 0; e < P::E; ++e) x[e] = neg_inf();
        if (turn == 0 || turn == turns + 1) {
            if (row.at != 0xffffffffu && (row.at < row.head) == (turn == 0)) {
                at = row.at;
                x[0] = row.edge;
            }
        } else {
            const uint32_t c = (turn - 1) * NT + threadIdx.x;
            at = row.head + c * P::E;
            if (c < row.n) P::open(row.words[c], x);
        }
#pragma unroll
        for (int e = 0; e < P::E; ++e) equal += x[e] == value;
        uint32_t before = equal;
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t other = __shfl_up(before, d);
            if ((int)(threadIdx.x & 63) >= d) before += other;
        }
        if ((threadIdx.x & 63) == 63) totals[threadIdx.x >> 6] = before;
        __syncthreads();
        uint32_t all = 0;
        before -= equal;
        for (uint32_t w = 0; w < Group<NT>::WAVES; ++w) {
            if (w < threadIdx.x >> 6) before += totals[w];
            all += totals[w];
        }
        before += have;
#pragma unroll
        for (int e = 0; e < P::E; ++e)
            if (x[e] == value && before < k) best[before++] = Keys<T, Key>::of(x[e], at + e);
        have += all;
        __syncthreads();
    }
    return have < k ? have : k;
}

// The k-th largest key digit by digit from the top: the counts of the next eight bits among the keys that agree with the
// digits chosen so far. For rows with more candidates than LDS has room for.
template <class T, int NT, class R> __device__ uint64_t least_by_digits(R &row, uint32_t k, uint32_t *count)
{
    __shared__ uint64_t least;
    __shared__ uint32_t need, done;
    if (threadIdx.x == 0) {
        least = 0;
        need = k;
        done = 0;
    }
#pragma unroll 1
    for (int shift = 56; shift >= 0; shift -= 8) {
        if (threadIdx.x < 256) count[threadIdx.x] = 0;
        __syncthreads();
        if (done) break;
        const uint64_t prefix = least;
        row.elements_again([&](float x, uint32_t v) {
            const uint64_t key = Keys<T, uint64_t>::of(x, v);
            if ((key >> 32) && (shift == 56 || (key >> (shift + 8)) == (prefix >> (shift + 8))))
                atomicAdd(&count[(key >> shift) & 255], 1u);
        });
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
    return least;
}

// The same within a wavefront: the k-th largest value, and among those equal to it the position of the last to be chosen, bit by
// bit with ballots. Stores the k best keys (all, if there are fewer) and returns their number.
template <class T, int NT, int NV, int BITS, class R, class Key> __device__ uint32_t best_of_many(R &row, uint32_t k, Key *best)
{
    using P = Pack<T>;
    constexpr uint32_t MASK = ~(uint32_t)(0xffffffffull >> BITS);
    auto count = [&](auto f) {
        uint32_t n = 0;
        row.each([&](Word4 w) {
            float x[P::E];
            P::open(w, x);
#pragma unroll
            for (int e = 0; e < P::E; ++e) n += (uint32_t)__popcll(__ballot(f(x[e], e)));
        });
        return n + (uint32_t)__popcll(__ballot(f(row.edge, P::E)));
    };
    uint32_t t = 0;
#pragma unroll 1
    for (uint32_t bit = 0x80000000u; bit & MASK; bit >>= 1)
        if (count([&](float x, int) { return order_of(x) >= (t | bit); }) >= k) t |= bit;
    // equal ones from the lowest position on: up to which
    const uint32_t left = k - count([&](float x, int) { return (order_of(x) & MASK) > t; });
    uint32_t low = 0, high = 0xffffffffu;
#pragma unroll 1
    while (t && low < high) {
        const uint32_t mid = low + (high - low) / 2;
        uint32_t n = 0;
        row.each_at([&](Word4 w, uint32_t v) {
            float x[P::E];
            P::open(w, x);
#pragma unroll
            for (int e = 0; e < P::E; ++e) n += (order_of(x[e]) & MASK) == t && v + e <= mid;
        });
        n += row.at != 0xffffffffu && (order_of(row.edge) & MASK) == t && row.at <= mid;
        if (across<Add, 64>(n) >= left) high = mid;
        else low = mid + 1;
    }
    uint32_t n = 0;
    const uint64_t below = (1ull << (threadIdx.x & 63)) - 1;
    auto keep = [&](float x, uint32_t v, bool has) {
        const uint32_t o = order_of(x) & MASK;
        const bool yes = has && order_of(x) && (o > t || (o == t && v <= high));
        const uint64_t b = __ballot(yes);
        if (yes) best[n + __popcll(b & below)] = Keys<T, Key>::of(x, v);
        n += (uint32_t)__popcll(b);
    };
#pragma unroll 1
    for (uint32_t c = 0; c < row.n; c += NT) {
        const bool has = c + (threadIdx.x & 63) < row.n;
        float x[P::E];
        P::open(has ? row.words[c + (threadIdx.x & 63)] : Word4{P::NONE, P::NONE, P::NONE, P::NONE}, x);
#pragma unroll
        for (int e = 0; e < P::E; ++e) keep(x[e], row.head + (c + (threadIdx.x & 63)) * P::E + e, has);
    }
    keep(row.edge, row.at, row.at != 0xffffffffu);
    Group<NT>::sync();
    return n;
}

// Two rounds over a row in registers.  The first gives the maximum of every thread; the `each`-th largest of a wavefront's
// maxima, the least of them over the wavefronts, is a bound that at least k elements reach.  (Few words or many slots: the
// bound comes from the elements themselves.)  The second collects what reaches it, usually little more than k, in LDS, where
// every candidate counts the larger ones: that is its place.  64 of 4096 x 131072 in bf16: 252 us, 4.3 TB/s (185 without the
// second round); vector ALU three quarters busy.  5 of 65536 x 100 in f16: 12 us, bound by its instructions.  (Four lanes to a
// candidate: 261 us; the next row's words requested as this row's are looked through: 302, the compiler keeps both.)
template <class T, int NT, int NV> __device__ __forceinline__ void top_of_row(const Rows &in, uint32_t k, int32_t *index, float *out)
{
    using G = Group<NT>;
    using P = Pack<T>;
    // rows of at most NT * NV * E elements where NT is not the most
    using Key = std::conditional_t<NT <= 64 && sizeof(T) == 2, uint32_t, uint64_t>;
    using K = Keys<T, Key>;
    constexpr int BITS = OrderBits<T>::N, ROOM = NT > 64 ? CANDIDATES : NT * NV * P::E < 1024 ? NT * NV * P::E : NV > 4 ? 512 : 1024;
    __shared__ Stats buf[G::WAVES];
    __shared__ uint32_t bounds[G::WAVES], found[G::ROWS], words;
    __shared__ __align__(16) Key best[G::ROWS][ROOM];
    const uint32_t group = G::row_in_group();
    const uint64_t r = in.first + (uint64_t)blockIdx.x * G::ROWS + group;
    if (r >= in.rows) return;                       // NT > 64: the whole workgroup
    Row<T, NT, NV> row;
    row.place((const T *)in.z + r * in.stride, in.classes);
    row.load();
    if (G::thread() == 0) found[group] = 0;
    if (threadIdx.x == 0) words = 0;
    float mine;
    Stats st = row.stats(LOG2E, mine);
    // wavefronts that have a word for every lane, or the only one
    const uint32_t full = NT <= 64 ? 1 : row.n / 64 < G::WAVES ? row.n / 64 : G::WAVES, each = (k + full - 1) / full;
    const uint32_t maxima = row.n < NT ? row.n : NT;
    uint32_t bound;
    if (NT == 16 && (in.classes <= 16 || (in.classes <= 48 && k > maxima))) {
        bound = 0;                                  // all of them: fewer comparisons than a search
    } else if (NV <= 4 && k > (NT < 64 ? maxima : maxima / 2)) {
        uint32_t keys[NV * P::E + 1];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float x[P::E];
            P::open(row.fresh(i), x);
#pragma unroll
            for (int e = 0; e < P::E; ++e) keys[i * P::E + e] = order_of(x[e]);
        }
        keys[NV * P::E] = order_of(row.edge);
        bound = nth_largest<NT, BITS, NV * P::E + 1>(keys, each);
    } else {
        const uint32_t key = order_of(mine);
        // of 16 maxima all that fewer than k exceed; 0 if there are not as many
        if constexpr (NT == 16) bound = across<Min, 16>(larger_of_16(key) < k ? key : 0xffffffffu);
        else bound = nth_largest<NT, BITS, 1>(&key, each);
    }
    G::put(st, buf);
    if (NT > 64 && (threadIdx.x & 63) == 0) bounds[G::wave()] = G::wave() < full ? bound : 0xffffffffu;
    G::sync();
    st = G::get(st, buf, LOG2E);
    if (NT > 64) {
        bound = bounds[0];
        for (int i = 1; i < G::WAVES; ++i) bound = bounds[i] < bound ? bounds[i] : bound;
    }
    const float log_s = __logf(st.s), m = st.m;
    // the least finite value leaves out -inf and NaN
    float least = bound ? value_of(bound) : -3.402823466e38f;
    auto keep = [&](float x, uint32_t v) {
        if (x >= least) {
            const uint32_t i = atomicAdd(&found[group], 1u);
            if (i < ROOM) best[group][i] = K::of(x, v);
        }
    };
    if (NT != 16 && row.at != 0xffffffffu) keep(row.edge, row.at);
    // A row with a NaN has a sum of NaN: there every word reaches, as max3 may lose what stands next to a signalling one.
    const float border = st.s == st.s ? least : neg_inf();
    auto reaches = [&](const float *x) {
        float most = x[0];
#pragma unroll
        for (int i = 1; i + 1 < P::E; i += 2) most = max3(most, x[i], x[i + 1]);
        return !(max3(most, x[P::E - 1], most) < border);
    };
    uint32_t taken = 0;
    if constexpr (NT == 16) {
        // every lane's places follow from the counts of the lanes before: no atomics, one after the other, for so few
        uint64_t mine = (uint64_t)(row.edge >= least) << NV * P::E;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float x[P::E];
            P::open(row.fresh(i), x);
#pragma unroll
            for (int e = 0; e < P::E; ++e) mine |= (uint64_t)(x[e] >= least) << (i * P::E + e);
        }
        const uint32_t count = (uint32_t)__popcll(mine);
        uint32_t at = before_in_16(count);
        taken = across<Add, 16>(count);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float x[P::E];
            P::open(row.fresh(i), x);
#pragma unroll
            for (int e = 0; e < P::E; ++e)
                if (mine >> (i * P::E + e) & 1) best[group][at++] = K::of(x[e], row.head + (i * NT + G::thread()) * P::E + e);
        }
        if (mine >> NV * P::E) best[group][at] = K::of(row.edge, row.at);
    } else if constexpr (NV <= 4 || NT <= 64) {
        row.each_at([&](Word4 w, uint32_t v) {
            float x[P::E];
            P::open(w, x);
            if (reaches(x))
#pragma unroll
                for (int i = 0; i < P::E; ++i) keep(x[i], v + i);
        });
    } else {
        // whole words first, their elements then one to a thread: a body of all elements of all words would not fit the
        // instruction cache
        __shared__ Word4 word[CANDIDATES];
        __shared__ uint32_t where[CANDIDATES];
        row.each_at([&](Word4 w, uint32_t v) {
            float x[P::E];
            P::open(w, x);
            if (reaches(x)) {
                const uint32_t i = atomicAdd(&words, 1u);
                if (i < CANDIDATES) {
                    word[i] = w;
                    where[i] = v;
                }
            }
        });
        __syncthreads();
        const uint32_t all = words;
        if (all <= CANDIDATES) {
            for (uint32_t i = threadIdx.x; i < all * P::E; i += NT)
                keep(to_float(((const T *)word)[i]), where[i / P::E] + i % P::E);
        } else if (threadIdx.x == 0) {
            found[0] = ROOM + 1;
        }
    }
    G::sync();
    uint32_t n = NT == 16 ? taken : found[group];
    if constexpr (NT <= 64 && NT * NV * P::E > ROOM) {
        if (n > ROOM) n = best_of_many<T, NT, NV, BITS>(row, k, best[group]);
    }
    if (NT > 64 && n > ROOM) {
        // Many equal to the bound, as in a row of few values (1024 x 131072 in bf16, zeros 123 us, -7 123; by digits 3240)?  What
        // exceeds it, and of the equal ones the first.  The bound has to be a value of the row for that: it lies below those that
        // it was made from where they are negative and of 16 bits, or where the search for it ended early.
        __syncthreads();
        if (threadIdx.x == 0) found[0] = 0;
        if (bound) {
            uint32_t low = 0xffffffffu;
            const auto lower = [&](float x) {
                if (order_of(x) >= bound) low = Min::of(low, order_of(x));
            };
            if constexpr (NV <= 4) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    float x[P::E];
                    P::open(row.fresh(i), x);
#pragma unroll
                    for (int e = 0; e < P::E; ++e) lower(x[e]);
                }
                lower(row.edge);
            } else {
                lower(mine);
            }
            low = across<Min, 64>(low);
            if ((threadIdx.x & 63) == 0) bounds[G::wave()] = low;
            __syncthreads();
            for (int i = 0; i < G::WAVES; ++i) low = Min::of(low, bounds[i]);
            least = value_of(low);
        }
        __syncthreads();
        row.elements_again([&](float x, uint32_t v) {
            if (x > least) {
                const uint32_t i = atomicAdd(&found[0], 1u);
                if (i < ROOM) best[0][i] = K::of(x, v);
            }
        });
        __syncthreads();
        n = found[0];
        if (n < k) n = equal_in_order<T, NT>(row, least, n, k, best[0]);
    }
    if (NT > 64 && n > ROOM) {
        __shared__ uint32_t count[256];
        const uint64_t last = least_by_digits<T, NT>(row, k, count);
        if (threadIdx.x == 0) found[0] = 0;
        __syncthreads();
        row.elements_again([&](float x, uint32_t v) {
            const uint64_t key = Keys<T, uint64_t>::of(x, v);
            if ((key >> 32) && key >= last) best[0][atomicAdd(&found[0], 1u)] = (Key)key;
        });
        __syncthreads();
        n = found[0];
    }
    auto put = [&](Key key, uint32_t place) {
        if (place >= k) return;
        index[r * k + place] = K::position(key);
        out[r * k + place] = (K::value(key) - m) - log_s;
    };
    if (NT == 16 && n <= 16) {
        const Key key = G::thread() < n ? best[group][G::thread()] : 0;
        const uint32_t place = larger_of_16(key);
        if (G::thread() < n) put(key, place);
    } else {
        for (uint32_t i = G::thread(); i < n; i += NT) {
            const Key key = best[group][i];
            uint32_t place = 0;
            for (uint32_t j = 0; j < n; ++j) place += best[group][j] > key;
            put(key, place);
        }
    }
    for (uint32_t i = n + G::thread(); i < k; i += NT) {
        index[r * k + i] = -1;
        out[r * k + i] = 0;
    }
}

template <class T, int NT, int NV>
__global__ void __launch_bounds__(Group<NT>::SIZE) k_top(Rows in, uint32_t k, int32_t *index, float *out)
{
    top_of_row<T, NT, NV>(in, k, index, out);
}

// 512 and 1024 threads of up to 8 words: with no more than 64 vector and 80 scalar registers to a wavefront a SIMD holds eight of
// them, two rows of up to 8192 words to a unit.  The vector registers come out so by themselves (float16 with 512 threads takes 70:
// seven wavefronts), the scalar ones are capped (64 of 2048 x 65536 in bf16 with 93 of them: 84 us instead of 64).  1024
// threads of 16 words take 93 vector registers: one row to a unit.
template <class T, int NT, int NV>
__global__ void __launch_bounds__(NT) __attribute__((amdgpu_num_sgpr(80))) k_top_long(Rows in, uint32_t k, int32_t *index, float *out)
{
    top_of_row<T, NT, NV>(in, k, index, out);
}

// ---- distillation ----------------------------------------------------------------------------------------

// What a row's threads have to know of each other's slots.
template <int NT> struct Taught {
    using G = Group<NT>;
    static constexpr uint32_t PLACES = 2 * G::TOP;
    int32_t v[G::ROWS][G::TOP];
    float u[G::ROWS][G::TOP];
    int32_t place[G::ROWS][PLACES];
    uint32_t twice[G::ROWS];
    Stats stats[G::WAVES];
    float loss[G::WAVES];

    __device__ void clear(uint32_t group)
    {
        for (uint32_t i = G::thread(); i < PLACES; i += NT) place[group][i] = -1;
        if (G::thread() == 0) twice[group] = 0;
    }
};

// The teacher's slots j of a row, slot j with thread j % NT: class (-1: empty) and sum of answers t, and their softmax:
// u = exp((t - m) * share) for the largest t of the wavefront, later of the row.  The difference comes before the product: a sum
// by itself, lowest values among them, may leave the range when it is divided by a temperature below 1.
template <int NT> struct Slots {
    using G = Group<NT>;
    int32_t v[G::SLOTS];
    float t[G::SLOTS], u[G::SLOTS];
    bool own[G::SLOTS];     // the class is in these threads' part of the row
    Stats st;

    __device__ void load(const Answers &a, uint64_t r, uint32_t classes)
    {
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i) {
            const uint32_t j = i * NT + G::thread();
            v[i] = -1;
            t[i] = neg_inf();
            if (j < a.k) {
                const int32_t c = a.index[r * a.k + j];
                const float s = a.sum[r * a.k + j];
                if ((uint32_t)c < classes && s != neg_inf()) {
                    v[i] = c;
                    t[i] = s;
                }
            }
            own[i] = v[i] >= 0;
        }
    }
    // u and its sum within the wavefront; and whether a class comes twice: of two slots of a class one finds the other in a
    // table of twice as many places as slots.  (All slots going through all others: 90 us instead of 63 for gradients of
    // 512 x 65537 with 250 slots, 527 instead of 471 for a step of 4096 x 131072 with 128.)
    __device__ void weigh(float share, Taught<NT> &lds, uint32_t group)
    {
        float m = neg_inf(), sum = 0;
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i) m = fmaxf(m, t[i]);
        m = across<Max, G::LANES>(m);
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i) {
            u[i] = 0;
            if (v[i] < 0) continue;
            u[i] = __builtin_amdgcn_exp2f((t[i] - m) * (share * LOG2E));
            sum += u[i];
            if (!own[i]) continue;
            constexpr uint32_t LAST = Taught<NT>::PLACES - 1;
            uint32_t h = ((uint32_t)v[i] * 0x9e3779b1u) >> 16 & LAST;
            while (true) {                          // ends: half of the places stay free
                const int32_t there = atomicCAS(&lds.place[group][h], -1, v[i]);
                if (there == v[i]) lds.twice[group] = 1;
                if (there < 0 || there == v[i]) break;
                h = (h + 1) & LAST;
            }
        }
        st = {m, across<Add, G::LANES>(sum)};
        G::put(st, lds.stats);
    }
    // After a barrier: u and its sum for the row.
    __device__ void join(uint32_t k, float share, Taught<NT> &lds, uint32_t group)
    {
        const Stats all = G::get(st, lds.stats, share * LOG2E);
        const float f = all.m == st.m ? 1.0f : __builtin_amdgcn_exp2f((st.m - all.m) * (share * LOG2E));
        st = all;
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i) {
            if (NT > 64) u[i] = v[i] >= 0 ? u[i] * f : 0.0f;
            const uint32_t j = i * NT + G::thread();
            if (j < k) {
                lds.v[group][j] = v[i];
                lds.u[group][j] = u[i];
            }
        }
    }
    // sum_j p_j (log p_j - (z_j / T - lse)) = A / U - log U + log S with the sum A of u_j ((t_j - m) * share - (z_j - m_z) / T); A
    // by wavefronts
    __device__ void part_of_loss(const float *x, Stats z, const Answers &a, Taught<NT> &lds)
    {
        float sum = 0;
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i)
            if (u[i] != 0.0f) sum += u[i] * ((t[i] - st.m) * a.share - (x[i] - z.m) * a.inv_t);
        sum = across<Add, G::LANES>(sum);
        if (NT <= 64) st.m = sum;
        else if ((threadIdx.x & 63) == 0) lds.loss[G::wave()] = sum;
    }
    // After a barrier
    __device__ float loss(Stats z, const Taught<NT> &lds) const
    {
        float sum = st.m;
        if (NT > 64) {
            sum = 0;
            for (uint32_t i = 0; i < (G::WAVES < 4 ? G::WAVES : 4); ++i) sum += lds.loss[i];      // 256 slots
        }
        return sum / st.s - __logf(st.s) + __logf(z.s);
    }
    // The u of slot i, or where classes come twice those of all slots of its class, added up in slot order: each of them is
    // stored with the same value.
    __device__ float of_class(int i, uint32_t k, const Taught<NT> &lds, uint32_t group) const
    {
        if (!lds.twice[group]) return u[i];
        float p = 0;
        for (uint32_t j = 0; j < k; ++j) p += lds.v[group][j] == v[i] ? lds.u[group][j] : 0.0f;
        return p;
    }
};

// A row that stays in registers between its statistics and its gradient.  4096 x 131072 in bf16: 435 us, 4.9 TB/s (read
// several times, 256 threads to a row: 1867); 2048 x 32768: 54.6 us; the loss alone of 777 x 50001 in f16: 18.1 us, 4.0
// TB/s on 777 workgroups of 512 places.  With 512 threads and 32 words each for the longest rows: 515 us.
template <class T, int NT, int NV, bool GRAD>
__global__ void __launch_bounds__(Group<NT>::SIZE) k_distill(Rows in, Answers a, float *loss, float *lse, T *grad, uint64_t grad_stride)
{
    using G = Group<NT>;
    __shared__ Stats buf[G::WAVES];
    __shared__ Taught<NT> taught;
    const uint32_t group = G::row_in_group();
    const uint64_t r = in.first + (uint64_t)blockIdx.x * G::ROWS + group;
    if (r >= in.rows) return;                       // NT > 64: the whole workgroup
    const float w = a.weight ? a.weight[r] : 1.0f, scale = a.inv_t * LOG2E;
    T *out = GRAD ? grad + r * grad_stride : nullptr;
    Slots<NT> slots;
    Row<T, NT, NV> row;
    slots.load(a, r, in.classes);
    row.place((const T *)in.z + r * in.stride, in.classes);
    // Padding is not read, where reading takes longer than waiting for the weight.
    if (NT > 64 && w == 0.0f) {
        if (threadIdx.x == 0) loss[r] = lse[r] = 0;
        if (GRAD) row.clear(out);
        return;
    }
    row.load();
    float x[G::SLOTS], mine;
#pragma unroll
    for (int i = 0; i < G::SLOTS; ++i) x[i] = slots.v[i] >= 0 ? to_float(row.z[slots.v[i]]) : 0.0f;
    taught.clear(group);
    G::sync();
    slots.weigh(a.share, taught, group);
    Stats st = row.stats(scale, mine);
    G::put(st, buf);
    G::sync();
    st = G::get(st, buf, scale);
    slots.join(a.k, a.share, taught, group);
    // neither a weight nor a filled slot, or all logits -inf
    const bool none = w == 0.0f || slots.st.s == 0.0f, excluded = !none && st.s == 0.0f;
    if (none || excluded) {
        if (G::thread() == 0) {
            loss[r] = 0;
            lse[r] = none ? 0.0f : neg_inf();
        }
        if (GRAD) row.clear(out);
        return;
    }
    const float g = w * a.inv_t, gs = g / st.s, gu = g / slots.st.s;
    slots.part_of_loss(x, st, a, taught);
    if (GRAD) row.store(out, st.m, scale, gs);
    G::sync();
    if (G::thread() == 0) {
        loss[r] = w * slots.loss(st, taught);
        lse[r] = st.m * a.inv_t + __logf(st.s);
    }
    // the teacher's classes, over the dense part
    if (GRAD)
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i)
            if (slots.v[i] >= 0)
                out[slots.v[i]] = (T)(__builtin_amdgcn_exp2f((x[i] - st.m) * scale) * gs - slots.of_class(i, a.k, taught, group) * gu);
}

// Long rows of which there are few are cut into parts of `per` words, a workgroup of 256 to each: 16 x 131072 in f32 take two
// launches of 3.4 and 5.4 us instead of one of 22, as a unit by itself moves some 50 bytes a nanosecond.
struct Parts {
    uint32_t count, per;
    Stats *stats;           // [rows][count]
};

template <class T, int NV> __global__ void __launch_bounds__(256) k_part_stats(Rows in, Parts parts, float scale)
{
    using G = Group<256>;
    __shared__ Stats buf[G::WAVES];
    const uint64_t r = blockIdx.x / parts.count;
    const uint32_t part = blockIdx.x % parts.count;
    Row<T, 256, NV> row;
    row.place((const T *)in.z + r * in.stride, in.classes, part * parts.per, parts.per);
    row.load();
    float mine;
    Stats st = row.stats(scale, mine);
    G::put(st, buf);
    G::sync();
    st = G::get(st, buf, scale);
    if (threadIdx.x == 0) parts.stats[blockIdx.x] = st;
}

// A row's parts, at most 256, to a wavefront's statistics: one part to a thread of a workgroup of 256.
__device__ inline Stats load_parts(const Parts &parts, uint64_t r)
{
    return threadIdx.x < parts.count ? parts.stats[r * parts.count + threadIdx.x] : Stats{neg_inf(), 0.0f};
}

// An lse from here on has a rounding of 2^-9 or more: exp(z / T - lse) would be off by as much, and by a factor of the number of
// classes in a row of nothing but the lowest value of 32 bits, whose lse has no bits left for log V.
constexpr float FAR_LSE = 32768.0f;

// Statistics of a whole row, read from memory by its group of threads, once per part: for what hardly ever runs (512 x 65537 in
// f32, 17 parts to a row, 804 us where all rows are such, 63 where none is).
template <class T, int NT> __device__ Stats stats_again(const T *z, uint32_t classes, float scale, Stats *buf)
{
    using G = Group<NT>;
    float m = neg_inf(), s = 0;
#pragma unroll 1
    for (uint32_t v = G::thread(); v < classes; v += NT) m = fmaxf(m, to_float(z[v]));
    m = across<Max, G::LANES>(m);
    if (m != neg_inf())
#pragma unroll 1
        for (uint32_t v = G::thread(); v < classes; v += NT) s += __builtin_amdgcn_exp2f((to_float(z[v]) - m) * scale);
    const Stats st = {m, across<Add, G::LANES>(s)};
    G::put(st, buf);
    G::sync();
    return G::get(st, buf, scale);
}

// The gradient of a part of a row, or with NT < 256 of a whole one, from its statistics: the lse of an earlier call, or with
// SPLIT the sums of its parts, where part 0 writes loss and lse as well.  Every part weighs the teacher's slots by itself, and
// fetches and stores those whose class it has (all parts fetching all: 63.8 us instead of 55 for 512 x 65537 in f32 with 250
// slots, 4.9 TB/s).  16384 x 1000 in bf16: 12.9 us, 5.1 TB/s.
template <class T, int NT, int NV, bool SPLIT, bool GRAD>
__global__ void __launch_bounds__(Group<NT>::SIZE)
k_gradient(Rows in, Answers a, Parts parts, float *loss, float *lse, T *grad, uint64_t grad_stride)
{
    using G = Group<NT>;
    using P = Pack<T>;
    __shared__ Stats buf[G::WAVES];
    __shared__ Taught<NT> taught;
    const uint32_t group = G::row_in_group(), count = GRAD ? parts.count : 1;
    const uint32_t part = NT < 256 ? 0 : blockIdx.x % count;
    const uint64_t r = in.first + (NT < 256 ? (uint64_t)blockIdx.x * G::ROWS + group : blockIdx.x / count);
    if (r >= in.rows) return;                       // NT > 64: the whole workgroup
    const float w = a.weight ? a.weight[r] : 1.0f, scale = a.inv_t * LOG2E, l = SPLIT ? 0.0f : lse[r];
    T *out = GRAD ? grad + r * grad_stride : nullptr;
    const T *z = (const T *)in.z + r * in.stride;
    Slots<NT> slots;
    Row<T, NT, NV> row;
    Stats st = {0.0f, 1.0f};
    slots.load(a, r, in.classes);
    if (SPLIT) st = load_parts(parts, r);
    if (GRAD) {
        row.place(z, in.classes, part * parts.per, parts.per);
        row.load();
    }
    // part 0 has the edges too: all classes before its words, and those behind the last part's
    const uint32_t end = row.head + row.n * P::E, words_end = in.classes - (in.classes - row.head) % P::E;
    float x[G::SLOTS];
#pragma unroll
    for (int i = 0; i < G::SLOTS; ++i) {
        const uint32_t v = slots.v[i];
        const bool filled = slots.v[i] >= 0;
        if (GRAD) slots.own[i] = filled && ((v >= row.head && v < end) || (part == 0 && (v < row.head || v >= words_end)));
        x[i] = slots.own[i] || (SPLIT && part == 0 && filled) ? to_float(z[v]) : 0.0f;
    }
    taught.clear(group);
    G::sync();
    slots.weigh(a.share, taught, group);
    if (SPLIT) {
        st = st.together<G::LANES>(scale);
        G::put(st, buf);
    }
    G::sync();
    if (SPLIT) st = G::get(st, buf, scale);
    slots.join(a.k, a.share, taught, group);
    const bool none = w == 0.0f || slots.st.s == 0.0f, far = !SPLIT && !none && fabsf(l) >= FAR_LSE;
    if (far) st = stats_again<T, NT>(z, in.classes, scale, buf);
    if (none || st.s == 0.0f) {
        if (SPLIT && part == 0 && threadIdx.x == 0) {
            loss[r] = 0;
            lse[r] = none ? 0.0f : neg_inf();
        }
        if (GRAD) row.clear(out);
        return;
    }
    const float g = w * a.inv_t, gs = g / st.s, gu = g / slots.st.s;
    // z / T is not rounded before lse is taken off
    auto student = [&](float z, bool by_stats) {
        return __builtin_amdgcn_exp2f(by_stats ? (z - st.m) * scale : __builtin_fmaf(z, a.inv_t, -l) * LOG2E) * gs;
    };
    if (SPLIT && part == 0) slots.part_of_loss(x, st, a, taught);
    if (GRAD) {
        auto store = [&](Word4 words, uint32_t v, bool by_stats) {
            float y[P::E];
            P::open(words, y);
#pragma unroll
            for (int i = 0; i < P::E; ++i) y[i] = student(y[i], by_stats);
            *(Word4Any *)(out + v) = P::close(y);
        };
        if (far) row.again_at([&](Word4 words, uint32_t v) { store(words, v, true); });
        else row.each_at([&](Word4 words, uint32_t v) { store(words, v, SPLIT); });
        if (row.at != 0xffffffffu) out[row.at] = (T)student(row.edge, SPLIT || far);
    }
    G::sync();
    if (SPLIT && part == 0 && threadIdx.x == 0) {
        loss[r] = w * slots.loss(st, taught);
        lse[r] = st.m * a.inv_t + __logf(st.s);
    }
    if (!GRAD) return;
#pragma unroll
    for (int i = 0; i < G::SLOTS; ++i)
        if (slots.own[i]) out[slots.v[i]] = (T)(student(x[i], SPLIT || far) - slots.of_class(i, a.k, taught, group) * gu);
}

// Log-probabilities of rows whose parts have been summed up.
template <class T> __global__ void __launch_bounds__(256) k_part_logprobs(Rows in, Parts parts, const int32_t *index, uint32_t k, float *out)
{
    using G = Group<256>;
    __shared__ Stats buf[G::WAVES];
    const uint64_t r = blockIdx.x;
    const uint32_t j = threadIdx.x;
    const int32_t at = j < k ? index[r * k + j] : -1;
    Stats st = load_parts(parts, r).together<64>(LOG2E);
    const bool filled = (uint32_t)at < in.classes;
    const float x = filled ? to_float(((const T *)in.z + r * in.stride)[at]) : 0.0f;
    G::put(st, buf);
    G::sync();
    st = G::get(st, buf, LOG2E);
    if (j < k) out[r * k + j] = !filled ? 0.0f : x == neg_inf() && st.s == st.s ? neg_inf() : (x - st.m) - __logf(st.s);
}

}  // namespace answers
}  // namespace d2
