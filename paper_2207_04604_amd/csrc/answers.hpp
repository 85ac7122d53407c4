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
    uint32_t first, rows, classes;      // the launch's rows: first .. rows - 1
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

// ---- 16 bytes of logits -----------------------------------------------------------------------------------

typedef uint32_t Word4 __attribute__((ext_vector_type(4)));
// any alignment of an element: the machine takes 16-byte accesses at odd addresses
typedef Word4 Word4Any __attribute__((aligned(2)));

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

// fmaxf without the quieting of signalling NaNs that it costs on values that come straight from memory
__device__ inline float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// ---- a row and the NT threads that work on it -------------------------------------------------------------

// A workgroup has 256 threads or NT, whichever is more; groups of up to a wavefront never meet a barrier.
template <int NT> struct Group {
    static constexpr int SIZE = NT < 256 ? 256 : NT, ROWS = SIZE / NT, WAVES = NT < 64 ? 1 : NT / 64;
    static constexpr int TOP = NT < 64 ? 64 : MAX_TOP, SLOTS = NT < TOP ? TOP / NT : 1;     // slots of a row, of a thread

    static __device__ uint32_t thread() { return threadIdx.x % NT; }
    static __device__ uint32_t row_in_group() { return threadIdx.x / NT; }
    static __device__ void sync()
    {
        if (NT > 64) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    // sums (or maxima) of N values over the group, to every thread; buf: WAVES * N floats that nobody reads any more
    template <class Op, int N> static __device__ void reduce(float *v, float *buf)
    {
#pragma unroll
        for (int d = (NT < 64 ? NT : 64) / 2; d; d >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = Op::of(v[i], __shfl_xor(v[i], d));
        if (NT > 64) {
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < N; ++i) buf[i * WAVES + (threadIdx.x >> 6)] = v[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float r = buf[i * WAVES];
#pragma unroll
                for (int k = 1; k < WAVES; ++k) r = Op::of(r, buf[i * WAVES + k]);
                v[i] = r;
            }
        }
    }
};

struct Max {
    static __device__ float of(float a, float b) { return fmaxf(a, b); }
};
struct Add {
    static __device__ float of(float a, float b) { return a + b; }
};

// The elements of a row: full 16-byte words from the first aligned address on, word c of the row with thread c % NT; the
// words 0 .. NV * NT - 1 stay in registers, any others are read again by every pass.  What lies before and behind the
// full words (at most 2 (E - 1) elements) goes one to a thread: `edge`, -inf where a thread has none.
template <class T, int NT, int NV> struct Row {
    using P = Pack<T>;
    static constexpr int E = P::E;
    const T *z;
    const Word4 *words;
    uint32_t head, n, at;           // elements before the words; words; position of the edge element (none: 0xffffffff)
    float edge;
    Word4 held[NV];

    // `first`, `count`: the words to take of the row, with the edges if the first is among them
    __device__ void load(const T *row, uint32_t classes, uint32_t first = 0, uint32_t count = 0xffffffffu)
    {
        const uint32_t t = Group<NT>::thread();
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
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            held[i] = Word4{P::NONE, P::NONE, P::NONE, P::NONE};
            if ((uint32_t)i * NT < n) {
                const uint32_t c = i * NT + t;
                if (c < n) held[i] = words[c];
            }
        }
        edge = at != 0xffffffffu ? to_float(row[at]) : neg_inf();
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
        for (uint32_t c = NV * NT + Group<NT>::thread(); c < n; c += NT) f(words[c]);
    }
    // f(16 bytes, position of their first element): the words of this thread that the row has
    template <class F> __device__ void each_at(F f)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((uint32_t)i * NT < n) {
                const uint32_t c = i * NT + Group<NT>::thread();
                if (c < n) f(fresh(i), head + c * E);
            }
        for (uint32_t c = NV * NT + Group<NT>::thread(); c < n; c += NT) f(words[c], head + c * E);
    }
    // f(element, its position): all words once more from memory
    template <class F> __device__ void elements_again(F f) const
    {
#pragma unroll 1
        for (uint32_t c = Group<NT>::thread(); c < n; c += NT) {
            float x[E];
            P::open(words[c], x);
#pragma unroll
            for (int i = 0; i < E; ++i) f(x[i], head + c * E + i);
        }
        if (at != 0xffffffffu) f(edge, at);
    }
    __device__ float max()
    {
        float m = edge;
        each([&](Word4 w) {
            float x[E];
            P::open(w, x);
#pragma unroll
            for (int i = 0; i < E; i += 2) m = max3(m, x[i], x[i + 1]);
        });
        return m;
    }
    // sum exp2((x - base) * scale).  The difference is rounded before the product, so that a row of the type's lowest value
    // gives 0 and not inf - inf.
    __device__ float sum(float base, float scale)
    {
        float s = __builtin_amdgcn_exp2f((edge - base) * scale);
        each([&](Word4 w) {
            float x[E], part = 0;
            P::open(w, x);
#pragma unroll
            for (int i = 0; i < E; ++i) part += __builtin_amdgcn_exp2f((x[i] - base) * scale);
            s += part;
        });
        return s;
    }
};

// ---- log-probabilities at given classes ------------------------------------------------------------------

template <class T, int NT, int NV>
__global__ void __launch_bounds__(Group<NT>::SIZE) k_logprobs_at(Rows in, const int32_t *index, uint32_t k, float *out)
{
    using G = Group<NT>;
    __shared__ float buf[2][G::WAVES];
    const uint64_t r = in.first + (uint64_t)blockIdx.x * G::ROWS + G::row_in_group();
    if (r >= in.rows) return;                       // NT > 64: the whole workgroup
    int32_t at[G::SLOTS];
#pragma unroll
    for (int i = 0; i < G::SLOTS; ++i) {
        const uint32_t j = i * NT + G::thread();
        at[i] = j < k ? index[r * k + j] : -1;
    }
    Row<T, NT, NV> row;
    row.load((const T *)in.z + r * in.stride, in.classes);
    float x[G::SLOTS];
#pragma unroll
    for (int i = 0; i < G::SLOTS; ++i) x[i] = (uint32_t)at[i] < in.classes ? to_float(row.z[at[i]]) : 0.0f;
    float m = row.max();
    G::template reduce<Max, 1>(&m, buf[0]);
    float s = row.sum(m == neg_inf() ? 0.0f : m, LOG2E);
    G::template reduce<Add, 1>(&s, buf[1]);
    const float log_s = __logf(s);
#pragma unroll
    for (int i = 0; i < G::SLOTS; ++i) {
        const uint32_t j = i * NT + G::thread();
        float lp = 0;
        if ((uint32_t)at[i] < in.classes) lp = x[i] == neg_inf() && s == s ? neg_inf() : (x[i] - m) - log_s;
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

// order and position in one key: of equal values the lower class is the larger key; no two keys of a row are alike
__device__ inline uint64_t key_of(float x, uint32_t v) { return (uint64_t)order_of(x) << 32 | (0xffffffffu - v); }

// The largest number t of the given leading bits with ballots for `count` of the keys at or above it, among the keys of all
// threads of the group's wavefront (N keys to a thread); 0 if there are not as many keys above 0.
template <int NT, int BITS, int N> __device__ inline uint32_t nth_largest(const uint32_t *keys, uint32_t count)
{
    uint32_t t = 0;
#pragma unroll 1
    for (uint32_t bit = 0x80000000u; bit >= (1u << (32 - BITS)) && bit; bit >>= 1) {
        uint32_t above = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t b = __ballot(keys[i] >= (t | bit));
            above += NT >= 64 ? (uint32_t)__popcll(b) : (uint32_t)__popc((uint32_t)(b >> (threadIdx.x & 63 & ~(NT - 1))) & ((1u << (NT & 31)) - 1));
        }
        if (above >= count) t |= bit;
    }
    return t;
}

// bits of order_of that tell the values of a type apart
template <class T> struct OrderBits { static constexpr int N = 32; };
template <> struct OrderBits<__bf16> { static constexpr int N = 16; };
template <> struct OrderBits<_Float16> { static constexpr int N = 19; };

constexpr uint32_t CANDIDATES = 1024;

// The k-th largest key digit by digit from the top: the counts of the next eight bits among the keys that agree with the
// digits chosen so far. For rows with more candidates than LDS has room for, such as many equal values.
template <int NT, class R> __device__ uint64_t least_by_digits(R &row, uint32_t k, uint32_t *count)
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
            const uint64_t key = key_of(x, v);
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

// Two rounds over a row in registers.  The first gives the maximum of every thread; the `each`-th largest of a wavefront's
// maxima, the least of them over the wavefronts, is a bound that at least k elements reach.  (Few words or many slots: the
// bound comes from the elements themselves.)  The second collects what reaches it, usually little more than k, in LDS, where
// every candidate counts the larger ones: that is its place.
template <class T, int NT, int NV>
__global__ void __launch_bounds__(Group<NT>::SIZE) k_top(Rows in, uint32_t k, int32_t *index, float *out)
{
    using G = Group<NT>;
    using P = Pack<T>;
    constexpr int BITS = OrderBits<T>::N, ROOM = NT < 64 ? 128 : CANDIDATES;
    __shared__ float buf[2][G::WAVES];
    __shared__ uint32_t bounds[G::WAVES], found[G::ROWS], words;
    __shared__ __align__(16) uint64_t best[G::ROWS][ROOM];
    const uint32_t group = G::row_in_group(), wave = NT > 64 ? threadIdx.x >> 6 : 0;
    const uint64_t r = in.first + (uint64_t)blockIdx.x * G::ROWS + group;
    if (r >= in.rows) return;                       // NT > 64: the whole workgroup
    Row<T, NT, NV> row;
    row.load((const T *)in.z + r * in.stride, in.classes);
    const float mine = row.max();
    float m = mine;
    if (G::thread() == 0) found[group] = 0;
    if (threadIdx.x == 0) words = 0;
    G::template reduce<Max, 1>(&m, buf[0]);
    // wavefronts that have a word for every lane, or the only one
    const uint32_t full = NT <= 64 ? 1 : row.n / 64 < G::WAVES ? row.n / 64 : G::WAVES, each = (k + full - 1) / full;
    uint32_t bound;
    if (NV <= 4 && 4 * k > (row.n < NT ? row.n : NT)) {
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
        bound = nth_largest<NT, BITS, 1>(&key, each);
    }
    if (NT > 64) {
        if ((threadIdx.x & 63) == 0) bounds[wave] = wave < full ? bound : 0xffffffffu;
    }
    float s = row.sum(m == neg_inf() ? 0.0f : m, LOG2E);
    G::template reduce<Add, 1>(&s, buf[1]);
    if (NT > 64) {
        bound = bounds[0];
        for (int i = 1; i < G::WAVES; ++i) bound = bounds[i] < bound ? bounds[i] : bound;
    }
    const float log_s = __logf(s);
    // the least finite value leaves out -inf and NaN
    const float least = bound ? value_of(bound) : -3.402823466e38f;
    auto keep = [&](float x, uint32_t v) {
        if (x >= least) {
            const uint32_t i = atomicAdd(&found[group], 1u);
            if (i < ROOM) best[group][i] = key_of(x, v);
        }
    };
    if (row.at != 0xffffffffu) keep(row.edge, row.at);
    auto reaches = [&](const float *x) {
        float most = x[0];
#pragma unroll
        for (int i = 1; i + 1 < P::E; i += 2) most = max3(most, x[i], x[i + 1]);
        return max3(most, x[P::E - 1], most) >= least;
    };
    if constexpr (NV <= 4) {
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
    uint32_t n = found[group];
    if (NT > 64 && n > ROOM) {
        __shared__ uint32_t count[256];
        const uint64_t last = least_by_digits<NT>(row, k, count);
        if (threadIdx.x == 0) found[0] = 0;
        __syncthreads();
        row.elements_again([&](float x, uint32_t v) {
            const uint64_t key = key_of(x, v);
            if ((key >> 32) && key >= last) best[0][atomicAdd(&found[0], 1u)] = key;
        });
        __syncthreads();
        n = found[0];
    }
    for (uint32_t i = G::thread(); i < n; i += NT) {
        const uint64_t key = best[group][i];
        uint32_t place = 0;
        for (uint32_t j = 0; j < n; ++j) place += best[group][j] > key;
        if (place < k) {
            index[r * k + place] = (int32_t)(0xffffffffu - (uint32_t)key);
            out[r * k + place] = (value_of((uint32_t)(key >> 32)) - m) - log_s;
        }
    }
    for (uint32_t i = n + G::thread(); i < k; i += NT) {
        index[r * k + i] = -1;
        out[r * k + i] = 0;
    }
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

    __device__ void clear(uint32_t group)
    {
        for (uint32_t i = G::thread(); i < PLACES; i += NT) place[group][i] = -1;
        if (G::thread() == 0) twice[group] = 0;
    }
};

// The teacher's slots j of a row, slot j with thread j % NT: class (-1: empty) and answer s_j / T.
template <int NT> struct Slots {
    using G = Group<NT>;
    int32_t v[G::SLOTS];
    float t[G::SLOTS], u[G::SLOTS];

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
                    t[i] = s * a.inv_members * a.inv_t;
                }
            }
        }
    }
    __device__ float max() const
    {
        float m = neg_inf();
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i) m = fmaxf(m, t[i]);
        return m;
    }
    // u = exp(t - base), 0 in empty slots; returns their sum.  Leaves classes and u in LDS, and there whether a class comes
    // twice: of two slots of a class one finds the other in a table of twice as many places as slots.
    __device__ float weigh(float base, uint32_t k, Taught<NT> &lds, uint32_t group)
    {
        float sum = 0;
        if (NT <= 64) G::sync();                    // others have met a barrier since the table was cleared
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i) {
            u[i] = 0;
            if (v[i] < 0) continue;
            t[i] -= base;
            u[i] = __builtin_amdgcn_exp2f(t[i] * LOG2E);
            sum += u[i];
            constexpr uint32_t LAST = Taught<NT>::PLACES - 1;
            uint32_t h = ((uint32_t)v[i] * 0x9e3779b1u) >> 16 & LAST;
            while (true) {                          // ends: half of the places stay free
                const int32_t there = atomicCAS(&lds.place[group][h], -1, v[i]);
                if (there == v[i]) lds.twice[group] = 1;
                if (there < 0 || there == v[i]) break;
                h = (h + 1) & LAST;
            }
        }
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i) {
            const uint32_t j = i * NT + G::thread();
            if (j < k) {
                lds.v[group][j] = v[i];
                lds.u[group][j] = u[i];
            }
        }
        return sum;
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

template <class T> __device__ inline void clear_row(T *out, uint32_t n, uint32_t t, uint32_t step)
{
    for (uint32_t v = t; v < n; v += step) out[v] = (T)0.0f;
}

// One pass over a row that stays in registers: its maximum m and S = sum exp((z - m) / T), then loss and gradient.  With
// u_j = exp(t_j - t_max), U their sum, the three sums S, U and A = sum_j u_j (t_j - t_max - (z_j - m) / T) come out of one
// reduction, and loss = A / U - log U + log S.
template <class T, int NT, int NV, bool GRAD>
__global__ void __launch_bounds__(Group<NT>::SIZE) k_distill(Rows in, Answers a, float *loss, float *lse, T *grad, uint64_t grad_stride)
{
    using G = Group<NT>;
    using P = Pack<T>;
    __shared__ float buf[5 * G::WAVES];
    __shared__ Taught<NT> taught;
    const uint32_t group = G::row_in_group();
    const uint64_t r = in.first + (uint64_t)blockIdx.x * G::ROWS + group;
    if (r >= in.rows) return;                       // NT > 64: the whole workgroup
    const float w = a.weight ? a.weight[r] : 1.0f, scale = a.inv_t * LOG2E;
    T *out = GRAD ? grad + r * grad_stride : nullptr;
    float m[2] = {neg_inf(), neg_inf()}, s[3] = {0, 0, 0};
    Row<T, NT, NV> row;
    Slots<NT> slots;
    float x[G::SLOTS];
    taught.clear(group);
    if (w != 0.0f) {
        slots.load(a, r, in.classes);
        row.load((const T *)in.z + r * in.stride, in.classes);
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i) x[i] = slots.v[i] >= 0 ? to_float(row.z[slots.v[i]]) : 0.0f;
        m[1] = slots.max();
        m[0] = row.max();
        G::template reduce<Max, 2>(m, buf);
        s[1] = slots.weigh(m[1], a.k, taught, group);
        const float base = m[0] == neg_inf() ? 0.0f : m[0];
        s[0] = row.sum(base, scale);
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i) {
            x[i] -= base;
            if (slots.u[i] != 0.0f) s[2] += slots.u[i] * (slots.t[i] - x[i] * a.inv_t);
        }
        G::template reduce<Add, 3>(s, buf + 2 * G::WAVES);
    }
    // neither a filled slot nor a weight, or all logits -inf
    const bool none = s[1] == 0.0f, excluded = !none && s[0] == 0.0f;
    if (none || excluded) {
        if (G::thread() == 0) {
            loss[r] = 0;
            lse[r] = none ? 0.0f : neg_inf();
        }
        if (GRAD) clear_row(out, in.classes, G::thread(), NT);
        return;
    }
    const float log_s = __logf(s[0]);
    if (G::thread() == 0) {
        loss[r] = w * (s[2] / s[1] - __logf(s[1]) + log_s);
        lse[r] = m[0] * a.inv_t + log_s;
    }
    if (!GRAD) return;
    const float g = w * a.inv_t, gs = g / s[0], gu = g / s[1];
    row.each_at([&](Word4 words, uint32_t v) {
        float y[P::E];
        P::open(words, y);
#pragma unroll
        for (int i = 0; i < P::E; ++i) y[i] = __builtin_amdgcn_exp2f((y[i] - m[0]) * scale) * gs;
        *(Word4Any *)(out + v) = P::close(y);
    });
    if (row.at != 0xffffffffu) out[row.at] = (T)(__builtin_amdgcn_exp2f((row.edge - m[0]) * scale) * gs);
    // the teacher's classes, over the dense part
    G::sync();
#pragma unroll
    for (int i = 0; i < G::SLOTS; ++i)
        if (slots.v[i] >= 0)
            out[slots.v[i]] = (T)(__builtin_amdgcn_exp2f(x[i] * scale) * gs - slots.of_class(i, a.k, taught, group) * gu);
}

// Rows of which there are few, or which no workgroup can hold, are cut into parts of `per` words, a workgroup of 256 to each.
struct Parts {
    uint32_t count, per;
    float2 *stats;          // [rows][count]: maximum and sum of every part
};

template <class T, int NV> __global__ void __launch_bounds__(256) k_part_stats(Rows in, Parts parts, float scale)
{
    using G = Group<256>;
    __shared__ float buf[2][G::WAVES];
    const uint64_t r = blockIdx.x / parts.count;
    const uint32_t part = blockIdx.x % parts.count;
    Row<T, 256, NV> row;
    row.load((const T *)in.z + r * in.stride, in.classes, part * parts.per, parts.per);
    float m = row.max();
    G::reduce<Max, 1>(&m, buf[0]);
    float s = row.sum(m == neg_inf() ? 0.0f : m, scale);
    G::reduce<Add, 1>(&s, buf[1]);
    if (threadIdx.x == 0) parts.stats[blockIdx.x] = make_float2(m, s);
}

// A thread's share of a row's parts, at most 256 parts: the maximum, then with the row's maximum its sum.
struct Joined {
    float m, s;
    __device__ void load(const Parts &parts, uint64_t r)
    {
        m = neg_inf();
        s = 0;
        if (threadIdx.x < parts.count) {
            const float2 v = parts.stats[r * parts.count + threadIdx.x];
            m = v.x;
            s = v.y;
        }
    }
    __device__ float sum(float base, float scale) const { return s == 0.0f ? 0.0f : s * __builtin_amdgcn_exp2f((m - base) * scale); }
};

// The gradient of a part of a row, or with NT < 256 of a whole one, from its statistics: the lse of an earlier call, or with
// SPLIT the sums of its parts, where part 0 writes loss and lse as well.  Every part weighs the teacher's slots by itself and
// stores those whose class it has.
template <class T, int NT, int NV, bool SPLIT, bool GRAD>
__global__ void __launch_bounds__(Group<NT>::SIZE)
k_gradient(Rows in, Answers a, Parts parts, float *loss, float *lse, T *grad, uint64_t grad_stride)
{
    using G = Group<NT>;
    using P = Pack<T>;
    __shared__ float buf[5 * G::WAVES];
    __shared__ Taught<NT> taught;
    const uint32_t group = G::row_in_group(), count = GRAD ? parts.count : 1;
    const uint32_t part = NT < 256 ? 0 : blockIdx.x % count;
    const uint64_t r = in.first + (NT < 256 ? (uint64_t)blockIdx.x * G::ROWS + group : blockIdx.x / count);
    if (r >= in.rows) return;                       // NT > 64: the whole workgroup
    const float w = a.weight ? a.weight[r] : 1.0f, scale = a.inv_t * LOG2E;
    T *out = GRAD ? grad + r * grad_stride : nullptr;
    const float l = SPLIT ? 0.0f : lse[r];
    float m[2] = {neg_inf(), neg_inf()}, s[3] = {0, 0, 0};
    Row<T, NT, NV> row;
    Slots<NT> slots;
    Joined joined;
    float x[G::SLOTS];
    taught.clear(group);
    const bool wanted = w != 0.0f && l != neg_inf();
    if (wanted) {
        slots.load(a, r, in.classes);
        if (SPLIT) joined.load(parts, r);
    }
    if (GRAD) row.load((const T *)in.z + r * in.stride, in.classes, part * parts.per, parts.per);
    if (wanted) {
#pragma unroll
        for (int i = 0; i < G::SLOTS; ++i)
            x[i] = slots.v[i] >= 0 ? to_float(((const T *)in.z + r * in.stride)[slots.v[i]]) : 0.0f;
        m[1] = slots.max();
        if (SPLIT) {
            m[0] = joined.m;
            G::template reduce<Max, 2>(m, buf);
        } else {
            G::template reduce<Max, 1>(m + 1, buf);
        }
        s[1] = slots.weigh(m[1], a.k, taught, group);
        if (SPLIT) {
            if (m[0] == neg_inf()) m[0] = 0;
            s[0] = joined.sum(m[0], scale);
#pragma unroll
            for (int i = 0; i < G::SLOTS; ++i)
                if (slots.u[i] != 0.0f) s[2] += slots.u[i] * (slots.t[i] - (x[i] - m[0]) * a.inv_t);
            G::template reduce<Add, 3>(s, buf + 2 * G::WAVES);
        } else {
            G::template reduce<Add, 1>(s + 1, buf + 2 * G::WAVES);
        }
    }
    const bool none = s[1] == 0.0f, excluded = SPLIT && !none && s[0] == 0.0f, zero = none || excluded;
    if (SPLIT && part == 0 && G::thread() == 0) {
        const float log_s = __logf(s[0]);
        loss[r] = zero ? 0.0f : w * (s[2] / s[1] - __logf(s[1]) + log_s);
        lse[r] = none ? 0.0f : excluded ? neg_inf() : m[0] * a.inv_t + log_s;
    }
    if (!GRAD) return;
    // the row's share: what is taken off z / T, and the factor of exp
    const float g = w * a.inv_t, gu = g / s[1], gs = zero ? 0.0f : SPLIT ? g / s[0] : g;
    auto student = [&](float z) {
        // z / T is not rounded before lse is taken off
        return __builtin_amdgcn_exp2f(SPLIT ? (z - m[0]) * scale : __builtin_fmaf(z, a.inv_t, -l) * LOG2E) * gs;
    };
    if (zero) {
        row.each_at([&](Word4, uint32_t v) { *(Word4Any *)(out + v) = Word4{0, 0, 0, 0}; });
        if (row.at != 0xffffffffu) out[row.at] = (T)0.0f;
        return;
    }
    row.each_at([&](Word4 words, uint32_t v) {
        float y[P::E];
        P::open(words, y);
#pragma unroll
        for (int i = 0; i < P::E; ++i) y[i] = student(y[i]);
        *(Word4Any *)(out + v) = P::close(y);
    });
    if (row.at != 0xffffffffu) out[row.at] = (T)student(row.edge);
    G::sync();
    // part 0 has the edges too: all classes before its words, and those behind the last part's
    const uint32_t end = row.head + row.n * P::E, words_end = in.classes - (in.classes - row.head) % P::E;
#pragma unroll
    for (int i = 0; i < G::SLOTS; ++i) {
        const uint32_t v = slots.v[i];
        if (slots.v[i] >= 0 && ((v >= row.head && v < end) || (part == 0 && (v < row.head || v >= words_end))))
            out[v] = (T)(student(x[i]) - slots.of_class(i, a.k, taught, group) * gu);
    }
}

// Log-probabilities of rows whose parts have been summed up.
template <class T> __global__ void __launch_bounds__(256) k_part_logprobs(Rows in, Parts parts, const int32_t *index, uint32_t k, float *out)
{
    using G = Group<256>;
    __shared__ float buf[2][G::WAVES];
    const uint64_t r = blockIdx.x;
    const T *z = (const T *)in.z + r * in.stride;
    Joined joined;
    joined.load(parts, r);
    const uint32_t j = threadIdx.x;
    const int32_t at = j < k ? index[r * k + j] : -1;
    const bool filled = (uint32_t)at < in.classes;
    const float x = filled ? to_float(z[at]) : 0.0f;
    float m = joined.m;
    G::reduce<Max, 1>(&m, buf[0]);
    float s = joined.sum(m == neg_inf() ? 0.0f : m, LOG2E);
    G::reduce<Add, 1>(&s, buf[1]);
    if (j < k) out[r * k + j] = !filled ? 0.0f : x == neg_inf() && s == s ? neg_inf() : (x - m) - __logf(s);
}

}  // namespace answers
}  // namespace d2
