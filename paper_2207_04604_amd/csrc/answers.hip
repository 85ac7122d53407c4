// C-ABI entry points of the exchange of answers (see include/d2mhe.h): argument checks and launches.
#include "answers.hpp"

using namespace d2::answers;

namespace {

bool misaligned(const void *p) { return ((uintptr_t)p & 15u) != 0; }

uint64_t word(uint32_t dtype) { return dtype == D2MHE_F32 ? 4 : 2; }

bool valid(const d2mhe_logits *z)
{
    return z->dtype <= D2MHE_BF16 && z->rows < (1u << 31) && z->classes >= 1 && z->classes < (1u << 31) &&
           z->row_stride >= z->classes && (z->rows == 0 || z->row_stride < (1ull << 60) / z->rows);
}

bool valid_k(uint32_t k) { return k >= 1 && k <= MAX_TOP; }

bool valid(const d2mhe_teacher *t)
{
    return valid_k(t->k) && t->members >= 1 && t->temperature >= 0.01f && t->temperature <= 100.0f;
}

// bytes from the first to behind the last used element
uint64_t span(uint64_t rows, uint64_t stride, uint64_t used, uint64_t bytes) { return ((rows - 1) * stride + used) * bytes; }

bool overlap(const void *a, uint64_t na, const void *b, uint64_t nb)
{
    return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

d2mhe_status check_gradient(const d2mhe_logits *z, const void *grad, uint64_t stride)
{
    if (stride < z->classes || (z->rows && stride >= (1ull << 60) / z->rows)) return D2MHE_ERR_RANGE;
    if (misaligned(grad)) return D2MHE_ERR_ALIGN;
    const uint64_t b = word(z->dtype);
    if (z->rows && overlap(z->logits, span(z->rows, z->row_stride, z->classes, b), grad, span(z->rows, stride, z->classes, b)))
        return D2MHE_ERR_RANGE;
    return D2MHE_OK;
}

Rows rows_of(const d2mhe_logits *z) { return {z->logits, z->row_stride, 0, z->rows, z->classes}; }

Answers answers_of(const d2mhe_teacher *t)
{
    return {t->index, t->sum, t->weight, t->k, (float)(1.0 / ((double)t->members * t->temperature)), 1.0f / t->temperature};
}

// f(T()) with the element type of the logits
template <class F> d2mhe_status with_type(uint32_t dtype, F f)
{
    if (dtype == D2MHE_F32) f(float());
    else if (dtype == D2MHE_F16) f((_Float16)0);
    else f((__bf16)0.0f);
    return hipGetLastError() == hipSuccess ? D2MHE_OK : D2MHE_ERR_HIP;
}

// Rows are cut into parts where 1024 threads would share one (beyond 8192 words) and up to 128 rows leave half of the units
// without.  Whole / in parts, us, 131072 classes: step of 64 rows in f32 35.5 / 22.5, of 96 39.3 / 32.6, of 128 42.3 / 43.8, of 128 in
// bf16 26.0 / 24.0; loss of 128 in f32 22.8 / 18.5, log-probabilities 20.7 / 17.0; 10^6 classes, step of 128 in f32 400 / 323.  One
// limit for all, as there is one size of scratch for all; next to both borders it loses: step of 128 x 40000 in f32 16.4 / 16.9, its
// loss 8.0 / 9.2, log-probabilities of 128 x 70000 in bf16 7.1 / 8.4.  With up to 8192 words the second launch costs more than it
// brings (step of 16 x 32768 in f32 8.1 / 10.4).  1024 workgroups instead of 512: step of 64 x 131072 25.8 -> 21.5.  A part has 4
// words for each of 256 threads.
constexpr uint32_t SPLIT_ROWS = 128, SPLIT_WORDS = 8192, SPLIT_GROUPS = 1024, PART_WORDS = 1024;

template <class T> uint32_t words_of(const d2mhe_logits *z) { return (z->classes + Pack<T>::E - 1) / Pack<T>::E; }

// threads to a row and 16-byte words per thread
template <int NT, int NV> struct Shape {
    static constexpr int THREADS = NT, WORDS = NV;
};

// f(T(), Shape()): threads and words that hold a row and its k slots; the longest rows keep a part of it.  Measured on 268 MB of
// bf16, us, shape taken / next best: loss of 512 classes 53 / 127 (64 x 2), 1000 49 / 77 (64 x 2), 4096 47 / 71 (256 x 4), 16384
// 47 / 52 (512 x 8); step of 8192 94 / 100 (128 x 8), 32768 55 / 57 (256 x 16); loss of 777 x 50001 in f16 19 / 25 (1024 x 8).
template <class F> d2mhe_status with_shape(const d2mhe_logits *z, uint32_t k, F f)
{
    return with_type(z->dtype, [&](auto zero) {
        const uint32_t words = words_of<decltype(zero)>(z);
        if (words <= 16 && k <= Group<16>::TOP) f(zero, Shape<16, 1>());
        else if (words <= 64 && k <= Group<16>::TOP) f(zero, Shape<16, 4>());
        else if (words <= 128 && k <= Group<16>::TOP) f(zero, Shape<16, 8>());
        else if (words <= 512) f(zero, Shape<64, 8>());
        else if (words <= 1024) f(zero, Shape<256, 4>());
        else if (words <= 2048) f(zero, Shape<256, 8>());
        else if (words <= 4096) f(zero, Shape<512, 8>());
        else if (words <= 8192) f(zero, Shape<512, 16>());
        else f(zero, Shape<1024, 16>());
    });
}

// How rows are cut into parts: not at all where there are rows enough to fill the chip.
Parts parts_of(const d2mhe_logits *z, void *scratch)
{
    const uint32_t e = z->dtype == D2MHE_F32 ? 4 : 8, words = (z->classes + e - 1) / e;
    Parts p = {1, words, (Stats *)scratch};
    if (z->rows == 0 || z->rows > SPLIT_ROWS || words <= SPLIT_WORDS) return p;
    uint32_t want = (SPLIT_GROUPS + z->rows - 1) / z->rows;
    const uint32_t most = (words + PART_WORDS - 1) / PART_WORDS;
    if (want > most) want = most;
    if (want > 256) want = 256;
    p.per = (words + want - 1) / want;
    p.count = (words + p.per - 1) / p.per;
    return p;
}

// launch(workgroups, rows from first on) until all rows are done: a launch has at most 2^20 workgroups
template <int NT, class F> void each_launch(const d2mhe_logits *z, uint32_t parts, F launch)
{
    constexpr uint32_t PER = Group<NT>::ROWS;
    const uint32_t most = parts < (1u << 20) ? (1u << 20) / parts : 1;          // rows (PER at a time) to a launch
    Rows in = rows_of(z);
    for (uint64_t first = 0; first < z->rows; first += (uint64_t)PER * most) {
        const uint64_t groups = (z->rows - first + PER - 1) / PER;
        in.first = (uint32_t)first;
        launch(dim3((unsigned)(groups < most ? groups : most) * parts), in);
    }
}

template <int NT, class F> void each_launch(const d2mhe_logits *z, F launch) { each_launch<NT>(z, 1, launch); }

}  // namespace

extern "C" {

size_t d2mhe_logits_scratch_bytes(const d2mhe_logits *z, uint32_t k)
{
    if (!z || !valid(z) || !valid_k(k)) return 0;
    const Parts p = parts_of(z, nullptr);
    return p.count == 1 ? 256 : ((uint64_t)z->rows * p.count * sizeof(Stats) + 255) / 256 * 256;
}

d2mhe_status d2mhe_top_logprobs(const d2mhe_logits *z, uint32_t k, int32_t *index, float *logprob, void *scratch,
                                size_t scratch_bytes, void *stream)
{
    if (!z || !z->logits || !index || !logprob || !scratch) return D2MHE_ERR_NULL;
    if (!valid(z) || !valid_k(k)) return D2MHE_ERR_RANGE;
    if (misaligned(z->logits) || misaligned(index) || misaligned(logprob) || misaligned(scratch)) return D2MHE_ERR_ALIGN;
    if (scratch_bytes < d2mhe_logits_scratch_bytes(z, k)) return D2MHE_ERR_WORKSPACE;
    if (z->rows == 0) return D2MHE_OK;
    const auto run = [&](auto zero, auto shape) {
        using T = decltype(zero);
        constexpr int NT = decltype(shape)::THREADS, NV = decltype(shape)::WORDS;
        each_launch<NT>(z, [&](dim3 grid, Rows in) {
            if constexpr (NT >= 512)
                hipLaunchKernelGGL((k_top_long<T, NT, NV>), grid, dim3(NT), 0, (hipStream_t)stream, in, k, index, logprob);
            else
                hipLaunchKernelGGL((k_top<T, NT, NV>), grid, dim3(Group<NT>::SIZE), 0, (hipStream_t)stream, in, k, index, logprob);
        });
    };
    // As many threads as give a close bound, four maxima to a slot (two in a wavefront by itself), and no more than it takes to
    // hold the row; measured in us, taken / next best: 5 of 32768 x 2048 in bf16 44 / 80 (256 x 4), 64 of 2048 x 65536 64 / 66 (512
    // x 16), 100 of 4096 x 32768 67 / 147 (1024 x 4), 5 of 131072 x 512 47 / 104 (64 x 2).
    return with_type(z->dtype, [&](auto zero) {
        const uint32_t words = words_of<decltype(zero)>(z);
        if (words <= 16 && k <= 16) run(zero, Shape<16, 1>());
        else if (words <= 64 && k <= 16) run(zero, Shape<16, 4>());
        else if (words <= 128) run(zero, Shape<64, 2>());
        else if (words <= 512 && k <= 32) run(zero, Shape<64, 8>());
        else if (words <= 1024) run(zero, Shape<256, 4>());
        else if (words <= 2048 && k <= 64) run(zero, Shape<256, 8>());
        else if (words <= 4096 && k <= 128) run(zero, Shape<512, 8>());
        else if (words <= 4096) run(zero, Shape<1024, 4>());
        else if (words <= 8192) run(zero, Shape<1024, 8>());
        else run(zero, Shape<1024, 16>());
    });
}

d2mhe_status d2mhe_logprobs_at(const d2mhe_logits *z, const int32_t *index, uint32_t k, float *logprob, void *scratch,
                               size_t scratch_bytes, void *stream)
{
    if (!z || !z->logits || !index || !logprob || !scratch) return D2MHE_ERR_NULL;
    if (!valid(z) || !valid_k(k)) return D2MHE_ERR_RANGE;
    if (misaligned(z->logits) || misaligned(index) || misaligned(logprob) || misaligned(scratch)) return D2MHE_ERR_ALIGN;
    if (scratch_bytes < d2mhe_logits_scratch_bytes(z, k)) return D2MHE_ERR_WORKSPACE;
    if (z->rows == 0) return D2MHE_OK;
    const Parts parts = parts_of(z, scratch);
    if (parts.count > 1)
        return with_type(z->dtype, [&](auto zero) {
            using T = decltype(zero);
            hipLaunchKernelGGL((k_part_stats<T, 4>), dim3(z->rows * parts.count), dim3(256), 0, (hipStream_t)stream, rows_of(z),
                               parts, LOG2E);
            hipLaunchKernelGGL(k_part_logprobs<T>, dim3(z->rows), dim3(256), 0, (hipStream_t)stream, rows_of(z), parts, index, k,
                               logprob);
        });
    return with_shape(z, k, [&](auto zero, auto shape) {
        constexpr int NT = decltype(shape)::THREADS, NV = decltype(shape)::WORDS;
        each_launch<NT>(z, [&](dim3 grid, Rows in) {
            hipLaunchKernelGGL((k_logprobs_at<decltype(zero), NT, NV>), grid, dim3(Group<NT>::SIZE), 0, (hipStream_t)stream, in,
                               index, k, logprob);
        });
    });
}

d2mhe_status d2mhe_distill(const d2mhe_logits *z, const d2mhe_teacher *teacher, float *loss, float *lse, void *grad,
                           uint64_t grad_stride, void *scratch, size_t scratch_bytes, void *stream)
{
    if (!z || !teacher || !z->logits || !teacher->index || !teacher->sum || !loss || !lse || !scratch) return D2MHE_ERR_NULL;
    if (!valid(z) || !valid(teacher)) return D2MHE_ERR_RANGE;
    if (misaligned(z->logits) || misaligned(teacher->index) || misaligned(teacher->sum) || misaligned(teacher->weight) ||
        misaligned(loss) || misaligned(lse) || misaligned(scratch))
        return D2MHE_ERR_ALIGN;
    if (grad)
        if (d2mhe_status s = check_gradient(z, grad, grad_stride)) return s;
    if (scratch_bytes < d2mhe_logits_scratch_bytes(z, teacher->k)) return D2MHE_ERR_WORKSPACE;
    if (z->rows == 0) return D2MHE_OK;
    const Parts parts = parts_of(z, scratch);
    const Answers a = answers_of(teacher);
    if (parts.count > 1)
        return with_type(z->dtype, [&](auto zero) {
            using T = decltype(zero);
            hipLaunchKernelGGL((k_part_stats<T, 4>), dim3(z->rows * parts.count), dim3(256), 0, (hipStream_t)stream, rows_of(z),
                               parts, a.inv_t * LOG2E);
            if (grad)
                hipLaunchKernelGGL((k_gradient<T, 256, 4, true, true>), dim3(z->rows * parts.count), dim3(256), 0,
                                   (hipStream_t)stream, rows_of(z), a, parts, loss, lse, (T *)grad, grad_stride);
            else
                hipLaunchKernelGGL((k_gradient<T, 256, 4, true, false>), dim3(z->rows), dim3(256), 0, (hipStream_t)stream,
                                   rows_of(z), a, parts, loss, lse, (T *)nullptr, 0);
        });
    return with_shape(z, teacher->k, [&](auto zero, auto shape) {
        using T = decltype(zero);
        constexpr int NT = decltype(shape)::THREADS, NV = decltype(shape)::WORDS;
        each_launch<NT>(z, [&](dim3 grid, Rows in) {
            if (grad)
                hipLaunchKernelGGL((k_distill<T, NT, NV, true>), grid, dim3(Group<NT>::SIZE), 0, (hipStream_t)stream, in,
                                   a, loss, lse, (T *)grad, grad_stride);
            else
                hipLaunchKernelGGL((k_distill<T, NT, NV, false>), grid, dim3(Group<NT>::SIZE), 0, (hipStream_t)stream, in,
                                   a, loss, lse, (T *)nullptr, 0);
        });
    });
}

d2mhe_status d2mhe_distill_backward(const d2mhe_logits *z, const d2mhe_teacher *teacher, const float *lse, void *grad,
                                    uint64_t grad_stride, void *stream)
{
    if (!z || !teacher || !z->logits || !teacher->index || !teacher->sum || !lse || !grad) return D2MHE_ERR_NULL;
    if (!valid(z) || !valid(teacher)) return D2MHE_ERR_RANGE;
    if (misaligned(z->logits) || misaligned(teacher->index) || misaligned(teacher->sum) || misaligned(teacher->weight) ||
        misaligned(lse))
        return D2MHE_ERR_ALIGN;
    if (d2mhe_status s = check_gradient(z, grad, grad_stride)) return s;
    if (z->rows == 0) return D2MHE_OK;
    const Answers a = answers_of(teacher);
    const auto run = [&](auto zero, auto shape, Parts parts) {
        using T = decltype(zero);
        constexpr int NT = decltype(shape)::THREADS, NV = decltype(shape)::WORDS;
        each_launch<NT>(z, parts.count, [&](dim3 grid, Rows in) {
            hipLaunchKernelGGL((k_gradient<T, NT, NV, false, true>), grid, dim3(Group<NT>::SIZE), 0, (hipStream_t)stream, in, a,
                               parts, nullptr, const_cast<float *>(lse), (T *)grad, grad_stride);
        });
    };
    return with_type(z->dtype, [&](auto zero) {
        const uint32_t words = words_of<decltype(zero)>(z);
        const Parts whole = {1, words, nullptr};
        // us on 268 MB of bf16, taken / next best: 256 classes 107 / 222 (64 x 2), 700 115 / 128 (16 x 8), 2048 94 / 130 (256 x 4),
        // 4096 93 / 98 (64 x 8)
        if (words <= 16 && teacher->k <= Group<16>::TOP) run(zero, Shape<16, 1>(), whole);
        else if (words <= 64 && teacher->k <= Group<16>::TOP) run(zero, Shape<16, 4>(), whole);
        else if (words <= 128) run(zero, Shape<64, 2>(), whole);
        else if (words <= 384) run(zero, Shape<64, 8>(), whole);
        else run(zero, Shape<256, 4>(), Parts{(words + PART_WORDS - 1) / PART_WORDS, PART_WORDS, nullptr});
    });
}

}  // extern "C"
