// C ABI of libdscores (include/dtree_scores.h): checks of arguments, then the launches.
#include "scores.hpp"

#include <string>

namespace {

thread_local std::string g_error;

dt_status fail(dt_status s, const char *msg) noexcept {
    try {
        g_error = msg;
    } catch (...) {
        g_error.clear();
    }
    return s;
}

dt_status hip_result(hipError_t e) noexcept {
    return e == hipSuccess ? DT_OK : fail(DT_ERR_HIP, hipGetErrorString(e));
}

int elem_bytes(dt_dtype t) {
    return t == DT_F32 ? 4 : t == DT_F16 || t == DT_BF16 ? 2 : t == DT_U8 ? 1 : 0;
}

bool misaligned(const void *p, int bytes) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(bytes) != 0; }

// The rows of an operator's first arguments; in.n == 0: nothing to do.
dt_status rows_of(const void *x, dt_dtype type, int64_t n, int32_t classes, int64_t ld, bool votes,
                  dscores::RowArgs *in) {
    const int es = elem_bytes(type);
    if (es == 0 || (type == DT_U8 && !votes)) return fail(DT_ERR_INVALID_ARG, "unknown type of scores");
    if (n < 0) return fail(DT_ERR_INVALID_ARG, "n must be >= 0");
    if (classes < 1) return fail(DT_ERR_INVALID_ARG, "n_classes must be >= 1");
    if (n > 1 && ld < classes) return fail(DT_ERR_INVALID_ARG, "ld must be >= n_classes");
    if (classes > DS_MAX_CLASSES) return fail(DT_ERR_UNSUPPORTED, "n_classes > 2^20");
    if (n > 0x7FFFFFFF) return fail(DT_ERR_UNSUPPORTED, "n > 2^31 - 1");
    if (n > 1 && ld > (int64_t(1) << 40)) return fail(DT_ERR_UNSUPPORTED, "ld > 2^40");
    if (n > 0 && !x) return fail(DT_ERR_INVALID_ARG, "null scores");
    if (misaligned(x, es)) return fail(DT_ERR_INVALID_ARG, "scores not aligned to their element");
    in->x = x;
    in->n = n;
    in->ld = n > 1 ? ld : classes;
    in->classes = classes;
    uintptr_t bits = reinterpret_cast<uintptr_t>(x) | 16u;
    if (n > 1) bits |= uintptr_t(ld) * uintptr_t(es);
    in->align = int(bits & (~bits + 1));       // the lowest set bit
    return DT_OK;
}

dt_status teacher_of(const float *values, const int32_t *index, int32_t k, float temperature,
                     dscores::DistillArgs *a) {
    if (k < 1 || k > DS_MAX_TOP) return fail(DT_ERR_INVALID_ARG, "k must be 1 .. 256");
    if (!(temperature > 0.0f && temperature <= DS_MAX_TEMPERATURE))
        return fail(DT_ERR_INVALID_ARG, "temperature must be positive and at most 2^60");
    if (!(1.5f / temperature <= 3.402823466e38f))      // log2 e over it is used
        return fail(DT_ERR_INVALID_ARG, "temperature is too small");
    if (a->in.n > 0 && (!values || !index)) return fail(DT_ERR_INVALID_ARG, "null teacher");
    if (misaligned(values, 4) || misaligned(index, 4))
        return fail(DT_ERR_INVALID_ARG, "misaligned teacher");
    a->values = values;
    a->index = index;
    a->k = k;
    a->temperature = temperature;
    return DT_OK;
}

dt_status grad_of(dt_dtype type, const float *g, void *grad, int64_t ld_grad,
                  dscores::DistillArgs *a) {
    if (a->in.n > 0 && (!g || !grad)) return fail(DT_ERR_INVALID_ARG, "null gradient");
    if (a->in.n > 1 && ld_grad < a->in.classes)
        return fail(DT_ERR_INVALID_ARG, "ld_grad must be >= n_classes");
    if (a->in.n > 1 && ld_grad > (int64_t(1) << 40))
        return fail(DT_ERR_UNSUPPORTED, "ld_grad > 2^40");
    if (misaligned(g, 4) || misaligned(grad, elem_bytes(type)))
        return fail(DT_ERR_INVALID_ARG, "misaligned gradient");
    a->g = g;
    a->grad = grad;
    a->ld_grad = a->in.n > 1 ? ld_grad : a->in.classes;
    return DT_OK;
}

}  // namespace

extern "C" {

const char *ds_last_error(void) { return g_error.c_str(); }

dt_status ds_top_scores(const void *d_x, dt_dtype type, int64_t n, int32_t n_classes, int64_t ld,
                        int32_t k, float *d_values, int32_t *d_index, float *d_lse, void *stream) {
    g_error.clear();
    dscores::TopArgs a{};
    const dt_status st = rows_of(d_x, type, n, n_classes, ld, true, &a.in);
    if (st != DT_OK) return st;
    if (k < 1 || k > DS_MAX_TOP || k > n_classes)
        return fail(DT_ERR_INVALID_ARG, "k must be 1 .. min(n_classes, 256)");
    if (n == 0) return DT_OK;
    if (!d_values || !d_index || !d_lse) return fail(DT_ERR_INVALID_ARG, "null output");
    if (misaligned(d_values, 4) || misaligned(d_index, 4) || misaligned(d_lse, 4))
        return fail(DT_ERR_INVALID_ARG, "misaligned output");
    a.k = k;
    a.values = d_values;
    a.index = d_index;
    a.lse = d_lse;
    return hip_result(dscores::launch_top(a, type, static_cast<hipStream_t>(stream)));
}

dt_status ds_sample(const void *d_x, dt_dtype type, int64_t n, int32_t n_classes, int64_t ld,
                    const float *d_u, const ds_sampling *settings, int32_t *d_labels, void *stream) {
    g_error.clear();
    dscores::SampleArgs a{};
    const dt_status st = rows_of(d_x, type, n, n_classes, ld, true, &a.in);
    if (st != DT_OK) return st;
    if (!settings) return fail(DT_ERR_INVALID_ARG, "null settings");
    a.set = *settings;
    if (!a.set.d_temperature && !(a.set.temperature >= 0.0f && a.set.temperature <= 3.402823466e38f))
        return fail(DT_ERR_INVALID_ARG, "temperature must be >= 0 and finite");
    if (!a.set.d_top_p && !(a.set.top_p >= 0.0f)) return fail(DT_ERR_INVALID_ARG, "top_p must be >= 0");
    if (!a.set.d_min_p && !(a.set.min_p >= 0.0f && a.set.min_p <= 1.0f))
        return fail(DT_ERR_INVALID_ARG, "min_p must be 0 .. 1");
    if (misaligned(a.set.d_temperature, 4) || misaligned(a.set.d_top_k, 4) ||
        misaligned(a.set.d_top_p, 4) || misaligned(a.set.d_min_p, 4) || misaligned(d_u, 4) ||
        misaligned(d_labels, 4))
        return fail(DT_ERR_INVALID_ARG, "misaligned pointer");
    if (n == 0) return DT_OK;
    if (!d_u || !d_labels) return fail(DT_ERR_INVALID_ARG, "null device pointer");
    a.u = d_u;
    a.labels = d_labels;
    return hip_result(dscores::launch_sample(a, type, static_cast<hipStream_t>(stream)));
}

int64_t ds_distill_work_bytes(int64_t n, int32_t n_classes) {
    if (n < 1 || n_classes < 1 || n_classes > DS_MAX_CLASSES) return 0;
    const int parts = dscores::distill_parts(n, n_classes);
    return parts > 1 ? n * parts * int64_t(sizeof(float2)) : 0;
}

dt_status ds_distill(const void *d_x, dt_dtype type, int64_t n, int32_t n_classes, int64_t ld,
                     const float *d_values, const int32_t *d_index, int32_t k, float temperature,
                     const float *d_g, float *d_loss, float *d_stats, void *d_grad, int64_t ld_grad,
                     void *d_work, int64_t work_bytes, void *stream) {
    g_error.clear();
    dscores::DistillArgs a{};
    dt_status st = rows_of(d_x, type, n, n_classes, ld, false, &a.in);
    if (st == DT_OK) st = teacher_of(d_values, d_index, k, temperature, &a);
    if (st != DT_OK) return st;
    if (d_g || d_grad) {
        st = grad_of(type, d_g, d_grad, ld_grad, &a);
        if (st != DT_OK) return st;
    }
    if (n == 0) return DT_OK;
    if (!d_loss || !d_stats) return fail(DT_ERR_INVALID_ARG, "null output");
    if (misaligned(d_loss, 4) || misaligned(d_stats, 8)) return fail(DT_ERR_INVALID_ARG, "misaligned output");
    const int64_t need = ds_distill_work_bytes(n, n_classes);
    if (need > 0 && (!d_work || work_bytes < need || misaligned(d_work, 8)))
        return fail(DT_ERR_INVALID_ARG, "workspace is null, too small or misaligned");
    a.loss = d_loss;
    a.stats = reinterpret_cast<float2 *>(d_stats);
    a.part = static_cast<float2 *>(d_work);
    a.parts = dscores::distill_parts(n, n_classes);
    return hip_result(dscores::launch_distill(a, type, static_cast<hipStream_t>(stream)));
}

dt_status ds_distill_backward(const void *d_x, dt_dtype type, int64_t n, int32_t n_classes,
                              int64_t ld, const float *d_values, const int32_t *d_index, int32_t k,
                              float temperature, const float *d_stats, const float *d_g,
                              void *d_grad, int64_t ld_grad, void *stream) {
    g_error.clear();
    dscores::DistillArgs a{};
    dt_status st = rows_of(d_x, type, n, n_classes, ld, false, &a.in);
    if (st == DT_OK) st = teacher_of(d_values, d_index, k, temperature, &a);
    if (st == DT_OK) st = grad_of(type, d_g, d_grad, ld_grad, &a);
    if (st != DT_OK || n == 0) return st;
    if (!d_stats || misaligned(d_stats, 8)) return fail(DT_ERR_INVALID_ARG, "null or misaligned d_stats");
    a.stats = reinterpret_cast<float2 *>(const_cast<float *>(d_stats));
    a.parts = 1;
    return hip_result(dscores::launch_distill_backward(a, type, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
