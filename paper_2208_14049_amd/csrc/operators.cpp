// C entries of the operators on rows in device memory: what the arguments have to be, and the launches on the caller's stream.  Nothing is
// allocated, copied or waited for here, so that a caller may capture the calls into a graph.
#include <cmath>

#include "../../include/ens.h"
#include "operators.h"

using namespace ens;

static int element_bytes(int dtype) { return dtype == ENS_FP32 ? 4 : dtype == ENS_BF16 || dtype == ENS_FP16 ? 2 : 0; }
static bool aligned(const void* p, int bytes) { return (uintptr_t)p % bytes == 0; }
// n rows of `len` elements, ld apart, that offsets in bytes can name
static bool rows_fit(int64_t n, int64_t len, int64_t ld) { return len <= ld && ld <= INT64_MAX / 8 / n; }
static bool row_buffer(const void* p, int dtype, int64_t n, int64_t len, int64_t ld) {
    return p && element_bytes(dtype) && aligned(p, element_bytes(dtype)) && rows_fit(n, len, ld);
}
static bool words(const void* p) { return p && aligned(p, 4); }
static bool words_or_null(const void* p) { return aligned(p, 4); }
// Temperatures at which every product of a logit is in reach of fp32 (Exp in rows.h).
static int temperature_status(float t) { return !(t > 0.f && std::isfinite(t)) ? ENS_E_INVALID : t < 0x1p-20f || t > 0x1p20f ? ENS_E_UNSUPPORTED : ENS_OK; }
static int status(hipError_t e) { return e == hipSuccess ? ENS_OK : e == hipErrorNoDevice ? ENS_E_NODEVICE : ENS_E_HIP; }

extern "C" {

static int route_args(const void* gates, int32_t dtype, int64_t ld, int64_t n, int32_t members, const ens_route_opts* o, RouteArgs* a) {
    if (!o || n < 0 || members < 1 || o->k < 1 || o->k > members) return ENS_E_INVALID;
    if (o->score != ENS_SCORE_SOFTMAX && o->score != ENS_SCORE_SIGMOID) return ENS_E_INVALID;
    if (!std::isfinite(o->scale)) return ENS_E_INVALID;
    const int groups = o->groups ? o->groups : 1, kept = o->groups_kept ? o->groups_kept : groups, best = o->group_best ? o->group_best : 2;
    if (groups < 1 || members % groups || kept < 1 || kept > groups || best < 1 || best > 2) return ENS_E_INVALID;
    if (o->k > members / groups * kept) return ENS_E_INVALID;
    if (members > ROUTE_MAX_MEMBERS || o->k > ROUTE_MAX_K || groups > ROUTE_MAX_GROUPS) return ENS_E_UNSUPPORTED;
    if (n > 0 && !row_buffer(gates, dtype, n, members, ld)) return ENS_E_INVALID;
    *a = RouteArgs{};
    a->gates = gates; a->ld = ld; a->n = n; a->dtype = dtype; a->members = members;
    a->k = o->k; a->score = o->score; a->groups = groups; a->groups_kept = kept; a->group_best = best;
    a->renormalise = o->renormalise != 0; a->scale = o->scale;
    return ENS_OK;
}

int ens_route(const void* gates, int32_t dtype, int64_t ld, int64_t n, int32_t members, const ens_route_opts* opts, const float* bias,
              int32_t* chosen, float* weights, int32_t* load, void* stream) {
    RouteArgs a;
    const int rc = route_args(gates, dtype, ld, n, members, opts, &a);
    if (rc != ENS_OK) return rc;
    if (n == 0) return ENS_OK;
    if (!words(chosen) || !words(weights) || !words_or_null(bias) || !words_or_null(load)) return ENS_E_INVALID;
    a.bias = bias; a.chosen = chosen; a.weights = weights; a.load = load;
    return status(launch_route(a, (hipStream_t)stream));
}

int ens_route_backward(const void* gates, int32_t dtype, int64_t ld, int64_t n, int32_t members, const ens_route_opts* opts,
                       const int32_t* chosen, const float* d_weights, void* d_gates, int64_t ld_d, void* stream) {
    RouteArgs a;
    const int rc = route_args(gates, dtype, ld, n, members, opts, &a);
    if (rc != ENS_OK) return rc;
    if (n == 0) return ENS_OK;
    if (!words(chosen) || !words(d_weights) || !row_buffer(d_gates, dtype, n, members, ld_d)) return ENS_E_INVALID;
    a.chosen = (int32_t*)chosen; a.d_weights = d_weights; a.d_gates = d_gates; a.ld_d = ld_d;
    return status(launch_route_backward(a, (hipStream_t)stream));
}

static int routed_args(const void* const* logits, int32_t dtype, int64_t ld, int64_t n, int32_t members, int32_t classes, const int32_t* chosen,
                       const float* weights, int32_t k, RoutedArgs* a) {
    if (n < 0 || members < 1 || classes < 1 || k < 1 || !logits) return ENS_E_INVALID;
    if (members > ROUTED_MAX_MEMBERS || k > ROUTED_MAX_K || classes > ROW_MAX) return ENS_E_UNSUPPORTED;
    *a = RoutedArgs{};
    if (n == 0) return ENS_OK;
    for (int m = 0; m < members; m++) {
        if (!row_buffer(logits[m], dtype, n, classes, ld)) return ENS_E_INVALID;
        a->logits[m] = logits[m];
    }
    if (!words(chosen) || !words(weights)) return ENS_E_INVALID;
    a->ld = ld; a->n = n; a->dtype = dtype; a->members = members; a->classes = classes; a->k = k;
    a->chosen = chosen; a->weights = weights;
    return ENS_OK;
}

int ens_combine_routed(const void* const* logits, int32_t dtype, int64_t ld, int64_t n, int32_t members, int32_t classes, const int32_t* chosen,
                       const float* weights, int32_t k, float* probs, float* state, void* stream) {
    RoutedArgs a;
    const int rc = routed_args(logits, dtype, ld, n, members, classes, chosen, weights, k, &a);
    if (rc != ENS_OK || n == 0) return rc;
    if (!words(probs) || !words_or_null(state) || !rows_fit(n, classes, classes)) return ENS_E_INVALID;
    a.probs = probs; a.state = state;
    return status(launch_combine_routed(a, (hipStream_t)stream));
}

int ens_combine_routed_backward(const void* const* logits, int32_t dtype, int64_t ld, int64_t n, int32_t members, int32_t classes,
                                const int32_t* chosen, const float* weights, int32_t k, const float* state, const float* d_probs,
                                float* d_weights, void* const* d_logits, int64_t ld_d, void* stream) {
    RoutedArgs a;
    const int rc = routed_args(logits, dtype, ld, n, members, classes, chosen, weights, k, &a);
    if (rc != ENS_OK || n == 0) return rc;
    if (!words(state) || !words(d_probs) || !words_or_null(d_weights)) return ENS_E_INVALID;
    a.state = (float*)state; a.d_probs = d_probs; a.d_weights = d_weights; a.ld_d = ld_d;
    bool any = d_weights != nullptr;
    for (int m = 0; m < members && d_logits; m++) {
        if (!d_logits[m]) continue;
        if (!row_buffer(d_logits[m], dtype, n, classes, ld_d)) return ENS_E_INVALID;
        a.d_logits[m] = d_logits[m];
        any = true;
    }
    if (!any) return ENS_E_INVALID;
    return status(launch_combine_routed_backward(a, (hipStream_t)stream));
}

int64_t ens_top_workspace(int64_t n, int32_t classes, int32_t k, int32_t dtype) {
    if (n < 0 || classes < 1 || k < 1 || k > classes || !element_bytes(dtype)) return ENS_E_INVALID;
    if (k > TOP_MAX_K || classes > ROW_MAX) return ENS_E_UNSUPPORTED;
    if (n > 0 && !rows_fit(n, classes, classes)) return ENS_E_INVALID;
    return n ? top_workspace(n, classes, k, dtype) : 0;
}

int ens_top(const void* values, int32_t dtype, int64_t ld, int64_t n, int32_t classes, int32_t k, int32_t form, float temperature,
            int32_t* index, float* value, void* workspace, int64_t workspace_bytes, void* stream) {
    const int64_t want = ens_top_workspace(n, classes, k, dtype);
    if (want < 0) return (int)want;
    if (form != ENS_TOP_VALUE && form != ENS_TOP_LOG && form != ENS_TOP_LOG_SOFTMAX) return ENS_E_INVALID;
    if (form == ENS_TOP_LOG_SOFTMAX && temperature_status(temperature) != ENS_OK) return temperature_status(temperature);
    if (n == 0) return ENS_OK;
    if (!row_buffer(values, dtype, n, classes, ld) || !words(index) || !words(value)) return ENS_E_INVALID;
    if (want > 0 && (!workspace || !aligned(workspace, 8) || workspace_bytes < want)) return ENS_E_INVALID;
    TopArgs a{};
    a.values = values; a.ld = ld; a.n = n; a.dtype = dtype; a.classes = classes; a.k = k; a.form = form;
    a.inv_temperature = form == ENS_TOP_LOG_SOFTMAX ? 1.f / temperature : 1.f;
    a.index = index; a.value = value; a.workspace = workspace;
    return status(launch_top(a, (hipStream_t)stream));
}

static int distill_sizes(int64_t n, int32_t classes, int32_t k, int32_t dtype) {
    if (n < 0 || classes < 1 || k < 1 || !element_bytes(dtype)) return ENS_E_INVALID;
    if (k > DISTILL_MAX_K || classes > ROW_MAX) return ENS_E_UNSUPPORTED;
    if (n > 0 && !rows_fit(n, classes, classes)) return ENS_E_INVALID;
    return ENS_OK;
}

int64_t ens_distill_workspace(int64_t n, int32_t classes, int32_t k, int32_t dtype) {
    const int rc = distill_sizes(n, classes, k, dtype);
    return rc != ENS_OK || n == 0 ? rc : distill_workspace(n, classes, k, dtype);
}

static int distill_args(const void* logits, int32_t dtype, int64_t ld, int64_t n, int32_t classes, const int32_t* index, const float* log_probs,
                        int32_t k, float temperature, int32_t tail, const float* row_weights, DistillArgs* a) {
    const int rc = distill_sizes(n, classes, k, dtype);
    if (rc != ENS_OK) return rc;
    if (temperature_status(temperature) != ENS_OK) return temperature_status(temperature);
    *a = DistillArgs{};
    if (n == 0) return ENS_OK;
    if (!row_buffer(logits, dtype, n, classes, ld) || !words(index) || !words(log_probs) || !words_or_null(row_weights)) return ENS_E_INVALID;
    a->logits = logits; a->ld = ld; a->n = n; a->dtype = dtype; a->classes = classes; a->k = k; a->tail = tail != 0;
    a->temperature = temperature; a->index = index; a->log_probs = log_probs; a->row_weights = row_weights;
    return ENS_OK;
}

int ens_distill(const void* logits, int32_t dtype, int64_t ld, int64_t n, int32_t classes, const int32_t* index, const float* log_probs,
                int32_t k, float temperature, int32_t tail, const float* row_weights, float* loss, float* state, void* d_logits, int64_t ld_d,
                void* workspace, int64_t workspace_bytes, void* stream) {
    DistillArgs a;
    const int rc = distill_args(logits, dtype, ld, n, classes, index, log_probs, k, temperature, tail, row_weights, &a);
    if (rc != ENS_OK || n == 0) return rc;
    if (!words(loss) || !words(state) || (d_logits && !row_buffer(d_logits, dtype, n, classes, ld_d))) return ENS_E_INVALID;
    if (d_logits == logits && ld_d != ld) return ENS_E_INVALID;
    const int64_t want = distill_workspace(n, classes, k, dtype);
    if (want > 0 && (!workspace || !aligned(workspace, 8) || workspace_bytes < want)) return ENS_E_INVALID;
    a.loss = loss; a.state = state; a.d_logits = d_logits; a.ld_d = ld_d; a.workspace = workspace;
    return status(launch_distill(a, (hipStream_t)stream));
}

int ens_distill_backward(const void* logits, int32_t dtype, int64_t ld, int64_t n, int32_t classes, const int32_t* index, const float* log_probs,
                         int32_t k, float temperature, int32_t tail, const float* state, const float* d_loss, void* d_logits, int64_t ld_d,
                         void* stream) {
    DistillArgs a;
    const int rc = distill_args(logits, dtype, ld, n, classes, index, log_probs, k, temperature, tail, d_loss, &a);
    if (rc != ENS_OK || n == 0) return rc;
    if (!words(state) || !row_buffer(d_logits, dtype, n, classes, ld_d)) return ENS_E_INVALID;
    if (d_logits == logits && ld_d != ld) return ENS_E_INVALID;
    a.state = (float*)state; a.d_logits = d_logits; a.ld_d = ld_d;
    return status(launch_distill_backward(a, (hipStream_t)stream));
}

}  // extern "C"
