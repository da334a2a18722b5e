// Operators on rows in device memory around an ensemble's answer: argument blocks and launchers.  operators.cpp checks the arguments; a
// launcher relies on that.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ens {

constexpr int ROUTE_MAX_MEMBERS = 512, ROUTE_MAX_K = 32, ROUTE_MAX_GROUPS = 64;
constexpr int ROUTED_MAX_MEMBERS = 64, ROUTED_MAX_K = 64;
constexpr int TOP_MAX_K = 128;
constexpr int DISTILL_MAX_K = 256;
constexpr int ROW_MAX = 1 << 24;             // classes of a row

struct RouteArgs {
    const void* gates;           // n rows of `members` values, ld apart
    int64_t ld, n;
    int dtype, members, k, score, groups, groups_kept, group_best, renormalise;
    float scale;
    const float* bias;           // or null
    int32_t* chosen;             // n x k
    float* weights;              // n x k
    int32_t* load;               // or null
    const float* d_weights;      // backward
    void* d_gates;
    int64_t ld_d;
};
hipError_t launch_route(const RouteArgs& a, hipStream_t s);
hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s);

struct RoutedArgs {
    const void* logits[ROUTED_MAX_MEMBERS];
    int64_t ld, n;
    int dtype, members, classes, k;
    const int32_t* chosen;       // n x k
    const float* weights;        // n x k
    float* probs;                // n x classes
    float* state;                // n x k x 2: maximum, logarithm of the sum of e^(z - maximum); or null (forward)
    const float* d_probs;        // backward
    float* d_weights;            // or null
    void* d_logits[ROUTED_MAX_MEMBERS];      // each or null
    int64_t ld_d;
};
hipError_t launch_combine_routed(const RoutedArgs& a, hipStream_t s);
hipError_t launch_combine_routed_backward(const RoutedArgs& a, hipStream_t s);

struct TopArgs {
    const void* values;
    int64_t ld, n;
    int dtype, classes, k, form;
    float inv_temperature;
    int32_t* index;              // n x k
    float* value;                // n x k
    void* workspace;
};
int64_t top_workspace(int64_t n, int classes, int k, int dtype);
hipError_t launch_top(const TopArgs& a, hipStream_t s);

struct DistillArgs {
    const void* logits;
    int64_t ld, n;
    int dtype, classes, k, tail;
    float temperature;
    const int32_t* index;        // n x k
    const float* log_probs;      // n x k
    const float* row_weights;    // n, or null for ones: what the gradient of a row is multiplied with
    float* loss;                 // n (forward)
    float* state;                // n x 3: maximum and logarithm of the sum of e^((x - maximum) / T), of all classes or with tail of those not listed; with tail ln(p of the listed / p of the others)
    void* d_logits;              // or null (forward)
    int64_t ld_d;
    void* workspace;
};
int64_t distill_workspace(int64_t n, int classes, int k, int dtype);
hipError_t launch_distill(const DistillArgs& a, hipStream_t s);
hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t s);

}  // namespace ens
