// Routing of rows to experts, their way there and back: what the host code and the kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace spinner {

constexpr int kMostRouted = 1024;         // experts of a router
constexpr int kMostChosen = 32;           // of which a row takes
constexpr int kMostRouteGroups = 64;

enum { kSoftmax = 0, kSigmoid = 1 };

struct RouteParams {
    const void* logits;
    const float* bias;                    // null: none
    const uint8_t* mask;                  // null: all rows are routed
    float* weights;                       // [rows][top]
    int* experts;                         // [rows][top]
    const float* dweights;                // (gradient)
    void* dlogits;
    long long stride, dstride;            // elements from one row of the logits (their gradient) to the next
    int rows, count, top;                 // count: experts
    int groups, top_groups, group_top;
    int log_groups;                       // (kernels) 2^log_groups >= groups
    int score;
    int renormalise;
    float scale;
};
hipError_t launch_route(const RouteParams& p, int dtype, hipStream_t s);
hipError_t launch_route_grad(const RouteParams& p, int dtype, hipStream_t s);

struct OrderParams {
    const int* experts;
    int* places;
    long long* ends;
    int* counts;                          // [blocks][count + 1], null where one workgroup does it all
    int entries, count;
    int blocks, share;                    // workgroups, entries of each
};
// p->blocks and p->share
void plan_order(OrderParams* p);
hipError_t launch_order(const OrderParams& p, hipStream_t s);

struct ExchangeParams {
    const char* x;                        // dispatch: rows; combine: rows at their places; gradient: those of combine's result
    const char* y;                        // (gradient) rows at their places
    char* out;
    const int* places;                    // [rows][top]
    const float* weights;                 // null: ones
    float* dweights;
    long long x_stride, y_stride, out_stride;      // bytes
    int rows, top, n;
};
hipError_t launch_dispatch(const ExchangeParams& p, int size, hipStream_t s);             // size: bytes of a number
hipError_t launch_combine(const ExchangeParams& p, int dtype, hipStream_t s);
hipError_t launch_combine_grad(const ExchangeParams& p, int dtype, hipStream_t s);

}  // namespace spinner
