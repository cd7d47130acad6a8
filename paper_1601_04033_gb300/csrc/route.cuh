// Internal interface of the routes and of the exchange between rows and places
// (experts.cu checks the arguments; route.cu and exchange.cu hold the kernels).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace fasgd {

struct RouteArgs {
    const int32_t* chosen;
    int32_t *offsets, *order, *place;
    int64_t n;               // rows * top
    int32_t experts;
    int32_t chunks;          // blocks that share the entries
    int64_t chunk;           // entries of each
    int32_t* part_counts;    // [chunks][experts] (chunks > 1)
};
// How many blocks share a route's entries, and how many entries each takes.
void route_chunks(int64_t n, int32_t experts, int32_t& chunks, int64_t& chunk);
cudaError_t launch_route(const RouteArgs& a, cudaStream_t stream);

struct ExchangeArgs {
    void* row_values;
    void* places;
    void* dplaces;
    const int32_t *order, *place;
    const float* weight;
    float* dweight;
    int64_t rows, top, cols, n;
    int64_t ld_rows, ld_places, ld_dplaces;
};
enum ExchangeKind { kGather, kCombine, kCombineGrad };
cudaError_t launch_exchange(const ExchangeArgs& a, ExchangeKind kind, int dtype, cudaStream_t stream);

}  // namespace fasgd
