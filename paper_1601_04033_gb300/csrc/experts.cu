// The routed experts' entry points (fasgd_route, fasgd_gather, fasgd_combine,
// fasgd_combine_grad, fasgd_multiply, fasgd_multiply_grad): argument checks, workspace
// layout, launches.  No handle; nothing is allocated and nothing is kept between calls.

#include <algorithm>

#include "checks.cuh"
#include "product.cuh"
#include "route.cuh"

namespace {

constexpr int64_t kPlacesMax = ((int64_t)1 << 31) - 1;

int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

int check_route_shape(const char* call, const fasgd_route_args& u) {
    if (u.experts < 1 || u.experts > FASGD_EXPERTS_MAX)
        return fail(FASGD_EINVAL, "%s: experts must be in [1, %d]", call, FASGD_EXPERTS_MAX);
    if (u.rows < 0 || u.rows > kRowsMax || u.top < 1 || u.top > kPlacesMax || (__int128)u.rows * u.top > kPlacesMax)
        return fail(FASGD_EINVAL, "%s: rows must be at least 0, top at least 1, rows * top below 2^31", call);
    return FASGD_OK;
}
int64_t lay_out(fasgd::RouteArgs& a, char* base) {
    fasgd::route_chunks(a.n, a.experts, a.chunks, a.chunk);
    a.part_counts = reinterpret_cast<int32_t*>(base);
    return up16(a.chunks > 1 ? (int64_t)4 * a.chunks * a.experts : 16);
}

int exchange(const char* call, const fasgd_exchange_args* u, fasgd::ExchangeKind kind, void* stream) {
    if (u == nullptr) return fail(FASGD_EINVAL, "%s: no arguments", call);
    if (int rc = check_shape(call, u->rows, u->cols, FASGD_COLS_MAX, u->dtype)) return rc;
    if (u->top < 1 || u->top > kPlacesMax || (__int128)u->rows * u->top > kPlacesMax)
        return fail(FASGD_EINVAL, "%s: top must be at least 1, rows * top below 2^31", call);
    const int64_t size = dtype_size(u->dtype), n = u->rows * u->top;
    const bool grad = kind == fasgd::kCombineGrad;
    fasgd::ExchangeArgs a = {};
    a.ld_rows = u->ld_rows;
    a.ld_places = u->ld_places;
    a.ld_dplaces = u->ld_dplaces;
    if (int rc = check_matrix(call, "row_values", u->row_values, a.ld_rows, u->rows, u->cols, size)) return rc;
    if (int rc = check_matrix(call, "places", u->places, a.ld_places, n, u->cols, size)) return rc;
    if (grad)
        if (int rc = check_matrix(call, "dplaces", u->dplaces, a.ld_dplaces, n, u->cols, size)) return rc;
    const bool by_order = kind != fasgd::kCombine, by_weight = kind != fasgd::kGather;
    if (u->place == nullptr || (by_order && u->order == nullptr) || (grad && u->weight == nullptr))
        return fail(FASGD_EINVAL, "%s: place, order and weight must not be NULL where they are needed", call);
    if (!aligned(u->place, 4) || (by_order && !aligned(u->order, 4)) || (by_weight && !aligned(u->weight, 4)) ||
        (grad && !aligned(u->dweight, 4)))
        return fail(FASGD_EINVAL, "%s: place, order, weight and dweight must be 4-byte aligned", call);
    const int64_t w = u->cols * size;
    const Region r[] = {{"row_values", u->row_values, u->rows, w, a.ld_rows * size, kind == fasgd::kCombine},
                        {"places", u->places, n, w, a.ld_places * size, kind == fasgd::kGather},
                        {"dplaces", grad ? u->dplaces : nullptr, n, w, a.ld_dplaces * size, true},
                        block("place", u->place, 4 * n, false),
                        block("order", by_order ? u->order : nullptr, 4 * n, false),
                        block("weight", by_weight ? u->weight : nullptr, 4 * n, false),
                        block("dweight", grad ? u->dweight : nullptr, 4 * n, true)};
    if (int rc = check_shared(call, r, sizeof r / sizeof r[0])) return rc;
    if (u->rows == 0) return FASGD_OK;
    a.row_values = u->row_values;
    a.places = u->places;
    a.dplaces = grad ? u->dplaces : nullptr;
    a.order = u->order;
    a.place = u->place;
    a.weight = by_weight ? u->weight : nullptr;
    a.dweight = grad ? u->dweight : nullptr;
    a.rows = u->rows;
    a.top = u->top;
    a.cols = u->cols;
    a.n = n;
    return cuda_status(fasgd::launch_exchange(a, kind, u->dtype, static_cast<cudaStream_t>(stream)), call);
}

// ---- products ---------------------------------------------------------------

// The experts' matrices: shape, row step, expert step (set to a whole matrix where there
// is one expert).
int check_experts(const char* call, const char* name, const void* p, int64_t& ld, int64_t& step, int64_t rows,
                  int64_t cols, int64_t experts, int64_t size) {
    if (int rc = check_matrix(call, name, p, ld, rows, cols, size)) return rc;
    const int64_t whole = (rows - 1) * ld + cols;
    if (experts == 1) step = whole;
    if (step < whole || (__int128)step * experts * size > ((__int128)1 << 62))
        return fail(FASGD_EINVAL, "%s: the experts' matrices of %s are %lld values apart, fewer than one has or too many",
                    call, name, (long long)step);
    return FASGD_OK;
}

struct Multiply {
    fasgd_multiply_args u;      // with ld and step set where they are not looked at
    bool grad;                  // checked for the gradients
    int64_t size, w_size;
    // Copies in the workspace (null: the argument itself serves), and the steps of what is read.
    void *w_copy, *x_copy, *dy_copy;
    int64_t w_ld, w_step, x_ld, dy_ld;
    bool planes;                // fp32 by planes on the tensor cores
    int64_t w_plane, x_plane, dy_plane;
    float* parts;               // of sums that are split
    const void* w() const { return w_copy != nullptr ? w_copy : u.w; }
    const void* x() const { return x_copy != nullptr ? x_copy : u.x; }
    const void* dy() const { return dy_copy != nullptr ? dy_copy : u.dy; }
};

int fill_multiply(const char* call, const fasgd_multiply_args& given, bool grad, Multiply& m) {
    m = Multiply();
    m.u = given;
    m.grad = grad;
    fasgd_multiply_args& u = m.u;
    if (int rc = check_shape(call, u.rows, u.inputs, FASGD_COLS_MAX, u.dtype)) return rc;
    if (u.rows > kPlacesMax || u.outputs < 1 || u.outputs > FASGD_COLS_MAX || u.experts < 1 ||
        u.experts > FASGD_EXPERTS_MAX)
        return fail(FASGD_EINVAL, "%s: rows must be below 2^31, outputs in [1, 2^20], experts in [1, %d]", call,
                    FASGD_EXPERTS_MAX);
    if (u.w_dtype != FASGD_F32 && u.w_dtype != u.dtype)
        return fail(FASGD_EINVAL, "%s: w_dtype must be FASGD_F32 or dtype", call);
    if ((u.w_flip | u.dw_flip) & ~1) return fail(FASGD_EINVAL, "%s: w_flip and dw_flip are 0 or 1", call);
    m.size = dtype_size(u.dtype);
    m.w_size = dtype_size(u.w_dtype);
    if (u.offsets == nullptr || !aligned(u.offsets, 4))
        return fail(FASGD_EINVAL, "%s: offsets must not be NULL, and 4-byte aligned", call);
    const bool by_x = !grad || u.dw != nullptr, by_w = !grad || u.dx != nullptr;
    if (by_x)
        if (int rc = check_matrix(call, "x", u.x, u.ld_x, u.rows, u.inputs, m.size)) return rc;
    if (by_w)
        if (int rc = check_experts(call, "w", u.w, u.ld_w, u.step_w, u.w_flip ? u.outputs : u.inputs,
                                   u.w_flip ? u.inputs : u.outputs, u.experts, m.w_size))
            return rc;
    if (!grad) return check_matrix(call, "y", u.y, u.ld_y, u.rows, u.outputs, m.size);
    if (u.dx == nullptr && u.dw == nullptr) return fail(FASGD_EINVAL, "%s: dx or dw must be given", call);
    if (int rc = check_matrix(call, "dy", u.dy, u.ld_dy, u.rows, u.outputs, m.size)) return rc;
    if (u.dx != nullptr)
        if (int rc = check_matrix(call, "dx", u.dx, u.ld_dx, u.rows, u.inputs, m.size)) return rc;
    if (u.dw != nullptr)
        if (int rc = check_experts(call, "dw", u.dw, u.ld_dw, u.step_dw, u.dw_flip ? u.outputs : u.inputs,
                                   u.dw_flip ? u.inputs : u.outputs, u.experts, m.w_size))
            return rc;
    return FASGD_OK;
}
fasgd::Product product(const Multiply& m) {
    fasgd::Product p = {};
    p.groups = (int32_t)m.u.experts;
    p.offsets = m.u.offsets;
    p.dtype = m.planes ? FASGD_BF16 : m.u.dtype;
    p.planes = p.exact = m.planes;
    p.ending = fasgd::kStore;
    p.out_dtype = m.u.dtype;
    p.factor = 1.0f;
    return p;
}
// y (or dx) by rows: `to` columns from `from`, w's side across or not.
fasgd::Product by_rows(const Multiply& m, int64_t from, int64_t to, bool across, const fasgd::Side& x, void* y, int64_t ld_y) {
    fasgd::Product p = product(m);
    p.a = {m.w(), m.w_ld, m.w_step, across, m.w_plane, m.planes ? 4 : 0};
    p.b = x;
    p.m = to;
    p.n = m.u.rows;
    p.k = from;
    p.ragged = fasgd::kRaggedN;
    p.out = y;
    p.ld_out = ld_y;
    return p;
}
fasgd::Product product_y(const Multiply& m) {
    return by_rows(m, m.u.inputs, m.u.outputs, !m.u.w_flip, {m.x(), m.x_ld, 0, 0, m.x_plane, m.planes ? 4 : 0}, m.u.y, m.u.ld_y);
}
fasgd::Product product_dx(const Multiply& m) {
    return by_rows(m, m.u.outputs, m.u.inputs, m.u.w_flip, {m.dy(), m.dy_ld, 0, 0, m.dy_plane, m.planes ? 4 : 0}, m.u.dx, m.u.ld_dx);
}
fasgd::Product by_experts(const Multiply& m) {
    const fasgd_multiply_args& u = m.u;
    fasgd::Product p = product(m);
    const fasgd::Side x = {m.x(), m.x_ld, 0, 1, m.x_plane, m.planes ? 4 : 0}, dy = {m.dy(), m.dy_ld, 0, 1, m.dy_plane, m.planes ? 4 : 0};
    p.a = u.dw_flip ? x : dy;
    p.b = u.dw_flip ? dy : x;
    p.m = u.dw_flip ? u.inputs : u.outputs;
    p.n = u.dw_flip ? u.outputs : u.inputs;
    p.k = u.rows;
    p.ragged = fasgd::kRaggedK;
    p.out = u.dw;
    p.ld_out = u.ld_dw;
    p.step_out = u.step_dw;
    p.out_dtype = u.w_dtype;
    p.exact = u.w_dtype == FASGD_F32;      // (one that is stored in 16 bits loses less than its rounding: launch_tiles sees to that)
    return p;
}

int64_t lay_out(Multiply& m, char* base) {
    const fasgd_multiply_args& u = m.u;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char* p = base + at;
        at += up256(bytes);
        return p;
    };
    m.w_ld = u.ld_w;
    m.w_step = u.step_w;
    m.x_ld = u.ld_x;
    m.dy_ld = u.ld_dy;
    m.w_copy = m.x_copy = m.dy_copy = nullptr;
    // The tensor cores' operands start and step on 16 bytes; fp32 ones are copied to planes, where
    // the products are large enough for the copies.
    m.planes = u.dtype == FASGD_F32 && fasgd::by_planes(u.rows, u.outputs, u.inputs);
    const bool tiles = u.dtype != FASGD_F32;
    const auto fits = [&](const void* p, int64_t ld, int64_t step, int64_t groups) {
        return !m.planes && (!tiles || fasgd::tile_side({p, ld, step, 0, 0, 0}, groups));
    };
    const auto copy = [&](int64_t values, int64_t& plane) {
        plane = values;
        return take(m.planes ? 8 * values : values * m.size);
    };
    if ((!m.grad || u.dx != nullptr) && (u.w_dtype != u.dtype || !fits(u.w, u.ld_w, u.step_w, u.experts))) {
        const int64_t rows = u.w_flip ? u.outputs : u.inputs, cols = u.w_flip ? u.inputs : u.outputs;
        m.w_ld = (cols + 7) / 8 * 8;
        m.w_step = rows * m.w_ld;
        m.w_copy = copy(u.experts * m.w_step, m.w_plane);
    }
    if ((!m.grad || u.dw != nullptr) && !fits(u.x, u.ld_x, 0, 1)) {
        m.x_ld = (u.inputs + 7) / 8 * 8;
        m.x_copy = copy(u.rows * m.x_ld, m.x_plane);
    }
    if (m.grad && !fits(u.dy, u.ld_dy, 0, 1)) {
        m.dy_ld = (u.outputs + 7) / 8 * 8;
        m.dy_copy = copy(u.rows * m.dy_ld, m.dy_plane);
    }
    // One product after the other takes the same room.
    int64_t parts = 0;
    if (u.rows > 0) {
        if (!m.grad) parts = fasgd::part_values(product_y(m));
        if (m.grad && u.dx != nullptr) parts = fasgd::part_values(product_dx(m));
        if (m.grad && u.dw != nullptr) parts = std::max(parts, fasgd::part_values(by_experts(m)));
    }
    m.parts = reinterpret_cast<float*>(take(4 * parts));
    return at;
}

int check_workspace(const char* call, const void* p, int64_t has, int64_t need) {
    if (need > 0 && (p == nullptr || !aligned(p, 256) || has < need))
        return fail(FASGD_EINVAL, "%s: workspace must be 256-byte aligned and hold %lld bytes", call, (long long)need);
    return FASGD_OK;
}

cudaError_t copy_w(const Multiply& m, cudaStream_t stream) {
    if (m.w_copy == nullptr) return cudaSuccess;
    const fasgd_multiply_args& u = m.u;
    fasgd::Pack p = {};
    p.from = u.w;
    p.to = m.w_copy;
    p.rows = u.w_flip ? u.outputs : u.inputs;
    p.cols = u.w_flip ? u.inputs : u.outputs;
    p.ld_from = u.ld_w;
    p.step_from = u.step_w;
    p.ld_to = m.w_ld;
    p.step_to = m.w_step;
    p.groups = (int32_t)u.experts;
    p.dtype_from = u.w_dtype;
    p.dtype_to = u.dtype;
    p.plane = m.planes ? m.w_plane : 0;
    p.offsets = u.offsets;
    return fasgd::launch_pack(p, stream);
}

cudaError_t copy_rows(const Multiply& m, const void* from, int64_t ld, int64_t cols, void* to, int64_t ld_to, int64_t plane,
                      cudaStream_t stream) {
    if (to == nullptr) return cudaSuccess;
    fasgd::Pack p = {};
    p.from = from;
    p.to = to;
    p.rows = m.u.rows;
    p.cols = cols;
    p.ld_from = ld;
    p.ld_to = ld_to;
    p.groups = 1;
    p.dtype_from = p.dtype_to = m.u.dtype;
    p.plane = m.planes ? plane : 0;
    return fasgd::launch_pack(p, stream);
}

// The arguments' memory, for check_shared.
int check_multiply_shared(const char* call, const Multiply& m) {
    const fasgd_multiply_args& u = m.u;
    const bool by_x = !m.grad || u.dw != nullptr, by_w = !m.grad || u.dx != nullptr;
    const auto matrix = [&](const char* name, const void* p, int64_t cols, int64_t ld, bool output) {
        return Region{name, p, u.rows, cols * m.size, ld * m.size, output};
    };
    const auto experts = [&](const char* name, const void* p, bool flip, int64_t ld, int64_t step, bool output) {
        const int64_t rows = flip ? u.outputs : u.inputs, cols = flip ? u.inputs : u.outputs;
        return Region{name, p, u.experts, ((rows - 1) * ld + cols) * m.w_size, step * m.w_size, output};
    };
    const Region r[] = {matrix("x", by_x ? u.x : nullptr, u.inputs, u.ld_x, false),
                        experts("w", by_w ? u.w : nullptr, u.w_flip, u.ld_w, u.step_w, false),
                        block("offsets", u.offsets, 4 * (u.experts + 1), false),
                        matrix("y", m.grad ? nullptr : u.y, u.outputs, u.ld_y, true),
                        matrix("dy", m.grad ? u.dy : nullptr, u.outputs, u.ld_dy, false),
                        matrix("dx", m.grad ? u.dx : nullptr, u.inputs, u.ld_dx, true),
                        experts("dw", m.grad ? u.dw : nullptr, u.dw_flip, u.ld_dw, u.step_dw, true),
                        block("workspace", u.workspace, u.workspace_bytes, true)};
    return check_shared(call, r, sizeof r / sizeof r[0]);
}

}  // namespace

extern "C" {

int64_t fasgd_route_workspace(const fasgd_route_args* u) {
    const char* call = "fasgd_route_workspace";
    if (u == nullptr) {
        fail(FASGD_EINVAL, "%s: no arguments", call);
        return -1;
    }
    if (check_route_shape(call, *u) != FASGD_OK) return -1;
    fasgd::RouteArgs a = {};
    a.n = u->rows * u->top;
    a.experts = (int32_t)u->experts;
    return lay_out(a, nullptr);
}

int fasgd_route(const fasgd_route_args* u, void* stream) {
    const char* call = "fasgd_route";
    if (u == nullptr) return fail(FASGD_EINVAL, "%s: no arguments", call);
    if (int rc = check_route_shape(call, *u)) return rc;
    if (u->chosen == nullptr || u->offsets == nullptr || u->order == nullptr || u->place == nullptr ||
        !aligned(u->chosen, 4) || !aligned(u->offsets, 4) || !aligned(u->order, 4) || !aligned(u->place, 4))
        return fail(FASGD_EINVAL, "%s: chosen, offsets, order and place must not be NULL, and 4-byte aligned", call);
    fasgd::RouteArgs a = {};
    a.n = u->rows * u->top;
    a.experts = (int32_t)u->experts;
    const int64_t need = lay_out(a, static_cast<char*>(u->workspace));
    if (u->workspace == nullptr || !aligned(u->workspace, 16) || u->workspace_bytes < need)
        return fail(FASGD_EINVAL, "%s: workspace must be 16-byte aligned and hold %lld bytes", call, (long long)need);
    const Region r[] = {block("chosen", u->chosen, 4 * a.n, false), block("offsets", u->offsets, 4 * (u->experts + 1), true),
                        block("order", u->order, 4 * a.n, true), block("place", u->place, 4 * a.n, true),
                        block("workspace", u->workspace, u->workspace_bytes, true)};
    if (int rc = check_shared(call, r, sizeof r / sizeof r[0])) return rc;
    a.chosen = u->chosen;
    a.offsets = u->offsets;
    a.order = u->order;
    a.place = u->place;
    return cuda_status(fasgd::launch_route(a, static_cast<cudaStream_t>(stream)), call);
}

int fasgd_gather(const fasgd_exchange_args* u, void* stream) {
    return exchange("fasgd_gather", u, fasgd::kGather, stream);
}
int fasgd_combine(const fasgd_exchange_args* u, void* stream) {
    return exchange("fasgd_combine", u, fasgd::kCombine, stream);
}
int fasgd_combine_grad(const fasgd_exchange_args* u, void* stream) {
    return exchange("fasgd_combine_grad", u, fasgd::kCombineGrad, stream);
}

int fasgd_client_sync(int32_t* late, void* stream_) {
    const char* call = "fasgd_client_sync";
    const auto stream = static_cast<cudaStream_t>(stream_);
    if (late == nullptr) return fail(FASGD_EINVAL, "%s: late is NULL", call);
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    const cudaError_t st = cudaStreamIsCapturing(stream, &capture);
    if (st != cudaSuccess) return cuda_status(st, call);
    if (capture != cudaStreamCaptureStatusNone) return fail(FASGD_EINVAL, "%s: the stream is being captured", call);
    return cuda_status(fasgd::read_late(late, stream), call);
}

int fasgd_selftest_product_wait(int64_t ns, void* stream) {
    const int rc = fasgd_selftest_product_limit(ns);
    return rc != FASGD_OK ? rc : cuda_status(fasgd::launch_expiry(static_cast<cudaStream_t>(stream)), "fasgd_selftest_product_wait");
}

int fasgd_selftest_product_limit(int64_t ns) {
    if (ns < 1000000 || ns > 1000000000) return fail(FASGD_EINVAL, "fasgd_selftest_product_limit: ns must be in [10^6, 10^9]");
    fasgd::set_wait_limit((uint64_t)ns);
    return FASGD_OK;
}

int64_t fasgd_multiply_workspace(const fasgd_multiply_args* u) {
    const char* call = "fasgd_multiply_workspace";
    if (u == nullptr) {
        fail(FASGD_EINVAL, "%s: no arguments", call);
        return -1;
    }
    Multiply m;
    if (fill_multiply(call, *u, u->dx != nullptr || u->dw != nullptr, m) != FASGD_OK) return -1;
    return lay_out(m, nullptr);
}

int fasgd_multiply(const fasgd_multiply_args* u, void* stream_) {
    const char* call = "fasgd_multiply";
    const auto stream = static_cast<cudaStream_t>(stream_);
    if (u == nullptr) return fail(FASGD_EINVAL, "%s: no arguments", call);
    Multiply m;
    if (int rc = fill_multiply(call, *u, false, m)) return rc;
    const int64_t need = lay_out(m, static_cast<char*>(u->workspace));
    if (int rc = check_workspace(call, u->workspace, u->workspace_bytes, need)) return rc;
    if (int rc = check_multiply_shared(call, m)) return rc;
    if (u->rows == 0) return FASGD_OK;
    cudaError_t st = copy_w(m, stream);
    if (st == cudaSuccess) st = copy_rows(m, m.u.x, m.u.ld_x, u->inputs, m.x_copy, m.x_ld, m.x_plane, stream);
    if (st == cudaSuccess)
        st = fasgd::launch_product(product_y(m), m.parts, stream);
    return cuda_status(st, call);
}

int fasgd_multiply_grad(const fasgd_multiply_args* u, void* stream_) {
    const char* call = "fasgd_multiply_grad";
    const auto stream = static_cast<cudaStream_t>(stream_);
    if (u == nullptr) return fail(FASGD_EINVAL, "%s: no arguments", call);
    Multiply m;
    if (int rc = fill_multiply(call, *u, true, m)) return rc;
    const int64_t need = lay_out(m, static_cast<char*>(u->workspace));
    if (int rc = check_workspace(call, u->workspace, u->workspace_bytes, need)) return rc;
    if (int rc = check_multiply_shared(call, m)) return rc;
    if (u->rows == 0) {      // no rows: no operands to copy or to describe
        m.u.dtype = FASGD_F32;
        m.planes = false;
        return cuda_status(u->dw != nullptr ? fasgd::launch_product(by_experts(m), m.parts, stream) : cudaSuccess, call);
    }
    cudaError_t st = copy_rows(m, m.u.dy, m.u.ld_dy, u->outputs, m.dy_copy, m.dy_ld, m.dy_plane, stream);
    if (st == cudaSuccess && u->dx != nullptr) {
        st = copy_w(m, stream);
        if (st == cudaSuccess)
            st = fasgd::launch_product(product_dx(m), m.parts, stream);
    }
    if (st == cudaSuccess && u->dw != nullptr) {
        st = copy_rows(m, m.u.x, m.u.ld_x, u->inputs, m.x_copy, m.x_ld, m.x_plane, stream);
        if (st == cudaSuccess) st = fasgd::launch_product(by_experts(m), m.parts, stream);
    }
    return cuda_status(st, call);
}

}  // extern "C"
