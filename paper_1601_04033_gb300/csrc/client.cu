// The client operators' entry points (fasgd_dropout, fasgd_join, fasgd_join_grad,
// fasgd_balance): argument checks, workspace layout, launch.  No handle; nothing
// is allocated and nothing is kept between calls.

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "client.cuh"

namespace fasgd {
void set_handleless_error(const char* msg);  // defined in runtime.cu
}

namespace {

constexpr int64_t kRowsMax = (int64_t)1 << 40;

int fail(int code, const char* fmt, ...) noexcept {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
        fasgd::set_handleless_error(buf);
    } catch (...) {       // out of memory for the text: the code says enough
    }
    return code;
}
int cuda_status(cudaError_t st, const char* call) {
    return st == cudaSuccess ? FASGD_OK : fail(FASGD_ECUDA, "%s: %s", call, cudaGetErrorString(st));
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int64_t dtype_size(int32_t dtype) { return dtype == FASGD_F32 ? 4 : 2; }

// An argument's memory: `rows` rows of `width` bytes, `step` bytes apart.
struct Region {
    const char* name;
    const void* p;
    int64_t rows, width, step;
    bool output;
};
Region block(const char* name, const void* p, int64_t bytes, bool output) {
    return {name, p, 1, bytes, bytes, output};
}
bool share(const Region& a, const Region& b) {
    if (a.p == nullptr || b.p == nullptr || a.rows == 0 || b.rows == 0 || a.width == 0 || b.width == 0)
        return false;
    const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
    const uintptr_t ea = pa + (uintptr_t)((a.rows - 1) * a.step + a.width);
    const uintptr_t eb = pb + (uintptr_t)((b.rows - 1) * b.step + b.width);
    if (ea <= pb || eb <= pa) return false;
    if (a.rows > 1 && b.rows > 1 && a.step == b.step) {   // columns of one wider matrix
        const uintptr_t off = (pa < pb ? pb - pa : pa - pb) % (uintptr_t)a.step;
        const int64_t first = pa < pb ? a.width : b.width, second = pa < pb ? b.width : a.width;
        if ((int64_t)off >= first && (int64_t)off + second <= a.step) return false;
    }
    return true;
}
// EINVAL where an output shares memory with another argument.
int check_shared(const char* call, const Region* r, int n) {
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if ((r[i].output || r[j].output) && share(r[i], r[j]))
                return fail(FASGD_EINVAL, "%s: %s and %s share memory", call, r[j].name, r[i].name);
    return FASGD_OK;
}

int check_shape(const char* call, int64_t rows, int64_t cols, int64_t cols_max, int32_t dtype) {
    if (rows < 0 || rows > kRowsMax || cols < 1 || cols > cols_max)
        return fail(FASGD_EINVAL, "%s: rows must be in [0, 2^40], cols in [1, %lld]", call, (long long)cols_max);
    if (dtype != FASGD_F32 && dtype != FASGD_BF16 && dtype != FASGD_F16)
        return fail(FASGD_EINVAL, "%s: dtype %d is not an fasgd_dtype", call, dtype);
    return FASGD_OK;
}
// A matrix argument: pointer, alignment of its type, row step.  ld is set to cols
// where there is no second row to step to.
int check_matrix(const char* call, const char* name, const void* p, int64_t& ld, int64_t rows, int64_t cols,
                 int64_t size) {
    if (p == nullptr) return fail(FASGD_EINVAL, "%s: %s is NULL", call, name);
    if (!aligned(p, (uintptr_t)size)) return fail(FASGD_EINVAL, "%s: %s is not aligned to its type", call, name);
    if (rows < 2) ld = cols;
    if (ld < cols || ld > kRowsMax || (__int128)ld * rows * size > ((__int128)1 << 62))
        return fail(FASGD_EINVAL, "%s: the rows of %s are %lld values apart, fewer than cols or too many", call,
                    name, (long long)ld);
    return FASGD_OK;
}

int fill_draws(const char* call, fasgd::DropArgs& d, double rate, uint64_t seed, int32_t client, uint64_t n,
               int64_t rows, int64_t cols) {
    if (!(rate >= 0.0 && rate <= 1.0)) return fail(FASGD_EINVAL, "%s: rate must be in [0, 1]", call);
    if (client < 0 || client >= (1 << 30)) return fail(FASGD_EINVAL, "%s: client must be in [0, 2^30)", call);
    if (n >> 48) return fail(FASGD_EINVAL, "%s: n must be below 2^48", call);
    if ((__int128)rows * cols >= ((__int128)1 << 51))
        return fail(FASGD_EINVAL, "%s: rows * cols must be below 2^51", call);
    fasgd::philox_key_schedule(seed, d.round_key0, d.round_key1);
    d.client_word = (uint32_t)client + (3u << 30);
    d.n_lo = (uint32_t)n;
    d.n_hi = (uint32_t)(n >> 32);
    d.cut = (uint32_t)std::floor(rate * 65536.0 + 0.5);
    d.last = d.cut == 0 ? 0u : d.cut >= 65536u ? ~0u : (d.cut << 16) - 1u;
    d.scale = d.cut < 65536u ? 65536.0f / (float)(65536u - d.cut) : 0.0f;
    return FASGD_OK;
}

cudaError_t sm_count(int& sms) {
    int dev = 0;
    const cudaError_t st = cudaGetDevice(&dev);
    return st != cudaSuccess ? st : cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
}

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// The checks that fasgd_join and fasgd_join_grad share, and the kernels' view.
int fill_join(const char* call, const fasgd_join_args& u, fasgd::JoinArgs& a) {
    if (int rc = check_shape(call, u.rows, u.cols, FASGD_COLS_MAX, u.dtype)) return rc;
    if (u.groups < 1 || u.groups > kRowsMax || u.rows % u.groups != 0)      // (of no rows there may be any number)
        return fail(FASGD_EINVAL, "%s: groups must be in [1, 2^40] and divide rows", call);
    if (u.norm != FASGD_RMS_NORM && u.norm != FASGD_LAYER_NORM)
        return fail(FASGD_EINVAL, "%s: norm %d is not an fasgd_norm", call, u.norm);
    if (!(u.eps > 0.f) || !std::isfinite(u.eps) || !std::isfinite(u.carry) || !std::isfinite(u.branch))
        return fail(FASGD_EINVAL, "%s: eps must be positive, and eps, carry and branch finite", call);
    if (u.y == nullptr && (u.post != nullptr || u.gate != nullptr || u.pre == nullptr))
        return fail(FASGD_EINVAL, "%s: without y there is no post or gate, and pre is needed", call);
    if ((u.post == nullptr && u.post_bias != nullptr) || (u.pre == nullptr && u.pre_bias != nullptr))
        return fail(FASGD_EINVAL, "%s: a bias without its norm", call);
    if (u.gate != nullptr && u.gate_dtype != FASGD_F32 && u.gate_dtype != u.dtype)
        return fail(FASGD_EINVAL, "%s: gate_dtype must be FASGD_F32 or dtype", call);
    const int64_t gate_size = u.gate_dtype == FASGD_F32 ? 4 : dtype_size(u.dtype);
    if (!aligned(u.post, 4) || !aligned(u.post_bias, 4) || !aligned(u.pre, 4) || !aligned(u.pre_bias, 4) ||
        !aligned(u.gate, (uintptr_t)gate_size))
        return fail(FASGD_EINVAL, "%s: a parameter is not aligned to its type", call);
    if (!aligned(u.stats, 16)) return fail(FASGD_EINVAL, "%s: stats must be 16-byte aligned", call);
    a = fasgd::JoinArgs();
    a.ld_x = u.ld_x;
    a.ld_y = u.ld_y;
    const int64_t size = dtype_size(u.dtype);
    if (int rc = check_matrix(call, "x", u.x, a.ld_x, u.rows, u.cols, size)) return rc;
    if (u.y != nullptr)
        if (int rc = check_matrix(call, "y", u.y, a.ld_y, u.rows, u.cols, size)) return rc;
    // Without y there is nothing to drop.
    const double rate = u.y != nullptr || !(u.rate >= 0.0 && u.rate <= 1.0) ? u.rate : 0.0;
    if (int rc = fill_draws(call, a.drop, rate, u.seed, u.client, u.n, u.rows, u.cols)) return rc;
    a.x = u.x;
    a.y = u.y;
    a.post = u.post;
    a.post_bias = u.post_bias;
    a.gate = u.gate;
    a.pre = u.pre;
    a.pre_bias = u.pre_bias;
    a.stats = reinterpret_cast<float4*>(u.stats);
    a.rows = u.rows;
    a.cols = u.cols;
    a.groups = u.groups;
    a.group_rows = u.rows / u.groups;
    a.layer = u.norm == FASGD_LAYER_NORM;
    a.gate_f32 = u.gate_dtype == FASGD_F32;
    a.eps = u.eps;
    a.carry = u.y != nullptr ? u.carry : 1.f;      // h = x
    a.branch = u.y != nullptr ? u.branch : 0.f;
    a.inv_cols = 1.0f / (float)u.cols;
    return FASGD_OK;
}
int fill_join_grad(const char* call, const fasgd_join_args& u, fasgd::JoinArgs& a) {
    if (int rc = fill_join(call, u, a)) return rc;
    const int64_t size = dtype_size(u.dtype);
    a.ld_dh = u.ld_dh;
    a.ld_dz = u.ld_dz;
    a.ld_dx = u.ld_dx;
    a.ld_dy = u.ld_dy;
    if (u.stats == nullptr) return fail(FASGD_EINVAL, "%s: stats is NULL", call);
    if ((u.pre != nullptr) != (u.dz != nullptr)) return fail(FASGD_EINVAL, "%s: dz goes with pre", call);
    if ((u.y != nullptr) != (u.dy != nullptr)) return fail(FASGD_EINVAL, "%s: dy goes with y", call);
    if ((u.dpost != nullptr && u.post == nullptr) || (u.dpost_bias != nullptr && u.post == nullptr) ||
        (u.dpre != nullptr && u.pre == nullptr) || (u.dpre_bias != nullptr && u.pre == nullptr) ||
        (u.dgate != nullptr && u.gate == nullptr))
        return fail(FASGD_EINVAL, "%s: the gradient of a parameter that is not there", call);
    const int64_t gate_size = u.gate_dtype == FASGD_F32 ? 4 : size;
    if (!aligned(u.dpost, 4) || !aligned(u.dpost_bias, 4) || !aligned(u.dpre, 4) || !aligned(u.dpre_bias, 4) ||
        !aligned(u.dgate, (uintptr_t)gate_size))
        return fail(FASGD_EINVAL, "%s: a parameter's gradient is not aligned to its type", call);
    if (u.dh != nullptr)
        if (int rc = check_matrix(call, "dh", u.dh, a.ld_dh, u.rows, u.cols, size)) return rc;
    if (u.dz != nullptr)
        if (int rc = check_matrix(call, "dz", u.dz, a.ld_dz, u.rows, u.cols, size)) return rc;
    if (int rc = check_matrix(call, "dx", u.dx, a.ld_dx, u.rows, u.cols, size)) return rc;
    if (u.dy != nullptr)
        if (int rc = check_matrix(call, "dy", u.dy, a.ld_dy, u.rows, u.cols, size)) return rc;
    a.dh = u.dh;
    a.dz = u.dz;
    a.dx = u.dx;
    a.dy = u.dy;
    a.out_param[0] = u.dpost;
    a.out_param[1] = u.dpost_bias;
    a.out_param[2] = u.dpre;
    a.out_param[3] = u.dpre_bias;
    a.out_gate = u.dgate;
    return FASGD_OK;
}

// The workspace of a gradient call: partial sums of the parameters' gradients,
// of the gate's, and the rows' means.
int64_t lay_out(fasgd::JoinArgs& a, const fasgd::JoinPlan& plan, char* base) {
    a.parts = plan.parts;
    a.splits = plan.splits;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char* p = base + at;
        at += up16(bytes);
        return p;
    };
    a.params = reinterpret_cast<float*>(take(20 * plan.parts * a.cols));
    a.gates = reinterpret_cast<float*>(
        take(a.out_gate != nullptr && a.groups > 1 && plan.splits > 1 ? 4 * a.groups * plan.splits * a.cols : 0));
    a.row_means = reinterpret_cast<float2*>(take(8 * plan.row_means));
    return at;
}

// fasgd_balance's shape, and its workspace.
int check_balance_shape(const char* call, const fasgd_balance_args& u) {
    if (int rc = check_shape(call, u.rows, u.cols, FASGD_EXPERTS_MAX, u.dtype)) return rc;
    if (u.groups < 1 || u.rows % u.groups != 0)
        return fail(FASGD_EINVAL, "%s: groups must be at least 1 and divide rows", call);
    if (u.top < 1 || u.top >= ((int64_t)1 << 31) || (__int128)u.rows * u.top >= ((__int128)1 << 31))
        return fail(FASGD_EINVAL, "%s: top must be at least 1, rows * top below 2^31", call);
    if ((__int128)u.groups * u.cols >= ((__int128)1 << 40))
        return fail(FASGD_EINVAL, "%s: groups * cols must be below 2^40", call);
    return FASGD_OK;
}
int64_t lay_out(fasgd::BalanceArgs& a, char* base) {
    a.splits = fasgd::balance_splits(a.rows, a.groups, a.top);
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char* p = base + at;
        at += up16(bytes);
        return p;
    };
    a.part_loss = reinterpret_cast<float2*>(take(8 * fasgd::kBalanceParts));
    a.ticket = reinterpret_cast<uint32_t*>(take(4));
    a.part_valid = reinterpret_cast<int32_t*>(take(4 * a.groups * a.splits));
    a.part_counts = reinterpret_cast<int32_t*>(take(a.splits > 1 ? 4 * a.groups * a.splits * a.cols : 0));
    return at;
}

}  // namespace

extern "C" {

int fasgd_dropout(const fasgd_dropout_args* u, void* stream) {
    const char* call = "fasgd_dropout";
    if (u == nullptr) return fail(FASGD_EINVAL, "%s: no arguments", call);
    if (int rc = check_shape(call, u->rows, u->cols, kRowsMax, u->dtype)) return rc;
    const int64_t size = dtype_size(u->dtype);
    fasgd::DropoutArgs a;
    a.ld_x = u->ld_x;
    a.ld_residual = u->ld_residual;
    a.ld_out = u->ld_out;
    if (int rc = check_matrix(call, "x", u->x, a.ld_x, u->rows, u->cols, size)) return rc;
    if (int rc = check_matrix(call, "out", u->out, a.ld_out, u->rows, u->cols, size)) return rc;
    if (u->residual != nullptr)
        if (int rc = check_matrix(call, "residual", u->residual, a.ld_residual, u->rows, u->cols, size)) return rc;
    if (int rc = fill_draws(call, a.drop, u->rate, u->seed, u->client, u->n, u->rows, u->cols)) return rc;
    const Region out = {"out", u->out, u->rows, u->cols * size, a.ld_out * size, true};
    const Region in[2] = {{"x", u->x, u->rows, u->cols * size, a.ld_x * size, false},
                          {"residual", u->residual, u->rows, u->cols * size, a.ld_residual * size, false}};
    for (const Region& r : in)
        if (!(r.p == out.p && r.step == out.step) && share(r, out))
            return fail(FASGD_EINVAL, "%s: out overlaps %s without being it", call, r.name);
    a.x = u->x;
    a.residual = u->residual;
    a.out = u->out;
    a.rows = u->rows;
    a.cols = u->cols;
    int sms = 0;
    cudaError_t st = sm_count(sms);
    if (st == cudaSuccess) st = fasgd::launch_dropout(a, u->dtype, sms, static_cast<cudaStream_t>(stream));
    return cuda_status(st, call);
}

int fasgd_join(const fasgd_join_args* u, void* stream) {
    const char* call = "fasgd_join";
    if (u == nullptr) return fail(FASGD_EINVAL, "%s: no arguments", call);
    fasgd::JoinArgs a;
    if (int rc = fill_join(call, *u, a)) return rc;
    const int64_t size = dtype_size(u->dtype);
    a.ld_h = u->ld_h;
    a.ld_z = u->ld_z;
    if ((u->y != nullptr) != (u->h != nullptr)) return fail(FASGD_EINVAL, "%s: h goes with y", call);
    if ((u->pre != nullptr) != (u->z != nullptr)) return fail(FASGD_EINVAL, "%s: z goes with pre", call);
    if (u->h != nullptr)
        if (int rc = check_matrix(call, "h", u->h, a.ld_h, u->rows, u->cols, size)) return rc;
    if (u->z != nullptr)
        if (int rc = check_matrix(call, "z", u->z, a.ld_z, u->rows, u->cols, size)) return rc;
    a.h = u->h;
    a.z = u->z;
    const int64_t w = u->cols * size, vec = u->cols * 4;
    const Region r[] = {{"x", u->x, u->rows, w, a.ld_x * size, false},
                        {"y", u->y, u->rows, w, a.ld_y * size, false},
                        {"h", u->h, u->rows, w, a.ld_h * size, true},
                        {"z", u->z, u->rows, w, a.ld_z * size, true},
                        block("post", u->post, vec, false),
                        block("post_bias", u->post_bias, vec, false),
                        block("gate", u->gate, u->groups * u->cols * (a.gate_f32 ? 4 : size), false),
                        block("pre", u->pre, vec, false),
                        block("pre_bias", u->pre_bias, vec, false),
                        block("stats", u->stats, u->rows * 16, true)};
    if (int rc = check_shared(call, r, sizeof r / sizeof r[0])) return rc;
    int sms = 0;
    cudaError_t st = sm_count(sms);
    if (st == cudaSuccess) st = fasgd::launch_join(a, u->dtype, sms, static_cast<cudaStream_t>(stream));
    return cuda_status(st, call);
}

int64_t fasgd_join_workspace(const fasgd_join_args* u) {
    const char* call = "fasgd_join_workspace";
    if (u == nullptr) {
        fail(FASGD_EINVAL, "%s: no arguments", call);
        return -1;
    }
    fasgd::JoinArgs a;
    if (fill_join_grad(call, *u, a) != FASGD_OK) return -1;
    int sms = 0;
    if (cuda_status(sm_count(sms), call) != FASGD_OK) return -1;
    return lay_out(a, fasgd::join_grad_plan(a, u->dtype, sms), nullptr);
}

int fasgd_join_grad(const fasgd_join_args* u, void* stream) {
    const char* call = "fasgd_join_grad";
    if (u == nullptr) return fail(FASGD_EINVAL, "%s: no arguments", call);
    fasgd::JoinArgs a;
    if (int rc = fill_join_grad(call, *u, a)) return rc;
    const int64_t size = dtype_size(u->dtype), w = u->cols * size, vec = u->cols * 4;
    const int64_t gates = u->groups * u->cols * (a.gate_f32 ? 4 : size);
    const Region r[] = {{"x", u->x, u->rows, w, a.ld_x * size, false},
                        {"y", u->y, u->rows, w, a.ld_y * size, false},
                        {"dh", u->dh, u->rows, w, a.ld_dh * size, false},
                        {"dz", u->dz, u->rows, w, a.ld_dz * size, false},
                        {"dx", u->dx, u->rows, w, a.ld_dx * size, true},
                        {"dy", u->dy, u->rows, w, a.ld_dy * size, true},
                        block("post", u->post, vec, false),
                        block("post_bias", u->post_bias, vec, false),
                        block("gate", u->gate, gates, false),
                        block("pre", u->pre, vec, false),
                        block("stats", u->stats, u->rows * 16, false),
                        block("dpost", u->dpost, vec, true),
                        block("dpost_bias", u->dpost_bias, vec, true),
                        block("dgate", u->dgate, gates, true),
                        block("dpre", u->dpre, vec, true),
                        block("dpre_bias", u->dpre_bias, vec, true),
                        block("workspace", u->workspace, u->workspace_bytes, true)};
    if (int rc = check_shared(call, r, sizeof r / sizeof r[0])) return rc;
    int sms = 0;
    cudaError_t st = sm_count(sms);
    if (st != cudaSuccess) return cuda_status(st, call);
    const int64_t need = lay_out(a, fasgd::join_grad_plan(a, u->dtype, sms), static_cast<char*>(u->workspace));
    if (need > 0 && (u->workspace == nullptr || !aligned(u->workspace, 16) || u->workspace_bytes < need))
        return fail(FASGD_EINVAL, "%s: workspace must be 16-byte aligned and hold %lld bytes", call,
                    (long long)need);
    st = fasgd::launch_join_grad(a, u->dtype, sms, static_cast<cudaStream_t>(stream));
    return cuda_status(st, call);
}

int64_t fasgd_balance_workspace(const fasgd_balance_args* u) {
    const char* call = "fasgd_balance_workspace";
    if (u == nullptr) {
        fail(FASGD_EINVAL, "%s: no arguments", call);
        return -1;
    }
    if (check_balance_shape(call, *u) != FASGD_OK) return -1;
    fasgd::BalanceArgs a = {};
    a.rows = u->rows;
    a.cols = u->cols;
    a.groups = u->groups;
    a.top = u->top;
    return lay_out(a, nullptr);
}

int fasgd_balance(const fasgd_balance_args* u, void* stream) {
    const char* call = "fasgd_balance";
    if (u == nullptr) return fail(FASGD_EINVAL, "%s: no arguments", call);
    if (int rc = check_balance_shape(call, *u)) return rc;
    const int64_t size = dtype_size(u->dtype);
    fasgd::BalanceArgs a = {};
    a.ld_logits = u->ld_logits;
    a.ld_dlogits = u->ld_dlogits;
    if (int rc = check_matrix(call, "logits", u->logits, a.ld_logits, u->rows, u->cols, size)) return rc;
    if (u->dlogits != nullptr)
        if (int rc = check_matrix(call, "dlogits", u->dlogits, a.ld_dlogits, u->rows, u->cols, size)) return rc;
    if (u->chosen == nullptr || !aligned(u->chosen, 4) || u->counts == nullptr || !aligned(u->counts, 4) ||
        !aligned(u->upstream, 4) || !aligned(u->loss, 4))
        return fail(FASGD_EINVAL, "%s: chosen and counts must not be NULL; upstream and loss are 4-byte aligned", call);
    if (!std::isfinite(u->balance_scale) || !std::isfinite(u->z_scale))
        return fail(FASGD_EINVAL, "%s: balance_scale and z_scale must be finite", call);
    a.rows = u->rows;
    a.cols = u->cols;
    a.groups = u->groups;
    a.group_rows = u->rows / u->groups;
    a.top = u->top;
    const int64_t need = lay_out(a, static_cast<char*>(u->workspace));
    if (u->workspace == nullptr || !aligned(u->workspace, 16) || u->workspace_bytes < need)
        return fail(FASGD_EINVAL, "%s: workspace must be 16-byte aligned and hold %lld bytes", call,
                    (long long)need);
    const Region r[] = {{"logits", u->logits, u->rows, u->cols * size, a.ld_logits * size, false},
                        {"dlogits", u->dlogits, u->rows, u->cols * size, a.ld_dlogits * size, true},
                        block("chosen", u->chosen, u->rows * u->top * 4, false),
                        block("valid", u->valid, u->rows, false),
                        block("upstream", u->upstream, 4, false),
                        block("counts", u->counts, u->groups * u->cols * 4, true),
                        block("loss", u->loss, 12, true),
                        block("workspace", u->workspace, u->workspace_bytes, true)};
    if (int rc = check_shared(call, r, sizeof r / sizeof r[0])) return rc;
    a.logits = u->logits;
    a.chosen = u->chosen;
    a.valid = u->valid;
    a.upstream = u->upstream;
    a.dlogits = u->dlogits;
    a.counts = u->counts;
    a.loss = u->loss;
    a.balance_scale = u->balance_scale;
    a.z_scale = u->z_scale;
    int sms = 0;
    cudaError_t st = sm_count(sms);
    if (st == cudaSuccess) st = fasgd::launch_balance(a, u->dtype, sms, static_cast<cudaStream_t>(stream));
    return cuda_status(st, call);
}

}  // extern "C"
