// The learner's operators of include/autoverse.h: argument checks, all before any device work,
// and the arguments in the kernels' form.  Nothing is allocated or kept.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <utility>

#include "av_internal.h"

using namespace av;

namespace {

av_status bad(const char *fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return set_error(AV_EINVAL, buf);
}

// Makes `device` current for a scope.
class OnDevice {
public:
    explicit OnDevice(int device) {
        err_ = hipGetDevice(&old_);
        if (err_ == hipSuccess && old_ != device) {
            err_ = hipSetDevice(device);
            moved_ = err_ == hipSuccess;
        }
    }
    ~OnDevice() {
        if (moved_) (void)hipSetDevice(old_);
    }
    OnDevice(const OnDevice &) = delete;
    OnDevice &operator=(const OnDevice &) = delete;
    hipError_t error() const { return err_; }

private:
    int old_ = 0;
    bool moved_ = false;
    hipError_t err_;
};

av_status launched(const char *what, hipError_t e) {
    if (e == hipSuccess) return AV_OK;
    char buf[256];
    snprintf(buf, sizeof buf, "%s failed: %s", what, hipGetErrorString(e));
    return set_error(AV_EDEVICE, buf);
}

size_t size_of(int dtype) { return dtype == AV_F32 ? 4 : 2; }

constexpr int64_t kBig = int64_t(1) << 31, kMostSteps = int64_t(1) << 30;
constexpr int64_t kMostColumns = int64_t(1) << 28;
// Rows too far apart for a wave's addressing take their steps one after another, at a microsecond
// each where the rows are few: this many end in a tenth of a second.
constexpr int64_t kMostFar = int64_t(1) << 16;

av_status check_scan(const av_scan_config *c) {
    if (!c) return bad("cfg is NULL");
    // steps are counted in 32 bits a tile past the end; a launch has fewer than 2^32 threads, up to
    // eight a column; and a lane's distance within a row, in bytes, fits 32 bits
    if (c->steps < 0 || c->steps > kMostSteps)
        return bad("steps %lld outside [0, 2^30]", (long long)c->steps);
    if (c->rows < 0 || c->width < 1 || c->rows > kMostColumns || c->width > kMostColumns ||
        c->rows * c->width > kMostColumns)
        return bad("rows %lld, width %lld: needs rows >= 0, width >= 1, rows x width <= 2^28",
                   (long long)c->rows, (long long)c->width);
    if (c->dtype != AV_F32 && c->dtype != AV_F16 && c->dtype != AV_BF16)
        return bad("unknown dtype %d", c->dtype);
    if (c->form != AV_SCAN_LINEAR && c->form != AV_SCAN_GATED) return bad("unknown form %d", c->form);
    if ((c->reverse != 0 && c->reverse != 1) || (c->gate_per_value != 0 && c->gate_per_value != 1))
        return bad("reverse and gate_per_value must be 0 or 1");
    return AV_OK;
}

// The elements of an output must not share a place: of two dimensions the one with the longer
// stride steps over all of the other.
bool spread(int64_t step, int64_t row, const av_scan_config &c) {
    std::pair<int64_t, int64_t> dim[2] = {{step, c.steps}, {row, c.rows}};
    if (dim[1].first < dim[0].first) std::swap(dim[0], dim[1]);
    int64_t extent = c.width;
    for (const auto &d : dim) {
        if (d.second <= 1) continue;
        if (d.first < extent) return false;
        extent = d.first * (d.second - 1) + extent;
    }
    return true;
}

struct Place {
    const void *p;
    int64_t step, row;
};

// Offsets are not negative and stay far inside 64 bits.
bool reachable(int64_t step, int64_t n) {
    return step >= 0 && __int128(step) * n < (__int128(1) << 60);
}

av_status check_workspace(const void *workspace, size_t bytes, size_t needed) {
    if (needed == 0) return AV_OK;
    if (!workspace || bytes < needed)
        return bad("workspace of %zu bytes; %zu are needed", workspace ? bytes : size_t(0), needed);
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return bad("workspace is not 16-byte aligned");
    return AV_OK;
}

// The most that any layout of these sizes takes: rows apart, or as one, or far apart (some, and not too
// many steps); and, in a gradient of a 16-bit type, with the states worked out again or not.
size_t workspace_of(const av_scan_config &c, bool back) {
    const int64_t N = c.rows * c.width;
    const bool sums = back && c.gate_per_value;
    size_t most = 0;
    for (const bool again : {false, true}) {
        if (again && !(back && c.dtype != AV_F32)) break;
        auto take = [&](int64_t rows, int64_t width, bool far) {
            const ScanPlan plan = scan_plan(c.steps, rows, width, c.dtype, far, again);
            most = std::max(most, scan_space(plan, c.steps, N, c.width, sums, again).bytes);
        };
        take(c.rows, c.width, false);
        take(1, N, false);
        if (c.rows > 1 && c.steps <= kMostFar) take(c.rows, c.width, true);
    }
    return most;
}

av_status scan(const av_scan_config *cfg, const void *x, const void *gate, const uint8_t *cut,
               const float *first, const float *h0, const void *y, const void *dy, void *out,
               void *dgate, float *final, void *workspace, size_t workspace_bytes, bool back) {
    const av_scan_config &c = *cfg;
    const bool col = c.gate_per_value != 0, gated = c.form == AV_SCAN_GATED;
    const bool some = c.steps > 0 && c.rows > 0;
    // a dimension of one element has no stride to speak of
    auto place = [&](const void *p, int64_t step, int64_t row) {
        return Place{p, c.steps > 1 ? step : 0, c.rows > 1 ? row : 0};
    };
    // nor has a gate per value, and what is not read takes no part in how the columns are shared out
    Place px = place(x, c.x_step, c.x_row);
    Place pg = col ? Place{gate, 0, 0} : place(gate, c.gate_step, c.gate_row);
    Place py = place(y, c.y_step, c.y_row), pdy = place(dy, c.dy_step, c.dy_row);
    Place po = back ? place(out, c.dx_step, c.dx_row) : place(out, c.y_step, c.y_row);
    Place pdg = col ? Place{dgate, 0, 0} : place(dgate, c.dgate_step, c.dgate_row);
    Place pc = place(cut, c.cut_step, c.cut_row);
    for (const Place *a : {&px, &pg, &py, &pdy, &po, &pdg, &pc})
        if (a->p && (!reachable(a->step, c.steps) || !reachable(a->row, c.rows)))
            return bad("a stride is out of range");
    if (!spread(po.step, po.row, c)) return bad("strides of %s overlap its elements", back ? "dx" : "y");
    if (back && dgate && !col && !spread(pdg.step, pdg.row, c))
        return bad("strides of dgate overlap its elements");
    const size_t size = size_of(c.dtype);
    // a 16-bit gradient works the states out again, unless x has become y, or is not there, or no one
    // asks for the gates' gradient (the gated kernels then do without marks)
    const bool again = back && size == 2 && x && (gated || (x != y && dgate));
    const bool reads_x = !back || gated || again;
    if (!reads_x) px = Place{nullptr, 0, 0};
    const void *all[] = {px.p, gate, y, dy, out, dgate};
    for (const void *p : all)
        if (reinterpret_cast<uintptr_t>(p) % size) return bad("a tensor is not aligned to its type");
    const float *floats[] = {first, h0, final};
    for (const float *p : floats)
        if (reinterpret_cast<uintptr_t>(p) % 4) return bad("a state is not aligned to its type");

    // rows that lie one behind the other are one long row, if no flags tell them apart or each
    // value has its own
    const bool each = cut && c.width == 1 && c.rows > 1 && c.cut_row == 1;
    bool merge = c.rows > 1 && (!cut || each);
    for (const Place *a : {&px, &pg, &py, &pdy, &po, &pdg})
        if (a->p && !(col && (a == &pg || a == &pdg))) merge = merge && a->row == c.width;
    const int64_t rows = merge ? 1 : c.rows, width = merge ? c.rows * c.width : c.width;
    if (merge)
        for (Place *a : {&px, &pg, &py, &pdy, &po, &pdg}) a->row = 0;

    // a wave reaches the rows of its columns by 32-bit distances (64 lanes of up to 4 columns)
    const int64_t span = std::min(rows, 4 * 64 / width + 2);
    bool far = false;
    for (const Place *a : {&px, &pg, &py, &pdy, &po, &pdg, &pc})
        if (a->p)
            far = far || span * a->row + width >= (int64_t(1) << 32) / int64_t(a == &pc ? 1 : size);
    if (far && c.steps > kMostFar)
        return bad("%lld steps of rows too far apart: more than %lld are taken only where %lld rows "
                   "lie within 2^32 bytes",
                   (long long)c.steps, (long long)kMostFar, (long long)span);
    const ScanPlan plan = scan_plan(c.steps, rows, width, c.dtype, far, again);
    const ScanSpace space = scan_space(plan, c.steps, c.rows * c.width, c.width, back && col, again);
    if (some) {
        if (av_status st = check_workspace(workspace, workspace_bytes, workspace_of(c, back)))
            return st;
    }

    // processing order: the gradient runs against the recurrence
    const bool down = (c.reverse != 0) != back;
    const int64_t last = std::max<int64_t>(0, c.steps - 1);
    auto turn = [&](const void *p, int64_t &step, size_t bytes) -> char * {
        char *q = static_cast<char *>(const_cast<void *>(p));
        if (!down || !q) return q;
        q += last * step * int64_t(bytes);
        step = -step;
        return q;
    };
    ScanArgs a{};
    a.T = c.steps; a.N = rows * width; a.D = width; a.width = c.width; a.chunk = plan.chunk;
    a.each = merge && each; a.runs = space.runs;
    a.x = turn(px.p, px.step, size); a.x_step = px.step; a.x_row = px.row;
    a.gate = col ? gate : turn(pg.p, pg.step, size);
    a.gate_step = pg.step; a.gate_row = pg.row;
    a.y = turn(py.p, py.step, size); a.y_step = py.step; a.y_row = py.row;
    a.dy = turn(pdy.p, pdy.step, size); a.dy_step = pdy.step; a.dy_row = pdy.row;
    a.out = turn(po.p, po.step, size); a.out_step = po.step; a.out_row = po.row;
    a.dgate = col ? dgate : turn(pdg.p, pdg.step, size);
    a.dgate_step = pdg.step; a.dgate_row = pdg.row;
    a.cut = reinterpret_cast<const uint8_t *>(turn(pc.p, pc.step, 1));
    a.cut_step = pc.step; a.cut_row = pc.row;
    a.first = first; a.h0 = h0; a.final = final;
    a.again = again;
    a.slots = some && plan.chunks > 1 ? workspace : nullptr;
    if (some && space.marks && (dgate || plan.chunks > 1)) {
        a.state_slots = static_cast<char *>(workspace) + space.states_off;
        a.marks = static_cast<char *>(workspace) + space.marks_off;
    }
    a.part = back && col && dgate && some
                 ? reinterpret_cast<float *>(static_cast<char *>(workspace) + space.part_off)
                 : nullptr;
    OnDevice on(c.device);
    if (on.error() != hipSuccess) return launched("hipSetDevice", on.error());
    return launched(back ? "av_scan_backward" : "av_scan",
                    launch_scan(a, plan, c.dtype, gated, col, back,
                                static_cast<hipStream_t>(c.stream)));
}

av_status check_tokens(const av_tokens_config *c) {
    if (!c) return bad("cfg is NULL");
    if (c->rows < 0 || c->rows >= kBig) return bad("rows %lld outside [0, 2^31)", (long long)c->rows);
    if (c->choices < 1 || c->choices > kBig - 1025)
        return bad("choices %lld outside [1, 2^31 - 1025]", (long long)c->choices);
    if (c->dtype != AV_F32 && c->dtype != AV_F16 && c->dtype != AV_BF16)
        return bad("unknown dtype %d", c->dtype);
    if (!reachable(c->row_stride, c->rows)) return bad("row_stride is out of range");
    if (c->ids_type != AV_IDS_U8 && c->ids_type != AV_IDS_I32 && c->ids_type != AV_IDS_I64)
        return bad("unknown ids_type %d", c->ids_type);
    return AV_OK;
}

av_status check_top(const av_tokens_config *c) {
    if (c->top < 0 || c->top > AV_TOP_MAX) return bad("top %d outside [0, %d]", c->top, AV_TOP_MAX);
    return AV_OK;
}

TokenArgs token_args(const av_tokens_config &c, const void *logits, const void *ids) {
    TokenArgs a{};
    a.N = c.rows; a.A = int(c.choices); a.ids_type = c.ids_type;
    a.stride = c.rows > 1 ? c.row_stride : 0;
    a.logits = logits; a.ids = ids;
    return a;
}

bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

size_t ids_size(int t) { return t == AV_IDS_U8 ? 1 : (t == AV_IDS_I32 ? 4 : 8); }

}  // namespace

extern "C" {

av_status av_scan_workspace(const av_scan_config *cfg, int32_t backward, size_t *bytes) {
    set_error(AV_OK, "");
    if (av_status st = check_scan(cfg)) return st;
    if (!bytes) return bad("bytes is NULL");
    *bytes = cfg->steps > 0 && cfg->rows > 0 ? workspace_of(*cfg, backward != 0) : 0;
    return AV_OK;
}

av_status av_scan(const av_scan_config *cfg, const void *x, const void *gate, const uint8_t *cut,
                  const float *h0, void *y, float *last, void *workspace, size_t workspace_bytes) {
    set_error(AV_OK, "");
    if (av_status st = check_scan(cfg)) return st;
    if (cfg->steps > 0 && cfg->rows > 0 && (!x || !gate || !y))
        return bad("x, gate and y must not be NULL");
    return scan(cfg, x, gate, cut, h0, nullptr, nullptr, nullptr, y, nullptr, last, workspace,
                workspace_bytes, false);
}

av_status av_scan_backward(const av_scan_config *cfg, const void *x, const void *gate,
                           const uint8_t *cut, const float *h0, const void *y, const void *dy,
                           const float *dlast, void *dx, void *dgate, float *dh0, void *workspace,
                           size_t workspace_bytes) {
    set_error(AV_OK, "");
    if (av_status st = check_scan(cfg)) return st;
    if (cfg->steps > 0 && cfg->rows > 0) {
        if (!gate || !y || !dy || !dx) return bad("gate, y, dy and dx must not be NULL");
        if (cfg->form == AV_SCAN_GATED && !x) return bad("x must not be NULL in the gated form");
    }
    return scan(cfg, x, gate, cut, dlast, h0, y, dy, dx, dgate, dh0, workspace, workspace_bytes,
                true);
}

av_status av_log_probs_workspace(const av_tokens_config *cfg, size_t *bytes) {
    set_error(AV_OK, "");
    if (av_status st = check_tokens(cfg)) return st;
    if (av_status st = check_top(cfg)) return st;
    if (!bytes) return bad("bytes is NULL");
    *bytes = tokens_plan(cfg->rows, cfg->choices, cfg->top, cfg->dtype).bytes;
    return AV_OK;
}

av_status av_log_probs(const av_tokens_config *cfg, const void *logits, const void *ids,
                       float *logp, float *entropy, float *stats, float *top_logp,
                       int32_t *top_ids, void *workspace, size_t workspace_bytes) {
    set_error(AV_OK, "");
    if (av_status st = check_tokens(cfg)) return st;
    if (av_status st = check_top(cfg)) return st;
    if (cfg->rows == 0) return AV_OK;
    if (!logits) return bad("logits is NULL");
    if ((logp != nullptr) != (ids != nullptr)) return bad("logp and ids go together");
    if (cfg->top > 0 && (!top_logp || !top_ids)) return bad("top_logp and top_ids must not be NULL");
    if (!aligned(logits, size_of(cfg->dtype)) || !aligned(ids, ids_size(cfg->ids_type)) ||
        !aligned(logp, 4) || !aligned(entropy, 4) || !aligned(stats, 8) || !aligned(top_logp, 4) ||
        !aligned(top_ids, 4))
        return bad("a tensor is not aligned to its type (stats: 8 bytes)");
    const TokenPlan plan = tokens_plan(cfg->rows, cfg->choices, cfg->top, cfg->dtype);
    if (plan.bytes > 0) {
        if (av_status st = check_workspace(workspace, workspace_bytes, plan.bytes)) return st;
    }
    TokenArgs a = token_args(*cfg, logits, ids);
    a.top = cfg->top;
    a.parts = plan.parts;
    a.part_stats = workspace;
    a.part_keys = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + plan.keys_off);
    a.logp = logp; a.entropy = entropy; a.stats = stats;
    a.top_logp = top_logp; a.top_ids = top_ids;
    OnDevice on(cfg->device);
    if (on.error() != hipSuccess) return launched("hipSetDevice", on.error());
    return launched("av_log_probs",
                    launch_log_probs(a, cfg->dtype, static_cast<hipStream_t>(cfg->stream)));
}

av_status av_log_probs_backward(const av_tokens_config *cfg, const void *logits, const void *ids,
                                const float *stats, const float *entropy, const float *dlogp,
                                const float *dentropy, void *dlogits) {
    set_error(AV_OK, "");
    if (av_status st = check_tokens(cfg)) return st;
    if (cfg->rows == 0) return AV_OK;
    if (!logits || !stats || !dlogits) return bad("logits, stats and dlogits must not be NULL");
    if (dlogp && !ids) return bad("dlogp needs ids");
    if (dentropy && !entropy) return bad("dentropy needs entropy");
    if (!reachable(cfg->drow_stride, cfg->rows)) return bad("drow_stride is out of range");
    if (cfg->rows > 1 && cfg->drow_stride < cfg->choices)
        return bad("drow_stride %lld: the rows of dlogits overlap", (long long)cfg->drow_stride);
    if (!aligned(logits, size_of(cfg->dtype)) || !aligned(dlogits, size_of(cfg->dtype)) ||
        !aligned(ids, ids_size(cfg->ids_type)) || !aligned(stats, 8) || !aligned(entropy, 4) ||
        !aligned(dlogp, 4) || !aligned(dentropy, 4))
        return bad("a tensor is not aligned to its type (stats: 8 bytes)");
    TokenArgs a = token_args(*cfg, logits, ids);
    a.in_stats = stats; a.in_entropy = entropy; a.dlogp = dlogp; a.dentropy = dentropy;
    a.dlogits = dlogits;
    a.dstride = cfg->rows > 1 ? cfg->drow_stride : 0;
    OnDevice on(cfg->device);
    if (on.error() != hipSuccess) return launched("hipSetDevice", on.error());
    return launched("av_log_probs_backward",
                    launch_log_probs_backward(a, cfg->dtype, static_cast<hipStream_t>(cfg->stream)));
}

av_status av_draw_actions(const av_tokens_config *cfg, const void *logits, const float *uniform,
                          uint8_t *actions, float *logp) {
    set_error(AV_OK, "");
    if (av_status st = check_tokens(cfg)) return st;
    if (cfg->choices > 256) return bad("choices %lld: an action is one byte, at most 256",
                                       (long long)cfg->choices);
    if (cfg->rows == 0) return AV_OK;
    if (!logits || !uniform || !actions) return bad("logits, uniform and actions must not be NULL");
    if (!aligned(logits, size_of(cfg->dtype)) || !aligned(uniform, 4) || !aligned(logp, 4))
        return bad("a tensor is not aligned to its type");
    TokenArgs a = token_args(*cfg, logits, nullptr);
    a.uniform = uniform; a.actions = actions; a.logp = logp;
    OnDevice on(cfg->device);
    if (on.error() != hipSuccess) return launched("hipSetDevice", on.error());
    return launched("av_draw_actions",
                    launch_draw(a, cfg->dtype, static_cast<hipStream_t>(cfg->stream)));
}

}  // extern "C"
