// The gated linear recurrence of a rollout (include/autoverse.h, av_scan, av_scan_backward):
//
//   s_t = a_t s_{t-1} + b_t,   b_t = x_t or (1 - a_t) x_t,   a step that is cut drops s_{t-1}.
//
// Steps compose: a span of steps maps the state s coming in to A s + B, with A the product of
// its gates and B what the span gives from nothing; spans (A1, B1), (A2, B2) in a row give
// (A2 A1, A2 B1 + B2).  A span holding a cut maps every state to B; its A is set to NaN, which
// says so (a span whose gates make A a NaN has a B that is NaN too, so the reading is the same).
//
// A workgroup owns 64 V neighbouring columns (b, d), V of them a lane, so that a wave's access is
// one row segment, and takes them through time in tiles of W x K steps: each of its W waves holds
// K consecutive steps in registers, reduces them to (A, B), shares that through LDS, composes
// the waves before it to get its own state, and writes its K steps.  Memory is read and
// written once.  Where the columns are too few to fill the device, time is cut into S chunks of whole
// tiles: a first kernel reduces every chunk but the last to its (A, B), and the chunk's workgroups
// compose the chunks before theirs.  The order of all sums is fixed by the sizes alone.
//
// The gradient is the same recurrence run the other way: with lam_t the gradient of s_t and
// c_t that of s_{t-1} through step t, lam_t = dy_t + c_{t+1} and c_t = a_t lam_t (0 where cut).
//
// Both directions and both time orders are one code: the host points every tensor at the first
// processed step and gives its step stride a sign; q counts processed steps.
#include <algorithm>

#include "av_internal.h"
#include "learn_types.h"

namespace av {
namespace {

constexpr int kWaves = 8;       // most waves of a workgroup
constexpr int kFill = 512;      // workgroups that fill the device's 256 compute units

// 1 / (1 + e^-g) and its complement, each to full relative precision.
__device__ inline void gate_pair(float g, float &a, float &rest) {
    const float e = __expf(-fabsf(g));
    const float big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
    a = g >= 0.0f ? big : small;
    rest = g >= 0.0f ? small : big;
}

__device__ inline float follow(float2 span, float s) {
    return span.x != span.x ? span.y : fmaf(span.x, s, span.y);
}

// What a lane keeps of its place: the column, and where its elements start.
template <int V> struct Column {
    int n;                      // first column, n = b * D + d
    bool live;
    int64_t b, d;
};

template <int V> __device__ inline Column<V> column_of(const ScanArgs &p, int lane) {
    Column<V> c;
    const int64_t n = (int64_t(blockIdx.x) * 64 + lane) * V;
    c.live = n < p.N;
    c.n = int(c.live ? n : p.N - V);          // a lane past the end repeats the last columns
    c.b = uint32_t(c.n) / uint32_t(p.D);
    c.d = c.n - c.b * p.D;
    return c;
}

// K steps of one wave as they come from memory.
template <typename T, int V, int K, bool kX, bool kGate> struct Steps {
    Vec<T, V> x[kX ? K : 1], g[kGate ? K : 1], e[K];
    uint8_t cut[K];
};

// The kernels' view of one direction.  kBack: e is dy, and x is read only where gated; else e
// holds x itself.
template <typename T, int V, int K, bool kGated, bool kCol, bool kBack>
struct Reader {
    static constexpr bool kX = kBack && kGated;
    using Raw = Steps<T, V, K, kX, !kCol>;
    const ScanArgs &p;
    const T *x, *g, *e;
    const uint8_t *cut;
    int64_t xs, gs, es;
    float ca[V], cr[V];                       // a gate per value: a and 1 - a

    __device__ Reader(const ScanArgs &p, const Column<V> &c) : p(p) {
        x = static_cast<const T *>(p.x) + c.b * p.x_row + c.d;
        xs = p.x_step;
        e = kBack ? static_cast<const T *>(p.dy) + c.b * p.dy_row + c.d : x;
        es = kBack ? p.dy_step : xs;
        g = static_cast<const T *>(p.gate) + (kCol ? c.d : c.b * p.gate_row + c.d);
        gs = p.gate_step;
        cut = p.cut ? p.cut + c.b * p.cut_row : nullptr;
        if (kCol) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                ca[v] = to_f32(g[v]);
                cr[v] = 1.0f;
                if (kGated) gate_pair(ca[v], ca[v], cr[v]);
            }
        }
    }

    // Steps q .. q + K - 1; past `end` the last step is read again.
    __device__ void load(Raw &r, int64_t q, int64_t end) const {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int64_t t = min(q + k, end - 1);
            if (kX) r.x[k] = *reinterpret_cast<const Vec<T, V> *>(x + t * xs);
            if (!kCol) r.g[k] = *reinterpret_cast<const Vec<T, V> *>(g + t * gs);
            r.e[k] = *reinterpret_cast<const Vec<T, V> *>(e + t * es);
        }
        if (cut) {
#pragma unroll
            for (int k = 0; k < K; ++k) r.cut[k] = cut[min(q + k, end - 1) * p.cut_step];
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) r.cut[k] = 0;
        }
    }

    __device__ void gate(const Raw &r, int k, int v, float &a, float &rest) const {
        if (kCol) {
            a = ca[v];
            rest = cr[v];
        } else {
            a = to_f32(r.g[k].v[v]);
            rest = 1.0f;
            if (kGated) gate_pair(a, a, rest);
        }
    }

    // The span of the n (<= K) steps held in r.
    __device__ void span(const Raw &r, int n, float2 (&s)[V]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = make_float2(1.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (k >= n) break;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float a, rest;
                gate(r, k, v, a, rest);
                const float in = to_f32(r.e[k].v[v]);
                if (kBack) {
                    s[v].y = r.cut[k] ? 0.0f : a * (s[v].y + in);
                } else {
                    const float b = kGated ? rest * in : in;
                    s[v].y = r.cut[k] ? b : fmaf(a, s[v].y, b);
                }
                s[v].x = r.cut[k] ? __builtin_nanf("") : s[v].x * a;
            }
        }
    }
};

// Composes the spans of the waves in LDS: `state` becomes the state after all of them, `mine`
// the one that wave w starts from.
template <int V>
__device__ inline void compose(const float2 *spans, int W, int w, int lane, float (&state)[V],
                               float (&mine)[V]) {
    for (int j = 0; j < W; ++j) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (j == w) mine[v] = state[v];
            state[v] = follow(spans[(j * 64 + lane) * V + v], state[v]);
        }
    }
}

// First kernel of a recurrence cut into chunks: slot 0 of the workspace takes the state coming in
// (as a span that gives it), slot s + 1 the span of chunk s.
template <typename T, int V, int K, bool kGated, bool kCol, bool kBack>
__global__ void __launch_bounds__(64 * kWaves) scan_chunks_kernel(ScanArgs p) {
    __shared__ float2 spans[kWaves * 64 * V];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int W = blockDim.x >> 6;
    const Column<V> c = column_of<V>(p, lane);
    const Reader<T, V, K, kGated, kCol, kBack> in(p, c);
    const int64_t begin = int64_t(blockIdx.y) * p.chunk, part = p.chunk / W;
    float2 total[V];
#pragma unroll
    for (int v = 0; v < V; ++v) total[v] = make_float2(1.0f, 0.0f);
    // the chunk is whole (the last one has no part here) and so is each wave's share of it
    const int64_t from = begin + w * part, to = from + part;
    for (int64_t q = from; q < to; q += K) {
        typename Reader<T, V, K, kGated, kCol, kBack>::Raw raw;
        in.load(raw, q, to);
        float2 s[V];
        in.span(raw, K, s);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float y = follow(s[v], total[v].y);
            total[v] = make_float2(s[v].x * total[v].x, y);
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) spans[(w * 64 + lane) * V + v] = total[v];
    __syncthreads();
    if (w != 0 || !c.live) return;
    float2 *slots = static_cast<float2 *>(p.slots);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float2 s = spans[lane * V + v];
        for (int j = 1; j < W; ++j) {
            const float2 next = spans[(j * 64 + lane) * V + v];
            s = make_float2(next.x * s.x, follow(next, s.y));
        }
        slots[int64_t(blockIdx.y + 1) * p.N + c.n + v] = s;
        if (blockIdx.y == 0)
            slots[c.n + v] = make_float2(__builtin_nanf(""), p.first ? p.first[c.n + v] : 0.0f);
    }
}

template <typename T, int V, int K, bool kGated, bool kCol, bool kBack>
__global__ void __launch_bounds__(64 * kWaves) scan_kernel(ScanArgs p) {
    __shared__ float2 spans[2][kWaves * 64 * V];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int W = blockDim.x >> 6;
    const Column<V> c = column_of<V>(p, lane);
    Reader<T, V, K, kGated, kCol, kBack> in(p, c);
    const int64_t begin = int64_t(blockIdx.y) * p.chunk;
    const int64_t end = min(p.T, begin + p.chunk);
    float state[V], mine[V];
    int par = 0;
    if (p.slots) {
        // the chunks before this one: each wave composes its share of them
        const float2 *slots = static_cast<const float2 *>(p.slots);
        const int have = int(blockIdx.y) + 1, share = (have + W - 1) / W;
        float2 s[V];
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = make_float2(1.0f, 0.0f);
        for (int j = w * share; j < min(have, (w + 1) * share); ++j) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float2 next = slots[int64_t(j) * p.N + c.n + v];
                s[v] = make_float2(next.x * s[v].x, follow(next, s[v].y));
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            spans[par][(w * 64 + lane) * V + v] = s[v];
            state[v] = 0.0f;
        }
        __syncthreads();
        compose<V>(spans[par], W, w, lane, state, mine);
        par ^= 1;
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) state[v] = p.first ? p.first[c.n + v] : 0.0f;
    }
    float sum[V] = {};                        // gradient of a gate per value
    for (int64_t tile = begin; tile < end; tile += int64_t(W) * K) {
        const int64_t q = tile + w * K;
        const int n = int(max(int64_t(0), min(int64_t(K), end - q)));   // this wave's steps
        typename Reader<T, V, K, kGated, kCol, kBack>::Raw raw;
        in.load(raw, min(q, end - 1), end);
        Vec<T, V> before[kBack ? K : 1];
        if (kBack) {
            // the state before processed step q of the gradient is the output one step on
            const T *y = static_cast<const T *>(p.y) + c.b * p.y_row + c.d;
#pragma unroll
            for (int k = 0; k < K; ++k)
                before[k] = *reinterpret_cast<const Vec<T, V> *>(
                    y + min(q + k + 1, p.T - 1) * p.y_step);
        }
        if (W > 1) {
            float2 s[V];
            in.span(raw, n, s);
#pragma unroll
            for (int v = 0; v < V; ++v) spans[par][(w * 64 + lane) * V + v] = s[v];
            __syncthreads();
            compose<V>(spans[par], W, w, lane, state, mine);
            par ^= 1;
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) mine[v] = state[v];
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (k >= n) break;
            Vec<T, V> out, dg;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float a, rest;
                in.gate(raw, k, v, a, rest);
                const float e = to_f32(raw.e[k].v[v]);
                if (kBack) {
                    const float lam = e + mine[v];
                    mine[v] = raw.cut[k] ? 0.0f : a * lam;
                    float h = to_f32(before[k].v[v]);
                    if (q + k == p.T - 1) h = p.h0 ? p.h0[c.n + v] : 0.0f;
                    if (raw.cut[k]) h = 0.0f;
                    float d = lam * h;
                    if (kGated) d = lam * (h - to_f32(raw.x[k].v[v])) * (a * rest);
                    out.v[v] = from_f32<T>(kGated ? lam * rest : lam);
                    if (kCol) sum[v] += d;
                    else dg.v[v] = from_f32<T>(d);
                } else {
                    const float b = kGated ? rest * e : e;
                    mine[v] = raw.cut[k] ? b : fmaf(a, mine[v], b);
                    out.v[v] = from_f32<T>(mine[v]);
                }
            }
            if (c.live) {
                T *to = static_cast<T *>(p.out) + c.b * p.out_row + c.d + (q + k) * p.out_step;
                *reinterpret_cast<Vec<T, V> *>(to) = out;
                if (kBack && !kCol && p.dgate) {
                    T *at = static_cast<T *>(p.dgate) + c.b * p.dgate_row + c.d +
                            (q + k) * p.dgate_step;
                    *reinterpret_cast<Vec<T, V> *>(at) = dg;
                }
            }
        }
        if (W == 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) state[v] = mine[v];
        }
    }
    if (p.final && w == 0 && c.live && end == p.T) {
#pragma unroll
        for (int v = 0; v < V; ++v) p.final[c.n + v] = state[v];
    }
    if (kBack && kCol && p.part) {
        __syncthreads();
        float *red = reinterpret_cast<float *>(spans);
#pragma unroll
        for (int v = 0; v < V; ++v) red[(w * 64 + lane) * V + v] = sum[v];
        __syncthreads();
        if (w == 0 && c.live) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float s = sum[v];
                for (int j = 1; j < W; ++j) s += red[(j * 64 + lane) * V + v];
                p.part[int64_t(blockIdx.y) * p.N + c.n + v] = s;
            }
        }
    }
}

// Sums m rows of `width` floats into one row (to_type T): a workgroup takes up to 64 values, its
// threads share the rows, blockIdx.y takes a run of `run` rows.
template <typename T>
__global__ void __launch_bounds__(256) sum_rows_kernel(const float *src, int64_t m, int64_t run,
                                                       int width, int lanes, T *dst) {
    __shared__ float red[256];
    const int d = int(blockIdx.x) * lanes + int(threadIdx.x) % lanes;
    const int part = int(threadIdx.x) / lanes, parts = 256 / lanes;
    const int64_t r0 = int64_t(blockIdx.y) * run, r1 = min(m, r0 + run);
    float s = 0.0f;
    if (d < width)
        for (int64_t r = r0 + part; r < r1; r += parts) s += src[r * width + d];
    red[threadIdx.x] = s;
    __syncthreads();
    for (int half = parts / 2; half > 0; half >>= 1) {
        if (part < half) red[threadIdx.x] += red[threadIdx.x + half * lanes];
        __syncthreads();
    }
    if (part == 0 && d < width) dst[int64_t(blockIdx.y) * width + d] = from_f32<T>(red[threadIdx.x]);
}

__global__ void __launch_bounds__(256) copy_state_kernel(const float *src, float *dst, int n) {
    const int i = int(blockIdx.x) * 256 + int(threadIdx.x);
    if (i < n) dst[i] = src ? src[i] : 0.0f;
}

template <typename T>
__global__ void __launch_bounds__(256) zero_kernel(T *dst, int n) {
    const int i = int(blockIdx.x) * 256 + int(threadIdx.x);
    if (i < n) dst[i] = from_f32<T>(0.0f);
}

template <typename T, int V, int K, bool kGated, bool kCol, bool kBack>
hipError_t launch(const ScanArgs &a, const ScanPlan &plan, hipStream_t s) {
    const unsigned tiles = unsigned((a.N / V + 63) / 64);
    if (plan.chunks > 1)
        hipLaunchKernelGGL((scan_chunks_kernel<T, V, K, kGated, kCol, kBack>),
                           dim3(tiles, plan.chunks - 1), dim3(64 * plan.waves), 0, s, a);
    hipLaunchKernelGGL((scan_kernel<T, V, K, kGated, kCol, kBack>), dim3(tiles, plan.chunks),
                       dim3(64 * plan.waves), 0, s, a);
    return hipGetLastError();
}

template <typename T, int V, bool kGated>
hipError_t pick(const ScanArgs &a, const ScanPlan &plan, bool col, bool back, hipStream_t s) {
    if (back)
        return col ? launch<T, V, kScanSteps, kGated, true, true>(a, plan, s)
                   : launch<T, V, kScanSteps, kGated, false, true>(a, plan, s);
    return col ? launch<T, V, kScanSteps, kGated, true, false>(a, plan, s)
               : launch<T, V, kScanSteps, kGated, false, false>(a, plan, s);
}

template <typename T>
hipError_t run(const ScanArgs &a, const ScanPlan &plan, bool gated, bool col, bool back,
               hipStream_t s) {
    hipError_t e;
    if (plan.vec == 2)
        e = gated ? pick<T, 2, true>(a, plan, col, back, s) : pick<T, 2, false>(a, plan, col, back, s);
    else
        e = gated ? pick<T, 1, true>(a, plan, col, back, s) : pick<T, 1, false>(a, plan, col, back, s);
    if (e != hipSuccess || !back || !col || !a.dgate) return e;
    // the workgroups' sums of a gate per value: [chunks * B][D] rows, first in runs, then all
    const int64_t m = int64_t(plan.chunks) * (a.N / a.D);
    const int D = int(a.D);
    int lanes = 1;
    while (lanes < 64 && lanes < D) lanes *= 2;
    const unsigned blocks = unsigned((D + lanes - 1) / lanes);
    const float *src = a.part;
    int64_t rows = m;
    if (plan.runs > 1) {
        const int64_t each = (m + plan.runs - 1) / plan.runs;
        float *mid = a.part + m * D;
        hipLaunchKernelGGL((sum_rows_kernel<float>), dim3(blocks, plan.runs), dim3(256), 0, s, src,
                           m, each, D, lanes, mid);
        src = mid;
        rows = plan.runs;
    }
    hipLaunchKernelGGL((sum_rows_kernel<T>), dim3(blocks, 1), dim3(256), 0, s, src, rows, rows, D,
                       lanes, static_cast<T *>(a.dgate));
    return hipGetLastError();
}

size_t round16(size_t n) { return (n + 15) & ~size_t(15); }

}  // namespace

// How the sizes are shared out.  vec: two columns a lane where every access then stays one
// aligned word.  Waves: as many as the steps have use for.  Chunks of time: only where the
// columns alone leave compute units idle, and of at least one tile.
ScanPlan scan_plan(int64_t T, int64_t B, int64_t D, bool pairs, bool col, bool back) {
    ScanPlan plan;
    const int64_t N = B * D;
    plan.vec = pairs ? 2 : 1;
    plan.waves = int(std::max<int64_t>(1, std::min<int64_t>(kWaves, (T + kScanSteps - 1) / kScanSteps)));
    const int64_t tile = int64_t(plan.waves) * kScanSteps;
    const int64_t groups = (N / plan.vec + 63) / 64;
    const int64_t want = std::max<int64_t>(1, std::min((kFill + groups - 1) / groups,
                                                       (T + tile - 1) / tile));
    const int64_t tiles_each = (T + tile * want - 1) / (tile * want);
    plan.chunk = std::max<int64_t>(1, tiles_each) * tile;
    plan.chunks = int(std::max<int64_t>(1, (T + plan.chunk - 1) / plan.chunk));
    size_t bytes = 0;
    if (plan.chunks > 1) bytes = round16(size_t(plan.chunks) * size_t(N) * sizeof(float2));
    plan.part_off = bytes;
    plan.runs = 1;
    if (back && col) {
        const int64_t m = int64_t(plan.chunks) * B;
        if (m > 1024) plan.runs = int(std::min<int64_t>(64, m / 256));
        bytes += size_t(m) * size_t(D) * sizeof(float);
        if (plan.runs > 1) bytes += size_t(plan.runs) * size_t(D) * sizeof(float);
    }
    plan.bytes = bytes;
    return plan;
}

hipError_t launch_scan(const ScanArgs &a, const ScanPlan &plan, int dtype, bool gated, bool col,
                       bool back, hipStream_t s) {
    if (a.N == 0 || a.T == 0) {
        const unsigned blocks = unsigned((a.N + 255) / 256);
        if (a.final && a.N)
            hipLaunchKernelGGL(copy_state_kernel, dim3(blocks), dim3(256), 0, s, a.first, a.final,
                               int(a.N));
        if (back && col && a.dgate) {
            const int D = int(a.D);
            const dim3 g(unsigned((D + 255) / 256));
            if (dtype == AV_F32)
                hipLaunchKernelGGL((zero_kernel<float>), g, dim3(256), 0, s,
                                   static_cast<float *>(a.dgate), D);
            else
                hipLaunchKernelGGL((zero_kernel<_Float16>), g, dim3(256), 0, s,
                                   static_cast<_Float16 *>(a.dgate), D);
        }
        return hipGetLastError();
    }
    switch (dtype) {
        case AV_F32: return run<float>(a, plan, gated, col, back, s);
        case AV_F16: return run<_Float16>(a, plan, gated, col, back, s);
        default: return run<bf16_t>(a, plan, gated, col, back, s);
    }
}

}  // namespace av
