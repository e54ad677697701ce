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
// The gates' gradient takes the states.  In 32 bits they are the outputs y.  A 16-bit y has lost what a sum
// over many steps, or a difference from x, needs (one gate, 4187 rows of 5 steps in bf16: off by 19
// times the sum), so there the states are worked out again: marks, the spans from a chunk's first step to
// each of its tiles, come from a pass over x and the gates (over dy too where time is cut, in place of
// the chunks' pass), and a tile takes its waves' spans in both directions through LDS, with one barrier
// still.  One tile needs no marks.  (128 x 1024 x 256 in bf16 both ways: 138 us, with the rounded states
// 111; 65536 x 2 x 320 in f16: 212 us, 189.)
//
// Both directions and both time orders are one code: the host points every tensor at the first
// processed step and gives its step stride a sign; q counts processed steps.
#include <algorithm>

#include "av_internal.h"
#include "learn_types.h"

namespace av {
namespace {

// Steps a wave holds, and most waves of a workgroup: a lane with one column holds 8 steps, one with
// a word of columns 4, which leaves registers for more waves a SIMD (a gradient that works the states out
// takes 92 for 2 columns x 4 steps, and 160, two waves a SIMD, for 4 x 4).
constexpr int steps_of(int V) { return V == 1 ? 8 : 4; }
constexpr int waves_of(int V) { return V == 1 ? 16 : 8; }
template <typename T> constexpr int kWide = 8 / sizeof(T);      // columns of a lane's 8-byte word
constexpr int kFill = 512;      // workgroups that fill the device's 256 compute units

// 1 / (1 + e^-g) and its complement, neither as 1 less the other: each is off by up to (8 + 1.25 |g|) 2^-24 of
// itself, of which |g| comes from the exponent's rounding, and is 0 below 2^-126.  (With the rounding put
// right, 8 of them: 128 x 1024 x 256 in bf16 both ways 138 us, so 141, for weights that are small anyway.)
__device__ inline void gate_pair(float g, float &a, float &rest) {
    const float e = __expf(-fabsf(g));
    const float big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
    a = g >= 0.0f ? big : small;
    rest = g >= 0.0f ? small : big;
}

__device__ inline float follow(float2 span, float s) {
    return span.x != span.x ? span.y : fmaf(span.x, s, span.y);
}

// A lane's place: V columns of row b from value d on, n = b D + d counted over all rows.  A row takes
// lanes of V columns each; its last lane's start where V are left, so that `skip` of them are
// the lane before's too: it works on them but stores nothing of them.  A lane past the end repeats
// the last one's place and stores nothing.
struct Column {
    int n, skip;
    bool live;
    uint32_t b, d;
    bool odd;                         // some lane of the wave skips columns
};

template <int V> __device__ inline Column column_of(const ScanArgs &p, int64_t place) {
    Column c;
    const uint32_t lanes = uint32_t(p.lanes);                 // of a row
    c.live = place < p.places;
    const uint32_t at = uint32_t(c.live ? place : p.places - 1);
    c.b = at / lanes;
    const uint32_t from = (at - c.b * lanes) * V;
    c.d = min(from, uint32_t(p.D) - V);
    c.skip = int(from - c.d);
    c.n = int(c.b * uint32_t(p.D) + c.d);
    c.odd = V > 1 && __ballot(c.skip != 0) != 0;
    return c;
}

// V states of neighbouring columns.
template <int V> __device__ inline Word<float, V> states_at(const float *p, const Column &c) {
    Word<float, V> s{};
    if (p) s = load_any<Word<float, V>>(p + c.n);
    return s;
}
template <int V, typename T> __device__ inline void put_states(T *p, const Column &c,
                                                               const T (&v)[V]) {
    if (!c.odd || c.skip == 0) {
        __builtin_memcpy(p + c.n, v, sizeof v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i >= c.skip) p[c.n + i] = v[i];
    }
}

// The workgroup's group of columns.  Workgroups are dealt to the 8 XCDs in turn; here each XCD takes
// one contiguous eighth of the groups.  Neighbouring groups then meet in one XCD's cache, whose
// channels lie 256 bytes apart: dealt in turn, a wave's 256-byte rows, a power of two of bytes from
// step to step, would all fall into two of that cache's sixteen channels.
__device__ inline int64_t group_of_columns() {
    const uint32_t eighth = gridDim.x / 8, x = blockIdx.x;
    return gridDim.x % 8 ? x : x % 8 * eighth + x / 8;
}

// A tensor as one workgroup sees it: a base and a step stride in bytes that are the same for the
// whole wave, and the lane's own distance, which the host has made sure fits 32 bits; an access
// is then one scalar address and one 32-bit register.
struct Lanes {
    const char *base;
    int64_t step;
    uint32_t off;

    __device__ Lanes(const void *p, int64_t step_, int64_t row, int size, uint32_t b0,
                     const Column &c, bool rows = true)
        : base(static_cast<const char *>(p) + (rows ? b0 * row : 0) * size), step(step_ * size),
          off(((rows ? (c.b - b0) * uint32_t(row) : 0u) + c.d) * uint32_t(size)) {}
    // A place that moves along the steps; get and put access the lane's element there.
    struct Cursor {
        const char *p;
        int64_t step;
        uint32_t off;
        template <typename E> __device__ E get() const { return load_any<E>(p + off); }
        // Written past the caches: outputs are not read again by the kernel, and the inputs that
        // other workgroups still want stay (65536 x 2 x 320 in f16 both ways: 210 us, through them 227).
        // c.odd is the same for the wave, so that most waves never look at their lanes' skip.
        template <typename T, int V> __device__ void put(const Word<T, V> &e, const Column &c) const {
            char *to = const_cast<char *>(p) + off;
            if (!c.odd || c.skip == 0) {
                store_past(to, e);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (v >= c.skip) store_past(to + v * sizeof(T), e.v[v]);
            }
        }
        __device__ void next() { p += step; }
    };
    __device__ Cursor at(int q) const { return Cursor{base + q * step, step, off}; }
};

// K consecutive steps of V columns as they come from memory; kEach: with V flags, one for
// each column.
template <typename T, int V, int K, bool kX, bool kGate, bool kBefore, bool kEach> struct Raw {
    Word<T, V> e[K], g[kGate ? K : 1], x[kX ? K : 1], before[kBefore ? K : 1];
    Word<uint8_t, kEach ? V : 1> cut[K];
};

// The same in 32 bits: a step takes the state s to a s + b (to b where it is cut), with
// b = x or (1 - a) x, or, in the gradient, c to a (c + e) (to 0), e the gradient of the output.
template <int V, int K, bool kRest, bool kEach> struct Work {
    float a[K][V], b[K][V], rest[kRest ? K : 1][V];
    Word<uint8_t, kEach ? V : 1> flags[K];
    __device__ bool cut(int k, int v) const { return flags[k].v[kEach ? v : 0] != 0; }
};

// What of a tile's tensors is read: all, or only what a span of the recurrence that is processed needs, or,
// in the gradient, a span of the states.
enum Part { kAll, kSpan, kStates };

// One direction's view of the tensors.  kBack: e is dy and `before` the state before the step, of which
// kAgain reads none but x; without it x is read only where gated.  Else e is x.
template <typename T, int V, int K, bool kGated, bool kCol, bool kBack, bool kAgain, bool kEach>
struct Reader {
    static constexpr bool kX = kBack && (kGated || kAgain), kRest = kBack && kGated;
    static constexpr bool kBefore = kBack && !kAgain;
    using In = Raw<T, V, K, kX, !kCol, kBefore, kEach>;
    using Out = Work<V, K, kRest, kEach>;
    using Values = Word<T, V>;
    using Flags = Word<uint8_t, kEach ? V : 1>;
    Lanes x, g, e, y, cut;
    int steps;
    bool cuts;
    float ca[V], cr[V];                       // a gate per value: a and 1 - a

    __device__ Reader(const ScanArgs &p, const Column &c, uint32_t b0)
        : x(p.x, p.x_step, p.x_row, sizeof(T), b0, c),
          g(p.gate, p.gate_step, p.gate_row, sizeof(T), b0, c, !kCol),
          e(kBack ? p.dy : p.x, kBack ? p.dy_step : p.x_step, kBack ? p.dy_row : p.x_row, sizeof(T),
            b0, c),
          y(p.y, p.y_step, p.y_row, sizeof(T), b0, c),
          cut(p.cut, p.cut_step, p.cut_row, 1, b0,
              Column{c.n, 0, c.live, c.b, p.each ? c.d : 0, false}),
          steps(int(p.T)), cuts(p.cut != nullptr) {
        if (kCol) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t d = uint32_t(c.n + i) % uint32_t(p.width);
                ca[i] = to_f32(static_cast<const T *>(p.gate)[d]);
                cr[i] = 1.0f;
                if (kGated) gate_pair(ca[i], ca[i], cr[i]);
            }
        }
    }

    // Steps q .. q + K - 1; past `end` the last step is read again.
    template <Part kPart> __device__ void load(In &r, int q, int end) const {
        q = min(q, end - 1);
        // the state before processed step q of the gradient is the output one step on
        Lanes::Cursor pe = e.at(q), pg = g.at(q), px = x.at(q), pc = cut.at(q),
                      py = y.at(min(q + 1, steps - 1));
        const bool whole = q + K < end;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (kPart != kStates) r.e[k] = pe.template get<Values>();
            if (!kCol) r.g[k] = pg.template get<Values>();
            if (kX && kPart != kSpan) r.x[k] = px.template get<Values>();
            if (kBefore && kPart == kAll) r.before[k] = py.template get<Values>();
            if (whole || q + k + 1 < end) {
                pe.next();
                if (!kCol) pg.next();
                if (kX) px.next();
            }
            if (kBefore && (whole || q + k + 2 < steps)) py.next();
        }
        if (cuts) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                r.cut[k] = pc.template get<Flags>();
                if (whole || q + k + 1 < end) pc.next();
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) r.cut[k] = Flags{};
        }
    }

    // The first n steps in r in 32 bits; the others become steps that change nothing.
    __device__ void unpack(In &r, int n, Out &o) const {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            o.flags[k] = r.cut[k];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float a = ca[v], rest = cr[v];
                if (!kCol) {
                    a = to_f32(r.g[k].v[v]);
                    rest = 1.0f;
                    if (kGated) gate_pair(a, a, rest);
                }
                const float in = to_f32(r.e[k].v[v]);
                o.a[k][v] = a;
                o.b[k][v] = !kBack && kGated ? rest * in : in;
                if (kRest) o.rest[k][v] = rest;
            }
        }
        if (n < K) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (k < n) continue;
                o.flags[k] = Flags{};
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    o.a[k][v] = 1.0f;
                    o.b[k][v] = 0.0f;
                    if (kRest) o.rest[k][v] = 0.0f;
                }
                if (kAgain) r.x[k] = Values{};
            }
        }
    }

    static __device__ void span(const Out &o, float2 (&s)[V]) {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = make_float2(1.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (kBack) s[v].y = o.cut(k, v) ? 0.0f : o.a[k][v] * (s[v].y + o.b[k][v]);
                else s[v].y = o.cut(k, v) ? o.b[k][v] : fmaf(o.a[k][v], s[v].y, o.b[k][v]);
                s[v].x = o.cut(k, v) ? __builtin_nanf("") : s[v].x * o.a[k][v];
            }
    }

    // What step k of the recurrence adds to its state, for the gradient.
    static __device__ float taken(const In &r, const Out &o, int k, int v) {
        const float x = to_f32(r.x[kX ? k : 0].v[v]);
        return kGated ? o.rest[kRest ? k : 0][v] * x : x;
    }
    // The span of the states over these steps, which the gradient holds last step first.
    static __device__ void states_span(const In &r, const Out &o, float2 (&s)[V]) {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = make_float2(1.0f, 0.0f);
#pragma unroll
        for (int k = K - 1; k >= 0; --k)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float b = taken(r, o, k, v);
                s[v].y = o.cut(k, v) ? b : fmaf(o.a[k][v], s[v].y, b);
                s[v].x = o.cut(k, v) ? __builtin_nanf("") : s[v].x * o.a[k][v];
            }
    }
    // The states before these steps, from the one before the first of them (step K - 1 here), which is
    // taken through all.
    static __device__ void states(const In &r, const Out &o, float (&s)[V], float (&came)[K][V]) {
#pragma unroll
        for (int k = K - 1; k >= 0; --k)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float b = taken(r, o, k, v);
                came[k][v] = o.cut(k, v) ? 0.0f : s[v];
                s[v] = o.cut(k, v) ? b : fmaf(o.a[k][v], s[v], b);
            }
    }

    // Takes V states through step k: the output, and the gradient of the gate.  first: this is the
    // recurrence's first step (the gradient's last), whose state before is h; or came holds those of
    // all steps.
    static __device__ void step(const In &r, const Out &o, int k, bool first, const Word<float, V> &h,
                                const float (&came)[kAgain ? K : 1][V], float (&state)[V],
                                float (&out)[V], float (&dgate)[V]) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float a = o.a[k][v];
            if (kBack) {
                const float lam = o.b[k][v] + state[v];
                state[v] = o.cut(k, v) ? 0.0f : a * lam;
                float s;
                if constexpr (kAgain) {
                    s = came[k][v];
                } else {
                    s = first ? h.v[v] : to_f32(r.before[k].v[v]);
                    s = o.cut(k, v) ? 0.0f : s;
                }
                out[v] = kGated ? lam * o.rest[k][v] : lam;
                // lam (s - x) a (1 - a), or lam s
                dgate[v] = kGated ? out[v] * a * (s - to_f32(r.x[k].v[v])) : lam * s;
            } else {
                state[v] = o.cut(k, v) ? o.b[k][v] : fmaf(a, state[v], o.b[k][v]);
                out[v] = state[v];
            }
        }
    }
};

template <typename T, int V> __device__ inline Word<T, V> rounded(const float (&f)[V]) {
    Word<T, V> o;
#pragma unroll
    for (int v = 0; v < V; ++v) o.v[v] = from_f32<T>(f[v]);
    return o;
}

// First kernel of a recurrence cut into chunks: slot 0 of the workspace takes the state coming in
// (as a span that gives it), slot s + 1 the span of chunk s.
template <typename T, int V, bool kGated, bool kCol, bool kBack, bool kEach>
__global__ void __launch_bounds__(64 * waves_of(V)) scan_chunks_kernel(ScanArgs p) {
    constexpr int K = steps_of(V);
    __shared__ float2 spans[waves_of(V) * 64 * V];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int W = blockDim.x >> 6;
    const Column c = column_of<V>(p, group_of_columns() * 64 + lane);
    using R = Reader<T, V, K, kGated, kCol, kBack, false, kEach>;
    const R in(p, c, __builtin_amdgcn_readfirstlane(c.b));
    const int begin = int(blockIdx.y) * int(p.chunk), part = int(p.chunk) / W;
    float2 total[V];
#pragma unroll
    for (int v = 0; v < V; ++v) total[v] = make_float2(1.0f, 0.0f);
    // the chunk is whole (the last one has no part here) and so is each wave's share of it
    const int from = begin + w * part, to = from + part;
    typename R::In raw;
    in.template load<kSpan>(raw, from, to);
    for (int q = from; q < to; q += K) {
        typename R::Out work;
        in.unpack(raw, K, work);
        if (q + K < to) in.template load<kSpan>(raw, q + K, to);
        float2 s[V];
        R::span(work, s);
#pragma unroll
        for (int v = 0; v < V; ++v)
            total[v] = make_float2(s[v].x * total[v].x, follow(s[v], total[v].y));
    }
#pragma unroll
    for (int v = 0; v < V; ++v) spans[(w * 64 + lane) * V + v] = total[v];
    __syncthreads();
    if (w != 0 || !c.live) return;
    float2 *slots = static_cast<float2 *>(p.slots);
    const Word<float, V> first = states_at<V>(p.first, c);
    float2 mine[V], start[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        mine[v] = spans[lane * V + v];
        for (int j = 1; j < W; ++j) {
            const float2 next = spans[(j * 64 + lane) * V + v];
            mine[v] = make_float2(next.x * mine[v].x, follow(next, mine[v].y));
        }
        start[v] = make_float2(__builtin_nanf(""), first.v[v]);
    }
    put_states(slots + int64_t(blockIdx.y + 1) * p.N, c, mine);
    if (blockIdx.y == 0) put_states(slots, c, start);
}

// A span as the composition of `next` after it, and of two spans.
template <int V> __device__ inline void extend(float2 (&s)[V], const float2 (&next)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = make_float2(next[v].x * s[v].x, follow(next[v], s[v].y));
}

// First kernel of a gradient that works the states out again.  A workgroup goes through its chunk's tiles in
// the states' order, from the last to the first: marks[tile] takes the span of the states from the
// chunk's first step up to that tile (of the chunk's last tile nothing: they start there).  Where time is
// cut, slots take what scan_chunks_kernel says, and state_slots the same of the states, in their order of
// the chunks.  Each wave reduces its K steps of a tile; wave 0 composes the waves' spans while the others
// go on.  (128 x 1024 x 256 in bf16: 24 us, 4.9 TB/s; 65536 x 2 x 320 in f16, with the gradient's spans: 52 us.)
template <typename T, int V, bool kGated, bool kCol, bool kCut, bool kEach>
__global__ void __launch_bounds__(64 * waves_of(V)) scan_marks_kernel(ScanArgs p) {
    constexpr int K = steps_of(V), kMost = waves_of(V);
    __shared__ float2 spans[kCut ? 2 : 1][2][kMost * 64 * V];      // of the states, and of the gradient
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int W = blockDim.x >> 6, tile = W * K;
    const Column c = column_of<V>(p, group_of_columns() * 64 + lane);
    using R = Reader<T, V, K, kGated, kCol, true, true, kEach>;
    const R in(p, c, __builtin_amdgcn_readfirstlane(c.b));
    const int begin = int(blockIdx.y * uint32_t(p.chunk));
    const int end = int(min(p.T, begin + p.chunk));
    // no one asks for the span of the tile that the states reach last, unless there are more chunks
    const int stop = kCut ? begin : begin + tile;
    const int tiles = (end - begin + tile - 1) / tile;
    const int top = begin + (tiles - 1) * tile;
    int at = top;
    float2 total[V], back[V];
#pragma unroll
    for (int v = 0; v < V; ++v) total[v] = back[v] = make_float2(1.0f, 0.0f);
    float2 *marks = static_cast<float2 *>(p.marks);
    typename R::In next;
    auto load = [&](int from) { in.template load<kCut ? kAll : kStates>(next, from + w * K, end); };
    if (at >= stop) load(at);
    int par = 0;
    for (; at >= stop; at -= tile) {
        const int q = at + w * K, n = max(0, min(K, end - q));
        typename R::In raw = next;
        typename R::Out work;
        in.unpack(raw, n, work);
        if (at > stop) load(at - tile);
        float2 s[V], g[V];
        R::states_span(raw, work, s);
#pragma unroll
        for (int v = 0; v < V; ++v) spans[0][par][(w * 64 + lane) * V + v] = s[v];
        if (kCut) {
            R::span(work, g);
#pragma unroll
            for (int v = 0; v < V; ++v) spans[kCut][par][(w * 64 + lane) * V + v] = g[v];
        }
        __syncthreads();
        if (w == 0) {
            if (c.live && at < top) put_states(marks + int64_t(at / tile) * p.N, c, total);
            for (int j = W - 1; j >= 0; --j) {
#pragma unroll
                for (int v = 0; v < V; ++v) s[v] = spans[0][par][(j * 64 + lane) * V + v];
                extend(total, s);
            }
            if (kCut) {                                // the gradient comes to these steps before the others
#pragma unroll
                for (int v = 0; v < V; ++v) g[v] = spans[kCut][par][lane * V + v];
                for (int j = 1; j < W; ++j) {
#pragma unroll
                    for (int v = 0; v < V; ++v) s[v] = spans[kCut][par][(j * 64 + lane) * V + v];
                    extend(g, s);
                }
                extend(g, back);
#pragma unroll
                for (int v = 0; v < V; ++v) back[v] = g[v];
            }
        }
        par ^= 1;
    }
    if (w != 0 || !c.live) return;
    if (at >= begin && at < top) put_states(marks + int64_t(at / tile) * p.N, c, total);
    if (!kCut) return;
    const int chunks = int(gridDim.y), chunk = int(blockIdx.y);
    float2 *slots = static_cast<float2 *>(p.slots), *states = static_cast<float2 *>(p.state_slots);
    float2 start[V];
    if (chunk + 1 < chunks) put_states(slots + int64_t(chunk + 1) * p.N, c, back);
    if (chunk > 0) put_states(states + int64_t(chunks - chunk) * p.N, c, total);
    if (chunk == 0) {
        const Word<float, V> first = states_at<V>(p.first, c);
#pragma unroll
        for (int v = 0; v < V; ++v) start[v] = make_float2(__builtin_nanf(""), first.v[v]);
        put_states(slots, c, start);
    }
    if (chunk + 1 == chunks) {
        const Word<float, V> h = states_at<V>(p.h0, c);
#pragma unroll
        for (int v = 0; v < V; ++v) start[v] = make_float2(__builtin_nanf(""), h.v[v]);
        put_states(states, c, start);
    }
}

// The state that `have` slots lead to: each wave composes its share of them, all waves the shares.
template <int V>
__device__ inline void state_after(const void *of, int have, int64_t N, const Column &c, int w, int W,
                                   float2 *shares, float (&state)[V]) {
    const float2 *slots = static_cast<const float2 *>(of);
    const int lane = threadIdx.x & 63, share = (have + W - 1) / W;
    float2 s[V];
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = make_float2(1.0f, 0.0f);
    for (int j = w * share; j < min(have, (w + 1) * share); ++j) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float2 one = slots[int64_t(j) * N + c.n + v];
            s[v] = make_float2(one.x * s[v].x, follow(one, s[v].y));
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) shares[(w * 64 + lane) * V + v] = s[v];
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) state[v] = 0.0f;
    for (int j = 0; j < W; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) state[v] = follow(shares[(j * 64 + lane) * V + v], state[v]);
}

template <typename T, int V, bool kGated, bool kCol, bool kBack, bool kAgain, bool kEach>
__global__ void __launch_bounds__(64 * waves_of(V)) scan_kernel(ScanArgs p) {
    constexpr int K = steps_of(V), kMost = waves_of(V);
    // Loading a tile ahead pays where few workgroups share a compute unit; with many it only
    // costs registers, in the gradient too many (128 x 1024 x 256 in bf16: 81 us, without 76).
    constexpr bool kAhead = V == 1 || !kBack;
    __shared__ float2 spans[2][kMost * 64 * V];
    __shared__ float carry[2][64 * V];        // the state after a tile, for the next one
    __shared__ float2 state_spans[kAgain ? 2 : 1][kAgain ? kMost * 64 * V : 1];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int W = blockDim.x >> 6;
    const Column c = column_of<V>(p, group_of_columns() * 64 + lane);
    using R = Reader<T, V, K, kGated, kCol, kBack, kAgain, kEach>;
    const uint32_t b0 = __builtin_amdgcn_readfirstlane(c.b);
    const R in(p, c, b0);
    // at most 2^30 steps: kMost K more do not pass 31 bits
    const int begin = int(blockIdx.y * uint32_t(p.chunk));
    const int end = int(min(p.T, begin + p.chunk)), tile = W * K;
    typename R::In next;
    if (kAhead) in.template load<kAll>(next, begin + w * K, end);
    const Word<float, V> h = states_at<V>(kBack ? p.h0 : nullptr, c);
    float state[V];
    int par = 0;
    float reach[V];                           // the state that the recurrence brings to this chunk
    if (p.slots) {
        state_after(p.slots, int(blockIdx.y) + 1, p.N, c, w, W, spans[1], state);
        if constexpr (kAgain)
            state_after(p.state_slots, int(gridDim.y - blockIdx.y), p.N, c, w, W, state_spans[1], reach);
    } else {
        const Word<float, V> first = states_at<V>(p.first, c);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            state[v] = first.v[v];
            reach[v] = h.v[v];
        }
    }
    const Lanes out(p.out, p.out_step, p.out_row, sizeof(T), b0, c);
    const Lanes dgate(p.dgate, p.dgate_step, p.dgate_row, sizeof(T), b0, c);
    const bool with_gate = kBack && !kCol && p.dgate;
    float sum[V] = {};                        // gradient of a gate per value
    for (int at = begin; at < end; at += tile) {
        const int q = at + w * K;
        const int n = max(0, min(K, end - q));                          // this wave's steps
        if (!kAhead) in.template load<kAll>(next, q, end);
        float s0[V];                          // the state before this tile's steps, then this wave's
        if constexpr (kAgain) {
            Word<float2, V> mark;
#pragma unroll
            for (int v = 0; v < V; ++v) mark.v[v] = make_float2(1.0f, 0.0f);
            if (p.marks && at + tile < end)
                mark = load_any<Word<float2, V>>(static_cast<const float2 *>(p.marks) +
                                                 int64_t(at / tile) * p.N + c.n);
#pragma unroll
            for (int v = 0; v < V; ++v) s0[v] = follow(mark.v[v], reach[v]);
        }
        typename R::In raw = next;
        typename R::Out work;
        in.unpack(raw, n, work);
        // the next tile is on its way while this one is worked on
        if (kAhead && at + tile < end) in.template load<kAll>(next, q + tile, end);
        if (W > 1) {
            float2 s[V];
            R::span(work, s);
#pragma unroll
            for (int v = 0; v < V; ++v) spans[par][(w * 64 + lane) * V + v] = s[v];
            if constexpr (kAgain) {
                R::states_span(raw, work, s);
#pragma unroll
                for (int v = 0; v < V; ++v) state_spans[par][(w * 64 + lane) * V + v] = s[v];
            }
            __syncthreads();
            // from the state before the tile through the waves before this one
            if (at > begin) {
#pragma unroll
                for (int v = 0; v < V; ++v) state[v] = carry[par][lane * V + v];
            }
#pragma unroll 4
            for (int j = 0; j < w; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    state[v] = follow(spans[par][(j * 64 + lane) * V + v], state[v]);
            if constexpr (kAgain) {
#pragma unroll 4
                for (int j = W - 1; j > w; --j)
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        s0[v] = follow(state_spans[par][(j * 64 + lane) * V + v], s0[v]);
            }
            par ^= 1;
        }
        float came[kAgain ? K : 1][V];
        if constexpr (kAgain) R::states(raw, work, s0, came);
        Lanes::Cursor po = out.at(q), pg = dgate.at(q);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float o[V], dg[V];
            R::step(raw, work, k, q + k == in.steps - 1, h, came, state, o, dg);
            if (k < n) {                      // the others change nothing and are no one's output
                if (c.live) po.put(rounded<T, V>(o), c);
                if (with_gate && c.live) pg.put(rounded<T, V>(dg), c);
                if (kBack && kCol) {
#pragma unroll
                    for (int v = 0; v < V; ++v) sum[v] += dg[v];
                }
            }
            po.next();
            pg.next();
        }
        if (W > 1 && w == W - 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) carry[par][lane * V + v] = state[v];
        }
    }
    // the last wave went through every step (those past the end change nothing)
    if (p.final && w == W - 1 && c.live && end == in.steps) put_states(p.final, c, state);
    if (kBack && kCol && p.part) {
        __syncthreads();
        float *red = reinterpret_cast<float *>(spans);
#pragma unroll
        for (int v = 0; v < V; ++v) red[(w * 64 + lane) * V + v] = sum[v];
        __syncthreads();
        if (w == 0 && c.live) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                for (int j = 1; j < W; ++j) sum[v] += red[(j * 64 + lane) * V + v];
            put_states(p.part + int64_t(blockIdx.y) * p.N, c, sum);
        }
    }
}

// A few steps (an agent's acting step is one): a lane takes its columns through all of them.  Its
// addresses are 64 bits a lane, so any distance between rows will do.  The states are worked out again for
// four steps at a time, from h0 or, of more than 32 steps (rows far apart), from the state at the next
// border of 32, which a first pass leaves in the workspace.
constexpr int kShortSteps = 4, kShortMark = 32;
template <typename T, int V, bool kGated, bool kCol, bool kBack, bool kAgain, bool kEach>
__global__ void __launch_bounds__(256) scan_short_kernel(ScanArgs p) {
    constexpr int K = kAgain ? kShortSteps : 1;
    const Column c = column_of<V>(p, int64_t(blockIdx.x) * 256 + threadIdx.x);
    if (!c.live) return;
    using R = Reader<T, V, K, kGated, kCol, kBack, kAgain, kEach>;
    const R in(p, c, c.b);
    const Word<float, V> h = states_at<V>(kBack ? p.h0 : nullptr, c);
    Word<float, V> state = states_at<V>(p.first, c);
    const Lanes out(p.out, p.out_step, p.out_row, sizeof(T), c.b, c);
    const Lanes dgate(p.dgate, p.dgate_step, p.dgate_row, sizeof(T), c.b, c);
    float sum[V] = {};
    typename R::In raw;
    typename R::Out work;
    float came[kAgain ? K : 1][V];
    const int last = (in.steps - 1) / K * K;           // where the recurrence's first steps are
    float *marks = static_cast<float *>(p.marks);
    // takes the states from before steps from .. from + K - 1 (the recurrence's last of them first) through
    auto through = [&](int from, Word<float, V> &s) {
        if constexpr (kAgain) {
            in.template load<kStates>(raw, from, in.steps);
            in.unpack(raw, min(K, in.steps - from), work);
            R::states(raw, work, s.v, came);
        }
    };
    if (kAgain && marks) {
        Word<float, V> s = h;
        for (int at = last; at >= kShortMark; at -= K) {
            through(at, s);
            if (at % kShortMark == 0) put_states(marks + int64_t(at / kShortMark - 1) * p.N, c, s.v);
        }
    }
    for (int at = 0; at < in.steps; at += K) {
        if constexpr (kAgain) {
            const int group = at / kShortMark;
            Word<float, V> s = h;
            if (marks && group < last / kShortMark)
                __builtin_memcpy(s.v, marks + int64_t(group) * p.N + c.n, sizeof s.v);
            for (int f = min(last, (group + 1) * kShortMark - K); f > at; f -= K) through(f, s);
            in.template load<kAll>(raw, at, in.steps);
            in.unpack(raw, min(K, in.steps - at), work);
            R::states(raw, work, s.v, came);
        } else {
            in.template load<kAll>(raw, at, in.steps);
            in.unpack(raw, K, work);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int q = at + k;
            if (q >= in.steps) break;
            float o[V], dg[V];
            R::step(raw, work, k, q == in.steps - 1, h, came, state.v, o, dg);
            out.at(q).put(rounded<T, V>(o), c);
            if (kBack && !kCol && p.dgate) dgate.at(q).put(rounded<T, V>(dg), c);
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += kBack && kCol ? dg[v] : 0.0f;
        }
    }
    if (p.final) put_states(p.final, c, state.v);
    if (kBack && kCol && p.part) put_states(p.part, c, sum);
}

// Sums m rows of `width` floats into one row (to type T): a workgroup takes `lanes` values at a time,
// its threads share the rows, blockIdx.y takes a run of `run` rows.
template <typename T>
__global__ void __launch_bounds__(1024) sum_rows_kernel(const float *src, int64_t m, int64_t run,
                                                        int width, int lanes, T *dst) {
    __shared__ float red[1024];
    const int part = int(threadIdx.x) / lanes, parts = 1024 / lanes;
    const int64_t r0 = int64_t(blockIdx.y) * run, r1 = min(m, r0 + run);
    for (int from = int(blockIdx.x) * lanes; from < width; from += int(gridDim.x) * lanes) {
        const int d = from + int(threadIdx.x) % lanes;
        float s = 0.0f;
        if (d < width) {
#pragma unroll 4
            for (int64_t r = r0 + part; r < r1; r += parts) s += src[r * width + d];
        }
        red[threadIdx.x] = s;
        __syncthreads();
        for (int half = parts / 2; half > 0; half >>= 1) {
            if (part < half) red[threadIdx.x] += red[threadIdx.x + half * lanes];
            __syncthreads();
        }
        if (part == 0 && d < width)
            dst[int64_t(blockIdx.y) * width + d] = from_f32<T>(red[threadIdx.x]);
    }
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

// Lanes that B rows of D values take, V columns each.
int64_t scan_places(int64_t B, int64_t D, int V) { return B * ((D + V - 1) / V); }

// Workgroups over the columns; from 64 on a multiple of 8 (group_of_columns), the last ones empty.
unsigned scan_groups(int64_t places) {
    const int64_t n = (places + 63) / 64;
    return unsigned(n < 64 ? n : (n + 7) / 8 * 8);
}

template <typename T, int V, bool kGated, bool kCol, bool kBack, bool kAgain, bool kEach>
hipError_t launch(const ScanArgs &all, const ScanPlan &plan, hipStream_t s) {
    ScanArgs a = all;
    a.lanes = scan_places(1, a.D, V);
    a.places = a.N / a.D * a.lanes;
    if (plan.waves == 0) {
        const unsigned blocks = unsigned((a.places + 255) / 256);
        hipLaunchKernelGGL((scan_short_kernel<T, V, kGated, kCol, kBack, kAgain, kEach>), dim3(blocks),
                           dim3(256), 0, s, a);
        return hipGetLastError();
    }
    const unsigned groups = scan_groups(a.places);
    const dim3 block(64 * plan.waves);
    if constexpr (kAgain) {
        if (plan.chunks > 1)
            hipLaunchKernelGGL((scan_marks_kernel<T, V, kGated, kCol, true, kEach>),
                               dim3(groups, plan.chunks), block, 0, s, a);
        else if (a.marks)
            hipLaunchKernelGGL((scan_marks_kernel<T, V, kGated, kCol, false, kEach>), dim3(groups),
                               block, 0, s, a);
    } else if (plan.chunks > 1) {
        hipLaunchKernelGGL((scan_chunks_kernel<T, V, kGated, kCol, kBack, kEach>),
                           dim3(groups, plan.chunks - 1), block, 0, s, a);
    }
    hipLaunchKernelGGL((scan_kernel<T, V, kGated, kCol, kBack, kAgain, kEach>),
                       dim3(groups, plan.chunks), block, 0, s, a);
    return hipGetLastError();
}

template <typename T, int V, bool kGated, bool kEach>
hipError_t pick(const ScanArgs &a, const ScanPlan &plan, bool col, bool back, hipStream_t s) {
    if constexpr (sizeof(T) == 2 && V <= 2) {          // the gated form's gradient always has x
        if (back && (kGated || a.again))
            return col ? launch<T, V, kGated, true, true, true, kEach>(a, plan, s)
                       : launch<T, V, kGated, false, true, true, kEach>(a, plan, s);
    }
    if constexpr (sizeof(T) == 4 || !kGated) {
        if (back)
            return col ? launch<T, V, kGated, true, true, false, kEach>(a, plan, s)
                       : launch<T, V, kGated, false, true, false, kEach>(a, plan, s);
    }
    if (back) return hipErrorInvalidValue;             // no plan leads here
    return col ? launch<T, V, kGated, true, false, false, kEach>(a, plan, s)
               : launch<T, V, kGated, false, false, false, kEach>(a, plan, s);
}

template <typename T, int V>
hipError_t pick(const ScanArgs &a, const ScanPlan &plan, bool gated, bool col, bool back,
                hipStream_t s) {
    if constexpr (V > 1) {
        if (a.each)
            return gated ? pick<T, V, true, true>(a, plan, col, back, s)
                         : pick<T, V, false, true>(a, plan, col, back, s);
    }
    return gated ? pick<T, V, true, false>(a, plan, col, back, s)
                 : pick<T, V, false, false>(a, plan, col, back, s);
}

template <typename T>
hipError_t run(const ScanArgs &a, const ScanPlan &plan, bool gated, bool col, bool back,
               hipStream_t s) {
    const hipError_t e = plan.vec == 1   ? pick<T, 1>(a, plan, gated, col, back, s)
                         : plan.vec == 2 ? pick<T, 2>(a, plan, gated, col, back, s)
                                         : pick<T, kWide<T>>(a, plan, gated, col, back, s);
    if (e != hipSuccess || !back || !col || !a.dgate) return e;
    // the workgroups' sums of a gate per value: [chunks * B][D] rows, first in runs, then all
    const int64_t m = int64_t(plan.chunks) * (a.N / a.width);
    const int D = int(a.width);
    int lanes = 1;
    while (lanes < 16 && lanes < D) lanes *= 2;
    // a launch has fewer than 2^32 threads, 1024 a workgroup: very wide sums loop
    const unsigned blocks = unsigned(std::min((D + lanes - 1) / lanes, 1 << 20));
    const float *src = a.part;
    int64_t rows = m;
    if (a.runs > 1) {
        const int64_t each = (m + a.runs - 1) / a.runs;
        float *mid = a.part + m * D;
        hipLaunchKernelGGL((sum_rows_kernel<float>), dim3(blocks, a.runs), dim3(1024), 0, s, src,
                           m, each, D, lanes, mid);
        src = mid;
        rows = a.runs;
    }
    hipLaunchKernelGGL((sum_rows_kernel<T>), dim3(blocks, 1), dim3(1024), 0, s, src, rows, rows, D,
                       lanes, static_cast<T *>(a.dgate));
    return hipGetLastError();
}

size_t round16(size_t n) { return (n + 15) & ~size_t(15); }

}  // namespace

// How the sizes are shared out.  B rows of D values, all rows as one where they lie one behind the
// other; far: rows too far apart for a wave's addressing.
//   A lane takes a word of columns of up to 8 bytes, in a gradient that works the states out again of up to
//   4 (128 x 1024 x 256 in bf16: 76 us, with 8 it needs 160 registers and 87 us), as long as that leaves
//   at most a fifth of the lanes' columns to no one.  Odd widths too in 16 bits (30230 x 325 in bf16 both ways: 87 us,
//   with single columns 106), but not in 32 (777 x 33 x 129: 42 us, with single columns 39).
//   A few steps, or far rows: a lane takes its columns through all of them.
//   Else words where they still fill the device, for their longer row segments (128 x 1024 x 256 in
//   bf16: 42 us forward, with single columns 50), and one column where only that does (2048 x 64 x
//   256: 58 us, with words 151).  Where neither does, and there are more than three tiles of sixteen
//   waves of single columns (at some 2 us a tile; below that a second launch costs more), time is
//   cut into chunks, and words are taken again, smaller ones where they leave fewer lanes idle
//   (65536 x 2 x 320 in f16: 210 us both ways, with the longest 223).
//   Waves: eight, or sixteen where there is at most one uncut workgroup a compute unit, which has to
//   hide its own latency (1000 x 16384 in f32: 26.3 us, with eight 27.7; but 300 x 500 x 33, some
//   units with two workgroups: 22.1 with sixteen, 18.4 with eight).  No more of them than share an
//   uncut recurrence's tiles evenly (300 x 16384 in f32: 14.4 us, so 13.5; 140 x 500 x 40: 11.6, so
//   11.0), but with words, where memory is the bound, only if that drops more than a quarter (40 x
//   1024 x 256 in f32: 27.5 us, so 23.9; but 80 x 8192 x 64 in f16, a quarter less: 58.4, so 59.3).
ScanPlan scan_plan(int64_t T, int64_t B, int64_t D, int dtype, bool far, bool again) {
    ScanPlan plan{};
    plan.chunks = 1;
    plan.chunk = std::max<int64_t>(1, T);
    plan.vec = dtype == AV_F32 || again ? 2 : 4;
    while (plan.vec > 1 && (plan.vec > D || scan_places(1, D, plan.vec) * plan.vec * 4 > D * 5 ||
                            (dtype == AV_F32 && D % plan.vec)))
        plan.vec /= 2;
    if (B == 0 || T < 8 || far) return plan;
    const int64_t fill = int64_t(64) * kFill, N = B * D;
    const bool cut = N < fill / 2 && T > 3 * 16 * steps_of(1);
    if (!cut && scan_places(B, D, plan.vec) < fill) plan.vec = 1;
    // columns that whole workgroups have room for
    const auto room = [&](int64_t V) { return (scan_places(B, D, V) + 63) / 64 * 64 * V; };
    while (cut && plan.vec > 1 && room(plan.vec / 2) * 10 < room(plan.vec) * 9) plan.vec /= 2;
    const int64_t K = steps_of(plan.vec), groups = scan_groups(scan_places(B, D, plan.vec));
    plan.waves = int(std::min<int64_t>(cut || groups > kFill / 2 ? 8 : waves_of(plan.vec),
                                       (T + K - 1) / K));
    if (!cut) {
        const int64_t shares = (T + K - 1) / K, tiles = (shares + plan.waves - 1) / plan.waves;
        const int even = int((shares + tiles - 1) / tiles);
        if (plan.vec == 1 || even * 4 < plan.waves * 3) plan.waves = even;
    }
    if (cut) {
        const int64_t tile = plan.waves * K, tiles = (T + tile - 1) / tile;
        const int64_t want = std::min((kFill + groups - 1) / groups, tiles);
        plan.chunk = (tiles + want - 1) / want * tile;
        plan.chunks = int((T + plan.chunk - 1) / plan.chunk);
    }
    return plan;
}

// The workspace of a plan: the chunks' spans, of the states too where they are worked out again, then the
// marks of each tile (or a lane's states at its borders), then, for a gradient of `width` gates, the sums of
// them that the workgroups leave: one row of `width` for each chunk and row of the recurrence.
ScanSpace scan_space(const ScanPlan &plan, int64_t T, int64_t N, int64_t width, bool sums, bool again) {
    ScanSpace space{0, 0, 0, 0, 1, false};
    const size_t row = size_t(N) * sizeof(float2);
    if (plan.chunks > 1) space.bytes = round16(size_t(plan.chunks) * row);
    space.states_off = space.marks_off = space.bytes;
    if (again) {
        if (plan.chunks > 1) space.bytes += round16(size_t(plan.chunks) * row);
        space.marks_off = space.bytes;
        if (plan.waves == 0) {
            const int64_t n = (T + kShortMark - 1) / kShortMark;
            if (n > 1) space.bytes += round16(size_t(n - 1) * size_t(N) * sizeof(float));
        } else {
            const int64_t tile = plan.waves * steps_of(plan.vec), n = (T + tile - 1) / tile;
            if (n > 1) space.bytes += round16(size_t(plan.chunks > 1 ? n : n - 1) * row);
        }
        space.marks = space.bytes > space.marks_off;
    }
    space.part_off = space.bytes;
    if (sums) {
        const int64_t m = plan.chunks * (N / width);
        if (m > 1024) space.runs = int(std::min<int64_t>(64, m / 256));
        space.bytes += size_t(m) * size_t(width) * sizeof(float);
        if (space.runs > 1) space.bytes += size_t(space.runs) * size_t(width) * sizeof(float);
    }
    return space;
}

hipError_t launch_scan(const ScanArgs &a, const ScanPlan &plan, int dtype, bool gated, bool col,
                       bool back, hipStream_t s) {
    if (a.N == 0 || a.T == 0) {
        const unsigned blocks = unsigned((a.N + 255) / 256);
        if (a.final && a.N)
            hipLaunchKernelGGL(copy_state_kernel, dim3(blocks), dim3(256), 0, s, a.first, a.final,
                               int(a.N));
        if (back && col && a.dgate) {
            const int D = int(a.width);
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
