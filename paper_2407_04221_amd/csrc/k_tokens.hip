// Log-probabilities of given tokens with entropy and alternatives, their gradient, and the drawing
// of actions (include/autoverse.h, av_log_probs, av_log_probs_backward, av_draw_actions).
//
// With m the row's largest logit and L = log2 e,
//   t_i = (l_i - m) L,  S = sum 2^t_i,  w = sum t_i 2^t_i,
//   log p_i = (l_i - m) - ln 2 log2 S,  H = ln 2 (log2 S - w / S);
// the gradient is given (m, log2 S).  The difference is taken before the multiplication: l L - m L
// as one fused operation is shorter, but m L passes the largest number where all logits are the
// type's lowest.  A masked choice has t = -inf and adds nothing; t is bounded below in the product
// t 2^t so that its 0 is not -inf x 0.  A NaN or +inf among the logits makes S a NaN.
//
// One pass over the logits: each thread keeps its own (m, S, w) and rescales S and w when its m
// grows.  A thread takes a whole row of up to 16 choices, a wave of up to kWaveRow, else a
// workgroup.  Rows are read as aligned 16-byte words, the row's two ends element by element.
#include <algorithm>

#include "av_internal.h"
#include "learn_types.h"

namespace av {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr int kThreadRow = 16;      // longest row of one thread
constexpr int kWaveRow = 2048;      // longest row of one wave
constexpr float kNone = -__builtin_inff();

__device__ inline int64_t id_of(const TokenArgs &a, int64_t row) {
    if (a.ids_type == AV_IDS_U8) return static_cast<const uint8_t *>(a.ids)[row];
    if (a.ids_type == AV_IDS_I32) return static_cast<const int32_t *>(a.ids)[row];
    return static_cast<const int64_t *>(a.ids)[row];
}

__device__ inline float exp2_of(float t) { return __builtin_amdgcn_exp2f(t); }

// (m, S, w) of a set of logits.
struct Stat { float m, s, w; };

// What is taken from the logits: m, or 0 while every one is masked (-inf less -inf is no number).
__device__ inline float origin(float m) { return m == kNone ? 0.0f : m; }

// Moves the sums to a larger maximum.
__device__ inline void raise(Stat &a, float m) {
    const float d = (origin(a.m) - origin(m)) * kLog2e;
    const float c = a.m == kNone ? 0.0f : exp2_of(d);     // nothing summed yet: d says nothing
    a.w = c == 0.0f ? 0.0f : c * fmaf(a.s, d, a.w);
    a.s = c == 0.0f && a.s == a.s ? 0.0f : c * a.s;       // a NaN stays
    a.m = m;
}

__device__ inline void add(Stat &a, float l) {
    const float t = (l - origin(a.m)) * kLog2e;
    const float e = exp2_of(t);
    a.s += e;
    a.w = fmaf(fmaxf(t, -1.0e4f), e, a.w);
}

__device__ inline void join(Stat &a, Stat b) {
    const float m = fmaxf(a.m, b.m);
    raise(a, m);
    raise(b, m);
    a.s += b.s;
    a.w += b.w;
}

template <int kLanes> __device__ inline Stat join_lanes(Stat a) {
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) {
        Stat b;
        b.m = __shfl_xor(a.m, d);
        b.s = __shfl_xor(a.s, d);
        b.w = __shfl_xor(a.w, d);
        // both lanes of a pair add the same two parts in the same order
        const bool low = (threadIdx.x & d) == 0;
        Stat x = low ? a : b;
        join(x, low ? b : a);
        a = x;
    }
    return a;
}

// The row's results from its (m, S, w).
struct Row { float m, lse, entropy; bool bad; };

__device__ inline Row row_of(const Stat &a) {
    Row r;
    r.m = origin(a.m);
    r.bad = !(a.s < __builtin_inff());
    r.lse = a.m == kNone ? 0.0f : log2f(a.s);
    r.entropy = a.m == kNone ? 0.0f : fmaxf(0.0f, kLn2 * (r.lse - a.w / a.s));
    if (r.bad) r.m = r.lse = r.entropy = __builtin_nanf("");
    return r;
}

__device__ inline float logp_of(const Row &r, float l) { return fmaf(-kLn2, r.lse, l - r.m); }

// A choice as a number that grows with its logit and, of equal ones, with a lower index; 0: none.
__device__ inline uint64_t key_of(float l, int i) {
    if (!(l > kNone)) return 0;
    const uint32_t b = __float_as_uint(l + 0.0f);       // -0 counts as 0
    const uint32_t u = b & 0x80000000u ? ~b : b | 0x80000000u;
    return uint64_t(u) << 32 | uint32_t(~i);
}
__device__ inline float key_logit(uint64_t k) {
    const uint32_t u = uint32_t(k >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}

__device__ inline uint64_t max_lanes(uint64_t k) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const uint64_t o = __shfl_xor(static_cast<unsigned long long>(k), d);
        k = o > k ? o : k;
    }
    return k;
}

__device__ inline void put_top(const TokenArgs &a, const Row &r, int64_t row, int j, uint64_t k) {
    const bool none = k == 0 || r.bad;
    a.top_ids[row * a.top + j] = none ? -1 : int32_t(~uint32_t(k));
    a.top_logp[row * a.top + j] = r.bad ? __builtin_nanf("") : none ? kNone : logp_of(r, key_logit(k));
}

template <typename T>
__device__ inline void put_row(const TokenArgs &a, const Row &r, int64_t row, const T *l) {
    if (a.logp) {
        const int64_t id = id_of(a, row);
        float v = 0.0f;
        if (id >= 0 && id < a.A) {
            const float x = to_f32(l[id]);
            v = r.bad ? __builtin_nanf("") : x == kNone ? kNone : logp_of(r, x);
        }
        a.logp[row] = v;
    }
    if (a.entropy) a.entropy[row] = r.entropy;
    if (a.stats) {
        a.stats[2 * row] = r.m;
        a.stats[2 * row + 1] = r.lse;
    }
}

// ---- rows of at most 16 choices: one thread each ----

template <typename T, int kA> __device__ inline void load_small(const T *l, int A, float (&v)[kA]) {
#pragma unroll
    for (int i = 0; i < kA; ++i) v[i] = i < A ? to_f32(l[i]) : kNone;
}

template <typename T, int kA>
__global__ void __launch_bounds__(256) small_rows_kernel(TokenArgs a) {
    const int64_t row = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (row >= a.N) return;
    const T *l = static_cast<const T *>(a.logits) + row * a.stride;
    float v[kA];
    load_small(l, a.A, v);
    Stat st{kNone, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kA; ++i) st.m = fmaxf(st.m, v[i]);
#pragma unroll
    for (int i = 0; i < kA; ++i) add(st, v[i]);
    const Row r = row_of(st);
    put_row(a, r, row, l);
    if (a.top) {
        uint64_t last = ~uint64_t(0);
        for (int j = 0; j < a.top; ++j) {
            uint64_t best = 0;
#pragma unroll
            for (int i = 0; i < kA; ++i) {
                const uint64_t k = key_of(v[i], i);
                if (k < last && k > best) best = k;
            }
            put_top(a, r, row, j, best);
            last = best;
        }
    }
}

// What the gradient of one row needs: log2 p_i = (l - m) L - lse, d = p (c0 + c1 log2 p).
struct Back { float m, lse, g, c0, c1; int id; };

__device__ inline Back back_of(const TokenArgs &a, int64_t row) {
    Back b;
    b.m = a.in_stats[2 * row];
    b.lse = a.in_stats[2 * row + 1];
    const int64_t id = a.dlogp ? id_of(a, row) : -1;
    b.id = id >= 0 && id < a.A ? int(id) : -1;
    b.g = b.id >= 0 ? a.dlogp[row] : 0.0f;
    const float gh = a.dentropy ? a.dentropy[row] : 0.0f;
    b.c1 = -gh * kLn2;
    b.c0 = -b.g - (a.dentropy ? gh * a.in_entropy[row] : 0.0f);
    return b;
}

__device__ inline float slope(const Back &b, float l) {
    const float t = fmaf(l - b.m, kLog2e, -b.lse);
    return exp2_of(t) * fmaf(b.c1, fmaxf(t, -1.0e4f), b.c0);
}

// The gradients of n neighbouring choices from index `at` on.
template <int n> __device__ inline void slopes(const Back &b, int at, float (&v)[n]) {
    const int own = b.id - at;                 // the given token among them, unless it is masked
    float extra[n];
    const bool here = b.id >= 0 && own >= 0 && own < n;
#pragma unroll
    for (int i = 0; i < n; ++i) extra[i] = here && i == own && v[i] != kNone ? b.g : 0.0f;
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = slope(b, v[i]);
    if (here) {
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] += extra[i];
    }
}

template <typename T, int kA>
__global__ void __launch_bounds__(256) small_back_kernel(TokenArgs a) {
    const int64_t row = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (row >= a.N) return;
    const T *l = static_cast<const T *>(a.logits) + row * a.stride;
    T *d = static_cast<T *>(a.dlogits) + row * a.dstride;
    const Back b = back_of(a, row);
    float v[kA];
    load_small(l, a.A, v);
    slopes(b, 0, v);
#pragma unroll
    for (int i = 0; i < kA; ++i)
        if (i < a.A) d[i] = from_f32<T>(v[i]);
}

// ---- longer rows, as aligned words of kPer elements ----

template <typename T> struct Words {
    static constexpr int kPer = 16 / sizeof(T);
    const T *l;
    int skip, A, count;         // elements of the first word before the row, and words of the row

    __device__ Words(const TokenArgs &a, int64_t row)
        : l(static_cast<const T *>(a.logits) + row * a.stride), A(a.A) {
        skip = int(reinterpret_cast<uintptr_t>(l) / sizeof(T) % kPer);
        count = int((int64_t(skip) + A + kPer - 1) / kPer);
    }
    __device__ int first(int word) const { return word * kPer - skip; }
    __device__ bool whole(int word) const {
        return word < count && first(word) >= 0 && int64_t(first(word)) + kPer <= A;
    }
    // Elements first(word) .. + kPer - 1; -inf outside the row.
    __device__ void load(int word, float (&v)[kPer]) const {
        const int at = first(word);
        if (whole(word)) {
            const Vec<T, kPer> q = *reinterpret_cast<const Vec<T, kPer> *>(l + at);
#pragma unroll
            for (int i = 0; i < kPer; ++i) v[i] = to_f32(q.v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                v[i] = word < count && at + i >= 0 && at + i < A ? to_f32(l[at + i]) : kNone;
        }
    }
};

template <int kPer> __device__ inline float largest(const float (&v)[kPer]) {
    float m = v[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) m = fmaxf(m, v[i]);
    return m;
}

template <int kPer> __device__ inline uint64_t best_key(const float (&v)[kPer], int at) {
    uint64_t k = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const uint64_t o = key_of(v[i], at + i);
        k = o > k ? o : k;
    }
    return k;
}

// One wave per row of at most kWaveRow choices, held in registers.
template <typename T, int kWords>
__global__ void __launch_bounds__(256) wave_rows_kernel(TokenArgs a) {
    constexpr int kPer = Words<T>::kPer;
    const int lane = threadIdx.x & 63;
    const int64_t row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= a.N) return;
    const Words<T> in(a, row);
    float v[kWords][kPer];
#pragma unroll
    for (int j = 0; j < kWords; ++j) in.load(j * 64 + lane, v[j]);
    Stat st{kNone, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < kWords; ++j) st.m = fmaxf(st.m, largest(v[j]));
#pragma unroll
    for (int j = 0; j < kWords; ++j)
#pragma unroll
        for (int i = 0; i < kPer; ++i) add(st, v[j][i]);
    st = join_lanes<64>(st);
    const Row r = row_of(st);
    if (lane == 0) put_row(a, r, row, in.l);
    if (a.top) {
        uint64_t last = ~uint64_t(0);
        for (int n = 0; n < a.top; ++n) {
            uint64_t best = 0;
#pragma unroll
            for (int j = 0; j < kWords; ++j)
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const uint64_t k = key_of(v[j][i], in.first(j * 64 + lane) + i);
                    if (k < last && k > best) best = k;
                }
            best = max_lanes(best);
            if (lane == 0) put_top(a, r, row, n, best);
            last = best;
        }
    }
}

// One workgroup per row of any length.
template <typename T, int kThreads>
__global__ void __launch_bounds__(kThreads) long_rows_kernel(TokenArgs a) {
    constexpr int kPer = Words<T>::kPer, kWaves = kThreads / 64;
    __shared__ Stat stats[kWaves];
    __shared__ unsigned long long keys[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t row = blockIdx.x;
    const Words<T> in(a, row);
    Stat st{kNone, 0.0f, 0.0f};
    uint64_t best = 0;
    for (int word = tid; word < in.count; word += kThreads) {
        float v[kPer];
        in.load(word, v);
        const float m = largest(v);
        if (m > st.m) {                               // the first of equal ones stays the best
            if (a.top) best = best_key(v, in.first(word));
            raise(st, m);
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) add(st, v[i]);
    }
    st = join_lanes<64>(st);
    if (lane == 0) stats[w] = st;
    __syncthreads();
    st = stats[0];
    for (int j = 1; j < kWaves; ++j) join(st, stats[j]);
    const Row r = row_of(st);
    if (tid == 0) put_row(a, r, row, in.l);
    // alternatives one after another: the best of the threads' best; the wave that held it
    // finds its thread's next in that thread's words
    for (int n = 0; n < a.top; ++n) {
        const uint64_t mine = max_lanes(best);
        if (lane == 0) keys[w] = mine;
        __syncthreads();
        uint64_t top = keys[0];
        for (int j = 1; j < kWaves; ++j) top = keys[j] > top ? keys[j] : top;
        if (tid == 0) put_top(a, r, row, n, top);
        if (top != 0 && mine == top) {
            const int owner = __ffsll(__ballot(best == top)) - 1;
            uint64_t next = 0;
            for (int word = w * 64 + owner + lane * kThreads; word < in.count;
                 word += 64 * kThreads) {
                float v[kPer];
                in.load(word, v);
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const uint64_t k = key_of(v[i], in.first(word) + i);
                    if (k < top && k > next) next = k;
                }
            }
            next = max_lanes(next);
            if (lane == owner) best = next;
        }
        __syncthreads();
    }
}

// Gradient of rows of any length; kSame: dlogits' rows are as far into a word as the logits'.
// blockIdx.y, and the threads, share a row's words.
template <typename T, bool kSame>
__global__ void __launch_bounds__(256) long_back_kernel(TokenArgs a, int per_row) {
    constexpr int kPer = Words<T>::kPer;
    const int64_t row = blockIdx.x;
    const Words<T> in(a, row);
    T *d = static_cast<T *>(a.dlogits) + row * a.dstride;
    const Back b = back_of(a, row);
    for (int word = int(blockIdx.y) * 256 + threadIdx.x; word < in.count; word += per_row * 256) {
        float v[kPer];
        in.load(word, v);
        const int at = in.first(word);
        slopes(b, at, v);
        Vec<T, kPer> o;
#pragma unroll
        for (int i = 0; i < kPer; ++i) o.v[i] = from_f32<T>(v[i]);
        if (kSame && in.whole(word)) {
            *reinterpret_cast<Vec<T, kPer> *>(d + at) = o;
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (at + i >= 0 && at + i < a.A) d[at + i] = o.v[i];
        }
    }
}

// The same for rows of at most kWaveRow choices, a wave each.
template <typename T, bool kSame>
__global__ void __launch_bounds__(256) wave_back_kernel(TokenArgs a) {
    constexpr int kPer = Words<T>::kPer;
    const int64_t row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= a.N) return;
    const Words<T> in(a, row);
    T *d = static_cast<T *>(a.dlogits) + row * a.dstride;
    const Back b = back_of(a, row);
    for (int word = threadIdx.x & 63; word < in.count; word += 64) {
        float v[kPer];
        in.load(word, v);
        const int at = in.first(word);
        slopes(b, at, v);
        Vec<T, kPer> o;
#pragma unroll
        for (int i = 0; i < kPer; ++i) o.v[i] = from_f32<T>(v[i]);
        if (kSame && in.whole(word)) {
            *reinterpret_cast<Vec<T, kPer> *>(d + at) = o;
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (at + i >= 0 && at + i < a.A) d[at + i] = o.v[i];
        }
    }
}

// ---- drawing ----

// In 64 bits, so that where the sum passes u is a property of the logits and not of the order or
// the type of the sum.  Rows of up to kA = 4 kLanes choices, four neighbouring ones a lane.
template <typename T, int kLanes>
__global__ void __launch_bounds__(256) draw_kernel(TokenArgs a) {
    const int lane = threadIdx.x % kLanes;
    const int64_t row = int64_t(blockIdx.x) * (256 / kLanes) + threadIdx.x / kLanes;
    const bool live = row < a.N;
    const T *l = static_cast<const T *>(a.logits) + (live ? row : a.N - 1) * a.stride;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = lane * 4 + i < a.A ? to_f32(l[lane * 4 + i]) : kNone;
    float m = largest(v);
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, kLanes));
    double e[4], sum = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e[i] = v[i] == kNone ? 0.0 : exp(double(v[i]) - double(m));
        sum += e[i];
        e[i] = sum;                                   // up to and with choice i
    }
    double upto = sum;                                // of the lanes up to and with this one
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) {
        const double o = __shfl_up(upto, d, kLanes);
        if (lane >= d) upto += o;
    }
    const double total = __shfl(upto, kLanes - 1, kLanes);
    double before = __shfl_up(upto, 1, kLanes);
    if (lane == 0) before = 0.0;
    const double aim = live ? double(a.uniform[row]) * total : 0.0;
    int pick = 1 << 20, alive = -1;
#pragma unroll
    for (int i = 3; i >= 0; --i) {
        if (v[i] > kNone && alive < 0) alive = lane * 4 + i;
        if (v[i] > kNone && before + e[i] > aim) pick = lane * 4 + i;
    }
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) {
        pick = min(pick, __shfl_xor(pick, d, kLanes));
        alive = max(alive, __shfl_xor(alive, d, kLanes));
    }
    if (pick == 1 << 20) pick = alive;
    if (!live || lane != 0) return;
    float logp = kNone;
    if (!(total < double(__builtin_inff()))) {        // a NaN, or a +inf
        pick = 0;
        logp = __builtin_nanf("");
    } else if (pick < 0) {
        pick = 0;
    } else {
        logp = float(double(to_f32(l[pick])) - double(m) - log(total));
    }
    a.actions[row] = uint8_t(pick);
    if (a.logp) a.logp[row] = logp;
}

unsigned blocks_of(int64_t n, int64_t per) { return unsigned((n + per - 1) / per); }

template <typename T> int words_of(const TokenArgs &a) {     // most words a row can take
    return int((int64_t(a.A) + 16 / sizeof(T) - 2) / (16 / sizeof(T))) + 1;
}

template <typename T> hipError_t forward(const TokenArgs &a, hipStream_t s) {
    const dim3 b(256);
    if (a.A <= kThreadRow) {
        const dim3 g(blocks_of(a.N, 256));
        if (a.A <= 4) hipLaunchKernelGGL((small_rows_kernel<T, 4>), g, b, 0, s, a);
        else if (a.A <= 8) hipLaunchKernelGGL((small_rows_kernel<T, 8>), g, b, 0, s, a);
        else hipLaunchKernelGGL((small_rows_kernel<T, 16>), g, b, 0, s, a);
        return hipGetLastError();
    }
    const int lanes = blocks_of(words_of<T>(a), 64);
    if (a.A <= kWaveRow && lanes <= 8) {
        const dim3 g(blocks_of(a.N, 4));
        if (lanes <= 1) hipLaunchKernelGGL((wave_rows_kernel<T, 1>), g, b, 0, s, a);
        else if (lanes <= 2) hipLaunchKernelGGL((wave_rows_kernel<T, 2>), g, b, 0, s, a);
        else if (lanes <= 4) hipLaunchKernelGGL((wave_rows_kernel<T, 4>), g, b, 0, s, a);
        else hipLaunchKernelGGL((wave_rows_kernel<T, 8>), g, b, 0, s, a);
        return hipGetLastError();
    }
    if (a.N >= 512)
        hipLaunchKernelGGL((long_rows_kernel<T, 256>), dim3(unsigned(a.N)), b, 0, s, a);
    else
        hipLaunchKernelGGL((long_rows_kernel<T, 1024>), dim3(unsigned(a.N)), dim3(1024), 0, s, a);
    return hipGetLastError();
}

template <typename T> hipError_t backward(const TokenArgs &a, hipStream_t s) {
    const dim3 b(256);
    if (a.A <= kThreadRow) {
        const dim3 g(blocks_of(a.N, 256));
        if (a.A <= 4) hipLaunchKernelGGL((small_back_kernel<T, 4>), g, b, 0, s, a);
        else if (a.A <= 8) hipLaunchKernelGGL((small_back_kernel<T, 8>), g, b, 0, s, a);
        else hipLaunchKernelGGL((small_back_kernel<T, 16>), g, b, 0, s, a);
        return hipGetLastError();
    }
    constexpr int kPer = 16 / sizeof(T);
    const bool same = (reinterpret_cast<uintptr_t>(a.logits) -
                       reinterpret_cast<uintptr_t>(a.dlogits)) % 16 == 0 &&
                      (a.stride - a.dstride) % kPer == 0;
    if (a.A <= kWaveRow) {
        const dim3 g(blocks_of(a.N, 4));
        if (same) hipLaunchKernelGGL((wave_back_kernel<T, true>), g, b, 0, s, a);
        else hipLaunchKernelGGL((wave_back_kernel<T, false>), g, b, 0, s, a);
        return hipGetLastError();
    }
    // enough workgroups for the device where the rows are few
    const int words = words_of<T>(a);
    const int per_row = int(std::max<int64_t>(1, std::min<int64_t>(blocks_of(words, 256),
                                                                   (2048 + a.N - 1) / a.N)));
    const dim3 g(unsigned(a.N), unsigned(per_row));
    if (same) hipLaunchKernelGGL((long_back_kernel<T, true>), g, b, 0, s, a, per_row);
    else hipLaunchKernelGGL((long_back_kernel<T, false>), g, b, 0, s, a, per_row);
    return hipGetLastError();
}

template <typename T> hipError_t draw(const TokenArgs &a, hipStream_t s) {
    const dim3 b(256);
    if (a.A <= 8) hipLaunchKernelGGL((draw_kernel<T, 2>), dim3(blocks_of(a.N, 128)), b, 0, s, a);
    else if (a.A <= 64) hipLaunchKernelGGL((draw_kernel<T, 16>), dim3(blocks_of(a.N, 16)), b, 0, s, a);
    else hipLaunchKernelGGL((draw_kernel<T, 64>), dim3(blocks_of(a.N, 4)), b, 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_log_probs(const TokenArgs &a, int dtype, hipStream_t s) {
    switch (dtype) {
        case AV_F32: return forward<float>(a, s);
        case AV_F16: return forward<_Float16>(a, s);
        default: return forward<bf16_t>(a, s);
    }
}

hipError_t launch_log_probs_backward(const TokenArgs &a, int dtype, hipStream_t s) {
    switch (dtype) {
        case AV_F32: return backward<float>(a, s);
        case AV_F16: return backward<_Float16>(a, s);
        default: return backward<bf16_t>(a, s);
    }
}

hipError_t launch_draw(const TokenArgs &a, int dtype, hipStream_t s) {
    switch (dtype) {
        case AV_F32: return draw<float>(a, s);
        case AV_F16: return draw<_Float16>(a, s);
        default: return draw<bf16_t>(a, s);
    }
}

}  // namespace av
