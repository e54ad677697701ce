// Log-probabilities of given tokens with entropy and alternatives, their gradient, and the drawing
// of actions (include/autoverse.h, av_log_probs, av_log_probs_backward, av_draw_actions).
//
// With m the row's largest logit and L = log2 e,
//   t_i = (l_i - m) L,  S = sum 2^t_i,  w = sum t_i 2^t_i,
//   log p_i = (l_i - m) - ln 2 log2 S,  H = ln 2 (log2 S - w / S);
// the gradient is given (m, log2 S).  An S below 1.5 is 1, the largest itself, and little else: the
// others are then summed on their own, R = S - 1, so that log2 S = log2 e log1p R keeps the bits that
// 1 + R drops (logits 0 and four of -16: log p = -4.50e-7, from the sum -4.77e-7), and with it log p
// and H, which is a sum of two terms that are not negative.  (1638400 rows of 5 in f32, many of them like
// this, both ways: 29.9 us, without 29.0.)  The difference is taken before the multiplication: l L - m L
// as one fused operation is shorter, but m L passes the largest number where all logits are the
// type's lowest.  A masked choice has t = -inf and adds nothing; t is bounded below in the product
// t 2^t so that its 0 is not -inf x 0.  A NaN or +inf among the logits makes S a NaN.
//
// One pass over the logits: each thread keeps its own (m, S, w) and rescales S and w when its m
// grows.  A thread takes a whole row of up to 16 choices, 4 to 64 lanes one of up to kWaveRow, else
// a workgroup, or several.  Longer rows are read as 16-byte words wherever they start.
#include <algorithm>

#include "av_internal.h"
#include "learn_types.h"

namespace av {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr int kThreadRow = 16;      // longest row of one thread
// Longest row of one wave: 64 numbers a lane.  (20000 x 3000: in bf16 44 us as workgroups, so 31, in f32
// 50 and 46; of 4096 in f32 59 and 61; of 8192 in bf16 73 and 127.)
constexpr int kWaveRow = 4096;
// Longest row of one wave in the gradient, in 16-byte words: longer ones give each thread of a workgroup
// a word (50000 x 2040 in f32: 205 us as waves, so 139; x 1600 in bf16: 60 and 70).
constexpr int kTeamBack = 256;
// Words of all rows from which few lanes take a row, with several words each: fewer reductions and row
// results an instruction, but fewer waves.  (300000 x 148 in f32: 84 us as waves, so 37; 8000 of them
// 4.1 and 3.3; 8000 x 30 in f32 3.4 and 3.2, 8000 x 113 in f16 3.3 and 3.6.)  With alternatives, which cost
// each lane its words, only up to 64 words for kFew of them and 32 for more (200000 x 1000 in f16, 32 lanes
// or a wave: none 83 and 97, four of them 193 and 156).  The gradient four times as
// many, where the lanes' idle words are more than the last of a line (300000 x 66 in f16: 26.7 us, so
// 18.8; x 148 in f32 114 and 69; but x 113 in f16, fifteen of sixteen lanes, 30.0 and 34.4 to 46; 30000 x
// 148 in f32 10.2 and 8.9; 8000 x 300 in f16 5.3 and 5.0, x 256 in f32 4.4 and 5.3).
constexpr int64_t kMany = int64_t(1) << 18;
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

__device__ inline float add(Stat &a, float l) {
    const float t = (l - origin(a.m)) * kLog2e;
    const float e = exp2_of(t);
    a.s += e;
    a.w = fmaf(fmaxf(t, -1.0e4f), e, a.w);
    return e;
}

// Reductions over a wave by DPP: within rows of 16 lanes, then lane 15 of a row into the next and
// lane 31 into the upper half; lane 63 holds the result, which all lanes get.
template <int kCtrl, int kRows> __device__ inline uint32_t from_lane(uint32_t x, uint32_t none) {
    return uint32_t(__builtin_amdgcn_update_dpp(int(none), int(x), kCtrl, kRows, 0xF, false));
}
template <typename Op> __device__ inline uint32_t over_wave(uint32_t x, uint32_t none, Op op) {
    x = op(x, from_lane<0x111, 0xF>(x, none));        // row_shr:1, 2, 4, 8
    x = op(x, from_lane<0x112, 0xF>(x, none));
    x = op(x, from_lane<0x114, 0xF>(x, none));
    x = op(x, from_lane<0x118, 0xF>(x, none));
    x = op(x, from_lane<0x142, 0xA>(x, none));        // row_bcast:15 into rows 1 and 3
    x = op(x, from_lane<0x143, 0xC>(x, none));        // row_bcast:31 into rows 2 and 3
    return uint32_t(__builtin_amdgcn_readlane(int(x), 63));
}
__device__ inline float wave_max(float v) {
    return __uint_as_float(over_wave(__float_as_uint(v), __float_as_uint(kNone),
                                     [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
}
__device__ inline float wave_sum(float v) {
    return __uint_as_float(over_wave(__float_as_uint(v), 0u, [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}
__device__ inline uint32_t wave_max(uint32_t v) {
    return over_wave(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ inline uint64_t wave_max(uint64_t k) {
    const uint32_t hi = wave_max(uint32_t(k >> 32));
    return uint64_t(hi) << 32 | wave_max(uint32_t(k >> 32) == hi ? uint32_t(k) : 0u);
}

// The sum of the lanes' sets: all are raised to the largest maximum and added.
__device__ inline Stat join_lanes(Stat a) {
    raise(a, wave_max(a.m));
    a.s = wave_sum(a.s);
    a.w = wave_sum(a.w);
    return a;
}

// Whether a row's results, or a part's sums, are worked out from the weights of all but the largest.
__device__ inline bool certain(float s) { return s < 1.5f; }
__device__ inline float weight_below(float l, float m) {
    return l < m ? exp2_of((l - m) * kLog2e) : 0.0f;
}
// A weight, or 0 for the largest's, which rows of one thread or of few lanes sum beside S: one instruction and
// an addition an element, whatever the logits (300000 x 148 in f32: 29.3 us, without 28; only for rows that need
// it, 28.7 where none does and 31.4 where many do; x 300 in f16 47, without 40, and 43.6 and 50.7).  One
// that rounds to 1 is left out too, but then S is not certain().
__device__ inline float below_one(float e) { return __builtin_amdgcn_fractf(e); }

// log (1 + x) for 0 <= x <= 1/2, twice the area hyperbolic tangent of z = x / (2 + x) <= 1/5: z (1 + z^2 / 3 +
// .. + z^10 / 11), of which the next term is 3e-10.  Within 4 roundings of itself.
__device__ inline float log1p_half(float x) {
    const float z = x * __builtin_amdgcn_rcpf(2.0f + x), q = z * z;
    float s = fmaf(1.0f / 11.0f, q, 1.0f / 9.0f);
    s = fmaf(s, q, 1.0f / 7.0f);
    s = fmaf(s, q, 0.2f);
    s = fmaf(s, q, 1.0f / 3.0f);
    return 2.0f * fmaf(z * q, s, z);
}

// The row's results from its (m, S, w), and, where S is certain(), S - 1.
struct Row { float m, lse, entropy; bool bad; };

__device__ inline Row row_of(const Stat &a, float others) {
    Row r;
    r.m = origin(a.m);
    r.bad = !(a.s < __builtin_inff());
    r.lse = certain(a.s) ? kLog2e * log1p_half(others) : log2f(a.s);
    if (a.m == kNone) r.lse = 0.0f;
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

__device__ inline void put_top(const TokenArgs &a, const Row &r, int64_t row, int j, uint64_t k) {
    const bool none = k == 0 || r.bad;
    a.top_ids[row * a.top + j] = none ? -1 : int32_t(~uint32_t(k));
    a.top_logp[row * a.top + j] = r.bad ? __builtin_nanf("") : none ? kNone : logp_of(r, key_logit(k));
}

// The given token's logit, fetched before the row is worked on; inside: it is one of the choices.
struct Given { bool inside; float l; };

template <typename T> __device__ inline Given given_of(const TokenArgs &a, int64_t row, const T *l) {
    Given g{false, kNone};
    if (a.logp) {
        const int64_t id = id_of(a, row);
        g.inside = id >= 0 && id < a.A;
        if (g.inside) g.l = to_f32(l[id]);
    }
    return g;
}

__device__ inline void put_row(const TokenArgs &a, const Row &r, int64_t row, const Given &g) {
    if (a.logp)
        a.logp[row] = !g.inside ? 0.0f : r.bad ? __builtin_nanf("") : g.l == kNone ? kNone
                                                                          : logp_of(r, g.l);
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

// The rows of a workgroup, which lie one behind the other, between memory and LDS as 16-byte
// words (and what is left over at the end of the last workgroup's rows element by element).
template <typename T, bool kIn> __device__ inline void move_rows(T *tile, T *rows, int elements) {
    typedef uint32_t Word __attribute__((ext_vector_type(4)));
    constexpr int kPer = 16 / sizeof(T);
    const int words = elements / kPer;
    for (int w = threadIdx.x; w < words; w += 256) {
        if (kIn) reinterpret_cast<Word *>(tile)[w] = reinterpret_cast<const Word *>(rows)[w];
        else __builtin_nontemporal_store(reinterpret_cast<Word *>(tile)[w],
                                         reinterpret_cast<Word *>(rows) + w);
    }
    for (int i = words * kPer + threadIdx.x; i < elements; i += 256) {
        if (kIn) tile[i] = rows[i];
        else rows[i] = tile[i];
    }
}

template <typename T, int kA, bool kTile>
__global__ void __launch_bounds__(256) small_rows_kernel(TokenArgs a) {
    __shared__ __attribute__((aligned(16))) T tile[kTile ? 256 * kA : 1];
    const int64_t row0 = int64_t(blockIdx.x) * 256, row = row0 + threadIdx.x;
    const T *l = static_cast<const T *>(a.logits) + row * a.stride;
    if (kTile) {
        const T *rows = static_cast<const T *>(a.logits) + row0 * a.stride;
        move_rows<T, true>(tile, const_cast<T *>(rows), int(min(int64_t(256), a.N - row0)) * a.A);
        __syncthreads();
        l = tile + threadIdx.x * a.A;
    }
    if (row >= a.N) return;
    const Given given = given_of(a, row, l);
    float v[kA];
    load_small(l, a.A, v);
    Stat st{kNone, 0.0f, 0.0f};
    float others = 0.0f;
#pragma unroll
    for (int i = 0; i < kA; ++i) st.m = fmaxf(st.m, v[i]);
#pragma unroll
    for (int i = 0; i < kA; ++i) {
        others += below_one(add(st, v[i]));
    }
    const Row r = row_of(st, others);
    put_row(a, r, row, given);
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

// What the gradient of one row needs: log2 p_i = (l - m) L - lse, d = p (c0 + c1 log2 p), and of the
// given token p (ch + c1 log2 p) + g (1 - p).  strange: 0 times what stands in the brackets need not be 0.
struct Back { float m, lse, g, c0, c1, ch; int id; bool strange; };

__device__ inline Back back_of(const TokenArgs &a, int64_t row) {
    Back b;
    b.m = a.in_stats[2 * row];
    b.lse = a.in_stats[2 * row + 1];
    const int64_t id = a.dlogp ? id_of(a, row) : -1;
    b.id = id >= 0 && id < a.A ? int(id) : -1;
    b.g = b.id >= 0 ? a.dlogp[row] : 0.0f;
    const float gh = a.dentropy ? a.dentropy[row] : 0.0f;
    b.c1 = -gh * kLn2;
    b.ch = a.dentropy ? -gh * a.in_entropy[row] : 0.0f;
    b.c0 = b.ch - b.g;
    b.strange = !(fmaf(1.0e4f, fabsf(b.c1), fabsf(b.c0)) < __builtin_inff());
    return b;
}

__device__ inline float slope(const Back &b, float l) {
    const float t = fmaf(l - b.m, kLog2e, -b.lse);
    return exp2_of(t) * fmaf(b.c1, fmaxf(t, -1.0e4f), b.c0);
}
// The given token's.  Of 1 - p little is left where p is all but 1: above e^-1/2 it is the series of
// 1 - e^x, x = log p, up to x^9 / 9! (the next term is 5e-10 of it), within 3 roundings of itself.
__device__ inline float own_slope(const Back &b, float l) {
    const float t = fmaf(l - b.m, kLog2e, -b.lse), p = exp2_of(t), x = kLn2 * t;
    float s = fmaf(1.0f / 362880.0f, x, 1.0f / 40320.0f);
    s = fmaf(s, x, 1.0f / 5040.0f);
    s = fmaf(s, x, 1.0f / 720.0f);
    s = fmaf(s, x, 1.0f / 120.0f);
    s = fmaf(s, x, 1.0f / 24.0f);
    s = fmaf(s, x, 1.0f / 6.0f);
    s = fmaf(s, x, 0.5f);
    const float rest = x > -0.5f ? -fmaf(x * x, s, x) : 1.0f - p;
    return fmaf(p, fmaf(b.c1, fmaxf(t, -1.0e4f), b.ch), b.g * rest);
}

// The gradients of n neighbouring choices from index `at` on.  A masked one's is 0: by its
// weight, or, in a strange row, by having been looked for (in all rows that costs 1638400 x 5 in f32 0.7 us
// of 30, 4096 x 32768 in bf16 2.5 of 140).  It is NaN in a row whose results are.
template <int n> __device__ inline void slopes(const Back &b, int at, float (&v)[n]) {
    const int own = b.id - at;                 // the given token among them, unless it is masked
    float mine = kNone;
    uint32_t masked = 0;                       // of a strange row
    if (unsigned(own) < unsigned(n)) {
#pragma unroll
        for (int i = 0; i < n; ++i) mine = i == own ? v[i] : mine;
    }
    if (b.strange) {
#pragma unroll
        for (int i = 0; i < n; ++i) masked |= v[i] == kNone ? 1u << i : 0u;
    }
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = slope(b, v[i]);
    if (mine != kNone) {
        mine = own_slope(b, mine);
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = i == own ? mine : v[i];
    }
    if (masked) {
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = masked >> i & 1 ? 0.0f * b.lse : v[i];
    }
}

template <typename T, int kA, bool kTile>
__global__ void __launch_bounds__(256) small_back_kernel(TokenArgs a) {
    __shared__ __attribute__((aligned(16))) T tile[kTile ? 256 * kA : 1];
    const int64_t row0 = int64_t(blockIdx.x) * 256, row = row0 + threadIdx.x;
    const int rows = int(min(int64_t(256), a.N - row0));
    const T *l = static_cast<const T *>(a.logits) + row * a.stride;
    T *d = static_cast<T *>(a.dlogits) + row * a.dstride;
    if (kTile) {
        const T *from = static_cast<const T *>(a.logits) + row0 * a.stride;
        move_rows<T, true>(tile, const_cast<T *>(from), rows * a.A);
        __syncthreads();
        l = d = tile + threadIdx.x * a.A;
    }
    if (row < a.N) {
        const Back b = back_of(a, row);
        float v[kA];
        load_small(l, a.A, v);
        slopes(b, 0, v);
#pragma unroll
        for (int i = 0; i < kA; ++i)
            if (i < a.A) d[i] = from_f32<T>(v[i]);
    }
    if (kTile) {
        __syncthreads();
        move_rows<T, false>(tile, static_cast<T *>(a.dlogits) + row0 * a.dstride, rows * a.A);
    }
}

// ---- longer rows, as words of kPer elements (16 bytes, at any address) ----

// A row's last word starts where kPer elements are left, so its first `skip` elements are the word
// before's too: they count as masked and are not stored.  The row has at least kPer.
template <typename T> struct Words {
    static constexpr int kPer = 16 / sizeof(T);
    const T *l;
    int A, count;

    __device__ Words(const TokenArgs &a, int64_t row)
        : l(static_cast<const T *>(a.logits) + row * a.stride), A(a.A),
          count((a.A + kPer - 1) / kPer) {}
    __device__ int first(int word) const { return min(word * kPer, A - kPer); }
    __device__ int skip(int word) const { return word * kPer - first(word); }
    __device__ Word<T, kPer> get(int word) const {
        return load_any<Word<T, kPer>>(l + first(word));
    }
    // Elements first(word) .. + kPer - 1; -inf where skipped, and all where there is no such word.
    __device__ void load(int word, float (&v)[kPer]) const {
        const bool there = word < count;
        const int at = there ? word : count - 1;
        const Word<T, kPer> q = get(at);
        const int from = there ? skip(at) : kPer;
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = i >= from ? to_f32(q.v[i]) : kNone;
    }
    // Stores the gradients of a word.
    template <bool kPast> __device__ void put(T *d, int word, const float (&v)[kPer]) const {
        const int at = first(word), from = skip(word);
        Word<T, kPer> o;
#pragma unroll
        for (int i = 0; i < kPer; ++i) o.v[i] = from_f32<T>(v[i]);
        if (from == 0) {
            if (kPast) store_past(d + at, o);
            else __builtin_memcpy(d + at, &o, sizeof o);
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (i >= from) store_past(d + at + i, o.v[i]);
        }
    }
};

template <int kPer> __device__ inline float largest(const float (&v)[kPer]) {
    float m = v[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) m = fmaxf(m, v[i]);
    return m;
}

// Reductions over the kLanes neighbouring lanes of a row: within four lanes and by mirroring eight and
// sixteen in one instruction each, wider through LDS.  Every lane gets the result, the same bits in
// all: the two of a pair add the same two numbers.
template <int kLanes, typename Op> __device__ inline uint32_t over_team(uint32_t x, Op op) {
    auto with = [&](uint32_t y) { x = op(x, y); };
    with(uint32_t(__builtin_amdgcn_mov_dpp(int(x), 0xB1, 0xF, 0xF, true)));    // quad 1 0 3 2
    with(uint32_t(__builtin_amdgcn_mov_dpp(int(x), 0x4E, 0xF, 0xF, true)));    // quad 2 3 0 1
    if (kLanes > 4) with(uint32_t(__builtin_amdgcn_mov_dpp(int(x), 0x141, 0xF, 0xF, true)));
    if (kLanes > 8) with(uint32_t(__builtin_amdgcn_mov_dpp(int(x), 0x140, 0xF, 0xF, true)));
    if (kLanes > 16) with(uint32_t(__shfl_xor(int(x), 16)));
    return x;
}
template <int kLanes> __device__ inline float team_max(float v) {
    return __uint_as_float(over_team<kLanes>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
}
template <int kLanes> __device__ inline float team_sum(float v) {
    return __uint_as_float(over_team<kLanes>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}

// The alternatives of a row that kLanes lanes hold, kWords words each: the largest left of all lanes,
// again and again, of equal ones the one of the lowest index.
template <int kLanes, int kWords, int kPer, typename Index>
__device__ inline void largest_first(const TokenArgs &a, const Row &r, int64_t row, bool live,
                                     const float (&v)[kWords][kPer], Index index) {
    const int lane = threadIdx.x % kLanes;
    uint32_t key[kWords][kPer];
#pragma unroll
    for (int w = 0; w < kWords; ++w)
#pragma unroll
        for (int i = 0; i < kPer; ++i) key[w][i] = uint32_t(key_of(v[w][i], 0) >> 32);
    const int shift = int(threadIdx.x & 63) / kLanes * kLanes;        // the team's first lane
    for (int j = 0; j < a.top; ++j) {
        uint32_t best = 0;
#pragma unroll
        for (int w = 0; w < kWords; ++w)
#pragma unroll
            for (int i = 0; i < kPer; ++i) best = max(best, key[w][i]);
        uint32_t top;
        if constexpr (kLanes == 64) top = wave_max(best);
        else top = over_team<kLanes>(best, [](uint32_t x, uint32_t y) { return max(x, y); });
        int which = 0;                                  // the lane's first of them
#pragma unroll
        for (int w = kWords - 1; w >= 0; --w)
#pragma unroll
            for (int i = kPer - 1; i >= 0; --i) which = key[w][i] == top ? w * kPer + i : which;
        const uint32_t at = best == top ? uint32_t(index(which / kPer, which % kPer)) : ~0u;
        bool mine;
        if constexpr (kWords == 1) {                    // the first lane's
            const uint64_t team = __ballot(best == top) >> shift & (~uint64_t(0) >> (64 - kLanes));
            mine = lane == __ffsll(static_cast<unsigned long long>(team)) - 1;
        } else {
            mine = at == over_team<kLanes>(at, [](uint32_t x, uint32_t y) { return min(x, y); });
        }
        if (!mine) continue;
#pragma unroll
        for (int w = 0; w < kWords; ++w)
#pragma unroll
            for (int i = 0; i < kPer; ++i) key[w][i] = w * kPer + i == which ? 0 : key[w][i];
        if (live) put_top(a, r, row, j, top ? uint64_t(top) << 32 | uint32_t(~at) : 0);
    }
}

// Rows of at most kLanes kWords words, kLanes (4 to 32) lanes each and kWords words a lane.
template <typename T, int kLanes, int kWords>
__global__ void __launch_bounds__(256) team_rows_kernel(TokenArgs a) {
    constexpr int kPer = Words<T>::kPer;
    const int lane = threadIdx.x % kLanes;
    const int64_t at = int64_t(blockIdx.x) * (256 / kLanes) + threadIdx.x / kLanes;
    const bool live = at < a.N;
    const int64_t row = live ? at : a.N - 1;
    const Words<T> in(a, row);
    Given given{};
    if (lane == 0) given = given_of(a, row, in.l);
    float v[kWords][kPer], m = kNone;
#pragma unroll
    for (int j = 0; j < kWords; ++j) in.load(j * kLanes + lane, v[j]);
#pragma unroll
    for (int j = 0; j < kWords; ++j) m = fmaxf(m, largest(v[j]));
    Stat st{team_max<kLanes>(m), 0.0f, 0.0f};
    float others = 0.0f;
#pragma unroll
    for (int j = 0; j < kWords; ++j)
#pragma unroll
        for (int i = 0; i < kPer; ++i) others += below_one(add(st, v[j][i]));
    st.s = team_sum<kLanes>(st.s);
    st.w = team_sum<kLanes>(st.w);
    others = team_sum<kLanes>(others);
    const Row r = row_of(st, others);
    if (lane == 0 && live) put_row(a, r, row, given);
    if (a.top == 0) return;
    largest_first<kLanes>(a, r, row, live, v,
                          [&](int j, int i) { return in.first(j * kLanes + lane) + i; });
}

// The k-th largest of the wave's 64 numbers (0 if fewer are set): bit by bit from the top, the
// largest number that k of them reach.
__device__ inline uint32_t kth_of_wave(uint32_t x, int k) {
    uint32_t t = 0;
#pragma unroll 4
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t up = t | 1u << bit;
        if (__popcll(__ballot(x >= up)) >= k) t = up;
    }
    return t;
}
// The same of keys; the lower halves are only looked at where the upper ones leave a tie.
__device__ inline uint64_t kth_of_wave(uint64_t key, int k) {
    const uint32_t hi = uint32_t(key >> 32), t = kth_of_wave(hi, k);
    const int above = __popcll(__ballot(hi > t)), equal = __popcll(__ballot(hi == t));
    if (t == 0 || above + equal == k) return uint64_t(t) << 32;
    return uint64_t(t) << 32 | kth_of_wave(hi == t ? uint32_t(key) : 0u, k - above);
}

// Adds a lane's words to its (empty) sums; sums[] takes what each word's weights come to.
template <int kWords, int kPer>
__device__ inline void add_words(Stat &st, const float (&v)[kWords][kPer], float (&sums)[kWords]) {
    float all = 0.0f;
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        st.s = 0.0f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) add(st, v[j][i]);
        sums[j] = st.s;
        all += st.s;
    }
    st.s = all;
}
// A lane's part of S - 1 where S is certain(): one word of one lane has the largest, m, and only its sum has lost
// bits to the 1, so only its weights are taken again (20000 x 3000 in bf16, logits of deviation 8: 24.8 us,
// with every word's 28.5; of deviation 2, where no row is certain, 22.8).
template <int kWords, int kPer>
__device__ inline float others_of(const float (&v)[kWords][kPer], const float (&sums)[kWords], float m) {
    float e = 0.0f, x[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = kNone;
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        const bool here = largest(v[j]) == m;
        e += here ? 0.0f : sums[j];
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[i] = here ? v[j][i] : x[i];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) e += weight_below(x[i], m);
    return e;
}

constexpr int kWaveList = 256;       // candidates for the alternatives of a wave's row

// One wave per row of at most kWaveRow choices, held in registers.  Alternatives: no one is smaller
// than the k-th largest of the lanes' maxima; the elements that reach it are listed in LDS, and a
// listed key's place is the number of larger ones.  Where they are too many (equal elements, or few
// choices left), the largest key below the last is taken again and again.  The bound costs much the
// same for any number; a few of a lane's single word are found sooner one after another (20000 x 300
// in bf16: 4 alternatives 16.2 us, with the bound 17.2; 6 of them 19.8 and 17.7), and so is one of a few
// words (20000 x 1000 in bf16: 14.0, with the bound 20.0; of eight words 66.8 and 64.8).
constexpr int kFew = 4, kFewWords = 4;
template <typename T, int kWords>
__global__ void __launch_bounds__(256) wave_rows_kernel(TokenArgs a) {
    constexpr int kPer = Words<T>::kPer;
    __shared__ unsigned long long lists[4][kWaveList];
    const int lane = threadIdx.x & 63;
    const int64_t row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= a.N) return;
    const Words<T> in(a, row);
    Given given{};
    if (lane == 0) given = given_of(a, row, in.l);
    float v[kWords][kPer];
#pragma unroll
    for (int j = 0; j < kWords; ++j) in.load(j * 64 + lane, v[j]);
    float m = kNone;
#pragma unroll
    for (int j = 0; j < kWords; ++j) m = fmaxf(m, largest(v[j]));
    Stat st{wave_max(m), 0.0f, 0.0f};
    float sums[kWords];
    add_words(st, v, sums);
    st.s = wave_sum(st.s);
    st.w = wave_sum(st.w);
    float others = 0.0f;
    if (certain(st.s)) others = wave_sum(others_of(v, sums, st.m));      // the same in all lanes
    const Row r = row_of(st, others);
    if (lane == 0) put_row(a, r, row, given);
    if (a.top == 0) return;
    if constexpr (kWords == 1) if (a.top <= kFew) {
        largest_first<64>(a, r, row, true, v, [&](int, int i) { return in.first(lane) + i; });
        return;
    }
    if (kWords <= kFewWords && a.top == 1) {
        int at = 0;
#pragma unroll
        for (int j = kWords - 1; j >= 0; --j)
#pragma unroll
            for (int i = kPer - 1; i >= 0; --i) at = v[j][i] == m ? in.first(j * 64 + lane) + i : at;
        const uint64_t best = wave_max(key_of(m, at));
        if (lane == 0) put_top(a, r, row, 0, best);
        return;
    }
    unsigned long long *list = lists[threadIdx.x >> 6];
    const uint64_t bound = uint64_t(kth_of_wave(uint32_t(key_of(m, 0) >> 32), a.top)) << 32;
    const float least = bound == 0 ? -__FLT_MAX__ : key_logit(bound);
    int n = 0;
#pragma unroll
    for (int j = 0; j < kWords; ++j)
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint64_t who = __ballot(v[j][i] >= least);
            const int at = n + int(__builtin_amdgcn_mbcnt_hi(uint32_t(who >> 32),
                                   __builtin_amdgcn_mbcnt_lo(uint32_t(who), 0u)));
            if (v[j][i] >= least && at < kWaveList)
                list[at] = key_of(v[j][i], in.first(j * 64 + lane) + i);
            n += __popcll(who);
        }
    if (n <= kWaveList) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        for (int i = lane; i < n; i += 64) {
            const uint64_t k = list[i];
            int place = 0;
            for (int j = 0; j < n; ++j) place += list[j] > k;
            if (place < a.top) put_top(a, r, row, place, k);
        }
        for (int j = n + lane; j < a.top; j += 64) put_top(a, r, row, j, 0);
        return;
    }
    uint64_t last = ~uint64_t(0);
    for (int t = 0; t < a.top; ++t) {
        uint64_t next = 0;
#pragma unroll
        for (int j = 0; j < kWords; ++j)
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const uint64_t k = key_of(v[j][i], in.first(j * 64 + lane) + i);
                if (k < last && k > next) next = k;
            }
        next = wave_max(next);
        if (lane == 0) put_top(a, r, row, t, next);
        last = next;
    }
}

// The words of one of `parts` parts of a row.
template <typename T> struct Parts : Words<T> {
    int from, to;

    __device__ Parts(const TokenArgs &a, int64_t row, int part = 0, int parts = 1)
        : Words<T>(a, row) {
        const int each = (this->count + parts - 1) / parts;
        from = min(this->count, part * each);
        to = min(this->count, from + each);
    }
};

constexpr int kList = 2048;          // candidates for the alternatives

// Alternatives of a row; m is the largest of the thread's own elements.
//
// Where k threads of one wave hold an element of at least x, no alternative is smaller than x.  The
// largest such bound over the waves leaves a few k threads with a larger element; all threads share
// those threads' words, list what reaches the bound, and a listed key's place is the number of larger
// ones.  Where the list is too small because many elements are equal, the bound is taken over keys,
// which also tell equal elements apart; where it still is (thousands of the largest in a few
// threads' hands, or fewer than k choices in any wave), the alternatives are found one after another,
// each in a pass over the row.
//
// put(place, key) takes them; a key of 0 says that there is none.
template <typename T, int kThreads, typename Put>
__device__ void alternatives(const TokenArgs &a, const Parts<T> &in, float m, Put put) {
    constexpr int kPer = Parts<T>::kPer, kWaves = kThreads / 64;
    __shared__ unsigned long long list[kList], keys[kWaves];
    __shared__ uint16_t holders[kThreads];
    __shared__ int listed, held;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int each = (in.to - in.from + kThreads - 1) / kThreads;     // words of a thread
    uint64_t best = key_of(m, 0);                              // at least any key of the thread's
    for (int exact = 0; exact < 2; ++exact) {
        if (exact) {
            best = 0;
            for (int word = in.from + tid; word < in.to; word += kThreads) {
                float v[kPer];
                in.load(word, v);
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (v[i] == m) best = max(best, key_of(m, in.first(word) + i));
            }
        }
        const uint64_t mine = exact ? kth_of_wave(best, a.top)
                                    : uint64_t(kth_of_wave(uint32_t(best >> 32), a.top)) << 32;
        __syncthreads();
        if (lane == 0) keys[w] = mine;
        if (tid == 0) listed = held = 0;
        __syncthreads();
        uint64_t bound = 1;                           // a masked choice's key is 0
        for (int j = 0; j < kWaves; ++j) bound = max(bound, uint64_t(keys[j]));
        if (best >= bound) holders[atomicAdd(&held, 1)] = uint16_t(tid);
        __syncthreads();
        auto offer = [&](float v, int i) {
            const uint64_t k = key_of(v, i);
            if (k < bound) return;
            const int at = atomicAdd(&listed, 1);
            if (at < kList) list[at] = k;
        };
        const int tasks = held * each;
        for (int t = tid; t < tasks; t += kThreads) {
            const int word = in.from + holders[t / each] + t % each * kThreads;
            if (word >= in.to) continue;
            float v[kPer];
            in.load(word, v);
#pragma unroll
            for (int i = 0; i < kPer; ++i) offer(v[i], in.first(word) + i);
        }
        __syncthreads();
        const int n = listed;
        if (n > kList) continue;
        for (int i = tid; i < n; i += kThreads) {
            const uint64_t k = list[i];
            int place = 0;
            for (int j = 0; j < n; ++j) place += list[j] > k;
            if (place < a.top) put(place, k);
        }
        for (int j = n + tid; j < a.top; j += kThreads) put(j, uint64_t(0));
        return;
    }
    uint64_t last = ~uint64_t(0);
    for (int j = 0; j < a.top; ++j) {
        uint64_t next = 0;
        auto look = [&](float v, int i) {
            const uint64_t k = key_of(v, i);
            if (k < last && k > next) next = k;
        };
        for (int word = in.from + tid; word < in.to; word += kThreads) {
            float v[kPer];
            in.load(word, v);
#pragma unroll
            for (int i = 0; i < kPer; ++i) look(v[i], in.first(word) + i);
        }
        next = wave_max(next);
        __syncthreads();
        if (lane == 0) keys[w] = next;
        __syncthreads();
        for (int i = 0; i < kWaves; ++i) next = max(next, uint64_t(keys[i]));
        if (tid == 0) put(j, next);
        last = next;
    }
}

// A row's, or a part's, S - 1, where S is certain() and so one thread has the largest; st the thread's own
// sums, m the row's largest.  That thread's sum is the one that has lost bits to the 1: its wave takes
// its words once more, one a lane.
template <typename T, int kThreads>
__device__ float others_of(const Parts<T> &in, const Stat &st, float m) {
    constexpr int kPer = Parts<T>::kPer, kWaves = kThreads / 64;
    __shared__ float sums[kWaves];
    const int lane = threadIdx.x & 63, first = threadIdx.x & ~63;
    const unsigned long long who = __ballot(st.m == m);
    Stat up = st;
    raise(up, m);
    float e = st.m == m ? 0.0f : up.s;
    if (who) {
        const int holder = first + __ffsll(who) - 1;
        for (int word = in.from + holder + lane * kThreads; word < in.to; word += 64 * kThreads) {
            float v[kPer];
            in.load(word, v);
#pragma unroll
            for (int i = 0; i < kPer; ++i) e += weight_below(v[i], m);
        }
    }
    e = wave_sum(e);
    if (lane == 0) sums[threadIdx.x >> 6] = e;
    __syncthreads();
    return wave_sum(lane < kWaves ? sums[lane] : 0.0f);
}

// One workgroup per row of any length, or, kSplit, per part of it (blockIdx.y), whose m, S - 1 and w and
// alternatives go to the workspace.  A thread has kWords 16-byte words on their way at once; the
// largest of their elements is found first, so that the sums are rescaled at most once for all.  Four
// words, or eight for many long rows (2500 x 60001 in f32: 122 us, with four 129; but 777 x 50021 in
// f16 31 and 26.6, and 4096 x 9000 in bf16, which have no round of eight, 21.6 and 18.1).
template <typename T, int kThreads, int kWords, bool kSplit>
__global__ void __launch_bounds__(kThreads) long_rows_kernel(TokenArgs a) {
    constexpr int kPer = Parts<T>::kPer, kWaves = kThreads / 64;
    __shared__ Stat stats[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t row = blockIdx.x;
    const Parts<T> in(a, row, kSplit ? blockIdx.y : 0, kSplit ? a.parts : 1);
    Given given{};
    if (!kSplit && tid == 0) given = given_of(a, row, in.l);
    Stat st{kNone, 0.0f, 0.0f};
    for (int word = in.from + tid; word < in.to; word += kWords * kThreads) {
        Word<T, kPer> q[kWords];
        // all of this round's words are there, and none is the row's last, which may skip elements
        const bool whole = word + (kWords - 1) * kThreads < min(in.to, in.count - 1);
        float m = st.m;
        if (whole) {
#pragma unroll
            for (int j = 0; j < kWords; ++j) q[j] = in.get(word + j * kThreads);
#pragma unroll
            for (int j = 0; j < kWords; ++j)
#pragma unroll
                for (int i = 0; i < kPer; ++i) m = fmaxf(m, to_f32(q[j].v[i]));
            if (m > st.m) raise(st, m);
#pragma unroll
            for (int j = 0; j < kWords; ++j)
#pragma unroll
                for (int i = 0; i < kPer; ++i) add(st, to_f32(q[j].v[i]));
        } else {
#pragma unroll
            for (int j = 0; j < kWords; ++j) q[j] = in.get(min(word + j * kThreads, in.to - 1));
#pragma unroll
            for (int j = 0; j < kWords; ++j) {
                const int at = word + j * kThreads;
                if (at >= in.to) continue;
                const int from = in.skip(at);
                float v[kPer];
#pragma unroll
                for (int i = 0; i < kPer; ++i) v[i] = i >= from ? to_f32(q[j].v[i]) : kNone;
                m = largest(v);
                if (m > st.m) raise(st, m);
#pragma unroll
                for (int i = 0; i < kPer; ++i) add(st, v[i]);
            }
        }
    }
    const Stat own = st;
    const float mine = st.m;
    st = join_lanes(st);
    if (lane == 0) stats[w] = st;
    __syncthreads();
    Stat all{kNone, 0.0f, 0.0f};
    if (lane < kWaves) all = stats[lane];
    all = join_lanes(all);                              // the same in all waves
    float others = all.s - 1.0f;
    if (certain(all.s)) others = others_of<T, kThreads>(in, own, all.m);
    if (kSplit) {
        const int64_t at = row * a.parts + blockIdx.y;
        if (tid == 0) static_cast<Stat *>(a.part_stats)[at] = Stat{all.m, others, all.w};
        if (a.top) {
            uint64_t *keys = a.part_keys + at * a.top;
            alternatives<T, kThreads>(a, in, mine, [&](int place, uint64_t k) { keys[place] = k; });
        }
        return;
    }
    const Row r = row_of(all, others);
    if (tid == 0) put_row(a, r, row, given);
    if (a.top)
        alternatives<T, kThreads>(a, in, mine, [&](int place, uint64_t k) {
            put_top(a, r, row, place, k);
        });
}

// The rows from their parts (at most 64).  A part's last alternative, if it has that many, has `top`
// keys from itself up, so what is smaller than the largest of these is no alternative of the row;
// of the keys left, a little more than `top`, a key's place is the number of larger ones.  (Placing
// all 256 keys of sixteen parts took 3 us more.)
template <typename T> __global__ void __launch_bounds__(256) join_rows_kernel(TokenArgs a) {
    __shared__ uint64_t list[64 * AV_TOP_MAX];
    __shared__ int listed;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t row = blockIdx.x;
    const int n = a.parts * a.top;
    const uint64_t *keys = a.part_keys + row * n;
    const bool part = lane < a.parts;
    Stat all{kNone, 0.0f, 0.0f};
    if (part) all = static_cast<const Stat *>(a.part_stats)[row * a.parts + lane];
    uint64_t bound = a.top && part ? keys[lane * a.top + a.top - 1] : 0;
    uint64_t mine = tid < n ? keys[tid] : 0;
    Given given{};
    if (tid == 0) {
        given = given_of(a, row, static_cast<const T *>(a.logits) + row * a.stride);
        listed = 0;
    }
    // what a part without a choice has for S - 1 is 0, or a NaN
    const float rest = all.s;
    all.s = all.m == kNone ? rest : 1.0f + rest;
    Stat sum = all;
    raise(sum, wave_max(all.m));
    // of the one part with the row's largest, if the row is certain(), S - 1; of the others all
    const float others = wave_sum(all.m == sum.m ? rest : sum.s);
    sum.s = wave_sum(sum.s);
    sum.w = wave_sum(sum.w);
    const Row r = row_of(sum, others);
    if (tid == 0) put_row(a, r, row, given);
    if (a.top == 0) return;
    bound = max(wave_max(bound), uint64_t(1));
    __syncthreads();
    for (int i = tid; i < n; i += 256) {
        if (i >= 256) mine = keys[i];
        if (mine >= bound) list[atomicAdd(&listed, 1)] = mine;
    }
    __syncthreads();
    const int m = listed;
    for (int i = tid; i < m; i += 256) {
        const uint64_t k = list[i];
        int place = 0;
        for (int j = 0; j < m; ++j) place += list[j] > k;
        if (place < a.top) put_top(a, r, row, place, k);
    }
    for (int j = m + tid; j < a.top; j += 256) put_top(a, r, row, j, 0);
}

// Gradient of rows of any length; blockIdx.y, and the threads, share a row's words.  The gradient
// goes past the caches: it is not read again here, and the logits, which the forward pass has just
// read, stay (4096 x 32768 in bf16, both passes: 169 us, so 139).
template <typename T>
__global__ void __launch_bounds__(256) long_back_kernel(TokenArgs a) {
    constexpr int kPer = Words<T>::kPer;
    const int64_t row = blockIdx.x;
    const Words<T> in(a, row);
    T *d = static_cast<T *>(a.dlogits) + row * a.dstride;
    const Back b = back_of(a, row);
    const int stride = int(gridDim.y) * 256;
    for (int word = int(blockIdx.y) * 256 + threadIdx.x; word < in.count; word += stride) {
        const Word<T, kPer> q = in.get(word);
        float v[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = to_f32(q.v[i]);
        slopes(b, in.first(word), v);
        in.template put<true>(d, word, v);
    }
}

// The same for rows of at most kTeamBack words, kLanes lanes each and kWords words a lane on their way.  A
// lane with one word has the whole row's stores in one instruction, which may go past the caches;
// several leave lines in pieces, which the caches put together (300000 x 148 in f32: 69 us, past
// them 83).
template <typename T, int kLanes, int kWords>
__global__ void __launch_bounds__(256) team_back_kernel(TokenArgs a) {
    constexpr int kPer = Words<T>::kPer;
    const int64_t row = int64_t(blockIdx.x) * (256 / kLanes) + threadIdx.x / kLanes;
    if (row >= a.N) return;
    const Words<T> in(a, row);
    T *d = static_cast<T *>(a.dlogits) + row * a.dstride;
    const Back b = back_of(a, row);
    for (int word = threadIdx.x % kLanes; word < in.count; word += kLanes * kWords) {
        Word<T, kPer> q[kWords];
#pragma unroll
        for (int j = 0; j < kWords; ++j) q[j] = in.get(min(word + j * kLanes, in.count - 1));
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
            const int at = word + j * kLanes;
            if (at >= in.count) continue;
            float v[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) v[i] = to_f32(q[j].v[i]);
            slopes(b, in.first(at), v);
            in.template put<kWords == 1>(d, at, v);
        }
    }
}

// ---- drawing ----

// Sums of the lanes up to and with this one, of a row's kLanes; and the row's total.
template <int kLanes, typename F> __device__ inline F upto_lane(F x, int lane) {
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) {
        const F o = __shfl_up(x, d, kLanes);
        if (lane >= d) x += o;
    }
    return x;
}

constexpr int kNoChoice = 1 << 20;

// Rows of up to kEach kLanes choices, kEach neighbouring ones a lane.  Where the sum passes u is a
// property of the logits in 64 bits, but is found in 32 unless it is close.  With e_i = 2^t_i,
// t_i <= 0, a weight is off by at most (1 + |t_i| ln 2) 2^-23 of itself and sum p_i |t_i| <= log2 A <= 8,
// so that a running sum, with its fourteen additions, and u times the total are off by less than
// 16 x 2^-23 of the total: a sum further than 2^-17 of the total from u x total is on the side it
// seems to be.  The rows of a wave that holds a closer one (a row of 256 choices in some 250 does,
// one of 5 in 13000) are drawn again in 64 bits (26421 rows of 135 choices: 11 us, all in 64 bits 22).
template <typename T, int kLanes, int kEach>
__global__ void __launch_bounds__(256) draw_kernel(TokenArgs a) {
    const int lane = threadIdx.x % kLanes;
    const int64_t row = int64_t(blockIdx.x) * (256 / kLanes) + threadIdx.x / kLanes;
    const bool live = row < a.N;
    const T *l = static_cast<const T *>(a.logits) + (live ? row : a.N - 1) * a.stride;
    const float u = a.uniform[live ? row : a.N - 1];
    float v[kEach];
    if (lane * kEach + kEach <= a.A) {
        const Word<T, kEach> q = load_any<Word<T, kEach>>(l + lane * kEach);
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = to_f32(q.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            v[i] = lane * kEach + i < a.A ? to_f32(l[lane * kEach + i]) : kNone;
    }
    float m = largest(v);
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, kLanes));
    float e[kEach], sum = 0.0f;
    int alive = -1;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        e[i] = v[i] == kNone ? 0.0f : exp2_of((v[i] - m) * kLog2e);
        sum += e[i];
        e[i] = sum;                                   // up to and with choice i
        if (v[i] > kNone) alive = lane * kEach + i;
    }
    const float upto = upto_lane<kLanes>(sum, lane), total = __shfl(upto, kLanes - 1, kLanes);
    float before = __shfl_up(upto, 1, kLanes);
    if (lane == 0) before = 0.0f;
    const float aim = u * total;
    int pick = kNoChoice;
    bool close = false;
#pragma unroll
    for (int i = kEach - 1; i >= 0; --i) {
        if (!(v[i] > kNone)) continue;
        const float over = before + e[i] - aim;
        if (over > 0.0f) pick = lane * kEach + i;
        close |= fabsf(over) <= total * 0x1p-17f;
    }
    if (__any(close)) {
        double w[kEach], s = 0.0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            s += v[i] == kNone ? 0.0 : exp(double(v[i]) - double(m));
            w[i] = s;
        }
        const double to = upto_lane<kLanes>(s, lane);
        const double goal = double(u) * __shfl(to, kLanes - 1, kLanes);
        double from = __shfl_up(to, 1, kLanes);
        if (lane == 0) from = 0.0;
        pick = kNoChoice;
#pragma unroll
        for (int i = kEach - 1; i >= 0; --i)
            if (v[i] > kNone && from + w[i] > goal) pick = lane * kEach + i;
    }
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) {
        pick = min(pick, __shfl_xor(pick, d, kLanes));
        alive = max(alive, __shfl_xor(alive, d, kLanes));
    }
    if (pick == kNoChoice) pick = alive;
    float log_total = kLn2 * log2f(total);
    if (__any(total < 1.5f)) {
        // a row with one all but certain choice: log (1 + the others' weights), whose small numbers
        // the 1 would leave no bits for
        float others = 0.0f;
#pragma unroll
        for (int i = 0; i < kEach; ++i) others += weight_below(v[i], m);
#pragma unroll
        for (int d = kLanes / 2; d > 0; d >>= 1) others += __shfl_xor(others, d, kLanes);
        if (total < 1.5f) log_total = log1pf(others);
    }
    if (!live || lane != 0) return;
    float logp = kNone;
    if (!(total < __builtin_inff())) {                // a NaN, or a +inf
        pick = 0;
        logp = __builtin_nanf("");
    } else if (pick < 0) {
        pick = 0;
    } else {
        logp = to_f32(l[pick]) - m - log_total;
    }
    a.actions[row] = uint8_t(pick);
    if (a.logp) a.logp[row] = logp;
}

unsigned blocks_of(int64_t n, int64_t per) { return unsigned((n + per - 1) / per); }

template <typename T> int words_of(const TokenArgs &a) {
    constexpr int kPer = 16 / sizeof(T);
    return (a.A + kPer - 1) / kPer;
}

// Rows one behind the other from a 16-byte border on: moved through LDS.
bool packed_rows(const TokenArgs &a, const void *p, int64_t stride) {
    return (stride == a.A || a.N == 1) && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

template <typename T, bool kTile> hipError_t small_forward(const TokenArgs &a, hipStream_t s) {
    const dim3 g(blocks_of(a.N, 256)), b(256);
    if (a.A <= 4) hipLaunchKernelGGL((small_rows_kernel<T, 4, kTile>), g, b, 0, s, a);
    else if (a.A <= 8) hipLaunchKernelGGL((small_rows_kernel<T, 8, kTile>), g, b, 0, s, a);
    else hipLaunchKernelGGL((small_rows_kernel<T, 16, kTile>), g, b, 0, s, a);
    return hipGetLastError();
}

template <typename T, bool kTile> hipError_t small_backward(const TokenArgs &a, hipStream_t s) {
    const dim3 g(blocks_of(a.N, 256)), b(256);
    if (a.A <= 4) hipLaunchKernelGGL((small_back_kernel<T, 4, kTile>), g, b, 0, s, a);
    else if (a.A <= 8) hipLaunchKernelGGL((small_back_kernel<T, 8, kTile>), g, b, 0, s, a);
    else hipLaunchKernelGGL((small_back_kernel<T, 16, kTile>), g, b, 0, s, a);
    return hipGetLastError();
}

template <typename T> hipError_t forward(const TokenArgs &a, hipStream_t s) {
    const dim3 b(256);
    if (a.A <= kThreadRow) {
        if (packed_rows(a, a.logits, a.stride)) return small_forward<T, true>(a, s);
        return small_forward<T, false>(a, s);
    }
    const int words = words_of<T>(a);
    if (a.A <= kWaveRow) {
        auto rows = [&](int lanes) { return dim3(blocks_of(a.N, 256 / lanes)); };
        const bool many = a.all * words >= kMany, few = a.top <= kFew;
        if (words <= 4) hipLaunchKernelGGL((team_rows_kernel<T, 4, 1>), rows(4), b, 0, s, a);
        else if (many && words <= 8)
            hipLaunchKernelGGL((team_rows_kernel<T, 4, 2>), rows(4), b, 0, s, a);
        else if (many && words <= 12)
            hipLaunchKernelGGL((team_rows_kernel<T, 4, 3>), rows(4), b, 0, s, a);
        else if (many && words <= 16)
            hipLaunchKernelGGL((team_rows_kernel<T, 4, 4>), rows(4), b, 0, s, a);
        else if (many && words <= 24)
            hipLaunchKernelGGL((team_rows_kernel<T, 8, 3>), rows(8), b, 0, s, a);
        else if (many && words <= 32)
            hipLaunchKernelGGL((team_rows_kernel<T, 8, 4>), rows(8), b, 0, s, a);
        else if (many && few && words <= 48)
            hipLaunchKernelGGL((team_rows_kernel<T, 16, 3>), rows(16), b, 0, s, a);
        else if (many && few && words <= 64)
            hipLaunchKernelGGL((team_rows_kernel<T, 16, 4>), rows(16), b, 0, s, a);
        else if (many && a.top == 0 && words <= 96)
            hipLaunchKernelGGL((team_rows_kernel<T, 32, 3>), rows(32), b, 0, s, a);
        else if (many && a.top == 0 && words <= 128)
            hipLaunchKernelGGL((team_rows_kernel<T, 32, 4>), rows(32), b, 0, s, a);
        else if (words <= 8) hipLaunchKernelGGL((team_rows_kernel<T, 8, 1>), rows(8), b, 0, s, a);
        else if (words <= 16) hipLaunchKernelGGL((team_rows_kernel<T, 16, 1>), rows(16), b, 0, s, a);
        else if (words <= 32) hipLaunchKernelGGL((team_rows_kernel<T, 32, 1>), rows(32), b, 0, s, a);
        else if (words <= 64) hipLaunchKernelGGL((wave_rows_kernel<T, 1>), rows(64), b, 0, s, a);
        else if (words <= 128) hipLaunchKernelGGL((wave_rows_kernel<T, 2>), rows(64), b, 0, s, a);
        else if (words <= 192) hipLaunchKernelGGL((wave_rows_kernel<T, 3>), rows(64), b, 0, s, a);
        else if (words <= 256) hipLaunchKernelGGL((wave_rows_kernel<T, 4>), rows(64), b, 0, s, a);
        else if (words <= 384) hipLaunchKernelGGL((wave_rows_kernel<T, 6>), rows(64), b, 0, s, a);
        else if (words <= 512) hipLaunchKernelGGL((wave_rows_kernel<T, 8>), rows(64), b, 0, s, a);
        else if constexpr (sizeof(T) == 4) {
            if (words <= 768) hipLaunchKernelGGL((wave_rows_kernel<T, 12>), rows(64), b, 0, s, a);
            else hipLaunchKernelGGL((wave_rows_kernel<T, 16>), rows(64), b, 0, s, a);
        }
        return hipGetLastError();
    }
    const dim3 g(unsigned(a.N), unsigned(a.parts));
    if (a.parts > 1) {
        hipLaunchKernelGGL((long_rows_kernel<T, 256, 4, true>), g, b, 0, s, a);
        hipLaunchKernelGGL((join_rows_kernel<T>), dim3(unsigned(a.N)), b, 0, s, a);
    } else if (a.N >= 2048 && words >= 4096) {
        hipLaunchKernelGGL((long_rows_kernel<T, 256, 8, false>), g, b, 0, s, a);
    } else if (a.N >= 2048) {
        hipLaunchKernelGGL((long_rows_kernel<T, 256, 4, false>), g, b, 0, s, a);
    } else if (a.N >= 512) {
        hipLaunchKernelGGL((long_rows_kernel<T, 512, 4, false>), g, dim3(512), 0, s, a);
    } else {
        hipLaunchKernelGGL((long_rows_kernel<T, 1024, 4, false>), g, dim3(1024), 0, s, a);
    }
    return hipGetLastError();
}

template <typename T> hipError_t backward(const TokenArgs &a, hipStream_t s) {
    const dim3 b(256);
    if (a.A <= kThreadRow) {
        if (packed_rows(a, a.logits, a.stride) && packed_rows(a, a.dlogits, a.dstride))
            return small_backward<T, true>(a, s);
        return small_backward<T, false>(a, s);
    }
    const int words = words_of<T>(a);
    if (words <= kTeamBack) {
        auto rows = [&](int lanes) { return dim3(blocks_of(a.N, 256 / lanes)); };
        const bool many = a.all * words >= 4 * kMany;
        if (words <= 4) hipLaunchKernelGGL((team_back_kernel<T, 4, 1>), rows(4), b, 0, s, a);
        else if (words <= 8) hipLaunchKernelGGL((team_back_kernel<T, 8, 1>), rows(8), b, 0, s, a);
        else if (many && words <= 12)
            hipLaunchKernelGGL((team_back_kernel<T, 4, 3>), rows(4), b, 0, s, a);
        else if (words <= 16) hipLaunchKernelGGL((team_back_kernel<T, 16, 1>), rows(16), b, 0, s, a);
        else if (many && words <= 24)
            hipLaunchKernelGGL((team_back_kernel<T, 8, 3>), rows(8), b, 0, s, a);
        else if (many && words <= 32)
            hipLaunchKernelGGL((team_back_kernel<T, 16, 2>), rows(16), b, 0, s, a);
        else if (many && words <= 48)
            hipLaunchKernelGGL((team_back_kernel<T, 16, 3>), rows(16), b, 0, s, a);
        else if (many && words <= 64)
            hipLaunchKernelGGL((team_back_kernel<T, 16, 4>), rows(16), b, 0, s, a);
        else if (many && words <= 96)
            hipLaunchKernelGGL((team_back_kernel<T, 32, 3>), rows(32), b, 0, s, a);
        else if (words <= 32) hipLaunchKernelGGL((team_back_kernel<T, 32, 1>), rows(32), b, 0, s, a);
        else hipLaunchKernelGGL((team_back_kernel<T, 64, 1>), rows(64), b, 0, s, a);
        return hipGetLastError();
    }
    // enough workgroups for the device where the rows are few
    const int per_row = int(std::max<int64_t>(1, std::min<int64_t>(blocks_of(words, 256),
                                                                   (2048 + a.N - 1) / a.N)));
    hipLaunchKernelGGL((long_back_kernel<T>), dim3(unsigned(a.N), unsigned(per_row)), b, 0, s, a);
    return hipGetLastError();
}

template <typename T> hipError_t draw(const TokenArgs &a, hipStream_t s) {
    const dim3 b(256);
    if (a.A <= 8) hipLaunchKernelGGL((draw_kernel<T, 2, 4>), dim3(blocks_of(a.N, 128)), b, 0, s, a);
    else if (a.A <= 64)
        hipLaunchKernelGGL((draw_kernel<T, 8, 8>), dim3(blocks_of(a.N, 32)), b, 0, s, a);
    else if (a.A <= 128)
        hipLaunchKernelGGL((draw_kernel<T, 16, 8>), dim3(blocks_of(a.N, 16)), b, 0, s, a);
    else hipLaunchKernelGGL((draw_kernel<T, 32, 8>), dim3(blocks_of(a.N, 8)), b, 0, s, a);
    return hipGetLastError();
}

}  // namespace

// Few long rows are cut into parts, so that their exponentials (which bound a row that one compute
// unit takes alone: 131072 choices, 12 us) are shared: up to two parts a compute unit, each of 1024
// words or more (four a thread).
TokenPlan tokens_plan(int64_t N, int64_t A, int top, int dtype) {
    TokenPlan plan{1, 0, 0};
    const int64_t words = A / (dtype == AV_F32 ? 4 : 8);
    if (A > kWaveRow && N > 0 && N <= 256 && words >= 2048) {
        plan.parts = int(std::min<int64_t>({64, 512 / N, words / 1024}));
        plan.keys_off = (size_t(N) * plan.parts * sizeof(Stat) + 15) & ~size_t(15);
        plan.bytes = plan.keys_off + size_t(N) * plan.parts * size_t(top) * sizeof(uint64_t);
    }
    return plan;
}

// Calls f for runs of at most 2^22 rows: a launch has fewer than 2^32 threads, at most 512 a row
// where the rows are many.
template <typename F> static hipError_t in_runs(const TokenArgs &all, int dtype, F f) {
    constexpr int64_t kRun = int64_t(1) << 22;
    const int64_t size = dtype == AV_F32 ? 4 : 2;
    const int64_t id = all.ids_type == AV_IDS_U8 ? 1 : all.ids_type == AV_IDS_I32 ? 4 : 8;
    for (int64_t row = 0; row < all.N; row += kRun) {
        TokenArgs a = all;
        a.N = std::min(kRun, all.N - row);
        a.all = all.N;
        a.logits = static_cast<const char *>(all.logits) + row * all.stride * size;
        if (all.ids) a.ids = static_cast<const char *>(all.ids) + row * id;
        if (all.logp) a.logp += row;
        if (all.entropy) a.entropy += row;
        if (all.stats) a.stats += 2 * row;
        if (all.top_logp) a.top_logp += row * all.top;
        if (all.top_ids) a.top_ids += row * all.top;
        if (all.in_stats) a.in_stats += 2 * row;
        if (all.in_entropy) a.in_entropy += row;
        if (all.dlogp) a.dlogp += row;
        if (all.dentropy) a.dentropy += row;
        if (all.dlogits)
            a.dlogits = static_cast<char *>(all.dlogits) + row * all.dstride * size;
        if (all.uniform) a.uniform += row;
        if (all.actions) a.actions += row;
        const hipError_t e = f(a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_log_probs(const TokenArgs &all, int dtype, hipStream_t s) {
    return in_runs(all, dtype, [&](const TokenArgs &a) {
        switch (dtype) {
            case AV_F32: return forward<float>(a, s);
            case AV_F16: return forward<_Float16>(a, s);
            default: return forward<bf16_t>(a, s);
        }
    });
}

hipError_t launch_log_probs_backward(const TokenArgs &all, int dtype, hipStream_t s) {
    return in_runs(all, dtype, [&](const TokenArgs &a) {
        switch (dtype) {
            case AV_F32: return backward<float>(a, s);
            case AV_F16: return backward<_Float16>(a, s);
            default: return backward<bf16_t>(a, s);
        }
    });
}

hipError_t launch_draw(const TokenArgs &all, int dtype, hipStream_t s) {
    return in_runs(all, dtype, [&](const TokenArgs &a) {
        switch (dtype) {
            case AV_F32: return draw<float>(a, s);
            case AV_F16: return draw<_Float16>(a, s);
            default: return draw<bf16_t>(a, s);
        }
    });
}

}  // namespace av
