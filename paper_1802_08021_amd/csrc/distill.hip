// Distillation on gfx950: divergence of the student's rows from a teacher's
// lists of likely tokens, joined with the loss of given tokens, and its
// gradient.
//
// The outcomes of a row are the listed tokens i, with the teacher's q_i and the
// student's p_i, and, where the rest counts, all other tokens together, with r
// and p_r.  With f the divergence's derivative by ln p of an outcome (-q; p ln(p
// / q); (1 - beta) p ln(p / m)) and F the sum of all f, a logit's derivative is
// f_i - p_i F on the list and p_v (f_r / p_r - F) off it; a given token adds p_v
// - [v == label].  p_r is the sum over the unlisted tokens by itself: as one
// minus the listed it would be lost where the student is sure.  Off the list
// exponentials are taken against the largest unlisted logit, so that p_v / p_r
// is right however small p_r is.
//
// A list's marks, a bit a token, lie in LDS while a row is summed; what is
// computed of a list's entries is in fp64 (a few hundred a row), with logarithms
// within 10^-7, and what is kept of each (q, e, its gradient) in fp32.
#include "rows_device.h"

#include <algorithm>

namespace sparcml {
namespace {

// ---------------------------------------------------------------- a row's list

__device__ __forceinline__ float value_of(const DistillArgs& a, uint64_t i)
{
    if (a.type == kF32) return static_cast<const float*>(a.value)[i];
    if (a.type == kBf16) return (float)static_cast<const __bf16*>(a.value)[i];
    return (float)static_cast<const _Float16*>(a.value)[i];
}

// Entry i of row t: a token that is there, or none (v >= V).
struct Entry {
    uint32_t v;
    float value;
    __device__ __forceinline__ Entry(const DistillArgs& a, uint64_t t, uint32_t i, uint32_t V) : v(0xFFFFFFFFu), value(0.0f)
    {
        if (i >= a.count) return;
        const uint32_t id = (uint32_t)a.id[t * a.ld + i];
        value = value_of(a, t * a.ld + i);
        if (id < V && value != -INFINITY) v = id;
    }
};

__device__ __forceinline__ bool distilled(const Logits& in, const DistillArgs& a, uint64_t t)
{
    return !(in.label && !has_token(in, t)) && !(a.weight && a.weight[t] == 0.0f);
}

// A row's terms of the sums over rows.
struct DistillTerms {
    float div, nll, covered;
};
// What its gradient is made of: off the list A 2^(c (x - top)); the given
// token's part.
struct DistillRow {
    float A, top, given;
};

// e^x in fp64, within 10^-11 of itself: 2^n e^g with |g| <= ln 2 / 2, the
// series of e^g up to g^9.  (The library's own, inlined where it is needed here,
// takes 160 registers.)
__device__ __forceinline__ double exp64(double x)
{
    const double n = rint(fmin(fmax(x, -2000.0), 2000.0) * 1.4426950408889634);
    const double g = __builtin_fma(n, -0.6931471805599453, fmin(fmax(x, -2000.0), 2000.0));
    double y = 1.0 / 362880.0;
    const double series[9] = {1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0};
#pragma unroll
    for (int i = 0; i < 9; ++i) y = __builtin_fma(y, g, series[i]);
    y = ldexp(y, (int)n);
    return x != x ? x : x == -INFINITY ? 0.0 : y;
}
// ln x in fp64, as part_ln takes it: within 10^-7.
__device__ __forceinline__ double ln64(double x)
{
    if (!(x > 0.0 && x < INFINITY)) return x == 0.0 ? -INFINITY : x;
    int e;
    double m = frexp(x, &e);
    if (m < 0.7071067811865476) {
        m *= 2.0;
        --e;
    }
    // (what is left of the rounding to fp32 is its own logarithm's first term)
    const float f = (float)m;
    return ((double)e + (double)__builtin_amdgcn_logf(f)) * 0.6931471805599453 + (m - (double)f) / (double)f;
}

// One outcome's share of the divergence and its derivative by the student's
// log probability (lq, lp: log probabilities; a probability of 0 takes an
// infinity away).
struct Share {
    double div, f;
};
__device__ __forceinline__ double product(double p, double x) { return p == 0.0 ? 0.0 : p * x; }
__device__ __forceinline__ Share share_of(float beta, double lq, double lp)
{
    const double q = exp64(lq), p = exp64(lp), b = (double)beta;
    Share r;
    if (beta == 0.0f) {
        r.div = product(q, lq - lp);
        r.f = -q;
    } else if (beta == 1.0f) {
        r.div = r.f = product(p, lp - lq);
    } else {
        const double lm = ln64(b * q + (1.0 - b) * p);
        r.f = (1.0 - b) * product(p, lp - lm);
        r.div = b * product(q, lq - lm) + r.f;
    }
    if (lp == -INFINITY) r.f = 0.0;  // (a logit of -Inf does not move)
    return r;
}

// LDS accesses of one wave before and behind this keep their order.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A row's list in LDS, made by one wave: entries lane, lane + 64, ...  What
// depends on the list alone (take, prepare) is there before the row's sum, so
// that little is left to do behind it (finish).
struct List {
    uint32_t id[kMaxTop];
    float value[kMaxTop], x[kMaxTop];  // the teacher's value, the student's logit
    float q[kMaxTop], e[kMaxTop];      // the teacher's probability; e^(scale (x - top)), then the token's gradient
    uint32_t dup;
    DistillRow row;
    DistillTerms terms;

    __device__ __forceinline__ bool there(uint32_t i, uint32_t V) const { return id[i] < V; }
    // Entries that repeat an earlier one go (dup: there is one).
    __device__ __forceinline__ void drop_repeats(uint32_t count)
    {
        wave_fence();
        if (!dup) return;
        const uint32_t lane = threadIdx.x & 63;
        uint32_t v[kMaxTop / 64], again = 0;
#pragma unroll
        for (uint32_t k = 0; k < kMaxTop / 64; ++k) v[k] = lane + 64 * k < count ? id[lane + 64 * k] : 0u;
#pragma unroll 8
        for (uint32_t j = 0; j < count; ++j) {
            const uint32_t w = id[j];
#pragma unroll
            for (uint32_t k = 0; k < kMaxTop / 64; ++k) again |= (uint32_t)(w == v[k] && j < lane + 64 * k) << k;
        }
        wave_fence();
#pragma unroll
        for (uint32_t k = 0; k < kMaxTop / 64; ++k)
            if (lane + 64 * k < count && (again >> k & 1u)) id[lane + 64 * k] = 0xFFFFFFFFu;
        wave_fence();
    }
};

// Sums over a list: its largest logit (-Inf: there is none), ln q = value ts - off,
// Q = sum q, Z = sum e, and with the weights that beta needs (q, or e for beta 1),
// as the list holds them in fp32, the products with logarithms (u against lq, w
// against scale (x - top)) and the weights themselves without tokens of -Inf:
// roundings of the weights then weigh differences of logarithms alone, which are
// 0 where student and teacher agree.
struct ListSums {
    float top;
    double ts, off, Q, Z, u, w, mass;
};
__device__ __forceinline__ ListSums prepare_list(const DistillArgs& a, double scale, uint32_t V, List& list)
{
    const uint32_t lane = threadIdx.x & 63;
    ListSums s = {-INFINITY, a.rest ? 1.0 : (double)a.teacher_scale, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
    float best = -INFINITY;
    for (uint32_t i = lane; i < a.count; i += 64)
        if (list.there(i, V)) {
            s.top = fmaxf(s.top, list.x[i]);
            best = fmaxf(best, list.value[i]);
        }
    s.top = wave_join<false>(s.top);
    best = a.rest ? 0.0f : wave_join<false>(best);
    const float top = s.top == -INFINITY ? 0.0f : s.top;
#pragma unroll 1
    for (uint32_t i = lane; i < a.count; i += 64)
        if (list.there(i, V)) {
            const double q = exp64(((double)list.value[i] - (double)best) * s.ts);
            const double e = exp64(((double)list.x[i] - (double)top) * scale);
            list.q[i] = (float)q;
            list.e[i] = (float)e;
            s.Q += q;
            s.Z += e;
        }
    s.Q = wave_sum(s.Q);
    s.Z = wave_sum(s.Z);
    double each = 1.0;
    if (!a.rest && s.Q != 0.0) {
        s.off = (double)best * s.ts + ln64(s.Q);
        each = 1.0 / s.Q;
        s.Q = s.Q == s.Q ? 1.0 : s.Q;
    }
    const bool back = a.beta == 1.0f;  // (otherwise only beta == 0 has a use for these)
    for (uint32_t i = lane; i < a.count; i += 64)
        if (list.there(i, V)) {
            const double q = (double)list.q[i] * each, p = back ? (double)list.e[i] : q;
            list.q[i] = (float)q;
            s.u += product(p, (double)list.value[i] * s.ts - s.off);
            s.w += product(p, ((double)list.x[i] - (double)top) * scale);
            s.mass += list.x[i] == -INFINITY ? 0.0 : p;
        }
    s.u = wave_sum(s.u);
    s.w = wave_sum(s.w);
    s.mass = wave_sum(s.mass);
    return s;
}

// A row's terms and its list's gradients from the sum over the unlisted tokens,
// by the same wave; at: the given token's logit, label the token or none.
__device__ __forceinline__ void finish_list(const DistillArgs& a, double scale, uint32_t V, const ListSums& s,
                                            const Part& rest, uint32_t label, float at, double weight, List& list)
{
    const uint32_t lane = threadIdx.x & 63;
    const bool outside = rest.sum != 0.0f;
    const float M = fmaxf(s.top, outside ? rest.top : -INFINITY);
    if (M == -INFINITY && s.Z == 0.0) {  // nothing but -Inf (a sum of NaN has no largest)
        for (uint32_t i = lane; i < a.count; i += 64) list.e[i] = 0.0f;
        if (lane == 0) {
            list.row = DistillRow{0.0f, 0.0f, __builtin_nanf("")};
            list.terms = DistillTerms{0.0f, 0.0f, 0.0f};
        }
        return;
    }
    // against M: the list's part, the rest's; ln p = scale (x - top) - ln
    const float top = s.top == -INFINITY ? M : s.top;
    const double step = ((double)top - (double)M) * scale, far = outside ? ((double)rest.top - (double)M) * scale : 0.0;
    const double g = exp64(step), h = outside ? exp64(far) : 0.0;
    const double total = g * s.Z + h * (double)rest.sum, all = ln64(total), ln = all - step, one = g / total;
    double div, F;
    if (a.beta == 0.0f) {
        div = s.u - s.w + ln * s.mass;  // (w takes a token of -Inf)
        F = -s.mass;
    } else if (a.beta == 1.0f) {
        div = F = one * (s.w - s.u - ln * s.mass);
    } else {
        div = F = 0.0;
        const double b = (double)a.beta;
#pragma unroll 1
        for (uint32_t i = lane; i < a.count; i += 64)
            if (list.there(i, V)) {
                const double lp = ((double)list.x[i] - (double)top) * scale - ln, q = (double)list.q[i];
                const double p = (double)list.e[i] * one, lm = ln64(b * q + (1.0 - b) * p);
                const double f = (1.0 - b) * product(p, lp - lm);
                div += b * product(q, (double)list.value[i] * s.ts - s.off - lm) + f;
                F += f;
                list.q[i] = (float)f;
            }
        div = wave_sum(div);
        F = wave_sum(F);
    }
    Share out = {0.0, 0.0};
    if (a.rest && outside) out = share_of(a.beta, ln64(fmax(1.0 - s.Q, 0x1p-24)), far + part_ln(rest.sum) - all);
    div += out.div;
    F += out.f;
    // (NaN among the values: a token that the student gives nothing hides it
    // from every product, but not from Q)
    if (s.Q != s.Q) div = F = s.Q;
    const double soft = 1.0 - (double)a.hard, hard = at != -INFINITY ? (double)a.hard : 0.0;
    const double k0 = (double)within((float)(weight * (double)a.grad_scale * scale));
    const double both = hard - soft * F;
    bool listed = false;
    for (uint32_t i = lane; i < a.count; i += 64)
        if (list.there(i, V)) {
            const double p = (double)list.e[i] * one;
            double f = a.beta == 0.0f ? list.x[i] == -INFINITY ? 0.0 : -(double)list.q[i] : (double)list.q[i];
            if (a.beta == 1.0f)
                f = product(p, ((double)list.x[i] - (double)top) * scale - ln - ((double)list.value[i] * s.ts - s.off));
            const bool given = list.id[i] == label;
            list.e[i] = within((float)(k0 * (soft * f + p * both - (given ? hard : 0.0))));
            listed |= given;
        }
    listed = __any(listed);
    if (lane == 0) {
        const float A = outside ? within((float)(k0 * (soft * out.f / (double)rest.sum + both * h / total))) : 0.0f;
        // (NaN where the token has its place on the list, or none)
        const float given = listed || hard == 0.0
                                ? __builtin_nanf("")
                                : within((float)((double)A * exp64(((double)at - (double)rest.top) * scale) - k0 * hard));
        list.row = DistillRow{A, rest.top, given};
        const double nll = label < V ? all - ((double)at - (double)M) * scale : 0.0;
        list.terms = DistillTerms{(float)div, (float)nll, (float)(s.Z * one)};
    }
}

// Marks of a piece's elements (a bit each) and what is left of the piece
// without them.
template <int TYPE>
__device__ __forceinline__ uint32_t marks_of(const uint32_t* marks, uint32_t j)
{
    constexpr uint32_t N = Piece<TYPE>::N;
    return marks[j * N / 32] >> (j * N % 32) & ((1u << N) - 1);
}
template <int TYPE>
__device__ __forceinline__ void hide(Piece<TYPE>& x, uint32_t marks)
{
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t two = marks >> (i * Piece<TYPE>::N / 4);
        const uint32_t m = TYPE == kF32 ? (two & 1u ? ~0u : 0u) : (two & 1u ? 0xFFFFu : 0u) | (two & 2u ? 0xFFFF0000u : 0u);
        x.w[i] = (x.w[i] & ~m) | (Piece<TYPE>::kNone & m);
    }
}

// ---------------------------------------------------------------- sums

constexpr uint32_t kWindow = 4096;  // pieces whose marks lie in LDS at a time

// What the first of two launches leaves of a row's list: five arrays of `count`
// (tokens, values, logits, q, e), and its sums.
struct Prepared {
    float* arrays;  // [rows][5][count]
    ListSums* sums;
    float* at_label;
};
constexpr uint32_t kTable = 1024;  // places for a list's tokens, to find repeats

// Slice s of a row, as k_slices takes them: (M, Z) over the unlisted tokens.
// Slice S is the row's list.
template <int TYPE>
__global__ void __launch_bounds__(256) k_rest_slices(Logits in, DistillArgs a, uint32_t S, uint32_t W, float c, Part* part,
                                                     Prepared to, uint32_t* ticket)
{
    typedef typename Elem<TYPE>::type E;
    constexpr uint32_t N = Piece<TYPE>::N, kMarks = kWindow * N / 32, kListWords = (sizeof(List) + 3) / 4 + kTable;
    __shared__ float s_top[4], s_sum[4];
    __shared__ uint32_t s_words[kMarks > kListWords ? kMarks : kListWords], s_single[4];
    uint32_t* const s_marks = s_words;
    const uint32_t tid = threadIdx.x, V = (uint32_t)in.vocab;
    if (blockIdx.x == 0 && tid == 0) *ticket = 0;  // for k_distill_grad
    for (uint64_t b = blockIdx.x; b < in.rows * (S + 1); b += gridDim.x) {
        const uint64_t t = b / (S + 1);
        const uint32_t s = (uint32_t)(b % (S + 1));
        if (!distilled(in, a, t)) continue;
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        if (s == S) {
            List& list = *reinterpret_cast<List*>(s_words + kTable);
            const Entry e(a, t, tid, V);
            for (uint32_t i = tid; i < kTable; i += 256) s_words[i] = 0xFFFFFFFFu;
            if (tid == 0) list.dup = 0;
            list.id[tid] = e.v;
            list.value[tid] = e.value;
            list.x[tid] = e.v < V ? (float)row[e.v] : -INFINITY;
            if (tid == 0) to.at_label[t] = in.label ? (float)row[in.label[t]] : -INFINITY;
            __syncthreads();
            if (e.v < V)
                for (uint32_t h = e.v * 2654435761u >> 22;; h = (h + 1) % kTable) {  // (a quarter of them are taken at most)
                    const uint32_t was = atomicCAS(&s_words[h], 0xFFFFFFFFu, e.v);
                    if (was == e.v) list.dup = 1;
                    if (was == e.v || was == 0xFFFFFFFFu) break;
                }
            __syncthreads();
            if (tid < 64) {
                list.drop_repeats(a.count);
                const ListSums sums = prepare_list(a, (double)in.scale, V, list);
                if (tid == 0) to.sums[t] = sums;
            }
            __syncthreads();
            if (tid < a.count) {
                float* out = to.arrays + t * 5 * a.count + tid;
                out[0] = __uint_as_float(list.id[tid]);
                out[a.count] = list.value[tid];
                out[2 * a.count] = list.x[tid];
                out[3 * a.count] = list.q[tid];
                out[4 * a.count] = list.e[tid];
            }
            __syncthreads();
            continue;
        }
        const RowCut<TYPE> r(row, V);
        const uint32_t first = (uint32_t)min((uint64_t)r.full, (uint64_t)s * W);
        const uint32_t end = (uint32_t)min((uint64_t)r.full, (uint64_t)(s + 1) * W);
        const Entry mine(a, t, tid, V);
        if (tid < 4) s_single[tid] = 0;
        Own own = {-INFINITY, 0.0f};
        for (uint32_t at = first; at < end || at == first; at += kWindow) {
            const uint32_t stop = min(end, at + kWindow);
            for (uint32_t i = tid; i < (stop - at) * N / 32 + 1 && i < kWindow * N / 32; i += 256) s_marks[i] = 0;
            __syncthreads();
            if (mine.v < V) {
                if (r.in_piece(mine.v)) {
                    const uint32_t bit = mine.v - r.head - at * N;  // (below the window: wraps beyond it)
                    if ((mine.v - r.head) / N >= at && bit < (stop - at) * N) atomicOr(&s_marks[bit / 32], 1u << (bit % 32));
                } else if (at == first) {
                    const uint32_t i = mine.v < r.head ? mine.v : mine.v - r.full * N;
                    atomicOr(&s_single[i / 32], 1u << (i % 32));
                }
            }
            __syncthreads();
            if (at == first && s == 0 && tid < r.singles && !(s_single[tid / 32] >> (tid % 32) & 1u)) {
                const float x = (float)row[r.single(tid)];
                own = Own{x, x == -INFINITY ? 0.0f : 1.0f};
            }
            for (uint32_t j = at + tid; j < stop; j += 256) {
                Piece<TYPE> x[1];
                x[0].w = load_vec<u32x4, true>(row + r.piece(j));
                const uint32_t marks = marks_of<TYPE>(s_marks, j - at);
                if (marks) hide(x[0], marks);
                own.add(x, 1, c);
            }
            __syncthreads();
        }
        float high = join_waves<false>(own.top, s_top);
        if (high == -INFINITY) high = 0.0f;
        const float sum = join_waves<true>(own.sum * exp2_fast((own.top - high) * c), s_sum);
        if (tid == 0) part[t * S + s] = Part{high, sum};
        __syncthreads();
    }
}

// ---------------------------------------------------------------- a workgroup a row

// Row blockIdx.x by one workgroup, whose first wave has the list, and the others
// the row, as k_row takes it (the first NV pieces of a thread in registers
// between the passes, LP more in LDS, the rest read once more): the list's
// marks, the sum over the unlisted tokens beside the list's own sums, the row's
// terms, the gradient, and behind it the listed and the given token's places
// once more.
template <int TYPE, int THREADS, int NV, int LP>
__global__ void __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(8)))
k_distill_row(Logits in, DistillArgs a, float c, float* div, DistillTerms* terms, void* dlogits, uint64_t ldd)
{
    typedef typename Elem<TYPE>::type E;
    constexpr int N = Piece<TYPE>::N;
    extern __shared__ uint32_t s_marks[];
    __shared__ u32x4 s_keep[LP ? LP * (THREADS - 64) : 1];
    __shared__ Part s_part[THREADS / 64];
    __shared__ uint32_t s_single[4];
    __shared__ List s_list;
    const uint64_t t = blockIdx.x;
    const uint32_t V = (uint32_t)in.vocab, lane = threadIdx.x & 63;
    const E* row = static_cast<const E*>(in.x) + t * in.ld;
    E* out = static_cast<E*>(dlogits) + t * ldd;
    if (!distilled(in, a, t)) {
        if (threadIdx.x == 0) {
            div[t] = 0.0f;
            terms[t] = DistillTerms{0.0f, 0.0f, 0.0f};
        }
        if (dlogits) clear_row<TYPE>(out, V);
        return;
    }
    const RowCut<TYPE> r(row, V);
    const uint32_t words = (r.full * N + 31) / 32;
    for (uint32_t i = threadIdx.x; i < words; i += blockDim.x) s_marks[i] = 0;
    if (threadIdx.x < 4) s_single[threadIdx.x] = 0;
    if (threadIdx.x == 4) s_list.dup = 0;
    // (a branch of whole waves: both sides have their own barriers, five each, or
    // three without a gradient)
    if ((uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x) < 64) {
        const double scale = (double)in.scale;
        for (uint32_t i = lane; i < a.count; i += 64) {
            const Entry e(a, t, i, V);
            s_list.id[i] = e.v;
            s_list.value[i] = e.value;
        }
        __syncthreads();
        for (uint32_t i = lane; i < a.count; i += 64) {
            const uint32_t v = s_list.id[i];
            if (v >= V) continue;
            const bool in_piece = r.in_piece(v);
            const uint32_t bit = in_piece ? v - r.head : v < r.head ? v : v - r.full * N;
            uint32_t* word = (in_piece ? s_marks : s_single) + bit / 32;
            if (atomicOr(word, 1u << (bit % 32)) >> (bit % 32) & 1u) s_list.dup = 1;
        }
        __syncthreads();
        s_list.drop_repeats(a.count);
        for (uint32_t i = lane; i < a.count; i += 64) {
            const uint32_t v = s_list.id[i];
            if (v < V) s_list.x[i] = (float)row[v];
        }
        const uint32_t label = in.label ? (uint32_t)in.label[t] : 0xFFFFFFFFu;
        const float at = in.label ? (float)row[label] : -INFINITY;
        const double weight = a.weight ? (double)a.weight[t] : 1.0;
        const ListSums sums = prepare_list(a, scale, V, s_list);
        __syncthreads();
        finish_list(a, scale, V, sums, join_slices(s_part, blockDim.x / 64 - 1, 64, c), label, at, weight, s_list);
        wave_fence();
        if (lane == 0) {
            div[t] = s_list.terms.div;
            terms[t] = s_list.terms;
        }
        if (!dlogits) return;
        __syncthreads();
        __syncthreads();
        for (uint32_t i = lane; i < a.count; i += 64)
            if (s_list.id[i] < V) out[s_list.id[i]] = (E)s_list.e[i];
        if (lane == 0 && s_list.row.given == s_list.row.given) out[label] = (E)s_list.row.given;
        return;
    }
    const uint32_t tid = threadIdx.x - 64, step = blockDim.x - 64;
    const int used = (int)min((r.full + step - 1) / step, (uint32_t)NV);
    Piece<TYPE> x[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        x[j].none();
        if (tid + step * j < r.full) x[j].w = load_vec<u32x4>(row + r.piece(tid + step * j));
    }
    float single = tid < r.singles ? (float)row[r.single(tid)] : -INFINITY;
    __syncthreads();
    __syncthreads();
    if (tid < r.singles && s_single[tid / 32] >> (tid % 32) & 1u) single = -INFINITY;
    Own own = {single, single == -INFINITY ? 0.0f : 1.0f};
    for (uint32_t j = tid + step * NV, slot = tid; j < r.full; j += step, slot += step) {
        Piece<TYPE> q[1];
        q[0].w = load_vec<u32x4, true>(row + r.piece(j));
        const uint32_t marks = marks_of<TYPE>(s_marks, j);
        if (marks) hide(q[0], marks);
        own.add(q, 1, c);
        if (LP && slot < LP * step) s_keep[slot] = q[0].w;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i >= used) break;
        const uint32_t j = tid + step * i, marks = j < r.full ? marks_of<TYPE>(s_marks, j) : 0u;
        if (marks) hide(x[i], marks);
    }
    own.add(x, used, c);
    {
        float top = wave_join<false>(own.top);
        if (top == -INFINITY) top = 0.0f;
        const float sum = wave_join<true>(own.sum * exp2_fast((own.top - top) * c));
        if (lane == 0) s_part[tid >> 6] = Part{top, sum};
    }
    __syncthreads();
    if (!dlogits) return;
    uint32_t j = tid + step * (NV + LP);
    Piece<TYPE> next;
    if (j < r.full) next.w = load_vec<u32x4>(row + r.piece(j));
    __syncthreads();
    const float A = s_list.row.A, top = s_list.row.top;
    auto write = [&](Piece<TYPE>& q, uint32_t at) {
        q.repack();
        float z[N];
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = entry(q.get(i), c, top, A);
        q.put(z);
        if (at < r.full) store_vec(out + r.piece(at), q.w);
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i >= used) break;
        write(x[i], tid + step * i);
    }
    for (uint32_t i = 0; i < (uint32_t)LP && tid + step * (NV + i) < r.full; ++i) {
        Piece<TYPE> now;
        now.w = s_keep[tid + step * i];
        write(now, tid + step * (NV + i));
    }
    for (; j < r.full; j += step) {
        Piece<TYPE> now = next;
        if (j + step < r.full) next.w = load_vec<u32x4>(row + r.piece(j + step));
        write(now, j);
    }
    if (tid < r.singles) out[r.single(tid)] = (E)entry(single, c, top, A);
    // (every store before this is done before the next ones begin)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// ---------------------------------------------------------------- gradient by slices

// A factor of 0 takes an infinity away (not NaN).
__device__ __forceinline__ double weighed(double w, double x) { return w == 0.0 && x == x ? 0.0 : w * x; }

// The sums over rows, by one workgroup (fixed order).
template <int U, class Load>
__device__ __forceinline__ void put_distill_stats(const Logits& in, const DistillArgs& a, double (*s_w)[4], float* stats,
                                                  Load load)
{
    double x[4] = {0.0, 0.0, 0.0, 0.0};
    const double soft = 1.0 - (double)a.hard;
    // (U rows' loads under way at a time)
    for (uint64_t t0 = threadIdx.x; t0 < in.rows; t0 += U * blockDim.x) {
        DistillTerms d[U];
        float w[U];
        bool use[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint64_t t = min(t0 + u * blockDim.x, in.rows - 1);
            d[u] = load(t);
            w[u] = a.weight ? a.weight[t] : 1.0f;
            use[u] = (!in.label || has_token(in, t)) & (w[u] != 0.0f) & (t0 + u * blockDim.x < in.rows);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!use[u]) continue;
            const double v = (double)w[u];
            x[0] += v * (weighed(soft, (double)d[u].div) + weighed((double)a.hard, (double)d[u].nll));
            x[1] += v * (double)d[u].div;
            x[2] += v * (double)d[u].nll;
            x[3] += v * (double)d[u].covered;
        }
    }
    block_sum(x, s_w, 4);
    if (threadIdx.x == 0)
        for (int i = 0; i < 4; ++i) stats[i] = (float)x[i];
}
__global__ void __launch_bounds__(1024) k_distill_stats(Logits in, DistillArgs a, const DistillTerms* terms, float* stats)
{
    __shared__ double s_w[16][4];
    put_distill_stats<8>(in, a, s_w, stats, [&](uint64_t t) { return terms[t]; });
}

constexpr int kDistillU = 2;

// Slice s of a gradient row, 256 kDistillU pieces; every workgroup finds its
// row's terms, a row's first writes them, and the last of these to finish sums
// them up.  (Without a gradient: G == 1, nothing but that.)
template <int TYPE>
__global__ void __launch_bounds__(256) k_distill_grad(Logits in, DistillArgs a, uint32_t S, uint32_t G, float c,
                                                      const Part* part, Prepared from, DistillTerms* terms,
                                                      uint32_t* ticket, float* div, float* stats, void* dlogits,
                                                      uint64_t ldd)
{
    typedef typename Elem<TYPE>::type E;
    constexpr int N = Piece<TYPE>::N, U = kDistillU;
    __shared__ double s_w[4][4];
    __shared__ List s_list;
    __shared__ uint32_t s_last;
    const uint32_t tid = threadIdx.x, V = (uint32_t)in.vocab;
    bool last = false;
    for (uint64_t b = blockIdx.x; b < in.rows * G; b += gridDim.x) {
        const uint64_t t = b / G;
        const uint32_t s = (uint32_t)(b % G);
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        E* out = static_cast<E*>(dlogits) + t * ldd;
        const RowCut<TYPE> r(row, dlogits ? V : 0);
        const uint32_t first = min(r.full, s * (256 * U)), end = min(r.full, first + 256 * U);
        const bool use = distilled(in, a, t);
        float single = -INFINITY;
        Piece<TYPE> y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            y[u].none();
            if (use && first + tid + 256 * u < end) y[u].w = load_vec<u32x4>(row + r.piece(first + tid + 256 * u));
        }
        if (use && s == 0 && tid < r.singles) single = (float)row[r.single(tid)];
        DistillTerms d = {0.0f, 0.0f, 0.0f};
        if (use) {
            if (tid < a.count) {
                const float* list = from.arrays + t * 5 * a.count + tid;
                s_list.id[tid] = __float_as_uint(list[0]);
                s_list.value[tid] = list[a.count];
                s_list.x[tid] = list[2 * a.count];
                s_list.q[tid] = list[3 * a.count];
                s_list.e[tid] = list[4 * a.count];
            }
            const ListSums sums = from.sums[t];
            __syncthreads();
            if (tid < 64)
                finish_list(a, (double)in.scale, V, sums, join_slices(part + t * S, S, 64, c),
                            in.label ? (uint32_t)in.label[t] : 0xFFFFFFFFu, from.at_label[t],
                            a.weight ? (double)a.weight[t] : 1.0, s_list);
            __syncthreads();
            d = s_list.terms;
        }
        if (s == 0 && tid == 0) {
            div[t] = d.div;
            // (device-scope accesses, each done before the next)
            float* w = &terms[t].div;
            for (int i = 0; i < 3; ++i)
                __hip_atomic_store(w + i, i == 0 ? d.div : i == 1 ? d.nll : d.covered, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            last = atomicAdd(ticket, 1u) == (uint32_t)in.rows - 1;
        }
        if (!dlogits) {
            __syncthreads();
            continue;
        }
        const float A = use ? s_list.row.A : 0.0f, top = use ? s_list.row.top : 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float z[N];
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = A == 0.0f ? 0.0f : entry(y[u].get(i), c, top, A);
            y[u].put(z);
            if (first + tid + 256 * u < end) store_vec(out + r.piece(first + tid + 256 * u), y[u].w);
        }
        if (s == 0 && tid < r.singles) out[r.single(tid)] = (E)(A == 0.0f ? 0.0f : entry(single, c, top, A));
        // (every store before this is done before the next ones begin)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (use) {
            auto inside = [&](uint32_t v) {
                if (v >= V) return false;
                if (!r.in_piece(v)) return s == 0;
                return (v - r.head) / N >= first && (v - r.head) / N < end;
            };
            if (tid < a.count && inside(s_list.id[tid])) out[s_list.id[tid]] = (E)s_list.e[tid];
            const float given = s_list.row.given;
            if (tid == 0 && given == given && inside((uint32_t)in.label[t])) out[in.label[t]] = (E)given;
        }
        __syncthreads();
    }
    if (tid == 0) s_last = last;
    __syncthreads();
    if (!s_last) return;
    put_distill_stats<1>(in, a, s_w, stats, [&](uint64_t t) {
        float w[3];
        for (int i = 0; i < 3; ++i)
            w[i] = __hip_atomic_load(&terms[t].div + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return DistillTerms{w[0], w[1], w[2]};
    });
}

// ---------------------------------------------------------------- host

constexpr uint32_t kDistillGrid = 1u << 22;
constexpr uint64_t kDistillSlices = 1024;   // of few rows together
// From so many rows on a workgroup a row, whose pieces it holds (bf16 with 64
// tokens: 64 x 131072 30 us against 25 by slices and two launches, 128 x 131072
// 30 against 38; 64 x 32000 16 against 15, 200 x 32000 17 against 24),
constexpr uint64_t kDistillMany = 128;
// of at most so many logits, 20 KB of marks.  (The two forms do not cross here: bf16
// with 64 tokens 4096 x 163840 527 us against 1219 by slices, and with 32 KB of marks
// 201088 661 against 1509, 262144 1000 against 1922, 128 x 200000 44 against 53; 512
// x 170000 fp32 156 against 278.  Longer rows would gain by more room for marks.)
constexpr uint64_t kMarked = 5 * 32768;
constexpr uint64_t kDistillRows = 1u << 21; // of a launch with a workgroup a row (fewer than 2^32 threads)
constexpr uint32_t kDistillHold = 8, kDistillHoldLds = 3;

struct DistillCut {
    uint32_t S, W, G;
    uint64_t pieces;
    bool many;
};
uint64_t most_rest_slices(uint64_t pieces) { return std::min<uint64_t>(64, (pieces + 511) / 512); }
DistillCut cut_distill(uint64_t rows, uint64_t vocab, uint32_t type)
{
    DistillCut r;
    r.pieces = vocab / (type == kF32 ? 4 : 8) + 1;
    r.many = rows >= kDistillMany && vocab <= kMarked;
    const uint64_t want = kDistillSlices / std::min(rows, kDistillSlices);
    const uint64_t S = std::max<uint64_t>(1, std::min(most_rest_slices(r.pieces), want));
    r.W = (uint32_t)((r.pieces + S - 1) / S);
    r.S = (uint32_t)((r.pieces + r.W - 1) / r.W);
    r.G = (uint32_t)((r.pieces + 256 * kDistillU - 1) / (256 * kDistillU));
    return r;
}

struct DistillSpace {
    DistillTerms* terms;
    uint32_t* ticket;
    Part* part;
    Prepared lists;
};
DistillSpace carve_distill(void* ws, uint64_t rows, uint64_t sliced, uint64_t parts, uint32_t count, size_t* bytes)
{
    Carve c(ws);
    DistillSpace r;
    r.terms = c.take<DistillTerms>(rows);
    r.ticket = c.take<uint32_t>(1);
    r.part = c.take<Part>(parts);
    r.lists.arrays = c.take<float>(sliced * 5 * count);
    r.lists.sums = c.take<ListSums>(sliced);
    r.lists.at_label = c.take<float>(sliced);
    if (bytes) *bytes = c.used;
    return r;
}

}  // namespace

// (Enough for every type and every call of fewer rows, a smaller vocabulary or
// shorter lists: what is counted are the rows that may go by slices.)
size_t distill_workspace(uint32_t count, uint64_t rows, uint64_t vocab)
{
    size_t b = 0;
    const uint64_t sliced = vocab > kMarked ? rows : std::min(rows, kDistillMany - 1);
    const uint64_t parts = std::max(sliced, std::min(kDistillSlices, sliced * most_rest_slices(vocab / 4 + 1)));
    carve_distill(nullptr, rows, sliced, parts, count, &b);
    return b;
}

hipError_t distill_run(const Logits& in0, const DistillArgs& a0, float* div, float* stats, void* dlogits, uint64_t ldd,
                       void* ws, hipStream_t s)
{
    Logits in = in0;
    DistillArgs a = a0;
    const DistillCut cut = cut_distill(in.rows, in.vocab, in.type);
    const float c = log2_scale(in.scale);
    if (!cut.many) {
        const DistillSpace sp = carve_distill(ws, in.rows, in.rows, in.rows * cut.S, a.count, nullptr);
        const uint32_t slices = (uint32_t)std::min<uint64_t>(in.rows * (cut.S + 1), kDistillGrid);
        const uint32_t G = dlogits ? cut.G : 1, grads = (uint32_t)std::min<uint64_t>(in.rows * G, kDistillGrid);
        by_type(in.type, [&](auto ty) {
            constexpr int TY = decltype(ty)::value;
            timer_begin(kTLossRows, s);
            hipLaunchKernelGGL((k_rest_slices<TY>), dim3(slices), dim3(256), 0, s, in, a, cut.S, cut.W, c, sp.part, sp.lists,
                               sp.ticket);
            timer_end(kTLossRows, s);
            timer_begin(kTLossGrad, s);
            hipLaunchKernelGGL((k_distill_grad<TY>), dim3(grads), dim3(256), 0, s, in, a, cut.S, G, c, sp.part, sp.lists,
                               sp.terms, sp.ticket, div, stats, dlogits, ldd);
            timer_end(kTLossGrad, s);
        });
        return hipGetLastError();
    }
    const DistillSpace sp = carve_distill(ws, in.rows, 0, 0, a.count, nullptr);
    // Threads of a row: 512 up to 7168 pieces (4096 x 56000 bf16 with 64 tokens 179
    // us against 183 with 1024, 60000 197 against 189; 2000 x 30000 fp32 99 against
    // 95), with pieces in LDS too (50001: 155 us against 166 without, 172 with 1024
    // threads; where several batches in turn leave nothing in cache 191, 195 with
    // 1024 threads).
    const uint64_t most = cut.pieces <= 7168 ? 512 : 1024, size = in.type == kF32 ? 4 : 2;
    const uint64_t threads = 64 + std::max<uint64_t>(kMinThreads, (cut.pieces + kDistillHold * 64 - 1) / (kDistillHold * 64) * 64);
    const size_t lds = (in.vocab + 31) / 32 * 4 + 4;
    timer_begin(kTLossRows, s);
    by_type(in.type, [&](auto ty) {
        constexpr int TY = decltype(ty)::value;
        for (uint64_t r0 = 0; r0 < in0.rows; r0 += kDistillRows) {
            const dim3 grid((uint32_t)std::min(in0.rows - r0, kDistillRows)), block((uint32_t)std::min(threads, most));
            in.x = static_cast<const uint8_t*>(in0.x) + r0 * in.ld * size;
            in.label = in0.label ? in0.label + r0 : nullptr;
            a.id = a0.id + r0 * a.ld;
            a.value = static_cast<const uint8_t*>(a0.value) + r0 * a.ld * (a.type == kF32 ? 4 : 2);
            a.weight = a0.weight ? a0.weight + r0 : nullptr;
            void* d = dlogits ? static_cast<uint8_t*>(dlogits) + r0 * ldd * size : nullptr;
            auto go = [&](auto kern) {
                hipLaunchKernelGGL(kern, grid, block, lds, s, in, a, c, div + r0, sp.terms + r0, d, ldd);
            };
            if (most == 512)
                go(k_distill_row<TY, 512, kDistillHold, kDistillHoldLds>);
            else
                go(k_distill_row<TY, 1024, kDistillHold, kDistillHoldLds>);
        }
    });
    timer_end(kTLossRows, s);
    timer_begin(kTLossGrad, s);
    hipLaunchKernelGGL(k_distill_stats, dim3(1), dim3(1024), 0, s, in0, a0, sp.terms, stats);
    timer_end(kTLossGrad, s);
    return hipGetLastError();
}

}  // namespace sparcml
