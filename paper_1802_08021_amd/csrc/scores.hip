// What rows of logits say, on gfx950: log probability of each row's token, log
// of the row's sum, entropy, and the most likely tokens in order; and the
// gradient of a loss over these.
//
// With x the row's logits, M their maximum, s the inverse temperature, c = s
// log2(e), d_v = c (x_v - M), Z = sum_v 2^d_v and U = sum_v -d_v 2^d_v: log
// probabilities are ln 2 (d_v - log2 Z), the entropy is ln 2 (log2 Z + U / Z).
// Both of its terms are positive, so nothing cancels.  U moves with the maximum
// as Z does: from M to M' it becomes 2^-h (U + h Z), h = c (M' - M).
//
// The n most likely tokens of a row: every thread of a workgroup has the
// largest logit that it has seen, and the n-th largest of these is a bound
// that at least n logits reach, few more do (of 1024 threads about 66 for n =
// 64).  The rows of threads below it need no second look; those of the others
// are looked through once more, and what reaches the bound is put in order.
#include "rows_device.h"

#include <algorithm>

namespace sparcml {
namespace {

// ---------------------------------------------------------------- parts

// M, Z and U of a part of a row; nothing (or nothing but -Inf): zeros.
struct ScorePart {
    float top, sum, bend;
};

// h above, held where 2^-h is 0 anyway (an infinity would leave NaN; the NaN of
// two logits of +Inf comes through).
__device__ __forceinline__ float rise(float from, float to, float c)
{
    const float h = (to - from) * c;
    return h > 1e30f ? 1e30f : h;
}
__device__ __forceinline__ ScorePart moved(ScorePart p, float top, float c)
{
    if (p.sum == 0.0f) return ScorePart{top, 0.0f, 0.0f};
    const float h = rise(p.top, top, c), f = exp2_fast(-h);
    return ScorePart{top, p.sum * f, f * (p.bend + h * p.sum)};
}

// What a thread has of its row so far.
struct Tally {
    float top, sum, bend;
    template <int TYPE, int U>
    __device__ __forceinline__ void add(Piece<TYPE> (&x)[U], float c)
    {
        float high = top;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < Piece<TYPE>::N; ++i) high = fmaxf(high, x[u].get(i));
        const float base = high == -INFINITY ? 0.0f : high;
        // (top may be -Inf: the sum is 0 then)
        const float h = rise(top, base, c), f = exp2_fast(-h);
        float z[2] = {sum * f, 0.0f}, b[2] = {f * (bend + h * sum), 0.0f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u].repack();
#pragma unroll
            for (int i = 0; i < Piece<TYPE>::N; ++i) {
                const float d = (x[u].get(i) - base) * c, e = exp2_fast(d);
                z[i & 1] += e;
                b[i & 1] = __builtin_fmaf(-fmaxf(d, -1e4f), e, b[i & 1]);  // (-Inf times 0 is none)
            }
        }
        sum = z[0] + z[1];
        bend = b[0] + b[1];
        top = high;
    }
};

__device__ __forceinline__ float part_entropy(const ScorePart& p)
{
    return p.sum == 0.0f ? 0.0f : (float)(part_ln(p.sum) + (double)p.bend / (double)p.sum * 0.693147180559945309);
}

// A row's numbers but its list.
__device__ __forceinline__ void put_scores(const ScoresOut& o, uint64_t t, const ScorePart& p, bool has, float at,
                                           float scale)
{
    const Part q = {p.top, p.sum};
    if (o.logp) o.logp[t] = has ? (float)part_logp(q, at, scale) : 0.0f;
    if (o.lse) o.lse[t] = part_lse(q, scale);
    if (o.entropy) o.entropy[t] = part_entropy(p);
    if (o.norm) {
        o.norm[2 * t] = p.top;
        o.norm[2 * t + 1] = p.sum == 0.0f ? -INFINITY : (float)part_ln(p.sum);
    }
}
__device__ __forceinline__ void put_unused(const ScoresOut& o, uint64_t t)
{
    if (threadIdx.x == 0) {
        if (o.logp) o.logp[t] = 0.0f;
        if (o.lse) o.lse[t] = 0.0f;
        if (o.entropy) o.entropy[t] = 0.0f;
        if (o.norm) o.norm[2 * t] = o.norm[2 * t + 1] = 0.0f;
    }
    for (uint32_t i = threadIdx.x; i < o.top; i += blockDim.x) {
        o.top_id[t * o.top + i] = -1;
        o.top_logp[t * o.top + i] = -INFINITY;
    }
}

// ---------------------------------------------------------------- order

// A logit's place in the order of all fp32 numbers: 0 for -Inf and NaN, which
// are on no list; the same for both zeros.
__device__ __forceinline__ uint32_t place(float x)
{
    const int b = __float_as_int(x + 0.0f);
    return x > -INFINITY ? (uint32_t)(b ^ ((b >> 31) | (int)0x80000000)) : 0u;
}
__device__ __forceinline__ float placed(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
// No two tokens of a row share a key; the lower index comes first.
__device__ __forceinline__ uint64_t key_of(uint32_t place, uint32_t v) { return (uint64_t)place << 32 | (uint32_t)~v; }

constexpr uint32_t kCands = 2048;  // candidates that are put in order
constexpr uint32_t kRanked = 512;  // up to here by counting the larger ones

struct TopSpace {
    uint32_t high[1024];  // the threads' largest
    uint32_t who[1024];   // threads at or above the bound
    uint64_t key[kCands], out[kMaxTop];
    uint32_t count, threads, bound;
    uint32_t hist[256];
};

// Largest bound (about) that at least n of the threads' numbers reach, at
// least 1; by one wave.
__device__ __forceinline__ uint32_t find_bound(const uint32_t* high, uint32_t n)
{
    uint32_t v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = 64u * i + threadIdx.x < blockDim.x ? high[64 * i + threadIdx.x] : 0u;
    uint32_t t = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t more = t | 1u << bit;
        uint32_t count = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) count += (uint32_t)__popcll(__ballot(v[i] >= more));
        if (count >= n) {
            t = more;
            if (count <= n + n / 8) break;
        }
    }
    return t ? t : 1u;
}

// The n largest of s.key[0, count) in order to s.out, count <= kCands.
__device__ __forceinline__ void put_in_order(TopSpace& s, uint32_t count, uint32_t n)
{
    const uint32_t tid = threadIdx.x, step = blockDim.x;
    if (count <= kRanked) {
        for (uint32_t i = tid; i < count; i += step) {
            const uint64_t k = s.key[i];
            uint32_t rank = 0;
            for (uint32_t j = 0; j < count; ++j) rank += s.key[j] > k;
            if (rank < n) s.out[rank] = k;
        }
        __syncthreads();
        return;
    }
    uint32_t size = kRanked;
    while (size < count) size *= 2;
    for (uint32_t i = count + tid; i < size; i += step) s.key[i] = 0;
    __syncthreads();
    for (uint32_t run = 2; run <= size; run *= 2)
        for (uint32_t gap = run / 2; gap; gap /= 2) {
            for (uint32_t i = tid; i < size / 2; i += step) {
                const uint32_t a = 2 * i - (i & (gap - 1)), b = a + gap;
                const uint64_t x = s.key[a], y = s.key[b];
                if ((x < y) == ((a & run) == 0)) {
                    s.key[a] = y;
                    s.key[b] = x;
                }
            }
            __syncthreads();
        }
    for (uint32_t i = tid; i < n; i += step) s.out[i] = s.key[i];
    __syncthreads();
}

// Pieces [first, end) of a row and, with `singles`, its singles.
template <int TYPE>
struct Span {
    typedef typename Elem<TYPE>::type E;
    const E* row;
    RowCut<TYPE> r;
    uint32_t first, end;
    bool singles;
    // Calls f(key) for every token that can be on a list.
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        if (singles && threadIdx.x < r.singles) {
            const uint32_t v = r.single(threadIdx.x), p = place((float)row[v]);
            if (p) f(key_of(p, v));
        }
        for (uint32_t j = first + threadIdx.x; j < end; j += blockDim.x) {
            Piece<TYPE> x;
            x.w = load_vec<u32x4, true>(row + r.piece(j));
#pragma unroll
            for (int i = 0; i < Piece<TYPE>::N; ++i) {
                const uint32_t p = place(x.get(i));
                if (p) f(key_of(p, r.piece(j) + i));
            }
        }
    }
};

// The n-th largest key of a span that has more than n, eight bits a pass: for
// rows where too many logits reach the bound (most of them equal).
template <int TYPE>
__device__ uint64_t nth_key(TopSpace& s, const Span<TYPE>& span, uint32_t n)
{
    uint64_t prefix = 0;
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (uint32_t i = threadIdx.x; i < 256; i += blockDim.x) s.hist[i] = 0;
        __syncthreads();
        span.each([&](uint64_t k) {
            if (shift < 56 && k >> (shift + 8) != prefix) return;
            const uint32_t bin = (uint32_t)(k >> shift) & 255u;
            // (a wave whose keys share a bin adds once)
            const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane((int)bin);
            if (__ballot(bin == first) == __ballot(true)) {
                const uint64_t on = __ballot(true);
                if ((threadIdx.x & 63) == (uint32_t)__ffsll((unsigned long long)on) - 1)
                    atomicAdd(&s.hist[bin], (uint32_t)__popcll(on));
            } else {
                atomicAdd(&s.hist[bin], 1u);
            }
        });
        __syncthreads();
        if (threadIdx.x == 0) {
            int bin = 255;
            uint32_t above = 0;
            for (; bin > 0 && above + s.hist[bin] < n; --bin) above += s.hist[bin];
            s.bound = (uint32_t)bin;
            s.count = above;
        }
        __syncthreads();
        prefix = prefix << 8 | s.bound;
        n -= s.count;
        __syncthreads();
    }
    return prefix;
}

// The n most likely tokens of a span in order in s.out; returns how many there
// are (at most n).  high: the thread's largest logit, single: its single.
template <int TYPE>
__device__ uint32_t top_of(TopSpace& s, const Span<TYPE>& span, uint32_t n, float high, float single)
{
    constexpr int N = Piece<TYPE>::N;
    const uint32_t tid = threadIdx.x, step = blockDim.x;
    const uint32_t mine = place(high);
    s.high[tid] = mine;
    if (tid == 0) s.count = s.threads = 0;
    __syncthreads();
    if (tid < 64) {
        const uint32_t b = find_bound(s.high, n);
        if (tid == 0) s.bound = b;
    }
    __syncthreads();
    const uint32_t bound = s.bound;
    if (mine >= bound) s.who[atomicAdd(&s.threads, 1u)] = tid;
    auto add = [&](uint64_t k) {
        const uint32_t at = atomicAdd(&s.count, 1u);
        if (at < kCands) s.key[at] = k;
    };
    if (span.singles && tid < span.r.singles && place(single) >= bound) add(key_of(place(single), span.r.single(tid)));
    __syncthreads();
    const uint32_t threads = s.threads, rounds = (span.end - span.first + step - 1) / step;
    for (uint32_t i = tid; i < threads * rounds; i += step) {
        const uint32_t j = span.first + s.who[i % threads] + step * (i / threads);
        if (j >= span.end) continue;
        Piece<TYPE> x;
        x.w = load_vec<u32x4, true>(span.row + span.r.piece(j));
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (place(x.get(e)) >= bound) add(key_of(place(x.get(e)), span.r.piece(j) + e));
    }
    __syncthreads();
    uint32_t count = s.count;
    if (count > kCands) {
        const uint64_t least = nth_key(s, span, n);
        if (tid == 0) s.count = 0;
        __syncthreads();
        span.each([&](uint64_t k) {
            if (k >= least) add(k);
        });
        __syncthreads();
        count = s.count;
    }
    put_in_order(s, count, n);
    return min(count, n);
}

__device__ __forceinline__ void put_top(const ScoresOut& o, uint64_t t, const TopSpace& s, uint32_t found, Part p,
                                        float scale)
{
    for (uint32_t i = threadIdx.x; i < o.top; i += blockDim.x) {
        const uint64_t k = i < found ? s.out[i] : 0;
        o.top_id[t * o.top + i] = i < found ? (int32_t)~(uint32_t)k : -1;
        o.top_logp[t * o.top + i] = i < found ? (float)part_logp(p, placed((uint32_t)(k >> 32)), scale) : -INFINITY;
    }
}

// ---------------------------------------------------------------- forward

__device__ __forceinline__ bool scored(const Logits& in, uint64_t t) { return !in.label || has_token(in, t); }

// Slice s of a row: pieces [s W, (s + 1) W); slice 0 takes the singles too.
// With one slice a row its scores at once, else its part and its list.
template <int TYPE>
__global__ void __launch_bounds__(1024) k_scores(Logits in, ScoresOut o, uint32_t S, uint32_t W, float c,
                                                 ScorePart* part, uint64_t* keys)
{
    typedef typename Elem<TYPE>::type E;
    __shared__ float s_top[16], s_sum[16], s_bend[16];
    __shared__ TopSpace s_space;
    const uint32_t tid = threadIdx.x, step = blockDim.x, n = o.top;
    for (uint64_t b = blockIdx.x; b < in.rows * S; b += gridDim.x) {
        const uint64_t t = b / S;
        const uint32_t s = (uint32_t)(b % S);
        if (!scored(in, t)) {
            if (S == 1) put_unused(o, t);
            continue;
        }
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        const RowCut<TYPE> r(row, (uint32_t)in.vocab);
        const uint32_t first = (uint32_t)min((uint64_t)r.full, (uint64_t)s * W);
        const uint32_t end = (uint32_t)min((uint64_t)r.full, (uint64_t)(s + 1) * W);
        const Span<TYPE> span = {row, r, first, end, s == 0};
        const float single = s == 0 && tid < r.singles ? (float)row[r.single(tid)] : -INFINITY;
        const float at = tid == 0 && in.label ? (float)row[in.label[t]] : 0.0f;
        Tally own = {single, single == -INFINITY ? 0.0f : 1.0f, 0.0f};
        for (uint32_t j = first + tid; j < end; j += 4 * step) {
            Piece<TYPE> x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                x[u].none();
                if ((uint64_t)j + step * u < end) x[u].w = load_vec<u32x4, true>(row + r.piece(j + step * u));
            }
            own.add(x, c);
        }
        float high = join_waves<false>(own.top, s_top);
        if (high == -INFINITY) high = 0.0f;
        const ScorePart q = moved(ScorePart{own.top, own.sum, own.bend}, high, c);
        const float sum = join_waves<true>(q.sum, s_sum), bend = join_waves<true>(q.bend, s_bend);
        const ScorePart p = {high, sum, bend};
        if (tid == 0) {
            if (S > 1)
                part[b] = p;
            else
                put_scores(o, t, p, in.label != nullptr, at, in.scale);
        }
        if (n) {
            const uint32_t found = top_of(s_space, span, n, own.top, single);
            if (S > 1)
                for (uint32_t i = tid; i < n; i += step) keys[b * n + i] = i < found ? s_space.out[i] : 0;
            else
                put_top(o, t, s_space, found, Part{p.top, p.sum}, in.scale);
        }
        __syncthreads();
    }
}

// A row's slices joined (at most 64 of them, at most kCands keys together).
template <int TYPE>
__global__ void __launch_bounds__(256) k_join_scores(Logits in, ScoresOut o, uint32_t S, float c,
                                                     const ScorePart* part, const uint64_t* keys)
{
    typedef typename Elem<TYPE>::type E;
    __shared__ TopSpace s_space;
    const uint32_t tid = threadIdx.x, n = o.top;
    for (uint64_t t = blockIdx.x; t < in.rows; t += gridDim.x) {
        if (!scored(in, t)) {
            put_unused(o, t);
            continue;
        }
        // every wave joins the parts for itself, a lane a slice
        const uint32_t lane = tid & 63;
        const ScorePart mine = lane < S ? part[t * S + lane] : ScorePart{0.0f, 0.0f, 0.0f};
        float top = wave_join<false>(mine.sum == 0.0f ? -INFINITY : mine.top);
        if (top == -INFINITY) top = 0.0f;
        const ScorePart q = moved(mine, top, c);
        const ScorePart p = {top, wave_join<true>(q.sum), wave_join<true>(q.bend)};
        if (tid == 0) {
            const float at = in.label ? (float)(static_cast<const E*>(in.x) + t * in.ld)[in.label[t]] : 0.0f;
            put_scores(o, t, p, in.label != nullptr, at, in.scale);
            s_space.count = 0;
        }
        if (n) {
            __syncthreads();
            for (uint32_t i = tid; i < S * n; i += 256) {
                const uint64_t k = keys[t * S * n + i];
                if (k) s_space.key[atomicAdd(&s_space.count, 1u)] = k;
            }
            __syncthreads();
            const uint32_t count = s_space.count;
            put_in_order(s_space, count, n);
            put_top(o, t, s_space, min(count, n), Part{p.top, p.sum}, in.scale);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- gradient

constexpr int kScoreU = 2;

// The gradient of slice s of a row, W pieces: with p_v = 2^(d_v - log2 Z) the
// softmax, s p_v (on - entropy' (ln p_v + H)) everywhere, and in the places of
// the row's token and of its list their own derivatives beside it, stored once
// more behind the slice's other entries.
template <int TYPE, bool ENTROPY>
__global__ void __launch_bounds__(256) k_scores_grad(Logits in, ScoresGrad a, uint32_t S, uint32_t W, void* dlogits,
                                                     uint64_t ldd)
{
    typedef typename Elem<TYPE>::type E;
    constexpr int N = Piece<TYPE>::N, U = kScoreU;
    __shared__ double s_w[4][4];
    __shared__ uint32_t s_id[kMaxTop + 1], s_n[5];
    __shared__ float s_x[kMaxTop + 1], s_g[kMaxTop + 1];
    const uint32_t tid = threadIdx.x, V = (uint32_t)in.vocab;
    const float c = in.scale * kLog2e;
    for (uint64_t b = blockIdx.x; b < in.rows * S; b += gridDim.x) {
        const uint64_t t = b / S;
        const uint32_t s = (uint32_t)(b % S);
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        E* out = static_cast<E*>(dlogits) + t * ldd;
        const RowCut<TYPE> r(row, V);
        const uint32_t first = (uint32_t)min((uint64_t)r.full, (uint64_t)s * W);
        const uint32_t end = (uint32_t)min((uint64_t)r.full, (uint64_t)(s + 1) * W);
        const uint32_t label = in.label ? (uint32_t)in.label[t] : 0xFFFFFFFFu;
        const bool use = scored(in, t) && a.norm[2 * t + 1] > -INFINITY;
        // the token and the list, an entry a thread
        const float d_logp = a.d_logp && in.label ? a.d_logp[t] : 0.0f;
        const float d_lse = a.d_lse ? a.d_lse[t] : 0.0f, d_h = ENTROPY ? a.d_entropy[t] : 0.0f;
        uint32_t id = 0xFFFFFFFFu;
        float g = 0.0f, x = -INFINITY;
        if (a.d_top && tid < a.top) {
            id = (uint32_t)a.top_id[t * a.top + tid];
            g = a.d_top[t * a.top + tid];
        }
        float at = -INFINITY;
        bool any = false;
        if (use) {
            if (id < V) x = (float)row[id];
            if (x == -INFINITY) g = 0.0f;
            if (label < V) at = (float)row[label];
        }
        const float one = at == -INFINITY ? 0.0f : d_logp;
        double total[1] = {(double)g};
        if (a.d_top) block_sum(total, s_w, 1);
        any = use && (one != 0.0f || d_lse != 0.0f || d_h != 0.0f || __syncthreads_or(g != 0.0f));
        if (!any) {
            const u32x4 zero = {0u, 0u, 0u, 0u};
            for (uint32_t j = first + tid; j < end; j += 256) store_vec(out + r.piece(j), zero);
            if (s == 0 && tid < r.singles) out[r.single(tid)] = (E)0.0f;
            __syncthreads();
            continue;
        }
        const float top = a.norm[2 * t], l2 = a.norm[2 * t + 1] * kLog2e;
        const float on = in.scale * (float)((double)d_lse - (double)one - total[0]);
        const float A = ENTROPY ? on - in.scale * d_h * a.entropy[t] : on;
        const float B = ENTROPY ? -in.scale * d_h * 0.693147180559945309f : 0.0f;
        auto entry_of = [&](float v) {
            const float d = (v - top) * c - l2, e = exp2_fast(d);
            return ENTROPY ? e * (A + B * fmaxf(d, -1e4f)) : e * A;
        };
        const float single = s == 0 && tid < r.singles ? (float)row[r.single(tid)] : -INFINITY;
        __syncthreads();
        for (uint32_t j = first + tid; j < end; j += 256 * U) {
            Piece<TYPE> y[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                y[u].none();
                if ((uint64_t)j + 256 * u < end) y[u].w = load_vec<u32x4>(row + r.piece(j + 256 * u));
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float e[N];
#pragma unroll
                for (int i = 0; i < N; ++i) e[i] = entry_of(y[u].get(i));
                y[u].put(e);
                if ((uint64_t)j + 256 * u < end) store_vec(out + r.piece(j + 256 * u), y[u].w);
            }
        }
        if (s == 0 && tid < r.singles) out[r.single(tid)] = (E)entry_of(single);
        // what lies in this slice of the list, in its order, and the token
        auto inside = [&](uint32_t v, float x) {
            if (v >= V || x == -INFINITY) return false;
            if (!r.in_piece(v)) return s == 0;
            const uint32_t j = (v - r.head) / N;
            return j >= first && j < end;
        };
        const bool mine = inside(id, x);
        const uint64_t mask = __ballot(mine);
        if ((tid & 63) == 0) s_n[tid >> 6] = (uint32_t)__popcll(mask);
        // (every store before this is done before the next ones begin)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        uint32_t before = 0, count = 0;
        for (uint32_t w = 0; w < 4; ++w) {
            if (w < tid >> 6) before += s_n[w];
            count += s_n[w];
        }
        if (mine) {
            const uint32_t i = before + (uint32_t)__popcll(mask & ((1ull << (tid & 63)) - 1));
            s_id[i] = id;
            s_x[i] = x;
            s_g[i] = g;
        }
        const bool token = inside(label, at);
        if (token && tid == 0) {
            s_id[count] = label;
            s_x[count] = at;
            s_g[count] = one;
        }
        count += token;
        __syncthreads();
        for (uint32_t i = tid; i < count; i += 256) {
            // (a token that is there twice: its first entry takes all of them)
            float more = 0.0f;
            bool lead = true;
            for (uint32_t k = 0; k < count; ++k)
                if (s_id[k] == s_id[i]) {
                    more += s_g[k];
                    lead &= k >= i;
                }
            if (lead) out[s_id[i]] = (E)(entry_of(s_x[i]) + in.scale * more);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- host

constexpr uint32_t kScoreGrid = 1u << 21;  // (of up to 1024 threads each)
constexpr uint64_t kScoreSlices = 1024;  // of few rows together

struct ScoreCut {
    uint32_t S, W, threads;
};
// Slices of a row at most: 64, and their lists together are put in order.
uint64_t most_score_slices(uint64_t pieces, uint32_t top)
{
    return std::min<uint64_t>(std::min<uint64_t>(64, (pieces + 511) / 512), top ? kCands / top : 64);
}
ScoreCut cut_scores(uint64_t rows, uint64_t vocab, uint32_t type, uint32_t top)
{
    ScoreCut r;
    const uint64_t pieces = vocab / (type == kF32 ? 4 : 8) + 1;
    const uint64_t want = kScoreSlices / std::min(rows, kScoreSlices);
    const uint64_t S = std::max<uint64_t>(1, std::min(most_score_slices(pieces, top), want));
    r.W = (uint32_t)((pieces + S - 1) / S);
    r.S = (uint32_t)((pieces + r.W - 1) / r.W);
    const uint64_t threads = std::max<uint64_t>((r.W + 255) / 256 * 64, 2 * top);
    r.threads = threads <= 128 ? 128 : threads <= 256 ? 256 : threads <= 512 ? 512 : 1024;
    return r;
}

struct ScoreSpace {
    ScorePart* part;
    uint64_t* keys;
};
ScoreSpace carve_scores(void* ws, uint64_t parts, uint32_t top, size_t* bytes)
{
    Carve c(ws);
    ScoreSpace r;
    r.part = c.take<ScorePart>(parts);
    r.keys = c.take<uint64_t>(parts * top);
    if (bytes) *bytes = c.used;
    return r;
}

}  // namespace

// (Enough for every type and for every call of fewer rows, a smaller
// vocabulary or shorter lists: parts are counted by what bounds them.)
size_t scores_workspace(uint32_t top, uint64_t rows, uint64_t vocab)
{
    const uint64_t pieces = vocab / 4 + 1;
    size_t b = 0;
    Carve c(nullptr);
    const uint64_t parts = std::min(kScoreSlices, rows * std::min<uint64_t>(64, (pieces + 511) / 512));
    c.take<ScorePart>(parts);
    c.take<uint64_t>(parts * top);
    b = c.used;
    return b;
}

hipError_t scores_run(const Logits& in, const ScoresOut& o, void* ws, hipStream_t s)
{
    const ScoreCut cut = cut_scores(in.rows, in.vocab, in.type, o.top);
    const ScoreSpace sp = carve_scores(ws, cut.S > 1 ? in.rows * cut.S : 0, o.top, nullptr);
    const float c = in.scale * kLog2e;
    const uint32_t grid = (uint32_t)std::min<uint64_t>(in.rows * cut.S, kScoreGrid);
    timer_begin(kTScores, s);
    by_type(in.type, [&](auto ty) {
        constexpr int TY = decltype(ty)::value;
        hipLaunchKernelGGL((k_scores<TY>), dim3(grid), dim3(cut.threads), 0, s, in, o, cut.S, cut.W, c, sp.part, sp.keys);
        if (cut.S > 1)
            hipLaunchKernelGGL((k_join_scores<TY>), dim3((uint32_t)std::min<uint64_t>(in.rows, kScoreGrid)), dim3(256), 0,
                               s, in, o, cut.S, c, sp.part, sp.keys);
    });
    timer_end(kTScores, s);
    return hipGetLastError();
}

hipError_t scores_grad_run(const Logits& in, const ScoresGrad& a, void* dlogits, uint64_t ldd, hipStream_t s)
{
    const uint64_t pieces = in.vocab / (in.type == kF32 ? 4 : 8) + 1;
    // (in place, a row's token and list are read before any of it is written:
    // one workgroup a row)
    const bool whole = dlogits == in.x && (a.d_logp || a.d_top);
    const uint32_t W = whole ? (uint32_t)pieces : 256 * kScoreU, S = (uint32_t)((pieces + W - 1) / W);
    const uint32_t grid = (uint32_t)std::min<uint64_t>(in.rows * S, kScoreGrid);
    timer_begin(kTScoresGrad, s);
    by_type(in.type, [&](auto ty) {
        constexpr int TY = decltype(ty)::value;
        if (a.d_entropy)
            hipLaunchKernelGGL((k_scores_grad<TY, true>), dim3(grid), dim3(256), 0, s, in, a, S, W, dlogits, ldd);
        else
            hipLaunchKernelGGL((k_scores_grad<TY, false>), dim3(grid), dim3(256), 0, s, in, a, S, W, dlogits, ldd);
    });
    timer_end(kTScoresGrad, s);
    return hipGetLastError();
}

}  // namespace sparcml
