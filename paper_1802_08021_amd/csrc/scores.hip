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
// The n most likely tokens of a row: every thread of a workgroup keeps the
// largest logit of each of four groups of its pieces, and the n-th largest of
// all groups' is a bound that at least n logits reach and few more do (of 2048
// groups about 65 for n = 64).  Groups below it need no second look; those of
// the others are looked through once more, and what reaches the bound is put in
// order.
#include "rows_device.h"

#include <algorithm>

namespace sparcml {
namespace {

// ---------------------------------------------------------------- parts

// M, Z and U of a part of a row; nothing (or nothing but -Inf): M is -Inf or 0,
// Z and U are 0.
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

// What a thread has of its row so far: its largest logit, and sums of 2^d and
// -d 2^d with d = c x - ref, one fused multiply-add.  ref is a whole number
// (so that sums move from one to the other exactly) that follows the largest c
// x only where it is left more than four powers of two behind.  Logits so large
// that c x has no place for d (kFar) leave sums of no use: whoever finds one
// largest in a row sums that row again, taking differences first.  Logits so
// small are 0 beside all others.
constexpr float kFar = 1048576.0f;
// The largest of three, NaN aside (the compiler would quiet NaN before each of
// its own: twice the instructions).
__device__ __forceinline__ float largest(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
struct Tally {
    float top = -INFINITY, ref = -INFINITY, r = 0.0f, sum = 0.0f, bend = 0.0f;
    // (r: ref, 0 while there is none)
    __device__ __forceinline__ void follow(float most, float c)
    {
        top = largest(top, most, most);
        const float y = most * c;
        const bool behind = y > ref + 4.0f && y > -kFar;
        if (__ballot(behind)) {
            if (behind) {
                const float to = rintf(y), h = fminf(to - ref, 1e30f), f = exp2_fast(-h);
                bend = f * (bend + h * sum);
                sum *= f;
                ref = r = to;
            }
        }
    }
    // Adds K pieces; their largest logit.
    template <int TYPE, int K>
    __device__ __forceinline__ float add(Piece<TYPE>* x, float* most, float c)
    {
        constexpr int N = Piece<TYPE>::N;
        float high = -INFINITY;
#pragma unroll
        for (int u = 0; u < K; ++u) {
            most[u] = largest(x[u].get(0), x[u].get(1), x[u].get(2));
#pragma unroll
            for (int i = 3; i + 1 < N; i += 2) most[u] = largest(most[u], x[u].get(i), x[u].get(i + 1));
            most[u] = largest(most[u], x[u].get(N - 1), x[u].get(N - 1));
        }
#pragma unroll
        for (int u = 0; u < K; u += 2) high = largest(high, most[u], most[u + 1]);
        follow(high, c);
        float z[2] = {sum, 0.0f}, b[2] = {bend, 0.0f};
#pragma unroll
        for (int u = 0; u < K; ++u) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float d = __builtin_fmaf(x[u].get(i), c, -r), e = exp2_fast(d);
                z[i & 1] += e;
                b[i & 1] = __builtin_fmaf(-fmaxf(d, -1e4f), e, b[i & 1]);  // (-Inf times 0 is none)
            }
        }
        sum = z[0] + z[1];
        bend = b[0] + b[1];
        return high;
    }
    __device__ __forceinline__ void add_one(float x, float c)
    {
        follow(x, c);
        const float d = __builtin_fmaf(x, c, -r), e = exp2_fast(d);
        sum += e;
        bend = __builtin_fmaf(-fmaxf(d, -1e4f), e, bend);
    }
    // The wave's part, in every lane: against its largest logit again.
    __device__ __forceinline__ ScorePart join_lanes(float c) const
    {
        const float high = wave_join<false>(top), to = wave_join<false>(ref);
        const float h = fminf(to - ref, 1e30f), f = ref == -INFINITY ? 0.0f : exp2_fast(-h);
        const float z = wave_join<true>(sum == 0.0f ? 0.0f : f * sum);
        const float b = wave_join<true>(sum == 0.0f ? 0.0f : f * (bend + h * sum));
        if (z == 0.0f) return ScorePart{high, 0.0f, 0.0f};
        const float off = __builtin_fmaf(-c, high, to), g = exp2_fast(off);
        return ScorePart{high, z * g, g * __builtin_fmaf(-off, z, b)};
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

constexpr int kScoreU = 4;       // pieces of a thread where a row is one turn,
constexpr uint32_t kGroups = 4;  // groups of them: a piece each; else
constexpr uint32_t kSubs = 16;   // smaller ones that are looked through again
static_assert(kScoreU == kGroups, "a piece a group");

// What a workgroup puts a row together in.
template <int THREADS, bool ONE>
struct TopSpace {
    static constexpr uint32_t kWaves = THREADS / 64, kCands = THREADS < 256 ? 512 : 1024;
    static constexpr uint32_t kHeld = ONE ? 1 : kSubs;  // numbers a thread keeps here
    struct Wave {
        float top, sum, bend;
        uint32_t there, low, high;  // of its groups: how many hold a logit, ~least, largest
    } wave[kWaves];
    uint32_t reach[3][3];  // (a step's, the next one's, the one's behind it)
    uint32_t count, groups, bound, above;
    union {
        uint32_t high[kHeld * THREADS];  // the groups' largest (read before there are candidates)
        uint64_t key[kCands];            // candidates
    };
    union {
        uint16_t who[kCands];  // groups at or above the bound
        struct {
            uint64_t out[kMaxTop];
            uint32_t hist[256];
        };
    };
};

// The waves' parts joined (nothing: M is -Inf); M in every thread, the sums in
// the first `lanes`.
template <int WAVES, class W>
__device__ __forceinline__ ScorePart join_parts(const W* wave, float c, uint32_t lanes)
{
    ScorePart p = {-INFINITY, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) p.top = fmaxf(p.top, wave[w].top);
    if (threadIdx.x >= ((lanes + 63) & ~63u)) return p;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const ScorePart q = moved(ScorePart{wave[w].top, wave[w].sum, wave[w].bend}, p.top, c);
        p.sum += q.sum;
        p.bend += q.bend;
    }
    return p;
}

template <class Space>
__device__ __forceinline__ void clear_counts(Space& s)
{
    if (threadIdx.x < 9) s.reach[threadIdx.x / 3][threadIdx.x % 3] = 0;
    if (threadIdx.x == 9) s.count = s.groups = 0;
}

// What each wave has of its row, by its first lane.
template <class Space>
__device__ __forceinline__ void put_wave(Space& s, const ScorePart& q, const uint32_t (&v)[kGroups])
{
    uint32_t there = 0, low = 0, high = 0;
#pragma unroll
    for (uint32_t i = 0; i < kGroups; ++i) {
        there += (uint32_t)__popcll(__ballot(v[i] != 0));
        low = max(low, v[i] ? ~v[i] : 0u);
        high = max(high, v[i]);
    }
    low = wave_max(low);
    high = wave_max(high);
    if ((threadIdx.x & 63) == 0) s.wave[threadIdx.x >> 6] = {q.top, q.sum, q.bend, there, low, high};
}

// A bound that at least n of the threads' numbers v reach (1 if fewer are not
// 0) and few more do: two bits a step from the first in which they differ.
template <class Space>
__device__ __forceinline__ uint32_t find_bound(Space& s, const uint32_t (&v)[kGroups], uint32_t n)
{
    constexpr uint32_t kWaves = Space::kWaves;
    uint32_t there = 0, low = 0, high = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) {
        there += s.wave[w].there;
        low = max(low, s.wave[w].low);
        high = max(high, s.wave[w].high);
    }
    if (there < n) return 1;
    low = (uint32_t)__builtin_amdgcn_readfirstlane((int)~low);
    high = (uint32_t)__builtin_amdgcn_readfirstlane((int)high);
    if (low == high) return low;
    int bit = 31 - __clz((int)(low ^ high));
    uint32_t t = high & ~((2u << bit) - 1);
    for (uint32_t turn = 0; bit >= 0; bit -= 2, turn = turn == 2 ? 0 : turn + 1) {
        const uint32_t shift = bit > 0 ? bit - 1 : 0, steps = bit > 0 ? 3 : 1;
        uint32_t reach[3] = {0, 0, 0};
#pragma unroll
        for (uint32_t k = 0; k < 3; ++k) {
            if (k >= steps) break;
#pragma unroll
            for (uint32_t i = 0; i < kGroups; ++i) reach[k] += (uint32_t)__popcll(__ballot(v[i] >= t + ((k + 1) << shift)));
        }
        if (kWaves > 1) {
            const uint32_t lane = threadIdx.x & 63;
            if (lane < 3) atomicAdd(&s.reach[turn][lane], lane == 0 ? reach[0] : lane == 1 ? reach[1] : reach[2]);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 3; ++k) reach[k] = (uint32_t)__builtin_amdgcn_readfirstlane((int)s.reach[turn][k]);
            // (read by all before the barrier above, added to behind the next)
            if (threadIdx.x < 3) s.reach[turn == 0 ? 2 : turn - 1][threadIdx.x] = 0;
        }
        const uint32_t best = reach[2] >= n ? 3 : reach[1] >= n ? 2 : reach[0] >= n ? 1 : 0;
        t += best << shift;
        if (best && reach[best - 1] <= n + n / 8 + 2) break;
    }
    return t ? t : 1u;
}

// The n largest of s.key[0, count) in order to s.out, count <= kCands: up to 128
// by counting the larger ones, beyond by waves that put 64 at a time in order
// and look up how many of each other 64 are larger.
template <class Space>
__device__ __forceinline__ void put_in_order(Space& s, uint32_t count, uint32_t n)
{
    constexpr uint32_t kWaves = Space::kWaves, kMost = Space::kCands / 64 / kWaves;
    const uint32_t tid = threadIdx.x;
    if (count <= 128) {
        for (uint32_t i = tid; i < count; i += 64 * kWaves) {
            const uint64_t k = s.key[i];
            uint32_t rank = 0, j = 0;
            for (; j + 8 <= count; j += 8)
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) rank += s.key[j + e] > k;
            for (; j < count; ++j) rank += s.key[j] > k;
            if (rank < n) s.out[rank] = k;
        }
        __syncthreads();
        return;
    }
    const uint32_t lane = tid & 63, wave = tid >> 6, blocks = (count + 63) / 64;
    for (uint32_t b = wave; b < blocks; b += kWaves) {
        uint64_t k = 64 * b + lane < count ? s.key[64 * b + lane] : 0;
        for (uint32_t run = 2; run <= 64; run *= 2)
            for (uint32_t gap = run / 2; gap; gap /= 2) {
                const uint64_t o = __shfl_xor((unsigned long long)k, (int)gap);
                const bool larger = ((lane & run) == 0) == ((lane & gap) == 0);  // who keeps the larger one
                k = (o > k) == larger ? o : k;
            }
        s.key[64 * b + lane] = k;
    }
    __syncthreads();
    for (uint32_t b = wave; b < blocks; b += kWaves) {
        const uint64_t k = s.key[64 * b + lane];
        uint32_t rank = lane;
        if (lane >= n) continue;  // (its own 64 hold n larger ones)
        for (uint32_t w = 0; w < blocks; ++w) {
            if (w == b) continue;
            const uint64_t* list = s.key + 64 * w;
            uint32_t at = 0;  // of the list, how many are larger
#pragma unroll
            for (uint32_t half = 32; half; half /= 2)
                if (list[at + half - 1] > k) at += half;
            rank += at + (at == 63 && list[63] > k);
        }
        if (k && rank < n) s.out[rank] = k;
    }
    __syncthreads();
}

// Piece u of a thread's K in a turn over a long row.  (Side by side, what is
// looked through again would lie in half the lines or a quarter, but the first
// pass is slower: 2048 x 131072 fp32 298 us against 156.)
template <int K, int THREADS>
__device__ __forceinline__ uint64_t long_piece(uint64_t turn, uint32_t u, uint32_t tid)
{
    return (turn * K + u) * THREADS + tid;
}

// Pieces [first, end) of a row and, with `singles`, its singles.
template <int TYPE>
struct Span {
    typedef typename Elem<TYPE>::type E;
    const E* row;
    RowCut<TYPE> r;
    uint32_t first, end;
    bool singles;
    // Calls f(logit, token) for every token.
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        if (singles && threadIdx.x < r.singles) f((float)row[r.single(threadIdx.x)], r.single(threadIdx.x));
        for (uint64_t j = first + threadIdx.x; j < end; j += blockDim.x) {
            Piece<TYPE> x;
            x.w = load_vec<u32x4, true>(row + r.piece((uint32_t)j));
#pragma unroll
            for (int i = 0; i < Piece<TYPE>::N; ++i) f(x.get(i), r.piece((uint32_t)j) + i);
        }
    }
};

// A span's part once more, its largest logit known and so large that the
// difference has to be taken first.
template <int TYPE, int THREADS>
__device__ __attribute__((noinline)) ScorePart far_part(Span<TYPE> span, float top, float c, float (*s_far)[THREADS / 64])
{
    float z = 0.0f, b = 0.0f;
    span.each([&](float x, uint32_t) {
        const float d = (x - top) * c, e = exp2_fast(d);
        z += e;
        b = __builtin_fmaf(-fmaxf(d, -1e4f), e, b);
    });
    z = wave_join<true>(z);
    b = wave_join<true>(b);
    if ((threadIdx.x & 63) == 0) {
        s_far[0][threadIdx.x >> 6] = z;
        s_far[1][threadIdx.x >> 6] = b;
    }
    __syncthreads();
    z = b = 0.0f;
    for (int w = 0; w < THREADS / 64; ++w) {
        z += s_far[0][w];
        b += s_far[1][w];
    }
    __syncthreads();
    return ScorePart{top, z, b};
}

// The n largest of more than n keys, that each(f) calls f with, to s.key, eight
// bits a pass: for rows where too many logits reach the bound (most of them
// equal).
template <class Space, class Each>
__device__ void narrow(Space& s, uint32_t n, Each each)
{
    const uint32_t all = n;
    uint64_t prefix = 0;
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (uint32_t i = threadIdx.x; i < 256; i += 64 * Space::kWaves) s.hist[i] = 0;
        __syncthreads();
        each([&](uint64_t k) {
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
            s.above = above;
        }
        __syncthreads();
        prefix = prefix << 8 | s.bound;
        n -= s.above;
        __syncthreads();
    }
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
    each([&](uint64_t k) {
        if (k >= prefix) s.key[min(atomicAdd(&s.count, 1u), all - 1)] = k;  // (no two are the same)
    });
    __syncthreads();
}

// The n most likely tokens of a span in order in s.out; returns how many there
// are (at most n).  v: the thread's groups' largest.  ONE: its pieces are
// groups, and still in x; else s.high has those of kSubs smaller groups, of
// `per` turns of K pieces.  single: the thread's single.  (After put_wave and a
// barrier.)
template <int TYPE, int THREADS, bool ONE>
__device__ __forceinline__ uint32_t top_of(TopSpace<THREADS, ONE>& s, const Span<TYPE>& span, uint32_t n, uint32_t per,
                                           Piece<TYPE> (&x)[kScoreU], const uint32_t (&v)[kGroups], float single)
{
    constexpr int N = Piece<TYPE>::N, K = 16 / N;
    constexpr uint32_t kCands = TopSpace<THREADS, ONE>::kCands;
    const uint32_t tid = threadIdx.x;
    const uint32_t bound = find_bound(s, v, n);
    const float least = bound > place(-3.402823466e38f) ? placed(bound) : -3.402823466e38f;
    auto add = [&](uint32_t at, float y, uint32_t j) {
        if (at < kCands) s.key[at] = key_of(place(y), j);
    };
    if (ONE) {
        if (span.singles && single >= least) add(atomicAdd(&s.count, 1u), single, span.r.single(tid));
        // counted first, so that a wave asks for its places once
        uint32_t mine = 0;
        const bool some = max(max(v[0], v[1]), max(v[2], v[3])) >= bound;
        if (__ballot(some)) {
            // (unpacked again each time: nothing is kept from the sums to here)
            if (some)
#pragma unroll
                for (int u = 0; u < kScoreU; ++u) {
                    x[u].repack();
#pragma unroll
                    for (int e = 0; e < N; ++e) mine += x[u].get(e) >= least;
                }
            const uint32_t upto = wave_scan(mine);
            uint32_t at = 0;
            if ((tid & 63) == 63) at = atomicAdd(&s.count, upto);
            at = (uint32_t)__builtin_amdgcn_readlane((int)at, 63) + upto - mine;
            if (some)
#pragma unroll
                for (int u = 0; u < kScoreU; ++u) {
                    x[u].repack();
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (x[u].get(e) >= least) add(at++, x[u].get(e), span.r.piece(span.first + tid + THREADS * u) + e);
                }
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < kGroups; ++i)
            if (v[i] >= bound)
                for (uint32_t q = i * (kSubs / kGroups); q < (i + 1) * (kSubs / kGroups); ++q)
                    if (s.high[q * THREADS + tid] >= bound) {
                        const uint32_t at = atomicAdd(&s.groups, 1u);
                        if (at < kCands) s.who[at] = (uint16_t)(q * THREADS + tid);
                    }
        __syncthreads();
        if (span.singles && single >= least) add(atomicAdd(&s.count, 1u), single, span.r.single(tid));
        // a lane a group, and the lanes that are left over at its further pieces
        // (each group has a candidate: too many groups are too many of these)
        const uint32_t groups = s.groups, wide = groups <= 1 ? 0 : 32 - __clz((int)(groups - 1));
        const uint32_t lanes = min(1u << wide, (uint32_t)THREADS), apart = THREADS / lanes;
        if (groups > kCands && tid == 0) s.count = kCands + 1;
        for (uint32_t g = tid & (lanes - 1); g < groups && groups <= kCands; g += lanes) {
            const uint32_t w = s.who[g], at = w % THREADS;
            for (uint32_t nth = tid / lanes; nth < per * K; nth += apart) {
                const uint64_t j = span.first + long_piece<K, THREADS>((uint64_t)(w / THREADS) * per + nth / K, nth % K, at);
                if (j >= span.end) break;
                Piece<TYPE> y;
                y.w = load_vec<u32x4, true>(span.row + span.r.piece((uint32_t)j));
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (y.get(e) >= least) add(atomicAdd(&s.count, 1u), y.get(e), span.r.piece((uint32_t)j) + e);
            }
        }
    }
    __syncthreads();
    if (s.count > kCands)
        narrow(s, n, [&](auto f) {
            span.each([&](float y, uint32_t token) {
                if (place(y)) f(key_of(place(y), token));
            });
        });
    const uint32_t count = s.count;
    put_in_order(s, count, n);
    return min(count, n);
}

template <class Space>
__device__ __forceinline__ void put_top(const ScoresOut& o, uint64_t t, const Space& s, uint32_t found,
                                        Part p, float scale)
{
    for (uint32_t i = threadIdx.x; i < o.top; i += 64 * Space::kWaves) {
        const uint64_t k = i < found ? s.out[i] : 0;
        o.top_id[t * o.top + i] = i < found ? (int32_t)~(uint32_t)k : -1;
        o.top_logp[t * o.top + i] = i < found ? (float)part_logp(p, placed((uint32_t)(k >> 32)), scale) : -INFINITY;
    }
}

// ---------------------------------------------------------------- forward

__device__ __forceinline__ bool scored(const Logits& in, uint64_t t) { return !in.label || has_token(in, t); }

// Slice s of a row: pieces [s W, (s + 1) W); slice 0 takes the singles too.
// With one slice a row its scores at once, else its part and its list.  ONE: a
// slice is a turn, kScoreU pieces a thread.
template <int TYPE, int THREADS, bool LIST, bool ONE>
__global__ void __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(LIST ? 5 : 6)))
k_scores(Logits in, ScoresOut o, uint32_t S, uint32_t W, float c, ScorePart* part, uint64_t* keys)
{
    typedef typename Elem<TYPE>::type E;
    constexpr int K = 16 / Piece<TYPE>::N;
    __shared__ TopSpace<LIST ? THREADS : 64, ONE || !LIST> s_list;
    __shared__ typename TopSpace<THREADS, ONE>::Wave s_wave[LIST ? 1 : THREADS / 64];
    __shared__ float s_far[2][THREADS / 64];
    const uint32_t tid = threadIdx.x, n = o.top;
    for (uint64_t b = blockIdx.x; b < in.rows * S; b += gridDim.x) {
        const uint64_t t = b / S;
        const uint32_t s = (uint32_t)(b % S);
        if (!scored(in, t)) {
            if (S == 1) put_unused(o, t);
            continue;
        }
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        // (one wave has no lane for each single beside a line)
        const RowCut<TYPE> r = THREADS == 64 ? RowCut<TYPE>((uint32_t)in.vocab) : RowCut<TYPE>(row, (uint32_t)in.vocab);
        const uint32_t first = (uint32_t)min((uint64_t)r.full, (uint64_t)s * W);
        const uint32_t end = (uint32_t)min((uint64_t)r.full, (uint64_t)(s + 1) * W);
        auto fetch = [&](Piece<TYPE>& x, uint64_t j) {
            x.none();
            if (j < end) x.w = load_vec<u32x4>(row + r.piece((uint32_t)j));
        };
        const float single = s == 0 && tid < r.singles ? (float)row[r.single(tid)] : -INFINITY;
        const float at = tid == 0 && in.label ? (float)row[in.label[t]] : 0.0f;
        Piece<TYPE> x[kScoreU];
        float most[kScoreU];
        uint32_t v[kGroups] = {0, 0, 0, 0}, per = 0;
        Tally own;
        if constexpr (ONE) {
#pragma unroll
            for (int u = 0; u < kScoreU; ++u) fetch(x[u], (uint64_t)first + tid + THREADS * u);
            own.add_one(single, c);
#pragma unroll
            for (int u = 0; u < kScoreU; u += K) own.add<TYPE, K>(x + u, most + u, c);
            if (LIST)
#pragma unroll
                for (int u = 0; u < kScoreU; ++u) v[u] = place(most[u]);
        } else {
            // K pieces at a time, the next ones under way (loads past the end
            // read the last piece, and count for nothing)
            const uint32_t count = end - first, turns = (count + K * THREADS - 1) / (K * THREADS);
            const uint32_t below = tid & ~63u;  // a wave has mine of the turns
            const uint32_t mine = count > below ? (count - below + K * THREADS - 1) / (K * THREADS) : 0u;
            per = (turns + kSubs - 1) / kSubs;
            const uint8_t* from = reinterpret_cast<const uint8_t*>(row + r.piece(first));
            const uint32_t last = count ? (count - 1) * 16 : 0;
            Piece<TYPE> y[K];
            auto ask = [&](Piece<TYPE>(&q)[K], uint32_t turn) {
#pragma unroll
                for (int u = 0; u < K; ++u)
                    q[u].w = load_vec<u32x4>(reinterpret_cast<const E*>(
                        from + min((uint32_t)long_piece<K, THREADS>(turn, u, tid) * 16, last)));
            };
            float group = -INFINITY;
            uint32_t left = per, sub = 0;
            if (LIST)
#pragma unroll
                for (uint32_t q = 0; q < kSubs; ++q) s_list.high[q * THREADS + tid] = 0;  // (its own places: no barrier)
            auto take = [&](Piece<TYPE>(&q)[K], uint32_t turn) {
                if (turn + 1 == mine)
#pragma unroll
                    for (int u = 0; u < K; ++u)
                        if (long_piece<K, THREADS>(turn, u, tid) >= count) q[u].none();
                const float high = own.add<TYPE, K>(q, most, c);
                if (LIST) {
                    group = largest(group, high, high);
                    if (--left == 0 || turn + 1 == mine) {
                        s_list.high[sub * THREADS + tid] = place(group);
                        group = -INFINITY;
                        left = per;
                        ++sub;
                    }
                }
            };
            Piece<TYPE>(&z)[K] = reinterpret_cast<Piece<TYPE>(&)[K]>(x);
            if (mine) ask(z, 0);
            own.add_one(single, c);
            for (uint32_t turn = 0; turn < mine; turn += 2) {
                if (turn + 1 < mine) ask(y, turn + 1);
                take(z, turn);
                if (turn + 1 >= mine) break;
                if (turn + 2 < mine) ask(z, turn + 2);
                take(y, turn + 1);
            }
            if (LIST)
#pragma unroll
                for (uint32_t q = 0; q < kSubs; ++q)
                    v[q / (kSubs / kGroups)] = max(v[q / (kSubs / kGroups)], s_list.high[q * THREADS + tid]);
        }
        const Span<TYPE> span = {row, r, first, end, s == 0};
        ScorePart p = own.join_lanes(c);
        if constexpr (LIST) {
            put_wave(s_list, p, v);
            clear_counts(s_list);
            __syncthreads();
            p = join_parts<THREADS / 64>(s_list.wave, c, max(n, 1u));
        } else {
            if ((tid & 63) == 0) s_wave[tid >> 6] = {p.top, p.sum, p.bend, 0, 0, 0};
            __syncthreads();
            p = join_parts<THREADS / 64>(s_wave, c, 1u);
        }
        if (p.top != -INFINITY && !(fabsf(p.top * c) < kFar)) {
            __syncthreads();  // (s_far lies apart, but the waves' parts are read above)
            p = far_part<TYPE, THREADS>(span, p.top, c, s_far);
        }
        if (p.top == -INFINITY) p.top = 0.0f;
        if (tid == 0) {
            if (S > 1)
                part[b] = p;
            else
                put_scores(o, t, p, in.label != nullptr, at, in.scale);
        }
        if constexpr (LIST) {
            const uint32_t found = top_of<TYPE, THREADS, ONE>(s_list, span, n, per, x, v, single);
            if (S > 1)
                for (uint32_t i = tid; i < n; i += THREADS) keys[b * n + i] = i < found ? s_list.out[i] : 0;
            else
                put_top(o, t, s_list, found, Part{p.top, p.sum}, in.scale);
        }
        __syncthreads();
    }
}

// A row's slices joined (at most 64 of them).
template <int TYPE>
__global__ void __launch_bounds__(256) k_join_scores(Logits in, ScoresOut o, uint32_t S, float c,
                                                     const ScorePart* part, const uint64_t* keys)
{
    typedef typename Elem<TYPE>::type E;
    __shared__ TopSpace<256, true> s_space;
    const uint32_t tid = threadIdx.x, n = o.top;
    for (uint64_t t = blockIdx.x; t < in.rows; t += gridDim.x) {
        if (!scored(in, t)) {
            put_unused(o, t);
            continue;
        }
        // a lane of the first wave a slice, and the first of every slice's list
        // for a bound: 2 n keys and more (at most 2 n + 64 of them)
        const uint64_t* list = keys + t * S * n;
        const uint32_t heads = n ? min(n, (2 * n + S - 1) / S) : 0;
        uint32_t v[kGroups];
#pragma unroll
        for (uint32_t k = 0; k < kGroups; ++k) {
            const uint32_t i = tid + 256 * k;
            v[k] = i < S * heads ? (uint32_t)(list[(uint64_t)(i / heads) * n + i % heads] >> 32) : 0u;
        }
        ScorePart p = tid < S ? part[t * S + tid] : ScorePart{0.0f, 0.0f, 0.0f};
        if (p.sum == 0.0f) p.top = -INFINITY;
        const float top = wave_join<false>(p.top);
        p = moved(p, top, c);
        put_wave(s_space, ScorePart{top, wave_join<true>(p.sum), wave_join<true>(p.bend)}, v);
        clear_counts(s_space);
        __syncthreads();
        p = join_parts<4>(s_space.wave, c, max(n, 1u));
        if (p.top == -INFINITY) p.top = 0.0f;
        if (tid == 0) {
            const float at = in.label ? (float)(static_cast<const E*>(in.x) + t * in.ld)[in.label[t]] : 0.0f;
            put_scores(o, t, p, in.label != nullptr, at, in.scale);
        }
        if (n) {
            constexpr uint32_t kCands = TopSpace<256, true>::kCands;
            const uint32_t bound = find_bound(s_space, v, n);
            auto each = [&](auto f) {
                for (uint32_t i = tid; i < S * n; i += 256)
                    if (const uint64_t k = list[i]) f(k);
            };
            each([&](uint64_t k) {
                if ((uint32_t)(k >> 32) < bound) return;
                const uint32_t at = atomicAdd(&s_space.count, 1u);
                if (at < kCands) s_space.key[at] = k;
            });
            __syncthreads();
            if (s_space.count > kCands) narrow(s_space, n, each);
            const uint32_t count = s_space.count;
            put_in_order(s_space, count, n);
            put_top(o, t, s_space, min(count, n), Part{p.top, p.sum}, in.scale);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- gradient

constexpr int kScoreGradU = 2;

// The gradient of slice s of a row, W pieces: with p_v = 2^(d_v - log2 Z) the
// softmax, s p_v (on - entropy' (ln p_v + H)) everywhere, and in the places of
// the row's token and of its list their own derivatives beside it, stored once
// more behind the slice's other entries.  A row's first pieces are under way
// while its factors are found.
template <int TYPE, int THREADS, bool ENTROPY, bool LIST>
__global__ void __launch_bounds__(THREADS)
k_scores_grad(Logits in, ScoresGrad a, uint32_t S, uint32_t W, void* dlogits, uint64_t ldd)
{
    typedef typename Elem<TYPE>::type E;
    constexpr int N = Piece<TYPE>::N, U = kScoreGradU;
    constexpr uint32_t kWaves = THREADS < kMaxTop ? THREADS / 64 : kMaxTop / 64;  // that have entries of a list
    __shared__ double s_sum[kWaves];
    __shared__ uint32_t s_id[LIST ? kMaxTop : 1], s_n[kWaves], s_some[kWaves], s_token;
    __shared__ float s_x[LIST ? kMaxTop : 1], s_g[LIST ? kMaxTop : 1];
    const uint32_t tid = threadIdx.x, V = (uint32_t)in.vocab;
    const float c = in.scale * kLog2e;
    for (uint64_t b = blockIdx.x; b < in.rows * S; b += gridDim.x) {
        const uint64_t t = b / S;
        const uint32_t s = (uint32_t)(b % S);
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        E* out = static_cast<E*>(dlogits) + t * ldd;
        // (one wave has no lane for each single beside a line)
        const RowCut<TYPE> r = THREADS == 64 ? RowCut<TYPE>(V) : RowCut<TYPE>(row, V);
        const uint32_t first = (uint32_t)min((uint64_t)r.full, (uint64_t)s * W);
        const uint32_t end = (uint32_t)min((uint64_t)r.full, (uint64_t)(s + 1) * W);
        const uint32_t label = in.label ? (uint32_t)in.label[t] : 0xFFFFFFFFu;
        const bool scored = !in.label || label < V;
        Piece<TYPE> y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            y[u].none();
            if (scored && (uint64_t)first + tid + THREADS * u < end) y[u].w = load_vec<u32x4>(row + r.piece(first + tid + THREADS * u));
        }
        // the token and the list, an entry a thread
        uint32_t id = 0xFFFFFFFFu;
        float g = 0.0f, x = -INFINITY, at = -INFINITY, single = -INFINITY;
        if (LIST && scored && tid < a.top) {
            id = (uint32_t)a.top_id[t * a.top + tid];
            g = a.d_top[t * a.top + tid];
        }
        const float top = a.norm[2 * t], ln = a.norm[2 * t + 1];
        const float d_logp = a.d_logp ? a.d_logp[t] : 0.0f, d_lse = a.d_lse ? a.d_lse[t] : 0.0f;
        const float d_h = ENTROPY ? a.d_entropy[t] : 0.0f;
        if (scored && label < V) at = (float)row[label];
        if (scored && s == 0 && tid < r.singles) single = (float)row[r.single(tid)];
        const float one = at == -INFINITY ? 0.0f : d_logp;
        double total = 0.0;
        bool any = scored && ln > -INFINITY && (one != 0.0f || d_lse != 0.0f || d_h != 0.0f);
        if constexpr (LIST) {
            if (id < V) x = (float)row[id];
            if (x == -INFINITY) g = 0.0f;
            if (tid < 64 * kWaves) {
                const double sum = wave_sum((double)g);
                const bool some = __any(g != 0.0f);
                if ((tid & 63) == 0) {
                    s_sum[tid >> 6] = sum;
                    s_some[tid >> 6] = some;
                }
            }
            if (tid == 0) s_token = 1;
            __syncthreads();
            uint32_t some = 0;
#pragma unroll
            for (uint32_t w = 0; w < kWaves; ++w) {
                total += s_sum[w];
                some |= s_some[w];
            }
            any = any || (some && scored && ln > -INFINITY);
        }
        if (!any) {
            const u32x4 zero = {0u, 0u, 0u, 0u};
            for (uint64_t j = first + tid; j < end; j += THREADS) store_vec(out + r.piece((uint32_t)j), zero);
            if (s == 0 && tid < r.singles) out[r.single(tid)] = (E)0.0f;
            if (LIST) __syncthreads();
            continue;
        }
        const float l2 = ln * kLog2e, on = in.scale * (float)((double)d_lse - (double)one - total);
        const float A = ENTROPY ? on - in.scale * d_h * a.entropy[t] : on;
        const float B = ENTROPY ? -in.scale * d_h * 0.693147180559945309f : 0.0f;
        auto entry_of = [&](float v) {
            const float d = (v - top) * c - l2, e = exp2_fast(d);
            return ENTROPY ? e * __builtin_fmaf(B, fmaxf(d, -1e4f), A) : e * A;
        };
        // (in place, the token and the list are read before any of it is written)
        __syncthreads();
        for (uint64_t j = first + tid; j < end; j += THREADS * U) {
            Piece<TYPE> next[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                next[u].none();
                if (j + THREADS * (U + u) < end) next[u].w = load_vec<u32x4>(row + r.piece((uint32_t)j + THREADS * (U + u)));
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float e[N];
#pragma unroll
                for (int i = 0; i < N; ++i) e[i] = entry_of(y[u].get(i));
                y[u].put(e);
                if (j + THREADS * u < end) store_vec(out + r.piece((uint32_t)j + THREADS * u), y[u].w);
                y[u] = next[u];
            }
        }
        if (s == 0 && tid < r.singles) out[r.single(tid)] = (E)entry_of(single);
        auto inside = [&](uint32_t v, float x) {
            if (v >= V || x == -INFINITY) return false;
            if (!r.in_piece(v)) return s == 0;
            const uint32_t j = (v - r.head) / N;
            return j >= first && j < end;
        };
        const bool token = inside(label, at);
        // (every store before this is done before the next ones begin)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if constexpr (!LIST) {
            __syncthreads();
            if (token && tid == 0) out[label] = (E)(entry_of(at) + in.scale * one);
        } else {
            // what lies in this slice of the list, in its order
            const bool mine = inside(id, x);
            const uint64_t mask = __ballot(mine);
            if ((tid & 63) == 0 && tid < 64 * kWaves) s_n[tid >> 6] = (uint32_t)__popcll(mask);
            __syncthreads();
            uint32_t before = 0, count = 0;
#pragma unroll
            for (uint32_t w = 0; w < kWaves; ++w) {
                if (w < tid >> 6) before += s_n[w];
                count += s_n[w];
            }
            if (mine) {
                const uint32_t i = before + (uint32_t)__popcll(mask & ((1ull << (tid & 63)) - 1));
                s_id[i] = id;
                s_x[i] = x;
                s_g[i] = g;
            }
            __syncthreads();
            for (uint32_t i = tid; i < count; i += THREADS) {
                // (a token that is there twice: its first entry takes all of them)
                float more = 0.0f;
                bool lead = true;
                for (uint32_t k = 0; k < count; ++k)
                    if (s_id[k] == s_id[i]) {
                        more += s_g[k];
                        lead &= k >= i;
                    }
                if (s_id[i] == label) {
                    more += one;
                    s_token = 0;  // (it has its place on the list)
                }
                if (lead) out[s_id[i]] = (E)(entry_of(s_x[i]) + in.scale * more);
            }
            __syncthreads();
            if (token && tid == 0 && s_token) out[label] = (E)(entry_of(at) + in.scale * one);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- host

constexpr uint32_t kScoreGrid = 1u << 21;  // (of up to 1024 threads each)
constexpr int kLongThreads = 256;  // of a row of several turns
constexpr uint64_t kScoreSlices = 1024;  // of few rows together

struct ScoreCut {
    uint32_t S, W, threads;
};
// Slices of a row at most.
uint64_t most_score_slices(uint64_t pieces) { return std::min<uint64_t>(64, (pieces + 511) / 512); }
ScoreCut cut_scores(uint64_t rows, uint64_t vocab, uint32_t type, uint32_t top)
{
    ScoreCut r;
    const uint64_t pieces = vocab / (type == kF32 ? 4 : 8) + 1;
    const uint64_t want = kScoreSlices / std::min(rows, kScoreSlices);
    const uint64_t S = std::max<uint64_t>(1, std::min(most_score_slices(pieces), want));
    r.W = (uint32_t)((pieces + S - 1) / S);
    r.S = (uint32_t)((pieces + r.W - 1) / r.W);
    const uint32_t threads = (r.W + kScoreU - 1) / kScoreU;
    r.threads = threads <= 64 ? 64 : threads <= 128 ? 128 : threads <= 256 ? 256 : 512;
    if (top > 64) r.threads = std::max(r.threads, 256u);
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
    const uint64_t parts = std::min(kScoreSlices, rows * most_score_slices(pieces));
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
        auto go = [&](auto kern, uint32_t threads) {
            hipLaunchKernelGGL(kern, dim3(grid), dim3(threads), 0, s, in, o, cut.S, cut.W, c, sp.part, sp.keys);
        };
        auto with = [&](auto threads, auto one) {
            constexpr int T = decltype(threads)::value;
            constexpr bool O = decltype(one)::value;
            o.top ? go(k_scores<TY, T, true, O>, T) : go(k_scores<TY, T, false, O>, T);
        };
        typedef std::true_type Y;
        switch (cut.threads) {
        case 64: with(std::integral_constant<int, 64>(), Y()); break;
        case 128: with(std::integral_constant<int, 128>(), Y()); break;
        case 256: with(std::integral_constant<int, 256>(), Y()); break;
        default:
            if (cut.W <= kScoreU * 512)
                with(std::integral_constant<int, 512>(), Y());
            else
                with(std::integral_constant<int, kLongThreads>(), std::false_type());
        }
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
    // (in place, a row's token and list are read before any of it is written: one
    // workgroup a row)
    const bool whole = dlogits == in.x && (a.d_logp || a.d_top);
    // Slices of 1024 pieces, of 512 where there are few (37 x 32000 fp32 4.6 us
    // against 5.2), of 2048 with long lists, which every slice looks through (8192
    // x 131072 bf16 and 64 tokens 724 us against 754; without a list 689 with
    // 1024, 762 with 512, 746 with 2048, 807 by whole rows).
    const bool few = in.rows * pieces < 1024 * 1024;
    const uint32_t W = whole ? (uint32_t)pieces : few ? 512 : a.top > 32 ? 2048 : 1024;
    // One wave for the shortest rows; for whole rows, few and long, 1024 threads.
    const uint32_t T = pieces <= 64 * kScoreGradU && a.top <= 64 ? 64 : whole && pieces > 1024 && in.rows < 1024 ? 1024 : 256;
    const uint32_t S = (uint32_t)((pieces + W - 1) / W);
    const uint32_t grid = (uint32_t)std::min<uint64_t>(in.rows * S, kScoreGrid);
    timer_begin(kTScoresGrad, s);
    by_type(in.type, [&](auto ty) {
        constexpr int TY = decltype(ty)::value;
        auto go = [&](auto kern, uint32_t threads) {
            hipLaunchKernelGGL(kern, dim3(grid), dim3(threads), 0, s, in, a, S, W, dlogits, ldd);
        };
        auto with = [&](auto entropy, auto list) {
            constexpr bool H = decltype(entropy)::value, L = decltype(list)::value;
            T == 64    ? go(k_scores_grad<TY, 64, H, L>, 64)
            : T == 256 ? go(k_scores_grad<TY, 256, H, L>, 256)
                       : go(k_scores_grad<TY, 1024, H, L>, 1024);
        };
        typedef std::true_type Y;
        typedef std::false_type N;
        if (a.d_entropy)
            a.d_top ? with(Y(), Y()) : with(Y(), N());
        else
            a.d_top ? with(N(), Y()) : with(N(), N());
    });
    timer_end(kTScoresGrad, s);
    return hipGetLastError();
}

}  // namespace sparcml
