// What rows of logits say, on gfx950: log probability of each row's token, log
// of the row's sum, entropy, and the most likely tokens in order; and the
// gradient of a loss over these.
//
// With x the row's logits, M their maximum, s the inverse temperature, c = s
// log2(e), d_v = c (x_v - M), Z = sum_v 2^d_v and U = sum_v -d_v 2^d_v: log
// probabilities are ln 2 (d_v - log2 Z), the entropy is ln 2 (log2 Z + U / Z).
// Neither of its terms is below 0, so they do not cancel each other.  U moves
// with the maximum as Z does: from M to M' it becomes 2^-h (U + h Z), h = c (M' -
// M).  Sums are taken against a whole number near c M and moved to it behind the
// pass, where Z is held at 1 and U at 0: an entropy near 0 is off by some 10^-7
// (up to 6e-7 at 3001 logits, however small it is), but not below 0, and no log
// probability above.
//
// The n most likely tokens of a row: the pass over its logits leaves the largest
// of each of up to 1024 groups of its lines (128 bytes; of up to 2048 groups of
// a lane's pieces where a list is long for its row), and the n-th largest of
// these is a bound that at least n logits reach and few more do (of 1024 groups
// about 66 for n = 64).  A second launch finds it, looks through the groups that
// reach it once more, and puts what it finds in order.  In the pass' own
// workgroups, where a list keeps these from their next row, it takes 190 us
// against 212 at 4096 x 131072 bf16 with 64 tokens, but 15.5 against 11.7 at 5 x
// 131072 f32 with 20, 93 against 87 at 4096 x 50001 bf16 and 80 against 53 at
// 8192 x 8000; without a list these are 163, 7, 66 and 33 us, of which the reads
// alone take 151, 0.4, 58 and 18.
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
        // (rounding leaves them a few 2^-24 off: the largest logit's own term is 1
        // and 0; comparisons, as NaN has to stay)
        const float Z = z * g, B = g * __builtin_fmaf(-off, z, b);
        return ScorePart{high, Z < 1.0f ? 1.0f : Z, B < 0.0f ? 0.0f : B};
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

constexpr int kScoreU = 4;  // pieces of a thread where a row is one turn
constexpr uint32_t kLineGroups = 1024, kLaneGroups = 2048;  // groups of a row at most

// The waves' parts joined (nothing: M is -Inf).
template <int WAVES>
__device__ __forceinline__ ScorePart join_parts(const ScorePart* wave, float c)
{
    ScorePart p = {-INFINITY, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) p.top = fmaxf(p.top, wave[w].top);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const ScorePart q = moved(wave[w], p.top, c);
        p.sum += q.sum;
        p.bend += q.bend;
    }
    return p;
}

// A row's cut into pieces, for a pass of `threads`: one wave has no lane for
// each single beside a line.
template <int TYPE>
__device__ __forceinline__ RowCut<TYPE> cut_of(const void* row, uint32_t V, bool one_wave)
{
    return one_wave ? RowCut<TYPE>(V) : RowCut<TYPE>(row, V);
}

// Another lane's word, `gap` apart (an exclusive or): within rows of 16 by moves
// of the vector unit.
template <int CTRL>
__device__ __forceinline__ uint32_t moved_word(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
template <int GAP>
__device__ __forceinline__ uint32_t across(uint32_t x)
{
    if constexpr (GAP == 1) return moved_word<0xB1>(x);                     // quad_perm 1 0 3 2
    if constexpr (GAP == 2) return moved_word<0x4E>(x);                     // quad_perm 2 3 0 1
    if constexpr (GAP == 4) return moved_word<0x1B>(moved_word<0x141>(x));  // row_half_mirror, quad_perm 3 2 1 0
    if constexpr (GAP == 8) return moved_word<0x128>(x);                    // row_ror 8
    return (uint32_t)__shfl_xor((int)x, GAP);
}
// The largest of eight neighbours' values.
__device__ __forceinline__ float largest_of_8(float x)
{
    auto with = [](float x, uint32_t y) { return largest(x, __uint_as_float(y), x); };
    x = with(x, across<1>(__float_as_uint(x)));
    x = with(x, across<2>(__float_as_uint(x)));
    return with(x, moved_word<0x141>(__float_as_uint(x)));
}

// Groups of a row's pieces: LANES adjacent lanes' (1 or 8), `units` of each, a
// pass' threads apart; `each` groups a slice, of S slices.
struct Groups {
    uint32_t* largest;  // places, [rows][S each]
    uint32_t units, each;
};

// ---------------------------------------------------------------- the pass

__device__ __forceinline__ bool scored(const Logits& in, uint64_t t) { return !in.label || has_token(in, t); }

// A part once more of pieces [first, end) and, with `singles`, the singles: its
// largest logit is known, and so large that the difference has to be taken first.
template <int TYPE, int THREADS>
__device__ __attribute__((noinline)) ScorePart far_part(const typename Elem<TYPE>::type* row, RowCut<TYPE> r, uint32_t first,
                                                        uint32_t end, bool singles, float top, float c,
                                                        float (*s_far)[THREADS / 64])
{
    float z = 0.0f, b = 0.0f;
    auto take = [&](float x) {
        const float d = (x - top) * c, e = exp2_fast(d);
        z += e;
        b = __builtin_fmaf(-fmaxf(d, -1e4f), e, b);
    };
    if (singles && threadIdx.x < r.singles) take((float)row[r.single(threadIdx.x)]);
    for (uint64_t j = first + threadIdx.x; j < end; j += THREADS) {
        Piece<TYPE> x;
        x.w = load_vec<u32x4, true>(row + r.piece((uint32_t)j));
#pragma unroll
        for (int i = 0; i < Piece<TYPE>::N; ++i) take(x.get(i));
    }
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

// Slice s of a row: pieces [s W, (s + 1) W); slice 0 takes the singles too.
// With one slice a row its numbers at once, and its part where its list needs
// it or there are more; LANES: the groups' for a list, or 0.  ONE: a slice is a
// turn, kScoreU pieces a thread.
template <int TYPE, int THREADS, int LANES, bool ONE>
__global__ void __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(6)))
k_scores(Logits in, ScoresOut o, uint32_t S, uint32_t W, float c, ScorePart* part, Groups groups)
{
    typedef typename Elem<TYPE>::type E;
    constexpr int K = 16 / Piece<TYPE>::N;
    __shared__ ScorePart s_wave[THREADS / 64];
    __shared__ float s_far[2][THREADS / 64];
    __shared__ uint32_t s_largest[LANES == 8 ? kLineGroups : 1];
    const uint32_t tid = threadIdx.x;
    for (uint64_t b = blockIdx.x; b < in.rows * S; b += gridDim.x) {
        const uint64_t t = b / S;
        const uint32_t s = (uint32_t)(b % S);
        if (!scored(in, t)) {
            if (S == 1) put_unused(o, t);
            continue;
        }
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        const RowCut<TYPE> r = cut_of<TYPE>(row, (uint32_t)in.vocab, THREADS == 64);
        const uint32_t first = (uint32_t)min((uint64_t)r.full, (uint64_t)s * W);
        const uint32_t end = (uint32_t)min((uint64_t)r.full, (uint64_t)(s + 1) * W);
        const uint32_t count = end - first;
        const float single = s == 0 && tid < r.singles ? (float)row[r.single(tid)] : -INFINITY;
        const float at = tid == 0 && in.label ? (float)row[in.label[t]] : 0.0f;
        // group number g of the thread's lanes
        uint32_t* largest_of = LANES ? groups.largest + b * groups.each : nullptr;
        auto note = [&](float most, uint32_t g) {
            if (LANES == 1) largest_of[g * THREADS + tid] = place(most);
            if (LANES == 8) {
                most = largest_of_8(most);
                if ((tid & 7) == 0) s_largest[g * (THREADS / 8) + tid / 8] = place(most);
            }
        };
        Piece<TYPE> x[kScoreU];
        float most[kScoreU];
        Tally own;
        if constexpr (ONE) {
#pragma unroll
            for (int u = 0; u < kScoreU; ++u) {
                x[u].none();
                if (tid + THREADS * u < count) x[u].w = load_vec<u32x4>(row + r.piece(first + tid + THREADS * u));
            }
            own.add_one(single, c);
#pragma unroll
            for (int u = 0; u < kScoreU; u += K) own.add<TYPE, K>(x + u, most + u, c);
            if (LANES) {
                if (groups.units == 1) {
#pragma unroll
                    for (int u = 0; u < kScoreU; ++u) note(most[u], u);
                } else if (groups.units == 2) {
                    note(fmaxf(most[0], most[1]), 0);
                    note(fmaxf(most[2], most[3]), 1);
                } else {
                    note(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])), 0);
                }
            }
        } else {
            // K pieces at a time, the next ones under way (loads past the end
            // read the last piece, and count for nothing)
            const uint32_t below = tid & ~63u;  // a wave has mine of the turns
            const uint32_t mine = count > below ? (count - below + K * THREADS - 1) / (K * THREADS) : 0u;
            const uint8_t* from = reinterpret_cast<const uint8_t*>(row + r.piece(first));
            const uint32_t last = count ? (count - 1) * 16 : 0, per = LANES ? groups.units / K : 0;
            Piece<TYPE> y[K];
            Piece<TYPE>(&z)[K] = reinterpret_cast<Piece<TYPE>(&)[K]>(x);
            auto ask = [&](Piece<TYPE>(&q)[K], uint32_t turn) {
#pragma unroll
                for (int u = 0; u < K; ++u)
                    q[u].w = load_vec<u32x4>(reinterpret_cast<const E*>(from + min(((turn * K + u) * THREADS + tid) * 16, last)));
            };
            float group = -INFINITY;
            uint32_t left = per, g = 0;
            auto take = [&](Piece<TYPE>(&q)[K], uint32_t turn) {
                if (turn + 1 == mine)
#pragma unroll
                    for (int u = 0; u < K; ++u)
                        if ((turn * K + u) * THREADS + tid >= count) q[u].none();
                const float high = own.add<TYPE, K>(q, most, c);
                if (LANES) {
                    group = largest(group, high, high);
                    if (--left == 0 || turn + 1 == mine) {
                        note(group, g++);
                        group = -INFINITY;
                        left = per;
                    }
                }
            };
            if (mine) ask(z, 0);
            own.add_one(single, c);
            for (uint32_t turn = 0; turn < mine; turn += 2) {
                if (turn + 1 < mine) ask(y, turn + 1);
                take(z, turn);
                if (turn + 1 >= mine) break;
                if (turn + 2 < mine) ask(z, turn + 2);
                take(y, turn + 1);
            }
            if (LANES)  // (groups that this wave has no piece of)
                for (; g * THREADS < groups.each * LANES; ++g) note(-INFINITY, g);
        }
        ScorePart p = own.join_lanes(c);
        if (THREADS > 64) {
            if ((tid & 63) == 0) s_wave[tid >> 6] = p;
            __syncthreads();
            p = join_parts<THREADS / 64>(s_wave, c);
        }
        if (p.top != -INFINITY && !(fabsf(p.top * c) < kFar)) {
            __syncthreads();
            p = far_part<TYPE, THREADS>(row, r, first, end, s == 0, p.top, c, s_far);
        }
        if (LANES == 8 && THREADS == 64) __syncthreads();
        if (LANES == 8)
            for (uint32_t i = tid; i < groups.each; i += THREADS) largest_of[i] = s_largest[i];
        if (p.top == -INFINITY) p.top = 0.0f;
        if (tid == 0) {
            if (LANES || S > 1) part[b] = p;
            if (S == 1) put_scores(o, t, p, in.label != nullptr, at, in.scale);
        }
        if (THREADS > 64) __syncthreads();
    }
}

// ---------------------------------------------------------------- lists

// What a row's list is found in; up to kCands candidates.  (Little, where a wave
// has a row: the waves of a CU wait for memory in turn.)
constexpr uint32_t kShortTop = 64;
template <int THREADS>
struct TopSpace {
    static constexpr uint32_t kWaves = THREADS / 64, kCands = THREADS == 64 ? 256 : 1024;
    static constexpr uint32_t kTop = THREADS == 64 ? kShortTop : kMaxTop;
    uint32_t count, groups, bound, above;
    uint32_t there[kWaves], low[kWaves], high[kWaves];
    ScorePart part;
    alignas(16) uint32_t hist[256];
    union {
        uint32_t who[kCands];  // first pieces of groups at or above the bound
        uint64_t out[kTop];    // the list in order
    };
    uint64_t key[kCands];  // candidates
};

// A bound that at least n of the numbers that each(f) calls f with reach (1 if
// fewer are not 0) and few more do: the range that holds the n-th largest is cut
// into 256, until few are left in its part (once, as a rule).
template <int THREADS, class Each>
__device__ __forceinline__ uint32_t find_bound(TopSpace<THREADS>& s, uint32_t n, Each each)
{
    constexpr uint32_t kWaves = THREADS / 64;
    const uint32_t lane = threadIdx.x & 63;
    uint32_t there = 0, low = 0, high = 0;  // low: of the complements
    each([&](uint32_t v) {
        there += v != 0;
        low = max(low, v ? ~v : 0u);
        high = max(high, v);
    });
    there = (uint32_t)__builtin_amdgcn_readlane((int)wave_scan(there), 63);
    low = wave_max(low);
    high = wave_max(high);
    if (lane == 0) {
        s.there[threadIdx.x >> 6] = there;
        s.low[threadIdx.x >> 6] = low;
        s.high[threadIdx.x >> 6] = high;
    }
    for (uint32_t i = threadIdx.x; i < 256; i += THREADS) s.hist[i] = 0;
    __syncthreads();
    if (kWaves > 1) {
        there = 0;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) {
            there += s.there[w];
            low = max(low, s.low[w]);
            high = max(high, s.high[w]);
        }
    }
    if (there < n) return 1;
    low = (uint32_t)__builtin_amdgcn_readfirstlane((int)~low);
    high = (uint32_t)__builtin_amdgcn_readfirstlane((int)high);
    for (uint32_t above = 0;;) {  // above: how many lie beyond high
        const uint32_t range = high - low, shift = range < 256 ? 0 : 24 - __clz((int)range);
        each([&](uint32_t v) {
            if (v >= low && v <= high) atomicAdd(&s.hist[(v - low) >> shift], 1u);
        });
        __syncthreads();
        // (every wave for itself: a lane four parts, the highest first)
        const u32x4 h = *reinterpret_cast<const u32x4*>(&s.hist[252 - 4 * lane]);
        const uint32_t all = h[0] + h[1] + h[2] + h[3], upto = wave_scan(all) + above;
        const int at = __ffsll((unsigned long long)__ballot(upto >= n)) - 1;
        uint32_t more = upto - all, cut = 255 - 4 * lane;
#pragma unroll
        for (int k = 3; k >= 0; --k)
            if (more < n) {
                more += h[k];
                cut = 252 - 4 * lane + k;
            }
        more = (uint32_t)__builtin_amdgcn_readlane((int)more, at);
        cut = (uint32_t)__builtin_amdgcn_readlane((int)cut, at);
        const uint32_t from = low + (cut << shift);
        if (more <= n + n / 4 + 8 || shift == 0) return from;
        above = more - s.hist[cut];
        low = from;
        high = from + ((1u << shift) - 1);
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < 256; i += THREADS) s.hist[i] = 0;
        __syncthreads();
    }
}

template <int RUN, int GAP>
__device__ __forceinline__ void exchange(uint64_t& k)
{
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t o = (uint64_t)across<GAP>((uint32_t)(k >> 32)) << 32 | across<GAP>((uint32_t)k);
    const bool larger = ((lane & RUN) == 0) == ((lane & GAP) == 0);  // who keeps the larger one
    k = (o > k) == larger ? o : k;
    if constexpr (GAP > 1) exchange<RUN, GAP / 2>(k);
}
template <int RUN>
__device__ __forceinline__ void sort_lanes(uint64_t& k)
{
    if constexpr (RUN > 2) sort_lanes<RUN / 2>(k);
    exchange<RUN, RUN / 2>(k);
}

// The n largest of s.key[0, count) in order to s.out, count <= kCands: waves put
// 64 at a time in order and look up how many of each other 64 are larger.
template <int THREADS>
__device__ __forceinline__ void put_in_order(TopSpace<THREADS>& s, uint32_t count, uint32_t n)
{
    constexpr uint32_t kWaves = THREADS / 64;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, blocks = (count + 63) / 64;
    for (uint32_t b = wave; b < blocks; b += kWaves) {
        uint64_t k = 64 * b + lane < count ? s.key[64 * b + lane] : 0;
        sort_lanes<64>(k);
        s.key[64 * b + lane] = k;
    }
    __syncthreads();
    for (uint32_t b = wave; b < blocks; b += kWaves) {
        if (lane >= n) continue;  // (its own 64 hold n larger ones)
        const uint64_t k = s.key[64 * b + lane];
        uint32_t rank = lane;
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

// The n largest of more than n keys, that each(f) calls f with, to s.key, eight
// bits a pass: for rows where too many logits reach the bound (most of them
// equal).
template <int THREADS, class Each>
__device__ __attribute__((noinline)) void narrow(TopSpace<THREADS>& s, uint32_t n, Each each)
{
    const uint32_t all = n;
    uint64_t prefix = 0;
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (uint32_t i = threadIdx.x; i < 256; i += THREADS) s.hist[i] = 0;
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

// A row's list, from its parts and groups; with more than one slice (at most 64)
// its numbers too, by the last wave.  R groups a thread; threads: of the pass.
template <int TYPE, int THREADS, int LANES, int R>
__global__ void __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(THREADS == 64 && R <= 16 ? 5 : 4)))
k_lists(Logits in, ScoresOut o, uint32_t S, uint32_t W, float c, const ScorePart* part, Groups groups, uint32_t threads)
{
    typedef typename Elem<TYPE>::type E;
    constexpr int N = Piece<TYPE>::N;
    constexpr uint32_t kCands = TopSpace<THREADS>::kCands;
    __shared__ TopSpace<THREADS> s;
    const uint32_t tid = threadIdx.x, n = o.top;
    for (uint64_t t = blockIdx.x; t < in.rows; t += gridDim.x) {
        if (!scored(in, t)) {
            if (S > 1) put_unused(o, t);
            continue;
        }
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        const RowCut<TYPE> r = cut_of<TYPE>(row, (uint32_t)in.vocab, threads == 64);
        const bool last = tid >= THREADS - 64;
        const uint32_t lane = tid & 63;
        ScorePart p = {0.0f, 0.0f, 0.0f};
        float at = 0.0f;
        if (last && lane < S) p = part[t * S + lane];
        if (last && S > 1 && in.label) at = (float)row[in.label[t]];
        uint32_t v[LANES ? R : 1];
        if (LANES) {
            const uint32_t* group = groups.largest + t * S * groups.each;
#pragma unroll
            for (int e = 0; e < R; ++e) v[e] = tid + e * THREADS < S * groups.each ? group[tid + e * THREADS] : 0u;
        }
        if (tid == 0) s.count = s.groups = 0;
        if (last) {
            // (a lane a slice)
            if (p.sum == 0.0f) p.top = -INFINITY;
            const float top = wave_join<false>(p.top);
            p = moved(p, top, c);
            p = {top == -INFINITY ? 0.0f : top, wave_join<true>(p.sum), wave_join<true>(p.bend)};
            if (lane == 0) s.part = p;
        }
        if constexpr (LANES > 0) {
            const uint32_t bound = find_bound(s, n, [&](auto f) {
#pragma unroll
                for (int e = 0; e < R; ++e) f(v[e]);
            });
            const float least = bound > place(-3.402823466e38f) ? placed(bound) : -3.402823466e38f;
            auto add = [&](float y, uint32_t token) {
                const uint32_t at = atomicAdd(&s.count, 1u);
                if (at < kCands) s.key[at] = key_of(place(y), token);
            };
#pragma unroll
            for (int e = 0; e < R; ++e)
                if (v[e] >= bound) {
                    const uint32_t i = tid + e * THREADS, at = atomicAdd(&s.groups, 1u);
                    // the group's first piece
                    const uint32_t slice = S == 1 ? 0 : i / groups.each, g = i - slice * groups.each;
                    const uint32_t row_of = threads / LANES;
                    if (at < kCands) s.who[at] = slice * W + g / row_of * groups.units * threads + g % row_of * LANES;
                }
            for (uint32_t i = tid; i < r.singles; i += THREADS) {
                const float y = (float)row[r.single(i)];
                if (y >= least) add(y, r.single(i));
            }
            __syncthreads();
            // a lane a piece (each group has a candidate: too many groups are too
            // many of these)
            const uint32_t found = s.groups, pieces = groups.units * LANES, shift = 31 - __clz((int)pieces);
            if (found > kCands && tid == 0) s.count = kCands + 1;
            auto piece_of = [&](uint32_t i) {
                const uint32_t k = i & (pieces - 1);
                return s.who[i >> shift] + k / LANES * threads + k % LANES;
            };
            auto stop_of = [&](uint32_t j) { return S == 1 ? r.full : min(r.full, (j / W + 1) * W); };
            // (several of a lane's under way: a round trip to memory is 2 us)
            constexpr int U = THREADS == 64 ? 4 : 8;
            for (uint32_t i = tid; i < found << shift && found <= kCands; i += U * THREADS) {
                Piece<TYPE> y[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    y[u].none();
                    if (i - tid + u * THREADS >= found << shift) continue;  // (of the whole workgroup)
                    const uint32_t at = min(i + u * THREADS, (found << shift) - 1), j = piece_of(at);
                    if (at == i + u * THREADS && j < stop_of(s.who[at >> shift])) y[u].w = load_vec<u32x4, true>(row + r.piece(j));
                }
                if constexpr (THREADS > 64) {
                    // (all marks of a lane's in one run, their logits read again: 5 x 131072
                    // fp32 with 256 tokens 23 us against 29)
                    uint64_t marks = 0;
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int e = 0; e < N; ++e) marks |= (uint64_t)(y[u].get(e) >= least) << (N * u + e);
                    while (marks) {
                        const uint32_t bit = (uint32_t)__ffsll((unsigned long long)marks) - 1;
                        marks &= marks - 1;
                        const uint32_t token = r.piece(piece_of(i + bit / N * THREADS)) + bit % N;
                        add((float)row[token], token);
                    }
                } else {
                    // (a piece's marks at a time, selected from registers: 4096 x 50001 bf16
                    // with 20 tokens 87 us against 93; a place in the code for every element
                    // takes longer to fetch)
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (i - tid + u * THREADS >= found << shift) continue;
                        uint32_t marks = 0;
#pragma unroll
                        for (int e = 0; e < N; ++e) marks |= (uint32_t)(y[u].get(e) >= least) << e;
                        while (__any(marks != 0)) {
                            if (marks) {
                                const int e = __ffs((int)marks) - 1;
                                marks &= marks - 1;
                                float v = y[u].get(0);
#pragma unroll
                                for (int q = 1; q < N; ++q) v = e == q ? y[u].get(q) : v;
                                add(v, r.piece(piece_of(i + u * THREADS)) + e);
                            }
                        }
                    }
                }
            }
            __syncthreads();
            if (s.count > kCands)
                // (by value: what a call might change stays in memory for all of the
                // kernel, 88 against 93 us at 4096 x 50001 bf16 with 20 tokens)
                narrow(s, n, [=, known = found <= kCands, of = s.who](auto f) {
                    for (uint32_t i = tid; i < r.singles; i += THREADS)
                        if (const uint32_t k = place((float)row[r.single(i)])) f(key_of(k, r.single(i)));
                    // the groups that reach the bound, where they are known
                    const uint32_t all = known ? found << shift : r.full;
                    for (uint32_t i = tid; i < all; i += THREADS) {
                        uint32_t j = i;
                        if (known) {
                            const uint32_t k = i & (pieces - 1), first = of[i >> shift];
                            j = first + k / LANES * threads + k % LANES;
                            if (j >= (S == 1 ? r.full : min(r.full, (first / W + 1) * W))) continue;
                        }
                        Piece<TYPE> y;
                        y.w = load_vec<u32x4, true>(row + r.piece(j));
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            if (const uint32_t k = place(y.get(e))) f(key_of(k, r.piece(j) + e));
                    }
                });
            const uint32_t count = s.count;
            put_in_order(s, count, n);
            const Part q = {s.part.top, s.part.sum};
            for (uint32_t i = tid; i < n; i += THREADS) {
                const uint64_t k = i < count ? s.out[i] : 0;
                o.top_id[t * n + i] = i < count ? (int32_t)~(uint32_t)k : -1;
                o.top_logp[t * n + i] = i < count ? (float)part_logp(q, placed((uint32_t)(k >> 32)), in.scale) : -INFINITY;
            }
        }
        if (S > 1 && tid == THREADS - 64) put_scores(o, t, p, in.label != nullptr, at, in.scale);
        __syncthreads();
    }
}

// ---------------------------------------------------------------- gradient

constexpr int kScoreGradU = 2;

// Factors of the softmax, from derivatives that are finite, held where no product
// with a logarithm (at least kNoShare, where 2^d is 0) leaves fp32: tokens without
// probability, 0 times the factor, would have NaN.
constexpr float kNoShare = -160.0f;
__device__ __forceinline__ float held(double x)
{
    return (float)(fabs(x) > 1e36 && fabs(x) < INFINITY ? copysign(1e36, x) : x);
}

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
    const float c = log2_scale(in.scale);
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
        bool any = scored && ln != -INFINITY && (one != 0.0f || d_lse != 0.0f || d_h != 0.0f);
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
            any = any || (some && scored && ln != -INFINITY);
        }
        if (!any) {
            const u32x4 zero = {0u, 0u, 0u, 0u};
            for (uint64_t j = first + tid; j < end; j += THREADS) store_vec(out + r.piece((uint32_t)j), zero);
            if (s == 0 && tid < r.singles) out[r.single(tid)] = (E)0.0f;
            if (LIST) __syncthreads();
            continue;
        }
        const float l2 = ln * kLog2e;
        const double scale = (double)in.scale, on = (double)d_lse - (double)one - total, h = (double)d_h;
        const float A = held(scale * (ENTROPY ? on - h * (double)a.entropy[t] : on));
        const float B = ENTROPY ? held(-scale * h * 0.693147180559945309) : 0.0f;
        auto entry_of = [&](float v) {
            const float d = (v - top) * c - l2, e = exp2_fast(d);
            return ENTROPY ? e * __builtin_fmaf(B, fmaxf(d, kNoShare), A) : e * A;
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
// Slices of few rows together (300 x 131072 bf16 with 20 tokens 28 us against 38
// with 512, 130 20 against 21, 300 x 32000 19.6 against 18.1; 2048: the same).
constexpr uint64_t kScoreSlices = 1024;
constexpr int kLongThreads = 256;          // of a row of several turns

// S slices of W pieces; groups of `lanes` (0: no list) and `units`, `each` a
// slice.
struct ScoreCut {
    uint32_t S, W, threads, lanes, units, each;
    bool one;
};
// Slices of a row at most.
uint64_t most_score_slices(uint64_t pieces) { return std::min<uint64_t>(64, (pieces + 511) / 512); }
ScoreCut cut_scores(uint64_t rows, uint64_t vocab, uint32_t type, uint32_t top)
{
    ScoreCut r;
    const uint64_t pieces = std::max<uint64_t>(1, vocab / (type == kF32 ? 4 : 8));
    const uint64_t want = kScoreSlices / std::min(rows, kScoreSlices);
    for (uint64_t S = std::max<uint64_t>(1, std::min(most_score_slices(pieces), want));; S /= 2) {
        r.W = (uint32_t)(((pieces + S - 1) / S + 7) / 8 * 8);
        r.S = (uint32_t)((pieces + r.W - 1) / r.W);
        const uint32_t threads = (r.W + kScoreU - 1) / kScoreU;
        r.one = threads <= 512;
        r.threads = threads <= 64 ? 64 : threads <= 128 ? 128 : threads <= 256 ? 256 : r.one ? 512 : kLongThreads;
        // (a group of lines of each lane at least)
        if (!top || S == 1 || r.S * (r.threads / 8) <= kLineGroups) break;
    }
    r.lanes = r.units = r.each = 0;
    if (!top) return r;
    // Groups of lines, unless the list is more than two thirds as long as those
    // that hold anything are many: few groups are a low bound (4096 rows bf16: 8000
    // with 64 tokens, 125 lines' groups, 40 us against 49 by lanes; 32000 with 200,
    // 250 of these, 127 against 106; 1000 with 25, 15 of these, 147 against 17).
    // Lines also where many slices leave no room for a group of each lane.
    const uint32_t least = r.one ? 1 : type == kF32 ? 4 : 2, all = r.one ? kScoreU : (r.W + r.threads - 1) / r.threads;
    for (r.lanes = 8;; r.lanes = 1) {
        const uint32_t most = r.lanes == 8 ? kLineGroups : kLaneGroups;
        for (r.units = least;; r.units *= 2) {
            r.each = (all + r.units - 1) / r.units * (r.threads / r.lanes);
            if (r.S * r.each <= most || r.units >= all) break;
        }
        if (r.lanes == 1 || r.S * r.threads > kLaneGroups) return r;
        if (2 * std::min<uint64_t>(r.S * r.each, pieces / (8 * r.units)) >= 3 * top) return r;
    }
}

// Rows whose lists are by a wave each, of at most kShortTop tokens; fewer have
// 256 threads each (bf16: 512 x 131072 with 20 tokens 36 us against 41 by waves,
// 1000 x 32000 with 64 27 against 35; 1500 x 32000 39 against 41, 8192 x 32000
// 152 against 129, 8192 x 8000 with 20 82 against 53).
constexpr uint64_t kManyLists = 1024;

struct ScoreSpace {
    ScorePart* part;
    uint32_t* largest;
};
ScoreSpace carve_scores(void* ws, uint64_t parts, uint64_t groups, size_t* bytes)
{
    Carve c(ws);
    ScoreSpace r;
    r.part = c.take<ScorePart>(parts);
    r.largest = c.take<uint32_t>(groups);
    if (bytes) *bytes = c.used;
    return r;
}

}  // namespace

// (Enough for every type and for every call of fewer rows, a smaller vocabulary
// or shorter lists: parts and groups are counted by what bounds them.)
size_t scores_workspace(uint32_t top, uint64_t rows, uint64_t vocab)
{
    size_t b = 0;
    // (a wave's lanes with kScoreU groups each, or a group for every piece where the
    // threads round up to a power of two: at most two for each of the row's)
    const uint64_t groups = std::min<uint64_t>(kLaneGroups, std::max<uint64_t>(256, vocab + 4));
    carve_scores(nullptr, std::max(rows, std::min(kScoreSlices, rows * most_score_slices(vocab / 4 + 1))),
                 top ? rows * groups : 0, &b);
    return b;
}

hipError_t scores_run(const Logits& in, const ScoresOut& o, void* ws, hipStream_t s)
{
    const ScoreCut cut = cut_scores(in.rows, in.vocab, in.type, o.top);
    const ScoreSpace sp = carve_scores(ws, in.rows * cut.S, in.rows * cut.S * cut.each, nullptr);
    const Groups groups = {sp.largest, cut.units, cut.each};
    const bool many = in.rows >= kManyLists;
    const float c = log2_scale(in.scale);
    const uint32_t grid = (uint32_t)std::min<uint64_t>(in.rows * cut.S, kScoreGrid);
    const uint32_t rows = (uint32_t)std::min<uint64_t>(in.rows, kScoreGrid);
    timer_begin(kTScores, s);
    by_type(in.type, [&](auto ty) {
        constexpr int TY = decltype(ty)::value;
        typedef std::true_type Y;
        auto by_lanes = [&](auto f) {
            if (cut.lanes == 8)
                f(std::integral_constant<int, 8>());
            else if (cut.lanes == 1)
                f(std::integral_constant<int, 1>());
            else
                f(std::integral_constant<int, 0>());
        };
        auto pass = [&](auto threads, auto one) {
            by_lanes([&](auto lanes) {
                constexpr int T = decltype(threads)::value;
                hipLaunchKernelGGL((k_scores<TY, T, decltype(lanes)::value, decltype(one)::value>), dim3(grid), dim3(T), 0, s,
                                   in, o, cut.S, cut.W, c, sp.part, groups);
            });
        };
        if (!cut.one)
            pass(std::integral_constant<int, kLongThreads>(), std::false_type());
        else if (cut.threads == 64)
            pass(std::integral_constant<int, 64>(), Y());
        else if (cut.threads == 128)
            pass(std::integral_constant<int, 128>(), Y());
        else if (cut.threads == 256)
            pass(std::integral_constant<int, 256>(), Y());
        else
            pass(std::integral_constant<int, 512>(), Y());
        if (!cut.lanes && cut.S == 1) return;
        by_lanes([&](auto lanes) {
            constexpr int L = decltype(lanes)::value;
            auto go = [&](auto threads, auto held) {
                constexpr int T = decltype(threads)::value;
                hipLaunchKernelGGL((k_lists<TY, T, L, decltype(held)::value>), dim3(rows), dim3(T), 0, s, in, o, cut.S, cut.W, c,
                                   sp.part, groups, cut.threads);
            };
            typedef std::integral_constant<int, 64> One;
            typedef std::integral_constant<int, 256> Four;
            const uint32_t all = cut.S * cut.each;
            if (many && o.top <= kShortTop && L) {
                if (all <= 256)
                    go(One(), std::integral_constant<int, 4>());
                else if (all <= 512)
                    go(One(), std::integral_constant<int, 8>());
                else if (all <= 1024)
                    go(One(), std::integral_constant<int, 16>());
                else
                    go(One(), std::integral_constant<int, L == 1 ? 32 : 16>());
            } else {
                go(Four(), std::integral_constant<int, L == 1 ? 8 : 4>());
            }
        });
    });
    timer_end(kTScores, s);
    return hipGetLastError();
}

hipError_t scores_grad_run(const Logits& in, const ScoresGrad& a, void* dlogits, uint64_t ldd, hipStream_t s)
{
    const uint64_t pieces = in.vocab / (in.type == kF32 ? 4 : 8) + 1;
    // (in place, a row's token and list are read before any of it is written: one
    // workgroup a row, which takes longer than slices into another tensor do: 5 x
    // 131072 fp32 with 20 tokens 14.9 us against 5.0, 37 x 32000 with the row's token
    // 5.8 against 4.7; bf16 4096 x 50001 with 20 tokens 155 against 147, 8192 x
    // 131072 with the row's token 805 against 686)
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
