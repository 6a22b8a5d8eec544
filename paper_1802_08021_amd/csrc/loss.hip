// Losses over rows of logits on gfx950: log probability of each row's token,
// clipped policy loss with a KL term, loss of paired log ratios, and their
// gradients.
//
// With x the row's logits, M their maximum, s the inverse temperature, c = s
// log2(e) and Z = sum_v 2^(c (x_v - M)): the token's log probability is ln 2
// (c (x_label - M) - log2 Z), and for a loss whose derivative by it is q the
// gradient is s q ([v == label] - 2^(c (x_v - M)) / Z).  The difference is
// taken first (c x - c M in one fused multiply-add would overflow where all of
// a row is masked by the type's lowest value).
//
// Many rows: a workgroup a row, the row in registers between the passes over
// it, so that the logits are read once even where the gradient follows
// (k_row).  Few rows, or rows beyond the registers: slices of rows, a
// workgroup each, whose (M, Z) are joined by whoever reads them (k_slices,
// then the gradient by slices again).
#include "internal.h"
#include "types_device.h"

#include <algorithm>

namespace sparcml {
namespace {

constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// ---------------------------------------------------------------- rows

// 16 bytes of a row.
template <int TYPE>
struct Piece {
    typedef typename Elem<TYPE>::type E;
    static constexpr int N = TYPE == kF32 ? 4 : 8;  // elements
    // A word of a piece that holds nothing but -Inf.
    static constexpr uint32_t kNone = TYPE == kF32 ? 0xFF800000u : TYPE == kBf16 ? 0xFF80FF80u : 0xFC00FC00u;
    u32x4 w;
    __device__ __forceinline__ float get(int i) const { return unpack<TYPE>(w, i); }
    // The elements rounded to nearest.
    __device__ __forceinline__ void put(const float* x)
    {
        E y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = (E)x[i];
        w = __builtin_bit_cast(u32x4, y);
    }
    __device__ __forceinline__ void none() { w = u32x4{kNone, kNone, kNone, kNone}; }
    // Keeps the compiler from carrying the unpacked values from one pass to
    // the next (twice to four times the registers).
    __device__ __forceinline__ void repack() { asm volatile("" : "+v"(w)); }
};

// Where a row's pieces lie: from its first 128-byte line on (a wave's accesses
// then take whole lines; the gradient, at the same distance from a line where
// rows and strides agree, leaves none half written), `head` elements in front
// of them, the rest behind.  Single i (head and rest) is element single(i).
constexpr uint32_t kLine = 128;
template <int TYPE>
struct RowCut {
    static constexpr uint32_t N = Piece<TYPE>::N, kHeads = N * (kLine / 16);  // elements of a line
    static constexpr uint32_t kSingles = kHeads + N - 2;                      // singles at most
    uint32_t head, full, singles;
    __device__ __forceinline__ RowCut(const void* row, uint32_t V)
    {
        head = min(V, (uint32_t)((0 - reinterpret_cast<uintptr_t>(row)) / (16 / N)) % kHeads);
        full = (V - head) / N;
        singles = V - full * N;
    }
    __device__ __forceinline__ uint32_t piece(uint32_t j) const { return head + j * N; }
    __device__ __forceinline__ uint32_t single(uint32_t i) const { return i < head ? i : i + full * N; }
    __device__ __forceinline__ bool in_piece(uint32_t v) const { return v >= head && (v - head) / N < full; }
};
constexpr uint32_t kMinThreads = 128;  // a thread for each single

__device__ __forceinline__ bool has_token(const Logits& in, uint64_t t)
{
    return (uint32_t)in.label[t] < (uint32_t)in.vocab;
}
// Whether a row is read at all.
__device__ __forceinline__ bool in_use(const Logits& in, const float* weight, uint64_t t)
{
    return has_token(in, t) && !(weight && weight[t] == 0.0f);
}

// M of a part of a row and the sum of 2^(c (x - M)) over it; nothing (or
// nothing but -Inf): (0, 0).
struct Part {
    float top, sum;
};

// The parts of a row's S slices joined by a group of g lanes (g a power of two
// up to 64, S <= g; every lane of the wave takes part).
__device__ __forceinline__ Part join_slices(const Part* part, uint32_t S, uint32_t g, float c)
{
    const uint32_t i = threadIdx.x & (g - 1);
    const Part p = i < S ? part[i] : Part{0.0f, 0.0f};
    float top = p.sum == 0.0f ? -INFINITY : p.top;  // (without a sum, top means nothing)
    for (uint32_t o = 1; o < g; o <<= 1) top = fmaxf(top, __shfl_xor(top, (int)o));
    if (top == -INFINITY) top = 0.0f;
    float sum = p.sum == 0.0f ? 0.0f : p.sum * exp2_fast((p.top - top) * c);
    for (uint32_t o = 1; o < g; o <<= 1) sum += __shfl_xor(sum, (int)o);
    return Part{top, sum};
}

// ln of a part's sum in fp64: its power of two and log2 of what is left of it,
// in [sqrt(1/2), sqrt(2)), apart (fp32's log of a sum of thousands would be off
// by 5e-7; exactly 0 for 1).
__device__ __forceinline__ double part_ln(float sum)
{
    int e;
    float m = frexpf(sum, &e);
    if (m < 0.707106781f) {
        m *= 2.0f;
        --e;
    }
    return ((double)e + (double)__builtin_amdgcn_logf(m)) * 0.693147180559945309;
}
__device__ __forceinline__ double part_logp(Part p, float x, float scale)
{
    return p.sum == 0.0f ? (double)-INFINITY : ((double)x - (double)p.top) * (double)scale - part_ln(p.sum);
}
__device__ __forceinline__ float part_lse(Part p, float scale)
{
    return p.sum == 0.0f ? -INFINITY : (float)((double)p.top * (double)scale + part_ln(p.sum));
}

// A row's coefficient: beyond fp32, its largest number (an infinity would leave
// NaN where the row has no probability).
__device__ __forceinline__ float within(float x) { return fabsf(x) == INFINITY ? copysignf(3.402823466e38f, x) : x; }

// One gradient entry before the label's own term.
__device__ __forceinline__ float entry(float x, float c, float top, float k) { return k * exp2_fast((x - top) * c); }

// Zeros in the row of the calling workgroup.
template <int TYPE>
__device__ __forceinline__ void clear_row(typename Elem<TYPE>::type* out, uint32_t V)
{
    typedef typename Elem<TYPE>::type E;
    const RowCut<TYPE> r(out, V);
    const u32x4 zero = {0u, 0u, 0u, 0u};
    for (uint32_t j = threadIdx.x; j < r.full; j += blockDim.x) store_vec(out + r.piece(j), zero);
    for (uint32_t i = threadIdx.x; i < r.singles; i += blockDim.x) out[r.single(i)] = (E)0.0f;
}

// ---------------------------------------------------------------- policy terms

// One token's inputs of the policy loss.
struct PolicyRow {
    float w, old, adv, ref;
    PolicyRow() = default;
    __device__ __forceinline__ PolicyRow(const PolicyArgs& a, uint64_t t)
        : w(a.weight[t]), old(a.old_logp[t]), adv(a.adv[t]), ref(a.ref_logp ? a.ref_logp[t] : 0.0f)
    {
    }
    // In scalar registers (the same row in the whole wave).
    __device__ __forceinline__ PolicyRow scalar() const
    {
        auto s = [](float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); };
        PolicyRow r;
        r.w = s(w);
        r.old = s(old);
        r.adv = s(adv);
        r.ref = s(ref);
        return r;
    }
};

// Log probabilities are -Inf where a token cannot come: two that are the same
// infinity are 0 apart, and a factor of 0 takes an infinity away (NaN stays).
__device__ __forceinline__ double apart(double x, double y) { return x == y ? 0.0 : x - y; }
template <class T>
__device__ __forceinline__ T times(T a, T x)
{
    return a == (T)0 && fabs(x) == (T)INFINITY ? (T)0 : a * x;
}

// Its terms and the loss' derivative by its log probability, all with the
// weight.  A row that holds nothing but -Inf has none; a log probability of
// -Inf does not move with the row's logits.
struct PolicyTerms {
    float gain, k, clipped, coef;
};
__device__ __forceinline__ PolicyTerms policy_terms(const PolicyArgs& a, const PolicyRow& q, const Part& p, double lp)
{
    PolicyTerms r;
    const bool none = p.sum == 0.0f;
    const float rho = exp2_fast((float)(apart(lp, (double)q.old) * 1.44269504088896341));
    const float u = times(q.adv, rho), held = times(q.adv, fminf(fmaxf(rho, a.lo), a.hi));
    const bool clipped = u > held;
    r.gain = none ? 0.0f : q.w * (clipped ? held : u);  // (a NaN of u comes through)
    r.clipped = clipped && !none ? q.w : 0.0f;
    r.k = 0.0f;
    r.coef = clipped ? 0.0f : -u;
    if (a.ref_logp) {
        const float far = (float)apart((double)q.ref, lp), em = expm1f(far);
        r.k = none ? 0.0f : q.w * (far == INFINITY ? far : em - far);
        r.coef = r.coef - times(a.kl, em);
    }
    r.coef = lp == -INFINITY ? 0.0f : within(q.w * r.coef);
    return r;
}

// Sums of `count` numbers over a workgroup, in every thread (fixed order).
__device__ __forceinline__ void block_sum(double* x, double (*s_w)[4], int count)
{
    for (int o = 1; o < 64; o <<= 1)
        for (int i = 0; i < count; ++i) x[i] += __shfl_xor(x[i], o);
    if ((threadIdx.x & 63) == 0)
        for (int i = 0; i < count; ++i) s_w[threadIdx.x >> 6][i] = x[i];
    __syncthreads();
    for (int i = 0; i < count; ++i) {
        x[i] = s_w[0][i];
        for (uint32_t q = 1; q < blockDim.x >> 6; ++q) x[i] += s_w[q][i];
    }
}

__device__ __forceinline__ void add_terms(const PolicyTerms& r, double* x)
{
    x[0] += (double)r.gain;
    x[1] += (double)r.k;
    x[2] += (double)r.clipped;
}

__device__ __forceinline__ void put_policy_stats(const PolicyArgs& a, double* x, double (*s_w)[4], float* stats)
{
    block_sum(x, s_w, 3);
    if (threadIdx.x == 0) {
        stats[0] = (float)((a.ref_logp ? times((double)a.kl, x[1]) : 0.0) - x[0]);
        stats[1] = (float)-x[0];
        stats[2] = (float)x[1];
        stats[3] = (float)x[2];
    }
}

// The sums over tokens of their terms (eight rows a thread in flight).  8192
// rows: 6.4 us after a pass over short rows, 8.7 after one over 2 GB, when the
// terms come from HBM.
__global__ void __launch_bounds__(1024) k_policy_stats(uint64_t rows, PolicyArgs a, const PolicyTerms* terms,
                                                       float* stats)
{
    __shared__ double s_w[16][4];
    double x[3] = {0.0, 0.0, 0.0};
    for (uint64_t t = threadIdx.x; t < rows; t += 8192) {
        PolicyTerms r[8] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (t + 1024 * i < rows) r[i] = terms[t + 1024 * i];
#pragma unroll
        for (int i = 0; i < 8; ++i) add_terms(r[i], x);
    }
    put_policy_stats(a, x, s_w, stats);
}

// ---------------------------------------------------------------- a workgroup a row

template <bool SUM>
__device__ __forceinline__ float join_waves(float x, float* s)
{
    x = wave_join<SUM>(x);
    if (blockDim.x == 64) return x;
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    x = s[0];
    for (uint32_t i = 1; i < blockDim.x >> 6; ++i) x = SUM ? x + s[i] : fmaxf(x, s[i]);
    return x;
}

// What a thread has of its row so far: the maximum and the sum against it.
struct Own {
    float top, sum;
    // The first `used` of U pieces (the same in the whole wave).
    template <int TYPE, int U>
    __device__ __forceinline__ void add(Piece<TYPE> (&x)[U], int used, float c)
    {
        float high = top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u >= used) break;
#pragma unroll
            for (int i = 0; i < Piece<TYPE>::N; ++i) high = fmaxf(high, x[u].get(i));
        }
        const float base = high == -INFINITY ? 0.0f : high;
        float more[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u >= used) break;
            x[u].repack();
#pragma unroll
            for (int i = 0; i < Piece<TYPE>::N; ++i) more[i & 3] += exp2_fast((x[u].get(i) - base) * c);
        }
        sum = sum * exp2_fast((top - base) * c) + ((more[0] + more[1]) + (more[2] + more[3]));
        top = high;
    }
};

// Row blockIdx.x by one workgroup: the first NV pieces of a thread stay in
// registers between the two passes over them, LP more in LDS, the rest of a
// longer row is read once more (GRAD; from the 256 MB cache, so its first read
// is not marked nontemporal: 8192 x 131072 bf16 871 us with the mark, 770
// without), the singles one a thread.  Writes the log probability, lse and
// part where wanted, and with GRAD the gradient of the policy loss.
// At 64 registers a thread two workgroups of 1024 share a CU, and one's loads
// and stores go on under the other's exponentials: 8192 x 131072 bf16 770 us, 5.6
// TB/s of logits and gradient (two passes by slices 996; nothing in LDS 790;
// rows of 131072 wholly in registers, one workgroup a CU, 857), 1024 rows 108
// (131, 114), of fp32 222, 4.8 TB/s (250, 228).  Without its exponentials it
// takes as long: what bounds it is memory, at the rate that rows of 256 KB a
// workgroup are copied (5.5 to 6.0 TB/s).
template <int TYPE, int THREADS, int NV, int LP, bool GRAD, bool KEEP>
__global__ void __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(8)))
k_row(Logits in, PolicyArgs a, float c, float* logp, float* lse, Part* part, float* at_label, uint32_t* ticket,
      PolicyTerms* terms, void* dlogits, uint64_t ldd)
{
    typedef typename Elem<TYPE>::type E;
    constexpr int N = Piece<TYPE>::N;
    __shared__ float s_top[THREADS / 64], s_sum[THREADS / 64], s_x, s_coef;
    __shared__ u32x4 s_keep[LP ? LP * THREADS : 1];
    if (!GRAD && blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;  // for k_policy_grad
    const uint64_t t = blockIdx.x;
    const uint32_t V = (uint32_t)in.vocab, label = (uint32_t)in.label[t], tid = threadIdx.x, step = blockDim.x;
    const E* row = static_cast<const E*>(in.x) + t * in.ld;
    E* out = static_cast<E*>(dlogits) + t * ldd;
    if (!in_use(in, a.weight, t)) {
        if (tid == 0) {
            logp[t] = 0.0f;
            if (lse) lse[t] = 0.0f;
            if (terms) terms[t] = PolicyTerms{0.0f, 0.0f, 0.0f, 0.0f};
        }
        if (GRAD) clear_row<TYPE>(out, V);
        return;
    }
    PolicyRow q = {};
    if (terms) q = PolicyRow(a, t).scalar();
    const RowCut<TYPE> r(row, V);
    const int used = (int)min((r.full + step - 1) / step, (uint32_t)NV);
    Piece<TYPE> x[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        x[j].none();
        if (tid + step * j < r.full) x[j].w = load_vec<u32x4, KEEP>(row + r.piece(tid + step * j));
    }
    const float single = tid < r.singles ? (float)row[r.single(tid)] : -INFINITY;
    if (tid == 0) s_x = (float)row[label];
    Own own = {single, single == -INFINITY ? 0.0f : 1.0f};
    // (a thread's slots in LDS are its own: no barrier between the passes)
    for (uint32_t j = tid + step * NV, slot = tid; GRAD && j < r.full; j += step, slot += step) {
        Piece<TYPE> y[1];
        y[0].w = load_vec<u32x4, true>(row + r.piece(j));
        own.add(y, 1, c);
        if (LP && slot < LP * step) s_keep[slot] = y[0].w;
    }
    own.add(x, used, c);
    float top = join_waves<false>(own.top, s_top);
    if (top == -INFINITY) top = 0.0f;
    const Part p = {top, join_waves<true>(own.sum * exp2_fast((own.top - top) * c), s_sum)};
    if (tid == 0) {
        const double lp = part_logp(p, s_x, in.scale);
        logp[t] = (float)lp;
        if (lse) lse[t] = part_lse(p, in.scale);
        if (part) {
            part[t] = p;
            at_label[t] = s_x;
        }
        if (terms) {
            const PolicyTerms m = policy_terms(a, q, p, lp);
            terms[t] = m;
            if (GRAD) s_coef = within(a.grad_scale * in.scale * m.coef);
        }
    }
    if (!GRAD) return;
    // (the first piece that is read again is under way over the barrier)
    uint32_t j = tid + step * (NV + LP);
    Piece<TYPE> next;
    if (j < r.full) next.w = load_vec<u32x4>(row + r.piece(j));
    __syncthreads();
    const float coef = s_coef, xl = s_x;
    const float k = coef == 0.0f ? 0.0f : -coef / p.sum;
    auto write = [&](Piece<TYPE>& q, uint32_t at) {
        q.repack();
        float y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = entry(q.get(i), c, top, k);
        q.put(y);
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
    if (tid < r.singles) out[r.single(tid)] = (E)entry(single, c, top, k);
    // the label's own entry once more, by the thread that has just written it
    const bool mine = r.in_piece(label) ? (label - r.head) / N % step == tid
                                        : tid < r.singles && r.single(tid) == label;
    if (mine) out[label] = (E)(entry(xl, c, top, k) + coef);
}

// ---------------------------------------------------------------- slices of rows

// Slice s of a row: pieces [s W, (s + 1) W); slice 0 takes the singles too.
// (M, Z) of every slice of every row in use, the token's logit beside them;
// with one slice a row its log probability (lse, terms) at once.  Bound by HBM:
// 8192 x 131072 bf16 317 us, 6.8 TB/s (361 with plain loads).
template <int TYPE, bool KEEP>
__global__ void __launch_bounds__(256) k_slices(Logits in, const float* weight, uint32_t S, uint32_t W, float c,
                                                Part* part, float* at_label, float* logp, float* lse, PolicyArgs a,
                                                PolicyTerms* terms, uint32_t* ticket)
{
    typedef typename Elem<TYPE>::type E;
    __shared__ float s_top[4], s_sum[4];
    if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;  // for k_policy_grad
    for (uint64_t b = blockIdx.x; b < in.rows * S; b += gridDim.x) {
        const uint64_t t = b / S;
        const uint32_t s = (uint32_t)(b % S);
        if (!in_use(in, weight, t)) {
            if (S == 1 && threadIdx.x == 0) {
                logp[t] = 0.0f;
                if (lse) lse[t] = 0.0f;
                if (terms) terms[t] = PolicyTerms{0.0f, 0.0f, 0.0f, 0.0f};
            }
            continue;
        }
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        const RowCut<TYPE> r(row, (uint32_t)in.vocab);
        const uint32_t end = (uint32_t)min((uint64_t)r.full, (uint64_t)(s + 1) * W);
        const float single = s == 0 && threadIdx.x < r.singles ? (float)row[r.single(threadIdx.x)] : -INFINITY;
        const float at = threadIdx.x == 0 && s == 0 ? (float)row[in.label[t]] : 0.0f;
        Own own = {single, single == -INFINITY ? 0.0f : 1.0f};
        for (uint32_t j = s * W + threadIdx.x; j < end; j += 1024) {
            Piece<TYPE> x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                x[u].none();
                if (j + 256 * u < end) x[u].w = load_vec<u32x4, KEEP>(row + r.piece(j + 256 * u));
            }
            own.add(x, 4, c);
        }
        float high = join_waves<false>(own.top, s_top);
        if (high == -INFINITY) high = 0.0f;
        const float sum = join_waves<true>(own.sum * exp2_fast((own.top - high) * c), s_sum);
        if (threadIdx.x == 0) {
            const Part p = {high, sum};
            part[b] = p;
            if (s == 0) at_label[t] = at;
            if (S == 1) {
                const double lp = part_logp(p, at, in.scale);
                logp[t] = (float)lp;
                if (lse) lse[t] = part_lse(p, in.scale);
                if (terms) terms[t] = policy_terms(a, PolicyRow(a, t), p, lp);
            }
        }
        __syncthreads();
    }
}

// Calls f(t, lp, p) for rows first, first + 1, ... below end from one workgroup of 256
// threads, by the first lane of each row's group; lp and p are those of a row
// in use.
template <class F>
__device__ __forceinline__ void each_joined(const Logits& in, const float* weight, uint64_t first, uint64_t end,
                                            uint32_t S, uint32_t g, float c, const Part* part, const float* at_label,
                                            F f)
{
    for (uint64_t t0 = first; t0 < end; t0 += 256 / g) {
        const uint64_t t = t0 + threadIdx.x / g;
        const uint64_t in_range = t < end ? t : end - 1;
        const float at = at_label[in_range];
        const bool use = t < end && in_use(in, weight, in_range);
        const Part p = join_slices(part + in_range * S, S, g, c);
        if (t < end && (threadIdx.x & (g - 1)) == 0) f(t, use, use ? part_logp(p, at, in.scale) : 0.0, p);
    }
}

// Log probabilities from the slices, 256 / g rows a workgroup.
__global__ void __launch_bounds__(256) k_join(Logits in, const float* weight, uint32_t S, uint32_t g, float c,
                                              const Part* part, const float* at_label, float* logp, float* lse)
{
    const uint32_t rows = 256 / g;
    for (uint64_t t0 = (uint64_t)blockIdx.x * rows; t0 < in.rows; t0 += (uint64_t)gridDim.x * rows)
        each_joined(in, weight, t0, min(t0 + rows, in.rows), S, g, c, part, at_label,
                    [&](uint64_t t, bool use, double lp, Part p) {
                        logp[t] = (float)lp;
                        if (lse) lse[t] = use ? part_lse(p, in.scale) : 0.0f;
                    });
}

constexpr int kGradU = 2;

// Slice s of a gradient row, of 256 kGradU pieces.  The logits of a row in
// use are under way while its coefficient is found; zeros where that is 0.
template <int TYPE>
struct GradSlice {
    typedef typename Elem<TYPE>::type E;
    static constexpr int N = Piece<TYPE>::N, U = kGradU;
    const RowCut<TYPE> r;
    const uint32_t first;
    const bool singles;
    Piece<TYPE> x[U];
    float single;
    __device__ __forceinline__ GradSlice(const E* row, uint32_t V, uint32_t s, bool use)
        : r(row, V), first(s * (256 * U) + threadIdx.x), singles(s == 0 && threadIdx.x < r.singles), single(0.0f)
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u].none();
            if (use && first + 256 * u < r.full) x[u].w = load_vec<u32x4>(row + r.piece(first + 256 * u));
        }
        if (use && singles) single = (float)row[r.single(threadIdx.x)];
    }
    __device__ __forceinline__ void write(E* out, uint32_t label, float coef, Part p, float c)
    {
        coef = within(coef);
        const bool none = coef == 0.0f || p.sum == 0.0f;
        const float k = none ? 0.0f : -coef / p.sum;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t v = r.piece(first + 256 * u);
            if (first + 256 * u >= r.full) continue;
            float y[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                y[i] = none ? 0.0f : entry(x[u].get(i), c, p.top, k);
                if (!none && label - v == (uint32_t)i) y[i] += coef;
            }
            x[u].put(y);
            store_vec(out + v, x[u].w);
        }
        if (singles) {
            const uint32_t v = r.single(threadIdx.x);
            out[v] = (E)(none ? 0.0f : entry(single, c, p.top, k) + (v == label ? coef : 0.0f));
        }
    }
};

// The policy loss' gradient by slices (S of them for the parts, G for the
// gradient).  A row's first workgroup writes its log probability and terms;
// the last of them to finish sums the terms, in the rows' order.  (Without
// a gradient: G == 1, nothing but that.)
template <int TYPE>
__global__ void __launch_bounds__(256) k_policy_grad(Logits in, PolicyArgs a, uint32_t S, uint32_t g, uint32_t G,
                                                     float c, const Part* part, const float* at_label, float* logp,
                                                     PolicyTerms* terms, uint32_t* ticket, float* stats,
                                                     void* dlogits, uint64_t ldd)
{
    typedef typename Elem<TYPE>::type E;
    __shared__ double s_w[4][4];
    __shared__ uint32_t s_last;
    bool last = false;
    for (uint64_t b = blockIdx.x; b < in.rows * G; b += gridDim.x) {
        const uint64_t t = b / G;
        const uint32_t s = (uint32_t)(b % G);
        const bool use = in_use(in, a.weight, t);
        GradSlice<TYPE> slice(static_cast<const E*>(in.x) + t * in.ld, dlogits ? (uint32_t)in.vocab : 0, s, use);
        Part p = {0.0f, 0.0f};
        PolicyTerms m = {0.0f, 0.0f, 0.0f, 0.0f};
        double lp = 0.0;
        if (use) {
            const PolicyRow q(a, t);
            const float at = at_label[t];
            p = join_slices(part + t * S, S, g, c);
            lp = part_logp(p, at, in.scale);
            m = policy_terms(a, q, p, lp);
        }
        if (s == 0 && threadIdx.x == 0) {
            logp[t] = (float)lp;
            // (device-scope accesses, each done before the next)
            float* w = &terms[t].gain;
            for (int i = 0; i < 3; ++i)
                __hip_atomic_store(w + i, i == 0 ? m.gain : i == 1 ? m.k : m.clipped, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            last = atomicAdd(ticket, 1u) == (uint32_t)in.rows - 1;
        }
        if (dlogits)
            slice.write(static_cast<E*>(dlogits) + t * ldd, (uint32_t)in.label[t], a.grad_scale * in.scale * m.coef, p, c);
    }
    if (threadIdx.x == 0) s_last = last;
    __syncthreads();
    if (!s_last) return;
    double x[3] = {0.0, 0.0, 0.0};
    for (uint64_t t = threadIdx.x; t < in.rows; t += 256)
        for (int i = 0; i < 3; ++i)
            x[i] += (double)__hip_atomic_load(&terms[t].gain + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    put_policy_stats(a, x, s_w, stats);
}

struct PairSums {
    double x[4];  // loss, 1 if in order, rewards
};

// A pair's loss from the sums of its two sequences' log ratios, and the
// derivative by the preferred one's.
struct PairLoss {
    PairSums sums;
    float coef;
};
__device__ __forceinline__ PairLoss pair_loss(const PreferenceArgs& a, uint32_t pairs, double good, double bad)
{
    good = times((double)a.beta, good);
    bad = times((double)a.beta, bad);
    const double h = apart(good, bad), z = exp(-fabs(h)), soft = log1p(z);
    const double up = h >= 0.0 ? 1.0 / (1.0 + z) : z / (1.0 + z);    // sigmoid(h)
    const double down = h >= 0.0 ? z / (1.0 + z) : 1.0 / (1.0 + z);  // sigmoid(-h)
    const double eps = (double)a.smoothing;
    PairLoss r;
    r.sums = PairSums{{times(1.0 - eps, soft - fmin(h, 0.0)) + times(eps, soft + fmax(h, 0.0)), h > 0.0 ? 1.0 : 0.0, good, bad}};
    r.coef = (float)((double)a.beta * (eps * up - (1.0 - eps) * down) / (double)pairs);
    return r;
}
// A token's log ratio; none in a row that holds nothing but -Inf.  (Without a
// branch, so that the loads are under way together.)
__device__ __forceinline__ double log_ratio(const PreferenceArgs& a, uint64_t t, double lp, Part p)
{
    const double x = apart(lp, a.ref_logp ? (double)a.ref_logp[t] : 0.0);
    return p.sum == 0.0f ? 0.0 : x;
}

constexpr uint32_t kFewPairs = 32;
struct FewBounds {
    uint32_t words[2 * kFewPairs + 1];
};

// Pair blockIdx.x: its tokens' log probabilities (S > 1: from the slices),
// rewards of its two sequences, loss, and the derivative by every token's log
// probability.  The sequences' bounds: the launch's arguments, or a table.
__global__ void __launch_bounds__(256) k_pairs(Logits in, PreferenceArgs a, uint32_t pairs, FewBounds few,
                                               const uint32_t* many, uint32_t S, uint32_t g, float c, const Part* part,
                                               const float* at_label, float* logp, float* coef, PairSums* sums)
{
    __shared__ double s_w[4][4];
    const uint32_t b = blockIdx.x;
    const uint32_t lo = many ? many[2 * b] : few.words[2 * b], mid = many ? many[2 * b + 1] : few.words[2 * b + 1];
    const uint32_t end = many ? many[2 * b + 2] : few.words[2 * b + 2];
    double x[2] = {0.0, 0.0};
    auto add = [&](uint64_t t, bool use, double lp, Part p) {
        if (S > 1) logp[t] = (float)lp;
        if (use) x[t < mid ? 0 : 1] += log_ratio(a, t, lp, p);
    };
    if (S > 1)
        each_joined(in, nullptr, lo, end, S, g, c, part, at_label, add);
    else
        for (uint64_t t = (uint64_t)lo + threadIdx.x; t < end; t += 256) add(t, has_token(in, t), logp[t], part[t]);
    block_sum(x, s_w, 2);
    const PairLoss r = pair_loss(a, pairs, x[0], x[1]);
    for (uint64_t t = (uint64_t)lo + threadIdx.x; t < end; t += 256) {
        // (a token whose own logit is -Inf: its log probability does not move)
        const float at = at_label[t];
        coef[t] = has_token(in, t) && at != -INFINITY ? (t < mid ? r.coef : -r.coef) : 0.0f;
    }
    if (threadIdx.x == 0) sums[b] = r.sums;
}

__device__ __forceinline__ void put_pair_stats(double* x, double (*s_w)[4], uint32_t pairs, float* stats)
{
    block_sum(x, s_w, 4);
    if (threadIdx.x == 0)
        for (int q = 0; q < 4; ++q) stats[q] = (float)(x[q] / pairs);
}

// The gradient by slices from coefficients that are there: of a policy loss
// whose rows are one slice each (its terms), or of pairs (coef).  Workgroup 0:
// the sums over tokens or pairs.  Bound by HBM: 8192 x 131072 bf16 680 us of
// a policy loss, 750 of pairs, 5.7 to 6.3 TB/s, with 2 pieces a thread (with one
// 896, with four 709 where two took 690).
template <int TYPE, bool POLICY>
__global__ void __launch_bounds__(256) k_grad(Logits in, PolicyArgs a, const PolicyTerms* terms, uint32_t pairs,
                                              const float* coef, const PairSums* sums, float factor, uint32_t S,
                                              uint32_t g, uint32_t G, float c, const Part* part, float* stats,
                                              void* dlogits, uint64_t ldd)
{
    typedef typename Elem<TYPE>::type E;
    __shared__ double s_w[4][4];
    if (blockIdx.x == 0) {
        double x[4] = {0.0, 0.0, 0.0, 0.0};
        if (POLICY) {
            for (uint64_t t = threadIdx.x; t < in.rows; t += 256) add_terms(terms[t], x);
            put_policy_stats(a, x, s_w, stats);
        } else {
            for (uint32_t i = threadIdx.x; i < pairs; i += 256)
                for (int q = 0; q < 4; ++q) x[q] += sums[i].x[q];
            put_pair_stats(x, s_w, pairs, stats);
        }
        return;
    }
    for (uint64_t b = blockIdx.x - 1; b < in.rows * G; b += gridDim.x - 1) {
        const uint64_t t = b / G;
        const bool use = in_use(in, POLICY ? a.weight : nullptr, t);
        GradSlice<TYPE> slice(static_cast<const E*>(in.x) + t * in.ld, (uint32_t)in.vocab, (uint32_t)(b % G), use);
        const float q = factor * (POLICY ? terms[t].coef : coef[t]);
        Part p = {0.0f, 0.0f};
        if (use) p = POLICY ? part[t] : join_slices(part + t * S, S, g, c);
        slice.write(static_cast<E*>(dlogits) + t * ldd, (uint32_t)in.label[t], q, p, c);
    }
}

// The gradient of a preference loss of few pairs and rows without a launch for
// the pairs: every workgroup sums its own row's pair (the logits are under way
// meanwhile), workgroup 0 all of them.  Up to 256 rows (us, bf16, without / with
// that launch): one pair of 64 x 8000 9.3 / 12.7, 128 x 1000 9.5 / 12.4, 256 x
// 1000 11.9 / 12.8, 256 x 32000 17.6 / 17.2, 512 x 1000 17.9 / 12.9, 512 x 32000
// 27.5 / 25.4; eight pairs of 256 x 8000 10.4 / 12.8, 512 x 8000 12.9 / 14.1, 512 x
// 32000 25.5 / 24.3 (the rows of a pair count, but the crossing is near 256).
constexpr uint32_t kPairRows = 256;
template <int TYPE>
__global__ void __launch_bounds__(256) k_few_pairs(Logits in, PreferenceArgs a, uint32_t pairs, FewBounds bounds,
                                                   uint32_t G, float c, const Part* part, const float* at_label,
                                                   const float* logp, float* stats, void* dlogits, uint64_t ldd)
{
    typedef typename Elem<TYPE>::type E;
    __shared__ double s_w[4][4], s_ratio[kPairRows], s_seq[2 * kFewPairs];
    if (blockIdx.x == 0) {
        // a thread a sequence, from ratios that all threads have fetched
        for (uint32_t t = threadIdx.x; t < (uint32_t)in.rows; t += 256)
            s_ratio[t] = has_token(in, t) ? log_ratio(a, t, (double)logp[t], part[t]) : 0.0;
        __syncthreads();
        if (threadIdx.x < 2 * pairs) {
            double sum = 0.0;
            for (uint32_t t = bounds.words[threadIdx.x]; t < bounds.words[threadIdx.x + 1]; ++t) sum += s_ratio[t];
            s_seq[threadIdx.x] = sum;
        }
        __syncthreads();
        PairSums r = {{0.0, 0.0, 0.0, 0.0}};
        if (threadIdx.x < pairs)
            r = pair_loss(a, pairs, s_seq[2 * threadIdx.x], s_seq[2 * threadIdx.x + 1]).sums;
        put_pair_stats(r.x, s_w, pairs, stats);
        return;
    }
    const uint32_t b = blockIdx.x - 1, t = b / G;
    const bool use = has_token(in, t);
    GradSlice<TYPE> slice(static_cast<const E*>(in.x) + t * in.ld, (uint32_t)in.vocab, b % G, use);
    Part p = {0.0f, 0.0f};
    float q = 0.0f;
    if (use) {
        uint32_t i = 0;  // the row's pair: the last one that begins at or before it
        while (bounds.words[2 * i + 2] <= t) ++i;
        const uint32_t lo = bounds.words[2 * i], mid = bounds.words[2 * i + 1], end = bounds.words[2 * i + 2];
        p = part[t];
        double x[2] = {0.0, 0.0};
        for (uint32_t u = lo + threadIdx.x; u < end; u += 256)
            if (has_token(in, u)) x[u < mid ? 0 : 1] += log_ratio(a, u, (double)logp[u], part[u]);
        block_sum(x, s_w, 2);
        const float d = pair_loss(a, pairs, x[0], x[1]).coef;
        q = at_label[t] == -INFINITY ? 0.0f : a.grad_scale * in.scale * (t < mid ? d : -d);
    }
    slice.write(static_cast<E*>(dlogits) + t * ldd, (uint32_t)in.label[t], q, p, c);
}

// ---------------------------------------------------------------- host

// How a call's rows are taken.  `row`: log probabilities by a workgroup a
// row (k_row), else by S slices of W pieces (k_slices), joined by groups of g
// lanes; `many`: a policy loss and its gradient by a workgroup a row; G: slices
// of a gradient pass.  The rules follow from (us, bf16 unless it says fp32, rows
// x vocabulary):
//   row, rows of up to 4096 pieces (32768 16-bit logits): 8 x 32000 5.2 against
//     6.1 by slices, 256 x 32000 6.4 / 8.3, 1000 x 32000 14.5 / 14.5; beyond,
//     slices: 8 x 65000 7.3 / 6.1, 1000 x 65000 28.3 / 24.1
//   many, from 128 rows on (one pass / two, inputs out of cache):
//      64 x 32000 12.6 / 10.2, fp32 15.9 / 13.3; 64 x 131072 26 / 20, fp32 37 / 27
//     128 x 32000 12.9 / 12.5, fp32 16.8 / 18.3; 128 x 131072 28 / 29, fp32 42 / 45
//     256 x 32000 14.1 / 16.0, fp32 21 / 30; 256 x 131072 35 / 48, fp32 63 / 81
//     512 x 32000 18 / 24, fp32 29 / 50; 512 x 131072 58 / 86, fp32 109 / 151
//     (shorter rows are launches: 128 x 1000 8.5 / 8.3, 256 x 8000 10.5 / 8.8, 512
//     x 1000 9.2 / 8.3, 512 x 8000 12.3 / 12.0, fp32 12.6 / 14.8)
//   slices of few rows: about 1024 workgroups together (300 x 131072 19 with as
//     many, 23 with four times as many), none of less than 512 pieces
struct Cut {
    uint32_t S, W, g, G;
    uint64_t pieces;  // of a row at most
    bool many, row;
};
constexpr uint64_t kManyRows = 128;
constexpr uint64_t kMaxRows = 1u << 21;  // of a launch with a workgroup a row (fewer than 2^32 threads)
constexpr uint32_t kMaxGrid = 1u << 22;
constexpr uint32_t kHold = 8;     // pieces a thread of k_row holds in registers,
constexpr uint32_t kHoldLds = 4;  // and one of 1024 in LDS (64 KB: two workgroups a CU)

constexpr uint64_t kMaxSlices = 1024;  // of few rows together

// Slices of a row at most.
uint64_t most_slices(uint64_t pieces) { return std::min<uint64_t>(64, (pieces + 511) / 512); }

Cut cut_rows(uint64_t rows, uint64_t vocab, uint32_t type)
{
    Cut r;
    r.pieces = vocab / (type == kF32 ? 4 : 8) + 1;
    r.G = (uint32_t)((r.pieces + 256 * kGradU - 1) / (256 * kGradU));
    r.many = rows >= kManyRows;
    r.row = r.pieces <= 512 * kHold;
    const uint64_t want = kMaxSlices / std::min(rows, kMaxSlices);
    const uint64_t S = r.row ? 1 : std::max<uint64_t>(1, std::min(most_slices(r.pieces), want));
    r.W = (uint32_t)((r.pieces + S - 1) / S);
    r.S = (uint32_t)((r.pieces + r.W - 1) / r.W);
    for (r.g = 1; r.g < r.S;) r.g *= 2;
    return r;
}

struct Space {
    Part* part;
    PolicyTerms* terms;
    uint32_t* ticket;
    float *at_label, *coef;
    PairSums* sums;
    uint32_t* bounds;
};
enum class Use { logprob, policy, preference };
Space carve(void* ws, Use use, uint64_t rows, uint64_t parts, uint32_t pairs, size_t* bytes)
{
    Carve c(ws);
    Space r;
    r.part = c.take<Part>(parts);
    r.terms = c.take<PolicyTerms>(use == Use::policy ? rows : 0);
    r.ticket = c.take<uint32_t>(1);
    r.at_label = c.take<float>(rows);
    r.coef = c.take<float>(use == Use::preference ? rows : 0);
    r.sums = c.take<PairSums>(pairs);
    r.bounds = c.take<uint32_t>(pairs ? 2 * (uint64_t)pairs + 1 : 0);
    if (bytes) *bytes = c.used;
    return r;
}
// Enough for every element type (fp32 has the most pieces) and for every call
// of fewer rows or a smaller vocabulary: rows * S falls where S does, so the
// parts are counted by what bounds it, which does not.
size_t workspace(Use use, uint32_t pairs, uint64_t rows, uint64_t vocab)
{
    const uint64_t pieces = cut_rows(rows, vocab, kF32).pieces;
    size_t b = 0;
    carve(nullptr, use, rows, std::max(rows, std::min(kMaxSlices, rows * most_slices(pieces))), pairs, &b);
    return b;
}

template <class F>
void by_type(uint32_t type, F f)
{
    if (type == kF32)
        f(std::integral_constant<int, kF32>());
    else if (type == kBf16)
        f(std::integral_constant<int, kBf16>());
    else
        f(std::integral_constant<int, kF16>());
}

// Of 512 threads up to twice the pieces that they hold (8192 x 50000 bf16: 280
// us, 302 with 1024), of 1024 beyond.
template <bool GRAD, bool KEEP>
void launch_row(const Cut& cut, Logits in, PolicyArgs a, float* logp, float* lse, const Space& sp, PolicyTerms* terms,
                void* dlogits, uint64_t ldd, hipStream_t s)
{
    const float c = in.scale * kLog2e;
    const uint64_t most = cut.pieces <= 1024 * kHold ? 512 : 1024;
    const uint64_t threads = std::max<uint64_t>(kMinThreads, (cut.pieces + kHold * 64 - 1) / (kHold * 64) * 64);
    const uint64_t rows = in.rows, size = in.type == kF32 ? 4 : 2;
    Part* part = GRAD ? nullptr : sp.part;
    float* at_label = sp.at_label;
    by_type(in.type, [&](auto ty) {
        constexpr int TY = decltype(ty)::value;
        for (uint64_t r0 = 0; r0 < rows; r0 += kMaxRows) {
            const dim3 grid((uint32_t)std::min(rows - r0, kMaxRows)), block((uint32_t)std::min(threads, most));
            auto go = [&](auto kern) {
                hipLaunchKernelGGL(kern, grid, block, 0, s, in, a, c, logp, lse, part, at_label, sp.ticket, terms, dlogits,
                                   ldd);
            };
            if (!GRAD || most == 512)  // (cut.row: 512 threads hold the row)
                go(k_row<TY, 512, kHold, 0, GRAD, KEEP>);
            else
                go(k_row<TY, 1024, kHold, kHoldLds, true, false>);
            // the next rows
            auto on = [](auto*& p, uint64_t n) {
                if (p) p += n;
            };
            in.x = static_cast<const uint8_t*>(in.x) + grid.x * in.ld * size;
            if (dlogits) dlogits = static_cast<uint8_t*>(dlogits) + grid.x * ldd * size;
            on(in.label, grid.x);
            on(a.old_logp, grid.x);
            on(a.ref_logp, grid.x);
            on(a.adv, grid.x);
            on(a.weight, grid.x);
            on(logp, grid.x);
            on(lse, grid.x);
            on(part, grid.x);
            on(at_label, grid.x);
            on(terms, grid.x);
        }
    });
}

// The rows in use: log probabilities (where S is 1, or a workgroup takes a
// row), else the parts for who joins them.
// KEEP: the logits are read again soon.
template <bool KEEP>
hipError_t rows_run(const Cut& cut, const Logits& in, const PolicyArgs* policy, const Space& sp, float* logp,
                    float* lse, hipStream_t s)
{
    const float c = in.scale * kLog2e;
    const PolicyArgs a = policy ? *policy : PolicyArgs{};
    PolicyTerms* terms = policy ? sp.terms : nullptr;
    timer_begin(kTLossRows, s);
    if (cut.row) {
        launch_row<false, KEEP>(cut, in, a, logp, lse, sp, terms, nullptr, 0, s);
    } else {
        const uint32_t grid = (uint32_t)std::min<uint64_t>(in.rows * cut.S, kMaxGrid);
        by_type(in.type, [&](auto ty) {
            hipLaunchKernelGGL((k_slices<decltype(ty)::value, KEEP>), dim3(grid), dim3(256), 0, s, in, a.weight, cut.S, cut.W,
                               c, sp.part, sp.at_label, logp, lse, a, terms, sp.ticket);
        });
    }
    timer_end(kTLossRows, s);
    return hipGetLastError();
}

}  // namespace

size_t logprob_workspace(uint64_t rows, uint64_t vocab) { return workspace(Use::logprob, 0, rows, vocab); }
size_t policy_workspace(uint64_t rows, uint64_t vocab) { return workspace(Use::policy, 0, rows, vocab); }
size_t preference_workspace(uint32_t pairs, uint64_t rows, uint64_t vocab)
{
    return workspace(Use::preference, pairs, rows, vocab);
}

hipError_t logprob_run(const Logits& in, float* logp, float* lse, void* ws, hipStream_t s)
{
    const Cut cut = cut_rows(in.rows, in.vocab, in.type);
    const Space sp = carve(ws, Use::logprob, in.rows, in.rows * cut.S, 0, nullptr);
    hipError_t e = rows_run<false>(cut, in, nullptr, sp, logp, lse, s);
    if (e != hipSuccess || cut.S == 1) return e;
    const uint32_t grid = (uint32_t)((in.rows * cut.g + 255) / 256);
    timer_begin(kTLossGrad, s);
    hipLaunchKernelGGL(k_join, dim3(grid), dim3(256), 0, s, in, (const float*)nullptr, cut.S, cut.g,
                       in.scale * kLog2e, sp.part, sp.at_label, logp, lse);
    timer_end(kTLossGrad, s);
    return hipGetLastError();
}

hipError_t policy_run(const Logits& in, const PolicyArgs& a, float* logp, float* stats, void* dlogits, uint64_t ldd,
                      void* ws, hipStream_t s)
{
    const Cut cut = cut_rows(in.rows, in.vocab, in.type);
    const Space sp = carve(ws, Use::policy, in.rows, in.rows * cut.S, 0, nullptr);
    const float c = in.scale * kLog2e;
    const bool fused = dlogits && cut.many;
    if (fused) {
        timer_begin(kTLossRows, s);
        launch_row<true, false>(cut, in, a, logp, nullptr, sp, sp.terms, dlogits, ldd, s);
        timer_end(kTLossRows, s);
    } else {
        hipError_t e = rows_run<false>(cut, in, &a, sp, logp, nullptr, s);
        if (e != hipSuccess) return e;
    }
    if (fused || (!dlogits && cut.S == 1)) {
        timer_begin(kTLossGrad, s);
        hipLaunchKernelGGL(k_policy_stats, dim3(1), dim3(1024), 0, s, in.rows, a, sp.terms, stats);
        timer_end(kTLossGrad, s);
        return hipGetLastError();
    }
    const uint32_t G = dlogits ? cut.G : 1;
    const uint32_t grid = (uint32_t)std::min<uint64_t>(in.rows * G, kMaxGrid);
    timer_begin(kTLossGrad, s);
    by_type(in.type, [&](auto ty) {
        constexpr int TY = decltype(ty)::value;
        if (cut.S == 1)
            hipLaunchKernelGGL((k_grad<TY, true>), dim3(grid + 1), dim3(256), 0, s, in, a, sp.terms, 0u,
                               (const float*)nullptr, (const PairSums*)nullptr, a.grad_scale * in.scale, 1u, 1u, G, c,
                               sp.part, stats, dlogits, ldd);
        else
            hipLaunchKernelGGL((k_policy_grad<TY>), dim3(grid), dim3(256), 0, s, in, a, cut.S, cut.g, G, c, sp.part,
                               sp.at_label, logp, sp.terms, sp.ticket, stats, dlogits, ldd);
    });
    timer_end(kTLossGrad, s);
    return hipGetLastError();
}

hipError_t preference_run(const Logits& in, const PreferenceArgs& a, uint32_t pairs, const uint32_t* bounds,
                          float* logp, float* stats, void* dlogits, uint64_t ldd, void* ws, hipStream_t s)
{
    const Cut cut = cut_rows(in.rows, in.vocab, in.type);
    const Space sp = carve(ws, Use::preference, in.rows, in.rows * cut.S, pairs, nullptr);
    const float c = in.scale * kLog2e;
    // logits that fit the 256 MB cache are found there by the gradient pass (1000
    // rows of 131072 bf16: 132 -> 127 us; 4000 rows: 498 -> 522, so not those)
    const bool fits = in.rows * in.ld * (in.type == kF32 ? 4 : 2) <= (256u << 20);
    hipError_t e = dlogits && fits ? rows_run<true>(cut, in, nullptr, sp, logp, nullptr, s)
                                   : rows_run<false>(cut, in, nullptr, sp, logp, nullptr, s);
    if (e != hipSuccess) return e;
    const size_t words = 2 * (size_t)pairs + 1;
    const uint32_t grid = dlogits ? (uint32_t)std::min<uint64_t>(in.rows * cut.G, kMaxGrid) + 1 : 1;
    FewBounds few = {};
    const uint32_t* many = nullptr;
    if (pairs <= kFewPairs) {
        std::copy(bounds, bounds + words, few.words);
        if (cut.S == 1 && in.rows <= kPairRows && in.rows * cut.G < kMaxGrid) {
            timer_begin(kTLossGrad, s);
            by_type(in.type, [&](auto ty) {
                hipLaunchKernelGGL((k_few_pairs<decltype(ty)::value>), dim3(grid), dim3(256), 0, s, in, a, pairs, few,
                                   cut.G, c, sp.part, sp.at_label, logp, stats, dlogits, ldd);
            });
            timer_end(kTLossGrad, s);
            return hipGetLastError();
        }
    } else {
        e = upload(sp.bounds, bounds, words * sizeof(uint32_t), s);
        if (e != hipSuccess) return e;
        many = sp.bounds;
    }
    timer_begin(kTLossGrad, s);
    hipLaunchKernelGGL(k_pairs, dim3(pairs), dim3(256), 0, s, in, a, pairs, few, many, cut.S, cut.g, c, sp.part,
                       sp.at_label, logp, sp.coef, sp.sums);
    by_type(in.type, [&](auto ty) {
        hipLaunchKernelGGL((k_grad<decltype(ty)::value, false>), dim3(grid), dim3(256), 0, s, in, PolicyArgs{},
                           (const PolicyTerms*)nullptr, pairs, sp.coef, sp.sums, a.grad_scale * in.scale, cut.S, cut.g,
                           cut.G, c, sp.part, stats, dlogits, ldd);
    });
    timer_end(kTLossGrad, s);
    return hipGetLastError();
}

}  // namespace sparcml
