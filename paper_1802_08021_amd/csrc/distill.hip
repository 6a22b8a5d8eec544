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
// computed of a list's entries is in fp64 (a few hundred a row).
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

// What a row's gradient is made of, and its terms of the sums over rows.
struct DistillRow {
    double ln, off, far;  // ln S; what makes log probabilities of the list's values; F
    float top, rest_top;  // M; the largest unlisted logit
    float A, k, hard;     // coefficient off the list; scales; of the given token
    float div, nll, covered;
};

// One outcome's share of the divergence and its derivative by the student's
// log probability (lq, lp: log probabilities; a probability of 0 takes an
// infinity away).
struct Share {
    double div, f;
};
__device__ __forceinline__ double product(double p, double x) { return p == 0.0 ? 0.0 : p * x; }
__device__ __forceinline__ Share share_of(float beta, double lq, double lp)
{
    const double q = exp(lq), p = exp(lp), b = (double)beta;
    Share r;
    if (beta == 0.0f) {
        r.div = product(q, lq - lp);
        r.f = -q;
    } else if (beta == 1.0f) {
        r.div = r.f = product(p, lp - lq);
    } else {
        const double lm = log(b * q + (1.0 - b) * p);
        r.f = (1.0 - b) * product(p, lp - lm);
        r.div = b * product(q, lq - lm) + r.f;
    }
    if (lp == -INFINITY) r.f = 0.0;  // (a logit of -Inf does not move)
    return r;
}

// A listed token's gradient.
__device__ __forceinline__ float listed_entry(const DistillArgs& a, const DistillRow& w, float value, float x, float scale)
{
    const double lp = ((double)x - (double)w.top) * (double)scale - w.ln;
    const Share e = share_of(a.beta, (double)value * (a.rest ? 1.0 : (double)a.teacher_scale) - w.off, lp);
    const double soft = 1.0 - (double)a.hard;
    return within((float)((double)w.k * (soft * e.f + exp(lp) * ((double)w.hard - soft * w.far))));
}

// ---------------------------------------------------------------- sums

constexpr uint32_t kWindow = 4096;  // pieces whose marks lie in LDS at a time

// Slice s of a row, as k_slices takes them: (M, Z) over the unlisted tokens.
template <int TYPE>
__global__ void __launch_bounds__(256) k_rest_slices(Logits in, DistillArgs a, uint32_t S, uint32_t W, float c, Part* part)
{
    typedef typename Elem<TYPE>::type E;
    constexpr uint32_t N = Piece<TYPE>::N;
    __shared__ float s_top[4], s_sum[4];
    __shared__ uint32_t s_marks[kWindow * N / 32], s_single[4];
    const uint32_t tid = threadIdx.x, V = (uint32_t)in.vocab;
    for (uint64_t b = blockIdx.x; b < in.rows * S; b += gridDim.x) {
        const uint64_t t = b / S;
        const uint32_t s = (uint32_t)(b % S);
        if (!distilled(in, a, t)) continue;
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
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
                const uint32_t marks = s_marks[(j - at) * N / 32] >> ((j - at) * N % 32) & ((1u << N) - 1);
                if (marks)
                    for (uint32_t i = 0; i < 4; ++i) {
                        const uint32_t two = marks >> (i * N / 4);
                        const uint32_t m = N == 4 ? (two & 1u ? ~0u : 0u)
                                                  : (two & 1u ? 0xFFFFu : 0u) | (two & 2u ? 0xFFFF0000u : 0u);
                        x[0].w[i] = (x[0].w[i] & ~m) | (Piece<TYPE>::kNone & m);
                    }
                own.add(x, 1, c);
            }
            __syncthreads();
        }
        float high = join_waves<false>(own.top, s_top);
        if (high == -INFINITY) high = 0.0f;
        const float sum = join_waves<true>(own.sum * exp2_fast((own.top - high) * c), s_sum);
        if (tid == 0) part[b] = Part{high, sum};
        __syncthreads();
    }
}

// ---------------------------------------------------------------- terms

// Row blockIdx.x: its terms from the slices' parts and its list, an entry a
// thread.
template <int TYPE>
__global__ void __launch_bounds__(256) k_distill_terms(Logits in, DistillArgs a, uint32_t S, float c, const Part* part,
                                                       DistillRow* terms, float* div)
{
    typedef typename Elem<TYPE>::type E;
    __shared__ double s_w[4][4], s_w2[4][4], s_w3[4][4];
    __shared__ float s_top[4], s_value[4];
    __shared__ uint32_t s_id[kMaxTop];
    const uint32_t tid = threadIdx.x, V = (uint32_t)in.vocab;
    for (uint64_t t = blockIdx.x; t < in.rows; t += gridDim.x) {
        if (!distilled(in, a, t)) {
            if (tid == 0) {
                terms[t] = DistillRow{};
                div[t] = 0.0f;
            }
            continue;
        }
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        Entry e(a, t, tid, V);
        // a token that is there twice counts by its first entry
        s_id[tid] = e.v;
        __syncthreads();
        if (e.v < V)
            for (uint32_t i = 0; i < tid; ++i)
                if (s_id[i] == e.v) {
                    e.v = 0xFFFFFFFFu;
                    break;
                }
        const bool there = e.v < V;
        const float x = there ? (float)row[e.v] : -INFINITY;
        const float at = in.label ? (float)row[in.label[t]] : -INFINITY;
        const Part rest = join_slices(part + t * S, S, 64, c);
        // the teacher's log probabilities: value * scale - off
        const double ts = a.rest ? 1.0 : (double)a.teacher_scale;
        double off = 0.0, left = 0.0;
        const float best = a.rest ? 0.0f : join_waves<false>(there ? e.value : -INFINITY, s_value);
        const float top_x = join_waves<false>(x, s_top);
        const float M = fmaxf(top_x, rest.sum == 0.0f ? -INFINITY : rest.top);
        const float top = M == -INFINITY ? 0.0f : M;
        const double near = ((double)x - (double)top) * (double)in.scale;
        double sums[2] = {there ? exp(a.rest ? (double)e.value : ((double)e.value - (double)best) * ts) : 0.0,
                          there ? exp(near) : 0.0};
        block_sum(sums, s_w, 2);
        if (a.rest)
            left = fmax(1.0 - sums[0], 0x1p-24);
        else if (sums[0] > 0.0)
            off = (double)best * ts + log(sums[0]);
        const double far = ((double)rest.top - (double)top) * (double)in.scale;
        const double outside = rest.sum == 0.0f ? 0.0 : exp(far) * (double)rest.sum;
        const double total = outside + sums[1], ln = log(total);
        Share own = {0.0, 0.0};
        double p = 0.0;
        if (there) {
            own = share_of(a.beta, (double)e.value * ts - off, near - ln);
            p = exp(near - ln);
        }
        double all[3] = {own.div, own.f, p};
        block_sum(all, s_w2, 3);
        if (tid == 0) {
            DistillRow w = {};
            if (total != 0.0) {
                Share out = {0.0, 0.0};
                if (a.rest && rest.sum != 0.0f) out = share_of(a.beta, log(left), far + part_ln(rest.sum) - ln);
                const double F = all[1] + out.f, soft = 1.0 - (double)a.hard;
                const double weight = a.weight ? (double)a.weight[t] : 1.0;
                const bool given = in.label && at != -INFINITY;
                w.ln = ln;
                w.off = off;
                w.far = F;
                w.top = top;
                w.rest_top = rest.top;
                w.k = within((float)(weight * (double)a.grad_scale * (double)in.scale));
                w.hard = given ? a.hard : 0.0f;
                if (rest.sum != 0.0f)
                    w.A = within((float)((double)w.k * (soft * out.f / (double)rest.sum +
                                                        ((double)w.hard - soft * F) * exp(far) / total)));
                w.div = (float)(all[0] + out.div);
                w.nll = in.label ? (float)(ln - ((double)at - (double)top) * (double)in.scale) : 0.0f;
                w.covered = (float)all[2];
            }
            terms[t] = w;
            div[t] = w.div;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- gradient

constexpr int kDistillU = 2;

// A factor of 0 takes an infinity away.
__device__ __forceinline__ double weighed(double w, double x) { return w == 0.0 ? 0.0 : w * x; }

// Slice s of a gradient row, 256 kDistillU pieces; workgroup 0: the sums over
// the rows.
template <int TYPE>
__global__ void __launch_bounds__(256) k_distill_grad(Logits in, DistillArgs a, uint32_t G, float c,
                                                      const DistillRow* terms, float* stats, void* dlogits, uint64_t ldd)
{
    typedef typename Elem<TYPE>::type E;
    constexpr int N = Piece<TYPE>::N, U = kDistillU;
    __shared__ double s_w[4][4];
    __shared__ uint32_t s_id[kMaxTop], s_n[4];
    __shared__ uint8_t s_given;
    const uint32_t tid = threadIdx.x, V = (uint32_t)in.vocab;
    if (blockIdx.x == 0) {
        double x[4] = {0.0, 0.0, 0.0, 0.0};
        for (uint64_t t = tid; t < in.rows; t += 256) {
            const DistillRow& w = terms[t];
            if (!distilled(in, a, t)) continue;
            const double weight = a.weight ? (double)a.weight[t] : 1.0, soft = 1.0 - (double)a.hard;
            x[0] += weight * (weighed(soft, (double)w.div) + weighed((double)a.hard, (double)w.nll));
            x[1] += weight * (double)w.div;
            x[2] += weight * (double)w.nll;
            x[3] += weight * (double)w.covered;
        }
        block_sum(x, s_w, 4);
        if (tid == 0)
            for (int i = 0; i < 4; ++i) stats[i] = (float)x[i];
        return;
    }
    for (uint64_t b = blockIdx.x - 1; b < in.rows * G; b += gridDim.x - 1) {
        const uint64_t t = b / G;
        const uint32_t s = (uint32_t)(b % G);
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        E* out = static_cast<E*>(dlogits) + t * ldd;
        const RowCut<TYPE> r(row, V);
        const uint32_t first = min(r.full, s * (256 * U)), end = min(r.full, first + 256 * U);
        const bool use = distilled(in, a, t);
        const DistillRow w = terms[t];
        const uint32_t label = in.label ? (uint32_t)in.label[t] : 0xFFFFFFFFu;
        auto inside = [&](uint32_t v) {
            if (v >= V) return false;
            if (!r.in_piece(v)) return s == 0;
            return (v - r.head) / N >= first && (v - r.head) / N < end;
        };
        Entry e(a, t, tid, V);
        const bool mine = use && inside(e.v);
        const float x = mine ? (float)row[e.v] : -INFINITY;
        const float at = use && inside(label) ? (float)row[label] : -INFINITY;
        const float single = use && s == 0 && tid < r.singles ? (float)row[r.single(tid)] : -INFINITY;
        Piece<TYPE> y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            y[u].none();
            if (use && first + tid + 256 * u < end) y[u].w = load_vec<u32x4>(row + r.piece(first + tid + 256 * u));
        }
        // the slice's part of the list, in its order
        const uint64_t mask = __ballot(mine);
        if ((tid & 63) == 0) s_n[tid >> 6] = (uint32_t)__popcll(mask);
        if (tid == 0) s_given = 0;
        // (in place, what is read above lies before what is written below)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        uint32_t before = 0, count = 0;
        for (uint32_t q = 0; q < 4; ++q) {
            if (q < tid >> 6) before += s_n[q];
            count += s_n[q];
        }
        const uint32_t place = before + (uint32_t)__popcll(mask & ((1ull << (tid & 63)) - 1));
        if (mine) s_id[place] = e.v;
        auto off = [&](float v) { return w.A == 0.0f ? 0.0f : entry(v, c, w.rest_top, w.A); };
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float z[N];
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = off(y[u].get(i));
            y[u].put(z);
            if (first + tid + 256 * u < end) store_vec(out + r.piece(first + tid + 256 * u), y[u].w);
        }
        if (s == 0 && tid < r.singles) out[r.single(tid)] = (E)off(single);
        // (every store before this is done before the next ones begin)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const float given = w.k * w.hard;
        if (mine) {
            bool lead = true;
            for (uint32_t i = 0; i < place; ++i) lead &= s_id[i] != e.v;
            if (lead) {
                out[e.v] = (E)(listed_entry(a, w, e.value, x, in.scale) - (e.v == label ? given : 0.0f));
                if (e.v == label) s_given = 1;
            }
        }
        __syncthreads();
        if (tid == 0 && at != -INFINITY && !s_given) out[label] = (E)(off(at) - given);
        __syncthreads();
    }
}

// ---------------------------------------------------------------- host

constexpr uint32_t kDistillGrid = 1u << 22;
constexpr uint64_t kDistillSlices = 1024;  // of few rows together

struct DistillCut {
    uint32_t S, W, G;
};
uint64_t most_rest_slices(uint64_t pieces) { return std::min<uint64_t>(64, (pieces + 511) / 512); }
DistillCut cut_distill(uint64_t rows, uint64_t vocab, uint32_t type)
{
    DistillCut r;
    const uint64_t pieces = vocab / (type == kF32 ? 4 : 8) + 1;
    const uint64_t want = kDistillSlices / std::min(rows, kDistillSlices);
    const uint64_t S = std::max<uint64_t>(1, std::min(most_rest_slices(pieces), want));
    r.W = (uint32_t)((pieces + S - 1) / S);
    r.S = (uint32_t)((pieces + r.W - 1) / r.W);
    r.G = (uint32_t)((pieces + 256 * kDistillU - 1) / (256 * kDistillU));
    return r;
}

struct DistillSpace {
    Part* part;
    DistillRow* terms;
};
DistillSpace carve_distill(void* ws, uint64_t rows, uint64_t parts, size_t* bytes)
{
    Carve c(ws);
    DistillSpace r;
    r.part = c.take<Part>(parts);
    r.terms = c.take<DistillRow>(rows);
    if (bytes) *bytes = c.used;
    return r;
}

}  // namespace

// (Enough for every type and every call of fewer rows, a smaller vocabulary or
// shorter lists.)
size_t distill_workspace(uint32_t, uint64_t rows, uint64_t vocab)
{
    size_t b = 0;
    const uint64_t parts = std::max(rows, std::min(kDistillSlices, rows * most_rest_slices(vocab / 4 + 1)));
    carve_distill(nullptr, rows, parts, &b);
    return b;
}

hipError_t distill_run(const Logits& in, const DistillArgs& a, float* div, float* stats, void* dlogits, uint64_t ldd,
                       void* ws, hipStream_t s)
{
    const DistillCut cut = cut_distill(in.rows, in.vocab, in.type);
    const DistillSpace sp = carve_distill(ws, in.rows, in.rows * cut.S, nullptr);
    const float c = in.scale * kLog2e;
    const uint32_t slices = (uint32_t)std::min<uint64_t>(in.rows * cut.S, kDistillGrid);
    const uint32_t rows = (uint32_t)std::min<uint64_t>(in.rows, kDistillGrid);
    const uint32_t grads = dlogits ? (uint32_t)std::min<uint64_t>(in.rows * cut.G, kDistillGrid) : 0;
    by_type(in.type, [&](auto ty) {
        constexpr int TY = decltype(ty)::value;
        timer_begin(kTLossRows, s);
        hipLaunchKernelGGL((k_rest_slices<TY>), dim3(slices), dim3(256), 0, s, in, a, cut.S, cut.W, c, sp.part);
        timer_end(kTLossRows, s);
        timer_begin(kTLossGrad, s);
        hipLaunchKernelGGL((k_distill_terms<TY>), dim3(rows), dim3(256), 0, s, in, a, cut.S, c, sp.part, sp.terms, div);
        hipLaunchKernelGGL((k_distill_grad<TY>), dim3(grads + 1), dim3(256), 0, s, in, a, cut.G, c, sp.terms, stats, dlogits,
                           ldd);
        timer_end(kTLossGrad, s);
    });
    return hipGetLastError();
}

}  // namespace sparcml
