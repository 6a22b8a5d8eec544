// Losses over rows of logits on gfx950: log probability of each row's token,
// clipped policy loss with a KL term, loss of paired log ratios, and their
// gradients.
//
// With x the row's logits, M their maximum, s the inverse temperature and
// Z = sum_v exp(s (x_v - M)): the token's log probability is s (x_label - M)
// - log Z, and for a loss whose derivative by it is q the gradient is
// s q ([v == label] - exp(s (x_v - M)) / Z).  A pass over the rows finds M and
// Z (one read, running maximum and sum), a second writes the gradient.  Rows
// are cut into slices, a workgroup each, whose (M, Z) are joined by whoever
// reads them.
#include "internal.h"
#include "types_device.h"

#include <algorithm>

namespace sparcml {
namespace {

constexpr uint32_t kStep = 2048;       // elements a workgroup takes at a time
constexpr float kLog2e = 1.44269504088896341f;

// Maximum of a part of a row and the sum of 2^(c (x - max)) over it;
// nothing (or nothing but -Inf): (-Inf, 0).
struct Part {
    float top, sum;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// What a part's sum counts for under the maximum `top`.
__device__ __forceinline__ float rescaled(Part p, float top, float c)
{
    return p.sum == 0.0f ? 0.0f : p.sum * exp2_fast((p.top - top) * c);
}

__device__ __forceinline__ Part join(Part a, Part b, float c)
{
    Part r;
    r.top = fmaxf(a.top, b.top);
    r.sum = rescaled(a, r.top, c) + rescaled(b, r.top, c);
    return r;
}

__device__ __forceinline__ Part join_slices(const Part* part, uint32_t S, float c)
{
    Part r = part[0];
    for (uint32_t i = 1; i < S; ++i) r = join(r, part[i], c);
    return r;
}

__device__ __forceinline__ bool has_token(const Logits& in, uint64_t t)
{
    return (uint32_t)in.label[t] < (uint32_t)in.vocab;
}

// Eight elements of a row from v on as fp32, -Inf past the end.
template <int TYPE>
__device__ __forceinline__ void get8(const typename Elem<TYPE>::type* row, uint64_t v, uint64_t end, float* x)
{
    if (v + 8 <= end) {
        const f32x4 a = __builtin_convertvector(load4<typename Elem<TYPE>::vec4>(row + v), f32x4);
        const f32x4 b = __builtin_convertvector(load4<typename Elem<TYPE>::vec4>(row + v + 4), f32x4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = a[i];
            x[4 + i] = b[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = v + i < end ? (float)row[v + i] : -INFINITY;
    }
}

// (M, Z) of every slice of every row in use; the token's logit beside them.
template <int TYPE>
__global__ void __launch_bounds__(256) k_rows(Logits in, const float* weight, uint32_t S, uint64_t W, float c,
                                              Part* part, float* at_label)
{
    typedef typename Elem<TYPE>::type E;
    __shared__ Part s_p[4];
    for (uint64_t b = blockIdx.x; b < in.rows * S; b += gridDim.x) {
        const uint64_t t = b / S, lo = (b % S) * W, end = min(lo + W, in.vocab);
        if (!has_token(in, t) || (weight && weight[t] == 0.0f)) continue;
        const E* row = static_cast<const E*>(in.x) + t * in.ld;
        Part p = {-INFINITY, 0.0f};
        for (uint64_t v = lo + threadIdx.x * 8; v < end; v += kStep) {
            float x[8];
            get8<TYPE>(row, v, end, x);
            float top = p.top;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, x[i]);
            const float base = top == -INFINITY ? 0.0f : top;
            float sum = p.sum * exp2_fast((p.top - base) * c);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += exp2_fast((x[i] - base) * c);
            p.top = top;
            p.sum = sum;
        }
        for (int o = 1; o < 64; o <<= 1) {
            const Part q = {__shfl_xor(p.top, o), __shfl_xor(p.sum, o)};
            p = join(p, q, c);
        }
        if ((threadIdx.x & 63) == 0) s_p[threadIdx.x >> 6] = p;
        __syncthreads();
        if (threadIdx.x == 0) {
            part[b] = join(join(s_p[0], s_p[1], c), join(s_p[2], s_p[3], c), c);
            if (lo == 0) at_label[t] = (float)row[in.label[t]];
        }
        __syncthreads();
    }
}

// Log probability and log sum of a row from its joined part.
__device__ __forceinline__ float row_logp(Part p, float x, float scale)
{
    return p.sum == 0.0f ? -INFINITY : (x - p.top) * scale - logf(p.sum);
}

__global__ void __launch_bounds__(256) k_logprob(Logits in, uint32_t S, float c, const Part* part,
                                                 const float* at_label, float* logp, float* lse)
{
    for (uint64_t t = (uint64_t)blockIdx.x * 256 + threadIdx.x; t < in.rows; t += (uint64_t)gridDim.x * 256) {
        float lp = 0.0f, l = 0.0f;
        if (has_token(in, t)) {
            const Part p = join_slices(part + t * S, S, c);
            lp = row_logp(p, at_label[t], in.scale);
            l = p.sum == 0.0f ? -INFINITY : p.top * in.scale + logf(p.sum);
        }
        logp[t] = lp;
        if (lse) lse[t] = l;
    }
}

// One token of the policy loss: its terms and the loss' derivative by its
// log probability (both before the weight).
struct PolicyToken {
    float gain, k, coef;
    bool clipped;
};
__device__ __forceinline__ PolicyToken policy_token(const PolicyArgs& a, uint64_t t, float lp)
{
    PolicyToken r;
    const float adv = a.adv[t], rho = expf(lp - a.old_logp[t]);
    const float u = rho * adv, held = fminf(fmaxf(rho, a.lo), a.hi) * adv;
    r.clipped = u > held;
    r.gain = r.clipped ? held : u;  // (a NaN of u comes through)
    r.k = 0.0f;
    r.coef = r.clipped ? 0.0f : -u;
    if (a.ref_logp) {
        const float far = a.ref_logp[t] - lp, em = expm1f(far);
        r.k = em - far;
        r.coef = r.coef - a.kl * em;
    }
    return r;
}

__device__ __forceinline__ double block_sum(double x, double* s_w)
{
    for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = x;
    __syncthreads();
    return (s_w[0] + s_w[1]) + (s_w[2] + s_w[3]);
}

// Elements [lo, end) of a gradient row: coef ([v == label] - 2^(c (x - M)) / Z),
// zeros where coef is 0 (the logits are then not read).
template <int TYPE>
__device__ __forceinline__ void grad_slice(const typename Elem<TYPE>::type* row, typename Elem<TYPE>::type* out,
                                           uint64_t lo, uint64_t end, uint32_t label, float coef, Part p, float c)
{
    typedef typename Elem<TYPE>::type E;
    typedef typename Elem<TYPE>::vec4 V;
    const bool none = coef == 0.0f || p.sum == 0.0f;
    const float k = -coef / p.sum;
    for (uint64_t v = lo + threadIdx.x * 8; v < end; v += kStep) {
        float x[8];
        if (none) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.0f;
        } else {
            get8<TYPE>(row, v, end, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = k * exp2_fast((x[i] - p.top) * c);
                if (v + i == label) x[i] += coef;
            }
        }
        if (v + 8 <= end) {
            const f32x4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
            store4(out + v, __builtin_convertvector(a, V));
            store4(out + v + 4, __builtin_convertvector(b, V));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (v + i < end) out[v + i] = (E)x[i];
        }
    }
}

// Workgroup 0: every token's log probability and the sums over tokens; the
// others a slice of the gradient each.
template <int TYPE>
__global__ void __launch_bounds__(256) k_policy(Logits in, PolicyArgs a, uint32_t S, uint64_t W, float c,
                                                const Part* part, const float* at_label, float* logp, float* stats,
                                                void* dlogits, uint64_t ldd)
{
    typedef typename Elem<TYPE>::type E;
    __shared__ double s_w[4];
    if (blockIdx.x == 0) {
        double gain = 0.0, k = 0.0, clipped = 0.0;
        for (uint64_t t = threadIdx.x; t < in.rows; t += 256) {
            const float w = a.weight[t];
            float lp = 0.0f;
            if (has_token(in, t) && w != 0.0f) {
                lp = row_logp(join_slices(part + t * S, S, c), at_label[t], in.scale);
                const PolicyToken r = policy_token(a, t, lp);
                gain += (double)w * (double)r.gain;
                k += (double)w * (double)r.k;
                clipped += r.clipped ? (double)w : 0.0;
            }
            logp[t] = lp;
        }
        gain = block_sum(gain, s_w);
        k = block_sum(k, s_w);
        clipped = block_sum(clipped, s_w);
        if (threadIdx.x == 0) {
            stats[0] = (float)((a.ref_logp ? (double)a.kl * k : 0.0) - gain);
            stats[1] = (float)-gain;
            stats[2] = (float)k;
            stats[3] = (float)clipped;
        }
        return;
    }
    for (uint64_t b = blockIdx.x - 1; b < in.rows * S; b += gridDim.x - 1) {
        const uint64_t t = b / S, lo = (b % S) * W, end = min(lo + W, in.vocab);
        const float w = a.weight[t];
        Part p = {0.0f, 0.0f};
        float coef = 0.0f;
        if (has_token(in, t) && w != 0.0f) {
            p = join_slices(part + t * S, S, c);
            coef = a.grad_scale * in.scale *
                   (w * policy_token(a, t, row_logp(p, at_label[t], in.scale)).coef);
        }
        grad_slice<TYPE>(static_cast<const E*>(in.x) + t * in.ld, static_cast<E*>(dlogits) + t * ldd, lo, end,
                         (uint32_t)in.label[t], coef, p, c);
    }
}

struct PairSums {
    double loss, won, good, bad;
};

// Pair blockIdx.x: rewards of its two sequences, loss, and the derivative by
// every token's log probability.
__global__ void __launch_bounds__(256) k_pairs(Logits in, PreferenceArgs a, uint32_t pairs, const uint32_t* bounds,
                                               uint32_t S, float c, const Part* part, const float* at_label,
                                               float* logp, float* coef, PairSums* sums)
{
    __shared__ double s_w[4];
    const uint32_t b = blockIdx.x;
    const uint32_t lo = bounds[2 * b], mid = bounds[2 * b + 1], end = bounds[2 * b + 2];
    double good = 0.0, bad = 0.0;
    for (uint64_t t = (uint64_t)lo + threadIdx.x; t < end; t += 256) {
        float lp = 0.0f;
        if (has_token(in, t)) {
            lp = row_logp(join_slices(part + t * S, S, c), at_label[t], in.scale);
            const double r = (double)lp - (a.ref_logp ? (double)a.ref_logp[t] : 0.0);
            (t < mid ? good : bad) += r;
        }
        logp[t] = lp;
    }
    good = (double)a.beta * block_sum(good, s_w);
    bad = (double)a.beta * block_sum(bad, s_w);
    const double h = good - bad, z = exp(-fabs(h)), soft = log1p(z);
    const double up = h >= 0.0 ? 1.0 / (1.0 + z) : z / (1.0 + z);    // sigmoid(h)
    const double down = h >= 0.0 ? z / (1.0 + z) : 1.0 / (1.0 + z);  // sigmoid(-h)
    const double eps = (double)a.smoothing;
    const float q = (float)((double)a.beta * (eps * up - (1.0 - eps) * down) / (double)pairs);
    for (uint64_t t = (uint64_t)lo + threadIdx.x; t < end; t += 256)
        coef[t] = has_token(in, t) ? (t < mid ? q : -q) : 0.0f;
    if (threadIdx.x == 0) {
        PairSums r;
        r.loss = (1.0 - eps) * (soft - fmin(h, 0.0)) + eps * (soft + fmax(h, 0.0));
        r.won = h > 0.0 ? 1.0 : 0.0;
        r.good = good;
        r.bad = bad;
        sums[b] = r;
    }
}

// Workgroup 0: the sums over pairs; the others a slice of the gradient each.
template <int TYPE>
__global__ void __launch_bounds__(256) k_preference(Logits in, PreferenceArgs a, uint32_t pairs, uint32_t S,
                                                    uint64_t W, float c, const Part* part, const float* coef,
                                                    const PairSums* sums, float* stats, void* dlogits, uint64_t ldd)
{
    typedef typename Elem<TYPE>::type E;
    __shared__ double s_w[4];
    if (blockIdx.x == 0) {
        double loss = 0.0, won = 0.0, good = 0.0, bad = 0.0;
        for (uint32_t i = threadIdx.x; i < pairs; i += 256) {
            loss += sums[i].loss;
            won += sums[i].won;
            good += sums[i].good;
            bad += sums[i].bad;
        }
        loss = block_sum(loss, s_w);
        won = block_sum(won, s_w);
        good = block_sum(good, s_w);
        bad = block_sum(bad, s_w);
        if (threadIdx.x == 0) {
            stats[0] = (float)(loss / pairs);
            stats[1] = (float)(won / pairs);
            stats[2] = (float)(good / pairs);
            stats[3] = (float)(bad / pairs);
        }
        return;
    }
    for (uint64_t b = blockIdx.x - 1; b < in.rows * S; b += gridDim.x - 1) {
        const uint64_t t = b / S, lo = (b % S) * W, end = min(lo + W, in.vocab);
        Part p = {0.0f, 0.0f};
        const float q = a.grad_scale * in.scale * coef[t];
        if (q != 0.0f) p = join_slices(part + t * S, S, c);
        grad_slice<TYPE>(static_cast<const E*>(in.x) + t * in.ld, static_cast<E*>(dlogits) + t * ldd, lo, end,
                         (uint32_t)in.label[t], q, p, c);
    }
}

// Slices a row: enough workgroups for the chip when there are few rows, none
// shorter than two steps of a workgroup.
struct Cut {
    uint32_t S;
    uint64_t W;
    uint32_t grid;
};
Cut cut_rows(uint64_t rows, uint64_t vocab)
{
    Cut r;
    const uint64_t most = (vocab + 2 * kStep - 1) / (2 * kStep), want = (1024 + rows - 1) / rows;
    uint64_t S = std::max<uint64_t>(1, std::min(most, want));
    r.W = ((vocab + S - 1) / S + kStep - 1) / kStep * kStep;
    r.S = (uint32_t)((vocab + r.W - 1) / r.W);
    r.grid = (uint32_t)std::min<uint64_t>(rows * r.S, 1u << 22);
    return r;
}

struct Space {
    Part* part;
    float *at_label, *coef;
    PairSums* sums;
    uint32_t* bounds;
};
Space carve(void* ws, uint64_t rows, const Cut& cut, uint32_t pairs, size_t* bytes)
{
    Carve c(ws);
    Space r;
    r.part = c.take<Part>(rows * cut.S);
    r.at_label = c.take<float>(rows);
    r.coef = c.take<float>(pairs ? rows : 0);
    r.sums = c.take<PairSums>(pairs);
    r.bounds = c.take<uint32_t>(pairs ? 2 * (uint64_t)pairs + 1 : 0);
    if (bytes) *bytes = c.used;
    return r;
}

hipError_t rows_run(const Logits& in, const float* weight, const Cut& cut, const Space& sp, float c, hipStream_t s)
{
    timer_begin(kTLossRows, s);
    if (in.type == kF32)
        hipLaunchKernelGGL((k_rows<kF32>), dim3(cut.grid), dim3(256), 0, s, in, weight, cut.S, cut.W, c, sp.part, sp.at_label);
    else if (in.type == kBf16)
        hipLaunchKernelGGL((k_rows<kBf16>), dim3(cut.grid), dim3(256), 0, s, in, weight, cut.S, cut.W, c, sp.part, sp.at_label);
    else
        hipLaunchKernelGGL((k_rows<kF16>), dim3(cut.grid), dim3(256), 0, s, in, weight, cut.S, cut.W, c, sp.part, sp.at_label);
    timer_end(kTLossRows, s);
    return hipGetLastError();
}

}  // namespace

size_t logprob_workspace(uint64_t rows, uint64_t vocab)
{
    size_t b;
    carve(nullptr, rows, cut_rows(rows, vocab), 0, &b);
    return b;
}
size_t policy_workspace(uint64_t rows, uint64_t vocab) { return logprob_workspace(rows, vocab); }
size_t preference_workspace(uint32_t pairs, uint64_t rows, uint64_t vocab)
{
    size_t b;
    carve(nullptr, rows, cut_rows(rows, vocab), pairs, &b);
    return b;
}

hipError_t logprob_run(const Logits& in, float* logp, float* lse, void* ws, hipStream_t s)
{
    const Cut cut = cut_rows(in.rows, in.vocab);
    const Space sp = carve(ws, in.rows, cut, 0, nullptr);
    const float c = in.scale * kLog2e;
    hipError_t e = rows_run(in, nullptr, cut, sp, c, s);
    if (e != hipSuccess) return e;
    const uint32_t grid = (uint32_t)std::min<uint64_t>((in.rows + 255) / 256, 4096);
    hipLaunchKernelGGL(k_logprob, dim3(grid), dim3(256), 0, s, in, cut.S, c, sp.part, sp.at_label, logp, lse);
    return hipGetLastError();
}

hipError_t policy_run(const Logits& in, const PolicyArgs& a, float* logp, float* stats, void* dlogits, uint64_t ldd,
                      void* ws, hipStream_t s)
{
    const Cut cut = cut_rows(in.rows, in.vocab);
    const Space sp = carve(ws, in.rows, cut, 0, nullptr);
    const float c = in.scale * kLog2e;
    hipError_t e = rows_run(in, a.weight, cut, sp, c, s);
    if (e != hipSuccess) return e;
    const dim3 grid(dlogits ? cut.grid + 1 : 1);
    timer_begin(kTLossGrad, s);
    if (in.type == kF32)
        hipLaunchKernelGGL((k_policy<kF32>), grid, dim3(256), 0, s, in, a, cut.S, cut.W, c, sp.part, sp.at_label, logp, stats, dlogits, ldd);
    else if (in.type == kBf16)
        hipLaunchKernelGGL((k_policy<kBf16>), grid, dim3(256), 0, s, in, a, cut.S, cut.W, c, sp.part, sp.at_label, logp, stats, dlogits, ldd);
    else
        hipLaunchKernelGGL((k_policy<kF16>), grid, dim3(256), 0, s, in, a, cut.S, cut.W, c, sp.part, sp.at_label, logp, stats, dlogits, ldd);
    timer_end(kTLossGrad, s);
    return hipGetLastError();
}

hipError_t preference_run(const Logits& in, const PreferenceArgs& a, uint32_t pairs, const uint32_t* bounds,
                          float* logp, float* stats, void* dlogits, uint64_t ldd, void* ws, hipStream_t s)
{
    const Cut cut = cut_rows(in.rows, in.vocab);
    const Space sp = carve(ws, in.rows, cut, pairs, nullptr);
    const float c = in.scale * kLog2e;
    hipError_t e = rows_run(in, nullptr, cut, sp, c, s);
    if (e == hipSuccess) e = upload(sp.bounds, bounds, (2 * (size_t)pairs + 1) * sizeof(uint32_t), s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_pairs, dim3(pairs), dim3(256), 0, s, in, a, pairs, sp.bounds, cut.S, c, sp.part, sp.at_label, logp, sp.coef, sp.sums);
    const dim3 grid(dlogits ? cut.grid + 1 : 1);
    timer_begin(kTLossGrad, s);
    if (in.type == kF32)
        hipLaunchKernelGGL((k_preference<kF32>), grid, dim3(256), 0, s, in, a, pairs, cut.S, cut.W, c, sp.part, sp.coef, sp.sums, stats, dlogits, ldd);
    else if (in.type == kBf16)
        hipLaunchKernelGGL((k_preference<kBf16>), grid, dim3(256), 0, s, in, a, pairs, cut.S, cut.W, c, sp.part, sp.coef, sp.sums, stats, dlogits, ldd);
    else
        hipLaunchKernelGGL((k_preference<kF16>), grid, dim3(256), 0, s, in, a, pairs, cut.S, cut.W, c, sp.part, sp.coef, sp.sums, stats, dlogits, ldd);
    timer_end(kTLossGrad, s);
    return hipGetLastError();
}

}  // namespace sparcml
