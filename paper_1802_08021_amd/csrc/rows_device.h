// Device helpers for operators over rows of logits: a row's pieces, parts of
// its sum, sums over a workgroup.
#pragma once

#include "internal.h"
#include "types_device.h"

#include <type_traits>

namespace sparcml {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
// c: the scale in powers of two, at most fp32's largest number (with an infinity
// equal logits, a difference of 0, would be NaN apart).
__host__ __device__ __forceinline__ float log2_scale(float scale)
{
    const float c = scale * kLog2e;
    return c < 3.402823466e38f ? c : 3.402823466e38f;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

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
    // From its first element on.
    __device__ __forceinline__ explicit RowCut(uint32_t V) : head(0), full(V / N), singles(V % N) {}
    __device__ __forceinline__ uint32_t piece(uint32_t j) const { return head + j * N; }
    __device__ __forceinline__ uint32_t single(uint32_t i) const { return i < head ? i : i + full * N; }
    __device__ __forceinline__ bool in_piece(uint32_t v) const { return v >= head && (v - head) / N < full; }
};
constexpr uint32_t kMinThreads = 128;  // a thread for each single

__device__ __forceinline__ bool has_token(const Logits& in, uint64_t t)
{
    return (uint32_t)in.label[t] < (uint32_t)in.vocab;
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

}  // namespace
}  // namespace sparcml
