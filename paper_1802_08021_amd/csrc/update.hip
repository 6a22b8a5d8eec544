// The update of Alg. 1 on gfx950: norm of a model's gradients, AdamW step
// over all its tensors, moments in 32 or in 8 bits.
//
// Both walk a list of pieces of 4096 elements that tensors_prepare_run lays out
// once, each with its tensor's addresses and rates: a workgroup knows what to do
// after one load, whatever the number and the lengths of the tensors, and one
// launch covers them all.  Both are bound by HBM: accesses are 16 bytes a lane (8 for
// 16-bit types of the step), marked nontemporal, and a piece of 32-bit moments
// begins at a line of its tensor (2^27 weights in 290 packed tensors: 725 us
// with pieces from the tensors' first elements, 655 to 667 so).
#include "internal.h"
#include "philox_device.h"
#include "types_device.h"

#include <algorithm>

namespace sparcml {
namespace {

// The pieces of tensor blockIdx.x.
__global__ void k_tensor_pieces(const TensorDesc* desc, TensorPiece* piece, uint32_t* ticket)
{
    const uint32_t t = blockIdx.x;
    if (t == 0 && threadIdx.x < kTickets) ticket[threadIdx.x * kTicketStride] = 0;
    TensorPiece p;
    p.d = desc[t];
    p.tensor = t;
    p.pad[0] = p.pad[1] = 0;
    const uint32_t pieces = p.d.n ? (uint32_t)((p.d.n + p.d.shift + kTensorChunk - 1) / kTensorChunk) : 0;
    for (p.index = threadIdx.x; p.index < pieces; p.index += blockDim.x) piece[p.d.first + p.index] = p;
}

// Element e of an array of n as fp32, zero outside it (e may lie before the
// array: below zero, as a large number).  Without a branch, so that the loads
// of a tensor's ends are under way together; n > 0.
template <class E>
__device__ __forceinline__ float get1(const E* p, uint64_t e, uint64_t n)
{
    const float x = (float)as_global(p)[e < n ? e : 0];
    return e < n ? x : 0.0f;
}

// Elements e .. e + 3 of an array of n, likewise.
template <int TYPE>
__device__ __forceinline__ f32x4 get4(const void* p, uint64_t e, uint64_t n)
{
    typedef typename Elem<TYPE>::type E;
    const E* q = static_cast<const E*>(p);
    if (e < n && e + 4 <= n) return __builtin_convertvector(load_vec<typename Elem<TYPE>::vec4>(q + e), f32x4);
    f32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = get1(q, e + i, n);
    return x;
}

// The same elements written, rounded to nearest where TYPE is narrower.
template <int TYPE>
__device__ __forceinline__ void put4(void* p, uint64_t e, uint64_t n, f32x4 x)
{
    typedef typename Elem<TYPE>::type E;
    E* q = static_cast<E*>(p) + e;
    if (e < n && e + 4 <= n) {
        store_vec(q, __builtin_convertvector(x, typename Elem<TYPE>::vec4));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e + i < n) as_global(q)[i] = (E)x[i];
    }
}

// Four codes as bytes of a word, zeros past the end.
__device__ __forceinline__ uint32_t get_codes(const void* p, uint64_t e, uint64_t n)
{
    const uint8_t* q = static_cast<const uint8_t*>(p);
    if (e + 4 <= n) return load_vec<uint32_t>(q + e);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = as_global(q)[e + i < n ? e + i : 0];
        w |= (e + i < n ? x : 0u) << (8 * i);
    }
    return w;
}

__device__ __forceinline__ void put_codes(void* p, uint64_t e, uint64_t n, uint32_t w)
{
    uint8_t* q = static_cast<uint8_t*>(p) + e;
    if (e + 4 <= n) {
        store_vec(q, w);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e + i < n) as_global(q)[i] = (uint8_t)(w >> (8 * i));
    }
}

__device__ __forceinline__ f32x4 decode4(uint32_t w, float scale)
{
    f32x4 x;
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0) * scale;
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * scale;
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * scale;
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * scale;
    return x;
}

// E4M3 codes of y, |y| <= 448: a code's neighbour above is taken when the
// value's bits below the code's last one and the draw's carry out of them
// (the conversion's stochastic form; the draw's 16 bits are its top ones).
__device__ __forceinline__ uint32_t encode4(f32x4 y, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3)
{
    int w = 0;
    w = __builtin_amdgcn_cvt_sr_fp8_f32(y[0], (int)r0, w, 0);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(y[1], (int)r1, w, 1);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(y[2], (int)r2, w, 2);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(y[3], (int)r3, w, 3);
    return (uint32_t)w;
}

// Biased exponent of the least power of two (at least 2^-100) that brings a
// block's largest magnitude to at most 448 = 1.75 * 2^8: the magnitude's own
// exponent less 8, one more above 1.75 * 2^e.
__device__ __forceinline__ uint32_t block_exponent(f32x4 x)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    const uint32_t e = (wave_max(top) + 0x1FFFFFu) >> 23;
    return max(e, 35u) - 8u;
}

// One AdamW step: a quarter of a piece a workgroup, four elements
// a lane, so that a wave holds exactly one block of the 8-bit form and its
// scale is one wave maximum.  Moments in 8 bits are rounded stochastically: the
// second one moves by 1 - beta2 of itself a step, far less than half a code, and
// rounding to nearest would hold it still.
// Bytes an element: 28 (32-bit moments, fp32 gradient) or 16 and 16/256 (8-bit).
// 20 M weights in 148 tensors, 32-bit: 91 to 95 us, 5.9 to 6.2 TB/s; 2^27 in 290, 8-bit:
// 387 to 395 us, 5.5 TB/s (a large copy: 6.2).  One vector a lane is the right size: with
// 4 vectors, before pieces began at lines, 2^27 took 838 us in 32 bits where one took
// 725, and 482 in 8 bits where one took 387 (more in flight, in less even order).  Without the generator, or with approximate roots and quotients, the
// 8-bit step is 2 to 3% faster, so neither is what bounds it.
template <int BITS, int GT, int CT>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(8)))
k_adamw(const TensorPiece* __restrict__ piece, uint64_t pieces, AdamwStep a, const float* __restrict__ clip)
{
    constexpr uint32_t kSub = kTensorChunk / 1024;
    float f = a.gs;
    if (clip) {
        const float c = clip[1];
        if (c == 0.0f) return;
        f = a.gs * c;
    }
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    for (uint64_t w = blockIdx.x; w < pieces * kSub; w += gridDim.x) {
        const TensorPiece at = piece[w / kSub];
        const TensorDesc& d = at.d;
        const float keep = (float)(1.0 - a.lr * (double)d.lr_scale * (double)d.decay);
        const float rate = (float)(a.rate * (double)d.lr_scale);
        // the wave's first element and the lane's (below zero: before the tensor)
        const uint64_t b = (uint64_t)at.index * kTensorChunk + (uint32_t)(w % kSub) * 1024 + (uint32_t)wv * 256 - d.shift;
        const uint64_t e = b + (uint32_t)lane * 4;
        if ((int64_t)b < (int64_t)d.n) {
            f32x4 p = get4<kF32>(d.param, e, d.n);
            const f32x4 g = get4<GT>(d.grad, e, d.n) * f;
            f32x4 m, v;
            if (BITS == 32) {
                m = get4<kF32>(d.m, e, d.n);
                v = get4<kF32>(d.v, e, d.n);
            } else {
                m = decode4(get_codes(d.m, e, d.n), as_global(d.m_scale)[b / kStateBlock]);
                v = decode4(get_codes(d.v, e, d.n), as_global(d.v_scale)[b / kStateBlock]);
                v = v * v;
            }
            m = a.b1 * m + a.omb1 * g;
            v = a.b2 * v + a.omb2 * (g * g);
            f32x4 r;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                r[i] = sqrtf(v[i]);  // (both correctly rounded)
                p[i] = p[i] * keep - rate * (m[i] / (r[i] * a.ibc2 + a.eps));
            }
            put4<kF32>(d.param, e, d.n, p);
            if (d.copy) put4<CT>(d.copy, e, d.n, p);
            if (BITS == 32) {
                put4<kF32>(d.m, e, d.n, m);
                put4<kF32>(d.v, e, d.n, v);
            } else {
                // lanes past the end hold zeros (of weights and states alike)
                const uint4 z = philox(make_uint4((uint32_t)(e >> 2), at.tensor, a.step, 0u), a.key0, a.key1);
                const uint32_t em = block_exponent(m), er = block_exponent(r);
                const f32x4 ym = m * __uint_as_float((254u - em) << 23);
                f32x4 yr = r * __uint_as_float((254u - er) << 23);
#pragma unroll
                for (int i = 0; i < 4; ++i) yr[i] = fmaxf(yr[i], 0x1p-9f);
                put_codes(d.m, e, d.n, encode4(ym, z.x << 16, z.y << 16, z.z << 16, z.w << 16));
                put_codes(d.v, e, d.n,
                          encode4(yr, z.x & 0xFFFF0000u, z.y & 0xFFFF0000u, z.z & 0xFFFF0000u, z.w & 0xFFFF0000u));
                if (lane == 0) {
                    as_global(d.m_scale)[b / kStateBlock] = __uint_as_float(em << 23);
                    as_global(d.v_scale)[b / kStateBlock] = __uint_as_float(er << 23);
                }
            }
        }
    }
}

__device__ __forceinline__ double block_sum(double x, double* s_w)
{
    for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = x;
    __syncthreads();
    return (s_w[0] + s_w[1]) + (s_w[2] + s_w[3]);
}

// Norm of all gradients: workgroup b sums the squares of pieces b, b + G, ...
// in fp64, the last workgroup to finish the partial sums, in their order (the
// same bits whichever it is).  2^27 in 290 tensors: fp32 81 us, 6.6 TB/s, bf16 43
// us (1024 workgroups; 94 and 48 with 2048, whose loads crowd the memory); 20 M
// bf16 in 148 tensors 10.4 us, where the chain piece, gradient and the last
// workgroup's sum count.
template <int GT>
__global__ void __launch_bounds__(256) k_norm(const TensorPiece* __restrict__ piece, uint64_t pieces, double* partial,
                                              uint32_t* ticket, double gs, double max_norm, float* out)
{
    __shared__ double s_w[4], s_end[4];
    __shared__ uint32_t s_last;
    double acc[2] = {0.0, 0.0};
    auto add = [&](const float* x, int n) {
#pragma unroll
        for (int i = 0; i < n; ++i) acc[i & 1] = fma((double)x[i], (double)x[i], acc[i & 1]);
    };
    constexpr int N = GT == kF32 ? 4 : 8, R = kTensorChunk / (256 * N);  // elements of 16 bytes; accesses a piece
    typedef typename Elem<GT>::type E;
    for (uint64_t c = blockIdx.x; c < pieces; c += gridDim.x) {
        const TensorPiece& at = piece[c];
        const E* grad = static_cast<const E*>(at.d.grad);
        const uint64_t n = at.d.n, e0 = (uint64_t)at.index * kTensorChunk - at.d.shift;
        if (e0 < n && e0 + kTensorChunk <= n) {  // a whole piece
            u32x4 w[R];
#pragma unroll
            for (int u = 0; u < R; ++u) w[u] = load_vec<u32x4>(grad + e0 + (threadIdx.x + u * 256) * N);
#pragma unroll
            for (int u = 0; u < R; ++u) {
                float x[N];
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = unpack<GT>(w[u], i);
                add(x, N);
            }
        } else {
            float x[kTensorChunk / 256];
#pragma unroll
            for (int i = 0; i < (int)kTensorChunk / 256; ++i) {
                x[i] = get1(grad, e0 + threadIdx.x + i * 256, n);
            }
            add(x, kTensorChunk / 256);
        }
    }
    const double sum = block_sum(acc[0] + acc[1], s_w);
    if (threadIdx.x == 0) {
        __hip_atomic_store(&partial[blockIdx.x], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        // Device-scope accesses only, each done before the next: they bypass
        // the XCDs' own L2s, which a fence would write back whole (22 ns a
        // workgroup); and a counter takes 12 ns an add, so the workgroups
        // count in groups and the groups' last ones in one.
        constexpr uint32_t kGroups = kTickets - 1;
        const uint32_t group = blockIdx.x % kGroups, size = (gridDim.x - group + kGroups - 1) / kGroups;
        uint32_t* mine = ticket + group * kTicketStride;
        uint32_t* top = ticket + kGroups * kTicketStride;
        bool last = false;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (atomicAdd(mine, 1u) == size - 1) {
            __hip_atomic_store(mine, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            last = atomicAdd(top, 1u) == min(gridDim.x, kGroups) - 1;
            if (last) __hip_atomic_store(top, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        s_last = last;
    }
    __syncthreads();
    if (!s_last) return;
    double all = 0.0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += 256)
        all += __hip_atomic_load(&partial[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    all = block_sum(all, s_end);
    if (threadIdx.x == 0) {
        const float norm = (float)(gs * sqrt(all));
        const float c = (float)(max_norm / ((double)norm + 1e-6));
        out[0] = norm;
        out[1] = isfinite(norm) ? fminf(1.0f, c) : 0.0f;
    }
}

template <int BITS, int GT, int CT>
void launch_adamw(const TensorTab& t, uint64_t pieces, const AdamwStep& a, const float* clip, hipStream_t s)
{
    const uint64_t grid = std::min<uint64_t>(pieces * (kTensorChunk / 1024), 1u << 22);
    hipLaunchKernelGGL((k_adamw<BITS, GT, CT>), dim3((uint32_t)grid), dim3(256), 0, s, t.piece, pieces, a, clip);
}

template <int BITS, int GT>
void launch_adamw(uint32_t ctype, const TensorTab& t, uint64_t pieces, const AdamwStep& a, const float* clip,
                  hipStream_t s)
{
    if (ctype == kF16)
        launch_adamw<BITS, GT, kF16>(t, pieces, a, clip, s);
    else
        launch_adamw<BITS, GT, kBf16>(t, pieces, a, clip, s);
}

template <int BITS>
void launch_adamw(uint32_t gtype, uint32_t ctype, const TensorTab& t, uint64_t pieces, const AdamwStep& a,
                  const float* clip, hipStream_t s)
{
    if (gtype == kF32)
        launch_adamw<BITS, kF32>(ctype, t, pieces, a, clip, s);
    else if (gtype == kBf16)
        launch_adamw<BITS, kBf16>(ctype, t, pieces, a, clip, s);
    else
        launch_adamw<BITS, kF16>(ctype, t, pieces, a, clip, s);
}

}  // namespace

TensorTab tensors_carve(void* ws, uint32_t count, uint64_t chunks, size_t* bytes)
{
    Carve c(ws);
    TensorTab t;
    t.desc = c.take<TensorDesc>(count);
    t.piece = c.take<TensorPiece>(chunks);
    t.partial = c.take<double>(kNormParts);
    t.ticket = c.take<uint32_t>(kTickets * kTicketStride);
    if (bytes) *bytes = c.used;
    return t;
}

hipError_t tensors_prepare_run(uint32_t count, const TensorDesc* host, uint64_t chunks, void* ws, hipStream_t s)
{
    const TensorTab t = tensors_carve(ws, count, chunks, nullptr);
    hipError_t e = upload(t.desc, host, count * sizeof(TensorDesc), s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_tensor_pieces, dim3(count), dim3(256), 0, s, t.desc, t.piece, t.ticket);
    return hipGetLastError();
}

hipError_t grad_norm_run(uint32_t count, uint64_t chunks, uint32_t gtype, double grad_scale, double max_norm,
                         float* out, void* ws, hipStream_t s)
{
    const TensorTab t = tensors_carve(ws, count, chunks, nullptr);
    const uint32_t parts = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(chunks, kNormParts));
    timer_begin(kTGradNorm, s);
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(parts), dim3(256), 0, s, t.piece, chunks, t.partial, t.ticket, grad_scale,
                           max_norm, out);
    };
    if (gtype == kF32)
        go(k_norm<kF32>);
    else if (gtype == kBf16)
        go(k_norm<kBf16>);
    else
        go(k_norm<kF16>);
    timer_end(kTGradNorm, s);
    return hipGetLastError();
}

hipError_t adamw_run(uint32_t count, uint64_t chunks, uint32_t gtype, uint32_t ctype, uint32_t bits,
                     const AdamwStep& a, const float* clip, void* ws, hipStream_t s)
{
    if (!chunks) return hipSuccess;
    const TensorTab t = tensors_carve(ws, count, chunks, nullptr);
    timer_begin(kTAdamw, s);
    if (bits == 32)
        launch_adamw<32>(gtype, ctype, t, chunks, a, clip, s);
    else
        launch_adamw<8>(gtype, ctype, t, chunks, a, clip, s);
    timer_end(kTAdamw, s);
    return hipGetLastError();
}

}  // namespace sparcml
