// Kernels over a list of tensors: global norm of the gradients, clipping, AdamW (see include/fastsnarf_train.h).
//
// All of them read the list from device memory and cut it into units of UNIT elements of one tensor, numbered through the list.  Every
// block takes one stretch of consecutive units, finds the tensor that it begins in, and walks on from tensor to tensor.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fs {

constexpr int UNIT = 2048;             // elements: 8 per thread
constexpr int TRAIN_BLOCKS = 4096;     // at most; a partial sum for each
constexpr int TICKET_GROUPS = 32, TICKET_STRIDE = 64;      // counters of last_block, each on lines of its own
constexpr int TICKETS = (1 + TICKET_GROUPS) * TICKET_STRIDE;

enum { TYPE_F32, TYPE_BF16, TYPE_F16 };
enum { KIND_TWO, KIND_MAX };

struct TensorD {                       // a tensor as the kernels see it, n > 0
    void *grad, *out, *param;
    float *master, *m, *v;
    long long n;
    int first;                         // its first unit
    int types;                         // of the gradients | of the parameters << 8
    float lr_scale, decay_scale;
};

struct ListD {
    const TensorD *tensors;
    const int *first;                  // [count + 1] first units, ascending: first[count] = units
    int count, units;
};

constexpr int PUT = 40;                // tensors that one launch of k_list_put carries in its arguments (3.2 KB of 4)
struct PutD { TensorD t[PUT]; };

// The list travels in kernel arguments: in the stream's order, without host memory that has to outlive the call, and as part of a captured graph.
__global__ __launch_bounds__(64) void k_list_put(PutD p, int at, int n, int count, int units, TensorD *__restrict__ tensors, int *__restrict__ first)
{
    const int i = threadIdx.x;
    if (i < n) {
        tensors[at + i] = p.t[i];
        first[at + i] = p.t[i].first;
    }
    if (i == 0 && at + n == count) first[count] = units;
}

__global__ void k_tickets_clear(unsigned *tickets)
{
    for (int i = threadIdx.x; i < TICKETS; i += blockDim.x) tickets[i] = 0u;
}

// ---- elements, four or eight at a time, aligned to the element only ----
// Pointers come out of the list, so the compiler is told that they are global memory: it would use flat instructions, which wait for LDS too.
#define FS_GLOBAL __attribute__((address_space(1)))
template <class T> using Global = FS_GLOBAL T *;
template <class T> __device__ __forceinline__ Global<T> global(void *p) { return (Global<T>)p; }

template <class T, int N> struct VecOf { typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T)))); };

template <class T, int N>
__device__ __forceinline__ void load(Global<T> p, float (&x)[N])
{
    const typename VecOf<T, N>::type v = *(const FS_GLOBAL typename VecOf<T, N>::type *)p;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)v[i];
}

template <class T, int N>
__device__ __forceinline__ void store(Global<T> p, const float (&x)[N])
{
    typename VecOf<T, N>::type v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (T)x[i];
    *(FS_GLOBAL typename VecOf<T, N>::type *)p = v;
}

// the first `n` of N elements, zeros behind
template <class T, int N>
__device__ __forceinline__ void load_some(Global<T> p, int n, float (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = 0.0f;
        if (i < n) x[i] = (float)p[i];
    }
}

template <class T, int N>
__device__ __forceinline__ void store_some(Global<T> p, int n, const float (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) p[i] = (T)x[i];
}

// ---- the walk over the list ----

// The tensor that unit u belongs to: every round, the wave's 64 lanes ask at 64 places of what is left.
__device__ __forceinline__ int find_tensor(const ListD &L, int u)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = L.count;
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lane * step;
        const bool at_or_before = i < n && L.first[lo + i] <= u;
        const int k = __popcll(__ballot(at_or_before)) - 1;       // lane 0 always says yes
        lo += k * step;
        n = min(step, n - k * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Calls f(tensor, begin, end) for the elements [begin, end) of every tensor that this block's stretch of units covers; begin is a multiple of UNIT.
template <class F>
__device__ __forceinline__ void walk(const ListD &L, F f)
{
    const int b = blockIdx.x, G = gridDim.x;
    int u = (int)((long long)L.units * b / G);
    const int end = (int)((long long)L.units * (b + 1) / G);
    if (u >= end) return;
    for (int i = find_tensor(L, u); u < end; ++i) {
        const TensorD t = L.tensors[i];
        const long long begin = (long long)(u - t.first) * UNIT, upto = (long long)(end - t.first) * UNIT;
        f(t, begin, upto < t.n ? upto : t.n);
        u = t.first + (int)((t.n + UNIT - 1) / UNIT);
    }
}

// ---- sums over a block, and over the blocks ----
__device__ __forceinline__ double join(double a, double b) { return a + b; }
__device__ __forceinline__ unsigned join(unsigned a, unsigned b) { return a > b ? a : b; }

// result in thread 0; every thread of the block calls it
template <class S>
__device__ __forceinline__ S block_join(S s)
{
    __shared__ S wave[4];
#pragma unroll
    for (int d = 32; d; d >>= 1) s = join(s, __shfl_xor(s, d));
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = s;
    __syncthreads();
    return join(join(wave[0], wave[1]), join(wave[2], wave[3]));
}

// True in every thread of the block that comes last, when all threads of all blocks have come here.  Blocks count themselves in groups, the last
// of a group counts it at the top: one counter serves a block in some 10 ns, so 2048 blocks that end together would stand 20 us in line at a
// single one.  The counters are 0 between kernels.  What a block leaves for the last one it stores with agent-scope atomics, which go past the caches;
// they are done when vmcnt is 0.  (A release at agent scope would write the whole L2 back and an acquire drop it, some 25 ns a block of 50 us in all.)
__device__ __forceinline__ unsigned count_in(unsigned *counter, unsigned of)
{
    const unsigned before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before != of - 1) return 0;
    __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return 1;
}

__device__ __forceinline__ bool last_block(unsigned *tickets)
{
    __shared__ unsigned last;
    __syncthreads();
    if (threadIdx.x == 0) {
        __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const unsigned groups = min((unsigned)TICKET_GROUPS, gridDim.x), mine = blockIdx.x % groups;
        last = count_in(tickets + (1 + mine) * TICKET_STRIDE, (gridDim.x - mine + groups - 1) / groups);
        if (last) last = count_in(tickets, groups);
    }
    __syncthreads();
    return last;
}

// ---- global norm ----

// Squares are added in 64 bits: fp32 gradients of any size neither overflow nor vanish, and the sum over 10^9 elements loses nothing.
// The largest magnitude is that of the bits without the sign, as integers: NaN is above infinity.
template <int KIND> struct Sum;
template <> struct Sum<KIND_TWO> {
    using type = double;
    static __device__ __forceinline__ double add(double s, float x) { return __builtin_fma((double)x, (double)x, s); }
    static __device__ __forceinline__ double value(double s) { return __builtin_sqrt(s); }
};
template <> struct Sum<KIND_MAX> {
    using type = unsigned;
    static __device__ __forceinline__ unsigned add(unsigned s, float x) { return join(s, __float_as_uint(x) & 0x7fffffffu); }
    static __device__ __forceinline__ double value(unsigned s) { return (double)__uint_as_float(s); }
};

template <int KIND, class T, class S>
__device__ __forceinline__ S sum_range(Global<T> g, long long begin, long long end, S s)
{
    constexpr int N = 16 / sizeof(T);                      // elements of one load
    for (long long at = begin; at < end; at += UNIT)
#pragma unroll
        for (int k = 0; k < UNIT; k += 256 * N) {
            const long long i = at + k + threadIdx.x * N;
            float x[N];
            if (i + N <= end) load<T, N>(g + i, x);
            else load_some<T, N>(g + i, (int)(end > i ? end - i : 0), x);
#pragma unroll
            for (int e = 0; e < N; ++e) s = Sum<KIND>::add(s, x[e]);
        }
    return s;
}

template <int KIND>
__global__ __launch_bounds__(256) void k_norm(ListD L, double scale, double *__restrict__ partial, unsigned *__restrict__ tickets, float *__restrict__ norm)
{
    using S = typename Sum<KIND>::type;
    S s = 0;
    walk(L, [&](const TensorD &t, long long begin, long long end) {
        switch (t.types & 255) {
        case TYPE_F32: s = sum_range<KIND>(global<float>(t.grad), begin, end, s); break;
        case TYPE_BF16: s = sum_range<KIND>(global<__bf16>(t.grad), begin, end, s); break;
        default: s = sum_range<KIND>(global<_Float16>(t.grad), begin, end, s); break;
        }
    });
    s = block_join(s);
    S *part = reinterpret_cast<S *>(partial);
    if (threadIdx.x == 0) __hip_atomic_store(part + blockIdx.x, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!last_block(tickets)) return;
    s = 0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += 256) s = join(s, __hip_atomic_load(part + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    s = block_join(s);
    if (threadIdx.x == 0) *norm = (float)(Sum<KIND>::value(s) * scale);
}

// ---- clipping ----

// s min(1, max_norm / (norm + 1e-6)), NaN for a norm that is NaN
__device__ __forceinline__ float clip_coef(const float *norm, double max_norm, double scale)
{
    if (max_norm == __builtin_inf()) return (float)scale;
    const double q = max_norm / ((double)*norm + 1e-6);
    return (float)((q >= 1.0 ? 1.0 : q) * scale);
}

template <class T>
__device__ __forceinline__ void scale_range(Global<T> g, Global<T> out, long long begin, long long end, float coef)
{
    constexpr int N = 16 / sizeof(T);
    for (long long at = begin; at < end; at += UNIT)
#pragma unroll
        for (int k = 0; k < UNIT; k += 256 * N) {
            const long long i = at + k + threadIdx.x * N;
            const int some = (int)(end - i < N ? end - i : N);
            float x[N];
            if (some == N) load<T, N>(g + i, x);
            else load_some<T, N>(g + i, some, x);
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] *= coef;
            if (some == N) store<T, N>(out + i, x);
            else store_some<T, N>(out + i, some, x);
        }
}

__global__ __launch_bounds__(256) void k_clip(ListD L, double max_norm, double scale, const float *__restrict__ norm)
{
    const float coef = clip_coef(norm, max_norm, scale);
    walk(L, [&](const TensorD &t, long long begin, long long end) {
        if (t.out == t.grad && coef == 1.0f) return;
        switch (t.types & 255) {
        case TYPE_F32: scale_range(global<float>(t.grad), global<float>(t.out), begin, end, coef); break;
        case TYPE_BF16: scale_range(global<__bf16>(t.grad), global<__bf16>(t.out), begin, end, coef); break;
        default: scale_range(global<_Float16>(t.grad), global<_Float16>(t.out), begin, end, coef); break;
        }
    });
}

// ---- AdamW ----

struct AdamD {
    double log_beta1, log_beta2, max_norm, scale;
    float lr, beta1, beta2, rest1, rest2, eps, decay;      // rest = 1 - beta, rounded once
    int skip_nonfinite;
};

// 1 - exp(y) for y <= 0 in 64 bits: y = k ln 2 + r, |r| <= ln 2 / 2, and the series of exp(r) - 1 up to r^13 / 13! (the rest is below 2^-58).
// For k = 0 nothing cancels, so 1 - beta^t of the first steps keeps its digits.
__device__ __forceinline__ double one_minus_exp(double y)
{
    y = y < -700.0 ? -700.0 : y;
    const double k = __builtin_rint(y * 1.4426950408889634);
    const double r = __builtin_fma(k, -1.9082149292705877e-10, __builtin_fma(k, -0.69314718036912382, y));      // ln 2 in two parts
    double e = 1.0;
#pragma unroll
    for (int n = 13; n >= 2; --n) e = __builtin_fma(e, r * (1.0 / n), 1.0);
    e *= r;
    const double p = __builtin_ldexp(1.0, (int)k);
    return -__builtin_fma(p, e, p - 1.0);
}

struct AdamC { float coef, lr, inv1, inv_sqrt2; };          // of this step

template <class P, class G, bool MASTER>
__device__ __forceinline__ void adam_range(const TensorD &t, long long begin, long long end, const AdamD &A, const AdamC &C)
{
    constexpr int N = 4;                                   // fp32 moments: 16 bytes of each
    const Global<G> grad = global<G>(t.grad);
    const Global<P> param = global<P>(t.param);
    const Global<float> tm = global<float>(t.m), tv = global<float>(t.v), master = global<float>(t.master);
    const float lr = C.lr * t.lr_scale, fade = lr * (A.decay * t.decay_scale), step = lr * C.inv1;
    for (long long at = begin; at < end; at += UNIT)
#pragma unroll
        for (int k = 0; k < UNIT; k += 256 * N) {
            const long long i = at + k + threadIdx.x * N;
            const int some = (int)(end - i < N ? end - i : N);
            if (some <= 0) continue;
            float g[N], p[N], m[N], v[N];
            if (some == N) {
                load<G, N>(grad + i, g);
                load<float, N>(tm + i, m);
                load<float, N>(tv + i, v);
                if (MASTER) load<float, N>(master + i, p);
                else load<P, N>(param + i, p);
            } else {
                load_some<G, N>(grad + i, some, g);
                load_some<float, N>(tm + i, some, m);
                load_some<float, N>(tv + i, some, v);
                if (MASTER) load_some<float, N>(master + i, some, p);
                else load_some<P, N>(param + i, some, p);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float x = g[e] * C.coef;
                m[e] = __builtin_fmaf(A.beta1, m[e], A.rest1 * x);
                v[e] = __builtin_fmaf(A.beta2, v[e], A.rest2 * x * x);
                p[e] -= __builtin_fmaf(fade, p[e], step * m[e] / __builtin_fmaf(__builtin_sqrtf(v[e]), C.inv_sqrt2, A.eps));
            }
            if (some == N) {
                store<float, N>(tm + i, m);
                store<float, N>(tv + i, v);
                if (MASTER) store<float, N>(master + i, p);
                store<P, N>(param + i, p);
            } else {
                store_some<float, N>(tm + i, some, m);
                store_some<float, N>(tv + i, some, v);
                if (MASTER) store_some<float, N>(master + i, some, p);
                store_some<P, N>(param + i, some, p);
            }
        }
}

template <class P, class G>
__device__ __forceinline__ void adam_tensor(const TensorD &t, long long begin, long long end, const AdamD &A, const AdamC &C)
{
    if (t.master) adam_range<P, G, true>(t, begin, end, A, C);
    else adam_range<P, G, false>(t, begin, end, A, C);
}

template <class P>
__device__ __forceinline__ void adam_types(const TensorD &t, long long begin, long long end, const AdamD &A, const AdamC &C)
{
    switch (t.types & 255) {
    case TYPE_F32: adam_tensor<P, float>(t, begin, end, A, C); break;
    case TYPE_BF16: adam_tensor<P, __bf16>(t, begin, end, A, C); break;
    default: adam_tensor<P, _Float16>(t, begin, end, A, C); break;
    }
}

__global__ __launch_bounds__(256) void k_adamw(ListD L, AdamD A, const float *__restrict__ lr, const float *__restrict__ norm,
                                               long long *__restrict__ steps, unsigned *__restrict__ tickets)
{
    if (A.skip_nonfinite && !(__builtin_fabsf(*norm) < __builtin_inff())) return;      // every block sees the same norm
    const long long before = *steps;
    const double time = (double)(before + 1);
    AdamC C;
    C.coef = clip_coef(norm, A.max_norm, A.scale);
    C.lr = lr ? *lr : A.lr;
    C.inv1 = (float)(1.0 / one_minus_exp(time * A.log_beta1));
    C.inv_sqrt2 = (float)(1.0 / __builtin_sqrt(one_minus_exp(time * A.log_beta2)));
    walk(L, [&](const TensorD &t, long long begin, long long end) {
        switch (t.types >> 8) {
        case TYPE_F32: adam_types<float>(t, begin, end, A, C); break;
        case TYPE_BF16: adam_types<__bf16>(t, begin, end, A, C); break;
        default: adam_types<_Float16>(t, begin, end, A, C); break;
        }
    });
    // the counter moves on when every block has read it
    if (last_block(tickets) && threadIdx.x == 0) *steps = before + 1;
}

}  // namespace fs
