// Kernels over a list of tensors: global norm of the gradients, clipping, AdamW (see include/fastsnarf_train.h).
//
// All of them read the list from device memory and cut it into units of UNIT elements of one tensor, numbered through the list.  Blocks
// take chunks of consecutive units in turn, find the tensor that a chunk begins in, and walk on from tensor to tensor.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fs {

constexpr int UNIT = 2048;             // elements: 8 per thread
constexpr int TRAIN_BLOCKS = 4096;     // at most; a partial sum for each
constexpr int LIST_LDS = 1024;          // places that a block keeps in LDS
constexpr int TICKET_GROUPS = 32, TICKET_STRIDE = 64;      // counters of last_block, each on lines of its own
constexpr int TICKETS = (1 + TICKET_GROUPS) * TICKET_STRIDE;

enum { TYPE_F32, TYPE_BF16, TYPE_F16 };
enum { KIND_TWO, KIND_MAX };

struct TensorD {                       // a tensor as the kernels see it, n > 0
    void *grad, *out, *param;
    float *master, *m, *v;
    long long n;
    int first, next;                   // its first unit, and the first of the tensor behind it
    int lead;                          // its first unit begins so many elements before the tensor, where memory is aligned
    int types;                         // of the gradients | of the parameters << 8
    float lr_scale, decay_scale;
};

struct ListD {
    const TensorD *tensors;
    const int *first;                  // [count] first units, ascending
    int count, units;
    int chunk;                         // units that a block takes at a time
};

constexpr int PUT = 40;                // tensors that one launch of k_list_put carries in its arguments (3.2 KB of 4)
struct PutD { TensorD t[PUT]; };

// The list travels in kernel arguments: in the stream's order, without host memory that has to outlive the call, and as part of a captured graph.
__global__ __launch_bounds__(64) void k_list_put(PutD p, int at, int n, TensorD *__restrict__ tensors, int *__restrict__ first)
{
    const int i = threadIdx.x;
    if (i >= n) return;
    tensors[at + i] = p.t[i];
    first[at + i] = p.t[i].first;
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
template <class T, int N> using Vec = typename VecOf<T, N>::type;

// STREAM: past the caches as far as that goes, for data that no later kernel finds there
template <bool STREAM, class T, int N>
__device__ __forceinline__ Vec<T, N> load(Global<T> p)
{
    const FS_GLOBAL Vec<T, N> *at = (const FS_GLOBAL Vec<T, N> *)p;
    return STREAM ? __builtin_nontemporal_load(at) : *at;
}

template <bool STREAM, class T, int N>
__device__ __forceinline__ void store(Global<T> p, Vec<T, N> v)
{
    FS_GLOBAL Vec<T, N> *at = (FS_GLOBAL Vec<T, N> *)p;
    if (STREAM) __builtin_nontemporal_store(v, at);
    else *at = v;
}

// ---- the walk over the list ----

// The tensor that unit u belongs to: every round, the wave's 64 lanes ask at 64 places of what is left.
template <class First>
__device__ __forceinline__ int find_tensor(First first, int count, int u)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = count;
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lane * step;
        const bool at_or_before = i < n && first[lo + i] <= u;
        const int k = __popcll(__ballot(at_or_before)) - 1;       // lane 0 always says yes
        lo += k * step;
        n = min(step, n - k * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// A tensor, by scalar loads: the list does not change while a kernel reads it.
__device__ __forceinline__ TensorD tensor_at(const ListD &L, int i)
{
    typedef const __attribute__((address_space(4))) TensorD *Constant;
    const Constant c = (Constant)L.tensors + i;
    return {c->grad, c->out, c->param, c->master, c->m, c->v, c->n, c->first, c->next, c->lead, c->types, c->lr_scale, c->decay_scale};
}

// A part of a tensor: elements [begin, end), of which those before 0 are not there (begin < 0 in a first unit with a lead).
struct Piece { long long begin, end; };

// Calls f(tensor, piece) for what this block's chunks of units cover of every tensor.  The next piece's tensor is found and asked for before
// the present piece is worked on.  BACK: the last chunk first.
template <bool BACK, class F>
__device__ __forceinline__ void walk(const ListD &L, F f)
{
    const int chunks = (int)(((long long)L.units + L.chunk - 1) / L.chunk);
    int c = blockIdx.x;
    if (c >= chunks) return;
    const bool kept = (int)gridDim.x < chunks && L.count <= LIST_LDS;      // several chunks: the places are asked for more than once
    __shared__ int s_first[LIST_LDS];
    if (kept) {
        for (int i = threadIdx.x; i < L.count; i += 256) s_first[i] = L.first[i];
        __syncthreads();
    }
    auto find = [&](int u) { return kept ? find_tensor(s_first, L.count, u) : find_tensor(L.first, L.count, u); };
    int u = (BACK ? chunks - 1 - c : c) * L.chunk, end = min(u + L.chunk, L.units), i = find(u);
    TensorD t = tensor_at(L, i);
    for (;;) {
        const long long upto = (long long)(end - t.first) * UNIT - t.lead;
        const Piece p = {(long long)(u - t.first) * UNIT - t.lead, upto < t.n ? upto : t.n};
        u = t.next;
        bool more = u < end;
        if (more) ++i;
        else {
            c += gridDim.x;
            more = c < chunks;
            if (more) {
                u = (BACK ? chunks - 1 - c : c) * L.chunk;
                end = min(u + L.chunk, L.units);
                i = find(u);
            }
        }
        const TensorD next = more ? tensor_at(L, i) : t;
        f(t, p);
        if (!more) return;
        t = next;
    }
}

// A piece in vectors of N elements.  Those at the tensor's ends that are not whole are left out; their elements, fewer than 2 N, are `edge`'s, one to a thread.
template <int N>
struct Vectors {
    int from, upto;                    // whole vectors, numbered from the piece's begin
    int heads, edges;                  // elements before them, and in all
    long long tail;                    // the first element behind them
    __device__ __forceinline__ explicit Vectors(const Piece &p)
    {
        const int before = p.begin < 0 ? (int)-p.begin : 0;
        const int there = (int)(p.end - p.begin);
        from = (before + N - 1) / N;
        upto = there / N;
        heads = min(from * N, there) - before;
        if (upto < from) upto = from;
        tail = p.begin + (long long)upto * N;
        edges = heads + (tail < p.end ? (int)(p.end - tail) : 0);
    }
    // the element of this thread, which is < edges
    __device__ __forceinline__ long long edge() const { return (int)threadIdx.x < heads ? (long long)threadIdx.x : tail + ((int)threadIdx.x - heads); }
};

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

// AHEAD loads of 16 bytes in every thread on their way.
#ifndef AHEAD_N
#define AHEAD_N 4
#define AHEAD_C 2
#define AHEAD_A 1
#endif
template <int KIND, bool STREAM, class T, class S>
__device__ __forceinline__ S sum_piece(Global<T> g, const Piece &p, S s)
{
    constexpr int N = 16 / sizeof(T), AHEAD = AHEAD_N;
    const Vectors<N> V(p);
    g += p.begin;
    Vec<T, N> x[AHEAD];
    auto add = [&](int k) {
#pragma unroll
        for (int e = 0; e < N; ++e) s = Sum<KIND>::add(s, (float)x[k][e]);
    };
    for (int j = 0; j < V.upto; j += 256 * AHEAD) {
        const int mine = j + threadIdx.x;
        if (j >= V.from && j + 256 * AHEAD <= V.upto) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) x[k] = load<STREAM, T, N>(g + (mine + k * 256) * N);
        } else {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                x[k] = (T)0.0f;
                if (mine + k * 256 >= V.from && mine + k * 256 < V.upto) x[k] = load<STREAM, T, N>(g + (mine + k * 256) * N);
            }
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) add(k);
    }
    if ((int)threadIdx.x < V.edges) s = Sum<KIND>::add(s, (float)g[V.edge() - p.begin]);
    return s;
}

template <int KIND, bool STREAM>
__global__ __launch_bounds__(256) void k_norm(ListD L, double scale, double *__restrict__ partial, unsigned *__restrict__ tickets, float *__restrict__ norm)
{
    using S = typename Sum<KIND>::type;
    S s = 0;
    walk<false>(L, [&](const TensorD &t, const Piece &p) {
        switch (t.types & 255) {
        case TYPE_F32: s = sum_piece<KIND, STREAM>(global<float>(t.grad), p, s); break;
        case TYPE_BF16: s = sum_piece<KIND, STREAM>(global<__bf16>(t.grad), p, s); break;
        default: s = sum_piece<KIND, STREAM>(global<_Float16>(t.grad), p, s); break;
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

template <bool STREAM, class T>
__device__ __forceinline__ void scale_piece(Global<T> g, Global<T> out, const Piece &p, float coef)
{
    constexpr int N = 16 / sizeof(T), AHEAD = AHEAD_C;
    const Vectors<N> V(p);
    g += p.begin;
    out += p.begin;
    Vec<T, N> x[AHEAD];
    auto scale = [&](int k) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[k][e] = (T)((float)x[k][e] * coef);
    };
    for (int j = 0; j < V.upto; j += 256 * AHEAD) {
        const int mine = j + threadIdx.x;
        if (j >= V.from && j + 256 * AHEAD <= V.upto) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) x[k] = load<STREAM, T, N>(g + (mine + k * 256) * N);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                scale(k);
                store<STREAM, T, N>(out + (mine + k * 256) * N, x[k]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (mine + k * 256 >= V.from && mine + k * 256 < V.upto) x[k] = load<STREAM, T, N>(g + (mine + k * 256) * N);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (mine + k * 256 >= V.from && mine + k * 256 < V.upto) {
                    scale(k);
                    store<STREAM, T, N>(out + (mine + k * 256) * N, x[k]);
                }
        }
    }
    if ((int)threadIdx.x < V.edges) {
        const long long i = V.edge() - p.begin;
        out[i] = (T)((float)g[i] * coef);
    }
}

template <bool STREAM>
__global__ __launch_bounds__(256) void k_clip(ListD L, double max_norm, double scale, const float *__restrict__ norm)
{
    const float coef = clip_coef(norm, max_norm, scale);
    walk<true>(L, [&](const TensorD &t, const Piece &p) {
        if (t.out == t.grad && coef == 1.0f) return;
        switch (t.types & 255) {
        case TYPE_F32: scale_piece<STREAM>(global<float>(t.grad), global<float>(t.out), p, coef); break;
        case TYPE_BF16: scale_piece<STREAM>(global<__bf16>(t.grad), global<__bf16>(t.out), p, coef); break;
        default: scale_piece<STREAM>(global<_Float16>(t.grad), global<_Float16>(t.out), p, coef); break;
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

// What a thread holds of one place: N elements of every array.
template <class P, class G, bool MASTER, int N>
struct Place {
    Vec<G, N> g;
    Vec<float, N> m, v, w;
    Vec<P, N> p;
};

struct AdamT { float coef, fade, step, inv_sqrt2, beta1, beta2, rest1, rest2, eps; };      // of one tensor

template <class P, class G, bool MASTER>
struct Arrays {
    Global<G> g;
    Global<P> p;
    Global<float> m, v, w;

    template <bool STREAM, int N>
    __device__ __forceinline__ void get(long long i, Place<P, G, MASTER, N> &x) const
    {
        x.g = load<STREAM, G, N>(g + i);
        x.m = load<STREAM, float, N>(m + i);
        x.v = load<STREAM, float, N>(v + i);
        if (MASTER) x.w = load<STREAM, float, N>(w + i);
        else x.p = load<STREAM, P, N>(p + i);
    }
    // Everything in fp32; the parameter in 16 bits is rounded once, from the new value.
    template <bool STREAM, int N>
    __device__ __forceinline__ void update(long long i, Place<P, G, MASTER, N> &x, const AdamT &A) const
    {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float g = (float)x.g[e] * A.coef, p = MASTER ? x.w[e] : (float)x.p[e];
            const float m = __builtin_fmaf(A.beta1, x.m[e], A.rest1 * g), v = __builtin_fmaf(A.beta2, x.v[e], A.rest2 * g * g);
            const float now = p - __builtin_fmaf(A.fade, p, A.step * m / __builtin_fmaf(__builtin_sqrtf(v), A.inv_sqrt2, A.eps));
            x.m[e] = m;
            x.v[e] = v;
            if (MASTER) x.w[e] = now;
            x.p[e] = (P)now;
        }
        store<STREAM, float, N>(m + i, x.m);
        store<STREAM, float, N>(v + i, x.v);
        if (MASTER) store<STREAM, float, N>(w + i, x.w);
        store<STREAM, P, N>(p + i, x.p);
    }
};

template <bool STREAM, class P, class G, bool MASTER>
__device__ __forceinline__ void adam_piece(const TensorD &t, const Piece &piece, const AdamT &A)
{
    constexpr int N = 4, AHEAD = AHEAD_A;
    const Vectors<N> V(piece);
    const long long at = piece.begin;
    const Arrays<P, G, MASTER> a = {global<G>(t.grad) + at, global<P>(t.param) + at, global<float>(t.m) + at, global<float>(t.v) + at, global<float>(t.master) + at};
    Place<P, G, MASTER, N> x[AHEAD];
    for (int j = 0; j < V.upto; j += 256 * AHEAD) {
        const int mine = j + threadIdx.x;
        if (j >= V.from && j + 256 * AHEAD <= V.upto) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) a.template get<STREAM>((mine + k * 256) * N, x[k]);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) a.template update<STREAM>((mine + k * 256) * N, x[k], A);
        } else {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (mine + k * 256 >= V.from && mine + k * 256 < V.upto) {
                    a.template get<STREAM>((mine + k * 256) * N, x[k]);
                    a.template update<STREAM>((mine + k * 256) * N, x[k], A);
                }
        }
    }
    if ((int)threadIdx.x < V.edges) {
        Place<P, G, MASTER, 1> y;
        a.template get<false>(V.edge() - at, y);
        a.template update<false>(V.edge() - at, y, A);
    }
}

template <bool STREAM, class P, class G>
__device__ __forceinline__ void adam_master(const TensorD &t, const Piece &p, const AdamT &A)
{
    if (t.master) adam_piece<STREAM, P, G, true>(t, p, A);
    else adam_piece<STREAM, P, G, false>(t, p, A);
}

template <bool STREAM, class P>
__device__ __forceinline__ void adam_grad(const TensorD &t, const Piece &p, const AdamT &A)
{
    switch (t.types & 255) {
    case TYPE_F32: adam_master<STREAM, P, float>(t, p, A); break;
    case TYPE_BF16: adam_master<STREAM, P, __bf16>(t, p, A); break;
    default: adam_master<STREAM, P, _Float16>(t, p, A); break;
    }
}

template <bool STREAM>
__global__ __launch_bounds__(256) void k_adamw(ListD L, AdamD A, const float *__restrict__ lr_word, const float *__restrict__ norm,
                                               long long *__restrict__ steps, unsigned *__restrict__ tickets)
{
    if (A.skip_nonfinite && !(__builtin_fabsf(*norm) < __builtin_inff())) return;      // every block sees the same norm
    const long long before = *steps;
    const double time = (double)(before + 1);
    const float coef = clip_coef(norm, A.max_norm, A.scale), rate = lr_word ? *lr_word : A.lr;
    const float inv1 = (float)(1.0 / one_minus_exp(time * A.log_beta1));
    const float inv_sqrt2 = (float)(1.0 / __builtin_sqrt(one_minus_exp(time * A.log_beta2)));
    walk<true>(L, [&](const TensorD &t, const Piece &p) {
        const float lr = rate * t.lr_scale;
        const AdamT T = {coef, lr * (A.decay * t.decay_scale), lr * inv1, inv_sqrt2, A.beta1, A.beta2, A.rest1, A.rest2, A.eps};
        switch (t.types >> 8) {
        case TYPE_F32: adam_grad<STREAM, float>(t, p, T); break;
        case TYPE_BF16: adam_grad<STREAM, __bf16>(t, p, T); break;
        default: adam_grad<STREAM, _Float16>(t, p, T); break;
        }
    });
    // the counter moves on when every block has read it
    if (last_block(tickets) && threadIdx.x == 0) *steps = before + 1;
}

}  // namespace fs
