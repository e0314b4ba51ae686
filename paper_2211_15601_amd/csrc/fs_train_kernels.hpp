// Kernels over a list of tensors: global norm of the gradients, clipping, AdamW (see include/fastsnarf_train.h).
//
// All of them read the list from device memory and cut it into units of UNIT elements of one tensor, numbered through the list.  Blocks
// take chunks of consecutive units in turn, find the tensor that a chunk begins in, and walk on from tensor to tensor: one launch, and even shares, whatever the
// number and the sizes of the tensors.  Every element is used once, so memory bounds all of it, and launches where there is little: what counts is how many
// bytes are on their way, in which order blocks go through the arrays (chunks in turn, not a stretch for each block: 1 GB read at 7.2 against 6.1 TB/s, copied at 6.1
// against 5.0), what goes past the caches, and how short the chains of dependent loads at a kernel's two ends are.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fs {

constexpr int UNIT = 2048;             // elements: 8 per thread
constexpr int TRAIN_BLOCKS = 2048;     // of k_norm at most; a partial sum for each
constexpr int SHORT_PART = 256;        // elements that a wave of a short list's second pass takes at a time
constexpr int LIST_LDS = 1024;         // places that a block keeps in LDS
constexpr int TICKET_GROUPS = 32, TICKET_STRIDE = 64;      // counters of take_ticket, each on lines of its own
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
    int chunks;                        // parts that blocks take in turn, alike to a unit: part c begins at unit c step / 2^STEP_BITS
    long long step;
};

constexpr int STEP_BITS = 20;
__host__ __device__ inline int chunk_begin(const ListD &L, int c) { const long long u = c * L.step >> STEP_BITS; return u < L.units ? (int)u : L.units; }

constexpr int PUT = 40;                // tensors that one launch of k_list_put carries in its arguments (3.2 KB of 4)
struct PutD { TensorD t[PUT]; };

// The list travels in kernel arguments: in the stream's order, without host memory that has to outlive the call, and as part of a captured graph.
// There it runs at every replay, and so does the clearing of the counters (`tickets`, or NULL), which would take a launch of its own some 2 us.
__global__ __launch_bounds__(64) void k_list_put(PutD p, int at, int n, TensorD *__restrict__ tensors, int *__restrict__ first, unsigned *__restrict__ tickets)
{
    const int i = threadIdx.x;
    if (tickets)
        for (int k = i; k < TICKETS; k += 64) tickets[k] = 0u;
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
__device__ __forceinline__ Piece piece_of(const TensorD &t, long long from, long long upto) { return {from - t.lead, min(upto - t.lead, t.n)}; }

// This block's way through the list: chunk after chunk, tensor after tensor.  Made early, so that the first tensor is on its way while the kernel gets its norm.
// BACK: the last chunk first.
template <bool BACK>
struct Walk {
    const ListD &L;
    const int *kept;                   // the places in LDS, where they are asked for more than once
    int c, u, end, i;                  // chunk, unit, first unit behind the chunk, tensor
    TensorD t;

    __device__ __forceinline__ explicit Walk(const ListD &list) : L(list), kept(nullptr), c(blockIdx.x)
    {
        __shared__ int s_first[LIST_LDS];
        if ((int)gridDim.x < L.chunks && L.count <= LIST_LDS) {
            for (int k = threadIdx.x; k < L.count; k += 256) s_first[k] = L.first[k];
            __syncthreads();
            kept = s_first;
        }
        if (c < L.chunks) {
            go();
            t = tensor_at(L, i);
        }
    }
    __device__ __forceinline__ void go()
    {
        const int at = BACK ? L.chunks - 1 - c : c;
        u = chunk_begin(L, at);
        end = chunk_begin(L, at + 1);
        i = kept ? find_tensor((const __attribute__((address_space(3))) int *)kept, L.count, u) : find_tensor(L.first, L.count, u);
    }
    // Calls f(tensor, piece, chunk) for what the block's chunks cover of every tensor.  The next piece's tensor is found and asked for before the present
    // piece is worked on.
    template <class F>
    __device__ __forceinline__ void each(F f)
    {
        while (c < L.chunks) {
            const Piece p = piece_of(t, (long long)(u - t.first) * UNIT, (long long)(end - t.first) * UNIT);
            const int now = c;
            u = t.next;
            if (u < end) ++i;
            else {
                c += gridDim.x;
                if (c < L.chunks) go();
            }
            const TensorD next = c < L.chunks ? tensor_at(L, i) : t;
            f(t, p, now);
            t = next;
        }
    }
};

// The same for short lists, a wave by itself: parts of PART elements, dealt out to `waves` waves of which this is number `wave`.
template <int PART, class F>
__device__ __forceinline__ void walk_short(const ListD &L, int wave, int waves, F f)
{
    constexpr int PARTS = UNIT / PART;
    for (int c = wave; c < L.units * PARTS; c += waves) {
        const TensorD t = tensor_at(L, find_tensor(L.first, L.count, c / PARTS));
        const long long at = (long long)(c / PARTS - t.first) * UNIT + c % PARTS * PART;
        const Piece p = piece_of(t, at, at + PART);
        if (p.begin < p.end && p.end > 0) f(t, p);
    }
}

// A piece in vectors of N elements, worked on by TEAM threads of which this is number `rank`.  Vectors at the tensor's ends that are not whole are left out;
// their elements, fewer than 2 N, are the edges, one to a thread.
template <int N, int TEAM>
struct Vectors {
    int from, upto;                    // whole vectors, numbered from the piece's begin
    int rank;
    bool edge;                         // this thread has an edge
    int at;                            // that element, from the piece's begin
    __device__ __forceinline__ explicit Vectors(const Piece &p) : rank(threadIdx.x & (TEAM - 1))
    {
        static_assert(2 * N <= TEAM, "an edge a thread");
        const int before = p.begin < 0 ? (int)-p.begin : 0, there = (int)(p.end - p.begin);
        from = (before + N - 1) / N;
        upto = max(from, there / N);
        const int heads = min(from * N, there) - before;
        at = rank < heads ? before + rank : upto * N + (rank - heads);
        edge = at < there;
    }
    // Calls f(first vector of this thread, all of its vectors are there) for every AHEAD * TEAM vectors; it has k * TEAM more behind it, see has().
    template <int AHEAD, class F>
    __device__ __forceinline__ void each(F f) const
    {
        for (int j = 0; j < upto; j += TEAM * AHEAD) f(j + rank, j >= from && j + TEAM * AHEAD <= upto);
    }
    __device__ __forceinline__ bool has(int j) const { return j >= from && j < upto; }
};

// ---- sums over a block, and over the blocks ----
__device__ __forceinline__ double join(double a, double b) { return a + b; }
__device__ __forceinline__ unsigned join(unsigned a, unsigned b) { return a > b ? a : b; }

// result in every thread; every thread of the block calls it
template <int WAVES, class S>
__device__ __forceinline__ S block_join(S s)
{
    __shared__ S wave[WAVES];
#pragma unroll
    for (int d = 32; d; d >>= 1) s = join(s, __shfl_xor(s, d));
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = s;
    __syncthreads();
    s = wave[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) s = join(s, wave[i]);
    return s;
}

// Which block comes last?  Blocks count themselves in groups, the last of a group counts it at the top: one counter serves a block in some 10 ns,
// so 1024 blocks that end together would stand 10 us in line at a single one.  The counters are 0 between kernels.  A release or acquire at agent scope would
// write the whole L2 back or drop it, 50 us with 2048 blocks; what a block leaves for the last one it stores with agent-scope atomics, which go past the
// caches, and has done so when vmcnt is 0.
struct Ticket { unsigned *counter; unsigned before, of; };

__device__ __forceinline__ unsigned count_in(unsigned *counter) { return __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// By one thread of a block, when all that the block does before the last one goes on is done.
__device__ __forceinline__ Ticket take_ticket(unsigned *tickets)
{
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const bool few = gridDim.x <= 2 * TICKET_GROUPS;
    const unsigned mine = blockIdx.x % TICKET_GROUPS;
    unsigned *counter = few ? tickets : tickets + (1 + mine) * TICKET_STRIDE;
    return {counter, count_in(counter), few ? gridDim.x : (gridDim.x - mine + TICKET_GROUPS - 1) / TICKET_GROUPS};
}

// By the same thread, then or later: is it the last block's?
__device__ __forceinline__ bool is_last(const Ticket &t, unsigned *tickets)
{
    if (t.before != t.of - 1) return false;
    __hip_atomic_store(t.counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (t.counter == tickets) return true;
    if (count_in(tickets) != TICKET_GROUPS - 1) return false;
    __hip_atomic_store(tickets, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
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

// AHEAD: loads of 16 bytes of an array that every thread has on their way.
constexpr int AHEAD_NORM = 4, AHEAD_CLIP = 2, AHEAD_ADAMW = 1;

template <int KIND, bool STREAM, int TEAM, int AHEAD, class T, class S>
__device__ __forceinline__ S sum_piece(Global<T> g, const Piece &p, S s)
{
    constexpr int N = 16 / sizeof(T);
    const Vectors<N, TEAM> V(p);
    g += p.begin;
    float edge = 0.0f;
    if (V.edge) edge = (float)g[V.at];
    V.template each<AHEAD>([&](int j, bool all) {
        Vec<T, N> x[AHEAD];
        if (all) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) x[k] = load<STREAM, T, N>(g + (j + k * TEAM) * N);
        } else {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                x[k] = (T)0.0f;
                if (V.has(j + k * TEAM)) x[k] = load<STREAM, T, N>(g + (j + k * TEAM) * N);
            }
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int e = 0; e < N; ++e) s = Sum<KIND>::add(s, (float)x[k][e]);
    });
    return Sum<KIND>::add(s, edge);
}

template <int KIND, bool STREAM, int TEAM, int AHEAD, class S>
__device__ __forceinline__ S sum_types(const TensorD &t, const Piece &p, S s)
{
    switch (t.types & 255) {
    case TYPE_F32: return sum_piece<KIND, STREAM, TEAM, AHEAD>(global<float>(t.grad), p, s);
    case TYPE_BF16: return sum_piece<KIND, STREAM, TEAM, AHEAD>(global<__bf16>(t.grad), p, s);
    default: return sum_piece<KIND, STREAM, TEAM, AHEAD>(global<_Float16>(t.grad), p, s);
    }
}

// Sums that blocks have left, joined by every thread's block in the same order.
template <class S>
__device__ __forceinline__ S join_parts(const S *part, int n)
{
    S s = 0;
    for (int i = threadIdx.x; i < n; i += 256) s = join(s, __hip_atomic_load(part + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    return block_join<4>(s);
}

// s sqrt(sum g^2) or s max |g|: each thread adds up what it reads, a block's waves join by shuffles and LDS, the block that comes last joins the blocks' sums, every
// time in the same order.  Bound by reading: 400 M fp32 in 226 us (7.1 TB/s), 45 M bf16 in 300 tensors 20 us (4.5, of which some 5 us are the two ends).  With the
// 64-bit sums it issues 3 instructions an element in fp32 and 5 in 16 bits, a seventh and a quarter of the time.
// The first `streamed` chunks are read past the caches, the others stay there for a pass that comes from the other end.
// norm == NULL: the blocks' sums stay in `partial`, and every block of the kernel behind this one joins them for itself (see norm_value()).
template <int KIND>
__global__ __launch_bounds__(256) void k_norm(ListD L, int streamed, double scale, double *__restrict__ partial, unsigned *__restrict__ tickets, float *__restrict__ norm)
{
    using S = typename Sum<KIND>::type;
    S s = 0;
    Walk<false>(L).each([&](const TensorD &t, const Piece &p, int c) {
        s = c < streamed ? sum_types<KIND, true, 256, AHEAD_NORM>(t, p, s) : sum_types<KIND, false, 256, AHEAD_NORM>(t, p, s);
    });
    s = block_join<4>(s);
    S *part = reinterpret_cast<S *>(partial);
    __shared__ bool last;
    if (threadIdx.x == 0) {
        __hip_atomic_store(part + blockIdx.x, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = norm && is_last(take_ticket(tickets), tickets);
    }
    __syncthreads();
    if (!last) return;
    s = join_parts(part, gridDim.x);
    if (threadIdx.x == 0) *norm = (float)(Sum<KIND>::value(s) * scale);
}

// Where a kernel gets the norm from: `parts` sums of k_norm, which it joins and writes to `norm`; or, parts == 0, from `norm` (NULL: nothing asks for it).
struct NormD {
    const double *partial;
    int parts, kind;
    double scale;
    float *norm;
};

// In 64 bits for what is made of it; only what is written out is rounded.
__device__ __forceinline__ double norm_value(const NormD &N)
{
    if (N.parts == 0) return N.norm ? (double)*N.norm : 0.0;
    const double v = N.kind == KIND_TWO ? Sum<KIND_TWO>::value(join_parts(N.partial, N.parts))
                                        : Sum<KIND_MAX>::value(join_parts(reinterpret_cast<const unsigned *>(N.partial), N.parts));
    const double n = v * N.scale;
    if (blockIdx.x == 0 && threadIdx.x == 0) *N.norm = (float)n;
    return n;
}

// ---- short lists ----
// Every block adds up the whole list, the same way, and needs to hear of no other: a list of SHORT_UNITS units is two trips to memory for its 16 waves.  One launch in
// place of two, and no counters: bound by the launch and the chain of loads (place, tensor, elements).  8 k elements: norm 3.0 us, clipping 4.4, AdamW 5.8.
constexpr int SHORT_THREADS = 1024, SHORT_WAVES = SHORT_THREADS / 64;
template <int KIND>
__device__ __forceinline__ double short_norm(const ListD &L, double scale)
{
    typename Sum<KIND>::type s = 0;
    walk_short<UNIT>(L, threadIdx.x >> 6, SHORT_WAVES, [&](const TensorD &t, const Piece &p) { s = sum_types<KIND, false, 64, 8>(t, p, s); });
    return Sum<KIND>::value(block_join<SHORT_WAVES>(s)) * scale;
}

template <int KIND>
__global__ __launch_bounds__(SHORT_THREADS) void k_norm_short(ListD L, double scale, float *__restrict__ norm)
{
    const double n = short_norm<KIND>(L, scale);
    if (threadIdx.x == 0) *norm = (float)n;
}

// ---- clipping ----

// s min(1, max_norm / (norm + 1e-6)), NaN for a norm that is NaN; rounded once.  (From a norm of 32 bits it would be off by about twice as much, and
// gradients whose norm 32 bits cannot hold would become zeros.)
__device__ __forceinline__ float clip_coef(double norm, double max_norm, double scale)
{
    if (max_norm == __builtin_inf()) return (float)scale;
    const double q = max_norm / (norm + 1e-6);
    return (float)((q >= 1.0 ? 1.0 : q) * scale);
}

template <bool STREAM, int TEAM, int AHEAD, class T>
__device__ __forceinline__ void scale_piece(Global<T> g, Global<T> out, const Piece &p, float coef)
{
    constexpr int N = 16 / sizeof(T);
    const Vectors<N, TEAM> V(p);
    g += p.begin;
    out += p.begin;
    V.template each<AHEAD>([&](int j, bool all) {
        Vec<T, N> x[AHEAD];
        auto get = [&](int k) { x[k] = load<STREAM, T, N>(g + (j + k * TEAM) * N); };
        auto put = [&](int k) {
#pragma unroll
            for (int e = 0; e < N; ++e) x[k][e] = (T)((float)x[k][e] * coef);
            store<STREAM, T, N>(out + (j + k * TEAM) * N, x[k]);
        };
        if (all) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) get(k);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) put(k);
        } else {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (V.has(j + k * TEAM)) get(k);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (V.has(j + k * TEAM)) put(k);
        }
    });
    if (V.edge) out[V.at] = (T)((float)g[V.at] * coef);
}

template <bool STREAM, int TEAM, int AHEAD>
__device__ __forceinline__ void scale_types(const TensorD &t, const Piece &p, float coef)
{
    if (t.out == t.grad && coef == 1.0f) return;
    switch (t.types & 255) {
    case TYPE_F32: scale_piece<STREAM, TEAM, AHEAD>(global<float>(t.grad), global<float>(t.out), p, coef); break;
    case TYPE_BF16: scale_piece<STREAM, TEAM, AHEAD>(global<__bf16>(t.grad), global<__bf16>(t.out), p, coef); break;
    default: scale_piece<STREAM, TEAM, AHEAD>(global<_Float16>(t.grad), global<_Float16>(t.out), p, coef); break;
    }
}

// Chunks from the list's end, where the norm has left gradients in the caches.  Bound by reading and writing: 250 M fp32 in 345 us (2 GB, 5.8 TB/s) behind
// 150 us of norm.
template <bool STREAM>
__global__ __launch_bounds__(256) void k_clip(ListD L, NormD N, int all_in_place, double max_norm, double scale)
{
    const float coef = clip_coef(norm_value(N), max_norm, scale);
    if (all_in_place && coef == 1.0f) return;              // what most steps end with: nothing is asked for before it is known
    Walk<true>(L).each([&](const TensorD &t, const Piece &p, int) { scale_types<STREAM, 256, AHEAD_CLIP>(t, p, coef); });
}

// Not in place: a block may have written while another still adds up.
template <int KIND>
__global__ __launch_bounds__(SHORT_THREADS) void k_clip_short(ListD L, double max_norm, double scale, float *__restrict__ norm)
{
    const double n = short_norm<KIND>(L, scale);
    const float coef = clip_coef(n, max_norm, scale);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    walk_short<SHORT_PART>(L, blockIdx.x * SHORT_WAVES + (threadIdx.x >> 6), gridDim.x * SHORT_WAVES, [&](const TensorD &t, const Piece &p) { scale_types<false, 64, 1>(t, p, coef); });
}

// ---- AdamW ----

struct AdamD {
    double log_beta1, log_beta2, max_norm, scale;
    float lr, beta1, beta2, rest1, rest2, eps, decay;      // rest = 1 - beta, rounded once
    int skip_nonfinite;
};

// 1 - exp(y) for y <= 0 in 64 bits: y = k ln 2 + r, |r| <= ln 2 / 2, and the series of exp(r) - 1 up to r^13 / 13! (the rest is below 2^-57).  ln 2 in two
// parts after Cody and Waite (1980): the double next to it, and the one next to what that leaves; each product is exact inside its fused multiply-add.
// For k = 0 nothing cancels, so 1 - beta^t of the first steps keeps its digits.  Off by less than 2 units in the last place (20000 values against 60 digits).
__device__ __forceinline__ double one_minus_exp(double y)
{
    y = y < -700.0 ? -700.0 : y;
    const double k = __builtin_rint(y * 1.4426950408889634);
    const double r = __builtin_fma(k, -2.3190468138462996e-17, __builtin_fma(k, -0.6931471805599453, y));
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

// What goes past the caches: nothing; all but the parameters, which the next forward pass reads; or all.
enum { ADAM_CACHED, ADAM_PARAM, ADAM_STREAM };

struct AdamT { float coef, fade, step, inv_sqrt2, beta1, beta2, rest1, rest2, eps; };      // of one tensor

template <class P, class G, bool MASTER>
struct Arrays {
    Global<G> g;
    Global<P> p;
    Global<float> m, v, w;

    template <int MODE, int N>
    __device__ __forceinline__ void get(long long i, Place<P, G, MASTER, N> &x) const
    {
        constexpr bool STREAM = MODE != ADAM_CACHED;
        x.g = load<STREAM, G, N>(g + i);
        x.m = load<STREAM, float, N>(m + i);
        x.v = load<STREAM, float, N>(v + i);
        if (MASTER) x.w = load<STREAM, float, N>(w + i);
        else x.p = load<STREAM, P, N>(p + i);
    }
    // Everything in fp32; the parameter in 16 bits is rounded once, from the new value.
    template <int MODE, int N>
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
        constexpr bool STREAM = MODE != ADAM_CACHED;
        store<STREAM, float, N>(m + i, x.m);
        store<STREAM, float, N>(v + i, x.v);
        if (MASTER) store<STREAM, float, N>(w + i, x.w);
        store<MODE == ADAM_STREAM, P, N>(p + i, x.p);
    }
};

template <int MODE, int TEAM, int AHEAD, class P, class G, bool MASTER>
__device__ __forceinline__ void adam_piece(const TensorD &t, const Piece &p, const AdamT &A)
{
    constexpr int N = 4;                                   // 16 bytes of every fp32 array
    const Vectors<N, TEAM> V(p);
    const Arrays<P, G, MASTER> a = {global<G>(t.grad) + p.begin, global<P>(t.param) + p.begin, global<float>(t.m) + p.begin, global<float>(t.v) + p.begin,
                                    global<float>(t.master) + p.begin};
    V.template each<AHEAD>([&](int j, bool all) {
        Place<P, G, MASTER, N> x[AHEAD];
        if (all) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) a.template get<MODE>((j + k * TEAM) * N, x[k]);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) a.template update<MODE>((j + k * TEAM) * N, x[k], A);
        } else {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (V.has(j + k * TEAM)) {
                    a.template get<MODE>((j + k * TEAM) * N, x[k]);
                    a.template update<MODE>((j + k * TEAM) * N, x[k], A);
                }
        }
    });
    if (V.edge) {
        Place<P, G, MASTER, 1> y;
        a.template get<ADAM_CACHED>(V.at, y);
        a.template update<ADAM_CACHED>(V.at, y, A);
    }
}

template <int MODE, int TEAM, int AHEAD, class P, class G>
__device__ __forceinline__ void adam_master(const TensorD &t, const Piece &p, const AdamT &A)
{
    if (t.master) adam_piece<MODE, TEAM, AHEAD, P, G, true>(t, p, A);
    else adam_piece<MODE, TEAM, AHEAD, P, G, false>(t, p, A);
}

template <int MODE, int TEAM, int AHEAD, class P>
__device__ __forceinline__ void adam_grad(const TensorD &t, const Piece &p, const AdamT &A)
{
    switch (t.types & 255) {
    case TYPE_F32: adam_master<MODE, TEAM, AHEAD, P, float>(t, p, A); break;
    case TYPE_BF16: adam_master<MODE, TEAM, AHEAD, P, __bf16>(t, p, A); break;
    default: adam_master<MODE, TEAM, AHEAD, P, _Float16>(t, p, A); break;
    }
}

struct AdamC { float coef, rate, inv1, inv_sqrt2; };       // of one step

// What the number of the step makes of the rate, by one wave for its block: the 64-bit arithmetic would take every wave some 0.8 us.  That wave's first
// lane also takes the ticket here, when it has read the counter, and looks at it at the end, when the answer has long come.
struct StepD { long long before; Ticket ticket; };
__device__ __forceinline__ StepD adam_begin(const AdamD &A, const float *lr_word, const long long *steps, unsigned *tickets, AdamC *shared)
{
    StepD s;
    s.before = *steps;
    const double time = (double)(s.before + 1);
    const AdamC C = {0.0f, lr_word ? *lr_word : A.lr, (float)(1.0 / one_minus_exp(time * A.log_beta1)), (float)(1.0 / __builtin_sqrt(one_minus_exp(time * A.log_beta2)))};
    if ((threadIdx.x & 63) == 0) {
        *shared = C;
        s.ticket = take_ticket(tickets);
    }
    return s;
}

// The counter moves on when every block has read it, unless the step was skipped.
__device__ __forceinline__ void adam_end(const StepD &s, bool skip, long long *steps, unsigned *tickets)
{
    if ((threadIdx.x & 63) == 0 && is_last(s.ticket, tickets) && !skip) *steps = s.before + 1;
}

template <int MODE, int TEAM, int AHEAD>
__device__ __forceinline__ void adam_types(const TensorD &t, const Piece &p, const AdamD &A, const AdamC &C)
{
    const float lr = C.rate * t.lr_scale;
    const AdamT T = {C.coef, lr * (A.decay * t.decay_scale), lr * C.inv1, C.inv_sqrt2, A.beta1, A.beta2, A.rest1, A.rest2, A.eps};
    switch (t.types >> 8) {
    case TYPE_F32: adam_grad<MODE, TEAM, AHEAD, float>(t, p, T); break;
    case TYPE_BF16: adam_grad<MODE, TEAM, AHEAD, __bf16>(t, p, T); break;
    default: adam_grad<MODE, TEAM, AHEAD, _Float16>(t, p, T); break;
    }
}

__device__ __forceinline__ bool is_finite(double x) { return __builtin_fabs(x) < __builtin_inf(); }

// Reads four arrays and writes three (of 16-bit parameters with masters, four and four), 28 bytes an element, once each; the counters say that no more is moved.
// 250 M elements in 1251 us (7.0 GB, 5.6 TB/s), 12.6 M fp32 in 57 (6.2).  Its 44 vector instructions an element take a quarter of that.  Four elements a thread, so
// that fp32 arrays are read 16 bytes at a time; more on its way per thread, or more blocks, makes no difference or costs pages in use (see grid_for).
template <int MODE>
__global__ __launch_bounds__(256) void k_adamw(ListD L, AdamD A, NormD N, const float *__restrict__ lr_word, long long *__restrict__ steps, unsigned *__restrict__ tickets)
{
    Walk<true> walk(L);
    __shared__ AdamC shared;
    StepD step;
    const bool first = threadIdx.x < 64;
    if (first) step = adam_begin(A, lr_word, steps, tickets, &shared);
    const double n = norm_value(N);
    __syncthreads();
    const bool skip = A.skip_nonfinite && !is_finite(n);   // every block sees the same norm
    if (!skip) {
        AdamC C = shared;
        C.coef = clip_coef(n, A.max_norm, A.scale);
        walk.each([&](const TensorD &t, const Piece &p, int) { adam_types<MODE, 256, AHEAD_ADAMW>(t, p, A, C); });
    }
    if (first) adam_end(step, skip, steps, tickets);
}

// With the norm in the same kernel, which is as good as the list is short.
__global__ __launch_bounds__(SHORT_THREADS) void k_adamw_short(ListD L, AdamD A, const float *__restrict__ lr_word, float *__restrict__ norm,
                                                               long long *__restrict__ steps, unsigned *__restrict__ tickets)
{
    __shared__ AdamC shared;
    StepD step;
    const int wave = threadIdx.x >> 6;
    const bool last_wave = wave == SHORT_WAVES - 1;        // the one with the least to add up
    if (last_wave) step = adam_begin(A, lr_word, steps, tickets, &shared);
    const double n = short_norm<KIND_TWO>(L, A.scale);     // waits for all of the block
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    const bool skip = A.skip_nonfinite && !is_finite(n);
    if (!skip) {
        AdamC C = shared;
        C.coef = clip_coef(n, A.max_norm, A.scale);
        walk_short<SHORT_PART>(L, blockIdx.x * SHORT_WAVES + wave, gridDim.x * SHORT_WAVES, [&](const TensorD &t, const Piece &p) { adam_types<ADAM_CACHED, 64, 1>(t, p, A, C); });
    }
    if (last_wave) adam_end(step, skip, steps, tickets);
}

}  // namespace fs
