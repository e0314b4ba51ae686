// Kernels of the networks' layers: products with their epilogue, the backward pass, dropout (see include/fastsnarf_net.h).
//
// Every product is D[p][q] = sum over t of P[p][t] Q[q][t], with p along the rows of the result in memory.  As operands of the matrix instructions P has their
// rows and Q their columns, so a lane's results are four neighbours p: a vector to store, and the words of one Philox call.
//   forward  p = outputs, q = rows,    t = inputs     P = weight (t along its rows), Q = X  (t along its rows)
//   dX       p = inputs,  q = rows,    t = outputs    P = weight (p along its rows), Q = dZ (t along its rows)
//   dweight  p = inputs,  q = outputs, t = rows       P = X      (p along its rows), Q = dZ (q along its rows)
// A matrix with t along its rows lies in LDS as it lies in memory and is read 16 bytes a lane; one with p or q along its rows, too, and is turned on the way
// to the registers by the LDS's transposing reads.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fs {

enum { NET_F32, NET_BF16, NET_F16 };
enum { ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU, ACT_SOFTPLUS };

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// A matrix in memory, `ld` elements from row to row.
struct MatD { const void *at; long long ld, rows, cols; };

struct DropD {
    const long long *at;               // seed and offset on the device, or NULL:
    unsigned long long seed, offset;
    unsigned least;                    // words from here on are kept
    int mode;                          // 0: nothing is dropped, 1: by the words, 2: everything is
    float scale;
};

// ---------------------------------------------------------------------------------------------------------------- elements

template <int TYPE> struct ElemOf { typedef unsigned short type; };
template <> struct ElemOf<NET_F32> { typedef float type; };

template <int TYPE> __device__ inline float widen(typename ElemOf<TYPE>::type v)
{
    if constexpr (TYPE == NET_F32) return v;
    else if constexpr (TYPE == NET_BF16) return __uint_as_float((unsigned)v << 16);
    else return (float)__builtin_bit_cast(_Float16, v);
}

template <int TYPE> __device__ inline typename ElemOf<TYPE>::type narrow(float v)
{
    if constexpr (TYPE == NET_F32) return v;
    else if constexpr (TYPE == NET_BF16) return __builtin_bit_cast(unsigned short, (__bf16)v);
    else return __builtin_bit_cast(unsigned short, (_Float16)v);
}

// N elements (a multiple of 16 bytes, or 8), as words.  In memory they lie at any address that is a multiple of one: the vector instructions take those.
template <int TYPE, int N> struct Packed {
    static constexpr int SIZE = TYPE == NET_F32 ? 4 : 2, WORDS = N * SIZE / 4;
    unsigned w[WORDS];
    typedef typename ElemOf<TYPE>::type T;

    __device__ inline T at(int i) const
    {
        if constexpr (TYPE == NET_F32) return __uint_as_float(w[i]);
        else return (T)(w[i / 2] >> (i & 1) * 16);
    }
    __device__ inline float wide(int i) const
    {
        if constexpr (TYPE == NET_BF16) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        else return widen<TYPE>(at(i));
    }
};

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
template <int SIZE> struct Loose;      // vectors at any address that is a multiple of SIZE
template <> struct Loose<2> { typedef u32x2 two __attribute__((aligned(2))); typedef u32x4 four __attribute__((aligned(2))); };
template <> struct Loose<4> { typedef u32x2 two __attribute__((aligned(4))); typedef u32x4 four __attribute__((aligned(4))); };

template <int TYPE, int N> __device__ inline Packed<TYPE, N> load_all(const typename ElemOf<TYPE>::type *at)
{
    typedef Packed<TYPE, N> R;
    R r;
    if constexpr (R::WORDS == 2) {
        const u32x2 v = *reinterpret_cast<const typename Loose<R::SIZE>::two *>(at);
        r.w[0] = v.x; r.w[1] = v.y;
    } else {
#pragma unroll
        for (int k = 0; k < R::WORDS; k += 4) {
            const u32x4 v = *reinterpret_cast<const typename Loose<R::SIZE>::four *>(at + k * 4 / R::SIZE);
            r.w[k] = v.x; r.w[k + 1] = v.y; r.w[k + 2] = v.z; r.w[k + 3] = v.w;
        }
    }
    return r;
}

// The first `n` (1 .. N) of N elements, zeros behind them.  Single elements are loaded without conditions, so that all are on their way at once.
template <int TYPE, int N> __device__ inline Packed<TYPE, N> load_some(const typename ElemOf<TYPE>::type *at, int n)
{
    if (n >= N) return load_all<TYPE, N>(at);
    Packed<TYPE, N> r;
#pragma unroll
    for (int k = 0; k < r.WORDS; ++k) {
        if constexpr (TYPE == NET_F32) {
            const unsigned x = __float_as_uint(at[k < n ? k : n - 1]);
            r.w[k] = k < n ? x : 0u;
        } else {
            const unsigned lo = at[2 * k < n ? 2 * k : n - 1], hi = at[2 * k + 1 < n ? 2 * k + 1 : n - 1];
            r.w[k] = (2 * k < n ? lo : 0u) | (2 * k + 1 < n ? hi : 0u) << 16;
        }
    }
    return r;
}

template <int TYPE, int N> __device__ inline void load_wide(float *v, const typename ElemOf<TYPE>::type *at, int n)
{
    const auto x = load_some<TYPE, N>(at, n);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = x.wide(i);
}

template <int TYPE, int N> __device__ inline void store_some(typename ElemOf<TYPE>::type *at, const float *v, int n)
{
    typedef Packed<TYPE, N> R;
    if (n < N) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) at[i] = narrow<TYPE>(v[i]);
        return;
    }
    unsigned w[R::WORDS];
#pragma unroll
    for (int k = 0; k < R::WORDS; ++k) {
        if constexpr (TYPE == NET_F32) w[k] = __float_as_uint(v[k]);
        else w[k] = (unsigned)narrow<TYPE>(v[2 * k]) | (unsigned)narrow<TYPE>(v[2 * k + 1]) << 16;
    }
    if constexpr (R::WORDS == 2) *reinterpret_cast<typename Loose<R::SIZE>::two *>(at) = u32x2{w[0], w[1]};
    else
#pragma unroll
        for (int k = 0; k < R::WORDS; k += 4) *reinterpret_cast<typename Loose<R::SIZE>::four *>(at + k * 4 / R::SIZE) = u32x4{w[k], w[k + 1], w[k + 2], w[k + 3]};
}

// ---------------------------------------------------------------------------------------------------------------- dropout

// Philox4x32-10.  Ten rounds take a large bf16 dropout 8 % longer than none at all: 268 M elements, 537 MB read and 537 MB written, in 229 and 212 us (seven rounds: 224).
__device__ inline uint4 philox(unsigned long long block, unsigned long long offset, unsigned long long seed)
{
    unsigned a = (unsigned)block, b = (unsigned)(block >> 32), c = (unsigned)offset, d = (unsigned)(offset >> 32);
    unsigned k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long p = 0xD2511F53ull * a, q = 0xCD9E8D57ull * c;
        a = __builtin_amdgcn_bitop3_b32((unsigned)(q >> 32), b, k0, 0x96);             // a ^ b ^ c
        b = (unsigned)q;
        c = __builtin_amdgcn_bitop3_b32((unsigned)(p >> 32), d, k1, 0x96);
        d = (unsigned)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(a, b, c, d);
}

struct Seed { unsigned long long seed, offset; };
__device__ inline Seed seed_of(const DropD &d)
{
    Seed s = {d.seed, d.offset};
    if (d.mode == 1 && d.at) {
        s.seed = (unsigned long long)d.at[0];
        s.offset = (unsigned long long)d.at[1];
    }
    return s;
}

// drop() of N (4 or 8) elements from element e on.
template <int N> __device__ inline void drop(float *v, unsigned long long e, const DropD &d, const Seed &s)
{
    if (d.mode == 0) return;
    if (d.mode == 2) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.0f;
        return;
    }
    const int shift = (int)(e & 3);
    unsigned w[N + 4];
#pragma unroll
    for (int b = 0; b < N / 4; ++b) {
        const uint4 x = philox((e >> 2) + b, s.offset, s.seed);
        w[4 * b] = x.x; w[4 * b + 1] = x.y; w[4 * b + 2] = x.z; w[4 * b + 3] = x.w;
    }
    if (shift) {                       // the elements begin inside a call's words
        const uint4 x = philox((e >> 2) + N / 4, s.offset, s.seed);
        w[N] = x.x; w[N + 1] = x.y; w[N + 2] = x.z; w[N + 3] = x.w;
        if (shift & 1)
#pragma unroll
            for (int i = 0; i < N + 3; ++i) w[i] = w[i + 1];
        if (shift & 2)
#pragma unroll
            for (int i = 0; i < N + 2; ++i) w[i] = w[i + 2];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = w[i] >= d.least ? v[i] * d.scale : 0.0f;
}

// ---------------------------------------------------------------------------------------------------------------- fp16's range

// dZ goes into 16 bits for the products.  fp16 has 40 powers of two, and dZ may lie below its least (gradients of a mean) or, divided by 1 - p, above its largest number: so it goes
// in times the power of two that takes the largest finite |G| / (1 - p) to 2^14 .. 2^15 (slopes are 1.13 at most), and the results are divided by that, both exactly.  What
// rounds to fp16's least steps is then below 2^-28 of the largest.  bf16 has fp32's range, and needs nothing.
struct Power { float to, back; };
__device__ inline Power power_of(unsigned most, const DropD &d)
{
    const float f = widen<NET_F16>((unsigned short)most) * (d.mode == 1 ? d.scale : 1.0f);
    if (!(f > 0.0f)) return {1.0f, 1.0f};
    const int e = (int)(__float_as_uint(f) >> 23) - 127;          // -24 .. 47
    return {__uint_as_float((unsigned)(127 + 14 - e) << 23), __uint_as_float((unsigned)(127 - 14 + e) << 23)};
}

// The largest finite fp16 numbers without signs, two columns of them, as bits and 0x0400: infinities and NaN are negative then.
typedef short s16x2 __attribute__((ext_vector_type(2)));
struct Largest {
    s16x2 most = {0x0400, 0x0400};

    __device__ inline void add(const Packed<NET_F16, 8> &x)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) most = __builtin_elementwise_max(most, __builtin_bit_cast(s16x2, x.w[k] & 0x7FFF7FFFu) + s16x2{0x0400, 0x0400});
    }
    __device__ inline unsigned bits() const { return (unsigned)(most.x > most.y ? most.x : most.y) - 0x0400u; }
};

// ... of a block's threads, of WAVES waves
template <int WAVES> __device__ inline unsigned largest_of(unsigned most, unsigned *s_most)
{
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) {
        const unsigned other = __shfl_xor(most, m);
        most = other > most ? other : most;
    }
    if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) most = s_most[w] > most ? s_most[w] : most;
    return most;
}

// ---------------------------------------------------------------------------------------------------------------- activations

// The hardware's 2^x, log2 and 1/x are good to a unit of the last place; what is built on them here is off by some units, of e^x |x| more (the rounding of x log2 e).
// The library's functions take 5 times the instructions, and an epilogue is bound by those: 65536 x 128 softplus took 33 us with them beside 35 for the product.
__device__ inline float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
__device__ inline float fast_rcp(float x) { return __builtin_amdgcn_rcpf(x); }

// ln(1 + u) of 0 <= u <= 1: ln of the rounded 1 + u, and what that rounding left out, at most 2^-24, times the slope 1 / (1 + u), for which 1 - u / 2 is near
// enough: it is off by u / 4 of that at most, 2^-26 of the result.
__device__ inline float log_of_one_more(float u)
{
    const float w = 1.0f + u, d = w - 1.0f;
    return __builtin_fmaf(__builtin_amdgcn_logf(w), 0.693147181f, (u - d) * __builtin_fmaf(d, -0.5f, 1.0f));
}

// Phi(z), and e^(-z^2/2), which it is made from: with u = |z| and t = 1 / (1 + 0.3 u), Phi(-u) = e^(-u^2/2) (t c0 + t^2 c1 + .. + t^10 c9), a polynomial fitted to
// the least relative error, 1e-7 (4e-7 in fp32 arithmetic).
__device__ inline float normal_of(float z, float &bell)
{
    constexpr float C[10] = {0.119682692f, 0.119680032f, 0.109011605f, 0.0859197751f, 0.068387121f, -0.0155361798f, 0.0995843709f, -0.147240862f, 0.0729390979f, -0.0124276103f};
    const float t = fast_rcp(__builtin_fmaf(fabsf(z), 0.3f, 1.0f));
    bell = fast_exp(-0.5f * z * z);
    float p = C[9];
#pragma unroll
    for (int i = 8; i >= 0; --i) p = __builtin_fmaf(p, t, C[i]);
    p *= t * bell;
    return z < 0.0f ? p : 1.0f - p;
}

template <int ACT> __device__ inline float act_of(float z, float beta, float over_beta)
{
    if constexpr (ACT == ACT_RELU) return z < 0.0f ? 0.0f : z;                                     // NaN stays
    else if constexpr (ACT == ACT_GELU) {
        float bell;
        return z * normal_of(z, bell);
    } else if constexpr (ACT == ACT_SILU) return z * fast_rcp(1.0f + fast_exp(-z));
    else if constexpr (ACT == ACT_SOFTPLUS) return __builtin_fmaf(log_of_one_more(fast_exp(-fabsf(z * beta))), over_beta, z < 0.0f ? 0.0f : z);
    else return z;
}

template <int ACT> __device__ inline float slope_of(float z, float beta)
{
    if constexpr (ACT == ACT_RELU) return z <= 0.0f ? 0.0f : 1.0f;
    else if constexpr (ACT == ACT_GELU) {
        float bell;
        const float n = normal_of(z, bell);
        return __builtin_fmaf(z * 0.39894228f, bell, n);
    } else if constexpr (ACT == ACT_SILU) {
        const float s = fast_rcp(1.0f + fast_exp(-z));
        return s * __builtin_fmaf(z, 1.0f - s, 1.0f);
    } else if constexpr (ACT == ACT_SOFTPLUS) return fast_rcp(1.0f + fast_exp(-z * beta));
    else return 1.0f;
}

template <int N> struct Int { static constexpr int value = N; };

// f(Int<act>()), the branch outside of the loops
template <class F> __device__ inline void with_act(int act, F f)
{
    switch (act) {
    case ACT_RELU: return f(Int<ACT_RELU>());
    case ACT_GELU: return f(Int<ACT_GELU>());
    case ACT_SILU: return f(Int<ACT_SILU>());
    case ACT_SOFTPLUS: return f(Int<ACT_SOFTPLUS>());
    default: return f(Int<ACT_NONE>());
    }
}

// ---------------------------------------------------------------------------------------------------------------- epilogue

enum { EPI_LAYER, EPI_STORE, EPI_PART };

// What becomes of D.  EPI_LAYER: the layer's Y (and Z), EPI_STORE: out = D in the type (fp16: times *factor, where that is not NULL), EPI_PART: fp32 sums of one part of the
// range of t into out, `part_stride` floats from part to part.
struct EpiD {
    int mode, act, bias_f32, z_f32;
    float beta, over_beta;
    const void *bias, *r;
    void *out, *z;
    long long ldr, ldo, ldz, part_stride;
    const float *factor;
    DropD drop;
};

template <int TYPE> __device__ inline void load_bias(float *b, const EpiD &E, long long p, int n)
{
    if (E.mode != EPI_LAYER || !E.bias || n <= 0) {
        b[0] = b[1] = b[2] = b[3] = 0.0f;
    } else if (E.bias_f32) {
        load_wide<NET_F32, 4>(b, static_cast<const float *>(E.bias) + p, n);
    } else {
        load_wide<TYPE, 4>(b, static_cast<const typename ElemOf<TYPE>::type *>(E.bias) + p, n);
    }
}

// Where a lane's results go, and what joins them there: addresses of one row, and of others by whole numbers of rows.
template <int TYPE> struct Place {
    typedef typename ElemOf<TYPE>::type T;
    T *out;
    char *z;
    const T *r;
    long long ldo, ldz, ldr;
    int zs;

    __device__ inline Place(const EpiD &E, long long q, long long p, int part)
    {
        zs = TYPE == NET_F32 || E.z_f32 ? 4 : 2;
        ldo = E.ldo;
        ldz = E.ldz * zs;
        ldr = E.ldr;
        if (E.mode == EPI_PART) out = reinterpret_cast<T *>(static_cast<float *>(E.out) + part * E.part_stride + q * E.ldo + p);
        else out = static_cast<T *>(E.out) + q * E.ldo + p;
        z = E.z ? static_cast<char *>(E.z) + q * ldz + p * zs : nullptr;
        r = E.r ? static_cast<const T *>(E.r) + q * E.ldr + p : nullptr;
    }
};

// What fp16 keeps of Z: finite numbers stay finite (the slopes at an infinity would be NaN, and are 0 and 1 at 65504 already), and positive ones positive (relu's slope is 1).
__device__ inline float half_z(float v)
{
    const float h = v > 0.0f && v < 0x1p-24f ? 0x1p-24f : __builtin_amdgcn_fmed3f(v, -65504.0f, 65504.0f);
    return fabsf(v) < INFINITY ? h : v;
}

// Four results, of which n (1 .. 4) are in the matrix, `rows` rows behind the place; e: the first one's number for drop(); r: their residual.
template <int TYPE, int ACT>
__device__ inline void finish4(float *v, const float *bias, const Packed<TYPE, 4> &r, const EpiD &E, const Seed &seed, const Place<TYPE> &at, int rows, unsigned long long e, int n)
{
    typedef typename ElemOf<TYPE>::type T;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += bias[i];
    if (E.z) {
        char *z = at.z + rows * at.ldz;
        if (E.z_f32) store_some<NET_F32, 4>(reinterpret_cast<float *>(z), v, n);
        else if constexpr (TYPE == NET_F16) {
            float h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = half_z(v[i]);
            store_some<TYPE, 4>(reinterpret_cast<T *>(z), h, n);
        } else store_some<TYPE, 4>(reinterpret_cast<T *>(z), v, n);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = act_of<ACT>(v[i], E.beta, E.over_beta);
    drop<4>(v, e, E.drop, seed);
    if (E.r)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += r.wide(i);
    store_some<TYPE, 4>(at.out + rows * at.ldo, v, n);
}

template <int TYPE> __device__ inline Packed<TYPE, 4> residual4(const EpiD &E, const Place<TYPE> &at, int rows, int n)
{
    Packed<TYPE, 4> r = {};
    if (E.r) r = load_some<TYPE, 4>(at.r + rows * at.ldr, n);
    return r;
}

template <int TYPE> __device__ inline float factor_of(const EpiD &E)
{
    if constexpr (TYPE == NET_F16) return E.factor ? *E.factor : 1.0f;
    else return 1.0f;
}

template <int TYPE> __device__ inline void plain4(float *v, float factor, const EpiD &E, const Place<TYPE> &at, int rows, int n)
{
    if constexpr (TYPE == NET_F16)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= factor;
    if (E.mode == EPI_PART) store_some<NET_F32, 4>(reinterpret_cast<float *>(at.out) + rows * at.ldo, v, n);
    else store_some<TYPE, 4>(at.out + rows * at.ldo, v, n);
}

// ---------------------------------------------------------------------------------------------------------------- products

// Where chunks of 8 elements lie in an LDS tile, so that the 16 lanes that are served together find theirs in 16 different places of 16 bytes.
// t along the rows: chunk c of row r; RP rows fill the 256 bytes of all banks.
template <int BT> __device__ inline int place_row(int r, int c)
{
    constexpr int RP = 128 / BT;
    return r * BT + ((c ^ ((r / RP) & (BT / 8 - 1))) * 8);
}
// p along the rows: a transposing read takes 32 bytes from each of four rows t, and its other half-wave's neighbours the next 32.
template <int B> __device__ inline int place_col(int t, int c)
{
    constexpr int RP = B >= 128 ? 1 : 128 / B;
    const int turn = B >= 64 ? 4 * ((t / RP) & (4 / RP - 1)) : 0;
    return t * B + ((c ^ turn) * 8);
}

template <int TYPE> __device__ inline f32x16 mfma(s16x8 a, s16x8 b, f32x16 c)
{
    if constexpr (TYPE == NET_F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// The operand of one matrix instruction from a tile with p along its rows: 32 of those from p0 on, t = 16 step + 8 (lane / 32) + 0 .. 7.
template <class Place> __device__ inline s16x8 turned(Place place, const short *tile, int p0, int step, int lane)
{
    // lane i of 16 hands in 4 elements of row t + i / 4 and gets those of column i
    const int i = lane & 15, t = 16 * step + 8 * (lane >> 5) + (i >> 2), p = p0 + (lane & 16) + 4 * (i & 3);
    const short *lo = tile + place(t, p >> 3) + (p & 7), *hi = tile + place(t + 4, p >> 3) + (p & 7);
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)lo), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)hi);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// The same from either kind of tile.
template <bool COL, int B, int BT> __device__ inline s16x8 operand(const short *tile, int p0, int step, int lane)
{
    if constexpr (COL) return turned([](int t, int c) { return place_col<B>(t, c); }, tile, p0, step, lane);
    else return *reinterpret_cast<const s16x8 *>(tile + place_row<BT>(p0 + (lane & 31), 2 * step + (lane >> 5)));
}

// Three bf16 parts of fp32 numbers: x = h + m + l to 24 bits and more, each part the rounded rest of those before it.  A rest that is no number
// (of infinities) gives results that are none either, which made_again() makes again.
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ inline void split8(const Packed<NET_F32, 8> &x, s16x8 *part)
{
    unsigned w[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {                      // two at a time, as the conversion does them
        f32x2 v = {x.wide(2 * i), x.wide(2 * i + 1)};
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            w[k][i] = __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
            v = f32x2{v.x - __uint_as_float(w[k][i] << 16), v.y - __uint_as_float(w[k][i] & 0xFFFF0000u)};
        }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) part[k] = __builtin_bit_cast(s16x8, u32x4{w[k][0], w[k][1], w[k][2], w[k][3]});
}

__device__ inline f32x16 mfma_bf16(s16x8 a, s16x8 b, f32x16 c) { return mfma<NET_BF16>(a, b, c); }
__device__ inline f32x4 mfma_bf16(s16x8 a, s16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0); }

// What eight numbers are beside infinities, as bf16: NaN, infinities and zeros themselves, 1 of the sign for all others.
__device__ inline s16x8 kinds8(const float (&x)[8])
{
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned u = __float_as_uint(x[i]), size = u & 0x7FFFFFFFu, k = (u >> 16 & 0x8000u) | (size > 0x7F800000u ? 0x7FC0u : size == 0x7F800000u ? 0x7F80u : size ? 0x3F80u : 0u);
        w[i / 2] = i & 1 ? w[i / 2] | k << 16 : k;
    }
    return __builtin_bit_cast(s16x8, u32x4{w[0], w[1], w[2], w[3]});
}

// A wave's results (those of one matrix instruction, get(i) and set(i, value)) that are no finite numbers, made again: they may be the parts' making (inf - inf, or a part
// of the largest numbers rounded up to infinity).  p(x, s) and q(x, s): a lane's elements of step s of the operands, in fp32.
//  1. A sum over the products of kinds is no finite number where NaN or infinities take part, and is then what theirs is.
//  2. Else the products or their parts passed 2^128: the parts of operands times 2^-64 do not.  What that takes from operands below 2^-38 is below 2^-62 times the
//     other's size, which sums beyond 2^128 do not hold.
// Bound by latency: a step's loads, past LDS, are waited for one step after another.  A batch of NaN, us, with it and without NaN: 2048 cubed forward 960 and 94, backward of
// 65536 x 128 x 128 270 and 50; finite sums beyond 2^128 take the second pass too (2048 cubed 1850).  A scalar sum for each result took 15200 and 7400.
template <class V, class P, class Q, class Get, class Set> __device__ inline void made_again(long long steps, P p, Q q, Get get, Set set)
{
    constexpr int N = sizeof(V) / 4;
    auto no_number = [&](int i) { return !(fabsf(get(i)) < INFINITY); };
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; ++i) bad |= no_number(i);
    if (!__any(bad)) return;
    constexpr int PA[6] = {0, 1, 2, 0, 1, 0}, PB[6] = {2, 1, 0, 1, 0, 0};
    unsigned left = 0;                 // bits of those that are left to the second pass
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        V sum;
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = 0.0f;
        auto parts = [&](const float (&x)[8], s16x8 *to) {
            if (pass == 0) {
                to[0] = kinds8(x);
                return;
            }
            Packed<NET_F32, 8> small;
#pragma unroll
            for (int i = 0; i < 8; ++i) small.w[i] = __float_as_uint(x[i] * 0x1p-64f);
            split8(small, to);
        };
#pragma unroll 1
        for (long long s = 0; s < steps; ++s) {
            s16x8 u[3], w[3];
            float x[8];
            p(x, s);
            parts(x, u);
            __builtin_amdgcn_sched_barrier(0);         // one operand after the other: few registers
            q(x, s);
            parts(x, w);
            if (pass == 0) sum = mfma_bf16(u[0], w[0], sum);
            else
#pragma unroll
                for (int i = 0; i < 6; ++i) sum = mfma_bf16(u[PA[i]], w[PB[i]], sum);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (pass == 0 && no_number(i)) {
                if (fabsf(sum[i]) < INFINITY) left |= 1u << i;
                else set(i, sum[i]);
            }
            if (pass == 1 && left >> i & 1) set(i, sum[i] * 0x1p64f * 0x1p64f);
        }
        if (!__any(left)) return;
    }
}

// ... of results in registers
template <class V, class P, class Q> __device__ inline void made_again(V &v, long long steps, P p, Q q)
{
    made_again<V>(steps, p, q, [&](int i) { return v[i]; }, [&](int i, float x) { v[i] = x; });
}

// Eight elements of row (COL: column) r from t on, zeros from t1 on.  t1 is at least 1.
template <int TYPE, bool COL> __device__ inline void eight(float (&x)[8], const MatD &M, long long r, long long t, long long t1)
{
    const typename ElemOf<TYPE>::type *at = static_cast<const typename ElemOf<TYPE>::type *>(M.at);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const long long n = t + k < t1 ? t + k : t1 - 1;
        x[k] = widen<TYPE>(at[COL ? n * M.ld + r : r * M.ld + n]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (t + k >= t1) x[k] = 0.0f;
}

// One operand's tile on its way from memory to LDS: B rows (p or q) by BT, in chunks of 8.
template <int TYPE, bool COL, int B, int BT, int THREADS> struct Stage {
    typedef typename ElemOf<TYPE>::type T;
    static constexpr int PLANES = TYPE == NET_F32 ? 3 : 1;
    static constexpr int ROWS = COL ? BT : B, COLS = COL ? B : BT, PER_ROW = COLS / 8, N = ROWS * PER_ROW / THREADS;
    static constexpr int LDS = PLANES * B * BT;            // 16-bit elements
    static_assert(ROWS * PER_ROW % THREADS == 0 && N >= 1, "tile");
    static constexpr int APART = THREADS / PER_ROW;        // rows between a thread's chunks
    static_assert(THREADS % PER_ROW == 0, "tile");
    Packed<TYPE, 8> chunk[N];

    // Where a thread's chunks of the tile that begins at row or column b0 lie, from its first element on.  Rows beyond the matrix: the last one, whose results go nowhere.
    struct Own { long long at[COL ? 1 : N]; };
    static __device__ inline Own own(const MatD &M, long long b0, int tid)
    {
        Own o;
        const int r = tid / PER_ROW, c = tid % PER_ROW * 8;
        if constexpr (COL) o.at[0] = r * M.ld + c;
        else
#pragma unroll
            for (int i = 0; i < N; ++i) o.at[i] = (b0 + r + i * APART < M.rows ? r + i * APART : M.rows - 1 - b0) * M.ld + c;
        return o;
    }

    // A tile of whole t, and, COL, whole chunks.  Addresses are a wave's and a lane's part, of which the latter stays the same.
    __device__ inline void fast(const MatD &M, long long b0, long long t0, const Own &o)
    {
        const T *at = static_cast<const T *>(M.at) + (COL ? t0 * M.ld + b0 : b0 * M.ld + t0);
#pragma unroll
        for (int i = 0; i < N; ++i) chunk[i] = load_all<TYPE, 8>(COL ? at + i * APART * M.ld + o.at[0] : at + o.at[COL ? 0 : i]);
    }

    // Any tile.  b0: first row or column p; t0: first t; t1: end of the range of t.
    __device__ inline void load(const MatD &M, long long b0, long long t0, long long t1, int tid)
    {
        const long long r0 = COL ? t0 : b0, c0 = COL ? b0 : t0, rows = COL ? t1 : M.rows, cols = COL ? M.cols : t1;
        const T *at = static_cast<const T *>(M.at) + r0 * M.ld + c0 + (tid / PER_ROW * M.ld + tid % PER_ROW * 8);
        const long long left = cols - (c0 + tid % PER_ROW * 8);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            chunk[i] = Packed<TYPE, 8>();
            if (r0 + tid / PER_ROW + i * APART < rows && left > 0) chunk[i] = load_some<TYPE, 8>(at + i * APART * M.ld, left < 8 ? (int)left : 8);
        }
    }

    // zeros where the matrix has nothing
    static __device__ inline Packed<TYPE, 8> guarded(const T *at, long long ld, long long r, long long c, long long rows, long long cols)
    {
        Packed<TYPE, 8> x = {};
        if (r < rows && c < cols) {
            const long long left = cols - c;
            x = load_some<TYPE, 8>(at + r * ld + c, left < 8 ? (int)left : 8);
        }
        return x;
    }

    static __device__ inline void put(const Packed<TYPE, 8> &x, short *tile, int u)
    {
        const int r = u / PER_ROW, c = u % PER_ROW;
        short *at = tile;
        if constexpr (COL) at += place_col<B>(r, c);
        else at += place_row<BT>(r, c);
        if constexpr (TYPE == NET_F32) {
            s16x8 part[3];
            split8(x, part);
#pragma unroll
            for (int k = 0; k < 3; ++k) *reinterpret_cast<s16x8 *>(at + k * B * BT) = part[k];
        } else {
            *reinterpret_cast<u32x4 *>(at) = u32x4{x.w[0], x.w[1], x.w[2], x.w[3]};
        }
    }

    __device__ inline void store(short *tile, int tid) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) put(chunk[i], tile, tid + i * THREADS);
    }

    // the whole way at once, chunk by chunk: few registers
    static __device__ inline void bring(const MatD &M, long long b0, long long t0, long long t1, short *tile, int tid)
    {
#pragma unroll 1
        for (int u = tid; u < ROWS * PER_ROW; u += THREADS)
            put(guarded(static_cast<const T *>(M.at), M.ld, (COL ? t0 : b0) + u / PER_ROW, (COL ? b0 : t0) + u % PER_ROW * 8, COL ? t1 : M.rows, COL ? M.cols : t1), tile, u);
    }
};

// The end of a product: a wave's results, MT by NT squares from (p0, q0) on, go through LDS (end_floats(MT) of its own), 32 rows q and up to 64 p at a time,
// so that rows leave in whole lines.  fp32: again(p, q, get, set) makes those of a square that are no finite numbers again.
constexpr __host__ __device__ int end_floats(int mt) { return 32 * ((mt > 1 ? 64 : 32) + 4); }

template <int TYPE, bool LAYER, int MT, int NT, class Again>
__device__ inline void product_end(const f32x16 (&acc)[MT][NT], float *out, int lane, long long p0, long long q0, long long np, long long nq, int part, const EpiD &E, Again again)
{
    constexpr int MG = MT > 1 ? 2 : 1, PW = 32 * MG, PITCH = PW + 4;
    static_assert(MT % MG == 0, "squares");
    const int col = 4 * (lane % (PW / 4));
    const Seed seed = seed_of(E.drop);
    const float factor = factor_of<TYPE>(E);
#pragma unroll 1
    for (int h = 0; h < NT * (MT / MG); ++h) {
        bool bad = false;
#pragma unroll
        for (int k = 0; k < NT * (MT / MG); ++k)           // a register's number is fixed
            if (k == h)
#pragma unroll
                for (int i = 0; i < MG; ++i)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x16 &x = acc[k / NT * MG + i][k % NT];
                        f32x4 v = {x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]};
                        *reinterpret_cast<f32x4 *>(out + (lane & 31) * PITCH + 32 * i + 8 * g + 4 * (lane >> 5)) = v;
                        if constexpr (TYPE == NET_F32)
#pragma unroll
                            for (int m = 0; m < 4; ++m) bad |= !(fabsf(v[m]) < INFINITY);
                    }
        if (TYPE == NET_F32 && __any(bad))
#pragma unroll 1
            for (int i = 0; i < MG; ++i) {             // each lane those that it wrote
                float *x = out + (lane & 31) * PITCH + 32 * i + 4 * (lane >> 5);
                again(p0 + h / NT * PW + 32 * i, q0 + h % NT * 32, [&](int k) { return x[8 * (k >> 2) + (k & 3)]; }, [&](int k, float v) { x[8 * (k >> 2) + (k & 3)] = v; });
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        constexpr int STEP = 64 / (PW / 4), PASSES = 32 / STEP, AHEAD = 4;
        const long long p = p0 + h / NT * PW + col, q1 = q0 + h % NT * 32 + lane / (PW / 4);
        const int n = np - p < 4 ? (int)(np - p) : 4, rows = nq - q1 < 32 ? (int)(nq - q1) : 32;      // of which this lane has every STEP-th
        const float *in = out + lane / (PW / 4) * PITCH + col;
        const Place<TYPE> at(E, q1, p, part);
        if (n > 0 && LAYER && E.mode == EPI_LAYER) {
            float bias[4];
            load_bias<TYPE>(bias, E, p, n);
            const unsigned long long e = (unsigned long long)q1 * np + p;
            with_act(E.act, [&](auto act) {
#pragma unroll 1
                for (int r = 0; r < PASSES; r += AHEAD) {
                    Packed<TYPE, 4> res[AHEAD];
#pragma unroll
                    for (int a = 0; a < AHEAD; ++a)
                        if ((r + a) * STEP < rows) res[a] = residual4<TYPE>(E, at, (r + a) * STEP, n);
#pragma unroll
                    for (int a = 0; a < AHEAD; ++a)
                        if ((r + a) * STEP < rows) {
                            const f32x4 x = *reinterpret_cast<const f32x4 *>(in + (r + a) * STEP * PITCH);
                            float v[4] = {x[0], x[1], x[2], x[3]};
                            finish4<TYPE, decltype(act)::value>(v, bias, res[a], E, seed, at, (r + a) * STEP, e + (unsigned long long)((r + a) * STEP) * np, n);
                        }
                }
            });
        } else if (n > 0)
#pragma unroll 2
            for (int r = 0; r < PASSES; ++r)
                if (r * STEP < rows) {
                    const f32x4 x = *reinterpret_cast<const f32x4 *>(in + r * STEP * PITCH);
                    float v[4] = {x[0], x[1], x[2], x[3]};
                    plain4<TYPE>(v, factor, E, at, r * STEP, n);
                }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

// Tiles of D in turn: blocks of one XCD (they are dealt round the 8 of them) get neighbouring tiles, whose operands then meet in its L2; among those,
// stripes of 8 tiles along q.
struct TilesD { int p, q; };
__device__ inline void tile_of(const TilesD &N, int block, int &tp, int &tq)
{
    const int all = N.p * N.q, even = all / 8 * 8;
    int i = block < even ? (block & 7) * (all / 8) + (block >> 3) : block;
    const int stripe = 8 * N.p, s = i / stripe, first = 8 * s, high = N.q - first < 8 ? N.q - first : 8;
    i -= s * stripe;
    tq = __builtin_amdgcn_readfirstlane(first + i % high);
    tp = __builtin_amdgcn_readfirstlane(i / high);
}

// D = P Q^T and what becomes of it.  BP x BQ results a block, WP x WQ waves; blockIdx.y: the part of the range of t, `t_part` long.
// 16 bits: bound by latency (1536 x 1024 x 768 fp16 12.7 us) and, at odd addresses, by the loads (8192 x 4096 x 4096 at odd elements 371 us).  fp32: by the arithmetic beside the matrix
// instructions, the parts (5.7 instructions an element) and the epilogue: 200003 x 256 x 256 with silu 177 us, 148 TFLOP/s, 8192 x 4096 x 4096 1293 us, 213 TFLOP/s (the library's
// 1822).  Two blocks of eight waves a compute unit, whose phases mix: three of four took 188, two of four (with 7.6 instructions an element) 247.
template <int TYPE, bool PCOL, bool QCOL, int BP, int BQ, int WP, int WQ, int BUFFERS, int AHEAD>
__global__ __launch_bounds__(64 * WP * WQ, TYPE == NET_F32 && BP * BQ == 128 * 128 && !QCOL ? 3 : 1) void k_product(MatD P, MatD Q, long long np, long long nq, long long nt, long long t_part, TilesD tiles, EpiD E)
{
    constexpr int THREADS = 64 * WP * WQ, BT = TYPE == NET_F32 ? 32 : 64, MT = BP / WP / 32, NT = BQ / WQ / 32;
    typedef Stage<TYPE, PCOL, BP, BT, THREADS> StageP;
    typedef Stage<TYPE, QCOL, BQ, BT, THREADS> StageQ;
    constexpr int TILE = StageP::LDS + StageQ::LDS;       // 16-bit elements
    constexpr int END = WP * WQ * end_floats(MT) * 4, BYTES = BUFFERS * TILE * 2 > END ? BUFFERS * TILE * 2 : END;
    __shared__ __attribute__((aligned(1024))) char s_mem[BYTES];
    short *lds = reinterpret_cast<short *>(s_mem);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wq = wave / WP;
    int tp, tq;
    tile_of(tiles, blockIdx.x, tp, tq);
    const long long p0 = (long long)tp * BP, q0 = (long long)tq * BQ;
    const int part = blockIdx.y;
    const long long t0 = part * t_part, t1 = t0 + t_part < nt ? t0 + t_part : nt;

    f32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.0f;

    int buffer = 0;
    auto compute = [&](int s) {
        const short *bp = lds + buffer * TILE, *bq = bp + StageP::LDS;
        constexpr int PL = StageP::PLANES;
        s16x8 a[MT][PL];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int k = 0; k < PL; ++k) a[i][k] = operand<PCOL, BP, BT>(bp + k * BP * BT, (wp * MT + i) * 32, s, lane);
        // of three parts each the six products that reach 2^-16 of the largest, the smaller parts of Q first
#pragma unroll
        for (int y = PL - 1; y >= 0; --y) {
            s16x8 b[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) b[j] = operand<QCOL, BQ, BT>(bq + y * BQ * BT, (wq * NT + j) * 32, s, lane);
#pragma unroll
            for (int x = PL - 1 - y; x >= 0; --x)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = mfma<TYPE>(a[i][x], b[j], acc[i][j]);
        }
    };
    const int whole = (int)((t1 - t0) / BT);
    const bool rest = t0 + (long long)whole * BT < t1;
    constexpr bool EARLY = BP * BQ <= 64 * 64;          // what is left of t is asked for first, where registers allow, and used last
    StageP rest_p;
    StageQ rest_q;
    if (EARLY && rest) {
        rest_p.load(P, p0, t0 + (long long)whole * BT, t1, tid);
        rest_q.load(Q, q0, t0 + (long long)whole * BT, t1, tid);
    }
    // AHEAD tiles on their way to registers, one or two in LDS.  EDGE: tiles that lie partly beyond the matrix along p or q in memory
    auto run = [&](auto edge) {
        constexpr bool EDGE = decltype(edge)::value;
        StageP sp[AHEAD];
        StageQ sq[AHEAD];
        const auto own_p = StageP::own(P, p0, tid);
        const auto own_q = StageQ::own(Q, q0, tid);
        // without a condition, so that the compiler can count the loads on their way: behind the last tile that one again, for nobody
        auto ask = [&](int k, StageP &x, StageQ &y) {
            const long long t = t0 + (long long)(k < whole ? k : whole - 1) * BT;
            if constexpr (EDGE && PCOL) x.load(P, p0, t, t1, tid);
            else x.fast(P, p0, t, own_p);
            if constexpr (EDGE && QCOL) y.load(Q, q0, t, t1, tid);
            else y.fast(Q, q0, t, own_q);
            __builtin_amdgcn_sched_barrier(0);         // in this order, which the waits go by
        };
        auto put = [&](int k, StageP &x, StageQ &y, int to) {
            x.store(lds + to * TILE, tid);
            y.store(lds + to * TILE + StageP::LDS, tid);
            ask(k + AHEAD, x, y);
        };
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) ask(k, sp[k], sq[k]);
        put(0, sp[0], sq[0], 0);
        __syncthreads();
        auto turn = [&](int k, StageP &np, StageQ &nq) {
            if constexpr (BUFFERS == 2) {
                // the next tile's writes to LDS among the products of this one
#pragma unroll
                for (int s = 0; s < BT / 32; ++s) compute(s);
                put(k + 1, np, nq, buffer ^ 1);
#pragma unroll
                for (int s = BT / 32; s < BT / 16; ++s) compute(s);
                buffer ^= 1;
            } else {
#pragma unroll
                for (int s = 0; s < BT / 16; ++s) compute(s);
                __syncthreads();
                put(k + 1, np, nq, 0);
            }
            __syncthreads();
        };
        int k = 0;
        for (; k + AHEAD <= whole; k += AHEAD)
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) turn(k + j, sp[(j + 1) % AHEAD], sq[(j + 1) % AHEAD]);
#pragma unroll
        for (int j = 0; j < AHEAD - 1; ++j)
            if (k + j < whole) turn(k + j, sp[(j + 1) % AHEAD], sq[(j + 1) % AHEAD]);
    };
    if (whole > 0) {
        if ((PCOL && p0 + BP > P.cols) || (QCOL && q0 + BQ > Q.cols)) run(Int<1>());
        else run(Int<0>());
    }
    if (rest) {
        buffer = 0;
        if (EARLY) {
            rest_p.store(lds, tid);
            rest_q.store(lds + StageP::LDS, tid);
        } else {
            StageP::bring(P, p0, t0 + (long long)whole * BT, t1, lds, tid);
            StageQ::bring(Q, q0, t0 + (long long)whole * BT, t1, lds + StageP::LDS, tid);
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < BT / 16; ++s) compute(s);
        __syncthreads();
    }

    auto again = [&](long long p, long long q, auto get, auto set) {            // rows beyond the last: the last one, whose results go nowhere
        p += lane & 31;
        q += lane & 31;
        p = p < np ? p : np - 1;
        q = q < nq ? q : nq - 1;
        auto at = [&](long long s) { return t0 + 16 * s + 8 * (lane >> 5); };
        made_again<f32x16>((t1 - t0 + 15) / 16, [&](float (&x)[8], long long s) { eight<NET_F32, PCOL>(x, P, p, at(s), t1); },
                           [&](float (&x)[8], long long s) { eight<NET_F32, QCOL>(x, Q, q, at(s), t1); }, get, set);
    };
    product_end<TYPE, !PCOL, MT, NT>(acc, reinterpret_cast<float *>(s_mem) + wave * end_floats(MT), lane, p0 + wp * MT * 32, q0 + wq * NT * 32, np, nq, part, E, again);
}

// The same for large products of 16-bit matrices whose rows lie at multiples of 16 bytes (and are, along p or q, a multiple of 8 long): 256 x 256 results a
// block of 8 waves.  Tiles of 64 t (whole lines of 128 bytes: with 32 the L2 has twice the requests) go from memory to LDS directly, into two buffers in turn.
// Bound by the matrix instructions and, with data that are not zeros, by power: 8192 x 4096 x 16384 bf16 932 us (1180 TFLOP/s; of zeros 826, the library's product
// 788).  128 squared through registers took 1736, tiles read straight before their products 1024; reads of a step among the products of the one before, over
// the barrier too, made it 932.
typedef __attribute__((address_space(3))) void lds_void;

// One operand's part of that: 256 rows (or, COL, columns) by 64 t are 32 KB, 1 KB an instruction, four instructions a wave.  A lane's chunk goes where the wave's place
// and its number say, so it is the chunk that is chosen: the one that place_row() or place_col() keep there.
template <bool COL> struct Direct {
    unsigned offset[4];                // bytes from the tile's first element
    const char *at;
    long long step;

    __device__ inline void begin(const MatD &M, long long b0, long long t0, int wave, int lane)
    {
        at = static_cast<const char *>(M.at) + (COL ? t0 * M.ld + b0 : b0 * M.ld + t0) * 2;
        step = (COL ? 64 * M.ld : 64) * 2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int u = wave * 4 + i;
            if constexpr (COL) {
                const int t = 2 * u + (lane >> 5), slot = lane & 31;
                long long c = (slot ^ (4 * (t & 3))) * 8;
                if (b0 + c >= M.cols) c = 0;                               // beyond the matrix: something of it, whose results go nowhere
                offset[i] = (unsigned)((t * M.ld + c) * 2);
            } else {
                const int r = 8 * u + (lane >> 3), slot = lane & 7;
                long long row = r;
                if (b0 + row >= M.rows) row = M.rows - 1 - b0;
                offset[i] = (unsigned)((row * M.ld + (slot ^ ((r >> 1) & 7)) * 8) * 2);
            }
        }
    }

    // By hand, since the compiler waits for all loads before it reads what such a load into the same array wrote once; who calls this waits.  A change of m0
    // needs a cycle before it is used here; nothing else in the kernel uses m0, which the compiler keeps no value in.
    __device__ inline void load(short *tile, int wave, bool more)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned to = (unsigned)(unsigned long long)(lds_void *)(tile + (wave * 4 + i) * 512);
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(offset[i]), "s"(at) : "memory");
        }
        at += more ? step : 0;
    }
};

template <int TYPE, bool PCOL, bool QCOL>
__global__ __launch_bounds__(512) void k_product_big(MatD P, MatD Q, long long np, long long nq, long long nt, long long t_part, TilesD tiles, EpiD E)
{
    constexpr int WP = 2, WAVES = 8, MT = 4, NT = 2, TILE = 256 * 64;
    static_assert(WAVES * end_floats(MT) * 4 <= 4 * TILE * 2, "results go through the buffers");
    __shared__ __attribute__((aligned(1024))) short s_mem[4 * TILE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wq = wave / WP;
    int tp, tq;
    tile_of(tiles, blockIdx.x, tp, tq);
    const long long p0 = (long long)tp * 256, q0 = (long long)tq * 256;
    const int part = blockIdx.y;
    const long long t0 = part * t_part, t1 = t0 + t_part < nt ? t0 + t_part : nt;
    f32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.0f;
    struct Step { s16x8 a[MT], b[NT]; };
    auto read = [&](Step &x, const short *bp, int s) {
#pragma unroll
        for (int i = 0; i < MT; ++i) x.a[i] = operand<PCOL, 256, 64>(bp, (wp * MT + i) * 32, s, lane);
#pragma unroll
        for (int j = 0; j < NT; ++j) x.b[j] = operand<QCOL, 256, 64>(bp + TILE, (wq * NT + j) * 32, s, lane);
    };
    auto multiply = [&](const Step &x) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = mfma<TYPE>(x.a[i], x.b[j], acc[i][j]);
    };
    constexpr int READS = MT * (PCOL ? 2 : 1) + NT * (QCOL ? 2 : 1), MFMAS = MT * NT, EACH = (READS + MFMAS - 1) / MFMAS;
    auto mixed = [&](int steps) {                      // a step's reads among the products of the one before
#pragma unroll
        for (int i = 0; i < steps * MFMAS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
    };
    const int whole = (int)((t1 - t0) / 64);
    if (whole > 0) {
        Direct<PCOL> dp;
        Direct<QCOL> dq;
        dp.begin(P, p0, t0, wave, lane);
        dq.begin(Q, q0, t0, wave, lane);
        int asked = 0;
        auto ask = [&](short *bp) {                    // behind the last tile: that one again, into a buffer that nobody reads
            ++asked;
            dp.load(bp, wave, asked < whole);
            dq.load(bp + TILE, wave, asked < whole);
        };
        auto arrived = [&] {                           // this wave's reads are done, and its loads
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0x0070);
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        };
        Step x, y;
        ask(s_mem);
        arrived();
        ask(s_mem + 2 * TILE);
        read(x, s_mem, 0);
        int at = 0;
        for (int k = 0; k < whole; ++k) {
            short *now = s_mem + at;
            at ^= 2 * TILE;
            read(y, now, 1);
            multiply(x);
            read(x, now, 2);
            multiply(y);
            read(y, now, 3);
            multiply(x);
            mixed(3);
            arrived();                                 // the next tile is there, and this one's buffer is read out
            ask(now);
            read(x, s_mem + at, 0);
            multiply(y);
            mixed(1);
        }
        __builtin_amdgcn_s_waitcnt(0x0070);
        __syncthreads();
    }
    if (t0 + whole * 64ll < t1) {                      // what is left of t
        Stage<TYPE, PCOL, 256, 64, 64 * WAVES>::bring(P, p0, t0 + whole * 64ll, t1, s_mem, tid);
        Stage<TYPE, QCOL, 256, 64, 64 * WAVES>::bring(Q, q0, t0 + whole * 64ll, t1, s_mem + TILE, tid);
        __syncthreads();
#pragma unroll 1
        for (int s = 0; s < 4; ++s) {
            Step x;
            read(x, s_mem, s);
            multiply(x);
        }
        __syncthreads();
    }
    product_end<TYPE, !PCOL, MT, NT>(acc, reinterpret_cast<float *>(s_mem) + wave * end_floats(MT), lane, p0 + wp * MT * 32, q0 + wq * NT * 32, np, nq, part, E, [](long long, long long, auto, auto) {});
}

// The parts' sums and what becomes of them, 256 neighbours p of one row q at a time.  SPLIT: a block's four waves add every fourth part each and the first of
// them finishes; else each wave has a strip of its own.  RESTS: `parts` parts more follow, of what rounding left of an operand.  They are left out where the others' sum
// is no finite number: a rest of 0 makes NaN of an infinity.
template <int TYPE, bool SPLIT, bool RESTS> __global__ __launch_bounds__(256) void k_parts(const float *__restrict__ part, long long part_stride, long long ldp, int parts, long long np, long long nq, EpiD E)
{
    constexpr int SUMS = RESTS ? 2 : 1;
    __shared__ float s_sum[SPLIT ? 3 * SUMS : 1][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = SPLIT ? wave : 0, step = SPLIT ? 4 : 1;
    const long long strips = (np + 255) / 256, all = strips * nq, each = SPLIT ? 1 : 4;
    const Seed seed = seed_of(E.drop);
    const float factor = factor_of<TYPE>(E);
    for (long long b = blockIdx.x * each + (SPLIT ? 0 : wave); b < all; b += gridDim.x * each) {
        const long long q = b / strips, p = b % strips * 256 + 4 * lane;
        const int n = np - p < 4 ? (int)(np - p) : 4;
        const Place<TYPE> to(E, q, p, 0);
        f32x4 sums[SUMS];
        Packed<TYPE, 4> r = {};
#pragma unroll
        for (int k = 0; k < SUMS; ++k) sums[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (n > 0) {
            if (!SPLIT || wave == 0) r = residual4<TYPE>(E, to, 0, n);
#pragma unroll
            for (int k = 0; k < SUMS; ++k) {
                const float *at = part + k * parts * part_stride + q * ldp + p;            // ldp is a multiple of 4
#pragma unroll 8
                for (int i = first; i < parts; i += step) sums[k] += *reinterpret_cast<const f32x4 *>(at + i * part_stride);
            }
        }
        if constexpr (SPLIT) {
            if (wave)
#pragma unroll
                for (int k = 0; k < SUMS; ++k) *reinterpret_cast<f32x4 *>(s_sum[3 * k + wave - 1] + 4 * lane) = sums[k];
            __syncthreads();
        }
        if (first == 0 && n > 0) {
            if constexpr (SPLIT)
#pragma unroll
                for (int k = 0; k < SUMS; ++k)
                    for (int w = 0; w < 3; ++w) sums[k] += *reinterpret_cast<const f32x4 *>(s_sum[3 * k + w] + 4 * lane);
            f32x4 sum = sums[0];
            if constexpr (RESTS)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] = fabsf(sum[i]) < INFINITY ? sum[i] + sums[1][i] : sum[i];
            float v[4] = {sum[0], sum[1], sum[2], sum[3]}, bias[4];
            if (E.mode == EPI_LAYER) {
                load_bias<TYPE>(bias, E, p, n);
                with_act(E.act, [&](auto act) { finish4<TYPE, decltype(act)::value>(v, bias, r, E, seed, to, 0, (unsigned long long)q * np + p, n); });
            } else plain4<TYPE>(v, factor, E, to, 0, n);
        }
        if constexpr (SPLIT) __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------------------- few rows

template <int TYPE> __device__ inline f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c)
{
    if constexpr (TYPE == NET_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

constexpr __host__ __device__ int few_ahead(bool f32, int mp, int nq) { return (f32 ? 2 : 4) * (mp * nq == 1 ? 2 : 1) / (f32 && mp * nq == 4 ? 2 : 1); }

// Forward with few rows: the weights are read once, past LDS, straight into the operands (16 outputs by 64 bytes an instruction), and that is all the time it takes.
// A block has MP times 16 outputs and all rows (NQ times 16); its waves have a stretch of t each and add up in LDS.  1 x 4096 x 16384 bf16 26.4 us where no cache holds the
// weights (5.1 TB/s), through the tiles 51.  Loads of steps that there are not cost as much as others: with a group too many a wave 31 us, and 8 x 1003 x 777
// 16.7 in place of 6.0.
template <int TYPE, int MP, int NQ>
__global__ __launch_bounds__(1024) void k_few(MatD W, MatD X, long long np, long long nq, long long nt, EpiD E)
{
    typedef typename ElemOf<TYPE>::type T;
    constexpr int PL = TYPE == NET_F32 ? 3 : 1, AHEAD = few_ahead(TYPE == NET_F32, MP, NQ);     // steps of 32 t on their way, a wave
    __shared__ __attribute__((aligned(16))) float s_sum[16][MP * NQ][64][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const long long p0 = blockIdx.x * (16ll * MP);
    // what the end needs, of the threads that take part in it: wave j has the results of outputs j / NQ and rows j % NQ
    const int j = threadIdx.x >> 6;
    const long long q = 16 * (j % NQ) + (lane & 15), p = p0 + 16 * (j / NQ) + 4 * (lane >> 4);
    const int n = j < MP * NQ && q < nq ? (np - p < 4 ? (int)(np - p) : 4) : 0;
    const Seed seed = seed_of(E.drop);
    float bias[4];
    load_bias<TYPE>(bias, E, p, n);
    Packed<TYPE, 4> r = {};
    const Place<TYPE> to(E, q, p, 0);
    if (n > 0) r = residual4<TYPE>(E, to, 0, n);

    // outputs and rows beyond the last: the last one, whose results go nowhere
    const T *w[MP], *x[NQ];
#pragma unroll
    for (int k = 0; k < MP; ++k) {
        const long long row = p0 + 16 * k + (lane & 15);
        w[k] = static_cast<const T *>(W.at) + (row < np ? row : np - 1) * W.ld + (lane >> 4) * 8;
    }
#pragma unroll
    for (int k = 0; k < NQ; ++k) {
        const long long row = 16 * k + (lane & 15);
        x[k] = static_cast<const T *>(X.at) + (row < nq ? row : nq - 1) * X.ld + (lane >> 4) * 8;
    }
    f32x4 acc[MP][NQ];
#pragma unroll
    for (int i = 0; i < MP; ++i)
#pragma unroll
        for (int k = 0; k < NQ; ++k) acc[i][k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    struct Step { Packed<TYPE, 8> a[MP], b[NQ]; };
    auto multiply = [&](const Step &c) {
        s16x8 u[MP][PL], v[PL];
#pragma unroll
        for (int i = 0; i < MP; ++i)
            if constexpr (PL == 3) split8(c.a[i], u[i]);
            else u[i][0] = __builtin_bit_cast(s16x8, u32x4{c.a[i].w[0], c.a[i].w[1], c.a[i].w[2], c.a[i].w[3]});
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
            if constexpr (PL == 3) split8(c.b[k], v);
            else v[0] = __builtin_bit_cast(s16x8, u32x4{c.b[k].w[0], c.b[k].w[1], c.b[k].w[2], c.b[k].w[3]});
#pragma unroll
            for (int y = PL - 1; y >= 0; --y)
#pragma unroll
                for (int z = PL - 1 - y; z >= 0; --z)
#pragma unroll
                    for (int i = 0; i < MP; ++i) acc[i][k] = mfma16<TYPE>(u[i][z], v[y], acc[i][k]);
        }
    };
    auto ask = [&](Step &y, long long s) {
#pragma unroll
        for (int k = 0; k < MP; ++k) y.a[k] = load_all<TYPE, 8>(w[k] + s * 32);
#pragma unroll
        for (int k = 0; k < NQ; ++k) y.b[k] = load_all<TYPE, 8>(x[k] + s * 32);
        __builtin_amdgcn_sched_barrier(0);             // in this order, which the waits go by
    };
    // a wave's stretch of groups of AHEAD steps, a group on its way; single steps behind them to one wave each
    const long long whole = nt / 32, groups = whole / AHEAD, first = groups * wave / waves * AHEAD, end = groups * (wave + 1) / waves * AHEAD;
    if (first < end) {
        Step c[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) ask(c[k], first + k);
        for (long long s = first + AHEAD; s < end; s += AHEAD)
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                multiply(c[k]);
                ask(c[k], s + k);
            }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) multiply(c[k]);
    }
    for (long long s = groups * AHEAD + wave; s < whole; s += waves) {
        Step c;
        ask(c, s);
        multiply(c);
    }
    if (whole * 32 < nt && wave == waves - 1) {
        Step c = {};
        const long long left = nt - whole * 32 - (lane >> 4) * 8;
        if (left > 0) {
#pragma unroll
            for (int k = 0; k < MP; ++k) c.a[k] = load_some<TYPE, 8>(w[k] + whole * 32, left < 8 ? (int)left : 8);
#pragma unroll
            for (int k = 0; k < NQ; ++k) c.b[k] = load_some<TYPE, 8>(x[k] + whole * 32, left < 8 ? (int)left : 8);
        }
        multiply(c);
    }
    if constexpr (TYPE == NET_F32) {
        // of its own steps: the stretch, single ones, and the end
        const long long rest = whole - groups * AHEAD - wave, stretch = end - first, steps = stretch + (rest > 0 ? (rest + waves - 1) / waves : 0) + (whole * 32 < nt && wave == waves - 1);
        auto at = [&](long long s) {
            const bool last = whole * 32 < nt && wave == waves - 1 && s == steps - 1;
            return 32 * (s < stretch ? first + s : last ? whole : groups * AHEAD + wave + (s - stretch) * waves) + 8 * (lane >> 4);
        };
#pragma unroll
        for (int i = 0; i < MP; ++i)
#pragma unroll
            for (int k = 0; k < NQ; ++k) {
                const long long p = p0 + 16 * i + (lane & 15), q = 16 * k + (lane & 15);
                made_again(acc[i][k], steps, [&](float (&x)[8], long long s) { eight<NET_F32, false>(x, W, p < np ? p : np - 1, at(s), nt); },
                           [&](float (&x)[8], long long s) { eight<NET_F32, false>(x, X, q < nq ? q : nq - 1, at(s), nt); });
            }
    }
#pragma unroll
    for (int i = 0; i < MP; ++i)
#pragma unroll
        for (int k = 0; k < NQ; ++k) *reinterpret_cast<f32x4 *>(s_sum[wave][i * NQ + k][lane]) = acc[i][k];
    __syncthreads();
    if (n <= 0) return;
    f32x4 sum = *reinterpret_cast<const f32x4 *>(s_sum[0][j][lane]);
#pragma unroll 4
    for (int i = 1; i < waves; ++i) sum += *reinterpret_cast<const f32x4 *>(s_sum[i][j][lane]);
    float v[4] = {sum[0], sum[1], sum[2], sum[3]};
    with_act(E.act, [&](auto act) { finish4<TYPE, decltype(act)::value>(v, bias, r, E, seed, to, 0, (unsigned long long)q * np + p, n); });
}

// ---------------------------------------------------------------------------------------------------------------- narrow layers

// Chunks of 8 elements of dZ in LDS, [rows][B]: read along the rows as an operand of dX, and turned as one of dweight.  16 rows have one chunk in 16 different places,
// and four rows 32 neighbours in 8.
template <int B> __device__ inline int place_both(int t, int c) { return t * B + ((c ^ 4 * (t & 3) ^ (t >> 2 & 3)) * 8); }

// What dZ is made from.
struct DzD { MatD G, Z; int z_f32, act; float beta; DropD drop; };

// Eight elements of it in fp32, k of them at (q(k), n(k)); zeros where there is none.
template <int TYPE, class Q, class N> __device__ inline void dz_eight(float (&x)[8], const DzD &D, const Seed &seed, Q q, N n)
{
    typedef typename ElemOf<TYPE>::type T;
    const long long rows = D.G.rows, cols = D.G.cols;
    float z[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const long long r = q(k) < rows ? q(k) : rows - 1, c = n(k) < cols ? n(k) : cols - 1;
        x[k] = widen<TYPE>(static_cast<const T *>(D.G.at)[r * D.G.ld + c]);
        z[k] = 0.0f;
        if (D.act != ACT_NONE) z[k] = TYPE == NET_F32 || D.z_f32 ? static_cast<const float *>(D.Z.at)[r * D.Z.ld + c] : widen<TYPE>(static_cast<const T *>(D.Z.at)[r * D.Z.ld + c]);
    }
    with_act(D.act, [&](auto kind) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= slope_of<decltype(kind)::value>(z[k], D.beta);
    });
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (D.drop.mode == 1) {
            const unsigned long long e = (unsigned long long)q(k) * cols + n(k);
            const uint4 w = philox(e >> 2, seed.offset, seed.seed);
            const unsigned word = e & 2 ? (e & 1 ? w.w : w.z) : (e & 1 ? w.y : w.x);
            x[k] = word >= D.drop.least ? x[k] * D.drop.scale : 0.0f;
            __builtin_amdgcn_sched_barrier(0);         // one after another: few registers
        }
        if (D.drop.mode == 2 || q(k) >= rows || n(k) >= cols) x[k] = 0.0f;
    }
}

// The backward pass of a layer of at most B inputs and B outputs, in one pass over its rows: G, Z and X are read once, dX is written, dweight stays in registers and the
// sums for dbias too, a part for each block.  The weights lie in LDS.  A block takes 32 rows at a time, the next ones on their way meanwhile.
//   dweight: WP x WQ waves share the B x B results, t = rows.  dX: 32 inputs a wave, t = outputs; where there are twice the waves, two share those.
// RESTS (16 bits): dZ goes in as two parts, itself rounded and what that leaves, for layers whose dZ has too few values to average its rounding out.  A rest of 0 would make
// a NaN of another operand's infinity: dX has sums of its own for the rests, and leaves them out where the others' are no finite numbers; dweight (whose second sums would
// take 437 registers, one block a compute unit) makes such results again.  Forward and backward of 1024 x 64 x 64 bf16, gelu, 20.8 us, by one part 16.6; of
// 65536 x 128 x 128, silu, 56, by one 50: there one part is taken.
// 65536 x 128 x 128 fp32 40 us (134 MB, 3.3 TB/s; matrix pipe busy 21 % of the time, vector instructions 26), bf16 31 (67 MB, 2.2 TB/s; 4 and 31): four barriers every 32
// rows, between which loads, parts and products follow one another.  For 256 x 256 in 16 bits, one
// block a compute unit, that took 624 us against 556 of the other kernels, so B is 128.
template <int TYPE, int B, int WAVES, bool RESTS>
__global__ __launch_bounds__(64 * WAVES, 2) void k_narrow(DzD D, MatD X, MatD W, void *dx, long long lddx, float *__restrict__ dw, long long ldw, double *__restrict__ sums)
{
    typedef typename ElemOf<TYPE>::type T;
    constexpr int THREADS = 64 * WAVES, R = 32, PL = TYPE == NET_F32 ? 3 : 1, PZ = TYPE == NET_F32 ? 3 : RESTS ? 2 : 1, WP = WAVES / 2, WQ = 2, MT = B / WP / 32, NT = B / WQ / 32;
    constexpr int HALVES = WAVES * 32 / B, STEPS = B / 16 / HALVES, UNITS = R * B / 8 / THREADS, PER_ROW = B / 8;
    static_assert(MT >= 1 && (HALVES == 1 || HALVES == 2) && THREADS % PER_ROW == 0, "shape");
    __shared__ __attribute__((aligned(1024))) short s_w[PL * B * B];
    __shared__ __attribute__((aligned(1024))) short s_in[(PZ + PL) * R * B];
    static_assert(HALVES * R * B * 4 <= (PZ + PL) * R * B * 2, "dX goes through the inputs' place");
    short *s_dz = s_in, *s_x = s_in + PZ * R * B;
    float *s_out = reinterpret_cast<float *>(s_in);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wq = wave / WP;
    const long long rows = D.G.rows, outputs = D.G.cols, inputs = X.cols;
    const Seed seed = seed_of(D.drop);
    if (dx) Stage<TYPE, true, B, B, THREADS>::bring(W, 0, 0, outputs, s_w, tid);

    f32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.0f;
    double db[8];                      // columns may cancel
#pragma unroll
    for (int i = 0; i < 8; ++i) db[i] = 0.0;

    Packed<TYPE, 8> g[UNITS];
    unsigned z[UNITS][8];
    Stage<TYPE, true, B, R, THREADS> sx;
    const int c8 = tid % PER_ROW * 8, left = outputs - c8 < 8 ? (int)(outputs - c8) : 8;
    constexpr int APART = THREADS / PER_ROW;
    const int r0 = tid / PER_ROW;
    const long long own_g = r0 * D.G.ld + c8, own_z = r0 * D.Z.ld + c8;
    auto load = [&](long long q0) {
        const T *at_g = static_cast<const T *>(D.G.at) + q0 * D.G.ld;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            g[i] = Packed<TYPE, 8>();
#pragma unroll
            for (int k = 0; k < 8; ++k) z[i][k] = 0u;
            if (q0 + r0 + i * APART < rows && left > 0) {
                g[i] = load_some<TYPE, 8>(at_g + i * APART * D.G.ld + own_g, left);
                if (D.act == ACT_NONE) continue;
                if (D.z_f32) {
                    const auto x = load_some<NET_F32, 8>(static_cast<const float *>(D.Z.at) + (q0 + i * APART) * D.Z.ld + own_z, left);
#pragma unroll
                    for (int k = 0; k < 8; ++k) z[i][k] = x.w[k];
                } else {
                    const auto x = load_some<TYPE, 8>(static_cast<const T *>(D.Z.at) + (q0 + i * APART) * D.Z.ld + own_z, left);
#pragma unroll
                    for (int k = 0; k < x.WORDS; ++k) z[i][k] = x.w[k];
                }
            }
        }
        if (dw) sx.load(X, 0, q0, rows, tid);
    };

    const long long stride = (long long)gridDim.x * R;
    long long q0 = (long long)blockIdx.x * R;
    Power power = {1.0f, 1.0f};
    if constexpr (TYPE == NET_F16)
        if (D.act != ACT_NONE || D.drop.mode == 1) {       // a block's own (see power_of): its rows of G are read twice
            __shared__ unsigned s_most[WAVES];
            Largest most;
            for (long long q = q0 + r0; q < rows + r0; q += stride)
#pragma unroll
                for (int i = 0; i < UNITS; ++i)
                    if (q + i * APART < rows && left > 0) most.add(load_some<TYPE, 8>(static_cast<const T *>(D.G.at) + (q + i * APART) * D.G.ld + c8, left));
            power = power_of(largest_of<WAVES>(most.bits(), s_most), D.drop);
        }
    load(q0);
    for (; q0 < rows; q0 += stride) {
        with_act(D.act, [&](auto kind) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int u = tid + i * THREADS, r = u / PER_ROW;
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[k] = g[i].wide(k);
                    if constexpr (decltype(kind)::value != ACT_NONE) {
                        float zk;
                        if (TYPE == NET_F32 || D.z_f32) zk = __uint_as_float(z[i][k]);
                        else {
                            Packed<TYPE, 8> x;
#pragma unroll
                            for (int m = 0; m < x.WORDS; ++m) x.w[m] = z[i][m];
                            zk = x.wide(k);
                        }
                        v[k] *= slope_of<decltype(kind)::value>(zk, D.beta);
                    }
                }
                drop<8>(v, (unsigned long long)(q0 + r) * outputs + c8, D.drop, seed);
                Packed<TYPE, 8> x;
#pragma unroll
                for (int k = 0; k < 8; ++k) db[k] += v[k];
                if constexpr (TYPE == NET_F32) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x.w[k] = __float_as_uint(v[k]);
                    s16x8 part[3];
                    split8(x, part);
#pragma unroll
                    for (int k = 0; k < 3; ++k) *reinterpret_cast<s16x8 *>(s_dz + k * R * B + place_both<B>(r, u % PER_ROW)) = part[k];
                } else {
                    if constexpr (TYPE == NET_F16)
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] *= power.to;
#pragma unroll
                    for (int k = 0; k < 4; ++k) x.w[k] = (unsigned)narrow<TYPE>(v[2 * k]) | (unsigned)narrow<TYPE>(v[2 * k + 1]) << 16;
                    *reinterpret_cast<u32x4 *>(s_dz + place_both<B>(r, u % PER_ROW)) = u32x4{x.w[0], x.w[1], x.w[2], x.w[3]};
                    if constexpr (RESTS) {             // and what that leaves, none where it is no finite number
                        float rest[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) rest[k] = fabsf(x.wide(k)) < INFINITY ? v[k] - x.wide(k) : 0.0f;
#pragma unroll
                        for (int k = 0; k < 4; ++k) x.w[k] = (unsigned)narrow<TYPE>(rest[2 * k]) | (unsigned)narrow<TYPE>(rest[2 * k + 1]) << 16;
                        *reinterpret_cast<u32x4 *>(s_dz + R * B + place_both<B>(r, u % PER_ROW)) = u32x4{x.w[0], x.w[1], x.w[2], x.w[3]};
                    }
                }
            }
        });
        if (dw) sx.store(s_x, tid);
        if (q0 + stride < rows) load(q0 + stride);
        __syncthreads();

        constexpr int PA[6] = {0, 1, 2, 0, 1, 0}, PB[6] = {2, 1, 0, 1, 0, 0};
        if (dw)
#pragma unroll
        for (int s = 0; s < R / 16; ++s) {
            s16x8 a[MT][PL], b[NT][PZ];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int k = 0; k < PL; ++k) a[i][k] = operand<true, B, R>(s_x + k * R * B, (wp * MT + i) * 32, s, lane);
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int k = 0; k < PZ; ++k) b[j][k] = turned([](int t, int c) { return place_both<B>(t, c); }, s_dz + k * R * B, (wq * NT + j) * 32, s, lane);
#pragma unroll
            for (int u = 0; u < (PL == 1 ? PZ : 6); ++u)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = mfma<TYPE>(a[i][PL == 1 ? 0 : PA[u]], b[j][PL == 1 ? PZ - 1 - u : PB[u]], acc[i][j]);
        }
        if (!dx) {
            __syncthreads();
            continue;
        }
        f32x16 d, rest;
#pragma unroll
        for (int k = 0; k < 16; ++k) d[k] = rest[k] = 0.0f;
        const int pb = wave % (B / 32) * 32, half = wave / (B / 32);
#pragma unroll 4
        for (int s = 0; s < STEPS; ++s) {
            const int step = half * STEPS + s;
            s16x8 a[PL], b[PZ];
#pragma unroll
            for (int k = 0; k < PL; ++k) a[k] = operand<true, B, B>(s_w + k * B * B, pb, step, lane);
#pragma unroll
            for (int k = 0; k < PZ; ++k) b[k] = *reinterpret_cast<const s16x8 *>(s_dz + k * R * B + place_both<B>(lane & 31, 2 * step + (lane >> 5)));
#pragma unroll
            for (int u = 0; u < (PL == 1 ? 1 : 6); ++u) d = mfma<TYPE>(a[PL == 1 ? 0 : PA[u]], b[PL == 1 ? 0 : PB[u]], d);
            if constexpr (RESTS) rest = mfma<TYPE>(a[0], b[1], rest);
        }
        if constexpr (RESTS)
#pragma unroll
            for (int k = 0; k < 16; ++k) d[k] = fabsf(d[k]) < INFINITY ? d[k] + rest[k] : d[k];
        __syncthreads();
        // row q of dX: B floats, its quarters of 16 bytes turned by q so that the lanes' writes spread over the banks
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
            const int q = lane & 31, quad = (pb + 8 * gq + 4 * (lane >> 5)) / 4;
            *reinterpret_cast<f32x4 *>(s_out + half * R * B + q * B + ((quad ^ (q & 15)) * 4)) = f32x4{d[4 * gq], d[4 * gq + 1], d[4 * gq + 2], d[4 * gq + 3]};
        }
        bool bad = false;
#pragma unroll
        for (int k = 0; k < 16; ++k) bad |= !(fabsf(d[k]) < INFINITY);
        if (TYPE == NET_F32 && __any(bad)) {
            const long long p = pb + (lane & 31) < inputs ? pb + (lane & 31) : inputs - 1, q = q0 + (lane & 31);
            float *row = s_out + half * R * B + (lane & 31) * B;
            auto place = [&](int i) { return row + ((((pb + 8 * (i >> 2) + 4 * (lane >> 5)) / 4 ^ (lane & 15)) * 4) + (i & 3)); };
            auto at = [&](long long s) { return 16 * (half * STEPS + s) + 8 * (lane >> 5); };
            made_again<f32x16>(STEPS, [&](float (&x)[8], long long s) { eight<TYPE, true>(x, W, p, at(s), outputs); },
                               [&](float (&x)[8], long long s) { dz_eight<TYPE>(x, D, seed, [&](int) { return q; }, [&](int k) { return at(s) + k; }); },
                               [&](int i) { return *place(i); }, [&](int i, float v) { *place(i) = v; });
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < R * B / 4 / THREADS; ++i) {
            const int u = tid + i * THREADS, r = u / (B / 4), quad = u % (B / 4);
            const long long q = q0 + r, p = 4 * quad;
            f32x4 x = *reinterpret_cast<const f32x4 *>(s_out + r * B + ((quad ^ (r & 15)) * 4));
            if constexpr (HALVES == 2) x += *reinterpret_cast<const f32x4 *>(s_out + R * B + r * B + ((quad ^ (r & 15)) * 4));
            if (q < rows && p < inputs) {
                const int n = inputs - p < 4 ? (int)(inputs - p) : 4;
                float v[4] = {x[0], x[1], x[2], x[3]};
                if constexpr (TYPE == NET_F16)
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] *= power.back;
                store_some<TYPE, 4>(static_cast<T *>(dx) + q * lddx + p, v, n);
            }
        }
        __syncthreads();
    }

    // dweight's part, [outputs][ldw]
    float *part = dw + (long long)blockIdx.x * outputs * ldw;
    auto put = [&](f32x16 v, int h) {
        if constexpr (TYPE == NET_F16) v *= power.back;
        const long long pb = (wp * MT + h / NT) * 32, qb = (wq * NT + h % NT) * 32;
        if constexpr (TYPE == NET_F32 || RESTS) {
            const long long p = pb + (lane & 31) < inputs ? pb + (lane & 31) : inputs - 1, q = qb + (lane & 31), groups = (rows - (long long)blockIdx.x * R + stride - 1) / stride;
            auto at = [&](long long s) { return (blockIdx.x + (s >> 1) * gridDim.x) * R + 16 * (s & 1) + 8 * (lane >> 5); };
            made_again(v, 2 * groups, [&](float (&x)[8], long long s) { eight<TYPE, true>(x, X, p, at(s), rows); },
                       [&](float (&x)[8], long long s) { dz_eight<TYPE>(x, D, seed, [&](int k) { return at(s) + k; }, [&](int) { return q; }); });
        }
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
            const long long p = pb + 8 * gq + 4 * (lane >> 5), q = qb + (lane & 31);
            if (p < inputs && q < outputs) *reinterpret_cast<f32x4 *>(part + q * ldw + p) = f32x4{v[4 * gq], v[4 * gq + 1], v[4 * gq + 2], v[4 * gq + 3]};
        }
    };
    if (dw) {
        if constexpr (TYPE == NET_F32 || RESTS) {
#pragma unroll 1
            for (int h = 0; h < MT * NT; ++h) {        // one copy of the code
                f32x16 v;
#pragma unroll
                for (int k = 0; k < MT * NT; ++k)
                    if (k == h) v = acc[k / NT][k % NT];
                put(v, h);
            }
        } else
#pragma unroll
            for (int h = 0; h < MT * NT; ++h) put(acc[h / NT][h % NT], h);
    }
    if (!sums) return;
    // dbias' part: a thread's columns are those of every PER_ROW-th other
    __syncthreads();
    double *s_db = reinterpret_cast<double *>(s_in);
    static_assert(THREADS * 8 * 8 <= (PZ + PL) * R * B * 2, "dbias goes through the inputs' place");
#pragma unroll
    for (int k = 0; k < 8; ++k) s_db[tid / PER_ROW * B + c8 + k] = db[k];
    __syncthreads();
    for (int n = tid; n < outputs; n += THREADS) {
        double all = 0.0;
        for (int r = 0; r < THREADS / PER_ROW; ++r) all += s_db[r * B + n];
        sums[blockIdx.x * outputs + n] = all;
    }
}

// The parts of k_narrow added up, dweight (of 256 neighbours by a block) and behind it dbias (of 64).
template <int TYPE> __global__ __launch_bounds__(1024) void k_narrow_end(const float *__restrict__ dw, long long ldp, int parts, long long inputs, long long outputs, void *out, long long ldo,
                                                                         const double *__restrict__ sums, void *dbias, int bias_f32, int blocks_dw)
{
    __shared__ __attribute__((aligned(16))) float s_sum[16][256];
    double (*s_db)[64] = reinterpret_cast<double (*)[64]>(s_sum);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if ((int)blockIdx.x < blocks_dw) {
        // rows of ldp floats, a multiple of 4, one after another
        const long long e = blockIdx.x * 256ll + 4 * lane, all = outputs * ldp;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        if (e < all)
#pragma unroll 8
            for (int i = wave; i < parts; i += 16) sum += *reinterpret_cast<const f32x4 *>(dw + i * all + e);
        *reinterpret_cast<f32x4 *>(s_sum[wave] + 4 * lane) = sum;
        __syncthreads();
        if (wave || e >= all) return;
        for (int w = 1; w < 16; ++w) sum += *reinterpret_cast<const f32x4 *>(s_sum[w] + 4 * lane);
        const long long q = e / ldp, p = e % ldp;
        const float v[4] = {sum[0], sum[1], sum[2], sum[3]};
        store_some<TYPE, 4>(static_cast<typename ElemOf<TYPE>::type *>(out) + q * ldo + p, v, inputs - p < 4 ? (int)(inputs - p) : 4);
        return;
    }
    const long long c = (blockIdx.x - blocks_dw) * 64ll + lane;
    double all = 0.0;
    if (c < outputs)
#pragma unroll 16
        for (int b = wave; b < parts; b += 16) all += sums[b * outputs + c];
    s_db[wave][lane] = all;
    __syncthreads();
    if (wave || c >= outputs) return;
    for (int w = 1; w < 16; ++w) all += s_db[w][lane];
    if (bias_f32) static_cast<float *>(dbias)[c] = (float)all;
    else static_cast<typename ElemOf<TYPE>::type *>(dbias)[c] = narrow<TYPE>((float)all);
}

// ---------------------------------------------------------------------------------------------------------------- elementwise

// `tx` threads (a power of 2) side by side, each with V neighbours of a row, and 256 / tx rows: a block's rows at a time.  Blocks take those in turn (a stretch for
// each would use the memory's channels less evenly).  The last row may be a shorter one, of `last` elements: of memory without gaps.
struct RowsD { long long rows, cols, last; int tx_bits; };

// f(first row, step, rows, neighbours in the matrix, Int<whole vectors?>) for a thread's rows.  Whole vectors first, in a loop of its own: what ends of rows need takes
// registers, and with them in one loop a dropout of 134 M bf16 took 245 us in place of 150.
template <int V, class F> __device__ inline void rows_of(const RowsD &N, long long c, int ty, F f)
{
    const long long at_once = 256 >> N.tx_bits, first = blockIdx.y * at_once + ty, step = gridDim.y * at_once, even = N.last == N.cols ? N.rows : N.rows - 1;
    const int n = N.cols - c < V ? (int)(N.cols - c) : V, end = N.last - c < V ? (int)(N.last - c) : V;
    if (n == V) f(first, step, even, V, Int<1>());
    else if (n > 0) f(first, step, even, n, Int<0>());
    if (even < N.rows && end > 0 && (N.rows - 1 - first) % step == 0 && first < N.rows) f(N.rows - 1, step, N.rows, end, Int<0>());
}

template <int TYPE, int V, bool WHOLE> __device__ inline Packed<TYPE, V> load_row(const MatD &M, long long q, long long c, int n)
{
    const typename ElemOf<TYPE>::type *at = static_cast<const typename ElemOf<TYPE>::type *>(M.at) + q * M.ld + c;
    if constexpr (WHOLE) return load_all<TYPE, V>(at);
    else return load_some<TYPE, V>(at, n);
}

// Y = R + drop(X).  Two rows' loads before the first one's store, which might be to the same memory.  Bound by memory: 134 M bf16 without residual 108 us (5.0 TB/s; with p = 0, a copy,
// 101), with residual 166 (4.9 TB/s; p = 0: 164).  Beside that vector instructions, most of them Philox's, keep the SIMDs busy for 65 % of the time, with residual 43 %.
template <int TYPE, int V> __global__ __launch_bounds__(256) void k_dropout(RowsD N, MatD X, MatD R, void *y, long long ldy, DropD D)
{
    typedef typename ElemOf<TYPE>::type T;
    const int x = threadIdx.x & ((1 << N.tx_bits) - 1), ty = threadIdx.x >> N.tx_bits;
    const Seed seed = seed_of(D);
    for (long long c = (((long long)blockIdx.x << N.tx_bits) + x) * V; c < N.cols; c += ((long long)gridDim.x << N.tx_bits) * V)
        rows_of<V>(N, c, ty, [&](long long first, long long step, long long rows, int n, auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            constexpr int U = WHOLE ? 2 : 1;
#pragma unroll 1
            for (long long q = first; q < rows; q += U * step) {
                Packed<TYPE, V> a[U], r[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u == 0 || q + u * step < rows) {
                        a[u] = load_row<TYPE, V, WHOLE>(X, q + u * step, c, n);
                        if (R.at) r[u] = load_row<TYPE, V, WHOLE>(R, q + u * step, c, n);
                    }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u == 0 || q + u * step < rows) {
                        float v[V];
#pragma unroll
                        for (int i = 0; i < V; ++i) v[i] = a[u].wide(i);
                        drop<V>(v, (unsigned long long)(q + u * step) * N.cols + c, D, seed);
                        if (R.at)
#pragma unroll
                            for (int i = 0; i < V; ++i) v[i] += r[u].wide(i);
                        store_some<TYPE, V>(static_cast<T *>(y) + (q + u * step) * ldy + c, v, WHOLE ? V : n);
                    }
            }
        });
}

// fp16: the largest finite |G| of each of LARGEST_BLOCKS blocks, for power_of().
constexpr int LARGEST_BLOCKS = 1024;
__global__ __launch_bounds__(256) void k_largest(RowsD N, MatD G, unsigned *__restrict__ most)
{
    __shared__ unsigned s_most[4];
    constexpr int U = 4;                               // loads before the first one's use
    const long long step = 256 >> N.tx_bits, first = blockIdx.x * U * step + (threadIdx.x >> N.tx_bits);
    Largest m;
    for (long long c = (threadIdx.x & ((1 << N.tx_bits) - 1)) * 8; c < N.cols; c += 8ll << N.tx_bits) {
        const unsigned short *at = static_cast<const unsigned short *>(G.at) + c;
        const int n = N.cols - c < 8 ? (int)(N.cols - c) : 8;
#pragma unroll 1
        for (long long q = first; q < N.rows; q += gridDim.x * U * step) {
            if (n == 8 && q + (U - 1) * step < N.rows) {
                Packed<NET_F16, 8> x[U];
#pragma unroll
                for (int u = 0; u < U; ++u) x[u] = load_all<NET_F16, 8>(at + (q + u * step) * G.ld);
#pragma unroll
                for (int u = 0; u < U; ++u) m.add(x[u]);
            } else
                for (int u = 0; u < U && q + u * step < N.rows; ++u) m.add(load_some<NET_F16, 8>(at + (q + u * step) * G.ld, n));
        }
    }
    const unsigned all = largest_of<4>(m.bits(), s_most);
    if (threadIdx.x == 0) most[blockIdx.x] = all;
}

// dZ = drop(G act'(Z)), and the sums of its columns over a block's rows (either may be NULL).  134 M bf16 with Z in fp32 241 us (1.07 GB, 4.5 TB/s), vector instructions busy
// for 46 % of that.
// fp16: dZ is written times a power of two, which goes by k_largest's `most` (where that is not NULL) and whose inverse goes to *factor.
// rest (16 bits, or NULL): what the rounding leaves of dZ, none where it is no finite number.
template <int TYPE, int V> __global__ __launch_bounds__(256) void k_dz(RowsD N, MatD G, MatD Z, int z_f32, int act, float beta, DropD D, void *dz, long long lddz, double *__restrict__ sums,
                                                                       const unsigned *__restrict__ most, float *__restrict__ factor, void *rest)
{
    typedef typename ElemOf<TYPE>::type T;
    __shared__ double s_sum[256 * V];
    const int tx = 1 << N.tx_bits, x = threadIdx.x & (tx - 1), ty = threadIdx.x >> N.tx_bits;
    float to = 1.0f;
    if constexpr (TYPE == NET_F16)
        if (most) {
            __shared__ unsigned s_most[4];
            unsigned m = 0;
#pragma unroll
            for (int i = 0; i < LARGEST_BLOCKS; i += 256) {
                const unsigned other = most[threadIdx.x + i];
                m = other > m ? other : m;
            }
            const Power power = power_of(largest_of<4>(m, s_most), D);
            to = power.to;
            if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *factor = power.back;
        }
    const long long c = (((long long)blockIdx.x << N.tx_bits) + x) * V;
    const Seed seed = seed_of(D);
    double sum[V];                     // columns may cancel
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0.0;
    with_act(act, [&](auto kind) {
        constexpr int ACT = decltype(kind)::value;
        rows_of<V>(N, c, ty, [&](long long first, long long step, long long rows, int n, auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            auto go = [&](auto wide_z) {
                constexpr int ZT = decltype(wide_z)::value ? NET_F32 : TYPE, U = WHOLE ? 2 : 1;
#pragma unroll 1
                for (long long q = first; q < rows; q += U * step) {
                    Packed<TYPE, V> g[U];
                    Packed<ZT, V> z[U];
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (u == 0 || q + u * step < rows) {
                            g[u] = load_row<TYPE, V, WHOLE>(G, q + u * step, c, n);
                            if constexpr (ACT != ACT_NONE) z[u] = load_row<ZT, V, WHOLE>(Z, q + u * step, c, n);
                        }
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (u == 0 || q + u * step < rows) {
                            float v[V];
#pragma unroll
                            for (int i = 0; i < V; ++i) {
                                v[i] = g[u].wide(i);
                                if constexpr (ACT != ACT_NONE) v[i] *= slope_of<ACT>(z[u].wide(i), beta);
                            }
                            drop<V>(v, (unsigned long long)(q + u * step) * N.cols + c, D, seed);
#pragma unroll
                            for (int i = 0; i < V; ++i) sum[i] += v[i];
                            if constexpr (TYPE == NET_F16)
#pragma unroll
                                for (int i = 0; i < V; ++i) v[i] *= to;
                            if (dz) store_some<TYPE, V>(static_cast<T *>(dz) + (q + u * step) * lddz + c, v, WHOLE ? V : n);
                            if (TYPE != NET_F32 && rest) {
#pragma unroll
                                for (int i = 0; i < V; ++i) {
                                    const float high = widen<TYPE>(narrow<TYPE>(v[i]));
                                    v[i] = fabsf(high) < INFINITY ? v[i] - high : 0.0f;
                                }
                                store_some<TYPE, V>(static_cast<T *>(rest) + (q + u * step) * lddz + c, v, WHOLE ? V : n);
                            }
                        }
                }
            };
            if (ACT != ACT_NONE && TYPE != NET_F32 && z_f32) go(Int<1>());
            else go(Int<TYPE == NET_F32>());
        });
    });
    if (!sums) return;
#pragma unroll
    for (int i = 0; i < V; ++i) s_sum[threadIdx.x * V + i] = sum[i];
    __syncthreads();
    for (int i = threadIdx.x; i < tx * V; i += 256) {
        double all = 0.0;
        for (int r = 0; r < 256 / tx; ++r) all += s_sum[r * tx * V + i];
        const long long k = ((long long)blockIdx.x << N.tx_bits) * V + i;
        if (k < N.cols) sums[blockIdx.y * N.cols + k] = all;
    }
}

// dbias from the blocks' sums: 64 columns a block, every 16th sum a wave
template <int TYPE> __global__ __launch_bounds__(1024) void k_dbias(const double *__restrict__ sums, int blocks, long long cols, void *out)
{
    __shared__ double s_sum[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long c = blockIdx.x * 64ll + lane;
    double all = 0.0;
    if (c < cols)
#pragma unroll 16
        for (int b = wave; b < blocks; b += 16) all += sums[b * cols + c];
    s_sum[wave][lane] = all;
    __syncthreads();
    if (wave == 0 && c < cols) {
        for (int w = 1; w < 16; ++w) all += s_sum[w][lane];
        static_cast<typename ElemOf<TYPE>::type *>(out)[c] = narrow<TYPE>((float)all);
    }
}

}  // namespace fs
