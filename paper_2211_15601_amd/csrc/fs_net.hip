// C ABI of the networks' layers (see include/fastsnarf_net.h): argument checks, shapes of launches, launches.  gfx950 only.
#include "../../include/fastsnarf_net.h"
#include "fs_net_kernels.hpp"

#include <hip/hip_runtime.h>
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

using namespace fs;

static_assert(int(FS_FLOAT_FULL) == NET_F32 && int(FS_FLOAT_BRAIN) == NET_BF16 && int(FS_FLOAT_HALF) == NET_F16, "types");
static_assert(int(FS_ACT_NONE) == ACT_NONE && int(FS_ACT_RELU) == ACT_RELU && int(FS_ACT_GELU) == ACT_GELU && int(FS_ACT_SILU) == ACT_SILU &&
              int(FS_ACT_SOFTPLUS) == ACT_SOFTPLUS, "activations");

namespace {

thread_local char net_err[256];

fs_status fail(fs_status s, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(net_err, sizeof net_err, fmt, ap);
    va_end(ap);
    return s;
}

fs_status launch_status(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FS_OK : fail(FS_E_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

bool type_ok(int32_t type) { return type == FS_FLOAT_FULL || type == FS_FLOAT_BRAIN || type == FS_FLOAT_HALF; }
int size_of(int32_t type) { return type == FS_FLOAT_FULL ? 4 : 2; }

// Memory of the current device?  The lookup in the runtime takes as long as a launch, and a program passes the same addresses again and again,
// so a thread remembers those it has confirmed, as fastsnarf.hip does.
bool on_device(int device, const void *p)
{
    static thread_local struct { const void *p; int device; } seen[64];
    const uintptr_t u = reinterpret_cast<uintptr_t>(p);
    const int h = (int)((u >> 9 ^ u >> 15 ^ u >> 21) & 63);
    if (seen[h].p == p && seen[h].device == device) return true;
    hipPointerAttribute_t a;
    if (hipPointerGetAttributes(&a, p) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    if ((a.type != hipMemoryTypeDevice && a.type != hipMemoryTypeManaged) || a.device != device) return false;
    seen[h] = {p, device};
    return true;
}

// An array of a call: `rows` rows of `cols` elements of `size` bytes, `ld` elements apart.
struct Array { const char *name; const void *at; int64_t rows, cols, ld; int size; bool written; };

bool empty(const Array &a) { return a.rows == 0 || a.cols == 0; }
uintptr_t begin_of(const Array &a) { return reinterpret_cast<uintptr_t>(a.at); }
unsigned __int128 extent(const Array &a) { return ((unsigned __int128)(a.rows - 1) * (uint64_t)a.ld + (uint64_t)a.cols) * a.size; }

// `same`: a written array may be that one itself.  Arrays whose address is NULL are left out by the caller where they may be.
fs_status check_arrays(const char *what, int device, const Array *a, int count, int y = -1, int same = -1)
{
    for (int i = 0; i < count; ++i) {
        if (empty(a[i]) || !a[i].at) continue;
        if (a[i].ld < 0 || (a[i].written && a[i].rows > 1 && a[i].ld < a[i].cols)) return fail(FS_E_SHAPE, "%s: rows of %s are %lld elements apart", what, a[i].name, (long long)a[i].ld);
        if (extent(a[i]) >> 56) return fail(FS_E_SHAPE, "%s: %s is too large", what, a[i].name);
        if (begin_of(a[i]) % a[i].size || !on_device(device, a[i].at)) return fail(FS_E_ARG, "%s: %s must be a device pointer aligned to its elements", what, a[i].name);
    }
    for (int i = 0; i < count; ++i) {
        if (!a[i].written || empty(a[i]) || !a[i].at) continue;
        for (int j = 0; j < count; ++j) {
            if (i == j || empty(a[j]) || !a[j].at || (a[j].written && j < i)) continue;
            if (i == y && j == same && a[i].at == a[j].at && (a[i].ld == a[j].ld || a[i].rows == 1)) continue;
            if (begin_of(a[i]) < begin_of(a[j]) + (uint64_t)extent(a[j]) && begin_of(a[j]) < begin_of(a[i]) + (uint64_t)extent(a[i]))
                return fail(FS_E_ARG, "%s: %s overlaps %s", what, a[i].name, a[j].name);
        }
    }
    return FS_OK;
}

fs_status check_drop(const char *what, const fs_drop &d)
{
    if (!(d.p >= 0.0 && d.p <= 1.0)) return fail(FS_E_ARG, "%s: the chance of dropping must be in 0 .. 1", what);
    return FS_OK;
}

// With the device known: where the seed lies.
fs_status check_seed(const char *what, int device, const fs_drop &d)
{
    if (d.p > 0.0 && d.d_seed && (reinterpret_cast<uintptr_t>(d.d_seed) % 8 || !on_device(device, d.d_seed)))
        return fail(FS_E_ARG, "%s: d_seed must be a device pointer aligned to 8 bytes", what);
    return FS_OK;
}

DropD drop_of(const fs_drop &d)
{
    DropD r = {};
    const double least = std::floor(d.p * 4294967296.0 + 0.5);
    r.mode = d.p == 0.0 ? 0 : least >= 4294967296.0 ? 2 : 1;
    if (r.mode != 1) return r;
    r.at = reinterpret_cast<const long long *>(d.d_seed);
    r.seed = d.seed;
    r.offset = d.offset;
    r.least = (unsigned)least;
    r.scale = (float)(1.0 / (1.0 - d.p));
    return r;
}

int act_kind(const fs_linear &l) { return l.act & FS_Z_FULL && l.act > 0 ? l.act - FS_Z_FULL : l.act; }
bool z_full(const fs_linear &l) { return (l.act & FS_Z_FULL) != 0 || l.bias_type == FS_FLOAT_FULL; }

fs_status check_layer(const char *what, const fs_linear *l)
{
    if (!l) return fail(FS_E_ARG, "%s: layer is NULL", what);
    if (l->rows < 0 || l->rows > 500000000ll || l->inputs < 0 || l->inputs > 1 << 24 || l->outputs < 0 || l->outputs > 1 << 24) return fail(FS_E_SHAPE, "%s: sizes out of range", what);
    if (!type_ok(l->type) || (l->bias_type != l->type && l->bias_type != FS_FLOAT_FULL)) return fail(FS_E_ARG, "%s: bad type", what);
    if (act_kind(*l) < FS_ACT_NONE || act_kind(*l) > FS_ACT_SOFTPLUS) return fail(FS_E_ARG, "%s: bad act", what);
    if (act_kind(*l) == FS_ACT_SOFTPLUS && !(l->beta > 0.0f && std::isfinite(l->beta))) return fail(FS_E_ARG, "%s: beta must be positive and finite", what);
    return check_drop(what, l->drop);
}

int cus_of(int device)
{
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess || n < 1) n = 256;
    (void)hipGetLastError();
    return n;
}

// ---------------------------------------------------------------------------------------------------------------- products

// Forward by k_few?  Up to 32 rows, where every wave has a stretch or two (few outputs with many inputs are better off in parts: 12 x 11000 x 300 bf16 takes it 16.2 us,
// the tiles 10.0), and where many weights do not make many blocks read the rows (4096 x 16384, 12 and 32 rows: 30.3 and 36.2 us, tiles 26.7 and 27.6; 8 rows 29; 4096 x 4096, 12
// and 32 rows: 10.4 and 14.3, tiles 13.0 and 13.6; 1024 x 1024: 4.5 and 5.6, tiles 8.0 and 8.3).
constexpr long long FEW_WAVES = 16;
bool is_few(int64_t rows, int64_t outputs, int64_t inputs, int cus)
{
    return rows <= 32 && (outputs >= 16ll * cus || inputs <= 4096) && (rows <= 8 || outputs * inputs <= 1 << 25);
}

// A layer's epilogue behind a range of t that is not longer: smaller blocks, of which some load while others end (524288 x 256 x 256 bf16 with residual and dropout 316 us, with
// the large tile 420; without an epilogue 228 and 169).
constexpr long long SHORT_T = 512;

// How a product is launched: tiles of `tile` squared, `parts` parts of the range of t, each t_part long; twice, if `rests`, with Q and with what its rounding left.
struct Plan {
    int tile, parts;
    bool rests;
    long long t_part, tiles_p, tiles_q, ldp;
    bool in_parts() const { return parts > 1 || rests; }
    int64_t part_bytes() const { return in_parts() ? (int64_t)parts * (rests ? 2 : 1) * part_stride * 4 : 0; }
    long long part_stride;
};

constexpr long long MAX_TILES = (1ll << 23) - 1;        // of 512 threads each at most: a launch has less than 2^32

// 64 squared unless there is a tile of 128 squared for every compute unit (bf16, us, 64 and 128: 2048 x 1024 x 1024 14.9 and 24.7, 4096 x 512 x 4096 49 and 37, 65536 x 128 x 128
// 18.9 and 15.8; fp32: 1024 cubed 25 and 30, 4096 x 1024 x 2048 130 and 103).  Parts, for two blocks a compute unit and none shorter than 256, where there are
// fewer tiles than three for four units (300 x 4096 x 300 bf16 12.7, without parts 22.1; dweight of 65536 x 256 x 256 85 and 372; with 288 tiles of 1536 x 1024 x 768
// fp16 17 in two parts, 12 in one).
Plan plan_product(int type, int64_t np, int64_t nq, int64_t nt, int cus, bool layer = false)
{
    Plan p = {};
    const long long bt = type == FS_FLOAT_FULL ? 32 : 64;
    auto tiles = [&](int64_t n, int b) { return (long long)((n + b - 1) / b); };
    auto area = [&](int b) { return tiles(np, b) * tiles(nq, b) * b * b; };
    p.tile = tiles(np, 128) * tiles(nq, 128) >= cus && np > 64 && nq > 64 ? 128 : 64;
    // a block of the 256 tile has a compute unit for itself: one each, in parts where t is long (dweight of 524288 x 256 x 256 bf16 132 us, with 64 squared 250 to 550;
    // of 8192 x 1024 x 1024 in two parts 110 with dX, with 128 squared 91)
    if (type != FS_FLOAT_FULL && !(layer && nt <= SHORT_T) && tiles(np, 256) * tiles(nq, 256) * std::max<long long>(1, nt / 2048) >= cus && area(256) <= area(128) / 4 * 5) p.tile = 256;
    p.tiles_p = tiles(np, p.tile);
    p.tiles_q = tiles(nq, p.tile);
    const long long all = std::max(1ll, p.tiles_p * p.tiles_q);
    const long long wanted = p.tile == 256 ? std::max(1ll, cus / all) : 4 * all >= 3 * cus ? 1 : std::min((2ll * cus + all - 1) / all, std::max<long long>(1, nt / 256));
    p.t_part = std::max(bt, ((long long)nt + wanted - 1) / wanted);
    p.t_part = (p.t_part + bt - 1) / bt * bt;
    p.parts = (int)std::max<long long>(1, (nt + p.t_part - 1) / p.t_part);
    p.ldp = (np + 3) / 4 * 4;
    p.part_stride = p.ldp * nq;
    return p;
}

Plan plan_forward(const fs_linear &l, int cus)
{
    Plan p = plan_product(l.type, l.outputs, l.rows, l.inputs, cus, true);
    if (is_few(l.rows, l.outputs, l.inputs, cus)) p.parts = 1;
    return p;
}

// May k_product_big read this operand?  Whole chunks of 16 bytes, and offsets in a tile that 32 bits hold.
bool direct_ok(const MatD &M, bool col) { return reinterpret_cast<uintptr_t>(M.at) % 16 == 0 && M.ld % 8 == 0 && M.ld <= 1 << 22 && (!col || M.cols % 8 == 0); }

template <int TYPE, bool PCOL, bool QCOL>
void launch_product(const Plan &p, const MatD &P, const MatD &Q, int64_t np, int64_t nq, int64_t nt, const EpiD &E, hipStream_t stream)
{
    long long tiles_p = p.tiles_p, tiles_q = p.tiles_q;
    if constexpr (TYPE != NET_F32)
        if (p.tile == 256) {
            if (direct_ok(P, PCOL) && direct_ok(Q, QCOL)) {
                const TilesD tiles = {(int)tiles_p, (int)tiles_q};
                k_product_big<TYPE, PCOL, QCOL><<<dim3((unsigned)(tiles_p * tiles_q), (unsigned)p.parts), 512, 0, stream>>>(P, Q, np, nq, nt, p.t_part, tiles, E);
                return;
            }
            tiles_p = (np + 127) / 128;
            tiles_q = (nq + 127) / 128;
        }
    const TilesD tiles = {(int)tiles_p, (int)tiles_q};
    const dim3 grid((unsigned)(tiles_p * tiles_q), (unsigned)p.parts);
    // By 8 waves (bf16 8192 x 1024 x 1024 forward 26 us, by 4 waves 30; backward 8192 x 4095 x 4095 1117 us, by 4 1232), fp32 backward by 4 (200003 x 256 x 256 474 us, by 8 503).
    // 16 bits have two buffers (524288 x 256 x 256 bf16 with residual and dropout 316 us, with one 337), fp32 one (200003 x 256 x 256 with residual and Z 254 us, with two 294).
    constexpr bool F32 = TYPE == NET_F32;
    if (p.tile < 128) k_product<TYPE, PCOL, QCOL, 64, 64, 2, 2, 2, 2><<<grid, 256, 0, stream>>>(P, Q, np, nq, nt, p.t_part, tiles, E);
    else if constexpr (F32 && PCOL) k_product<TYPE, PCOL, QCOL, 128, 128, 2, 2, 1, 1><<<grid, 256, 0, stream>>>(P, Q, np, nq, nt, p.t_part, tiles, E);
    else k_product<TYPE, PCOL, QCOL, 128, 128, 2, 4, F32 ? 1 : 2, 1><<<grid, 512, 0, stream>>>(P, Q, np, nq, nt, p.t_part, tiles, E);
}

template <int TYPE, bool RESTS>
void launch_parts(const Plan &p, const float *part, int64_t np, int64_t nq, const EpiD &E, hipStream_t stream)
{
    const long long all = (np + 255) / 256 * nq, blocks = p.parts >= 8 ? all : (all + 3) / 4;
    if (p.parts >= 8) k_parts<TYPE, true, RESTS><<<(unsigned)std::min<long long>(blocks, 1 << 16), 256, 0, stream>>>(part, p.part_stride, p.ldp, p.parts, np, nq, E);
    else k_parts<TYPE, false, RESTS><<<(unsigned)std::min<long long>(blocks, 1 << 16), 256, 0, stream>>>(part, p.part_stride, p.ldp, p.parts, np, nq, E);
}

// Waves a block: enough that every compute unit has some 16, and each a group of steps or more.
template <int TYPE> void launch_few(const MatD &W, const MatD &X, int64_t np, int64_t nq, int64_t nt, const EpiD &E, int cus, hipStream_t stream)
{
    // two times 16 outputs a block where that leaves a block for every unit: the rows are read half as often
    const int mp = nq > 4 && np > 16ll * cus ? 2 : 1, many = nq > 16 ? 2 : 1;
    const long long blocks = (np + 16 * mp - 1) / (16 * mp), groups = std::max<long long>(1, nt / 32 / few_ahead(TYPE == NET_F32, mp, many));
    const int waves = (int)std::max<long long>(mp * many, std::min(std::min(16ll, groups), std::max(4ll, FEW_WAVES * cus / blocks)));
    const dim3 grid((unsigned)blocks), block(64 * waves);
    if (mp == 1 && many == 1) k_few<TYPE, 1, 1><<<grid, block, 0, stream>>>(W, X, np, nq, nt, E);
    else if (mp == 1) k_few<TYPE, 1, 2><<<grid, block, 0, stream>>>(W, X, np, nq, nt, E);
    else if (many == 1) k_few<TYPE, 2, 1><<<grid, block, 0, stream>>>(W, X, np, nq, nt, E);
    else k_few<TYPE, 2, 2><<<grid, block, 0, stream>>>(W, X, np, nq, nt, E);
}

enum { NT, NN, TN };                   // forward, dX, dweight

// One product with its epilogue; `work`: part_bytes() of the plan; rest: of Q, where the plan has rests.
void product(int type, int kind, const Plan &p, const MatD &P, const MatD &Q, const MatD &rest, int64_t np, int64_t nq, int64_t nt, const EpiD &E, void *work, hipStream_t stream)
{
    if (np == 0 || nq == 0) return;
    EpiD part = E;
    if (p.in_parts()) {
        part = {};
        part.mode = EPI_PART;
        part.out = work;
        part.ldo = p.ldp;
        part.part_stride = p.part_stride;
    }
#define FS_NET_PRODUCT(TYPE, Q)                                                                        \
    do {                                                                                               \
        if (kind == NT) launch_product<TYPE, false, false>(p, P, Q, np, nq, nt, part, stream);         \
        else if (kind == NN) launch_product<TYPE, true, false>(p, P, Q, np, nq, nt, part, stream);     \
        else launch_product<TYPE, true, true>(p, P, Q, np, nq, nt, part, stream);                      \
    } while (0)
#define FS_NET_KIND(TYPE)                                                                              \
    do {                                                                                               \
        FS_NET_PRODUCT(TYPE, Q);                                                                       \
        if (p.rests) {                                                                                 \
            part.out = static_cast<float *>(work) + p.parts * p.part_stride;                           \
            FS_NET_PRODUCT(TYPE, rest);                                                                \
            launch_parts<TYPE, TYPE != NET_F32>(p, static_cast<const float *>(work), np, nq, E, stream); \
        } else if (p.parts > 1) {                                                                      \
            launch_parts<TYPE, false>(p, static_cast<const float *>(work), np, nq, E, stream);         \
        }                                                                                              \
    } while (0)
    if (type == FS_FLOAT_FULL) FS_NET_KIND(NET_F32);
    else if (type == FS_FLOAT_BRAIN) FS_NET_KIND(NET_BF16);
    else FS_NET_KIND(NET_F16);
#undef FS_NET_KIND
#undef FS_NET_PRODUCT
}

// ---------------------------------------------------------------------------------------------------------------- elementwise

struct RowsPlan { RowsD n; unsigned gx, gy; };

// last: elements of the last row
RowsPlan plan_rows(int type, int64_t rows, int64_t cols, int64_t last, long long blocks)
{
    RowsPlan p;
    const int v = type == FS_FLOAT_FULL ? 4 : 8;
    const long long units = (cols + v - 1) / v;
    p.n = {rows, cols, last, 0};
    while (p.n.tx_bits < 8 && 1ll << p.n.tx_bits < units) ++p.n.tx_bits;
    p.gx = (unsigned)std::min<long long>(1 << 16, std::max<long long>(1, (units + (1 << p.n.tx_bits) - 1) >> p.n.tx_bits));
    const long long at_once = 256 >> p.n.tx_bits, passes = std::max<long long>(1, (rows + at_once - 1) / at_once);
    p.gy = (unsigned)std::max(1ll, std::min(passes, blocks / p.gx));
    return p;
}

constexpr long long ROW_BLOCKS = 2048, DZ_BLOCKS = 1024;

// most, factor: of fp16, where dz is wanted; rest: where dz is and a product takes it (see k_dz)
template <int TYPE> void launch_dz(const RowsPlan &p, const MatD &G, const MatD &Z, const fs_linear &l, void *dz, void *rest, double *sums, unsigned *most, float *factor, hipStream_t stream)
{
    if (most) k_largest<<<LARGEST_BLOCKS, 256, 0, stream>>>(p.n, G, most);
    k_dz<TYPE, TYPE == NET_F32 ? 4 : 8><<<dim3(p.gx, p.gy), 256, 0, stream>>>(p.n, G, Z, z_full(l), act_kind(l), l.beta, drop_of(l.drop), dz, l.outputs, sums, most, factor, rest);
}

int64_t up(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// The backward pass's workspace: dZ (where it is not G itself), the sums of its columns, parts of either product, and of fp16 the factor and its numbers.
// narrow: k_narrow's, parts of dweight and of dbias by `blocks` blocks, and nothing else.
// Inputs and outputs of a layer whose backward pass is k_narrow's: two launches instead of five or six, 7 us each on the thread that runs backward passes, and no dZ in memory.
// Kernels, us, this and the others: fp32 1024 x 64 x 64 12.1 and 20.7, 65536 x 128 x 128 48 and 73, 524288 x 32 x 128 260 and 390; bf16 14.7 and 16.7, 40 and 47, 185 and 201,
// 262144 x 128 x 128 106 and 123.
constexpr int NARROW = 128;
// Products of 16 bits that take dZ in two parts, rounded and what that leaves.  The results' own rounding and dZ's make 1.41 times the error of the first alone, on average: of up
// to FEW results, or from up to FEW values of dZ, by chance more (64 results, dweight of 380289 x 8 x 8 bf16: 1.6 times; 2 x 27 x 2 fp16, silu: 3.2; 4 results of 3655
// values each, some of which cancel: 4.2).  With 4096 the squares' sums of normal results scatter by 2 %: 1.5 times is some six deviations off.
// Narrow layers take the parts up to NARROW_RESTS values of dZ, where that takes 4 us of 21 (1024 x 64 x 64 bf16).
// Others launch a product twice: backward of 5000 x 10 x 200 bf16 44 us, once 31, of 200000 x 300 x 8 185, once 123.
constexpr int64_t FEW = 4096, NARROW_RESTS = 1 << 17;
bool few_products(int64_t values, int64_t results) { return std::min(values, results) <= FEW; }
bool narrow_rests(const fs_linear &l)
{
    const int64_t values = l.rows * l.outputs;
    return l.type != FS_FLOAT_FULL && (values <= NARROW_RESTS || few_products(values, l.rows * l.inputs) || few_products(values, l.outputs * l.inputs));
}

struct Backward {
    Plan dx, dw;
    RowsPlan dz;
    bool has_dz;
    bool narrow;
    int blocks;
    int64_t rest, sums, part, factor, most, end;
};

int64_t narrow_ld(const fs_linear &l) { return (l.inputs + 3) / 4 * 4; }
int64_t narrow_sums(const fs_linear &l, const Backward &b) { return up((int64_t)b.blocks * l.outputs * narrow_ld(l) * 4); }

template <int TYPE>
void launch_narrow(const fs_linear &l, const Backward &b, const DzD &D, const MatD &X, const MatD &W, void *dx, int64_t lddx, void *dw, int64_t lddw, void *dbias, char *work, hipStream_t stream)
{
    float *part = dw ? reinterpret_cast<float *>(work) : nullptr;
    double *sums = dbias ? reinterpret_cast<double *>(work + narrow_sums(l, b)) : nullptr;
    const int64_t ld = narrow_ld(l);
    constexpr int WAVES = TYPE == NET_F32 ? 8 : 4;
    if (!narrow_rests(l)) k_narrow<TYPE, NARROW, WAVES, false><<<b.blocks, 64 * WAVES, 0, stream>>>(D, X, W, dx, lddx, part, ld, sums);
    else k_narrow<TYPE, NARROW, WAVES, TYPE != NET_F32><<<b.blocks, 64 * WAVES, 0, stream>>>(D, X, W, dx, lddx, part, ld, sums);
    const int blocks_dw = dw ? (int)((l.outputs * ld + 255) / 256) : 0, blocks_db = dbias ? (int)((l.outputs + 63) / 64) : 0;
    if (blocks_dw + blocks_db > 0) k_narrow_end<TYPE><<<blocks_dw + blocks_db, 1024, 0, stream>>>(part, ld, b.blocks, l.inputs, l.outputs, dw, lddw, sums, dbias, l.bias_type == FS_FLOAT_FULL, blocks_dw);
}

Backward plan_backward(const fs_linear &l, int cus)
{
    Backward b = {};
    b.dx = plan_product(l.type, l.inputs, l.rows, l.outputs, cus);
    b.dw = plan_product(l.type, l.inputs, l.outputs, l.rows, cus);
    b.dz = plan_rows(l.type, l.rows, l.outputs, l.outputs, DZ_BLOCKS);
    b.has_dz = act_kind(l) != FS_ACT_NONE || l.drop.p > 0.0;
    b.narrow = std::min({l.rows, l.inputs, l.outputs}) > 0 && std::max(l.inputs, l.outputs) <= NARROW;
    // as many as a compute unit holds: registers and LDS leave room for two blocks of 16 bits and one of fp32.  Forward and backward, us, of bf16 with two, three and four blocks:
    // 65536 x 128 x 128 57, 65 and 70, 131072 x 10 x 9 64, 77 and 70, 30000 x 128 x 128 38, 48 and 52.
    const long long per_cu = l.type != FS_FLOAT_FULL ? 2 : 1;
    b.blocks = (int)std::max<long long>(1, std::min<long long>(per_cu * cus, (l.rows + 31) / 32));
    if (b.narrow) {                    // no dZ, and no products' parts
        b.end = narrow_sums(l, b) + up((int64_t)b.blocks * l.outputs * 8);
        return b;
    }
    if (b.has_dz && l.type != FS_FLOAT_FULL) {
        b.dx.rests = few_products(l.rows * l.outputs, l.rows * l.inputs);
        b.dw.rests = few_products(l.rows * l.outputs, l.outputs * l.inputs);
    }
    b.rest = b.has_dz ? up(l.rows * l.outputs * size_of(l.type)) : 0;
    b.sums = b.dx.rests || b.dw.rests ? 2 * b.rest : b.rest;
    b.part = b.sums + up((int64_t)b.dz.gy * l.outputs * 8);
    b.factor = b.part + up(std::max(b.dx.part_bytes(), b.dw.part_bytes()));
    const bool scaled = b.has_dz && l.type == FS_FLOAT_HALF;
    b.most = b.factor + (scaled ? 256 : 0);
    b.end = b.most + (scaled ? up(LARGEST_BLOCKS * sizeof(unsigned)) : 0);
    return b;
}

bool too_many(const Plan &p) { return (unsigned __int128)p.tiles_p * p.tiles_q * (p.tile == 256 ? 4 : 1) > MAX_TILES; }

fs_status current_device(const char *what, int *device)
{
    if (hipGetDevice(device) == hipSuccess) return FS_OK;
    (void)hipGetLastError();
    return fail(FS_E_DEVICE, "%s: no device", what);
}

fs_status check_work(const char *what, int device, const void *work, int64_t bytes, int64_t needed)
{
    if (needed == 0) return FS_OK;
    if (!work || bytes < needed) return fail(FS_E_ARG, "%s: needs %lld bytes of workspace", what, (long long)needed);
    if (reinterpret_cast<uintptr_t>(work) % 256 || !on_device(device, work)) return fail(FS_E_ARG, "%s: the workspace must be a device pointer aligned to 256 bytes", what);
    return FS_OK;
}

#define FS_NET_TRY(x)                           \
    do {                                        \
        const fs_status try_status = (x);       \
        if (try_status != FS_OK) return try_status; \
    } while (0)

}  // namespace

extern "C" {

const char *fs_net_error(void) { return net_err; }

int64_t fs_linear_bytes(const fs_linear *layer, int32_t backward)
{
    if (check_layer("fs_linear_bytes", layer) != FS_OK) return -1;
    int device = 0;
    if (current_device("fs_linear_bytes", &device) != FS_OK) return -1;
    const int cus = cus_of(device);
    if (!backward) return up(plan_forward(*layer, cus).part_bytes());
    return plan_backward(*layer, cus).end;
}

fs_status fs_linear_forward(const fs_linear *layer, const void *d_x, int64_t ldx, const void *d_w, int64_t ldw, const void *d_bias, const void *d_r, int64_t ldr,
                            void *d_y, int64_t ldy, void *d_z, int64_t ldz, void *d_work, int64_t work_bytes, void *hip_stream)
{
    const char *what = "fs_linear_forward";
    FS_NET_TRY(check_layer(what, layer));
    const fs_linear &l = *layer;
    int device = 0;
    FS_NET_TRY(current_device(what, &device));
    const int64_t m = l.rows, n = l.outputs, k = l.inputs;
    const int cus = cus_of(device);
    const Plan p = plan_forward(l, cus);
    if (too_many(p)) return fail(FS_E_SHAPE, "%s: too many results", what);
    if (m > 0 && n > 0) {
        const int s = size_of(l.type);
        if (!d_y || (k > 0 && (!d_x || !d_w))) return fail(FS_E_ARG, "%s: d_x, d_w and d_y must not be NULL", what);
        const Array a[] = {{"d_x", d_x, m, k, ldx, s, false}, {"d_w", d_w, n, k, ldw, s, false}, {"d_bias", d_bias, 1, n, 0, size_of(l.bias_type), false},
                           {"d_r", d_r, m, n, ldr, s, false}, {"d_y", d_y, m, n, ldy, s, true}, {"d_z", d_z, m, n, ldz, z_full(l) ? 4 : s, true},
                           {"d_work", d_work, 1, p.part_bytes(), 0, 1, true}};
        FS_NET_TRY(check_arrays(what, device, a, 7, 4, 3));
        FS_NET_TRY(check_seed(what, device, l.drop));
        FS_NET_TRY(check_work(what, device, d_work, work_bytes, p.part_bytes()));
    }
    EpiD E = {};
    E.mode = EPI_LAYER;
    E.act = act_kind(l);
    E.beta = l.beta;
    E.over_beta = 1.0f / l.beta;
    E.bias = d_bias;
    E.bias_f32 = l.bias_type == FS_FLOAT_FULL;
    E.z_f32 = z_full(l);
    E.r = d_r;
    E.ldr = ldr;
    E.out = d_y;
    E.ldo = ldy;
    E.z = d_z;
    E.ldz = ldz;
    E.drop = drop_of(l.drop);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const MatD W = {d_w, ldw, n, k}, X = {d_x, ldx, m, k};
    if (m == 0 || n == 0) return FS_OK;
    if (!is_few(m, n, k, cus)) product(l.type, NT, p, W, X, {}, n, m, k, E, d_work, stream);
    else if (l.type == FS_FLOAT_FULL) launch_few<NET_F32>(W, X, n, m, k, E, cus, stream);
    else if (l.type == FS_FLOAT_BRAIN) launch_few<NET_BF16>(W, X, n, m, k, E, cus, stream);
    else launch_few<NET_F16>(W, X, n, m, k, E, cus, stream);
    return launch_status(what);
}

fs_status fs_linear_backward(const fs_linear *layer, const void *d_g, int64_t ldg, const void *d_x, int64_t ldx, const void *d_w, int64_t ldw, const void *d_z, int64_t ldz,
                             void *d_dx, int64_t lddx, void *d_dw, int64_t lddw, void *d_dbias, void *d_work, int64_t work_bytes, void *hip_stream)
{
    const char *what = "fs_linear_backward";
    FS_NET_TRY(check_layer(what, layer));
    const fs_linear &l = *layer;
    int device = 0;
    FS_NET_TRY(current_device(what, &device));
    const int64_t m = l.rows, n = l.outputs, k = l.inputs;
    const Backward b = plan_backward(l, cus_of(device));
    if (too_many(b.dx) || too_many(b.dw)) return fail(FS_E_SHAPE, "%s: too many results", what);
    const int s = size_of(l.type);
    const bool act = act_kind(l) != FS_ACT_NONE;
    if (m > 0 && n > 0 && (d_dbias || (k > 0 && (d_dx || d_dw)))) {
        if (!d_g || (act && !d_z) || (k > 0 && ((d_dx && !d_w) || (d_dw && !d_x)))) return fail(FS_E_ARG, "%s: an array that is needed is NULL", what);
    }
    const Array a[] = {{"d_g", d_g, m, n, ldg, s, false}, {"d_x", d_dw ? d_x : nullptr, m, k, ldx, s, false}, {"d_w", d_dx ? d_w : nullptr, n, k, ldw, s, false},
                       {"d_z", act ? d_z : nullptr, m, n, ldz, z_full(l) ? 4 : s, false}, {"d_dx", d_dx, m, k, lddx, s, true}, {"d_dw", d_dw, n, k, lddw, s, true},
                       {"d_dbias", d_dbias, 1, n, 0, size_of(l.bias_type), true}, {"d_work", d_work, 1, b.end, 0, 1, true}};
    FS_NET_TRY(check_arrays(what, device, a, 8));
    FS_NET_TRY(check_seed(what, device, l.drop));
    FS_NET_TRY(check_work(what, device, d_work, work_bytes, b.end));

    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    char *work = static_cast<char *>(d_work);
    double *sums = d_dbias ? reinterpret_cast<double *>(work + b.sums) : nullptr;
    const MatD G = {d_g, ldg, m, n}, Z = {d_z, ldz, m, n};
    if (b.narrow && (d_dx || d_dw || d_dbias)) {
        const DzD D = {G, Z, z_full(l), act_kind(l), l.beta, drop_of(l.drop)};
        const MatD X = {d_x, ldx, m, k}, W = {d_w, ldw, n, k};
        if (l.type == FS_FLOAT_FULL) launch_narrow<NET_F32>(l, b, D, X, W, d_dx, lddx, d_dw, lddw, d_dbias, work, stream);
        else if (l.type == FS_FLOAT_BRAIN) launch_narrow<NET_BF16>(l, b, D, X, W, d_dx, lddx, d_dw, lddw, d_dbias, work, stream);
        else launch_narrow<NET_F16>(l, b, D, X, W, d_dx, lddx, d_dw, lddw, d_dbias, work, stream);
        return launch_status(what);
    }
    const MatD dZ = b.has_dz ? MatD{work, n, m, n} : G;
    void *dz = b.has_dz && (d_dx || d_dw) ? work : nullptr;
    void *rest = dz && ((d_dx && b.dx.rests) || (d_dw && b.dw.rests)) ? work + b.rest : nullptr;
    float *factor = dz && n > 0 && l.type == FS_FLOAT_HALF ? reinterpret_cast<float *>(work + b.factor) : nullptr;
    if ((dz || sums) && n > 0) {
        if (l.type == FS_FLOAT_FULL) launch_dz<NET_F32>(b.dz, G, Z, l, dz, nullptr, sums, nullptr, nullptr, stream);
        else if (l.type == FS_FLOAT_BRAIN) launch_dz<NET_BF16>(b.dz, G, Z, l, dz, rest, sums, nullptr, nullptr, stream);
        else launch_dz<NET_F16>(b.dz, G, Z, l, dz, rest, sums, factor ? reinterpret_cast<unsigned *>(work + b.most) : nullptr, factor, stream);
        if (sums) {
            const unsigned blocks = (unsigned)((n + 63) / 64);
            if (l.bias_type == FS_FLOAT_FULL) k_dbias<NET_F32><<<blocks, 1024, 0, stream>>>(sums, (int)b.dz.gy, n, d_dbias);
            else if (l.bias_type == FS_FLOAT_BRAIN) k_dbias<NET_BF16><<<blocks, 1024, 0, stream>>>(sums, (int)b.dz.gy, n, d_dbias);
            else k_dbias<NET_F16><<<blocks, 1024, 0, stream>>>(sums, (int)b.dz.gy, n, d_dbias);
        }
    }
    EpiD E = {};
    E.mode = EPI_STORE;
    E.factor = factor;
    if (d_dx) {
        E.out = d_dx;
        E.ldo = lddx;
        product(l.type, NN, b.dx, {d_w, ldw, n, k}, dZ, {rest, n, m, n}, k, m, n, E, work + b.part, stream);
    }
    if (d_dw) {
        E.out = d_dw;
        E.ldo = lddw;
        product(l.type, TN, b.dw, {d_x, ldx, m, k}, dZ, {rest, n, m, n}, k, n, m, E, work + b.part, stream);
    }
    return launch_status(what);
}

fs_status fs_dropout(int32_t type, int64_t rows, int64_t columns, const fs_drop *drop, const void *d_x, int64_t ldx, const void *d_r, int64_t ldr, void *d_y, int64_t ldy,
                     void *hip_stream)
{
    const char *what = "fs_dropout";
    if (!drop) return fail(FS_E_ARG, "%s: drop is NULL", what);
    if (!type_ok(type)) return fail(FS_E_ARG, "%s: bad type", what);
    if (rows < 0 || columns < 0 || rows > 1ll << 36 || columns > 1ll << 36 || (unsigned __int128)rows * columns > (1ull << 40)) return fail(FS_E_SHAPE, "%s: sizes out of range", what);
    FS_NET_TRY(check_drop(what, *drop));
    if (rows == 0 || columns == 0) return FS_OK;
    int device = 0;
    FS_NET_TRY(current_device(what, &device));
    const int s = size_of(type);
    if (!d_x || !d_y) return fail(FS_E_ARG, "%s: d_x and d_y must not be NULL", what);
    const Array a[] = {{"d_x", d_x, rows, columns, ldx, s, false}, {"d_r", d_r, rows, columns, ldr, s, false}, {"d_y", d_y, rows, columns, ldy, s, true}};
    // Y may be either of what it is made from, element by element
    const Array xy[] = {a[0], a[2]}, ry[] = {a[1], a[2]};
    FS_NET_TRY(check_arrays(what, device, xy, 2, 1, 0));
    FS_NET_TRY(check_arrays(what, device, ry, 2, 1, 0));
    FS_NET_TRY(check_seed(what, device, *drop));
    // memory without gaps: rows of a block's width, whatever they were
    int64_t last = columns;
    if (ldx == columns && ldy == columns && (!d_r || ldr == columns)) {
        const int64_t all = rows * columns, width = type == FS_FLOAT_FULL ? 1024 : 2048;
        columns = std::min(all, width);
        rows = (all + columns - 1) / columns;
        last = all - (rows - 1) * columns;
        ldx = ldy = ldr = columns;
    }
    const RowsPlan p = plan_rows(type, rows, columns, last, ROW_BLOCKS);
    const MatD X = {d_x, ldx, rows, columns}, R = {d_r, ldr, rows, columns};
    const dim3 grid(p.gx, p.gy);
    const DropD D = drop_of(*drop);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (type == FS_FLOAT_FULL) k_dropout<NET_F32, 4><<<grid, 256, 0, stream>>>(p.n, X, R, d_y, ldy, D);
    else if (type == FS_FLOAT_BRAIN) k_dropout<NET_BF16, 8><<<grid, 256, 0, stream>>>(p.n, X, R, d_y, ldy, D);
    else k_dropout<NET_F16, 8><<<grid, 256, 0, stream>>>(p.n, X, R, d_y, ldy, D);
    return launch_status(what);
}

}  // extern "C"
