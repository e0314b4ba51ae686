// C ABI of the calls on a list of tensors (see include/fastsnarf_train.h): argument checks, the list's copy on the device,
// launches.  gfx950 only.
#include "../../include/fastsnarf_train.h"
#include "fs_train_kernels.hpp"

#include <hip/hip_runtime.h>
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <limits>
#include <new>

using namespace fs;

// The capture that a stream records for; `active` false: it records none.
struct Capture { bool active; unsigned long long id; };

struct fs_tensors {
    hipStream_t stream;
    int device, n_cus;
    int32_t asked;            // tensors as given
    fs_tensor *given;         // [asked] of the last create or update
    TensorD *host;            // [asked] those with elements, as they are on the device
    // what the tensors as a whole have
    bool params, moments, apart, in_place;      // in_place, apart: every `out` is, or none is, its gradient
    double grad_bytes, adam_bytes, param_bytes;
    ListD L;
    char *mem;                // device, see Places
    bool owned;               // `mem` was allocated here
    double *partial;
    unsigned *tickets;
    bool put;                 // the device's copy is that of `host`, for calls in the capture `put_in`; elsewhere too if that is none
    Capture put_in;
    const void *seen[8];      // words (d_norm, d_step, d_lr) that are known to be memory of the device, by address
    char err[256];
};

namespace {

fs_status fail(fs_tensors *t, fs_status s, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(t->err, sizeof t->err, fmt, ap);
    va_end(ap);
    return s;
}

fs_status launch_status(fs_tensors *t, const char *what)
{
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FS_OK : fail(t, FS_E_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

Capture capture_of(hipStream_t stream)
{
    Capture c = {false, 0};
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    if (!stream) return c;                                  // the default stream cannot be captured
    if (hipStreamGetCaptureInfo(stream, &status, &c.id) != hipSuccess) (void)hipGetLastError();
    else c.active = status == hipStreamCaptureStatusActive;
    return c;
}

// Is the device's list that of `host` where the next call on the list's stream runs?  A graph's update runs when the graph does, so until then, and
// for all that is no part of the graph, the device has another list.
bool there(const fs_tensors *t)
{
    if (!t->put || !t->put_in.active) return t->put;
    const Capture now = capture_of(t->stream);
    return now.active && now.id == t->put_in.id;
}

bool on_device(const fs_tensors *t, const void *p)
{
    hipPointerAttribute_t a;
    if (hipPointerGetAttributes(&a, p) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    return (a.type == hipMemoryTypeDevice || a.type == hipMemoryTypeManaged) && a.device == t->device;
}

// Null (where that is allowed) or aligned to an element of `size` bytes, and memory of the list's device: asked only where the
// pointer is not the one of the same place in the list before (`before`), which has been confirmed.
bool array_ok(const fs_tensors *t, const void *p, const void *before, bool nullable, int size)
{
    if (!p) return nullable;
    if (reinterpret_cast<uintptr_t>(p) % size) return false;
    return p == before || on_device(t, p);
}

// A word that a call reads or writes.  The lookup in the runtime takes as long as a launch, and a program passes the same words again and
// again, so those it has confirmed are remembered, as fastsnarf.hip does for its arrays.
bool word_ok(fs_tensors *t, const void *p, int size)
{
    const uintptr_t u = reinterpret_cast<uintptr_t>(p);
    if (!p || u % size) return false;
    const int h = (int)((u >> 3 ^ u >> 9) & 7);
    if (t->seen[h] == p) return true;
    if (!on_device(t, p)) return false;
    t->seen[h] = p;
    return true;
}

bool apart(const void *a, const void *b, size_t bytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x + bytes <= y || y + bytes <= x;
}

bool type_ok(int32_t type) { return type == FS_FLOAT_FULL || type == FS_FLOAT_BRAIN || type == FS_FLOAT_HALF; }
int size_of(int32_t type) { return type == FS_FLOAT_FULL ? 4 : 2; }
static_assert(int(FS_FLOAT_FULL) == TYPE_F32 && int(FS_FLOAT_BRAIN) == TYPE_BF16 && int(FS_FLOAT_HALF) == TYPE_F16, "types");
static_assert(int(FS_NORM_TWO) == KIND_TWO && int(FS_NORM_MAX) == KIND_MAX, "kinds");
constexpr int MAX_LEAD = 64;
static_assert(sizeof(PutD) + 64 <= 4096, "kernel arguments");

// Checks a list.  `before`: the list whose pointers are known to be memory of the device, or NULL.
fs_status check_list(fs_tensors *t, const char *what, const fs_tensor *list, int32_t count, const fs_tensor *before)
{
    long long units = 0;
    for (int32_t i = 0; i < count; ++i) {
        const fs_tensor &x = list[i];
        if (x.n < 0 || x.n > 1ll << 40) return fail(t, FS_E_SHAPE, "%s: tensor %d: n out of range", what, i);
        if (x.n == 0) continue;
        units += (x.n + MAX_LEAD + UNIT - 1) / UNIT;
        if (units >= 1ll << 31) return fail(t, FS_E_SHAPE, "%s: tensor %d: too many elements in all", what, i);
        if (!type_ok(x.grad_type) || (x.param && !type_ok(x.param_type))) return fail(t, FS_E_ARG, "%s: tensor %d: bad type", what, i);
        if (!std::isfinite(x.lr_scale) || !std::isfinite(x.decay_scale)) return fail(t, FS_E_ARG, "%s: tensor %d: lr_scale and decay_scale must be finite", what, i);
        fs_tensor old = {};
        if (before && before[i].n) old = before[i];
        const int gs = size_of(x.grad_type), ps = size_of(x.param_type);
        if (!array_ok(t, x.grad, old.grad, false, gs) || !array_ok(t, x.out, old.out, true, gs) || !array_ok(t, x.param, old.param, true, ps) ||
            !array_ok(t, x.master, old.master, true, 4) || !array_ok(t, x.exp_avg, old.exp_avg, true, 4) || !array_ok(t, x.exp_avg_sq, old.exp_avg_sq, true, 4))
            return fail(t, FS_E_ARG, "%s: tensor %d: arrays must be device pointers aligned to their elements (grad not NULL)", what, i);
        if (x.out && x.out != x.grad && !apart(x.out, x.grad, (size_t)x.n * gs))
            return fail(t, FS_E_ARG, "%s: tensor %d: out overlaps grad", what, i);
    }
    return FS_OK;
}

// Elements by which a tensor's first unit begins before it, so that units begin at 256 bytes of the moments (of the gradients, where there are none; 16-bit
// arrays then begin at 128).  Tensors packed without gaps lie anywhere: an AdamW step of 250 M elements in 16 bits took 1700 us with units that began with the
// tensors, 1450 with tensors at multiples of 64 elements.
int lead_of(const fs_tensor &x)
{
    const uintptr_t at = x.exp_avg ? reinterpret_cast<uintptr_t>(x.exp_avg) / 4 : reinterpret_cast<uintptr_t>(x.grad) / size_of(x.grad_type);
    return (int)(at % MAX_LEAD);
}

// Takes a checked list over: the host's copies, and the device's in the stream's order, with counters that are cleared (NULL: they are).
fs_status put_list(fs_tensors *t, const char *what, const fs_tensor *list, unsigned *tickets)
{
    t->put = false;
    int count = 0, units = 0;
    t->params = t->moments = t->apart = t->in_place = true;
    t->grad_bytes = t->adam_bytes = t->param_bytes = 0.0;
    for (int32_t i = 0; i < t->asked; ++i) {
        const fs_tensor &x = t->given[i] = list[i];
        if (x.n == 0) continue;
        TensorD &d = t->host[count++];
        d.grad = x.grad;
        d.out = x.out ? x.out : x.grad;
        d.param = x.param;
        d.master = x.master;
        d.m = x.exp_avg;
        d.v = x.exp_avg_sq;
        d.n = x.n;
        d.first = units;
        d.lead = lead_of(x);
        units += (int)((x.n + d.lead + UNIT - 1) / UNIT);
        d.next = units;
        d.types = x.grad_type | x.param_type << 8;
        d.lr_scale = x.lr_scale;
        d.decay_scale = x.decay_scale;
        t->params = t->params && x.param;
        t->moments = t->moments && x.exp_avg && x.exp_avg_sq;
        t->apart = t->apart && d.out != d.grad;
        t->in_place = t->in_place && d.out == d.grad;
        t->grad_bytes += (double)x.n * size_of(x.grad_type);
        if (x.param) t->param_bytes += (double)x.n * size_of(x.param_type);
        if (x.param) t->adam_bytes += (double)x.n * (size_of(x.grad_type) + 16 + (x.master ? 8 : size_of(x.param_type)) + size_of(x.param_type));
    }
    t->L.count = count;
    t->L.units = units;
    for (int at = 0; at < count || tickets; at += PUT, tickets = nullptr) {
        PutD p;
        const int n = std::min(PUT, count - at);
        std::memcpy(p.t, t->host + at, n * sizeof(TensorD));
        k_list_put<<<1, 64, 0, t->stream>>>(p, at, n, const_cast<TensorD *>(t->L.tensors), const_cast<int *>(t->L.first), tickets);
    }
    const fs_status s = launch_status(t, what);
    t->put = s == FS_OK;
    t->put_in = capture_of(t->stream);
    return s;
}

fs_status on_current_device(fs_tensors *t, const char *what)
{
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != t->device) {
        (void)hipGetLastError();
        return fail(t, FS_E_DEVICE, "%s: the list's device must be the current one", what);
    }
    return FS_OK;
}

#define FS_TRAIN_BEGIN(t, needs_list)                                                                                     \
    do {                                                                                                                  \
        if (!(t)) return FS_E_ARG;                                                                                        \
        const fs_status begin_status = on_current_device((t), __func__);                                                  \
        if (begin_status != FS_OK) return begin_status;                                                                   \
        if ((needs_list) && !there(t))                                                                                    \
            return fail((t), FS_E_STATE, "%s: the list has not reached the device%s", __func__,                           \
                        (t)->put ? ": its last update is part of a graph" : "");                                          \
    } while (0)

// Blocks of a kernel per compute unit, and how many units each takes at a time at most.  Few blocks with their chunks side by side keep the arrays' pages
// and channels evenly in use.  Measured for 2 / 4 / 8 blocks per unit, us: norm of 400 M fp32 226 / 234 / 241 and of 45 M bf16 in 300 tensors 23.5 / 20.9 /
// 21.2 (where a block's start is not hidden by what it has to do); clipping 20 M mixed 37 / 35 / 35; AdamW of 12.6 M fp32 70.6 / 73.3 / 73.1, of 250 M mixed
// 1365 / 1414 / 1415.  Chunks of 3 / 6 / 8 units in AdamW: 1351 / 1372 / 1384; of 1 unit 1600 (a block has too little on its way); of 6 / 8 / 32 in the norm of 45 M
// bf16 22.2 / 20.6 / 20.2, of 180 M 62.3 / 62.3 / 59.6.  Where that leaves less than `least` units a block, blocks are fewer, down to one a compute unit: a
// norm has fewer of them to wait for at its end, 2 M fp32 5.7 / 6.5, 4 M bf16 6.1 / 7.7, 16 M 11.2 / 11.1.
struct Shape { int per_cu, most, least; };
constexpr Shape NORM = {4, 32, 8}, NORM_LONG = {2, 8, 1}, CLIP = {4, 4, 1}, ADAMW = {2, 3, 1};

// Long lists mostly in fp32, where two blocks a unit read what they can: norm of 450 M fp32 254 us, with four 262; 900 M bf16, twice the arithmetic a byte, 296 and 263.
bool norm_is_long(const fs_tensors *t) { return t->L.units >= 1 << 16 && t->grad_bytes >= 3.0 * UNIT * t->L.units; }

struct Grid { int blocks; ListD L; };
Grid grid_for(const fs_tensors *t, const Shape &shape)
{
    const int wanted = std::max(t->n_cus, std::min(t->L.units / shape.least, shape.per_cu * t->n_cus));
    Grid g = {std::max(1, std::min(t->L.units, wanted)), t->L};
    const long long most = (long long)shape.most * g.blocks, rounds = std::max(1ll, (t->L.units + most - 1) / most);
    if (rounds > 16) {       // what the last round leaves undone is little, and chunks that are all alike are 2 % faster
        g.L.chunks = (int)(((long long)t->L.units + shape.most - 1) / shape.most);
        g.L.step = (long long)shape.most << STEP_BITS;
        return g;
    }
    g.L.chunks = (int)std::min<long long>(t->L.units, g.blocks * rounds);
    g.L.step = g.L.chunks ? (((long long)t->L.units << STEP_BITS) + g.L.chunks - 1) / g.L.chunks : 0;
    return g;
}

// Lists whose norm every block adds up for itself, in the kernel that needs it: two trips to memory for the 16 waves of a block.  Measured with 4 / 12 /
// 35 units, us, this and two kernels: clipping 4.4 / 5.2 / 7.0 and 7.4 / 7.4 / 7.6, AdamW 5.8 / 6.4 / 9.7 and 10.4 / 10.4 / 10.5; the norm alone by one block and by many
// 3.0 / 3.6 / 5.3 and 4.5 / 4.5 / 4.5.
constexpr int SHORT_UNITS = 32;
bool is_short(const fs_tensors *t) { return t->L.units <= SHORT_UNITS; }
int short_blocks(const fs_tensors *t) { return std::max(1, (t->L.units * (UNIT / SHORT_PART) + SHORT_WAVES - 1) / SHORT_WAVES); }

// Bytes at the end of the gradients that the norm leaves in the caches (256 MiB of them in front of the memory), for the pass behind it, which comes from that
// end (none for a norm alone).  What is before them streams: 400 M fp32 then take 234 us, not 259, and 228 where all of it streams.  Measured with 64 / 128 / 192 / 240
// MB, clipping 250 M fp32: 512 / 490 / 497 / 492 us.
constexpr double KEPT_BYTES = 192e6;

// What a pass leaves in the caches, by the bytes that it reads and writes (of AdamW's parameters, by theirs alone).  Measured with three lists in turn, us.
// Clipping, cached / past the caches: 5 M fp32 (40 MB) 15.6 / 17.1, 10 M 24.0 / 25.0, 20 M 50.6 / 43.5, 250 M 534 / 498.  AdamW, all cached / all but the
// parameters past the caches / all of it: 5 M fp32 (140 MB, 20 of parameters) 32.2 / 34.1 / 35.5, 10 M 67 / 57 / 60, 20 M 124 / 107 / 110, 40 M 248 / 221 / 208, 160 M
// 968 / 939 / 880; bf16 with masters 5 M 31.8 / 36.7 / 37.4, 20 M 122 / 107 / 112, 40 M (80 MB of parameters) 236 / 208 / 212, 160 M 933 / 861 / 842.
constexpr double CLIP_CACHED_BYTES = 112e6, ADAM_CACHED_BYTES = 192e6, ADAM_PARAM_BYTES = 96e6;

// The norm into d_norm, or, d_norm == NULL, as sums for the kernel behind it: their number is returned.
int launch_norm(fs_tensors *t, int32_t kind, double scale, float *d_norm)
{
    if (is_short(t) && d_norm) {
        if (kind == FS_NORM_TWO) k_norm_short<KIND_TWO><<<1, SHORT_THREADS, 0, t->stream>>>(t->L, scale, d_norm);
        else k_norm_short<KIND_MAX><<<1, SHORT_THREADS, 0, t->stream>>>(t->L, scale, d_norm);
        return 0;
    }
    const Grid g = grid_for(t, norm_is_long(t) ? NORM_LONG : NORM);
    const int streamed = t->grad_bytes > KEPT_BYTES ? (d_norm ? g.L.chunks : (int)(g.L.chunks * (1.0 - KEPT_BYTES / t->grad_bytes))) : 0;
    if (kind == FS_NORM_TWO) k_norm<KIND_TWO><<<g.blocks, 256, 0, t->stream>>>(g.L, streamed, scale, t->partial, t->tickets, d_norm);
    else k_norm<KIND_MAX><<<g.blocks, 256, 0, t->stream>>>(g.L, streamed, scale, t->partial, t->tickets, d_norm);
    return g.blocks;
}

// Where things lie in a list's memory: TensorD [count], int [count + 1], double [TRAIN_BLOCKS], unsigned [TICKETS].
struct Places { size_t first, partial, tickets, end; };
Places places_for(int32_t count)
{
    Places p;
    p.first = (size_t)count * sizeof(TensorD);
    p.partial = (p.first + ((size_t)count + 1) * sizeof(int) + 255) / 256 * 256;
    p.tickets = p.partial + TRAIN_BLOCKS * sizeof(double);
    p.end = p.tickets + TICKETS * sizeof(unsigned);
    return p;
}

bool scale_ok(double s) { return s > 0.0 && std::isfinite(s); }

// A list in memory of the caller's, or, workspace == NULL, of its own.
fs_status create(const fs_tensor *list, int32_t count, void *hip_stream, void *workspace, fs_tensors **out)
{
    if (out) *out = nullptr;
    if (!out || (!list && count > 0)) return FS_E_ARG;
    if (count < 0 || count > FS_MAX_TENSORS) return FS_E_SHAPE;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) {
        (void)hipGetLastError();
        return FS_E_DEVICE;
    }
    fs_tensors *t = new (std::nothrow) fs_tensors;
    if (!t) return FS_E_ALLOC;
    std::memset(t, 0, sizeof *t);
    t->stream = static_cast<hipStream_t>(hip_stream);
    t->device = dev;
    t->asked = count;
    t->given = new (std::nothrow) fs_tensor[count + 1];
    t->host = new (std::nothrow) TensorD[count + 1];
    fs_status s = t->given && t->host ? FS_OK : FS_E_ALLOC;
    if (s == FS_OK) s = check_list(t, "fs_tensors_create", list, count, nullptr);
    if (s == FS_OK && workspace && !on_device(t, workspace)) s = FS_E_ARG;
    if (s == FS_OK) {
        if (hipDeviceGetAttribute(&t->n_cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || t->n_cus < 1) t->n_cus = 256;
        (void)hipGetLastError();
        t->n_cus = std::min(t->n_cus, TRAIN_BLOCKS / NORM.per_cu);
        const Places at = places_for(count);
        t->mem = static_cast<char *>(workspace);
        t->owned = !workspace;
        if (t->owned && hipMalloc(reinterpret_cast<void **>(&t->mem), at.end) != hipSuccess) {
            (void)hipGetLastError();
            t->mem = nullptr;
            s = FS_E_ALLOC;
        } else {
            t->L.tensors = reinterpret_cast<TensorD *>(t->mem);
            t->L.first = reinterpret_cast<int *>(t->mem + at.first);
            t->partial = reinterpret_cast<double *>(t->mem + at.partial);
            t->tickets = reinterpret_cast<unsigned *>(t->mem + at.tickets);
            if (t->owned) k_tickets_clear<<<1, 256, 0, t->stream>>>(t->tickets);
            s = put_list(t, "fs_tensors_create", list, t->owned ? nullptr : t->tickets);
        }
    }
    if (s != FS_OK) {
        if (t->mem && t->owned) (void)hipFree(t->mem);
        delete[] t->given;
        delete[] t->host;
        delete t;
        return s;
    }
    *out = t;
    return FS_OK;
}

}  // namespace

extern "C" {

const char *fs_tensors_error(const fs_tensors *t) { return t ? t->err : "null list"; }

int64_t fs_tensors_bytes(int32_t count) { return count < 0 || count > FS_MAX_TENSORS ? 0 : (int64_t)places_for(count).end; }

fs_status fs_tensors_create(const fs_tensor *list, int32_t count, void *hip_stream, fs_tensors **out) { return create(list, count, hip_stream, nullptr, out); }

fs_status fs_tensors_create_noalloc(const fs_tensor *list, int32_t count, void *hip_stream, void *workspace, int64_t bytes, fs_tensors **out)
{
    if (out) *out = nullptr;
    if (count >= 0 && count <= FS_MAX_TENSORS && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || bytes < fs_tensors_bytes(count))) return FS_E_ARG;
    return create(list, count, hip_stream, workspace, out);
}

fs_status fs_tensors_destroy(fs_tensors *t)
{
    if (!t) return FS_OK;
    if (t->owned) {
        (void)hipStreamSynchronize(t->stream);
        const hipError_t e = hipFree(t->mem);
        (void)hipGetLastError();
        if (e != hipSuccess) return fail(t, FS_E_DEVICE, "fs_tensors_destroy: %s", hipGetErrorString(e));
    }
    delete[] t->given;
    delete[] t->host;
    delete t;
    return FS_OK;
}

fs_status fs_tensors_update(fs_tensors *t, const fs_tensor *list, int32_t count)
{
    FS_TRAIN_BEGIN(t, false);
    if (count != t->asked) return fail(t, FS_E_SHAPE, "fs_tensors_update: the list has %d tensors, not %d", t->asked, count);
    if (!list && count) return fail(t, FS_E_ARG, "fs_tensors_update: list is NULL");
    const fs_status s = check_list(t, "fs_tensors_update", list, count, t->given);
    return s == FS_OK ? put_list(t, "fs_tensors_update", list, nullptr) : s;
}

fs_status fs_tensors_set_stream(fs_tensors *t, void *hip_stream)
{
    if (!t) return FS_E_ARG;
    t->stream = static_cast<hipStream_t>(hip_stream);
    return FS_OK;
}

fs_status fs_tensors_ready(fs_tensors *t)
{
    FS_TRAIN_BEGIN(t, true);
    return FS_OK;
}

fs_status fs_grad_norm(fs_tensors *t, int32_t kind, double grad_scale, float *d_norm)
{
    FS_TRAIN_BEGIN(t, true);
    if (kind != FS_NORM_TWO && kind != FS_NORM_MAX) return fail(t, FS_E_ARG, "fs_grad_norm: bad kind");
    if (!scale_ok(grad_scale)) return fail(t, FS_E_ARG, "fs_grad_norm: grad_scale must be positive and finite");
    if (!word_ok(t, d_norm, 4)) return fail(t, FS_E_ARG, "fs_grad_norm: d_norm must be a device pointer");
    launch_norm(t, kind, grad_scale, d_norm);
    return launch_status(t, "fs_grad_norm");
}

fs_status fs_grad_clip(fs_tensors *t, int32_t kind, double max_norm, double grad_scale, int32_t norm_given, float *d_norm)
{
    FS_TRAIN_BEGIN(t, true);
    if (norm_given != 0 && norm_given != 1) return fail(t, FS_E_ARG, "fs_grad_clip: norm_given must be 0 or 1");
    if (!norm_given && kind != FS_NORM_TWO && kind != FS_NORM_MAX) return fail(t, FS_E_ARG, "fs_grad_clip: bad kind");
    if (!(max_norm >= 0.0)) return fail(t, FS_E_ARG, "fs_grad_clip: max_norm must not be negative");
    if (!scale_ok(grad_scale)) return fail(t, FS_E_ARG, "fs_grad_clip: grad_scale must be positive and finite");
    if (!word_ok(t, d_norm, 4)) return fail(t, FS_E_ARG, "fs_grad_clip: d_norm must be a device pointer");
    if (!norm_given && t->apart && is_short(t)) {
        if (kind == FS_NORM_TWO) k_clip_short<KIND_TWO><<<short_blocks(t), SHORT_THREADS, 0, t->stream>>>(t->L, max_norm, grad_scale, d_norm);
        else k_clip_short<KIND_MAX><<<short_blocks(t), SHORT_THREADS, 0, t->stream>>>(t->L, max_norm, grad_scale, d_norm);
        return launch_status(t, "fs_grad_clip");
    }
    const NormD N = {t->partial, norm_given ? 0 : launch_norm(t, kind, grad_scale, nullptr), kind, grad_scale, d_norm};
    const Grid g = grid_for(t, CLIP);
    if (2.0 * t->grad_bytes > CLIP_CACHED_BYTES) k_clip<true><<<g.blocks, 256, 0, t->stream>>>(g.L, N, t->in_place, max_norm, grad_scale);
    else k_clip<false><<<g.blocks, 256, 0, t->stream>>>(g.L, N, t->in_place, max_norm, grad_scale);
    return launch_status(t, "fs_grad_clip");
}

fs_status fs_adamw_step(fs_tensors *t, const fs_adamw *how, int64_t *d_step, float *d_norm)
{
    FS_TRAIN_BEGIN(t, true);
    if (!how) return fail(t, FS_E_ARG, "fs_adamw_step: how is NULL");
    const fs_adamw &h = *how;
    if (!std::isfinite(h.lr) || !std::isfinite(h.weight_decay)) return fail(t, FS_E_ARG, "fs_adamw_step: lr and weight_decay must be finite");
    if (!(h.beta1 >= 0.0 && h.beta1 < 1.0 && h.beta2 >= 0.0 && h.beta2 < 1.0)) return fail(t, FS_E_ARG, "fs_adamw_step: betas must be in [0, 1)");
    if (!(h.eps >= 0.0) || !std::isfinite(h.eps)) return fail(t, FS_E_ARG, "fs_adamw_step: eps must be finite and not negative");
    if (!(h.max_norm >= 0.0)) return fail(t, FS_E_ARG, "fs_adamw_step: max_norm must not be negative");
    if (!scale_ok(h.grad_scale)) return fail(t, FS_E_ARG, "fs_adamw_step: grad_scale must be positive and finite");
    if ((h.norm_given != 0 && h.norm_given != 1) || (h.skip_nonfinite != 0 && h.skip_nonfinite != 1))
        return fail(t, FS_E_ARG, "fs_adamw_step: norm_given and skip_nonfinite must be 0 or 1");
    if (!d_norm && (h.norm_given || h.skip_nonfinite || std::isfinite(h.max_norm)))
        return fail(t, FS_E_ARG, "fs_adamw_step: d_norm is NULL, but a norm is asked for");
    if (d_norm && !word_ok(t, d_norm, 4)) return fail(t, FS_E_ARG, "fs_adamw_step: d_norm must be a device pointer");
    if (!word_ok(t, d_step, 8)) return fail(t, FS_E_ARG, "fs_adamw_step: d_step must be a device pointer");
    if (h.d_lr && !word_ok(t, h.d_lr, 4)) return fail(t, FS_E_ARG, "fs_adamw_step: d_lr must be a device pointer or NULL");
    if (!t->params || !t->moments) return fail(t, FS_E_STATE, "fs_adamw_step: tensors without param, exp_avg or exp_avg_sq");
    AdamD A;
    A.log_beta1 = std::log(h.beta1);
    A.log_beta2 = std::log(h.beta2);
    A.max_norm = h.max_norm;
    A.scale = h.grad_scale;
    A.lr = (float)h.lr;
    A.beta1 = (float)h.beta1;
    A.beta2 = (float)h.beta2;
    A.rest1 = (float)(1.0 - h.beta1);
    A.rest2 = (float)(1.0 - h.beta2);
    A.eps = h.eps > 0.0 ? std::max((float)h.eps, std::numeric_limits<float>::denorm_min()) : 0.0f;      // 0 / (0 + eps) stays 0, not NaN
    A.decay = (float)h.weight_decay;
    A.skip_nonfinite = h.skip_nonfinite;
    long long *steps = reinterpret_cast<long long *>(d_step);
    const bool computed = d_norm && !h.norm_given;
    if (computed && is_short(t)) {
        k_adamw_short<<<short_blocks(t), SHORT_THREADS, 0, t->stream>>>(t->L, A, h.d_lr, d_norm, steps, t->tickets);
        return launch_status(t, "fs_adamw_step");
    }
    const NormD N = {t->partial, computed ? launch_norm(t, FS_NORM_TWO, h.grad_scale, nullptr) : 0, FS_NORM_TWO, h.grad_scale, d_norm};
    const Grid g = grid_for(t, ADAMW);
    if (t->param_bytes > ADAM_PARAM_BYTES) k_adamw<ADAM_STREAM><<<g.blocks, 256, 0, t->stream>>>(g.L, A, N, h.d_lr, steps, t->tickets);
    else if (t->adam_bytes > ADAM_CACHED_BYTES) k_adamw<ADAM_PARAM><<<g.blocks, 256, 0, t->stream>>>(g.L, A, N, h.d_lr, steps, t->tickets);
    else k_adamw<ADAM_CACHED><<<g.blocks, 256, 0, t->stream>>>(g.L, A, N, h.d_lr, steps, t->tickets);
    return launch_status(t, "fs_adamw_step");
}

}  // extern "C"
