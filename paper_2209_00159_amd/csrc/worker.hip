// The worker's side of a batch (C ABI in include/orloj.h, orloj_worker_*): the
// operators of a text model's step that depend on which requests the scheduler
// put together.
//
//   adapt_down_kernel, adapt_up_kernel   h = A_a x, then y = base + s B_a h
//   cache_write_kernel, cache_read_kernel  keys and values <-> 8-bit pages
//   attend_kernel                        attention of the rows over the pages

#include <hip/hip_fp8.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <new>
#include <vector>

#include "../../include/orloj.h"
#include "orloj_ctx.h"

struct orloj_worker {
    orloj_ctx* ctx;
    int device;                      // the context's: destroying may come after its end
    int* d_err;                      // device status word (data error bits)
    hipStream_t stream;              // of the last call
    std::vector<orloj_block> blocks; // scratch, the last one in use; captured calls may name any
};

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// Device-side data error bits (reported by orloj_worker_sync).
constexpr int kErrAdapter = 1;
constexpr int kErrRank = 2;
constexpr int kErrRows = 4;
constexpr int kErrLength = 8;
constexpr int kErrPage = 16;

constexpr float kTiny = 0x1p-100f;   // vectors below this are stored as zeros

// ---------------------------------------------------------------------------
// element types
// ---------------------------------------------------------------------------
struct F32 {
    using T = float;
    static __device__ __forceinline__ float up(T x) { return x; }
    static __device__ __forceinline__ T down(float x) { return x; }
};
struct F16 {
    using T = _Float16;
    static __device__ __forceinline__ float up(T x) { return (float)x; }
    static __device__ __forceinline__ T down(float x) { return (T)x; }
};
struct BF16 {
    using T = __bf16;
    static __device__ __forceinline__ float up(T x) { return (float)x; }
    static __device__ __forceinline__ T down(float x) { return (T)x; }
};

// ---------------------------------------------------------------------------
// adapters
// ---------------------------------------------------------------------------
struct AdaptArgs {
    int n, rank, d_in, d_out;
    int64_t rows, xs, bs, ys;
    const void *down, *up, *x, *base;
    void* y;
    const float* scale;
    const int32_t *ranks, *adapter;
    float* h;        // [rows][rank]
    int* err;
};

// Row t's adapter and its rank (0: none).
__device__ __forceinline__ int adapter_of(const AdaptArgs& a, int64_t t, int& rank) {
    int id = a.adapter[t];
    rank = 0;
    if (id < -1 || id >= a.n) {
        atomicOr(a.err, kErrAdapter);
        id = -1;
    }
    if (id >= 0) {
        rank = a.ranks ? a.ranks[id] : a.rank;
        if (rank < 0 || rank > a.rank) {
            atomicOr(a.err, kErrRank);
            rank = min(max(rank, 0), a.rank);
        }
    }
    return id;
}

// One workgroup per row, a wave per rank in turn: h[t][r] = A_a[r] . x_t.
template <class E>
__global__ __launch_bounds__(kThreads) void adapt_down_kernel(AdaptArgs a) {
    using T = typename E::T;
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int rank;
    const int id = adapter_of(a, t, rank);
    const T* x = (const T*)a.x + t * a.xs;
    for (int r = wave; r < rank; r += kWaves) {
        const T* w = (const T*)a.down + ((int64_t)id * a.rank + r) * a.d_in;
        float s = 0.0f;
        for (int k = lane; k < a.d_in; k += 64) s = fmaf(E::up(w[k]), E::up(x[k]), s);
        for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m, 64);
        if (lane == 0) a.h[t * a.rank + r] = s;
    }
}

// A thread per output element.
template <class E>
__global__ __launch_bounds__(kThreads) void adapt_up_kernel(AdaptArgs a) {
    using T = typename E::T;
    const int64_t t = blockIdx.x;
    const int o = blockIdx.y * kThreads + threadIdx.x;
    if (o >= a.d_out) return;
    int rank;
    const int id = adapter_of(a, t, rank);
    float s = 0.0f;
    if (rank) {
        const T* w = (const T*)a.up + ((int64_t)id * a.d_out + o) * a.rank;
        for (int r = 0; r < rank; ++r) s = fmaf(E::up(w[r]), a.h[t * a.rank + r], s);
        if (a.scale) s *= a.scale[id];
    }
    if (a.base) s += E::up(((const T*)a.base)[t * a.bs + o]);
    ((T*)a.y)[t * a.ys + o] = E::down(s);
}

// ---------------------------------------------------------------------------
// the cache
// ---------------------------------------------------------------------------
struct CacheArgs {
    int pages, page, shift, heads, dim, pad, format;
    uint8_t *k, *v;
    float *ks, *vs;
    int requests, max_pages, max_rows, max_length;
    int64_t rows;
    const int32_t *off, *len, *table;
    int* err;
};

// What a request's offsets and length say: false (and a data error) where they
// cannot be.
__device__ __forceinline__ bool request_of(const CacheArgs& c, int r, int64_t& first, int& rows, int& length) {
    const int a = c.off[r], b = c.off[r + 1];
    length = c.len[r];
    first = a;
    rows = b - a;
    int bad = 0;
    if (a < 0 || b < a || b > c.rows || rows > c.max_rows) bad |= kErrRows;
    if (length < rows || length > c.max_length || length > (int64_t)c.max_pages << c.shift) bad |= kErrLength;
    if (bad) atomicOr(c.err, bad);
    return !bad;
}

// Request and position of a row, found by the 16 lanes of a group together:
// each round's 16 probes cut the candidates to a sixteenth.
__device__ __forceinline__ bool place_of_row(const CacheArgs& c, int64_t row, int& req, int& pos) {
    const int lane = threadIdx.x & 63, sub = lane & 15;
    int lo = 0, n = c.requests;            // the request is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 15) >> 4;
        const int p = lo + (sub + 1) * step;   // first row of request p
        const bool past = p < lo + n && c.off[p] <= row;
        const uint64_t m = __ballot(past) >> (lane & 48) & 0xffff;
        const int k = __popcll(m);
        const int from = lo + k * step;
        n = min(step, lo + n - from);
        lo = from;
    }
    int64_t first;
    int rows, length;
    req = lo;
    if (!request_of(c, lo, first, rows, length)) return false;
    if (row < first || row >= first + rows) {
        atomicOr(c.err, kErrRows);
        return false;
    }
    pos = length - rows + (int)(row - first);
    return true;
}

// Offset of a token's slot among all (page, head, slot) triples, -1 where the
// table is wrong.
__device__ __forceinline__ int64_t slot_of(const CacheArgs& c, int req, int pos, int head) {
    const int p = c.table[(int64_t)req * c.max_pages + (pos >> c.shift)];
    if (p < 0 || p >= c.pages) {
        atomicOr(c.err, kErrPage);
        return -1;
    }
    return (((int64_t)p * c.heads + head) << c.shift) + (pos & (c.page - 1));
}

__device__ __forceinline__ uint8_t to_fp8(float x) {
    return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false);
}
__device__ __forceinline__ float from_code(int format, uint8_t b) {
    return format == ORLOJ_CACHE_INT8 ? (float)(int8_t)b : __builtin_amdgcn_cvt_f32_fp8(b, 0);
}

struct Vectors {
    void* d;
    int64_t row, head;
};

// 16 lanes a vector, 16 vectors a workgroup.
template <class E>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CacheArgs c, Vectors k, Vectors v) {
    using T = typename E::T;
    const int sub = threadIdx.x & 15;
    const int64_t i = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    const int64_t row = i / (2 * c.heads);
    const int which = (int)(i - row * 2 * c.heads);
    const int head = which % c.heads;
    if (row >= c.rows) return;
    int req, pos;
    if (!place_of_row(c, row, req, pos)) return;
    const int64_t slot = slot_of(c, req, pos, head);
    if (slot < 0) return;
    const Vectors& from = which < c.heads ? k : v;
    const T* x = (const T*)from.d + row * from.row + head * from.head;
    float amax = 0.0f;
    for (int d = sub; d < c.dim; d += 16) {
        const float a = fabsf(E::up(x[d]));
        amax = a > amax || a != a ? a : amax;
    }
    for (int m = 8; m; m >>= 1) {
        const float o = __shfl_xor(amax, m, 64);
        amax = o > amax || o != o ? o : amax;
    }
    const bool bad = !(amax < INFINITY), low = amax < kTiny;
    const float top = c.format == ORLOJ_CACHE_INT8 ? 127.0f : 448.0f;
    const float inv = (1.0f / (bad || low ? 1.0f : amax)) * top;
    uint8_t* code = (which < c.heads ? c.k : c.v) + slot * c.pad;
    for (int d = sub; d < c.pad; d += 16) {
        const float y = d < c.dim && !bad && !low ? E::up(x[d]) * inv : 0.0f;
        code[d] = c.format == ORLOJ_CACHE_INT8 ? (uint8_t)(int8_t)rintf(y) : to_fp8(y);
    }
    if (sub == 0) (which < c.heads ? c.ks : c.vs)[slot] = bad ? NAN : low ? 0.0f : amax * (1.0f / top);
}

template <class E>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CacheArgs c, Vectors k, Vectors v) {
    using T = typename E::T;
    const int sub = threadIdx.x & 15;
    const int64_t i = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    const int64_t row = i / (2 * c.heads);
    const int which = (int)(i - row * 2 * c.heads);
    const int head = which % c.heads;
    if (row >= c.rows) return;
    int req, pos;
    if (!place_of_row(c, row, req, pos)) return;
    const int64_t slot = slot_of(c, req, pos, head);
    if (slot < 0) return;
    const Vectors& to = which < c.heads ? k : v;
    T* x = (T*)to.d + row * to.row + head * to.head;
    const uint8_t* code = (which < c.heads ? c.k : c.v) + slot * c.pad;
    const float s = (which < c.heads ? c.ks : c.vs)[slot];
    for (int d = sub; d < c.dim; d += 16) x[d] = E::down(from_code(c.format, code[d]) * s);
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------
struct AttendArgs {
    CacheArgs c;
    Vectors q, out;
    const uint64_t* tree;
    float* lse;
    float scale;
    int q_heads, group;
};

// A wave per (request, row, query head): 64 tokens at a time, a token a lane for
// the scores, then a dimension a lane for the weighted sum.
template <class E>
__global__ __launch_bounds__(64) void attend_kernel(AttendArgs a) {
    using T = typename E::T;
    const CacheArgs& c = a.c;
    const int lane = threadIdx.x, r = blockIdx.z, i = blockIdx.x, qh = blockIdx.y, head = qh / a.group;
    __shared__ float q[ORLOJ_MAX_HEAD_DIM];
    int64_t first;
    int rows, length;
    if (!request_of(c, r, first, rows, length) || i >= rows) return;
    const T* x = (const T*)a.q.d + (first + i) * a.q.row + qh * a.q.head;
    for (int d = lane; d < c.dim; d += 64) q[d] = E::up(x[d]) * a.scale;
    __syncthreads();
    const int context = length - rows;
    const uint64_t mask = a.tree ? a.tree[first + i] : 0;
    float m = -INFINITY, l = 0.0f, o[4] = {};
    const int end = a.tree ? length : context + i + 1;
    for (int t0 = 0; t0 < end; t0 += 64) {
        const int t = t0 + lane;
        bool sees = t < end && (!a.tree || t < context || (mask >> (t - context) & 1));
        int64_t slot = -1;
        if (t < end) slot = slot_of(c, r, t, head);
        sees = sees && slot >= 0;
        float s = -INFINITY, w = 0.0f;
        if (sees) {
            const uint8_t* k = c.k + slot * c.pad;
            float dot = 0.0f;
            for (int d = 0; d < c.dim; ++d) dot = fmaf(q[d], from_code(c.format, k[d]), dot);
            s = dot * c.ks[slot];
        }
        float top = s;
        for (int k = 32; k; k >>= 1) {
            const float other = __shfl_xor(top, k, 64);
            top = other > top || other != other ? other : top;
        }
        top = m > top ? m : top;
        if (top == -INFINITY) continue;
        const float keep = __expf(m - top);
        if (sees) w = expf(s - top);
        m = top;
        float sum = w;
        for (int k = 32; k; k >>= 1) sum += __shfl_xor(sum, k, 64);
        l = l * keep + sum;
        for (int j = 0; j < 4; ++j) o[j] *= keep;
        for (int k = 0; k < 64; ++k) {
            if (!__shfl((int)sees, k, 64)) continue;
            const float p = __shfl(w, k, 64);
            const int64_t at = __shfl(slot, k, 64);
            const float pv = p * c.vs[at];
            for (int j = 0; j < 4; ++j)
                if (lane + 64 * j < c.dim) o[j] = fmaf(pv, from_code(c.format, c.v[at * c.pad + lane + 64 * j]), o[j]);
        }
    }
    T* y = (T*)a.out.d + (first + i) * a.out.row + qh * a.out.head;
    for (int j = 0; j < 4; ++j)
        if (lane + 64 * j < c.dim) y[lane + 64 * j] = E::down(l != 0.0f ? o[j] / l : 0.0f);
    if (a.lse && lane == 0) a.lse[(first + i) * a.q_heads + qh] = l != 0.0f ? m + logf(l) : -INFINITY;
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
int hip_err(orloj_ctx* ctx, hipError_t e, const char* what) {
    return orloj_ctx_fail(ctx, e == hipErrorOutOfMemory ? ORLOJ_E_NOMEM : ORLOJ_E_HIP, "%s: %s", what,
                          hipGetErrorString(e));
}

// What every call does first: the device, and the previous stream's work where
// the context's stream has changed (it may still use the scratch).
int enter(orloj_worker* w) {
    hipError_t e = hipSetDevice(w->ctx->device);
    if (e == hipSuccess && w->stream != w->ctx->stream) e = hipStreamSynchronize(w->stream);
    if (e != hipSuccess) return hip_err(w->ctx, e, "entering a worker call");
    w->stream = w->ctx->stream;
    return ORLOJ_OK;
}

int scratch(orloj_worker* w, size_t bytes, void** out) {
    if (w->blocks.empty() || w->blocks.back().bytes < bytes) {
        hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
        hipError_t e = hipStreamIsCapturing(w->ctx->stream, &st);
        if (e != hipSuccess) return hip_err(w->ctx, e, "hipStreamIsCapturing");
        if (st != hipStreamCaptureStatusNone)
            return orloj_ctx_fail(w->ctx, ORLOJ_E_INVALID,
                                  "the worker's scratch cannot grow to %zu bytes under capture: "
                                  "make a call of these sizes before it", bytes);
        // at least twice the last, so that what is kept of smaller ones stays below this one
        size_t want = std::max(bytes, w->blocks.empty() ? (size_t)1 << 20 : 2 * w->blocks.back().bytes);
        void* p = nullptr;
        e = hipMalloc(&p, want);
        if (e == hipErrorOutOfMemory && want > bytes) {
            (void)hipGetLastError();
            e = hipMalloc(&p, want = bytes);
        }
        if (e != hipSuccess) {
            (void)hipGetLastError();
            return hip_err(w->ctx, e, "growing the worker's scratch");
        }
        try {
            w->blocks.push_back(orloj_block{p, want});
        } catch (const std::bad_alloc&) {
            (void)hipFree(p);
            return orloj_ctx_fail(w->ctx, ORLOJ_E_NOMEM, "out of host memory");
        }
    }
    *out = w->blocks.back().p;
    return ORLOJ_OK;
}

// The launch's own status: the runtime's last error may be another library's.
template <class... A>
int launch(orloj_worker* w, const char* what, void (*kernel)(A...), dim3 grid, int threads, A... args) {
    void* p[] = {(void*)&args...};
    const hipError_t e = hipLaunchKernel((const void*)kernel, grid, dim3(threads), p, 0, w->ctx->stream);
    return e == hipSuccess ? ORLOJ_OK : hip_err(w->ctx, e, what);
}

int cache_args(orloj_worker* w, const orloj_cache* c, const orloj_batch* b, CacheArgs* a) {
    orloj_ctx* x = w->ctx;
    if (!c || !b) return orloj_ctx_fail(x, ORLOJ_E_INVALID, "cache or batch is NULL");
    int shift = 0;
    while (shift < 9 && 1 << shift != c->page_size) ++shift;
    if (shift < 4 || shift > 8)
        return orloj_ctx_fail(x, ORLOJ_E_INVALID, "page_size %d is not 16, 32, 64, 128 or 256", c->page_size);
    if (c->n_pages < 0 || c->n_heads < 1 || c->head_dim < 1)
        return orloj_ctx_fail(x, ORLOJ_E_INVALID, "n_pages %d, n_heads %d or head_dim %d out of range", c->n_pages,
                              c->n_heads, c->head_dim);
    if (c->head_dim > ORLOJ_MAX_HEAD_DIM)
        return orloj_ctx_fail(x, ORLOJ_E_UNSUPPORTED, "head_dim %d > %d", c->head_dim, ORLOJ_MAX_HEAD_DIM);
    if (c->format != ORLOJ_CACHE_INT8 && c->format != ORLOJ_CACHE_FP8)
        return orloj_ctx_fail(x, ORLOJ_E_INVALID, "unknown cache format %d", c->format);
    if (b->n_requests < 0 || b->max_pages < 0 || b->n_rows < 0 || b->max_rows < 0 || b->max_length < 0)
        return orloj_ctx_fail(x, ORLOJ_E_INVALID, "a size of the batch is negative");
    if (b->n_rows > INT32_MAX)
        return orloj_ctx_fail(x, ORLOJ_E_UNSUPPORTED, "n_rows %lld > 2^31 - 1", (long long)b->n_rows);
    if (b->n_requests == 0 && b->n_rows > 0)
        return orloj_ctx_fail(x, ORLOJ_E_INVALID, "%lld rows of no requests", (long long)b->n_rows);
    if (b->n_rows > 0) {
        if (!c->d_k || !c->d_v || !c->d_k_scale || !c->d_v_scale || !b->d_row_off || !b->d_length || !b->d_pages)
            return orloj_ctx_fail(x, ORLOJ_E_INVALID, "NULL buffer of the cache or the batch");
        if (((uintptr_t)c->d_k | (uintptr_t)c->d_v | (uintptr_t)c->d_k_scale | (uintptr_t)c->d_v_scale) & 15)
            return orloj_ctx_fail(x, ORLOJ_E_INVALID, "the cache is not aligned to 16 bytes");
    }
    *a = CacheArgs{c->n_pages, c->page_size, shift, c->n_heads, c->head_dim, (c->head_dim + 63) & ~63, c->format,
                   (uint8_t*)c->d_k, (uint8_t*)c->d_v, c->d_k_scale, c->d_v_scale, b->n_requests, b->max_pages,
                   b->max_rows, b->max_length, b->n_rows, b->d_row_off, b->d_length, b->d_pages, w->d_err};
    return ORLOJ_OK;
}

int vectors(orloj_worker* w, const orloj_vectors* v, int64_t rows, const char* name, Vectors* out) {
    if (!v) return orloj_ctx_fail(w->ctx, ORLOJ_E_INVALID, "%s is NULL", name);
    if (rows > 0 && !v->d) return orloj_ctx_fail(w->ctx, ORLOJ_E_INVALID, "%s has no buffer", name);
    if (v->row_stride < 0 || v->head_stride < 0)
        return orloj_ctx_fail(w->ctx, ORLOJ_E_INVALID, "%s has a negative stride", name);
    *out = Vectors{v->d, v->row_stride, v->head_stride};
    return ORLOJ_OK;
}

int cache_copy(orloj_worker* w, const orloj_cache* cache, const orloj_batch* batch, int32_t dtype,
               const orloj_vectors* k, const orloj_vectors* v, bool write) {
    if (!w) return ORLOJ_E_INVALID;
    CacheArgs c;
    Vectors kv, vv;
    if (int rc = cache_args(w, cache, batch, &c)) return rc;
    if (int rc = vectors(w, k, c.rows, "k", &kv)) return rc;
    if (int rc = vectors(w, v, c.rows, "v", &vv)) return rc;
    if (dtype != ORLOJ_F32 && dtype != ORLOJ_F16 && dtype != ORLOJ_BF16)
        return orloj_ctx_fail(w->ctx, ORLOJ_E_INVALID, "unknown dtype %d", dtype);
    const int64_t groups = (c.rows * 2 * c.heads + kThreads / 16 - 1) / (kThreads / 16);
    if (groups > INT32_MAX)
        return orloj_ctx_fail(w->ctx, ORLOJ_E_UNSUPPORTED, "%lld rows of %d heads are too many for one call",
                              (long long)c.rows, c.heads);
    if (int rc = enter(w)) return rc;
    if (c.rows == 0) return ORLOJ_OK;
    const dim3 g((unsigned)groups);
    if (write) {
        auto kernel = dtype == ORLOJ_F32 ? cache_write_kernel<F32> : dtype == ORLOJ_F16 ? cache_write_kernel<F16>
                                                                                   : cache_write_kernel<BF16>;
        return launch(w, "cache_write_kernel", kernel, g, kThreads, c, kv, vv);
    }
    auto kernel = dtype == ORLOJ_F32 ? cache_read_kernel<F32> : dtype == ORLOJ_F16 ? cache_read_kernel<F16>
                                                                               : cache_read_kernel<BF16>;
    return launch(w, "cache_read_kernel", kernel, g, kThreads, c, kv, vv);
}

}  // namespace

extern "C" {

int orloj_worker_create(orloj_worker** out, orloj_ctx* ctx) {
    if (!out) return ORLOJ_E_INVALID;
    *out = nullptr;
    if (!ctx) return ORLOJ_E_INVALID;
    orloj_worker* w = new (std::nothrow) orloj_worker;
    if (!w) return orloj_ctx_fail(ctx, ORLOJ_E_NOMEM, "out of host memory");
    w->ctx = ctx;
    w->device = ctx->device;
    w->d_err = nullptr;
    w->stream = ctx->stream;
    hipError_t e = hipSetDevice(ctx->device);
    if (e == hipSuccess) e = hipMalloc((void**)&w->d_err, sizeof(int));
    if (e == hipSuccess) e = hipMemset(w->d_err, 0, sizeof(int));
    if (e != hipSuccess) {
        if (w->d_err) (void)hipFree(w->d_err);
        delete w;
        return hip_err(ctx, e, "orloj_worker_create");
    }
    *out = w;
    return ORLOJ_OK;
}

void orloj_worker_destroy(orloj_worker* w) {
    if (!w) return;
    (void)hipSetDevice(w->device);
    (void)hipStreamSynchronize(w->stream);
    (void)hipFree(w->d_err);
    for (const orloj_block& b : w->blocks) (void)hipFree(b.p);
    delete w;
}

int orloj_worker_sync(orloj_worker* w) {
    if (!w) return ORLOJ_E_INVALID;
    if (int rc = enter(w)) return rc;
    hipError_t e = hipStreamSynchronize(w->stream);
    if (e != hipSuccess) return hip_err(w->ctx, e, "hipStreamSynchronize");
    int flags = 0;
    e = hipMemcpy(&flags, w->d_err, sizeof(int), hipMemcpyDeviceToHost);
    if (e == hipSuccess && flags) e = hipMemset(w->d_err, 0, sizeof(int));
    if (e != hipSuccess) return hip_err(w->ctx, e, "the worker's status word");
    if (flags)
        return orloj_ctx_fail(w->ctx, ORLOJ_E_DATA, "device data error:%s%s%s%s%s",
                              (flags & kErrAdapter) ? " adapter-id-out-of-range" : "",
                              (flags & kErrRank) ? " rank-out-of-range" : "",
                              (flags & kErrRows) ? " row-offsets-invalid" : "",
                              (flags & kErrLength) ? " length-invalid" : "",
                              (flags & kErrPage) ? " page-out-of-range" : "");
    return ORLOJ_OK;
}

int orloj_worker_adapt(orloj_worker* w, const orloj_adapters* ad, int64_t n_rows, const int32_t* d_adapter,
                       const void* d_x, int64_t x_stride, const void* d_base, int64_t base_stride, void* d_y,
                       int64_t y_stride) {
    if (!w) return ORLOJ_E_INVALID;
    orloj_ctx* x = w->ctx;
    if (!ad) return orloj_ctx_fail(x, ORLOJ_E_INVALID, "adapters is NULL");
    if (ad->n_adapters < 0 || ad->rank < 1 || ad->d_in < 1 || ad->d_out < 1 || n_rows < 0)
        return orloj_ctx_fail(x, ORLOJ_E_INVALID, "a size is out of range: %d adapters, rank %d, %d -> %d, %lld rows",
                              ad->n_adapters, ad->rank, ad->d_in, ad->d_out, (long long)n_rows);
    if (ad->rank > ORLOJ_MAX_RANK)
        return orloj_ctx_fail(x, ORLOJ_E_UNSUPPORTED, "rank %d > %d", ad->rank, ORLOJ_MAX_RANK);
    // so that the grid of rows by blocks of outputs stays within its limits
    if (ad->d_out > 65535 * kThreads) return orloj_ctx_fail(x, ORLOJ_E_UNSUPPORTED, "d_out %d is too wide", ad->d_out);
    if (n_rows > 1 << 20)
        return orloj_ctx_fail(x, ORLOJ_E_UNSUPPORTED, "%lld rows > 2^20", (long long)n_rows);
    if (ad->dtype != ORLOJ_F16 && ad->dtype != ORLOJ_BF16)
        return orloj_ctx_fail(x, ORLOJ_E_INVALID, "adapters are 16-bit floats, not dtype %d", ad->dtype);
    if (x_stride < ad->d_in || y_stride < ad->d_out || (d_base && base_stride < ad->d_out))
        return orloj_ctx_fail(x, ORLOJ_E_INVALID, "a stride is shorter than its row");
    if (n_rows && (!d_adapter || !d_x || !d_y || (ad->n_adapters && (!ad->d_down || !ad->d_up))))
        return orloj_ctx_fail(x, ORLOJ_E_INVALID, "NULL buffer");
    if (d_base && d_base == d_y && base_stride != y_stride)
        return orloj_ctx_fail(x, ORLOJ_E_INVALID, "d_base is d_y with another stride");
    if (int rc = enter(w)) return rc;
    if (!n_rows) return ORLOJ_OK;
    void* h;
    if (int rc = scratch(w, (size_t)n_rows * ad->rank * sizeof(float), &h)) return rc;
    const AdaptArgs a{ad->n_adapters, ad->rank, ad->d_in, ad->d_out, n_rows, x_stride, base_stride, y_stride,
                      ad->d_down, ad->d_up, d_x, d_base, d_y, ad->d_scale, ad->d_rank, d_adapter, (float*)h, w->d_err};
    const bool half = ad->dtype == ORLOJ_F16;
    const dim3 gd((unsigned)n_rows), gu((unsigned)n_rows, (ad->d_out + kThreads - 1) / kThreads);
    if (int rc = launch(w, "adapt_down_kernel", half ? adapt_down_kernel<F16> : adapt_down_kernel<BF16>, gd, kThreads, a))
        return rc;
    return launch(w, "adapt_up_kernel", half ? adapt_up_kernel<F16> : adapt_up_kernel<BF16>, gu, kThreads, a);
}

int orloj_worker_cache_write(orloj_worker* w, const orloj_cache* cache, const orloj_batch* batch, int32_t dtype,
                             const orloj_vectors* k, const orloj_vectors* v) {
    return cache_copy(w, cache, batch, dtype, k, v, true);
}

int orloj_worker_cache_read(orloj_worker* w, const orloj_cache* cache, const orloj_batch* batch, int32_t dtype,
                            const orloj_vectors* k, const orloj_vectors* v) {
    return cache_copy(w, cache, batch, dtype, k, v, false);
}

int orloj_worker_attend(orloj_worker* w, const orloj_cache* cache, const orloj_batch* batch, int32_t dtype,
                        int32_t n_q_heads, float scale, const orloj_vectors* q, const uint64_t* d_tree,
                        const orloj_vectors* out, float* d_lse) {
    if (!w) return ORLOJ_E_INVALID;
    AttendArgs a;
    if (int rc = cache_args(w, cache, batch, &a.c)) return rc;
    if (int rc = vectors(w, q, a.c.rows, "q", &a.q)) return rc;
    if (int rc = vectors(w, out, a.c.rows, "out", &a.out)) return rc;
    if (dtype != ORLOJ_F16 && dtype != ORLOJ_BF16)
        return orloj_ctx_fail(w->ctx, ORLOJ_E_INVALID, "queries are 16-bit floats, not dtype %d", dtype);
    if (n_q_heads < 1 || n_q_heads % a.c.heads)
        return orloj_ctx_fail(w->ctx, ORLOJ_E_INVALID, "%d query heads over %d key heads", n_q_heads, a.c.heads);
    if (!isfinite(scale)) return orloj_ctx_fail(w->ctx, ORLOJ_E_INVALID, "scale is not finite");
    if (d_tree && a.c.max_rows > ORLOJ_MAX_TREE)
        return orloj_ctx_fail(w->ctx, ORLOJ_E_UNSUPPORTED, "a tree of up to %d tokens > %d", a.c.max_rows,
                              ORLOJ_MAX_TREE);
    // grids hold at most 2^16 - 1 workgroups along their second and third axes
    if (n_q_heads > 65535 || a.c.requests > 65535)
        return orloj_ctx_fail(w->ctx, ORLOJ_E_UNSUPPORTED, "more than 65535 heads or requests");
    if (int rc = enter(w)) return rc;
    if (!a.c.rows || !a.c.max_rows) return ORLOJ_OK;
    a.tree = d_tree;
    a.lse = d_lse;
    a.scale = scale;
    a.q_heads = n_q_heads;
    a.group = n_q_heads / a.c.heads;
    const dim3 g(a.c.max_rows, n_q_heads, a.c.requests);
    return launch(w, "attend_kernel", dtype == ORLOJ_F16 ? attend_kernel<F16> : attend_kernel<BF16>, g, 64, a);
}

}  // extern "C"
