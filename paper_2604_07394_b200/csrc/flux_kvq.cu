// Filling and reading the 8-bit KV cache (layout and types: flux_kvq.h).
//
// One warp per (block of 16 positions, K or V, head): 16 rows of 256 bytes in, lane l holding channels 4 l .. 4 l + 3 of
// all 16 rows, so the block's largest magnitude is one warp reduction and both code orders are written from registers
// (K: 64-byte runs, V: 64 consecutive bytes per lane after a byte transposition).  Both directions are bound by memory:
// every byte is read once and written once.
//
// Tasks are numbered without knowing the requests' lengths on the host: request b's blocks start at task
// row_start[b] / 16 + 2 b, which leaves room for the at most n / 16 + 2 blocks that n rows at any position touch; the
// few numbers left over are skipped.  As many CTAs as the GPU holds take the tasks in strides, the requests' bounds in
// shared memory: a CTA per eight tasks spent most of its life on the chain row_start -> position -> rows (3.5 TB/s).
#include "flux_kvq.h"

namespace flux {
namespace {

constexpr int kWarps = 8;
constexpr int kCtasPerSm = 4;

struct KvqArgs {
    const void *src[2];              // store: K, V rows; row stride in bytes
    void *dst[2];                    // load: K, V rows, contiguous
    int64_t stride[2];
    void *const *caches[2];
    const int32_t *row_start;        // [B + 1]
    const int32_t *pos;              // [B]
    const int32_t *ctx_len;          // load: [B]
    const uint8_t *mask;
    int B, L, layer, Hkv, S, W, layout, max_context, total_rows;
    uint32_t tasks;
    uint32_t *status;
};

// Waits for the launches before, then lets the next one start: a launch that begins early (the decode with launch overlap) may
// read what they wrote, so the permission must not be passed on before they are done.
__device__ __forceinline__ void begin_launch()
{
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
}

// Rows [r0, r0 + n) exist, and so do the positions [p, p + n) of a cache of (up to) `ctx` tokens.
__device__ __forceinline__ bool bounds_ok(const KvqArgs &a, int r0, int n, int p, int ctx)
{
    return r0 >= 0 && n >= 0 && r0 <= a.total_rows - n && (n == 0 || (p >= 0 && n <= ctx && ctx <= a.max_context && p <= ctx - n));
}

// Request whose tasks include `slot`: the last b with row_start[b] / 16 + 2 b <= slot, 32 candidates at a time.
__device__ __forceinline__ int find_request(const int *row_start, int B, int slot, int lane)
{
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const int i = lo + lane * step;
        const bool le = i < hi && row_start[i] / kKvqBlock + 2 * i <= slot;
        const int c = __popc(__ballot_sync(0xffffffffu, le));
        lo += (c > 0 ? c - 1 : 0) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

// What the tasks have to know of the requests, in shared memory: read once by each CTA, the loads of a request independent of
// one another, where a task of its own would wait for one after the other before it asks for its rows (store and load
// of 32 tokens of 8 heads 7.2 -> 6.3 us, of four chunks, 57 MB, 22.4 -> 21.2).  32 bytes a request.
struct Requests {
    unsigned char **cache;     // [2][B]: K, V
    int *row_start;            // [B + 1]
    int *pos, *ctx;            // [B]
    int *kind;                 // [B]: 0 nothing to do (no rows, or a check failed), 1 every block is kept, 2 compact sparse cache
    __device__ __forceinline__ Requests(void *sh, int B)
        : cache((unsigned char **)sh), row_start((int *)(cache + 2 * B)), pos(row_start + B + 1), ctx(pos + B), kind(ctx + B) {}
};

__device__ __forceinline__ bool bad_cache(const void *cache) { return cache == nullptr || ((uintptr_t)cache & 15u) != 0; }

// Block 0 reports what the checks find.
__device__ __forceinline__ void stage_requests(const KvqArgs &a, const Requests &s)
{
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
        const int r0 = a.row_start[b], n = a.row_start[b + 1] - r0, p = a.pos[b];
        const int ctx = a.ctx_len != nullptr ? a.ctx_len[b] : a.max_context;
        const int mode = a.mask[(size_t)b * a.L + a.layer];
        unsigned char *k = (unsigned char *)a.caches[0][b], *v = (unsigned char *)a.caches[1][b];
        const bool fits = bounds_ok(a, r0, n, p, ctx), lost = bad_cache(k) || bad_cache(v);
        if (blockIdx.x == 0) {
            const uint32_t bits = !fits ? FLUX_STATUS_BAD_LENGTH
                                        : n == 0 ? 0u : (lost ? FLUX_STATUS_BAD_POINTER : 0u) | (mode > 1 ? FLUX_STATUS_BAD_MASK : 0u);
            if (bits != 0) atomicOr(a.status, bits);
        }
        s.cache[b] = k;
        s.cache[a.B + b] = v;
        s.row_start[b] = r0;
        if (b == a.B - 1) s.row_start[a.B] = r0 + n;
        s.pos[b] = p;
        s.ctx[b] = ctx;
        s.kind[b] = !fits || n == 0 || lost ? 0 : a.layout == FLUX_KV_COMPACT_SA && mode == 0 ? 2 : 1;
    }
    __syncthreads();
}

template <int kFmt>
__device__ __forceinline__ void store_task(const KvqArgs &a, const Requests &s, uint32_t task, int lane)
{
    const int slot = (int)(task / (2u * a.Hkv)), rem = (int)(task % (2u * a.Hkv));
    const int kv = rem >= a.Hkv ? 1 : 0, head = rem - kv * a.Hkv;
    const int b = find_request(s.row_start, a.B, slot, lane);
    if (s.kind[b] == 0) return;
    const int r0 = s.row_start[b], n = s.row_start[b + 1] - r0, p = s.pos[b];
    const int end = p + n, jf = p / kKvqBlock, jl = (end - 1) / kKvqBlock, j = jf + slot - (r0 / kKvqBlock + 2 * b);
    if (j < jf || j > jl) return;
    const bool compact = s.kind[b] == 2;
    unsigned char *cache = s.cache[kv * a.B + b];
    uint2 *tail = reinterpret_cast<uint2 *>(cache + (size_t)head * kKvqTailHeadBytes) + lane;
    const unsigned char *src = (const unsigned char *)a.src[kv] + (size_t)head * kRowBytes + (size_t)lane * 8;
    const int64_t stride = a.stride[kv];
    constexpr int kRow8 = kRowBytes / 8;
    bool bad = false;

    const bool complete = (j + 1) * kKvqBlock <= end;
    const bool wanted = complete && kvq_held(j, end, compact, a.S, a.W);
    // The rows of the call's last block go to the tail, even when they complete it, so that the newest block's tokens may be
    // stored again: beside those already there if the block is alone in this call; else by its own warp where the call's
    // first block starts afresh, or by the first block's warp, the only one that reads the tail, after it has done so.
    const bool begun = p % kKvqBlock != 0;
    const bool to_tail = jf == jl || (j == jl && !begun);
    if (wanted || to_tail) {
        uint2 x[kKvqBlock];
        const int first = j * kKvqBlock;
        if (first >= p && complete) {
            const unsigned char *row = src + (int64_t)(r0 + first - p) * stride;
#pragma unroll
            for (int i = 0; i < kKvqBlock; ++i, row += stride) x[i] = *reinterpret_cast<const uint2 *>(row);
        } else {
#pragma unroll
            for (int i = 0; i < kKvqBlock; ++i) {
                x[i] = make_uint2(0u, 0u);
                if (first + i < p) {
                    if (complete) x[i] = tail[i * kRow8];              // rows that were here before
                } else if (first + i < end) {
                    x[i] = *reinterpret_cast<const uint2 *>(src + (int64_t)(r0 + first + i - p) * stride);
                }
            }
        }
        bad = kvq_finite(x);
        if (to_tail) {
#pragma unroll
            for (int i = 0; i < kKvqBlock; ++i)
                if (first + i >= p && first + i < end) tail[i * kRow8] = x[i];
        }
        if (wanted) {
            uint32_t w[kKvqBlock];
            const float scale = kvq_encode_block<kFmt>(x, w);
            unsigned char *strip = cache + kvq_tail_bytes(a.Hkv) +
                                   (size_t)kvq_slot(j / 4, compact, a.S, a.W) * kvq_tile_stride(a.Hkv) + kvq_strip_at(head, j);
            kvq_put_block(strip + (j & 1) * kKvqBlockBytes, w, kv, lane);
            if (lane == 0) *reinterpret_cast<float *>(strip + kKvqStripCodes + (j & 1) * 4) = scale;
        }
    }
    if (begun && j == jf && jl > jf) {
        __syncwarp();
        const int first = jl * kKvqBlock;
        const unsigned char *row = src + (int64_t)(r0 + first - p) * stride;
        uint2 y[kKvqBlock];
#pragma unroll
        for (int i = 0; i < kKvqBlock; ++i, row += stride) y[i] = first + i < end ? *reinterpret_cast<const uint2 *>(row) : make_uint2(0u, 0u);
#pragma unroll
        for (int i = 0; i < kKvqBlock; ++i)
            if (first + i < end) tail[i * kRow8] = make_uint2(kvq_finite2(y[i].x, bad), kvq_finite2(y[i].y, bad));
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(a.status, FLUX_STATUS_NONFINITE);
}

template <int kFmt>
__global__ void __launch_bounds__(kWarps * 32, kCtasPerSm) kvq_store_kernel(KvqArgs a)
{
    extern __shared__ __align__(8) unsigned char sh[];
    const Requests s(sh, a.B);
    begin_launch();
    stage_requests(a, s);
    const int lane = threadIdx.x & 31;
    for (uint32_t task = blockIdx.x * kWarps + (threadIdx.x >> 5); task < a.tasks; task += gridDim.x * kWarps)
        store_task<kFmt>(a, s, task, lane);
}

template <int kFmt>
__device__ __forceinline__ void load_task(const KvqArgs &a, const Requests &s, uint32_t task, int lane)
{
    const int slot = (int)(task / (2u * a.Hkv)), rem = (int)(task % (2u * a.Hkv));
    const int kv = rem >= a.Hkv ? 1 : 0, head = rem - kv * a.Hkv;
    const int b = find_request(s.row_start, a.B, slot, lane);
    if (s.kind[b] == 0) return;
    const int r0 = s.row_start[b], n = s.row_start[b + 1] - r0, p = s.pos[b], ctx = s.ctx[b];
    const int jf = p / kKvqBlock, j = jf + slot - (r0 / kKvqBlock + 2 * b), first = j * kKvqBlock;
    if (j < jf || first >= p + n) return;
    const bool compact = s.kind[b] == 2;
    const unsigned char *cache = s.cache[kv * a.B + b];
    uint2 x[kKvqBlock];
    if (first + kKvqBlock <= ctx) {
        if (kvq_held(j, ctx, compact, a.S, a.W)) {
            const unsigned char *strip = cache + kvq_tail_bytes(a.Hkv) +
                                         (size_t)kvq_slot(j / 4, compact, a.S, a.W) * kvq_tile_stride(a.Hkv) + kvq_strip_at(head, j);
            const unsigned char *blk = strip + (j & 1) * kKvqBlockBytes;
            const float scale = *reinterpret_cast<const float *>(strip + kKvqStripCodes + (j & 1) * 4);
            uint32_t w[kKvqBlock];
            if (kv == 0) {
#pragma unroll
                for (int i = 0; i < kKvqBlock; ++i)
                    w[i] = *reinterpret_cast<const uint32_t *>(blk + ((2 * (lane >> 4) + (i >> 3)) * 8 + (i & 7)) * 64 + (lane & 15) * 4);
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const uint4 c = *reinterpret_cast<const uint4 *>(blk + lane * 64 + t * 16);
                    const uint4 y = transpose4(c.x, c.y, c.z, c.w);
                    w[2 * t] = y.x;
                    w[2 * t + 1] = y.y;
                    w[2 * t + 8] = y.z;
                    w[2 * t + 9] = y.w;
                }
            }
#pragma unroll
            for (int i = 0; i < kKvqBlock; ++i) x[i] = kvq_values4<kFmt>(w[i], scale);
        } else {
#pragma unroll
            for (int i = 0; i < kKvqBlock; ++i) x[i] = make_uint2(0u, 0u);
        }
    } else {
        const uint2 *tail = reinterpret_cast<const uint2 *>(cache + (size_t)head * kKvqTailHeadBytes) + lane;
#pragma unroll
        for (int i = 0; i < kKvqBlock; ++i) x[i] = first + i < ctx ? tail[i * (kRowBytes / 8)] : make_uint2(0u, 0u);
    }
    const size_t row = (size_t)a.Hkv * kRowBytes;
    unsigned char *dst = (unsigned char *)a.dst[kv] + (int64_t)(r0 + first - p) * (int64_t)row + (size_t)head * kRowBytes + (size_t)lane * 8;
    if (first >= p && first + kKvqBlock <= p + n) {
#pragma unroll
        for (int i = 0; i < kKvqBlock; ++i, dst += row) *reinterpret_cast<uint2 *>(dst) = x[i];
    } else {
#pragma unroll
        for (int i = 0; i < kKvqBlock; ++i, dst += row)
            if (first + i >= p && first + i < p + n) *reinterpret_cast<uint2 *>(dst) = x[i];
    }
}

template <int kFmt>
__global__ void __launch_bounds__(kWarps * 32, kCtasPerSm) kvq_load_kernel(KvqArgs a)
{
    extern __shared__ __align__(8) unsigned char sh[];
    const Requests s(sh, a.B);
    begin_launch();
    stage_requests(a, s);
    const int lane = threadIdx.x & 31;
    for (uint32_t task = blockIdx.x * kWarps + (threadIdx.x >> 5); task < a.tasks; task += gridDim.x * kWarps)
        load_task<kFmt>(a, s, task, lane);
}

}  // namespace

size_t kvq_cache_size(const flux_config &c, bool compact, int max_len)
{
    int64_t tiles = ((int64_t)max_len + kKvqTile - 1) / kKvqTile;
    const int64_t ring = (int64_t)kvq_sink_tiles(c.sink) + kvq_ring_tiles(c.window);
    if (compact && ring < tiles) tiles = ring;      // a request that never outgrows sink and window fills its tiles in order
    return kvq_tail_bytes(c.n_kv_heads) + (size_t)tiles * kvq_tile_stride(c.n_kv_heads);
}

int launch_kvq_move(flux_plan *p, int layer, int B, int fmt, const void *k, const void *v, int64_t k_stride, int64_t v_stride,
                    void *k_out, void *v_out, const int32_t *row_start, const int32_t *pos, const int32_t *ctx_len, int total_rows,
                    void *const *k_caches, void *const *v_caches, cudaStream_t st)
{
    const flux_config &c = p->cfg;
    KvqArgs a;
    a.src[0] = k; a.src[1] = v;
    a.dst[0] = k_out; a.dst[1] = v_out;
    a.stride[0] = k_stride * 2; a.stride[1] = v_stride * 2;
    a.caches[0] = k_caches; a.caches[1] = v_caches;
    a.row_start = row_start; a.pos = pos; a.ctx_len = ctx_len;
    a.mask = p->d_mask;
    a.B = B; a.L = c.n_layers; a.layer = layer; a.Hkv = c.n_kv_heads; a.S = c.sink; a.W = c.window;
    a.layout = c.kv_layout; a.max_context = c.max_context; a.total_rows = total_rows;
    a.status = (uint32_t *)((char *)p->ws + p->lay.status);
    const int64_t tasks = ((int64_t)total_rows / kKvqBlock + 2 * (int64_t)B) * 2 * c.n_kv_heads;
    if (tasks >= (1ll << 31)) return fail(FLUX_E_CAPACITY, "too many rows for one call");
    a.tasks = (uint32_t)tasks;
    const int64_t ctas = (tasks + kWarps - 1) / kWarps, most = (int64_t)kCtasPerSm * p->dev.n_sms;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)(ctas < most ? ctas : most));
    lc.blockDim = dim3(kWarps * 32);
    lc.dynamicSmemBytes = (size_t)B * 2 * sizeof(void *) + (size_t)(4 * B + 1) * sizeof(int);
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    const bool e4m3 = fmt == FLUX_KVQ_E4M3, load = k_out != nullptr;
    void (*fn)(KvqArgs) = load ? (e4m3 ? kvq_load_kernel<FLUX_KVQ_E4M3> : kvq_load_kernel<FLUX_KVQ_INT8>)
                               : (e4m3 ? kvq_store_kernel<FLUX_KVQ_E4M3> : kvq_store_kernel<FLUX_KVQ_INT8>);
    p->launches++;
    return check_cuda(cudaLaunchKernelEx(&lc, fn, a), load ? "kvq load kernel launch" : "kvq store kernel launch");
}

}  // namespace flux
