// Norm and rotation of query and key heads, rows to rows or into the pages of a cache, and pages back into rows.
//
// One pass over the data: a row's heads are read once and written once (bound by memory, 512 bytes a head); eight lanes share a head
// (flux_rope.h).  Two kernels: with few rows a warp takes four heads of one, which is all latency; with many it takes whole rows, finds
// their sines once for all heads, and has the next eight heads on their way while it works.
//
// Measured (32/8 heads): 32K rows into pages 129 us = 6.2 TB/s, 0.97 of the copy bandwidth; 24K rows to rows, whose fewer bytes a row leave
// less time for the same sines and norms, 87.6 us = 5.7 TB/s (issue slots 63 % used, 2400 instructions a row); a decode step's 32 rows 2.9
// us, which is the launch, one trip to memory for the row and its table entry, and the sines.
#include "flux_paged.h"
#include "flux_rope.h"

namespace flux {
namespace {

constexpr int kWarps = 8;
constexpr int kCtasPerSm = 2;
constexpr int kHeads = 32 / kHeadLanes;      // heads a warp takes at a time
constexpr int kRound = 2;            // so many of these make a slot of the ring
constexpr int kRing = 2;             // slots of a warp: with three or four the memory is no busier and serves rows less in order (132 and 134 us
                                     // for 32K rows into pages, with two 130)
constexpr int kSlotBytes = kRound * 2 * 32 * 16;

struct MoveArgs {
    RopeArgs rope;
    int turn;                        // 0: no rope, rows as they are
    const unsigned char *src[3];     // q, k, v rows, NULL: none
    int64_t src_stride[3];           // bytes
    unsigned char *dst[2];           // q, k rows out, NULL: none
    int64_t dst_stride[2];
    int heads[3];
    const int32_t *at;               // positions of the rows (rows to rows), else NULL and
    PageArgs pages;
    const int32_t *row_start, *pos;  // [B + 1], [B]
    int B, max_context, total_rows;
    uint32_t *status;
};

__device__ __forceinline__ void begin_launch()
{
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
}

// Bounds of the requests in shared memory: row_start, position of the first row, and whether its checks hold.
struct Requests {
    int *row_start, *pos, *ok;       // [B + 1], [B], [B]
    __device__ __forceinline__ Requests(int *sh, int B) : row_start(sh), pos(sh + B + 1), ok(sh + 2 * B + 1) {}
    // the request that row `r` belongs to, or -1
    __device__ __forceinline__ int of_row(int B, int r, int lane) const
    {
        int lo = 0, hi = B;          // row_start[lo] <= r, but for the first
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) >> 5, i = lo + lane * step;
            const int c = __popc(__ballot_sync(0xffffffffu, i < hi && row_start[i] <= r));
            lo += (c > 0 ? c - 1 : 0) * step;
            hi = min(hi, lo + step);
        }
        return row_start[lo] <= r && r < row_start[lo + 1] && ok[lo] ? lo : -1;
    }
};

__device__ __forceinline__ void stage_requests(const Requests &s, const int32_t *row_start, const int32_t *pos, const int32_t *ctx_len, int B,
                                               int total_rows, int64_t most, uint32_t *status)
{
    for (int b = threadIdx.x; b < B; b += blockDim.x) {
        const int r0 = row_start[b], r1 = row_start[b + 1], p = pos[b];
        const int64_t end = ctx_len != nullptr ? min((int64_t)ctx_len[b], most) : most;
        bool fits = r0 >= 0 && r1 >= r0 && r1 <= total_rows;
        if (fits && r1 > r0) fits = p >= 0 && (int64_t)p + (r1 - r0) <= end && (ctx_len == nullptr || ctx_len[b] <= most);
        if (!fits && blockIdx.x == 0) atomicOr(status, FLUX_STATUS_BAD_LENGTH);
        s.row_start[b] = r0;
        if (b == B - 1) s.row_start[B] = r1;
        s.pos[b] = p;
        s.ok[b] = fits;
    }
    __syncthreads();
}

__device__ __forceinline__ void stage_store(const MoveArgs &a, const Requests &s)
{
    if (a.at == nullptr)
        stage_requests(s, a.row_start, a.pos, nullptr, a.B, a.total_rows, min(a.pages.room(), (int64_t)a.max_context), a.status);
}

// Where a row goes.
struct Target {
    int p, entry;                    // position, table entry of its page
    bool live;                       // it belongs to a request, or rows go to rows
    __device__ __forceinline__ void find(const MoveArgs &a, const Requests &s, int row, int lane)
    {
        entry = FLUX_PAGE_NONE;
        live = row < a.total_rows;
        if (!live) return;
        if (a.at != nullptr) {
            p = a.at[row];
            return;
        }
        const int b = s.of_row(a.B, row, lane);
        live = b >= 0;
        if (!live) return;
        p = s.pos[b] + row - s.row_start[b];
        entry = a.pages.entry(b, p);
    }
    __device__ __forceinline__ unsigned char *page(const MoveArgs &a, int kv, int lane) const
    {
        if (entry >= 0 && entry < a.pages.n_pages) return (kv ? a.pages.pool[1] : a.pages.pool[0]) + a.pages.row(entry, p) * a.heads[1] * kRowBytes;
        if (entry != FLUX_PAGE_NONE && lane == 0) atomicOr(a.status, FLUX_STATUS_BAD_PAGE);
        return nullptr;
    }
};

// Few rows: a warp takes four heads.
template <bool kNeighbours>
__global__ void __launch_bounds__(kWarps * 32, kCtasPerSm) rope_few_kernel(MoveArgs a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    const Requests s(reinterpret_cast<int *>(smem), a.B);
    const int lane = threadIdx.x & 31;
    begin_launch();
    stage_store(a, s);
    RopeLane l;
    l.place(a.rope, lane);
    RopeFreqs freqs = {};
    if (a.turn) freqs.read(a.rope, lane);
    // fours of the three kinds
    const int u0 = a.src[0] != nullptr ? (a.heads[0] + kHeads - 1) / kHeads : 0, u1 = a.src[1] != nullptr ? (a.heads[1] + kHeads - 1) / kHeads : 0;
    const int units = u0 + u1 + (a.src[2] != nullptr ? (a.heads[2] + kHeads - 1) / kHeads : 0);
    for (int64_t task = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); task < (int64_t)a.total_rows * units; task += (int64_t)gridDim.x * kWarps) {
        const int row = (int)(task / units), u = (int)(task - (int64_t)row * units), kind = u < u0 ? 0 : u < u0 + u1 ? 1 : 2;
        const int h = kHeads * (u - (kind > 0 ? u0 : 0) - (kind > 1 ? u1 : 0)) + lane / kHeadLanes;
        const bool live = h < a.heads[kind];
        const __nv_bfloat16 *weight = kind == 0 ? a.rope.weight[0] : kind == 1 ? a.rope.weight[1] : nullptr;
        Pieces x = {};
        if (live) x = l.load(a.src[kind] + row * a.src_stride[kind] + h * kRowBytes);
        const Pieces weights = rope_weights(weight, l);      // (everything is asked for before anything is waited for)
        Target to;
        to.find(a, s, row, lane);
        if (!to.live) continue;
        RopeFactors f;
        if (kind < 2 && a.turn) {
            l.sines(a.rope, freqs, lane, to.p);
            f.fold(a.rope, l, weight != nullptr, weights);
        }
        if (kind < 2 && a.turn) x = to_pieces(f.turn(x, kNeighbours, weight != nullptr, a.rope.eps), kNeighbours);
        unsigned char *page = kind > 0 ? to.page(a, kind - 1, lane) : nullptr, *out = kind == 0 ? a.dst[0] : kind == 1 ? a.dst[1] : nullptr;
        if (live && out != nullptr) l.store(out + row * (kind == 0 ? a.dst_stride[0] : a.dst_stride[1]) + h * kRowBytes, x);
        if (live && page != nullptr) l.store(page + h * kRowBytes, x);
    }
}

// Many rows: a warp takes whole ones.  Every lane has a ring of its own pieces in shared memory, filled by asynchronous copies well ahead:
// what it copies it alone reads, so there is nothing to wait for but its own copies.
template <bool kNeighbours>
__global__ void __launch_bounds__(kWarps * 32, kCtasPerSm) rope_rows_kernel(MoveArgs a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    const Requests s(reinterpret_cast<int *>(smem + kWarps * kRing * kSlotBytes), a.B);
    const int lane = threadIdx.x & 31;
    begin_launch();
    stage_store(a, s);
    RopeLane l;
    l.place(a.rope, lane);
    const int n[3] = {a.src[0] != nullptr ? a.heads[0] : 0, a.src[1] != nullptr ? a.heads[1] : 0, a.src[2] != nullptr ? a.heads[2] : 0};
    const int first = blockIdx.x * kWarps + (threadIdx.x >> 5), step = gridDim.x * kWarps;
    unsigned char *ring = smem + (threadIdx.x >> 5) * kRing * kSlotBytes + lane * 16;
    const uint32_t ring_u32 = smem_u32(ring);

    struct Cursor {                  // eight heads (kHeads * kRound) of a kind of a row
        int kind, h;
        int64_t row;
    };
    auto next = [&](Cursor &c) {
        c.h += kHeads * kRound;
        while (c.h >= (c.kind == 0 ? n[0] : c.kind == 1 ? n[1] : n[2])) {
            c.h = 0;
            if (++c.kind == 3) {
                c.kind = 0;
                c.row += step;
            }
        }
    };
    Cursor cur = {0, -kHeads * kRound, first};
    next(cur);
    Cursor ld = cur;
    auto ask = [&](int slot) {
        if (ld.row < a.total_rows) {
            const unsigned char *src = ld.kind == 0 ? a.src[0] + ld.row * a.src_stride[0] : ld.kind == 1 ? a.src[1] + ld.row * a.src_stride[1]
                                                                                                        : a.src[2] + ld.row * a.src_stride[2];
            const int end = ld.kind == 0 ? n[0] : ld.kind == 1 ? n[1] : n[2], h = ld.h + lane / kHeadLanes;
#pragma unroll
            for (int i = 0; i < kRound; ++i) {
                const int m = h + kHeads * i;
                if (m < end) {
                    cp_async16(ring_u32 + slot * kSlotBytes + (2 * i) * 512, src + m * kRowBytes + l.a * 2, 16);
                    cp_async16(ring_u32 + slot * kSlotBytes + (2 * i + 1) * 512, src + m * kRowBytes + l.b * 2, 16);
                }
            }
            next(ld);
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) ask(i);
    Target to, after;                // of this row and the warp's next: its table entry is asked for a row ahead
    after.find(a, s, first, lane);
    int64_t at = -1;
    int slot = 0, folded = -1;
    unsigned char *pages[2] = {nullptr, nullptr};
    RopeFactors f;
    while (cur.row < a.total_rows) {
        if (cur.row != at) {
            at = cur.row;
            to = after;
            if (to.live) {
                pages[0] = to.page(a, 0, lane);
                pages[1] = to.page(a, 1, lane);
            }
            after.find(a, s, (int)min(at + step, (int64_t)a.total_rows), lane);
            folded = -1;
            if (to.live && a.turn) {         // frequencies and weights come from the L1: held across rows they cost registers, and 1.5 us of 90
                RopeFreqs freqs;
                freqs.read(a.rope, lane);
                l.sines(a.rope, freqs, lane, to.p);
            }
        }
        ask(slot == 0 ? kRing - 1 : slot - 1);       // the slot used last
        cp_async_wait<kRing - 1>();
        if (to.live) {
            const int end = cur.kind == 0 ? n[0] : cur.kind == 1 ? n[1] : n[2], h = cur.h + lane / kHeadLanes;
            if (cur.kind < 2 && a.turn && folded != cur.kind) {
                const __nv_bfloat16 *weight = cur.kind == 0 ? a.rope.weight[0] : a.rope.weight[1];
                f.fold(a.rope, l, weight != nullptr, rope_weights(weight, l));
                folded = cur.kind;
            }
            Pieces x[kRound];
#pragma unroll
            for (int i = 0; i < kRound; ++i)
                x[i] = {*reinterpret_cast<const uint4 *>(ring + slot * kSlotBytes + (2 * i) * 512),
                        *reinterpret_cast<const uint4 *>(ring + slot * kSlotBytes + (2 * i + 1) * 512)};
            if (cur.kind < 2 && a.turn) {                // (heads behind the last one: whatever the slot holds, and not stored)
                const bool norm = (cur.kind == 0 ? a.rope.weight[0] : a.rope.weight[1]) != nullptr;
#pragma unroll
                for (int i = 0; i < kRound; ++i) x[i] = to_pieces(f.turn(x[i], kNeighbours, norm, a.rope.eps), kNeighbours);
            }
            unsigned char *page = cur.kind == 0 ? nullptr : cur.kind == 1 ? pages[0] : pages[1];
            unsigned char *out = cur.kind == 0 ? a.dst[0] : cur.kind == 1 ? a.dst[1] : nullptr;
            if (out != nullptr) {
                out += cur.row * (cur.kind == 0 ? a.dst_stride[0] : a.dst_stride[1]) + h * kRowBytes;
#pragma unroll
                for (int i = 0; i < kRound; ++i)
                    if (h + kHeads * i < end) l.store(out + kHeads * i * kRowBytes, x[i]);
            }
            if (page != nullptr) {
                page += h * kRowBytes;
#pragma unroll
                for (int i = 0; i < kRound; ++i)
                    if (h + kHeads * i < end) l.store(page + kHeads * i * kRowBytes, x[i]);
            }
        }
        slot = slot + 1 == kRing ? 0 : slot + 1;
        next(cur);
    }
    cp_async_wait<0>();
}

struct LoadArgs {
    PageArgs pages;
    unsigned char *dst[2];
    const int32_t *row_start, *pos, *ctx_len;
    int B, Hkv, max_context, total_rows;
    uint32_t *status;
};

// Pages into rows: a warp per row and pool.
__global__ void __launch_bounds__(kWarps * 32) paged_load_kernel(LoadArgs a)
{
    extern __shared__ int sh[];
    const Requests s(sh, a.B);
    const int lane = threadIdx.x & 31;
    begin_launch();
    stage_requests(s, a.row_start, a.pos, a.ctx_len, a.B, a.total_rows, min(a.pages.room(), (int64_t)a.max_context), a.status);
    const int pieces = a.Hkv * (kRowBytes / 16);
    for (int64_t task = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); task < 2 * (int64_t)a.total_rows; task += (int64_t)gridDim.x * kWarps) {
        const int row = (int)(task >> 1), kv = (int)(task & 1);
        const int b = s.of_row(a.B, row, lane);
        if (b < 0) continue;
        const int p = s.pos[b] + row - s.row_start[b], page = a.pages.entry(b, p);
        const bool held = page >= 0 && page < a.pages.n_pages;
        if (!held && page != FLUX_PAGE_NONE && lane == 0) atomicOr(a.status, FLUX_STATUS_BAD_PAGE);
        const uint4 *src = reinterpret_cast<const uint4 *>(kv ? a.pages.pool[1] : a.pages.pool[0]) + (held ? a.pages.row(page, p) * pieces : 0);
        uint4 *dst = reinterpret_cast<uint4 *>(kv ? a.dst[1] : a.dst[0]) + (size_t)row * pieces;
        for (int i = lane; i < pieces; i += 4 * 32) {
            uint4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[k] = make_uint4(0u, 0u, 0u, 0u);
                if (held && i + 32 * k < pieces) x[k] = src[i + 32 * k];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + 32 * k < pieces) dst[i + 32 * k] = x[k];
        }
    }
}

template <class Args>
int launch(void (*fn)(Args), const Args &a, int64_t warps, size_t smem, flux_plan *p, int per_sm, cudaStream_t st, const char *what)
{
    const int64_t ctas = (warps + kWarps - 1) / kWarps, most = (int64_t)per_sm * p->dev.n_sms;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)(ctas < most ? ctas : most));
    lc.blockDim = dim3(kWarps * 32);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    p->launches++;
    return check_cuda(cudaLaunchKernelEx(&lc, fn, a), what);
}

constexpr size_t kRowsSmem = (size_t)kWarps * kRing * kSlotBytes;
size_t requests_bytes(int B) { return (size_t)(3 * B + 1) * sizeof(int); }

}  // namespace

RopeArgs rope_args(const flux_rope *r)
{
    RopeArgs a = {};
    a.scale = 1.f;
    if (r == nullptr) return a;
    a.weight[0] = (const __nv_bfloat16 *)r->q_weight;
    a.weight[1] = (const __nv_bfloat16 *)r->k_weight;
    a.freqs = r->freqs;
    a.eps = r->eps;
    a.offset = r->weight_offset;
    a.scale = r->scale;
    a.rot = r->rotary_dim;
    a.pairs = r->interleaved;
    return a;
}

int rope_setup(flux_plan *p)
{
    const size_t most = kRowsSmem + requests_bytes(kMaxBatch);
    if ((size_t)p->dev.smem_optin < most) return fail(FLUX_E_CUDA, "device offers %d bytes of shared memory per block, the norm and rotation kernel needs %zu", p->dev.smem_optin, most);
    int rc = check_cuda(cudaFuncSetAttribute(rope_rows_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most), "cudaFuncSetAttribute(rope_rows_kernel)");
    if (!rc) rc = check_cuda(cudaFuncSetAttribute(rope_rows_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most), "cudaFuncSetAttribute(rope_rows_kernel)");
    return rc;
}

int launch_rope_move(flux_plan *p, int B, const flux_rope *rope, const void *q, const void *k, const void *v, int64_t q_stride, int64_t k_stride,
                     int64_t v_stride, int total_rows, const int32_t *at, const int32_t *row_start, const int32_t *pos, const flux_pages *pages,
                     void *q_out, void *k_out, int64_t q_out_stride, int64_t k_out_stride, cudaStream_t st)
{
    const flux_config &c = p->cfg;
    MoveArgs a = {};
    a.rope = rope_args(rope);
    a.turn = rope != nullptr;
    a.src[0] = (const unsigned char *)q; a.src[1] = (const unsigned char *)k; a.src[2] = (const unsigned char *)v;
    a.src_stride[0] = q_stride * 2; a.src_stride[1] = k_stride * 2; a.src_stride[2] = v_stride * 2;
    a.dst[0] = (unsigned char *)q_out; a.dst[1] = (unsigned char *)k_out;
    a.dst_stride[0] = q_out_stride * 2; a.dst_stride[1] = k_out_stride * 2;
    a.heads[0] = c.n_q_heads; a.heads[1] = a.heads[2] = c.n_kv_heads;
    a.at = at;
    if (pages != nullptr) a.pages = page_args(*pages);
    a.row_start = row_start; a.pos = pos;
    a.B = pages != nullptr ? B : 0;
    a.max_context = c.max_context;
    a.total_rows = total_rows;
    a.status = (uint32_t *)((char *)p->ws + p->lay.status);
    // Up to three fours of heads for every warp that fits: those.  More: whole rows, whose sines are then found once.  (Into pages, us, fours /
    // whole rows: 32/8 heads, 512 rows 7.3 / 8.9, 1024 rows 11.1 / 8.9, 16384 rows 143 / 67; 8/2 heads, 1024 rows 5.7 / 5.8, 2048 rows 8.6 / 6.8.)
    const bool pairs = rope != nullptr && rope->interleaved;
    const int64_t places = (int64_t)kCtasPerSm * kWarps * p->dev.n_sms;
    const int units = (q != nullptr ? (a.heads[0] + kHeads - 1) / kHeads : 0) + (k != nullptr ? (a.heads[1] + kHeads - 1) / kHeads : 0) +
                      (v != nullptr ? (a.heads[2] + kHeads - 1) / kHeads : 0);
    if ((int64_t)total_rows * units > 3 * places)
        return launch(pairs ? rope_rows_kernel<true> : rope_rows_kernel<false>, a, total_rows, kRowsSmem + requests_bytes(a.B), p, kCtasPerSm, st,
                      "norm and rotation kernel launch");
    return launch(pairs ? rope_few_kernel<true> : rope_few_kernel<false>, a, (int64_t)total_rows * units, requests_bytes(a.B), p, kCtasPerSm, st,
                  "norm and rotation kernel launch");
}

int launch_paged_load(flux_plan *p, int B, const flux_pages &pages, const int32_t *ctx_len, int total_rows, const int32_t *row_start,
                      const int32_t *pos, void *k_out, void *v_out, cudaStream_t st)
{
    LoadArgs a;
    a.pages = page_args(pages);
    a.dst[0] = (unsigned char *)k_out; a.dst[1] = (unsigned char *)v_out;
    a.row_start = row_start; a.pos = pos; a.ctx_len = ctx_len;
    a.B = B; a.Hkv = p->cfg.n_kv_heads; a.max_context = p->cfg.max_context; a.total_rows = total_rows;
    a.status = (uint32_t *)((char *)p->ws + p->lay.status);
    return launch(paged_load_kernel, a, 2 * (int64_t)total_rows, requests_bytes(B), p, 6, st, "paged load kernel launch");
}

}  // namespace flux
