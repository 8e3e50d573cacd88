// Norm and rotation of query and key heads, rows to rows or into the pages of a cache, and pages back into rows.
//
// One pass over the data: a row's heads are read once and written once (bound by memory, 512 bytes a head); eight lanes share a head
// (flux_rope.h).  Two kernels: with few rows a warp takes four heads of one, which is all latency; with many it takes whole rows, finds
// their sines once for all heads, and has the next eight heads on their way while it works.
//
// Measured (32/8 heads): 32K rows into pages 131 to 133 us = 6.1 TB/s, 0.94 of the copy bandwidth; 24K rows to rows 83 us = 6.1 TB/s, 0.94; a
// decode step's 32 rows 2.9 us, which is the launch, one trip to memory for the row and its table entry, and the sines.  Pairs of
// neighbours: 186 and 118 us, since a lane's two pieces are half a sector each.  Pages into rows: 32K rows 49 us = 5.5 TB/s, 0.85.
#include "flux_paged.h"
#include "flux_rope.h"

namespace flux {
namespace {

constexpr int kWarps = 8;
constexpr int kCtasPerSm = 2;
constexpr int kHeads = 32 / kHeadLanes;      // heads a warp takes at a time
constexpr int kRound = 2;            // so many of these make a slot of the ring
constexpr int kRing = 2;             // slots of a warp
// Warps of an SM that take whole rows.  More of them, or more slots, ask for more at a time than the memory needs, and it serves reads and
// writes worse: 32K rows into pages / 24K rows to rows in 130 / 82 us with 14 warps, 132 / 85 with 12, 142 / 85 with 15, 144 / 89 with 16;
// slots of four heads instead of eight 147 / 95, of sixteen 138 / 87.
constexpr int kRowWarps = 14;
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
__global__ void __launch_bounds__(kRowWarps * 32, 1) rope_rows_kernel(MoveArgs a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    const Requests s(reinterpret_cast<int *>(smem + kRowWarps * kRing * kSlotBytes), a.B);
    const int lane = threadIdx.x & 31;
    begin_launch();
    stage_store(a, s);
    RopeLane l;
    l.place(a.rope, lane);
    const int n[3] = {a.src[0] != nullptr ? a.heads[0] : 0, a.src[1] != nullptr ? a.heads[1] : 0, a.src[2] != nullptr ? a.heads[2] : 0};
    const int first = blockIdx.x * kRowWarps + (threadIdx.x >> 5), step = gridDim.x * kRowWarps, mine = lane / kHeadLanes;
    const int oa = mine * kRowBytes + l.a * 2, ob = mine * kRowBytes + l.b * 2;      // this lane's pieces of its first head
    unsigned char *ring = smem + (threadIdx.x >> 5) * kRing * kSlotBytes + lane * 16;
    const uint32_t ring_u32 = smem_u32(ring);
    constexpr int kStep = kHeads * kRound;       // heads of a slot, all of one kind of one row
    int fill = 0, slot = 0;                      // slots filled next, used next

    auto ask = [&](int kind, int64_t row, int h) {
        const unsigned char *src = (kind == 0 ? a.src[0] + row * a.src_stride[0] : kind == 1 ? a.src[1] + row * a.src_stride[1]
                                                                                            : a.src[2] + row * a.src_stride[2]) + h * kRowBytes;
        const uint32_t to = ring_u32 + fill * kSlotBytes;
#pragma unroll
        for (int i = 0; i < kRound; ++i)
            if (h + mine + kHeads * i < (kind == 0 ? n[0] : kind == 1 ? n[1] : n[2])) {
                cp_async16(to + (2 * i) * 512, src + oa + kHeads * i * kRowBytes, 16);
                cp_async16(to + (2 * i + 1) * 512, src + ob + kHeads * i * kRowBytes, 16);
            }
        fill = fill + 1 == kRing ? 0 : fill + 1;
    };
    // the first heads of the first kind from `kind` on that there is, of this row or the warp's next
    auto ask_next = [&](int kind, int64_t row) {
        if (kind <= 0 && n[0] > 0) ask(0, row, 0);
        else if (kind <= 1 && n[1] > 0) ask(1, row, 0);
        else if (kind <= 2 && n[2] > 0) ask(2, row, 0);
        else if (row + step < a.total_rows) ask(n[0] > 0 ? 0 : 1, row + step, 0);       // (values never come alone)
    };
    static_assert(kRing == 2, "one slot is filled while the other one is used");
    if (first < a.total_rows) ask_next(0, first);
    cp_async_commit();
    Target to, after;                // of this row and the warp's next: its table entry is asked for a row ahead
    after.find(a, s, first, lane);
    for (int64_t row = first; row < a.total_rows; row += step) {
        to = after;
        unsigned char *pages[2] = {nullptr, nullptr};
        if (to.live) {
            pages[0] = to.page(a, 0, lane);
            pages[1] = to.page(a, 1, lane);
        }
        after.find(a, s, (int)min(row + step, (int64_t)a.total_rows), lane);
        if (to.live && a.turn) {         // frequencies and weights come from the L1: held across rows they cost registers, and 1.5 us of 90
            RopeFreqs freqs;
            freqs.read(a.rope, lane);
            l.sines(a.rope, freqs, lane, to.p);
        }
#pragma unroll
        for (int kind = 0; kind < 3; ++kind) {
            if (n[kind] == 0) continue;
            const __nv_bfloat16 *weight = kind == 0 ? a.rope.weight[0] : kind == 1 ? a.rope.weight[1] : nullptr;
            unsigned char *out = kind < 2 && a.dst[kind < 2 ? kind : 0] != nullptr ? a.dst[kind < 2 ? kind : 0] + row * a.dst_stride[kind < 2 ? kind : 0] : nullptr;
            unsigned char *page = kind == 0 ? nullptr : pages[kind == 1 ? 0 : 1];
            RopeFactors f;
            const bool turn = kind < 2 && a.turn && to.live;
            if (turn) f.fold(a.rope, l, weight != nullptr, rope_weights(weight, l));
            for (int h = 0; h < n[kind]; h += kStep) {
                if (h + kStep < n[kind]) ask(kind, row, h + kStep);
                else ask_next(kind + 1, row);
                cp_async_commit();
                cp_async_wait<kRing - 1>();
                Pieces x[kRound];
#pragma unroll
                for (int i = 0; i < kRound; ++i)
                    x[i] = {*reinterpret_cast<const uint4 *>(ring + slot * kSlotBytes + (2 * i) * 512),
                            *reinterpret_cast<const uint4 *>(ring + slot * kSlotBytes + (2 * i + 1) * 512)};
                slot = slot + 1 == kRing ? 0 : slot + 1;
                if (turn)                // (heads behind the last one: whatever the slot holds, and not stored)
#pragma unroll
                    for (int i = 0; i < kRound; ++i) x[i] = to_pieces(f.turn(x[i], kNeighbours, weight != nullptr, a.rope.eps), kNeighbours);
                if (!to.live) continue;
#pragma unroll
                for (int i = 0; i < kRound; ++i) {
                    if (h + mine + kHeads * i >= n[kind]) break;
                    const int at = (h + kHeads * i) * kRowBytes;
                    if (out != nullptr) {
                        *reinterpret_cast<uint4 *>(out + at + oa) = x[i].a;
                        *reinterpret_cast<uint4 *>(out + at + ob) = x[i].b;
                    }
                    if (page != nullptr) {
                        *reinterpret_cast<uint4 *>(page + at + oa) = x[i].a;
                        *reinterpret_cast<uint4 *>(page + at + ob) = x[i].b;
                    }
                }
            }
        }
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
int launch(void (*fn)(Args), const Args &a, int64_t warps, int cta_warps, size_t smem, flux_plan *p, int per_sm, cudaStream_t st, const char *what)
{
    const int64_t ctas = (warps + cta_warps - 1) / cta_warps, most = (int64_t)per_sm * p->dev.n_sms;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)(ctas < most ? ctas : most));
    lc.blockDim = dim3((unsigned)cta_warps * 32);
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

constexpr size_t kRowsSmem = (size_t)kRowWarps * kRing * kSlotBytes;
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
    // Whole rows once there is one for every other warp of their kernel, so that a warp finds a row's sines once; fewer are dealt out by fours
    // of heads.  (Into pages, us, fours / whole rows: 32/8 heads, 512 rows 6.4 / 8.4, 1024 rows 10.2 / 9.0, 16384 rows 144 / 66; 8/2 heads,
    // 1024 rows 4.9 / 5.4, 1500 rows 6.4 / 5.5.)
    const bool pairs = rope != nullptr && rope->interleaved;
    const int units = (q != nullptr ? (a.heads[0] + kHeads - 1) / kHeads : 0) + (k != nullptr ? (a.heads[1] + kHeads - 1) / kHeads : 0) +
                      (v != nullptr ? (a.heads[2] + kHeads - 1) / kHeads : 0);
    if (2 * (int64_t)total_rows >= (int64_t)kRowWarps * p->dev.n_sms)
        return launch(pairs ? rope_rows_kernel<true> : rope_rows_kernel<false>, a, total_rows, kRowWarps, kRowsSmem + requests_bytes(a.B), p, 1, st,
                      "norm and rotation kernel launch");
    return launch(pairs ? rope_few_kernel<true> : rope_few_kernel<false>, a, (int64_t)total_rows * units, kWarps, requests_bytes(a.B), p, kCtasPerSm, st,
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
    return launch(paged_load_kernel, a, 2 * (int64_t)total_rows, kWarps, requests_bytes(B), p, 6, st, "paged load kernel launch");
}

}  // namespace flux
