// Norm and rotation of query and key heads, rows to rows or into the pages of a cache, and pages back into rows.
//
// One pass over the data: a row's heads are read once and written once (bound by memory, 512 bytes a head).  A warp takes a row, or
// a part of its heads where there are few rows; its two half-warps take a head each (flux_rope.h), eight heads a round so that
// enough loads are on their way.  The sines of a row are found once for all its heads.
#include "flux_paged.h"
#include "flux_rope.h"

namespace flux {
namespace {

constexpr int kWarps = 8;
constexpr int kCtasPerSm = 3;
constexpr int kRound = 4;            // heads of a half-warp on their way at a time

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
    int B, max_context, total_rows, parts;
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

// Heads [h0, h1) of one kind, of one row: lanes 0-15 take the even ones of h0 .., lanes 16-31 the odd ones.
template <bool kTurn>
__device__ __forceinline__ void move_heads(const unsigned char *src, unsigned char *out, unsigned char *page, int h0, int h1, const RopeLane &l,
                                           const RopeFactors &f, int pairs, bool norm, float eps, int lane)
{
    for (int h = h0 + (lane >> 4); h - (lane >> 4) < h1; h += 2 * kRound) {
        uint2 pa[kRound], pb[kRound];
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            pa[i] = pb[i] = make_uint2(0u, 0u);
            if (h + 2 * i < h1) {
                pa[i] = *reinterpret_cast<const uint2 *>(src + (h + 2 * i) * kRowBytes + l.a * 2);
                pb[i] = *reinterpret_cast<const uint2 *>(src + (h + 2 * i) * kRowBytes + l.b * 2);
            }
        }
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            if (kTurn) f.apply(pa[i], pb[i], pairs, norm, eps);
            if (h + 2 * i < h1) {
                if (out != nullptr) {
                    *reinterpret_cast<uint2 *>(out + (h + 2 * i) * kRowBytes + l.a * 2) = pa[i];
                    *reinterpret_cast<uint2 *>(out + (h + 2 * i) * kRowBytes + l.b * 2) = pb[i];
                }
                if (page != nullptr) {
                    *reinterpret_cast<uint2 *>(page + (h + 2 * i) * kRowBytes + l.a * 2) = pa[i];
                    *reinterpret_cast<uint2 *>(page + (h + 2 * i) * kRowBytes + l.b * 2) = pb[i];
                }
            }
        }
    }
}

__global__ void __launch_bounds__(kWarps * 32, kCtasPerSm) rope_move_kernel(MoveArgs a)
{
    extern __shared__ int sh[];
    const Requests s(sh, a.B);
    const int lane = threadIdx.x & 31;
    begin_launch();
    if (a.at == nullptr)
        stage_requests(s, a.row_start, a.pos, nullptr, a.B, a.total_rows, min(a.pages.room(), (int64_t)a.max_context), a.status);
    // the heads of all kinds side by side; a part takes an equal share of them, in pairs
    const int n0 = a.src[0] != nullptr ? a.heads[0] : 0, n1 = a.src[1] != nullptr ? a.heads[1] : 0, n2 = a.src[2] != nullptr ? a.heads[2] : 0;
    const int units = (n0 + n1 + n2 + 1) / 2;
    RopeLane l;
    l.place(a.rope, lane);
    for (int64_t task = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); task < (int64_t)a.total_rows * a.parts; task += (int64_t)gridDim.x * kWarps) {
        const int row = (int)(task / a.parts), part = (int)(task - (int64_t)row * a.parts);
        const int u0 = 2 * (int)((int64_t)units * part / a.parts), u1 = min(2 * (int)((int64_t)units * (part + 1) / a.parts), n0 + n1 + n2);
        int p;
        unsigned char *kd = nullptr, *vd = nullptr;
        if (a.at != nullptr) {
            p = a.at[row];
        } else {
            const int b = s.of_row(a.B, row, lane);
            if (b < 0) continue;
            p = s.pos[b] + row - s.row_start[b];
            const int page = a.pages.entry(b, p);
            if (page >= 0 && page < a.pages.n_pages) {
                const size_t at = a.pages.row(page, p) * a.heads[1] * kRowBytes;
                kd = a.pages.pool[0] + at;
                vd = a.pages.pool[1] + at;
            } else if (page != FLUX_PAGE_NONE && lane == 0) {
                atomicOr(a.status, FLUX_STATUS_BAD_PAGE);
            }
        }
        if (a.turn) l.turn(a.rope, lane, p);
        if (u0 < n0) {
            RopeFactors f;
            f.fold(a.rope, l, 0);
            move_heads<true>(a.src[0] + (int64_t)row * a.src_stride[0], a.dst[0] + (int64_t)row * a.dst_stride[0], nullptr, u0, min(u1, n0), l, f,
                             a.rope.pairs, a.rope.weight[0] != nullptr, a.rope.eps, lane);
        }
        const int k0 = max(u0 - n0, 0), k1 = min(u1 - n0, n1), v0 = max(u0 - n0 - n1, 0), v1 = min(u1 - n0 - n1, n2);
        if (k0 < k1) {
            const unsigned char *src = a.src[1] + (int64_t)row * a.src_stride[1];
            unsigned char *out = a.dst[1] != nullptr ? a.dst[1] + (int64_t)row * a.dst_stride[1] : nullptr;
            RopeFactors f;
            if (a.turn) {
                f.fold(a.rope, l, 1);
                move_heads<true>(src, out, kd, k0, k1, l, f, a.rope.pairs, a.rope.weight[1] != nullptr, a.rope.eps, lane);
            } else {
                move_heads<false>(src, out, kd, k0, k1, l, f, 0, false, 0.f, lane);
            }
        }
        if (v0 < v1 && vd != nullptr) {
            const RopeFactors f = {};
            move_heads<false>(a.src[2] + (int64_t)row * a.src_stride[2], nullptr, vd, v0, v1, l, f, 0, false, 0.f, lane);
        }
    }
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
    // Few rows: their heads are dealt to several warps, down to two heads each, until the GPU has a warp in every place.
    const int units = ((q != nullptr ? a.heads[0] : 0) + (k != nullptr ? a.heads[1] : 0) + (v != nullptr ? a.heads[2] : 0) + 1) / 2;
    const int64_t places = (int64_t)kCtasPerSm * kWarps * p->dev.n_sms;
    const int64_t parts = (places + total_rows - 1) / total_rows;
    a.parts = (int)(parts < units ? parts : units);
    return launch(rope_move_kernel, a, (int64_t)total_rows * a.parts, requests_bytes(a.B), p, kCtasPerSm, st, "norm and rotation kernel launch");
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
