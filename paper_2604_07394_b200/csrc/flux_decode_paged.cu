// Decode attention over the paged KV cache (layout: flux_paged.h), one launch per layer; with flux_attn_decode_step_paged the norms, the
// rotation and the storing of the newest token are in the same launch.
//
// o = softmax(scale q K^T) V over the kept positions of every request.  Bound by memory: 256 bytes per kept position and head for each of
// K and V, and a table entry per page.
//
// Work: (request, KV head) segments of tiles of 16 positions, laid end to end and cut into one range per CTA, one CTA per SM, and
// again into one range per warp.  A tile never leaves a page, since a page has a multiple of 16 positions.  A warp walks its range with a
// ring of tiles of its own, brought in by asynchronous 16-byte copies (positions that the request does not keep are not read: zeros), so
// warps meet only once, at the end.  Table entries are read 32 tiles at a time, a lane for each.
//
// Products: mma.m16n8k16 in bf16 with the cache as the A operand -- S^T = K q^T (keys x heads) and O^T = V^T p^T (channels x heads)
// -- so up to 8 query heads fill the N dimension instead of padding M to 16: half the products and half the accumulators of the
// other way round.  Eight MACs per byte: tcgen05 would have nothing to do here.
//
// Softmax: fp32, log2 domain.  The maximum in use is raised when a tile's largest score exceeds it by 2^kRaise, and to that score.
// Weights go into the product with V as two bf16 numbers, the rounded weight and what the rounding leaves over (2^-16 of each), and so
// do query rows that are normed and rotated here: the memory leaves room for the products, and with weights of 8 bits the outputs'
// error against 64 bits was 0.0024 where their own rounding costs 0.0017 (with query rows of 8 bits as well 0.0033).
//
// With launch overlap the schedule and the first tiles -- all but those of the newest two positions, which the launch before may
// write -- run ahead of the grid-dependency wait.
//
// Merge: pieces of segments that a CTA's warps share are added up in shared memory; a segment spread over several CTAs goes on
// through partials in the workspace, and the CTA that finishes last (a ticket per segment) adds them up in the order of the
// CTAs; many of them in two steps, the groups' sums first.  No CTA waits for another.
//
// Measured (graph of back-to-back calls): 8 contexts of 64K, half sparse, 32/8 heads 173 us = 6.6 TB/s; 128K batch 1, 28/4 heads 52 us = 5.2
// TB/s; 64 steps of 100 to 4000 tokens 70 us = 5.7 TB/s.  From clock stamps: the memory is busy from 3 us after the dependency wait
// (lengths 0.9, place of the range 0.7, table entries and first requests 1.3), CTAs end within 2 % of one another, then 1 us to
// merge in the CTA, 1 us for the ticket, and the merge of the last CTA (4 heads of 10 partials 1.5 us, 7 of 37 5 us: 132 KB at what one SM
// gets from the L2).  Launch overlap hides most of the start: 170, 50 and 69 us.  Query rows are asked for ahead of the first tiles, whose
// requests wait for table entries, and a warp has scratch of its own for them, so its ring is refilled at once (64 steps 70 us, was 73).
#include "flux_decode_common.h"
#include "flux_paged.h"
#include "flux_rope.h"

namespace flux {
namespace {

constexpr int kWarps = 8;
constexpr int kTile = 16;                                       // positions of a tile
constexpr int kSlotV = kTile * kRowBytes;                       // slot: K rows | V rows, 16-byte pieces swizzled by the row
constexpr int kSlotBytes = 2 * kSlotV;
// Slots of a warp.  Two tiles of eight warps, 128 KB, are on their way in an SM.  Three (which fit beside pieces and scratch up to four heads, and
// up to eight before a warp had scratch of its own) are slower: all the memory can give is asked for either way (64 KB would do at an idle memory's latency), and with more requests in the queues some SMs get
// a sixth less than others, so CTAs with equal work end 148 to 180 us after the start (8 contexts of 64K: 181 us, with two slots 171).
constexpr int kRing = 2;
constexpr int kRowFloats = kHeadDim;                            // a piece: G rows of O, then G pairs (m, l)
constexpr int kMaxParts = 64;                                   // partials a CTA adds up in one round
// Rows (CTAs x heads) of partials from which on they are added up in two steps, groups of about the square root of the CTAs first.  One 128K
// context: 148 CTAs of 16 heads 33.4 us (in one step 47.5), of 8 24.9 (29.8), of 4 24.2 (26.0), 74 of 8 33.7 (34.9); 37 of 7 are done
// no sooner (53.3, in one 52.1).
constexpr int kManyRows = 384, kMinGroup = 4;
constexpr int kAppendCost = 2;                                  // storing the newest token costs a warp as much as that many tiles
constexpr int kShortSpan = 24;                                  // tiles a CTA's warps walk in about the time a merge across CTAs takes
constexpr float kRaise = 8.f;                                   // weights stay below 2^(kRaise + 1)

// Shared memory: slots | first pieces [kWarps][G rows, G pairs] | scratch of a warp (G <= 8) | flags | piece table | prefix, lengths
struct Smem {
    int piece_bytes, off_piece, off_scratch, off_flags, off_desc, off_table, total;
    __host__ __device__ __forceinline__ Smem(int G, int B)
    {
        piece_bytes = G * (kRowFloats + 2) * (int)sizeof(float);
        piece_bytes = (piece_bytes + 15) / 16 * 16;
        off_piece = kWarps * kRing * kSlotBytes;
        off_scratch = off_piece + kWarps * piece_bytes;
        off_flags = off_scratch + (G <= 8 ? kWarps * G * 2 * kRowBytes : 0);
        off_desc = off_flags + 16;
        off_table = off_desc + 2 * kWarps * (int)sizeof(int) * 2;
        total = off_table + (2 * B + 1) * (int)sizeof(int);
    }
};

struct PagedDecArgs {
    const unsigned char *q;          // rows of request b at q + b q_stride: [Hq][128] bf16
    int64_t q_stride;                // bytes
    PageArgs pages;
    const int32_t *ctx_len;
    const uint8_t *mask;
    int B, L, layer, Hq, Hkv, G, S, W, max_context;
    float scale_log2;
    float *part_o, *part_ml;         // [CTA + segment][G][128], [..][2]
    float *group_o, *group_ml;       // [first CTA + segment + group][G][128], [..][2]
    uint32_t *tickets, *group_tickets;       // [B * Hkv], [first CTA of a group + segment], zero between launches
    int32_t *debug;
    uint32_t *status;
    __nv_bfloat16 *out;
    uint32_t *touch;
    int touch_words;
    const unsigned char *k_new, *v_new;      // rows [Hkv][128] of the newest tokens, which this launch stores, or NULL
    int64_t k_stride, v_stride;
    RopeArgs rope;
    int turn;                        // norm and rotation of q and k_new (with k_new only)
    int overlap;                     // schedule and first tiles before the grid-dependency wait
};

// Tiles of a request of n tokens that a decode step reads: [0, e1) and [b2, b2 + count - e1); the last one holds the newest token.
struct Walk {
    int e1, b2, count;
    __device__ __forceinline__ Walk(int n, bool fa, int S, int W)
    {
        const int tiles = (n + kTile - 1) / kTile;
        if (fa || n <= S + W) {
            e1 = b2 = tiles;
        } else {
            e1 = min((S + kTile - 1) / kTile, tiles);
            b2 = max(e1, (n - W) / kTile);
        }
        count = e1 + max(0, tiles - b2);
    }
    __device__ __forceinline__ int tile(int t) const { return t < e1 ? t : b2 + t - e1; }
};

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
    return y;
}
// 16 bytes, all of them
__device__ __forceinline__ void cp_async16_whole(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cta_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// 2^(m - top) where a maximum may be -inf: nothing seen, weight 0
__device__ __forceinline__ float weight(float m, float top) { return m == -INFINITY ? 0.f : fast_exp2(m - top); }

// State of one warp for up to 8 kNT query heads: lane (g, t) holds heads 2 t, 2 t + 1 (+ 8) of rows g, g + 8 of every product.
template <int kNT>
struct State {
    float o[kNT][8][4];              // O^T: channel 16 mt + g + 8 (c >> 1), head 2 t + (c & 1)
    float m[kNT][2], l[kNT][2];      // maximum in use (the same in all lanes of a t), this lane's sum of weights
    __device__ __forceinline__ void reset()
    {
#pragma unroll
        for (int z = 0; z < kNT; ++z) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[z][i][c] = 0.f;
            m[z][0] = m[z][1] = -INFINITY;
            l[z][0] = l[z][1] = 0.f;
        }
    }
    // the row sums over the eight lanes of a t: afterwards each of them has the sum
    __device__ __forceinline__ void reduce_l()
    {
#pragma unroll
        for (int z = 0; z < kNT; ++z)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                l[z][c] += __shfl_xor_sync(0xffffffffu, l[z][c], 4);
                l[z][c] += __shfl_xor_sync(0xffffffffu, l[z][c], 8);
                l[z][c] += __shfl_xor_sync(0xffffffffu, l[z][c], 16);
            }
    }
    // O, times `f` of each row, as rows [G][128] in shared memory
    template <class F>
    __device__ __forceinline__ void put(float *dst, int G, int lane, const F &f) const
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int z = 0; z < kNT; ++z)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int hd = 8 * z + 2 * t + c;
                if (hd >= G) continue;
                const float x = f(z, c);
#pragma unroll
                for (int mt = 0; mt < 8; ++mt) {
                    dst[hd * kRowFloats + 16 * mt + g] = o[z][mt][c] * x;
                    dst[hd * kRowFloats + 16 * mt + g + 8] = o[z][mt][c + 2] * x;
                }
            }
    }
};

// One tile.  keep: bit r set where the request keeps row r (the others are zeros in the slot).
template <int kNT>
__device__ __forceinline__ void attend(State<kNT> &st, uint32_t slot, const uint32_t (&qf)[kNT][8][2], const uint32_t (&ql)[kNT][8][2], bool low,
                                       uint32_t keep, float scale_log2, int lane)
{
    const int mi = lane >> 3, rr = lane & 7, g = lane >> 2;
    // scores over the even and the odd steps apart: half the chain of dependent products
    float s[kNT][4], odd[kNT][4];
#pragma unroll
    for (int z = 0; z < kNT; ++z)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[z][c] = odd[z][c] = 0.f;
    const uint32_t krow = slot + ((mi & 1) * 8 + rr) * kRowBytes;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
        uint32_t a[4];
        ldmatrix_x4(a[0], a[1], a[2], a[3], krow + (((2 * kk + (mi >> 1)) ^ rr) << 4));
#pragma unroll
        for (int z = 0; z < kNT; ++z) mma_bf16(kk & 1 ? odd[z] : s[z], a, qf[z][kk][0], qf[z][kk][1]);
        if (low) {
#pragma unroll
            for (int z = 0; z < kNT; ++z) mma_bf16(kk & 1 ? odd[z] : s[z], a, ql[z][kk][0], ql[z][kk][1]);
        }
    }
#pragma unroll
    for (int z = 0; z < kNT; ++z)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[z][c] = (s[z][c] + odd[z][c]) * scale_log2;
    const uint32_t vrow = slot + kSlotV + ((mi >> 1) * 8 + rr) * kRowBytes;
    uint32_t va[4][4];                   // the first half of V, asked for before the softmax
#pragma unroll
    for (int mt = 0; mt < 4; ++mt) ldmatrix_x4_trans(va[mt][0], va[mt][1], va[mt][2], va[mt][3], vrow + (((2 * mt + (mi & 1)) ^ rr) << 4));
    if (keep != 0xffffu) {
        const bool keep0 = (keep >> g) & 1u, keep1 = (keep >> (g + 8)) & 1u;
#pragma unroll
        for (int z = 0; z < kNT; ++z)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                s[z][c] = keep0 ? s[z][c] : -INFINITY;
                s[z][c + 2] = keep1 ? s[z][c + 2] : -INFINITY;
            }
    }
    bool need = false;
#pragma unroll
    for (int z = 0; z < kNT; ++z)
#pragma unroll
        for (int c = 0; c < 2; ++c) need = need || fmaxf(s[z][c], s[z][c + 2]) > st.m[z][c] + kRaise;
    if (__any_sync(0xffffffffu, need)) {
#pragma unroll
        for (int z = 0; z < kNT; ++z)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float nm = fmaxf(st.m[z][c], fmaxf(s[z][c], s[z][c + 2]));
                nm = fmaxf(nm, __shfl_xor_sync(0xffffffffu, nm, 4));
                nm = fmaxf(nm, __shfl_xor_sync(0xffffffffu, nm, 8));
                nm = fmaxf(nm, __shfl_xor_sync(0xffffffffu, nm, 16));
                const float alpha = weight(st.m[z][c], nm);
                st.m[z][c] = nm;
                st.l[z][c] *= alpha;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    st.o[z][i][c] *= alpha;
                    st.o[z][i][c + 2] *= alpha;
                }
            }
    }
    uint32_t pb[kNT][4];                 // weights rounded, and what that leaves over
#pragma unroll
    for (int z = 0; z < kNT; ++z) {
        // nothing seen yet by this head: every score is -inf, every weight 0
        const float m0 = st.m[z][0] == -INFINITY ? 0.f : st.m[z][0], m1 = st.m[z][1] == -INFINITY ? 0.f : st.m[z][1];
        float p[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) p[c] = fast_exp2(s[z][c] - (c & 1 ? m1 : m0));
        st.l[z][0] += p[0] + p[2];
        st.l[z][1] += p[1] + p[3];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t x = pack_bf16(p[2 * h], p[2 * h + 1]);
            pb[z][h] = transpose_8x8(x);
            pb[z][2 + h] = transpose_8x8(pack_bf16(p[2 * h] - __uint_as_float(x << 16), p[2 * h + 1] - __uint_as_float(x & 0xffff0000u)));
        }
    }
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) {
        uint32_t (&a)[4] = va[mt & 3];
        if (mt >= 4) ldmatrix_x4_trans(a[0], a[1], a[2], a[3], vrow + (((2 * mt + (mi & 1)) ^ rr) << 4));
#pragma unroll
        for (int z = 0; z < kNT; ++z) {
            mma_bf16(st.o[z][mt], a, pb[z][0], pb[z][1]);
            mma_bf16(st.o[z][mt], a, pb[z][2], pb[z][3]);
        }
    }
}

// Running merge of rows: (m, l, four channels of this lane).
struct Row {
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    __device__ __forceinline__ void add(const float2 ml, const float4 v)
    {
        const float nm = fmaxf(m, ml.x), fo = weight(m, nm), fn = weight(ml.x, nm);
        o.x = fmaf(v.x, fn, o.x * fo);
        o.y = fmaf(v.y, fn, o.y * fo);
        o.z = fmaf(v.z, fn, o.z * fo);
        o.w = fmaf(v.w, fn, o.w * fo);
        l = fmaf(ml.y, fn, l * fo);
        m = nm;
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *dst) const
    {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    }
};

template <int kNT>
__global__ void __launch_bounds__(kWarps * 32, 1) decode_paged_kernel(PagedDecArgs a)
{
    extern __shared__ __align__(128) unsigned char smem[];
    const Smem lay(a.G, a.B);
    volatile int *last_flag = reinterpret_cast<volatile int *>(smem + lay.off_flags);        // [2]
    int2 *desc = reinterpret_cast<int2 *>(smem + lay.off_desc);  // pieces in tile order: segment (-1: none), bit 0 begins it, bit 1 ends it
    int *prefix = reinterpret_cast<int *>(smem + lay.off_table); // places before request b
    int *n_mode = prefix + a.B + 1;                              // length, sign bit set for sparse
    const uint32_t slots = smem_u32(smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool appending = a.k_new != nullptr;

    // Everything the launches before wrote is visible after the wait; the next launch may start early once every CTA has been through it.
    auto wait = [] { asm volatile("griddepcontrol.wait;\n" ::: "memory"); };
    auto release = [] { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); };
    if (!a.overlap) {
        wait();
        release();
    }

    // Places of a segment of request b (n > 0): 0 stands for its start, then all tiles but the last, kAppendCost empty ones where the
    // newest token is to be stored, the last tile.
    auto cost_of = [&](int b) {
        const int nm = n_mode[b];
        return 1 + Walk(nm & 0x7fffffff, nm >= 0, a.S, a.W).count + (appending ? kAppendCost : 0);
    };

    // ---- schedule ------------------------------------------------------------------------------
    uint32_t flags = 0;
    for (int b = tid; b < a.B; b += kWarps * 32) {
        const int n_raw = a.ctx_len[b], mode = a.mask[(size_t)b * a.L + a.layer];
        int n = max(n_raw, 0);
        if (mode > 1) flags |= FLUX_STATUS_BAD_MASK;
        if (n > a.max_context || n > a.pages.room()) {
            flags |= FLUX_STATUS_BAD_LENGTH;
            n = 0;               // its table has no such positions: a zero row
        }
        n_mode[b] = mode != 0 ? n : (int)((uint32_t)n | 0x80000000u);
        prefix[b + 1] = n > 0 ? cost_of(b) * a.Hkv : 0;
    }
    cta_sync();
    if (warp == 0) {
        int base = 0;
        for (int b0 = 0; b0 < a.B; b0 += 32) {
            const int b = b0 + lane;
            int x = b < a.B ? prefix[b + 1] : 0;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, d);
                if (lane >= d) x += y;
            }
            if (b < a.B) prefix[b + 1] = base + x;
            base += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0) prefix[0] = 0;
    }
    cta_sync();
    const int total = prefix[a.B];

    // Equal ranges, of at least one place per warp.  A range does not end inside a short segment: below kShortSpan the whole
    // segment costs a CTA no more time than merging across CTAs would, above it the ranges may differ by a 32nd (an eighth: 64 short contexts
    // 73.7 us instead of 72.7).
    const int span = max((total + (int)gridDim.x - 1) / (int)gridDim.x, kWarps);
    const int whole_below = span <= kShortSpan ? kShortSpan : span / 32;
    auto bound = [&](int k) {
        const int v = (int)min((int64_t)k * span, (int64_t)total);
        if (v == total) return v;
        const Place p(prefix, a.B, v, cost_of);
        return p.cost <= whole_below ? v - p.x : v;
    };
    const int c_begin = bound((int)blockIdx.x), c_end = bound((int)blockIdx.x + 1);
    const int v_begin = c_begin + (int)((int64_t)(c_end - c_begin) * warp / kWarps);
    const int v_end = c_begin + (int)((int64_t)(c_end - c_begin) * (warp + 1) / kWarps);

    // ---- a warp's tiles, one after the other ------------------------------------------------------
    struct Cursor {
        Place p;
        int v, t, t_end, n;              // place of the segment's first tile in range; tile at hand and end of the range's tiles of the segment
        Walk wk;
        bool fa, done;
        __device__ __forceinline__ Cursor(const Place &p_) : p(p_), wk(0, true, 0, 0) {}
    };
    // the tiles of the segment at c.p that lie in the range: those of places max(x, 1) .. x_end - 1
    auto enter = [&](Cursor &c) {
        const int nm = n_mode[c.p.b];
        c.n = nm & 0x7fffffff;
        c.fa = nm >= 0;
        c.wk = Walk(c.n, c.fa, a.S, a.W);
        const int x_end = min(c.p.cost, c.p.x + (v_end - c.v)), last = c.wk.count - 1;
        c.t = min(max(c.p.x, 1) - 1, last);
        c.t_end = x_end == c.p.cost ? c.wk.count : min(x_end - 1, last);
    };
    auto settle = [&](Cursor &c) {       // on to the next segment with a tile
        while (c.t >= c.t_end) {
            c.v += c.p.cost - c.p.x;
            if (c.v >= v_end) {
                c.done = true;
                return;
            }
            c.p.next_segment(prefix, a.Hkv, cost_of);
            enter(c);
        }
    };
    const bool any = v_begin < v_end;
    Cursor cur(any ? Place(prefix, a.B, v_begin, cost_of) : Place());
    cur.v = v_begin;
    cur.done = !any;
    if (any) {
        enter(cur);
        settle(cur);
    }
    Cursor ld = cur;

    // Rows of tile `u` of a request that are kept.
    auto kept = [&](const Cursor &c, int u) {
        const int p0 = u * kTile;
        uint32_t m = c.n - p0 >= kTile ? 0xffffu : (1u << (c.n - p0)) - 1u;
        const int lo = c.n - a.W;
        if (!c.fa && lo > a.S && p0 < lo && p0 + kTile > a.S) {          // sink: rows below S; window: rows from lo on
            const uint32_t sink = p0 < a.S ? (1u << (a.S - p0)) - 1u : 0u;
            m &= sink | (lo - p0 < kTile ? 0xffffu << (lo - p0) : 0u);
        }
        return m;
    };

    // loader: table entries of 32 tiles at a time, a lane for each
    int pg = FLUX_PAGE_NONE, pg_base = 0, pg_req = -1;
    const int lc = lane & 15, lr0 = lane >> 4;       // this lane's piece of a row, and its rows: lr0, lr0 + 2, ...
    const uint32_t row_bytes = (uint32_t)a.Hkv * kRowBytes;
    const unsigned char *lane_k = a.pages.pool[0] + lr0 * row_bytes + lc * 16, *lane_v = a.pages.pool[1] + lr0 * row_bytes + lc * 16;
    uint32_t place[4];                   // of rows lr0 + 2 i in a slot, swizzled; eight rows further on the same again
#pragma unroll
    for (int i = 0; i < 4; ++i) place[i] = slots + warp * kRing * kSlotBytes + (lr0 + 2 * i) * kRowBytes + ((lc ^ ((lr0 + 2 * i) & 7)) << 4);
    auto page_of = [&](const Cursor &c, int u) {
        if (c.p.b != pg_req || u < pg_base || u >= pg_base + 32) {
            pg_req = c.p.b;
            pg_base = u;
            pg = FLUX_PAGE_NONE;
            if ((u + lane) * kTile < c.n) pg = a.pages.entry(c.p.b, (u + lane) * kTile);
        }
        const int page = __shfl_sync(0xffffffffu, pg, u - pg_base);
        return page >= 0 && page < a.pages.n_pages ? page : FLUX_PAGE_NONE;
    };
    uint32_t lost = 0;                   // a needed page is missing: its positions count as masked
    auto issue = [&](int slot) {
        const int u = ld.wk.tile(ld.t), page = page_of(ld, u);
        uint32_t keep = kept(ld, u);
        if (page == FLUX_PAGE_NONE) {
            lost = FLUX_STATUS_BAD_PAGE;
            keep = 0;
        }
        const bool newest = ld.t == ld.wk.count - 1;
        if (a.touch != nullptr && ld.p.head == 0 && lane == 0) atomicOr(a.touch + (size_t)ld.p.b * a.touch_words + (u >> 1), keep << (16 * (u & 1)));
        if (newest && appending) keep &= ~(1u << ((ld.n - 1) & (kTile - 1)));          // it comes from k_new, v_new
        // (a pool has fewer than 2^32 positions)
        const uint64_t at = (uint64_t)(uint32_t)a.pages.row(max(page, 0), u * kTile) * row_bytes + (uint32_t)(ld.p.head * kRowBytes);
        const unsigned char *k = lane_k + at, *v = lane_v + at;
        const uint32_t dst = slot * kSlotBytes;
        if (keep == 0xffffu) {           // nearly all tiles
#pragma unroll
            for (int i = 0; i < kTile / 2; ++i, k += 2 * row_bytes, v += 2 * row_bytes) {
                cp_async16_whole(dst + place[i & 3] + (i / 4) * 8 * kRowBytes, k);
                cp_async16_whole(dst + place[i & 3] + (i / 4) * 8 * kRowBytes + kSlotV, v);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kTile / 2; ++i) {
                const int n = (keep >> (lr0 + 2 * i)) & 1u ? 16 : 0;
                const uint64_t off = n ? (uint64_t)(2 * i) * row_bytes : 0;
                const uint32_t d = dst + place[i & 3] + (i / 4) * 8 * kRowBytes;
                cp_async16(d, n ? k + off : a.pages.pool[0], n);
                cp_async16(d + kSlotV, n ? v + off : a.pages.pool[1], n);
            }
        }
        ++ld.t;
        settle(ld);
    };
    // Query rows and the newest token's rows of a segment, asked for.  Ordinary loads: with launch overlap the launch before may write the
    // rows while this kernel is resident.
    RopeLane turn;
    RopeFreqs freqs = {};
    Pieces weights[2] = {};
    Pieces rows[2 * kNT], fresh = {};    // fresh: pieces of the newest token's rows, lanes 0-7 of K, 8-15 of V
    int fresh_page = FLUX_PAGE_NONE;     // and the page that takes them
    if (a.turn || appending) turn.place(a.rope, lane);
    auto ask = [&](const Cursor &c) {
        if (a.turn) {
            const unsigned char *q = a.q + c.p.b * a.q_stride + (size_t)c.p.head * a.G * kRowBytes;
#pragma unroll
            for (int i = 0; i < 2 * kNT; ++i) {
                const int h = 4 * i + lane / kHeadLanes;
                rows[i].a = rows[i].b = make_uint4(0u, 0u, 0u, 0u);
                if (h < a.G) rows[i] = turn.load(q + h * kRowBytes);
            }
        }
        if (appending && c.t_end == c.wk.count) {
            fresh = turn.load((lane < kHeadLanes ? a.k_new + c.p.b * a.k_stride : a.v_new + c.p.b * a.v_stride) + c.p.head * kRowBytes);
            fresh_page = a.pages.entry(c.p.b, c.n - 1);
        }
    };
    auto ask_first = [&] {               // ahead of the first tiles, whose requests wait for table entries
        if (a.turn) {
            freqs.read(a.rope, lane);
            weights[0] = rope_weights(a.rope.weight[0], turn);
            weights[1] = rope_weights(a.rope.weight[1], turn);
        }
        if (!cur.done) ask(cur);
    };
    int primed = 0;
    if (!a.overlap) ask_first();
    if (a.overlap) {
        // the newest two positions may still be on their way
        while (primed < kRing && !ld.done && (ld.wk.tile(ld.t) + 1) * kTile <= ld.n - 2) {
            issue(primed++);
            cp_async_commit();
        }
        wait();
        release();
        ask_first();
    }
    for (; primed < kRing; ++primed) {
        if (!ld.done) issue(primed);
        cp_async_commit();
    }

    // ---- dispatch records, status bits, zero rows of inactive requests ------------------------------
    if (flags != 0 && blockIdx.x == 0) atomicOr(a.status, flags);
    if (blockIdx.x == 0)
        for (int b = tid; b < a.B; b += kWarps * 32) {
            const int nm = n_mode[b], n = nm & 0x7fffffff;
            const bool two = nm < 0 && n > a.S + a.W;
            int32_t *d = a.debug + (size_t)b * 8;
            d[0] = nm < 0 ? 0 : 1; d[1] = a.layer; d[2] = b; d[3] = n;
            d[4] = 0; d[5] = two ? a.S : n; d[6] = two ? n - a.W : 0; d[7] = two ? n : 0;
        }
    for (int b = blockIdx.x; b < a.B; b += gridDim.x)
        if (prefix[b + 1] == prefix[b])
            for (int i = tid; i < a.Hq * (kRowBytes / 16); i += kWarps * 32)
                reinterpret_cast<uint4 *>(a.out + (size_t)b * a.Hq * kHeadDim)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (c_begin >= c_end) return;        // the whole CTA

    // ---- attention -----------------------------------------------------------------------------------
    State<kNT> st;
    uint32_t qf[kNT][8][2], ql[kNT][8][2];       // query rows, and what rounding them has left over (only those turned here)
    int d_first = -1, d_last = -1, f_first = 0, f_last = 0;      // this warp's pieces: segment, flags
    unsigned char *ring = smem + warp * kRing * kSlotBytes;
    unsigned char *piece = smem + lay.off_piece + warp * lay.piece_bytes;
    // Memory of this warp that nothing is in: its scratch, or, where that does not fit, at first its piece, then the slot used last, which is
    // filled again only behind the next segment's query rows.
    constexpr bool kScratch = kNT == 1;
    unsigned char *spare = kScratch ? smem + lay.off_scratch + warp * a.G * 2 * kRowBytes : piece;
    int slot = 0, before = -1;           // slot of the tile at hand; one to be filled
    bool fresh_segment = true, asked = true, begins = false;
    while (!cur.done) {
        if (fresh_segment) {
            // Query rows as the B operand: lane (g, t) holds channels 16 kk + 2 t, + 1 and + 8, + 9 of head g (+ 8).
            fresh_segment = false;
            begins = cur.t == 0;
            st.reset();
            const unsigned char *q = a.q + cur.p.b * a.q_stride + (size_t)cur.p.head * a.G * kRowBytes;
            if (!asked) ask(cur);
            asked = false;
            if (a.turn) {
                turn.sines(a.rope, freqs, lane, cur.n - 1);
                RopeFactors f;
                f.fold(a.rope, turn, a.rope.weight[0] != nullptr, weights[0]);
#pragma unroll
                for (int i = 0; i < 2 * kNT; ++i) {
                    if (4 * i >= a.G) break;
                    const int h = 4 * i + lane / kHeadLanes;
                    Pairs y = f.turn(rows[i], a.rope.pairs != 0, a.rope.weight[0] != nullptr, a.rope.eps);
                    Pieces p = to_pieces(y, a.rope.pairs != 0);
                    const Pairs r = to_pairs(p, a.rope.pairs != 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        y.a[j].x -= r.a[j].x; y.a[j].y -= r.a[j].y;
                        y.b[j].x -= r.b[j].x; y.b[j].y -= r.b[j].y;
                    }
                    if (h < a.G) {
                        turn.store(spare + h * kRowBytes, p);
                        turn.store(spare + (a.G + h) * kRowBytes, to_pieces(y, a.rope.pairs != 0));
                    }
                }
                if (appending && cur.t_end == cur.wk.count) {
                    f.fold(a.rope, turn, a.rope.weight[1] != nullptr, weights[1]);
                    const Pieces p = to_pieces(f.turn(fresh, a.rope.pairs != 0, a.rope.weight[1] != nullptr, a.rope.eps), a.rope.pairs != 0);
                    if (lane < kHeadLanes) fresh = p;
                }
                __syncwarp();
                q = spare;
            }
            const int g = lane >> 2, t = lane & 3;
#pragma unroll
            for (int z = 0; z < kNT; ++z)
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const unsigned char *word = q + (8 * z + g) * kRowBytes + kk * 32 + e * 16 + t * 4;
                        qf[z][kk][e] = 8 * z + g < a.G ? *reinterpret_cast<const uint32_t *>(word) : 0u;
                        ql[z][kk][e] = a.turn && 8 * z + g < a.G ? *reinterpret_cast<const uint32_t *>(word + a.G * kRowBytes) : 0u;
                    }
            __syncwarp();
        }
        if (!kScratch && before >= 0) {
            if (!ld.done) issue(before);
            cp_async_commit();
        }
        cp_async_wait<kRing - 1>();
        __syncwarp();
        const int u = cur.wk.tile(cur.t);
        uint32_t keep = kept(cur, u);
        unsigned char *data = ring + slot * kSlotBytes;
        // a missing page: known to the loader, which is further on; asked again (rare: only once something is missing)
        if (lost != 0) {
            const int page = a.pages.entry(cur.p.b, u * kTile);
            if (page < 0 || page >= a.pages.n_pages) keep = 0;
        }
        if (appending && cur.t == cur.wk.count - 1 && fresh_page >= 0 && fresh_page < a.pages.n_pages) {
            const int pos = cur.n - 1, r = pos & (kTile - 1);
            if (lane < 2 * kHeadLanes) {
                const int kv = lane / kHeadLanes;
                turn.store((kv ? a.pages.pool[1] : a.pages.pool[0]) + ((int64_t)a.pages.row(fresh_page, pos) * a.Hkv + cur.p.head) * kRowBytes, fresh);
                unsigned char *row = data + kv * kSlotV + r * kRowBytes;
                *reinterpret_cast<uint4 *>(row + ((turn.a / 8 ^ (r & 7)) << 4)) = fresh.a;
                *reinterpret_cast<uint4 *>(row + ((turn.b / 8 ^ (r & 7)) << 4)) = fresh.b;
            }
            __syncwarp();
        }
        attend<kNT>(st, slots + (uint32_t)(warp * kRing + slot) * kSlotBytes, qf, ql, a.turn != 0, keep, a.scale_log2, lane);
        __syncwarp();
        if (kScratch) {
            if (!ld.done) issue(slot);
            cp_async_commit();
        } else {
            before = slot;
            spare = data;
        }
        slot = slot + 1 == kRing ? 0 : slot + 1;
        if (++cur.t == cur.t_end) {      // the range's part of the segment is done
            const bool ends = cur.t_end == cur.wk.count;
            const int seg = cur.p.b * a.Hkv + cur.p.head;
            st.reduce_l();
            if (begins && ends) {        // a whole segment in one warp: its output rows
                float *o = reinterpret_cast<float *>(spare);
                st.put(o, a.G, lane, [&](int z, int c) { return st.l[z][c] == 0.f ? 0.f : 1.f / st.l[z][c]; });
                __syncwarp();
                __nv_bfloat16 *orow = a.out + ((size_t)cur.p.b * a.Hq + (size_t)cur.p.head * a.G) * kHeadDim + 4 * lane;
                for (int h = 0; h < a.G; ++h) {
                    const float4 x = *reinterpret_cast<const float4 *>(o + h * kRowFloats + 4 * lane);
                    *reinterpret_cast<uint2 *>(orow + h * kHeadDim) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
                }
                __syncwarp();
            } else {
                float *dst = reinterpret_cast<float *>(piece);
                if (ends) {
                    d_first = seg;
                    f_first = 2;
                } else {                 // the warp's last segment: its piece goes over its ring, which has been used up
                    d_last = seg;
                    f_last = begins ? 1 : 0;
                    dst = reinterpret_cast<float *>(ring);
                    cp_async_wait<0>();
                    __syncwarp();
                }
                st.put(dst, a.G, lane, [](int, int) { return 1.f; });
                if (lane >> 2 == 0)
#pragma unroll
                    for (int z = 0; z < kNT; ++z)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int hd = 8 * z + 2 * lane + c;
                            if (hd < a.G) *reinterpret_cast<float2 *>(dst + a.G * kRowFloats + 2 * hd) = make_float2(st.m[z][c], st.l[z][c]);
                        }
                __syncwarp();
            }
            settle(cur);
            fresh_segment = true;
        }
    }
    cp_async_wait<0>();
    if (lost != 0 && lane == 0) atomicOr(a.status, lost);
    if (lane == 0) {
        desc[2 * warp] = make_int2(d_first, f_first);
        desc[2 * warp + 1] = make_int2(d_last, f_last);
    }
    cta_sync();

    // ---- segments that this CTA's warps share -------------------------------------------------------
    // Pieces of one segment are neighbours in `desc` (empty entries aside).  Groups are numbered in order; (group, head) rows
    // are dealt to the warps, four channels to a lane.
    int shared_seg[2] = {-1, -1};        // segments that go on in other CTAs: at most the range's first and last
    int group = 0, n_shared = 0;
    const int2 mine = lane < 2 * kWarps ? desc[lane] : make_int2(-1, 0);
    for (uint32_t left = __ballot_sync(0xffffffffu, mine.x >= 0); left != 0; ++group) {
        const int seg = __shfl_sync(0xffffffffu, mine.x, __ffs(left) - 1);
        const uint32_t pieces = __ballot_sync(0xffffffffu, mine.x == seg);
        const bool whole = __any_sync(0xffffffffu, mine.x == seg && (mine.y & 1)) && __any_sync(0xffffffffu, mine.x == seg && (mine.y & 2));
        left &= ~pieces;
        if (!whole) {
            if (n_shared == 0) shared_seg[0] = seg; else shared_seg[1] = seg;
            ++n_shared;
        }
        for (int hd = (warp - group * a.G % kWarps + kWarps) % kWarps; hd < a.G; hd += kWarps) {
            Row r;
            for (uint32_t todo = pieces; todo != 0; todo &= todo - 1) {
                const int j = __ffs(todo) - 1;
                const float *src = reinterpret_cast<const float *>(j & 1 ? smem + (j >> 1) * kRing * kSlotBytes
                                                                         : smem + lay.off_piece + (j >> 1) * lay.piece_bytes);
                r.add(*reinterpret_cast<const float2 *>(src + a.G * kRowFloats + 2 * hd), *reinterpret_cast<const float4 *>(src + hd * kRowFloats + 4 * lane));
            }
            if (whole) {
                r.store(a.out + ((size_t)(seg / a.Hkv) * a.Hq + (size_t)(seg % a.Hkv) * a.G + hd) * kHeadDim + 4 * lane);
            } else {
                const size_t e = ((size_t)blockIdx.x + seg) * a.G + hd;
                *reinterpret_cast<float4 *>(a.part_o + e * kHeadDim + 4 * lane) = r.o;
                if (lane == 0) *reinterpret_cast<float2 *>(a.part_ml + e * 2) = make_float2(r.m, r.l);
            }
        }
    }
    if (n_shared == 0) return;

    // ---- segments that several CTAs share -----------------------------------------------------------
    // The barrier orders this CTA's partial stores before thread 0's tickets (release); the CTA that draws a segment's last
    // ticket has acquired all the others' partials.
    cta_sync();
    // Many partials are added up in two steps, those of groups of neighbouring CTAs first, each by the last of the group: an SM gets 32
    // bytes a nanosecond from the L2, and 148 partials of 16 heads are 1.2 MB.
    struct Parts {
        int first, count, group;             // CTAs that hold tiles of the segment; how many make a group (0: no groups)
    };
    auto parts_of = [&](int seg) {           // of a segment longer than `whole_below` (a range is longer than the empty places)
        static_assert(kAppendCost < kWarps, "a CTA's range holds a tile of every segment it meets beyond place 0");
        const int sb = seg / a.Hkv, cost = (prefix[sb + 1] - prefix[sb]) / a.Hkv, begin = prefix[sb] + (seg % a.Hkv) * cost;
        Parts r;
        r.first = (begin + 1) / span;
        r.count = (begin + cost - 1) / span - r.first + 1;
        r.group = 0;                         // at most 32, a lane for each
        static_assert(kDecMaxCtas <= 32 * 32, "groups");
        if (r.count * a.G >= kManyRows)
            for (r.group = kMinGroup; r.group * r.group < r.count; ++r.group) {}
        return r;
    };
    auto draw = [&](uint32_t *ticket, int of) {          // true for the last of them, which makes it ready for the next launch
        unsigned seen;
        asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(seen) : "l"(ticket) : "memory");
        if (seen == (unsigned)(of - 1)) *ticket = 0u;
        return seen == (unsigned)(of - 1);
    };
    if (tid < n_shared) {
        const int seg = tid == 0 ? shared_seg[0] : shared_seg[1];
        const Parts r = parts_of(seg);
        uint32_t *ticket = a.tickets + seg;
        int of = r.count;
        if (r.group) {
            const int begin = ((int)blockIdx.x - r.first) / r.group * r.group;
            ticket = a.group_tickets + r.first + begin + seg;
            of = min(r.group, r.count - begin);
        }
        last_flag[tid] = draw(ticket, of);
    }
    cta_sync();
    for (int i = 0; i < n_shared; ++i) {
        if (!last_flag[i]) continue;
        const int seg = i == 0 ? shared_seg[0] : shared_seg[1];
        const Parts r = parts_of(seg);
        int n_part = r.count;
        const float *src = a.part_o + ((size_t)r.first + seg) * a.G * kHeadDim, *src_ml = a.part_ml + ((size_t)r.first + seg) * a.G * 2;
        if (r.group) {
            const int g = ((int)blockIdx.x - r.first) / r.group, np = min(r.group, r.count - g * r.group);
            const float *gp = src + (size_t)g * r.group * a.G * kHeadDim, *gp_ml = src_ml + (size_t)g * r.group * a.G * 2;
            for (int hd = warp; hd < a.G; hd += kWarps) {
                const float2 ml = lane < np ? __ldcg(reinterpret_cast<const float2 *>(gp_ml + ((size_t)lane * a.G + hd) * 2)) : make_float2(-INFINITY, 0.f);
                Row row;
                row.m = ml.x;
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) row.m = fmaxf(row.m, __shfl_xor_sync(0xffffffffu, row.m, d));
                const float w = weight(ml.x, row.m);
                row.l = ml.y * w;
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) row.l += __shfl_xor_sync(0xffffffffu, row.l, d);
#pragma unroll 8
                for (int p = 0; p < np; ++p) {
                    const float f = __shfl_sync(0xffffffffu, w, p);
                    const float4 v = __ldcg(reinterpret_cast<const float4 *>(gp + ((size_t)p * a.G + hd) * kHeadDim + 4 * lane));
                    row.o.x = fmaf(v.x, f, row.o.x);
                    row.o.y = fmaf(v.y, f, row.o.y);
                    row.o.z = fmaf(v.z, f, row.o.z);
                    row.o.w = fmaf(v.w, f, row.o.w);
                }
                const size_t e = ((size_t)r.first + seg + g) * a.G + hd;
                *reinterpret_cast<float4 *>(a.group_o + e * kHeadDim + 4 * lane) = row.o;
                if (lane == 0) *reinterpret_cast<float2 *>(a.group_ml + e * 2) = make_float2(row.m, row.l);
            }
            n_part = (r.count + r.group - 1) / r.group;
            cta_sync();
            if (tid == 0) last_flag[i] = draw(a.tickets + seg, n_part);
            cta_sync();
            if (!last_flag[i]) continue;
            src = a.group_o + ((size_t)r.first + seg) * a.G * kHeadDim;
            src_ml = a.group_ml + ((size_t)r.first + seg) * a.G * 2;
        }
        // All partials of the segment (neighbours in the workspace: entry (CTA + segment) G + head) come into the ring, which is idle
        // by now, in one round of asynchronous copies.
        const int fit = min(kWarps * kRing * kSlotBytes / (a.G * kRowFloats * 4), kMaxParts);
        Row rows[kNT];                                   // heads warp, warp + 8
        for (int p0 = 0; p0 < n_part; p0 += fit) {
            const int np = min(fit, n_part - p0);
            cta_sync();                                  // the ring's last readers (pieces, the round before) are done
            for (int z = tid; z < np * a.G * 32; z += kWarps * 32) cp_async16(slots + z * 16, src + (size_t)p0 * a.G * kHeadDim + (size_t)z * 4, 16);
            cp_async_commit();
            // meanwhile the weights, a lane per partial
            float w[kNT][kMaxParts / 32];
#pragma unroll
            for (int y = 0; y < kNT; ++y) {
                const int hd = warp + kWarps * y;
                float nm = rows[y].m;
                float2 ml[kMaxParts / 32];
#pragma unroll
                for (int z = 0; z < kMaxParts / 32; ++z) {
                    ml[z] = make_float2(-INFINITY, 0.f);
                    if (hd < a.G && 32 * z + lane < np) ml[z] = __ldcg(reinterpret_cast<const float2 *>(src_ml + ((size_t)(p0 + 32 * z + lane) * a.G + hd) * 2));
                    nm = fmaxf(nm, ml[z].x);
                }
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) nm = fmaxf(nm, __shfl_xor_sync(0xffffffffu, nm, d));
                float l = 0.f;
#pragma unroll
                for (int z = 0; z < kMaxParts / 32; ++z) {
                    w[y][z] = weight(ml[z].x, nm);
                    l = fmaf(ml[z].y, w[y][z], l);
                }
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
                const float fo = weight(rows[y].m, nm);
                rows[y].l = fmaf(rows[y].l, fo, l);
                rows[y].m = nm;
                rows[y].o.x *= fo; rows[y].o.y *= fo; rows[y].o.z *= fo; rows[y].o.w *= fo;
            }
            cp_async_wait<0>();
            cta_sync();
#pragma unroll
            for (int y = 0; y < kNT; ++y) {
                const int hd = warp + kWarps * y;
                if (hd >= a.G) continue;
#pragma unroll
                for (int z = 0; z < kMaxParts / 32; ++z)
#pragma unroll 4
                    for (int x = 0; x < min(32, np - 32 * z); ++x) {
                        const float f = __shfl_sync(0xffffffffu, w[y][z], x);
                        const float4 v = *reinterpret_cast<const float4 *>(smem + ((size_t)(32 * z + x) * a.G + hd) * kRowFloats * 4 + lane * 16);
                        rows[y].o.x = fmaf(v.x, f, rows[y].o.x);
                        rows[y].o.y = fmaf(v.y, f, rows[y].o.y);
                        rows[y].o.z = fmaf(v.z, f, rows[y].o.z);
                        rows[y].o.w = fmaf(v.w, f, rows[y].o.w);
                    }
            }
        }
#pragma unroll
        for (int y = 0; y < kNT; ++y)
            if (warp + kWarps * y < a.G)
                rows[y].store(a.out + ((size_t)(seg / a.Hkv) * a.Hq + (size_t)(seg % a.Hkv) * a.G + warp + kWarps * y) * kHeadDim + 4 * lane);
    }
}

using PagedDecFn = void (*)(PagedDecArgs);
PagedDecFn pick(int G) { return G <= 8 ? decode_paged_kernel<1> : decode_paged_kernel<2>; }

}  // namespace

int decode_paged_setup(flux_plan *p)
{
    if (p->dev.smem_optin < Smem(16, kMaxBatch).total)
        return fail(FLUX_E_CUDA, "device offers %d bytes of shared memory per block, the paged decode needs %d", p->dev.smem_optin,
                    Smem(16, kMaxBatch).total);
    for (int G = 8; G <= 16; G += 8) {
        const int rc = check_cuda(cudaFuncSetAttribute((const void *)pick(G), cudaFuncAttributeMaxDynamicSharedMemorySize, Smem(16, kMaxBatch).total),
                                  "cudaFuncSetAttribute(decode_paged_kernel)");
        if (rc) return rc;
    }
    return FLUX_OK;
}

int launch_decode_paged(flux_plan *p, int layer, int B, const flux_rope *rope, const void *q, int64_t q_stride, const void *k_new, const void *v_new,
                        int64_t k_stride, int64_t v_stride, const flux_pages &pages, const int32_t *ctx_len, void *out, cudaStream_t st)
{
    const flux_config &c = p->cfg;
    // the kernel numbers the places of all requests in 32 bits
    if ((int64_t)B * c.n_kv_heads * (c.max_context / kTile + 3 + kAppendCost + 1) >= (1ll << 30))
        return fail(FLUX_E_CAPACITY, "%d requests of %d KV heads and up to %d positions are too many for one call", B, c.n_kv_heads, c.max_context);
    char *ws = (char *)p->ws;
    PagedDecArgs a;
    a.q = (const unsigned char *)q;
    a.q_stride = q_stride * 2;
    a.k_new = (const unsigned char *)k_new;
    a.v_new = (const unsigned char *)v_new;
    a.k_stride = k_stride * 2; a.v_stride = v_stride * 2;
    a.pages = page_args(pages);
    a.ctx_len = ctx_len;
    a.mask = p->d_mask;
    a.B = B; a.L = c.n_layers; a.layer = layer; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = p->G;
    a.S = c.sink; a.W = c.window; a.max_context = c.max_context;
    a.scale_log2 = p->scale_log2;
    a.part_o = (float *)(ws + p->lay.part_o);
    a.part_ml = (float *)(ws + p->lay.part_ml);
    a.tickets = (uint32_t *)(ws + p->lay.kvq_tickets);
    a.group_o = (float *)(ws + p->lay.group_o);
    a.group_ml = (float *)(ws + p->lay.group_ml);
    a.group_tickets = (uint32_t *)(ws + p->lay.group_tickets);
    a.debug = (int32_t *)(ws + p->lay.debug);
    a.status = (uint32_t *)(ws + p->lay.status);
    a.out = (__nv_bfloat16 *)out;
    a.touch = p->touch;
    a.touch_words = p->touch_words;
    a.rope = rope_args(rope);
    a.turn = rope != nullptr;
    // (asked whatever the setting is, so that a page call is taken off with the decode behind it)
    const bool tables_change = p->page_calls.take(st);
    a.overlap = p->launch_overlap && !tables_change;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)p->dec_ctas);
    lc.blockDim = dim3(kWarps * 32);
    lc.dynamicSmemBytes = Smem(p->G, B).total;
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    const int rec = prof_begin(p, FLUX_KERNEL_DECODE, st);
    cudaError_t e = cudaLaunchKernelEx(&lc, pick(p->G), a);
    prof_end(p, rec, st);
    p->launches++;
    p->debug_records = B;
    return check_cuda(e, "paged decode kernel launch");
}

}  // namespace flux
