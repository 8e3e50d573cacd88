// Decode attention over the 8-bit KV cache (layout: flux_kvq.h), one launch per layer.
//
// o = softmax(scale q K~^T) V~ over the kept positions, K~ = s_K c_K and V~ = s_V c_V with one scale per block of 16
// positions.  Bound by memory: 128 bytes per kept position and head for each of K and V.
//
// Work: (request, KV head) segments of strips of 32 positions (plus the bf16 tail of the newest block as a unit of its
// own), laid end to end and cut into one range per CTA, one CTA per SM; a CTA's range is cut again into one range per
// consumer warp (0-7).  A warp therefore walks whole short segments alone, from query rows to output rows, and meets the
// other warps only once, at the end.  Every segment counts one unit more than it has, which is what starting and finishing it
// costs.  Warps 8-11 bring the units in by bulk copies, two consumers each (a strip of one head is one piece of 4 KB, codes
// and scales, for each of K and V; issuing the copies of all eight is too much for one warp).  Every consumer warp has a ring of slots of its own: the parity test of a barrier tells a phase only from its
// neighbours, so a slot must be waited for by one warp, in the order of its uses.
//
// Products: mma.m16n8k16 in fp16 with the cache as the A operand -- S^T = K q^T (keys x heads) and O^T = V^T p^T
// (channels x heads) -- so up to 8 query heads fill the N dimension instead of padding M to 16, and a lane's codes are
// contiguous 16-byte pieces.  Both code types are exact in fp16.  Query rows are scaled by a power of two to magnitude
// 1..2 (2..4 in the topmost binade) and rounded to fp16: bf16 values fit, and what falls below 2^-24 of the row's largest entry is
// below fp32's own rounding of the sum.
//
// Softmax: fp32, log2 domain, with one maximum for the row sum and one for O, since V's scales may lie anywhere in 2^-100 .. 2^119.
// The row sum adds p = 2^(s - m), m following the largest score s.  O adds p' c, p' = p scale 2^k, so it accumulates in the matrix unit
// without a scale per block; k = m - lim, where lim follows the largest s + e (e: exponent of the scale), keeps the largest p' within
// 2^10 .. 2^15.  p' is rounded to fp16: relative 2^-11, finer than the bf16 output, down to 2^-24 of the largest, and 2^-35 of it
// absolutely below that (k is at most 92, so weights times scales below 2^-106 lose bits: outputs below 2^-97).  The
// maxima are raised when a unit's largest exceeds what is in use by 2^4, and to that largest, whose weight then is a power of two (but
// for an int8 scale) that rounding leaves alone: a key that outweighs the others does so exactly.  O's units do not depend on m; when
// a piece is finished its row sum takes the same ones, l 2^k, which is in range for up to 2^30 keys.  (A single maximum, of s + e, with
// p' / scale in the row sum was the first form: 2^18 keys of the smallest scale, and fewer of rising scores, overflowed it, and it lost
// keys whose scale was 2^130 times smaller than another's.)
//
// flux_attn_decode_step_kvq: the warp that takes a segment's tail also stores the newest token -- its row in the tail, or, when it
// completes the block, the block's codes -- and attends to the stored values (append_token); a second launch cost 3 to 11 us.
//
// With launch overlap (flux_plan_set_launch_overlap) the schedule and the copies of every block but the newest run ahead of
// the grid-dependency wait, that is while the launch before is still merging: the caller has promised that it writes neither
// lengths, modes and addresses nor those blocks.
//
// Merge: at the end of a CTA the pieces of segments that its warps share are added up in shared memory; a segment spread
// over several CTAs goes on through partials in the workspace, and the CTA that finishes last (a ticket per segment) adds
// them up in the order of the CTAs.  No CTA waits for another.
#include "flux_decode_common.h"
#include "flux_kvq.h"
#include "flux_tc_util.h"

namespace flux {
namespace {

using tc::elect_one;
using tc::mbar_arrive;
using tc::mbar_expect_tx;
using tc::mbar_init;
using tc::mbar_try;
using tc::mbar_wait;

constexpr int kCons = 8;                                        // consumer warps
constexpr int kProd = 4;                                        // producer warps, each for kCons / kProd consumers
// Registers of a thread with two groups of heads (kNT 2), moved from the producers' warpgroup to the consumers' two at the fork: the state
// of 16 heads does not fit beside the rest in the 168 that 384 threads get.  The host checks that the launch covers the sum.
constexpr int kConsumerRegs = 208, kProducerRegs = 88;
constexpr int kStrip = kKvqStrip;
constexpr int kStripBlocks = kStrip / kKvqBlock;
constexpr int kSlotV = kKvqStripBytes;                          // slot: K strip | V strip, or K tail | V tail
constexpr int kSlotBytes = 2 * kKvqStripBytes;
static_assert(kKvqTailHeadBytes <= kKvqStripBytes, "a slot takes a strip or a tail");
constexpr int kMaxRing = 3;                                     // slots of one consumer warp (2 where the rest does not fit)
constexpr int kRowFloats = kHeadDim;                            // a piece: G rows of O, then G pairs (m, l)
constexpr int kMaxParts = 64;                                   // partials a CTA adds up in one round
constexpr int kAppendCost = 3;                                  // storing the newest token costs a warp as much as that many units
constexpr int kShortSpan = 24;                                  // units a CTA's warps walk in about the time a merge across CTAs takes

// Shared memory: slots | first pieces [kCons][G rows, G pairs] | full, empty barriers | flags | piece table | cache addresses | prefix, lengths
struct Smem {
    int ring, piece_bytes, off_piece, off_bars, off_flags, off_desc, off_caches, off_table, total;
    __host__ __device__ __forceinline__ Smem(int ring_, int G, int B) : ring(ring_)
    {
        piece_bytes = G * (kRowFloats + 2) * (int)sizeof(float);
        piece_bytes = (piece_bytes + 15) / 16 * 16;
        off_piece = kCons * ring * kSlotBytes;
        off_bars = off_piece + kCons * piece_bytes;
        off_flags = off_bars + 2 * kCons * ring * 8;
        off_desc = off_flags + 16;
        off_caches = off_desc + 2 * kCons * (int)sizeof(int) * 2;
        off_table = off_caches + 2 * B * (int)sizeof(void *);
        total = off_table + (2 * B + 1) * (int)sizeof(int);
    }
};
constexpr float kTop = 14.f, kRaise = 4.f;                      // weights for O stay below 2^(kTop + 1) < 65504
constexpr float kMaxK = 92.f;                                   // 2^kMaxK times a row sum of 2^30 keys, each up to 2^kRaise, is finite

struct KvqDecArgs {
    const unsigned char *q;          // bf16 rows [B][Hq][128]
    const void *const *k_caches;
    const void *const *v_caches;
    const int32_t *ctx_len;
    const uint8_t *mask;
    int B, L, layer, Hq, Hkv, G, S, W, layout, max_context;
    float scale_log2;
    float *part_o, *part_ml;         // [CTA + segment][G][128], [..][2]
    uint32_t *tickets;               // [B * Hkv], zero between launches
    int32_t *debug;
    uint32_t *status;
    __nv_bfloat16 *out;
    uint32_t *touch;
    int touch_words;
    int ring;
    const unsigned char *k_new, *v_new;      // rows [B][Hkv][128] of the newest tokens, which this launch stores, or NULL
    int overlap;                     // schedule and copies of all but the newest block before the grid-dependency wait
};

// Strips of a request of n tokens that a decode step reads: [0, e1) and [b2, b2 + count - e1); then the tail, if any.
// appending: the newest token is not in the cache yet; the block it belongs to is the tail, with 1 to 16 rows.
struct Walk {
    int blocks, e1, b2, count, tail;     // blocks: complete ones
    __device__ __forceinline__ Walk(int n, bool fa, int S, int W, bool appending)
    {
        blocks = (appending ? n - 1 : n) / kKvqBlock;
        const int e2 = (blocks + kStripBlocks - 1) / kStripBlocks;
        tail = n - blocks * kKvqBlock;
        if (fa || n <= S + W) {
            e1 = e2;
            b2 = e2;
        } else {
            e1 = min((S + kStrip - 1) / kStrip, e2);
            b2 = max(e1, (n - W) / kStrip);
        }
        count = e1 + max(0, e2 - b2);
    }
    __device__ __forceinline__ int units() const { return count + (tail ? 1 : 0); }
    __device__ __forceinline__ int strip(int x) const { return x < e1 ? x : b2 + x - e1; }
};

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the same with a zero accumulator
__device__ __forceinline__ void mma_f16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&v);
}
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// State of one warp for up to 8 kNT query heads: lane (g, t) holds heads 2 t, 2 t + 1 (+ 8) of rows g of every product.
template <int kNT>
struct State {
    float o[kNT][8][4];              // O^T: channel 32 (mt / 2) + 4 g + 2 (mt & 1) + (c >> 1), head 2 t + (c & 1)
    float m[kNT][2], l[kNT][2];      // this lane's rows: maximum in use, sum of 2^(s - m)
    float lim[kNT][2];               // the same in all lanes of a t: scores up to s + e = lim + kTop can be weighed for O
    __device__ __forceinline__ void reset()
    {
#pragma unroll
        for (int z = 0; z < kNT; ++z) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[z][i][c] = 0.f;
            m[z][0] = m[z][1] = lim[z][0] = lim[z][1] = kNegBig;
            l[z][0] = l[z][1] = 0.f;
        }
    }
    __device__ __forceinline__ float factor(int z, int c) const { return fast_exp2(m[z][c] - lim[z][c]); }         // 2^k
    // Raises the maxima where this unit's largest score (mx: this lane's rows) or largest s + e (my) exceeds what is in use.
    __device__ __forceinline__ void raise(const float (&mx)[kNT][2], const float (&my)[kNT][2])
    {
        bool need = false;
#pragma unroll
        for (int z = 0; z < kNT; ++z)
#pragma unroll
            for (int c = 0; c < 2; ++c) need = need || mx[z][c] > m[z][c] + kRaise || my[z][c] > lim[z][c] + kTop;
        if (!__any_sync(0xffffffffu, need)) return;
#pragma unroll
        for (int z = 0; z < kNT; ++z)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float nm = fmaxf(m[z][c], mx[z][c]);
                l[z][c] *= fast_exp2(m[z][c] - nm);
                m[z][c] = nm;
                float y = fmaxf(my[z][c] - (kTop - kRaise), nm - kMaxK);
                y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 4));
                y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 8));
                y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 16));
                const float nl = fmaxf(lim[z][c], y), alpha = fast_exp2(lim[z][c] - nl);
                lim[z][c] = nl;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    o[z][i][c] *= alpha;
                    o[z][i][c + 2] *= alpha;
                }
            }
    }
};

// One strip (scales beside its codes, or given apart: those of a block that has just been completed).  kFull: both blocks are
// complete and every key is kept.  Else blocks [i0, nb) are complete and held, and keys kept while pos < S or pos >= lo (lo = 0:
// all); the other blocks are left out altogether: they are whatever was in the slot or the cache before, NaN codes among it.
template <int kFmt, int kNT, bool kFull>
__device__ __forceinline__ void attend_strip(State<kNT> &st, const unsigned char *slot, const uint32_t (&qf)[kNT][8][2],
                                             const float (&qs)[kNT][2], int i0, int nb, int pos0, int S, int lo, int lane)
{
    const float2 ks2 = *reinterpret_cast<const float2 *>(slot + kKvqStripCodes);
    const float2 vs2 = *reinterpret_cast<const float2 *>(slot + kSlotV + kKvqStripCodes);
    const float ks[2] = {ks2.x, ks2.y};
    const float vs[2] = {vs2.x, vs2.y};
    const int g = lane >> 2;
    float s[kNT][kStripBlocks][4];
#pragma unroll
    for (int i = 0; i < kStripBlocks; ++i) {
        if (!kFull && (i < i0 || i >= nb)) continue;
        const unsigned char *kb = slot + i * kKvqBlockBytes + lane * 16;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const uint4 r0 = *reinterpret_cast<const uint4 *>(kb + (2 * p) * 512);
            const uint4 r1 = *reinterpret_cast<const uint4 *>(kb + (2 * p + 1) * 512);
            const uint32_t w0[4] = {r0.x, r0.y, r0.z, r0.w}, w1[4] = {r1.x, r1.y, r1.z, r1.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                uint32_t a[4];
                kvq_decode4<kFmt>(w0[u], a[0], a[2]);
                kvq_decode4<kFmt>(w1[u], a[1], a[3]);
#pragma unroll
                for (int z = 0; z < kNT; ++z) {
                    if (p == 0 && u == 0) mma_f16_first(s[z][i], a, qf[z][0][0], qf[z][0][1]);
                    else mma_f16(s[z][i], a, qf[z][4 * p + u][0], qf[z][4 * p + u][1]);
                }
            }
        }
    }
    float mx[kNT][2], my[kNT][2];
#pragma unroll
    for (int z = 0; z < kNT; ++z) mx[z][0] = mx[z][1] = my[z][0] = my[z][1] = -CUDART_INF_F;
    const bool masked = !kFull && lo > 0 && pos0 < lo && pos0 + kStrip > S;      // some position may be outside sink and window
#pragma unroll
    for (int i = 0; i < kStripBlocks; ++i) {
        if (!kFull && (i < i0 || i >= nb)) continue;
        const float e = __uint_as_float(0x4b000000u | (__float_as_uint(vs[i]) >> 23)) - (8388608.f + 127.f);       // its exponent
        bool keep0 = true, keep1 = true;
        if (!kFull && masked) {
            const int p0 = pos0 + i * kKvqBlock + g;
            keep0 = p0 < S || p0 >= lo;
            keep1 = p0 + 8 < S || p0 + 8 >= lo;
        }
#pragma unroll
        for (int z = 0; z < kNT; ++z)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float f = ks[i] * qs[z][c];
                s[z][i][c] *= f;
                s[z][i][c + 2] *= f;
                if (!kFull) {
                    if (!keep0) s[z][i][c] = -CUDART_INF_F;
                    if (!keep1) s[z][i][c + 2] = -CUDART_INF_F;
                }
                const float top = fmaxf(s[z][i][c], s[z][i][c + 2]);
                mx[z][c] = fmaxf(mx[z][c], top);
                my[z][c] = fmaxf(my[z][c], top + e);
            }
    }
    st.raise(mx, my);
    float f2k[kNT][2];
#pragma unroll
    for (int z = 0; z < kNT; ++z) {
        f2k[z][0] = st.factor(z, 0);
        f2k[z][1] = st.factor(z, 1);
    }
#pragma unroll
    for (int i = 0; i < kStripBlocks; ++i) {
        if (!kFull && (i < i0 || i >= nb)) continue;
        uint32_t pb[kNT][2];
#pragma unroll
        for (int z = 0; z < kNT; ++z) {
            float p[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) p[c] = fast_exp2(s[z][i][c] - st.m[z][c & 1]);
            st.l[z][0] += p[0] + p[2];
            st.l[z][1] += p[1] + p[3];
            // scale 2^k held finite: where it would be larger, every p here is 0 or below 2^-112
#pragma unroll
            for (int c = 0; c < 4; ++c) p[c] *= fminf(vs[i] * f2k[z][c & 1], 0x1p127f);
            pb[z][0] = transpose_8x8(pack_f16(p[0], p[1]));
            pb[z][1] = transpose_8x8(pack_f16(p[2], p[3]));
        }
        const unsigned char *vb = slot + kSlotV + i * kKvqBlockBytes + lane * 16;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint4 r = *reinterpret_cast<const uint4 *>(vb + q * 512);
            uint32_t a0[4], a1[4];
            kvq_decode4<kFmt>(r.x, a0[0], a0[2]);
            kvq_decode4<kFmt>(r.y, a0[1], a0[3]);
            kvq_decode4<kFmt>(r.z, a1[0], a1[2]);
            kvq_decode4<kFmt>(r.w, a1[1], a1[3]);
#pragma unroll
            for (int z = 0; z < kNT; ++z) {
                mma_f16(st.o[z][2 * q], a0, pb[z][0], pb[z][1]);
                mma_f16(st.o[z][2 * q + 1], a1, pb[z][0], pb[z][1]);
            }
        }
    }
}

// Query fragments of a segment: lane (g, t) holds channels 64 p + 16 t + 4 u .. + 3 of head g (+ 8) as the B operand of
// product step 4 p + u.  scaled: fp16 after division by the power of two in the row's largest entry, whose factor
// (times scale_log2) comes back for the heads of this lane's columns; else the bf16 bits as they are. Ordinary loads: with launch
// overlap the launch before may write the rows while this kernel is resident, which the read-only path does not allow.
template <int kNT>
__device__ __forceinline__ void load_q(const unsigned char *q, int G, bool scaled, float scale_log2, uint32_t (&qf)[kNT][8][2],
                                       float (&qs)[kNT][2], int lane)
{
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int z = 0; z < kNT; ++z) {
        const bool live = 8 * z + g < G;
        uint32_t w[2][8];
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint4 r = make_uint4(0u, 0u, 0u, 0u);
                if (live) r = *reinterpret_cast<const uint4 *>(q + (size_t)(8 * z + g) * kRowBytes + p * 128 + t * 32 + h * 16);
                w[p][4 * h] = r.x; w[p][4 * h + 1] = r.y; w[p][4 * h + 2] = r.z; w[p][4 * h + 3] = r.w;
            }
        if (scaled) {
            uint32_t top = 0;
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, max(w[p][i] & 0x7fff0000u, (w[p][i] << 16) & 0x7fff0000u));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = min(max((int)(top >> 23), 27), 253);              // 2^(e - 127), within 2^-100 .. 2^126
            const float down = __uint_as_float((uint32_t)(254 - e) << 23);
            const float up = top == 0 ? 1.f : __uint_as_float((uint32_t)e << 23);
#pragma unroll
            for (int c = 0; c < 2; ++c) qs[z][c] = __shfl_sync(0xffffffffu, up, (2 * t + c) * 4) * scale_log2;
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    w[p][i] = pack_f16(__uint_as_float(w[p][i] << 16) * down, __uint_as_float(w[p][i] & 0xffff0000u) * down);
        }
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                qf[z][4 * p + u][0] = w[p][2 * u];
                qf[z][4 * p + u][1] = w[p][2 * u + 1];
            }
    }
}

// The tail: up to 15 bf16 rows, one 16-key product in bf16 on the original query bits.  Rows from `count` on hold older
// or no data: their scores are masked and their V entries cleared.
template <int kNT>
__device__ __forceinline__ void attend_tail(State<kNT> &st, const unsigned char *slot, const unsigned char *q, int G, int count,
                                            int pos0, int S, int lo, float scale_log2, int lane)
{
    const int g = lane >> 2, t = lane & 3;
    uint32_t qf[kNT][8][2];
    float unused[kNT][2];
    load_q<kNT>(q, G, false, 0.f, qf, unused, lane);
    float s[kNT][4];
    float mx[kNT][2];
#pragma unroll
    for (int z = 0; z < kNT; ++z)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[z][c] = 0.f;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        uint32_t w[2][8];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint4 r = *reinterpret_cast<const uint4 *>(slot + (g + 8 * h) * kRowBytes + p * 128 + t * 32 + x * 16);
                w[h][4 * x] = r.x; w[h][4 * x + 1] = r.y; w[h][4 * x + 2] = r.z; w[h][4 * x + 3] = r.w;
            }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t a[4] = {w[0][2 * u], w[1][2 * u], w[0][2 * u + 1], w[1][2 * u + 1]};
#pragma unroll
            for (int z = 0; z < kNT; ++z) mma_bf16(s[z], a, qf[z][4 * p + u][0], qf[z][4 * p + u][1]);
        }
    }
    const bool keep0 = g < count && (pos0 + g < S || pos0 + g >= lo), keep1 = g + 8 < count && (pos0 + g + 8 < S || pos0 + g + 8 >= lo);
#pragma unroll
    for (int z = 0; z < kNT; ++z)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            s[z][c] = keep0 ? s[z][c] * scale_log2 : -CUDART_INF_F;
            s[z][c + 2] = keep1 ? s[z][c + 2] * scale_log2 : -CUDART_INF_F;
            mx[z][c] = fmaxf(s[z][c], s[z][c + 2]);
        }
    st.raise(mx, mx);                        // no scales: e = 0
    uint32_t pb[kNT][2];
#pragma unroll
    for (int z = 0; z < kNT; ++z) {
        float p[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            p[c] = fast_exp2(s[z][c] - st.m[z][c & 1]);
            st.l[z][c & 1] += p[c];
            p[c] *= st.factor(z, c & 1);
        }
        pb[z][0] = transpose_8x8(pack_bf16(p[0], p[1]));
        pb[z][1] = transpose_8x8(pack_bf16(p[2], p[3]));
    }
    const unsigned char *vrow = slot + kSlotV + 8 * g;
#pragma unroll
    for (int qd = 0; qd < 4; ++qd) {
        uint2 x[4];                                  // keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9; channels 32 qd + 4 g .. + 3
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int key = 2 * t + (k & 1) + 8 * (k >> 1);
            x[k] = *reinterpret_cast<const uint2 *>(vrow + key * kRowBytes + qd * 64);
            if (key >= count) x[k] = make_uint2(0u, 0u);
        }
        const uint32_t a0[4] = {__byte_perm(x[0].x, x[1].x, 0x5410), __byte_perm(x[0].x, x[1].x, 0x7632),
                                __byte_perm(x[2].x, x[3].x, 0x5410), __byte_perm(x[2].x, x[3].x, 0x7632)};
        const uint32_t a1[4] = {__byte_perm(x[0].y, x[1].y, 0x5410), __byte_perm(x[0].y, x[1].y, 0x7632),
                                __byte_perm(x[2].y, x[3].y, 0x5410), __byte_perm(x[2].y, x[3].y, 0x7632)};
#pragma unroll
        for (int z = 0; z < kNT; ++z) {
            mma_bf16(st.o[z][2 * qd], a0, pb[z][0], pb[z][1]);
            mma_bf16(st.o[z][2 * qd + 1], a1, pb[z][0], pb[z][1]);
        }
    }
}

// The newest token of (request, head) joins its block, whose earlier rows the slot's half holds (K or V tail): its row goes to the
// slot and to the cache's tail; when it completes the block (rows == 16) the block's codes and scale go to its tile and, in the
// same order, to the start of the half, so that the query meets the values every later step will read.  y: this lane's part of the
// row, finite.  (Not inlined, and with scalars for arguments: its rows would push the attention state out of registers.  Rolled
// loops: the code runs once per launch, so fetching it is most of what it costs.)
template <int kFmt>
__device__ __noinline__ void append_token(unsigned char *half, float *slot_scale, uint2 y, unsigned char *tail, unsigned char *blk, float *scale,
                                          int kv, int rows)
{
    const int lane = threadIdx.x & 31;
    *reinterpret_cast<uint2 *>(tail + (rows - 1) * kRowBytes + lane * 8) = y;
    unsigned char *mine = half + lane * 8;               // this lane's four channels of row i: mine + 256 i
    *reinterpret_cast<uint2 *>(mine + (rows - 1) * kRowBytes) = y;
    if (rows == kKvqBlock) {
        uint32_t two = 0;
#pragma unroll 4
        for (int i = 0; i < kKvqBlock; ++i) {
            const uint2 x = *reinterpret_cast<const uint2 *>(mine + i * kRowBytes);
            two = __vmaxu2(two, __vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu));
        }
        const uint32_t top = __reduce_max_sync(0xffffffffu, max(two & 0xffffu, two >> 16));
        const float s = kvq_scale<kFmt>(__uint_as_float(top << 16)), inv = __fdiv_rn(1.f, s);
#pragma unroll 2
        for (int i = 0; i < kKvqBlock; ++i) {
            const uint2 x = *reinterpret_cast<const uint2 *>(mine + i * kRowBytes);
            *reinterpret_cast<uint32_t *>(mine + i * kRowBytes) = kvq_encode4<kFmt>(x.x, x.y, s, inv);
        }
        uint32_t w[kKvqBlock];
#pragma unroll
        for (int i = 0; i < kKvqBlock; ++i) w[i] = *reinterpret_cast<const uint32_t *>(mine + i * kRowBytes);
        __syncwarp();                                    // every lane has its rows before the codes, in their order, overwrite them
        kvq_put_block(half, w, kv, lane);
        kvq_put_block(blk, w, kv, lane);
        if (lane == 0) *slot_scale = *scale = s;
    }
    __syncwarp();
}

// The row sums in O's units, summed over the eight lanes of a t: afterwards each of them has the sum.
template <int kNT>
__device__ __forceinline__ void reduce_l(State<kNT> &st)
{
#pragma unroll
    for (int z = 0; z < kNT; ++z)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float l = st.l[z][c] * st.factor(z, c);
            l += __shfl_xor_sync(0xffffffffu, l, 4);
            l += __shfl_xor_sync(0xffffffffu, l, 8);
            l += __shfl_xor_sync(0xffffffffu, l, 16);
            st.l[z][c] = l;
        }
}

// A whole segment in one warp: its output rows.
template <int kNT>
__device__ __forceinline__ void write_rows(State<kNT> &st, __nv_bfloat16 *orow, int G, int lane)
{
    reduce_l<kNT>(st);
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int z = 0; z < kNT; ++z)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int hd = 8 * z + 2 * t + c;
            if (hd >= G) continue;
            const float inv = 1.f / st.l[z][c];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<uint2 *>(orow + (size_t)hd * kHeadDim + 32 * q + 4 * g) =
                    make_uint2(pack_bf16(st.o[z][2 * q][c] * inv, st.o[z][2 * q][c + 2] * inv),
                               pack_bf16(st.o[z][2 * q + 1][c] * inv, st.o[z][2 * q + 1][c + 2] * inv));
        }
}

// A piece of a segment to shared memory.
template <int kNT>
__device__ __forceinline__ void write_piece(State<kNT> &st, float *dst, int G, int lane)
{
    reduce_l<kNT>(st);
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int z = 0; z < kNT; ++z)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int hd = 8 * z + 2 * t + c;
            if (hd >= G) continue;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<float4 *>(dst + hd * kRowFloats + 32 * q + 4 * g) =
                    make_float4(st.o[z][2 * q][c], st.o[z][2 * q][c + 2], st.o[z][2 * q + 1][c], st.o[z][2 * q + 1][c + 2]);
            if (g == 0) *reinterpret_cast<float2 *>(dst + G * kRowFloats + 2 * hd) = make_float2(st.lim[z][c], st.l[z][c]);
        }
}

// Running merge of rows: (lim, l, four channels of this lane).  Pieces' units may be further apart than fp32 reaches (where V's scales
// are): a factor is the square of ho / hn, so that a large row sum in small units keeps its part, while the O that goes with it may vanish.
struct Row {
    float m = kNegBig, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    __device__ __forceinline__ void add(const float2 ml, const float4 v)
    {
        const float nm = fmaxf(m, ml.x), ho = fast_exp2(0.5f * (m - nm)), hn = fast_exp2(0.5f * (ml.x - nm)), fo = ho * ho, fn = hn * hn;
        o.x = fmaf(v.x, fn, o.x * fo);
        o.y = fmaf(v.y, fn, o.y * fo);
        o.z = fmaf(v.z, fn, o.z * fo);
        o.w = fmaf(v.w, fn, o.w * fo);
        l = fmaf(ml.y * hn, hn, l * ho * ho);
        m = nm;
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *dst) const
    {
        const float inv = 1.f / l;
        *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    }
};

template <int kFmt, int kNT>
__global__ void __launch_bounds__((kCons + kProd) * 32, 1) decode_kvq_kernel(KvqDecArgs a)
{
    extern __shared__ __align__(128) unsigned char smem[];
    const Smem lay(a.ring, a.G, a.B);
    const int n_slots = kCons * a.ring;
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + lay.off_flags);
    volatile int *last_flag = abort_flag + 1;                    // [2]
    int2 *desc = reinterpret_cast<int2 *>(smem + lay.off_desc);  // pieces in unit order: segment (-1: none), bit 0 begins it, bit 1 ends it
    const unsigned char **caches = reinterpret_cast<const unsigned char **>(smem + lay.off_caches);   // K, V of request b
    int *prefix = reinterpret_cast<int *>(smem + lay.off_table); // places before request b
    int *n_mode = prefix + a.B + 1;                              // length, sign bit set for sparse
    const uint32_t bars = smem_u32(smem + lay.off_bars), slots = smem_u32(smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool appending = a.k_new != nullptr;

    if (tid == 0) {
        *abort_flag = 0;
        for (int i = 0; i < 2 * n_slots; ++i) mbar_init(bars + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    // Everything the launches before wrote is visible after the wait.  In overlap mode it comes later: each warp below waits before
    // it reads what the caller has not promised to be settled, or writes anything.
    // The next launch may start early once every CTA has been through its wait: not before, since it may then read what
    // the launches before this one wrote.
    auto wait = [] { asm volatile("griddepcontrol.wait;\n" ::: "memory"); };
    auto release = [] { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); };
    if (!a.overlap) {
        wait();
        release();
    }

    // Places of a segment of request b (n > 0): 0 stands for its start, 1 .. count are the strips, the last one is the tail, if any;
    // a launch that stores the newest token has kAppendCost empty places before it.
    auto cost_of = [&](int b) {
        const int nm = n_mode[b];
        return 1 + Walk(nm & 0x7fffffff, nm >= 0, a.S, a.W, appending).units() + (appending ? kAppendCost : 0);
    };

    // ---- schedule: the producer warps take 32 requests each, then one warp adds up ----------------------
    uint32_t flags = 0;
    if (warp >= kCons) {
        for (int b = (warp - kCons) * 32 + lane; b < a.B; b += kProd * 32) {
            const int n_raw = a.ctx_len[b], mode = a.mask[(size_t)b * a.L + a.layer];
            const uintptr_t kc = (uintptr_t)a.k_caches[b], vc = (uintptr_t)a.v_caches[b];
            int n = max(n_raw, 0);
            if (mode > 1) flags |= FLUX_STATUS_BAD_MASK;
            if (n > a.max_context) {
                flags |= FLUX_STATUS_BAD_LENGTH;
                n = 0;           // its cache cannot hold that many: a zero row instead of a read past its end
            }
            if (n > 0 && (kc == 0 || vc == 0 || ((kc | vc) & 15u) != 0)) {
                flags |= FLUX_STATUS_BAD_POINTER;
                n = 0;
            }
            caches[2 * b] = (const unsigned char *)kc;
            caches[2 * b + 1] = (const unsigned char *)vc;
            n_mode[b] = mode != 0 ? n : (int)((uint32_t)n | 0x80000000u);
            prefix[b + 1] = n > 0 ? cost_of(b) * a.Hkv : 0;
        }
    }
    __syncthreads();
    if (warp == kCons) {
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
    __syncthreads();
    const int total = prefix[a.B];
    // dispatch records, status bits, zero rows of inactive requests
    if (blockIdx.x == 0 && warp >= kCons) {
        wait();
        if (flags != 0) atomicOr(a.status, flags);
        for (int b = tid - kCons * 32; b < a.B; b += kProd * 32) {
            const int nm = n_mode[b], n = nm & 0x7fffffff;
            const bool two = nm < 0 && n > a.S + a.W;
            int32_t *d = a.debug + (size_t)b * 8;
            d[0] = nm < 0 ? 0 : 1; d[1] = a.layer; d[2] = b; d[3] = n;
            d[4] = 0; d[5] = two ? a.S : n; d[6] = two ? n - a.W : 0; d[7] = two ? n : 0;
        }
    }
    if (warp < kCons)
        for (int b = blockIdx.x; b < a.B; b += gridDim.x)
            if (prefix[b + 1] == prefix[b]) {
                wait();
                for (int i = tid; i < a.Hq * (kRowBytes / 16); i += kCons * 32)
                    reinterpret_cast<uint4 *>(a.out + (size_t)b * a.Hq * kHeadDim)[i] = make_uint4(0u, 0u, 0u, 0u);
            }
    if (total == 0) return;
    // Equal ranges, of at least one place per warp.  A range does not end inside a short segment: below kShortSpan the whole
    // segment costs a CTA no more time than merging across CTAs would, above it the ranges may differ by an eighth.
    const int span = max((total + (int)gridDim.x - 1) / (int)gridDim.x, kCons);
    const int keep = span <= kShortSpan ? kShortSpan : span / 8;
    auto bound = [&](int k) {
        const int v = min(k * span, total);
        if (v == total) return v;
        const Place p(prefix, a.B, v, cost_of);
        return p.cost <= keep ? v - p.x : v;
    };
    if ((int64_t)blockIdx.x * span >= total) return;
    const int c_begin = bound((int)blockIdx.x), c_end = bound((int)blockIdx.x + 1);
    if (c_begin >= c_end) return;

    if (warp >= kCons) {
        // ================= producers =================
        if (kNT > 1) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kProducerRegs));
        constexpr int kPer = kCons / kProd;
        static_assert(kPer == 2, "two consumers per producer");
        const size_t stride = kvq_tile_stride(a.Hkv);
        const int ring_end = kvq_sink_tiles(a.S) + kvq_ring_tiles(a.W);
        // What one consumer is to get next.  The strip's place in the cache is carried along: the next strip of a tile follows it,
        // the next tile is a stride away, a compact cache wraps at the end of its ring.
        struct Feed {
            Place p;
            int v, end, use, slot;       // place, end of the consumer's range, rounds of the ring so far, next slot of the ring
            int count, tail, e1, b2, strip, tile, n;     // of the segment; strip at place p.x and the slot of its tile
            bool compact;
            const unsigned char *kc, *vc;
            size_t at;
            __device__ __forceinline__ Feed(const Place &p_) : p(p_) {}
        };
        auto seek = [&](Feed &f) {       // a new strip, not the one after the last
            f.tile = kvq_slot(f.strip / 2, f.compact, a.S, a.W);
            f.at = kvq_tail_bytes(a.Hkv) + (size_t)f.tile * stride + (size_t)(2 * f.p.head + (f.strip & 1)) * kKvqStripBytes;
        };
        auto enter = [&](Feed &f) {      // the segment that place p is in
            const int nm = n_mode[f.p.b];
            f.n = nm & 0x7fffffff;
            const Walk wk(f.n, nm >= 0, a.S, a.W, appending);
            f.compact = a.layout == FLUX_KV_COMPACT_SA && nm < 0;
            f.count = wk.count;
            f.tail = wk.tail;
            f.e1 = wk.e1;
            f.b2 = wk.b2;
            f.strip = wk.strip(max(f.p.x, 1) - 1);
            f.kc = caches[2 * f.p.b];
            f.vc = caches[2 * f.p.b + 1];
            seek(f);
        };
        auto cut = [&](int c) { return c_begin + (int)((int64_t)(c_end - c_begin) * ((warp - kCons) * kPer + c) / kCons); };      // c_end may be the end of all
        Feed feeds[kPer] = {Place(prefix, a.B, min(cut(0), c_end - 1), cost_of), Place(prefix, a.B, min(cut(1), c_end - 1), cost_of)};
#pragma unroll
        for (int c = 0; c < kPer; ++c) {
            Feed &f = feeds[c];
            f.v = cut(c);
            f.end = cut(c + 1);
            f.use = f.slot = 0;
            enter(f);
        }
        bool ok = true, waited = a.overlap == 0;
        while (ok && (feeds[0].v < feeds[0].end || feeds[1].v < feeds[1].end)) {
#pragma unroll
            for (int c = 0; c < kPer; ++c) {
                Feed &f = feeds[c];
                if (!ok || f.v >= f.end) continue;
                const bool is_strip = f.p.x > 0 && f.p.x <= f.count;
                if (is_strip || f.p.x == f.p.cost - 1) {
                    const int s = ((warp - kCons) * kPer + c) * a.ring + f.slot;
                    ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * (n_slots + s), (uint32_t)((f.use & 1) ^ 1), abort_flag, a.status));
                    if (!ok) continue;
                    const uint32_t dst = slots + s * kSlotBytes, bar = bars + 8 * s;
                    // the newest two tokens' blocks: the tail, and the last block if it has been completed by one of them
                    if (!waited && (!is_strip || (f.tail <= 1 && f.p.x == f.count))) {
                        wait();
                        waited = true;
                    }
                    const size_t at = is_strip ? f.at : (size_t)f.p.head * kKvqTailHeadBytes;
                    const uint32_t bytes = is_strip ? kKvqStripBytes : kKvqTailHeadBytes;
                    if (elect_one()) {
                        mbar_expect_tx(bar, 2 * bytes);
                        bulk_copy(dst, f.kc + at, bytes, bar);
                        bulk_copy(dst + kSlotV, f.vc + at, bytes, bar);
                    }
                    if (a.touch != nullptr && f.p.head == 0 && lane == 0) {         // debug: the positions the unit holds
                        const int blocks = (appending ? f.n - 1 : f.n) / kKvqBlock, first = blocks * kKvqBlock;
                        uint32_t *words = a.touch + (size_t)f.p.b * a.touch_words;
                        if (is_strip) atomicOr(words + f.strip, blocks > kStripBlocks * f.strip + 1 ? 0xffffffffu : 0xffffu);
                        else atomicOr(words + (first >> 5), ((1u << f.tail) - 1u) << (first & 31));
                    }
                    if (++f.slot == a.ring) {
                        f.slot = 0;
                        ++f.use;
                    }
                    if (is_strip) {
                        if (++f.strip == f.e1) {                 // from the sink to the window
                            f.strip = f.b2;
                            seek(f);
                        } else if (f.strip & 1) {
                            f.at += kKvqStripBytes;
                        } else {
                            f.at += stride - kKvqStripBytes;
                            if (++f.tile == ring_end && f.compact) {
                                f.tile = kvq_sink_tiles(a.S);
                                f.at -= (size_t)kvq_ring_tiles(a.W) * stride;
                            }
                        }
                    }
                }
                if (++f.v < f.end && ++f.p.x == f.p.cost) {
                    f.p.next_segment(prefix, a.Hkv, cost_of);
                    enter(f);
                }
            }
        }
        if (*abort_flag) {       // a wait gave up: let the copies in flight land before the shared memory goes away
#pragma unroll
            for (int c = 0; c < kPer; ++c)
                for (int s = 0; s < a.ring; ++s) {
                    const int uses = feeds[c].use + (s < feeds[c].slot ? 1 : 0);      // of slot s
                    const uint32_t bar = bars + 8 * (((warp - kCons) * kPer + c) * a.ring + s);
                    for (int z = 0; uses > 0 && z < 200 && !mbar_try(bar, (uint32_t)((uses - 1) & 1)); ++z) __nanosleep(1000);
                }
        }
        return;
    }

    // ================= consumers =================
    if (kNT > 1) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kConsumerRegs));
    State<kNT> st;
    uint32_t qf[kNT][8][2];
    float qs[kNT][2];
    const int v_begin = c_begin + (int)((int64_t)(c_end - c_begin) * warp / kCons);
    const int v_end = c_begin + (int)((int64_t)(c_end - c_begin) * (warp + 1) / kCons);
    int d_first = -1, d_last = -1, f_first = 0, f_last = 0;      // this warp's pieces: segment, flags
    if (a.overlap) {
        wait();                          // query rows, and everything written from here on
        release();
    }
    if (v_begin < v_end) {
        Place p(prefix, a.B, v_begin, cost_of);
        int v = v_begin, slot = 0, use = 0;
        bool ok = true;
        for (;;) {
            const int nm = n_mode[p.b], n = nm & 0x7fffffff;
            const bool fa = nm >= 0;
            const Walk wk(n, fa, a.S, a.W, appending);
            const int S = a.S, lo = fa || n <= a.S + a.W ? 0 : n - a.W;
            const int x_end = min(p.cost, p.x + (v_end - v));    // this warp's places of the segment: [p.x, x_end)
            const int x0 = max(p.x, 1), x1 = min(wk.count + 1, x_end), n_strips = max(x1 - x0, 0);
            const bool has_tail = wk.tail > 0 && x_end == p.cost;
            v += p.cost - p.x;
            if (n_strips > 0 || has_tail) {
                const unsigned char *q = a.q + ((size_t)p.b * a.Hq + (size_t)p.head * a.G) * kRowBytes;
                st.reset();
                load_q<kNT>(q, a.G, true, a.scale_log2, qf, qs, lane);
                int strip = wk.strip(x0 - 1);
                for (int i = 0; i < n_strips + (has_tail ? 1 : 0); ++i) {
                    const int s = warp * a.ring + slot;
                    uint2 fresh[2];                      // this lane's part of the newest token's rows, asked for ahead of the wait
                    if (appending && i == n_strips) {
                        const size_t row = ((size_t)p.b * a.Hkv + p.head) * kRowBytes + lane * 8;
                        fresh[0] = *reinterpret_cast<const uint2 *>(a.k_new + row);
                        fresh[1] = *reinterpret_cast<const uint2 *>(a.v_new + row);
                    }
                    if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * s, (uint32_t)(use & 1), abort_flag, a.status));
                    if (ok) {
                        unsigned char *data = smem + s * kSlotBytes;
                        if (i < n_strips) {
                            const int pos0 = strip * kStrip, nb = wk.blocks - kStripBlocks * strip;
                            if (nb >= kStripBlocks && (pos0 >= lo || pos0 + kStrip <= S))
                                attend_strip<kFmt, kNT, true>(st, data, qf, qs, 0, kStripBlocks, pos0, S, lo, lane);
                            else     // behind the sink, blocks that end before the window may never have been written (kvq_held)
                                attend_strip<kFmt, kNT, false>(st, data, qf, qs, pos0 < S ? 0 : max(0, (lo - pos0) / kKvqBlock), min(kStripBlocks, nb), pos0, S,
                                                               lo, lane);
                            if (++strip == wk.e1) strip = wk.b2;
                        } else {
                            if (appending) {
                                const size_t strip_at = kvq_tail_bytes(a.Hkv) + kvq_strip_at(p.head, wk.blocks) + kvq_tile_stride(a.Hkv) *
                                                        (size_t)kvq_slot(wk.blocks / 4, a.layout == FLUX_KV_COMPACT_SA && !fa, a.S, a.W);
                                const int j = wk.blocks & 1;
                                bool bad = false;
#pragma unroll
                                for (int kv = 0; kv < 2; ++kv) {
                                    unsigned char *cache = const_cast<unsigned char *>(caches[2 * p.b + kv]);
                                    fresh[kv].x = kvq_finite2(fresh[kv].x, bad);
                                    fresh[kv].y = kvq_finite2(fresh[kv].y, bad);
                                    append_token<kFmt>(data + kv * kSlotV, reinterpret_cast<float *>(data + kv * kSlotV + kKvqStripCodes), fresh[kv],
                                                       cache + (size_t)p.head * kKvqTailHeadBytes, cache + strip_at + j * kKvqBlockBytes,
                                                       reinterpret_cast<float *>(cache + strip_at + kKvqStripCodes + 4 * j), kv, wk.tail);
                                }
                                if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(a.status, FLUX_STATUS_NONFINITE);
                            }
                            if (wk.tail == kKvqBlock)
                                attend_strip<kFmt, kNT, false>(st, data, qf, qs, 0, 1, wk.blocks * kKvqBlock, S, lo, lane);
                            else
                                attend_tail<kNT>(st, data, q, a.G, wk.tail, n - wk.tail, S, lo, a.scale_log2, lane);
                            if (appending) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the slot was written; the next copy into it must come after
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bars + 8 * (n_slots + s));
                    }
                    if (++slot == a.ring) {
                        slot = 0;
                        ++use;
                    }
                }
                const bool begins = n_strips > 0 ? x0 == 1 : wk.count == 0, ends = x_end == p.cost;
                const int seg = p.b * a.Hkv + p.head;
                if (begins && ends) {
                    write_rows<kNT>(st, a.out + ((size_t)p.b * a.Hq + (size_t)p.head * a.G) * kHeadDim, a.G, lane);
                } else if (ends) {
                    write_piece<kNT>(st, reinterpret_cast<float *>(smem + lay.off_piece + warp * lay.piece_bytes), a.G, lane);
                    d_first = seg;
                    f_first = 2;
                } else {
                    d_last = seg;        // the warp's last segment: its piece goes over the warp's own ring, which has been used up
                    f_last = begins ? 1 : 0;
                }
            }
            if (v >= v_end) break;
            p.next_segment(prefix, a.Hkv, cost_of);
        }
        if (d_last >= 0) {
            __syncwarp();
            write_piece<kNT>(st, reinterpret_cast<float *>(smem + warp * a.ring * kSlotBytes), a.G, lane);
        }
    }
    if (lane == 0) {
        desc[2 * warp] = make_int2(d_first, f_first);
        desc[2 * warp + 1] = make_int2(d_last, f_last);
    }
    consumers_sync();

    // ---- segments that this CTA's warps share -------------------------------------------------------
    // Pieces of one segment are neighbours in `desc` (empty entries aside).  Groups are numbered in order; (group, head) rows
    // are dealt to the warps, four channels to a lane.
    int shared_seg[2] = {-1, -1};        // segments that go on in other CTAs: at most the range's first and last
    int group = 0, n_shared = 0;
    const int2 mine = lane < 2 * kCons ? desc[lane] : make_int2(-1, 0);
    for (uint32_t left = __ballot_sync(0xffffffffu, mine.x >= 0); left != 0; ++group) {
        const int seg = __shfl_sync(0xffffffffu, mine.x, __ffs(left) - 1);
        const uint32_t pieces = __ballot_sync(0xffffffffu, mine.x == seg);
        const bool whole = __any_sync(0xffffffffu, mine.x == seg && (mine.y & 1)) && __any_sync(0xffffffffu, mine.x == seg && (mine.y & 2));
        left &= ~pieces;
        if (!whole) {
            if (n_shared == 0) shared_seg[0] = seg; else shared_seg[1] = seg;
            ++n_shared;
        }
        for (int hd = (warp - group * a.G % kCons + kCons) % kCons; hd < a.G; hd += kCons) {
            Row r;
            for (uint32_t todo = pieces; todo != 0; todo &= todo - 1) {
                const int j = __ffs(todo) - 1;
                const float *src = reinterpret_cast<const float *>(j & 1 ? smem + (j >> 1) * a.ring * kSlotBytes
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
    consumers_sync();
    auto parts_of = [&](int seg, int &c_first) {         // CTAs that hold units of a segment longer than `keep` (a range is longer than the empty places)
        static_assert(kAppendCost < kCons, "a CTA's range holds a unit of every segment it meets beyond place 0");
        const int sb = seg / a.Hkv, cost = (prefix[sb + 1] - prefix[sb]) / a.Hkv, begin = prefix[sb] + (seg % a.Hkv) * cost;
        c_first = (begin + 1) / span;
        return (begin + cost - 1) / span - c_first + 1;
    };
    if (tid < n_shared) {
        int c_first;
        const int seg = tid == 0 ? shared_seg[0] : shared_seg[1], n_part = parts_of(seg, c_first);
        unsigned seen;
        asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(seen) : "l"(a.tickets + seg) : "memory");
        last_flag[tid] = seen == (unsigned)(n_part - 1);
        if (seen == (unsigned)(n_part - 1)) a.tickets[seg] = 0u;      // ready for the next launch
    }
    consumers_sync();
    for (int i = 0; i < n_shared; ++i) {
        if (!last_flag[i]) continue;
        int c_first;
        const int seg = i == 0 ? shared_seg[0] : shared_seg[1], n_part = parts_of(seg, c_first);
        // All partials of the segment (neighbours in the workspace: entry (CTA + segment) G + head) come into the ring, which is idle
        // by now, in one round of asynchronous copies: one trip to L2 instead of one per 16 partials (7 us at 37 x 7 rows).
        const int fit = min(n_slots * kSlotBytes / (a.G * kRowBytes * 2), kMaxParts);
        const float *src = a.part_o + ((size_t)c_first + seg) * a.G * kHeadDim;
        const float *src_ml = a.part_ml + ((size_t)c_first + seg) * a.G * 2;
        Row rows[kNT];                                   // heads warp, warp + 8
        for (int p0 = 0; p0 < n_part; p0 += fit) {
            const int np = min(fit, n_part - p0);
            consumers_sync();                            // the ring's last readers (pieces, the round before) are done
            for (int z = tid; z < np * a.G * 32; z += kCons * 32) cp_async16(slots + z * 16, src + (size_t)p0 * a.G * kHeadDim + (size_t)z * 4, 16);
            cp_async_commit();
            // meanwhile the weights, a lane per partial
            float w[kNT][kMaxParts / 32];
#pragma unroll
            for (int y = 0; y < kNT; ++y) {
                const int hd = warp + kCons * y;
                float nm = rows[y].m;
                float2 ml[kMaxParts / 32];
#pragma unroll
                for (int z = 0; z < kMaxParts / 32; ++z) {
                    ml[z] = make_float2(kNegBig, 0.f);
                    if (hd < a.G && 32 * z + lane < np) ml[z] = __ldcg(reinterpret_cast<const float2 *>(src_ml + ((size_t)(p0 + 32 * z + lane) * a.G + hd) * 2));
                    nm = fmaxf(nm, ml[z].x);
                }
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) nm = fmaxf(nm, __shfl_xor_sync(0xffffffffu, nm, d));
                float l = 0.f;
#pragma unroll
                for (int z = 0; z < kMaxParts / 32; ++z) {
                    const float h = fast_exp2(0.5f * (ml[z].x - nm));        // as in Row::add
                    w[y][z] = h * h;
                    l = fmaf(ml[z].y * h, h, l);
                }
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
                const float ho = fast_exp2(0.5f * (rows[y].m - nm)), fo = ho * ho;
                rows[y].l = fmaf(rows[y].l * ho, ho, l);
                rows[y].m = nm;
                rows[y].o.x *= fo; rows[y].o.y *= fo; rows[y].o.z *= fo; rows[y].o.w *= fo;
            }
            cp_async_wait<0>();
            consumers_sync();
#pragma unroll
            for (int y = 0; y < kNT; ++y) {
                const int hd = warp + kCons * y;
                if (hd >= a.G) continue;
#pragma unroll
                for (int z = 0; z < kMaxParts / 32; ++z)
#pragma unroll 4
                    for (int x = 0; x < min(32, np - 32 * z); ++x) {
                        const float f = __shfl_sync(0xffffffffu, w[y][z], x);
                        const float4 v = *reinterpret_cast<const float4 *>(smem + ((size_t)(32 * z + x) * a.G + hd) * kRowBytes * 2 + lane * 16);
                        rows[y].o.x = fmaf(v.x, f, rows[y].o.x);
                        rows[y].o.y = fmaf(v.y, f, rows[y].o.y);
                        rows[y].o.z = fmaf(v.z, f, rows[y].o.z);
                        rows[y].o.w = fmaf(v.w, f, rows[y].o.w);
                    }
            }
        }
#pragma unroll
        for (int y = 0; y < kNT; ++y)
            if (warp + kCons * y < a.G)
                rows[y].store(a.out + ((size_t)(seg / a.Hkv) * a.Hq + (size_t)(seg % a.Hkv) * a.G + warp + kCons * y) * kHeadDim + 4 * lane);
    }
}

using KvqDecFn = void (*)(KvqDecArgs);
KvqDecFn pick(int fmt, int G)
{
    if (fmt == FLUX_KVQ_E4M3) return G <= 8 ? decode_kvq_kernel<FLUX_KVQ_E4M3, 1> : decode_kvq_kernel<FLUX_KVQ_E4M3, 2>;
    return G <= 8 ? decode_kvq_kernel<FLUX_KVQ_INT8, 1> : decode_kvq_kernel<FLUX_KVQ_INT8, 2>;
}
// Three slots per warp where they fit beside the pieces and the tables, else two.
int ring_for(int smem, int G, int B) { return Smem(kMaxRing, G, B).total <= smem ? kMaxRing : kMaxRing - 1; }

}  // namespace

int decode_kvq_setup(flux_plan *p)
{
    if (p->dev.smem_optin < Smem(2, 16, kMaxBatch).total)
        return fail(FLUX_E_CUDA, "device offers %d bytes of shared memory per block, the 8-bit decode needs %d", p->dev.smem_optin,
                    Smem(2, 16, kMaxBatch).total);
    for (int fmt = FLUX_KVQ_E4M3; fmt <= FLUX_KVQ_INT8; ++fmt)
        for (int G = 8; G <= 16; G += 8) {
            int rc = check_cuda(cudaFuncSetAttribute((const void *)pick(fmt, G), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                     p->dev.smem_optin),
                                "cudaFuncSetAttribute(decode_kvq_kernel)");
            if (rc) return rc;
            cudaFuncAttributes fa;
            rc = check_cuda(cudaFuncGetAttributes(&fa, (const void *)pick(fmt, G)), "cudaFuncGetAttributes(decode_kvq_kernel)");
            if (rc) return rc;
            if (G > 8 && fa.numRegs * (kCons + kProd) < kCons * kConsumerRegs + kProd * kProducerRegs)
                return fail(FLUX_E_CUDA, "8-bit decode kernel was built with %d registers per thread: too few for its register rebalancing",
                            fa.numRegs);
        }
    return FLUX_OK;
}

int launch_decode_kvq(flux_plan *p, int layer, int B, int fmt, const void *q, const void *const *k_caches, const void *const *v_caches,
                      const int32_t *ctx_len, void *out, cudaStream_t st, const void *k_new, const void *v_new)
{
    const flux_config &c = p->cfg;
    // the kernel numbers the places of all requests in 32 bits
    if ((int64_t)B * c.n_kv_heads * (c.max_context / kStrip + 2 + kAppendCost + 1) >= (1ll << 30))
        return fail(FLUX_E_CAPACITY, "%d requests of %d KV heads and up to %d positions are too many for one call", B, c.n_kv_heads, c.max_context);
    char *ws = (char *)p->ws;
    KvqDecArgs a;
    a.k_new = (const unsigned char *)k_new;
    a.v_new = (const unsigned char *)v_new;
    a.q = (const unsigned char *)q;
    a.k_caches = k_caches; a.v_caches = v_caches; a.ctx_len = ctx_len;
    a.mask = p->d_mask;
    a.B = B; a.L = c.n_layers; a.layer = layer; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = p->G;
    a.S = c.sink; a.W = c.window; a.layout = c.kv_layout; a.max_context = c.max_context;
    a.scale_log2 = p->scale_log2;
    a.part_o = (float *)(ws + p->lay.part_o);
    a.part_ml = (float *)(ws + p->lay.part_ml);
    a.tickets = (uint32_t *)(ws + p->lay.kvq_tickets);
    a.debug = (int32_t *)(ws + p->lay.debug);
    a.status = (uint32_t *)(ws + p->lay.status);
    a.out = (__nv_bfloat16 *)out;
    a.touch = p->touch;
    a.touch_words = p->touch_words;
    a.overlap = p->launch_overlap;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)p->dec_ctas);
    lc.blockDim = dim3((kCons + kProd) * 32);
    a.ring = ring_for(p->dev.smem_optin, p->G, B);
    lc.dynamicSmemBytes = Smem(a.ring, p->G, B).total;
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    const int rec = prof_begin(p, FLUX_KERNEL_DECODE, st);
    cudaError_t e = cudaLaunchKernelEx(&lc, pick(fmt, p->G), a);
    prof_end(p, rec, st);
    p->launches++;
    p->debug_records = B;
    return check_cuda(e, "8-bit decode kernel launch");
}

}  // namespace flux
