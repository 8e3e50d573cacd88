// Causal prefill of one routed layer on the sm_100a tensor cores (tcgen05 + TMEM + TMA).
//
// One CTA serves two query tiles at once: the same 128 query rows of two query
// heads that share a KV head (GQA) -- or, for a head left over by an odd group size (and
// for plain multi-head attention), two consecutive row tiles of one head -- so every
// K / V tile fetched by TMA feeds four MMAs.  Roles (warp-specialised, three warpgroups):
//   warps 0-3   softmax of query tile 0 (one thread per query row, TMEM lane = row)
//   warps 4-7   softmax of query tile 1
//   warp  8     TMA producer: Q once, then K_j, V_j through a ring of shared-memory slots
//   warp  9     MMA issuer: S = Q K^T (operands in shared memory), O += P V (P in TMEM)
//   warps 10-11 idle (they complete the third warpgroup, whose registers go to the softmax)
// Registers are rebalanced per warpgroup (setmaxnreg works on whole warpgroups and inside
// the CTA's own allocation): the third warpgroup shrinks to kOtherRegs, the two softmax
// warpgroups grow to kSoftmaxRegs; the host checks that the CTA's allocation covers that.
// TMEM (512 columns): S0 | S1 | O0 | O1, 128 fp32 columns each; P (bf16) overwrites the
// first 64 columns of its S.  The tensor pipe alternates between the two tiles, so the
// softmax of one tile overlaps the MMAs of the other.  Softmax is the online form in
// fp32 in the log2 domain; the running maximum is only raised when a tile exceeds it by
// more than 2^8 (the accumulator and the row sum stay consistent with the maximum in
// use, so the result is the same softmax), which makes rescaling O in TMEM rare.
// P is handed to the MMA issuer in two halves of 64 keys, so the first half of PV overlaps
// the exponentials of the second.
// An FA layer (Eq. 1) walks every KV tile up to the diagonal; an SA layer (Eq. 2 with the
// streaming subset) walks the sink tiles and the window tiles only.
//
// Packed prompts (flux_attn_prefill_packed) run on the same roles with another source of work: the query
// tiles of up to kPackReqs requests of different lengths and modes.  How long an item takes depends on its
// request's routing bit, which only the device knows, so items are handed out at run time, longest first:
// warp 10 draws the next number from a counter in the workspace, finds the item of that rank in the order of
// weights (key tiles) and passes it to the other roles through a two-entry ring.
// A request with few rows and many keys would leave most SMs idle: its items are cut along the keys into parts
// (entries of their own in the table of requests), whose accumulators go to the workspace, and the CTA that
// finishes an item's last part adds them up (split_epilogue).
//
// Every mbarrier wait is bounded: when it runs out the CTA raises
// FLUX_STATUS_WAIT_EXPIRED, stops issuing work, lets in-flight copies land, frees its
// TMEM and returns; CTAs that start after that return at once.
#include <cuda.h>
#include <limits.h>

#include "flux_internal.h"
#include "flux_tc_util.h"

namespace flux {
namespace {

using namespace tc;

constexpr int BM = 128, BN = 128;
constexpr int kHalfBytes = BM * 128;              // 128 rows x 64 bf16 (one 128-byte swizzle span per row)
constexpr int kTileBytes = 2 * kHalfBytes;        // a 128 x 128 bf16 tile = two halves (d 0-63 | d 64-127)
constexpr int kKvSlots = 5;                        // K and V tiles in flight (ring of 32 KB slots)
constexpr int kThreads = 384;
constexpr int kSoftmaxThreads = 128;
constexpr int kSoftmaxRegs = 224, kOtherRegs = 56;   // per-thread register targets after rebalancing

constexpr int OFF_Q = 0;                          // Q tile 0, Q tile 1
constexpr int OFF_KV = 2 * kTileBytes;
constexpr int OFF_BAR = OFF_KV + kKvSlots * kTileBytes;
// mbarriers: Q_FULL | KV_FULL[slots] | KV_EMPTY[slots] | S_FULL[2] | P_FULL[tile][half] | O_FULL[2] |
//            Q_EMPTY   (hands the Q tiles over from one work item to the next)
constexpr int BAR_Q_FULL = 0, BAR_KV_FULL = 1, BAR_KV_EMPTY = BAR_KV_FULL + kKvSlots,
              BAR_S_FULL = BAR_KV_EMPTY + kKvSlots, BAR_P_FULL = BAR_S_FULL + 2, BAR_O_FULL = BAR_P_FULL + 4,
              BAR_Q_EMPTY = BAR_O_FULL + 2, BAR_DRAIN = BAR_Q_EMPTY + 1,   // DRAIN: only used when a CTA gives up
              BAR_ITEM_FULL = BAR_DRAIN + 1, BAR_ITEM_EMPTY = BAR_ITEM_FULL + 2,   // packed prompts: the ring of items,
              BAR_GROUP = BAR_ITEM_EMPTY + 2,                                      // and a barrier of each softmax warpgroup
              BAR_ITEM_WANT = BAR_GROUP + 2,                                       // the producer is about to need the next item
              kNumBars = BAR_ITEM_WANT + 1;
static_assert(kNumBars <= 32, "barrier area");
constexpr int OFF_TMEM_PTR = OFF_BAR + 32 * 8;
constexpr int OFF_ABORT = OFF_TMEM_PTR + 4;
constexpr int OFF_ITEMS = OFF_ABORT + 12;         // int [2][4]: place of the request (-1: no more items), rank pair, rest, mode
constexpr int OFF_LAST = OFF_ITEMS + 32;          // int [2]: the warpgroup's part was its item's last
static_assert(OFF_ITEMS % 16 == 0 && OFF_LAST + 8 <= OFF_BAR + 512, "item ring");
constexpr int kItemReaders = 10;                  // producer, issuer and eight softmax warps read every item
constexpr int kSmemBytes = OFF_BAR + 512 + 1024;  // + slack to align the base to 1024 bytes

constexpr uint32_t kTmemCols = 512;
constexpr uint32_t TM_S = 0, TM_O = 256;          // + 128 * tile

constexpr float kRescaleThreshold = 8.0f;         // log2 units

// instruction descriptor, kind::f16: D fp32, A and B bf16, M 128, N 128
constexpr uint32_t kIdescBase = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
constexpr uint32_t kIdescQK = kIdescBase;               // A, B K-major
constexpr uint32_t kIdescPV = kIdescBase | (1u << 16);  // B (= V) MN-major

enum Mode { kRouted = 0, kBlocks = 1, kPacked = 2 };

constexpr int kPackReqs = 64;                     // requests (or parts) per launch of packed prompts (they travel as kernel arguments)
constexpr int kMaxParts = 16;                     // parts of an item at most
constexpr int kPartTiles = 4;                     // key tiles of a part at most, where there are accumulators for that many parts
struct PackReq {
    int req, q_row, k_row, nq, nk;                // routed request; first row in q and in k / v; new tokens; keys
    int part, parts, base;                        // this entry walks part `part` of `parts` of the key tiles; first accumulator
};
struct NoPack {};
struct PackArgs {
    PackReq r[kPackReqs];
    int n;
    int touch_words;
    uint32_t *counter;                            // items drawn so far beyond the first of every CTA; zero between launches
    uint32_t *tickets;                            // [accumulator][2]: parts of an item (that of its part 0) finished; zero between launches
    float4 *acc_o;                                // [accumulator][2 query tiles][32 channel quads][128 rows]
    float2 *acc_ml;                               // [accumulator][2][128]
};
template <int kMode> struct PackOf { using type = NoPack; };
template <> struct PackOf<kPacked> { using type = PackArgs; };

struct TcArgs {
    __nv_bfloat16 *out;
    const uint8_t *mask;
    int L, layer, req, Hq, G, S, W, q_start, Nq;
    int n_qt, n_kv, P, odd;      // query tiles, KV heads, head pairs per KV head, 1 if a head is left over
    int n_items;                 // work items of the launch
    float scale_log2;
    int32_t *debug;
    uint32_t *status;
    const uint8_t *bm;           // block-mask mode: uint8 [absolute query block][n_kb], blocks of 64 positions
    int n_kb;
    uint32_t *touch;             // debug bitmap of the KV positions loaded, or NULL
};

// KV tile index of the it-th tile a query tile keeps: sink tiles [0, e1), then window tiles from b2
__device__ __forceinline__ int tile_of(int it, int e1, int b2) { return it < e1 ? it : b2 + (it - e1); }

// Per-CTA constants shared by the three roles.
struct Cta {
    uint32_t sb;            // shared-window address of the 1024-byte aligned base
    uint32_t bar0;          // first mbarrier
    uint32_t tmem;          // TMEM base address
    volatile int *abort_flag;
    uint32_t *status;
    int kvh, nslots, q_end;
    int head0, head1, qt0, qt1, i00, i01;   // per query tile: query head, tile index in the chunk, first absolute position
    __device__ __forceinline__ int head(int t) const { return t ? head1 : head0; }
    __device__ __forceinline__ int qt(int t) const { return t ? qt1 : qt0; }
    __device__ __forceinline__ int i0(int t) const { return t ? i01 : i00; }
    int e1, b2, n_tiles;    // routed layers: KV tiles kept are [0, e1) and [b2, b2 + n_tiles - e1)
    bool fa;
    const uint8_t *bm;      // block-mask mode: mask, row length, last candidate KV tile
    int n_kb, last_tile;
    int req;                                // packed prompts: the item's request (debug bitmap)
    int t_begin, parts, acc, ticket;        // packed prompts: first tile of the part, parts that are not empty, accumulator, the item's ticket
    int q_start, q_row, k_row;              // packed prompts: position of the first query row, its row in q, the row of position 0 in k / v
    __device__ __forceinline__ uint32_t bar(int i) const { return bar0 + 8u * (uint32_t)i; }
    // every lane of the (converged) calling warp waits; the result is the same for all of them
    __device__ __forceinline__ bool wait(int i, uint32_t parity) const
    {
        return __all_sync(0xffffffffu, mbar_wait(bar(i), parity, abort_flag, status));
    }
};

// Work items, heaviest (latest query tiles) first.  An item is two query tiles that walk the
// same K / V tiles: the same 128 rows of two heads of a KV group, or -- for the head left
// over when the group size is odd -- two consecutive row tiles of that head (the earlier
// one simply finds its last KV tile fully masked).  Rank r = tiles counted from the end;
// ranks come in pairs (2k, 2k+1): n_kv * P head-pair items each, plus n_kv left-over items
// (tiles n_qt-1-2k and n_qt-2-2k) listed with the even rank.
__device__ __forceinline__ void decode_tiles(const TcArgs &a, int k2, int rem, int n_qt, int q_start, bool fa, Cta &c)
{
    int r = 2 * k2;
    bool leftover = false;
    if (rem < a.n_kv * a.P) {
    } else if (rem < a.n_kv * (a.P + a.odd)) {
        leftover = true;
        rem -= a.n_kv * a.P;
    } else {
        rem -= a.n_kv * (a.P + a.odd);
        r += 1;
    }
    const int qt = n_qt - 1 - r;
    if (!leftover) {
        c.kvh = rem / a.P;
        const int pi = rem % a.P;
        c.head0 = c.kvh * a.G + 2 * pi;
        c.head1 = c.head0 + 1;
        c.qt0 = c.qt1 = qt;
        c.nslots = 2;
    } else {
        c.kvh = rem;
        c.head0 = c.head1 = c.kvh * a.G + a.G - 1;
        c.qt0 = qt;
        c.qt1 = qt - 1;
        c.nslots = qt >= 1 ? 2 : 1;
    }
    c.i00 = q_start + c.qt0 * BM;
    c.i01 = q_start + c.qt1 * BM;
    const int i0_min = c.nslots == 2 ? c.i01 : c.i00;     // tile 1 is never later than tile 0
    const int i_hi = min(c.i00 + BM - 1, c.q_end - 1);
    const int e2 = i_hi / BN + 1;
    if (fa) {
        c.e1 = 0;
        c.b2 = 0;
    } else {
        c.e1 = min((a.S + BN - 1) / BN, e2);
        c.b2 = max(c.e1, max(0, i0_min - a.W + 1) / BN);
    }
    c.n_tiles = c.e1 + max(0, e2 - c.b2);
    c.last_tile = e2 - 1;
}

__device__ __forceinline__ void decode_item(const TcArgs &a, const NoPack &, int item, Cta &c)
{
    const int per2 = a.n_kv * (2 * a.P + a.odd);
    decode_tiles(a, item / per2, item % per2, a.n_qt, a.q_start, c.fa, c);
}

// The kernel is persistent: CTA b of G takes items b, 2G-1-b, 2G+b, 4G-1-b, ... (a serpentine over
// the weight-sorted list, so every CTA gets nearly the same amount of work).  Returns the k-th item
// of this CTA, or a number >= n_items when there is none.
__device__ __forceinline__ int item_of(int k)
{
    const int G = (int)gridDim.x, b = (int)blockIdx.x;
    return k * G + ((k & 1) ? G - 1 - b : b);
}

// The k-th item of this CTA for the calling (converged) warp; false when there is none, or the CTA is giving up.
__device__ __forceinline__ bool next_item(const TcArgs &a, const NoPack &pk, int k, Cta &c)
{
    const int item = item_of(k);
    if (item >= a.n_items) return false;
    decode_item(a, pk, item, c);
    return true;
}
// Parts of an item of n_tiles key tiles (fewer than the host assumed, if its request is sparse) whose request, of nq new tokens, is to
// be cut into `parts`.  Short items stay whole: cutting 8 tiles in two takes 1 row from 20.3 to 15.2 us, 64 rows from 20.4 to 17.8, 128
// rows from 21.3 to 20.7 (32/8 heads); 12 tiles of 128 rows in three 24.2 -> 22.3.  Parts of 4 against parts of 6: 1 row over 2048
// keys 16.0 / 22.0 us, 300 rows 23.7 / 27.9, from 8192 keys on the same.
__host__ __device__ __forceinline__ int parts_of(int parts, int n_tiles, int nq)
{
    if (n_tiles < (nq <= 64 ? 8 : 12)) return 1;
    const int most = (n_tiles + kPartTiles - 1) / kPartTiles;
    return most < parts ? most : parts;
}

__device__ __forceinline__ bool next_item(const TcArgs &a, const PackArgs &pk, int k, Cta &c)
{
    if (!c.wait(BAR_ITEM_FULL + (k & 1), (uint32_t)((k >> 1) & 1))) return false;
    int i, k2, rem, mode;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(i), "=r"(k2), "=r"(rem), "=r"(mode) : "r"(c.sb + OFF_ITEMS + 16 * (k & 1)) : "memory");
    __syncwarp();
    if (elect_one()) mbar_arrive(c.bar(BAR_ITEM_EMPTY + (k & 1)));
    if (i < 0) return false;
    const PackReq &r = pk.r[i];
    c.fa = mode != 0;
    c.req = r.req;
    c.q_start = r.nk - r.nq;
    c.q_end = r.nk;
    c.q_row = r.q_row;
    c.k_row = r.k_row;
    decode_tiles(a, k2, rem, (r.nq + BM - 1) / BM, c.q_start, c.fa, c);
    c.t_begin = 0;
    c.parts = 1;
    if (r.parts > 1) {
        c.parts = parts_of(r.parts, c.n_tiles, r.nq);
        c.ticket = r.base + (k2 * a.n_kv * (2 * a.P + a.odd) + rem) * r.parts;
        c.acc = c.ticket + r.part;
        c.t_begin = c.n_tiles * r.part / c.parts;
        c.n_tiles = c.n_tiles * (r.part + 1) / c.parts;
    }
    return true;
}

// Packed prompts: draws this CTA's items.  The first number is the CTA's own; each further one is the number of CTAs plus
// the counter.  Every CTA ends with one draw past the end, so a launch of n items draws n times in all, and whoever
// draws last puts the counter back to zero.
//
// Order: a pair is ranks 2 k, 2 k + 1 of one request (k < pairs: tiles counted from the end) with all their heads (per2 items; fewer in the
// last pair of an odd number of tiles);
// its weight is the number of key tiles its first rank walks, T - 2 k (T: tiles of all the request's keys), for a sparse
// request at most sink and window, divided by the parts it is cut into (at least 1).  Pairs are numbered by weight, heaviest first, then by request.  Request r has
// min(pairs, (T - w parts) / 2 + 1) pairs of weight w or more, so the weight of a given item is found by bisection over the sum
// of their items, which a warp adds up in a few instructions (kPackReqs / 32 requests per lane).
__device__ __forceinline__ void role_schedule(Cta &c, const TcArgs &a, const PackArgs &pk)
{
    constexpr int kPer = kPackReqs / 32;
    const int lane = threadIdx.x & 31;
    const int per2 = a.n_kv * (2 * a.P + a.odd);
    // The table is read with a different index in each lane: through a generic address, since the constant bank would serve the
    // lanes one by one.
    const PackReq *table = pk.r;
    asm("" : "+l"(table));
    const int cap_sa = (a.S + BN - 1) / BN + (a.W + BN - 1) / BN + 1;
    int tiles[kPer], pairs[kPer], items[kPer], cap[kPer], parts[kPer], top = 0;
    uint32_t dense = 0;
    PackReq mine[kPer];
#pragma unroll
    for (int z = 0; z < kPer; ++z) {
        mine[z].nq = -1;
        if (32 * z + lane < pk.n) mine[z] = table[32 * z + lane];
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    auto write_record = [&](const PackReq &r, int mode) {       // dispatch record (flux_debug_dispatch)
        const int n = r.nk;
        const bool two = mode == 0 && n > a.S + a.W;
        int32_t *d = a.debug + (size_t)r.req * 8;
        d[0] = mode; d[1] = a.layer; d[2] = r.req; d[3] = n;
        d[4] = 0; d[5] = two ? a.S : n; d[6] = two ? n - a.W : 0; d[7] = two ? n : 0;
    };
#pragma unroll
    for (int z = 0; z < kPer; ++z) {
        const PackReq &r = mine[z];
        tiles[z] = pairs[z] = items[z] = cap[z] = 0;
        parts[z] = 1;
        if (r.nq < 0) continue;
        if (r.nq == 0) {
            if (blockIdx.x == 0) write_record(r, -1);
            continue;
        }
        const int mode = a.mask[(size_t)r.req * a.L + a.layer];
        if (mode > 1 && blockIdx.x == 0) atomicOr(a.status, FLUX_STATUS_BAD_MASK);
        dense |= (mode != 0 ? 1u : 0u) << z;
        tiles[z] = (r.nk + BN - 1) / BN;
        pairs[z] = (r.nq + 2 * BM - 1) / (2 * BM);
        items[z] = pairs[z] * per2 - ((r.nq + BM - 1) / BM & 1) * a.n_kv * a.P;
        cap[z] = mode != 0 ? tiles[z] : min(tiles[z], cap_sa);
        parts[z] = r.parts;
        top = max(top, cap[z] / r.parts);
        if (blockIdx.x == 0 && r.part == 0) write_record(r, mode != 0 ? 1 : 0);
    }
    const bool expired = (*reinterpret_cast<volatile uint32_t *>(a.status) & FLUX_STATUS_WAIT_EXPIRED) != 0;
    top = max(1, __reduce_max_sync(0xffffffffu, top));
    auto count = [&](int z, int w) {     // items of weight w or more
        if (w <= 1) return items[z];
        const int n = w * parts[z] > cap[z] ? 0 : ((tiles[z] - w * parts[z]) >> 1) + 1;
        return n >= pairs[z] ? items[z] : n * per2;
    };
    auto total = [&](int w) {
        int s = 0;
#pragma unroll
        for (int z = 0; z < kPer; ++z) s += count(z, w);
        return __reduce_add_sync(0xffffffffu, s);
    };
    int above_top = 0;                   // total(top + 1)
    int item = expired ? a.n_items : (int)blockIdx.x;
    auto draw = [&]() {
        unsigned d = 0;
        if (lane == 0) {
            d = atomicAdd(pk.counter, 1u);
            if (d == (unsigned)(a.n_items - 1)) *pk.counter = 0u;
        }
        item = (int)gridDim.x + (int)__shfl_sync(0xffffffffu, d, 0);
    };
    for (int k = 0;; ++k) {
        int place = -1, k2 = 0, rem = 0, mode = 0;
        while (item < a.n_items) {
            int off = item;
            // the largest weight w with total(w) > off: at weight 1 all items count; numbers only grow, so w is at most the last one
            // (top), and mostly near it: steps down that double, then bisection
            int lo = top, hi = top + 1, above = above_top;       // total(hi) = above <= off
            for (int step = 1;; step *= 2) {
                const int n = total(lo);
                if (n > off) break;
                hi = lo;
                above = n;
                lo = max(1, lo - step);
            }
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1, n = total(mid);
                if (n > off) lo = mid; else { hi = mid; above = n; }
            }
            top = lo;
            above_top = above;
            off -= above;
            place = -1;
#pragma unroll
            for (int z = 0; z < kPer; ++z) {
                if (32 * z >= pk.n || place >= 0) break;
                const int before = count(z, hi), mine = count(z, lo) - before;
                int sum = mine;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, sum, d);
                    if (lane >= d) sum += y;
                }
                const uint32_t past = __ballot_sync(0xffffffffu, sum > off);
                if (past != 0) {
                    const int src = __ffs(past) - 1;
                    place = 32 * z + src;
                    rem = __shfl_sync(0xffffffffu, before + off - (sum - mine), src);
                    mode = (int)((__shfl_sync(0xffffffffu, dense, src) >> z) & 1u);
                }
                off -= __shfl_sync(0xffffffffu, sum, 31);
            }
            k2 = rem / per2;
            rem -= k2 * per2;
            bool real = true;                                   // an item of few tiles has fewer parts
            if (pk.r[place].part > 0) {
                const PackReq &r = pk.r[place];
                c.q_start = r.nk - r.nq;
                c.q_end = r.nk;
                decode_tiles(a, k2, rem, (r.nq + BM - 1) / BM, c.q_start, mode != 0, c);
                real = r.part < parts_of(r.parts, c.n_tiles, r.nq);
            }
            if (real) break;
            place = -1;
            draw();
        }
        if (!c.wait(BAR_ITEM_EMPTY + (k & 1), (uint32_t)(((k >> 1) & 1) ^ 1))) return;
        if (elect_one()) {
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(c.sb + OFF_ITEMS + 16 * (k & 1)), "r"(place), "r"(k2), "r"(rem), "r"(mode) : "memory");
            mbar_arrive(c.bar(BAR_ITEM_FULL + (k & 1)));
        }
        if (place < 0) return;
        if (!c.wait(BAR_ITEM_WANT, (uint32_t)(k & 1))) return;
        draw();
    }
}

// The KV tiles of a work item, in the order every role walks them.  Called by all lanes of a
// converged warp.  Routed FA / SA layers: a plain range.  Block-mask mode: the tiles [0, last_tile]
// in which at least one kept 64 x 64 block meets the item's rows; the warp inspects 32 candidate
// tiles at a time (one per lane) and hands out the non-empty ones.  pat: for query tile t, bit
// 4 t + 2 rb + cb says that the block (row half rb, key half cb) of the 128 x 128 tile is kept.
template <int kMode>
struct TileWalk {
    const Cta &c;
    int it = 0, base = 0;
    uint32_t bal = 0, mypat = 0;
    __device__ __forceinline__ explicit TileWalk(const Cta &cta) : c(cta)
    {
        if (kMode == kPacked) it = cta.t_begin;
    }
    __device__ __forceinline__ uint32_t pattern(int j) const
    {
        uint32_t pat = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (t >= c.nslots) break;
#pragma unroll
            for (int rb = 0; rb < 2; ++rb) {
                const int qb = c.i0(t) / 64 + rb;
                if (qb * 64 >= c.q_end) continue;
#pragma unroll
                for (int cb = 0; cb < 2; ++cb) {
                    const int kb = 2 * j + cb;
                    if (kb <= qb && kb < c.n_kb && c.bm[(size_t)qb * c.n_kb + kb] != 0) pat |= 1u << (4 * t + 2 * rb + cb);
                }
            }
        }
        return pat;
    }
    __device__ __forceinline__ bool next(int &jt, uint32_t &pat)
    {
        if (kMode != kBlocks) {
            if (it >= c.n_tiles) return false;
            jt = tile_of(it++, c.e1, c.b2);
            pat = 0xffu;
            return true;
        }
        const int lane = threadIdx.x & 31;
        while (bal == 0) {
            if (base > c.last_tile) return false;
            const int j = base + lane;
            mypat = j <= c.last_tile ? pattern(j) : 0u;
            bal = __ballot_sync(0xffffffffu, mypat != 0u);
            base += 32;
        }
        const int ln = __ffs(bal) - 1;
        bal &= bal - 1;
        jt = base - 32 + ln;
        pat = __shfl_sync(0xffffffffu, mypat, ln);
        ++it;
        return true;
    }
};

// ================= TMA producer (one warp, one issuing lane) =================
template <int kMode>
__device__ __forceinline__ void role_load(Cta &c, const TcArgs &a, const typename PackOf<kMode>::type &pk, const CUtensorMap *tm_q, const CUtensorMap *tm_k,
                                          const CUtensorMap *tm_v, int &qi, int &q_armed)
{
    // qi: K / V tiles requested so far (ring position); q_armed: items whose Q tiles have been requested.  Both are
    // the caller's, so that a CTA that gives up knows which copies may still be on their way.
    for (int k = 0;; ++k) {
        if (!next_item(a, pk, k, c)) break;
        // Q of the next item may overwrite Q of this one once its last QK^T has completed
        if (k > 0 && !c.wait(BAR_Q_EMPTY, (uint32_t)((k - 1) & 1))) return;
        q_armed = k + 1;
        if (elect_one()) {
            mbar_expect_tx(c.bar(BAR_Q_FULL), (uint32_t)(c.nslots * kTileBytes));
            for (int t = 0; t < c.nslots; ++t) {
                tma_load_3d(c.sb + OFF_Q + t * kTileBytes, tm_q, c.bar(BAR_Q_FULL), 0, c.head(t), (kMode == kPacked ? c.q_row : 0) + c.qt(t) * BM);
                tma_load_3d(c.sb + OFF_Q + t * kTileBytes + kHalfBytes, tm_q, c.bar(BAR_Q_FULL), 64, c.head(t), (kMode == kPacked ? c.q_row : 0) + c.qt(t) * BM);
            }
        }
        TileWalk<kMode> walk(c);
        int jt;
        uint32_t pat;
        bool asked = false;
        while (walk.next(jt, pat)) {
            // With two tiles to go the next item is asked for.  Not earlier: an item held back here is one that an idle CTA
            // could have started (each CTA drawing up to two ahead doubled the time of a single wave of items).
            if (kMode == kPacked && !asked && c.n_tiles - walk.it <= 2) {
                asked = true;
                if (elect_one()) mbar_arrive(c.bar(BAR_ITEM_WANT));
            }
            const int j0 = jt * BN, row = (kMode == kPacked ? c.k_row : 0) + j0;
            if (a.touch != nullptr) {   // debug: the positions of this tile that exist, 32 per lane 0..3
                const int lane = threadIdx.x & 31, first = j0 + 32 * lane;
                uint32_t *touch = a.touch;
                if constexpr (kMode == kPacked) touch += (size_t)c.req * pk.touch_words;
                if (lane < 4 && first < c.q_end)
                    atomicOr(touch + (first >> 5), c.q_end - first >= 32 ? 0xffffffffu : (1u << (c.q_end - first)) - 1u);
            }
#pragma unroll
            for (int kv = 0; kv < 2; ++kv, ++qi) {
                const int slot = qi % kKvSlots, use = qi / kKvSlots;
                if (!c.wait(BAR_KV_EMPTY + slot, (uint32_t)((use & 1) ^ 1))) return;
                const uint32_t dst = c.sb + OFF_KV + slot * kTileBytes;
                const CUtensorMap *tm = kv ? tm_v : tm_k;
                if (elect_one()) {
                    mbar_expect_tx(c.bar(BAR_KV_FULL + slot), (uint32_t)kTileBytes);
                    tma_load_3d(dst, tm, c.bar(BAR_KV_FULL + slot), 0, c.kvh, row);
                    tma_load_3d(dst + kHalfBytes, tm, c.bar(BAR_KV_FULL + slot), 64, c.kvh, row);
                }
            }
        }
    }
}

// ================= MMA issuer (one warp, one issuing lane) =================
// Issue order per KV tile j:  PV_0[j] QK_0[j+1] PV_1[j] QK_1[j+1]; the tensor pipe runs them in
// that order, so S_t[j+1] overwrites S_t / P_t only after PV_t[j] has read P_t[j].  (One issuer for
// both tiles: two issuing warps, whose MMAs interleave instruction by instruction, ran slower.)
// Across items the same order holds (the first QK^T of an item follows the last PV of the one
// before).  The first PV of an item overwrites O_t; it waits for that item's first P_t, which the
// softmax warps of tile t publish only after their epilogue has read the previous item's O_t.
template <int kMode>
__device__ __forceinline__ void role_mma(Cta &c, const TcArgs &a, const typename PackOf<kMode>::type &pk)
{
    // S_t = Q_t K^T, then up to two commits (tcgen05.commit belongs to the issuing lane; 0 = none)
    auto qk = [&](int t, int slot, uint32_t bar_a, uint32_t bar_b) {
        const uint32_t qb = c.sb + OFF_Q + t * kTileBytes, kb = c.sb + OFF_KV + slot * kTileBytes;
        if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) {
                const uint32_t off = (uint32_t)((kk >> 2) * kHalfBytes + (kk & 3) * 32);
                tc_mma_ss(c.tmem + TM_S + t * 128, smem_desc(qb + off, 16), smem_desc(kb + off, 16), kIdescQK,
                          kk > 0 ? 1u : 0u);
            }
            tc_commit(bar_a);
            if (bar_b) tc_commit(bar_b);
        }
    };
    // O_t (+)= P_t[:, 64 half ..] V[64 half ..]
    auto pv_half = [&](int t, int slot, int half, bool acc, uint32_t bar_a, uint32_t bar_b) {
        const uint32_t vb = c.sb + OFF_KV + slot * kTileBytes;
        if (elect_one()) {
#pragma unroll
            for (int k4 = 0; k4 < 4; ++k4) {
                const int kk = half * 4 + k4;
                tc_mma_ts(c.tmem + TM_O + t * 128, c.tmem + TM_S + t * 128 + kk * 8,
                          smem_desc(vb + kk * 2048, kHalfBytes), kIdescPV, (acc || kk > 0) ? 1u : 0u);
            }
            if (bar_a) tc_commit(bar_a);
            if (bar_b) tc_commit(bar_b);
        }
    };
    int qi = 0;                                      // K / V tiles consumed so far (ring position)
    int tiles[2] = {0, 0};                           // per query-tile slot: KV tiles done (barrier phases)
    for (int k = 0;; ++k) {
        if (!next_item(a, pk, k, c)) break;
        TileWalk<kMode> walk(c);
        int jt;
        uint32_t pat;
        bool more = walk.next(jt, pat);
        if (!c.wait(BAR_Q_FULL, (uint32_t)(k & 1))) return;
        if (!more) {    // (block-mask mode) the item keeps no block at all: nothing to accumulate
            if (elect_one()) {
                for (int t = 0; t < c.nslots; ++t) tc_commit(c.bar(BAR_O_FULL + t));
                tc_commit(c.bar(BAR_Q_EMPTY));
            }
            continue;
        }
        {
            const int kslot = qi % kKvSlots, kpar = (qi / kKvSlots) & 1;
            if (!c.wait(BAR_KV_FULL + kslot, (uint32_t)kpar)) return;
            tc_fence_after();
            for (int t = 0; t < c.nslots; ++t)
                qk(t, kslot, c.bar(BAR_S_FULL + t), t == c.nslots - 1 ? c.bar(BAR_KV_EMPTY + kslot) : 0u);
            ++qi;
        }
        for (bool first = true; more; first = false) {
            const int vslot = qi % kKvSlots, vpar = (qi / kKvSlots) & 1;
            const int kslot = (qi + 1) % kKvSlots, kpar = ((qi + 1) / kKvSlots) & 1;
            more = walk.next(jt, pat);
            if (!c.wait(BAR_KV_FULL + vslot, (uint32_t)vpar)) return;
            // no QK^T of this item is left to issue once its last tile is reached: Q may be replaced
            if (!more && elect_one()) tc_commit(c.bar(BAR_Q_EMPTY));
            for (int t = 0; t < c.nslots; ++t) {
                const bool last = t == c.nslots - 1;
                if (!c.wait(BAR_P_FULL + 2 * t, (uint32_t)(tiles[t] & 1))) return;
                tc_fence_after();
                pv_half(t, vslot, 0, !first, 0u, 0u);
                if (!c.wait(BAR_P_FULL + 2 * t + 1, (uint32_t)(tiles[t] & 1))) return;
                tc_fence_after();
                // after the second half: the V slot is free once the last tile's PV is done; O is complete on the last KV tile
                pv_half(t, vslot, 1, !first, last ? c.bar(BAR_KV_EMPTY + vslot) : 0u, more ? 0u : c.bar(BAR_O_FULL + t));
                tiles[t]++;
                if (more) {
                    if (t == 0) {
                        if (!c.wait(BAR_KV_FULL + kslot, (uint32_t)kpar)) return;
                        tc_fence_after();
                    }
                    qk(t, kslot, c.bar(BAR_S_FULL + t), last ? c.bar(BAR_KV_EMPTY + kslot) : 0u);
                }
            }
            qi += more ? 2 : 1;
        }
    }
}

// Bits 0 .. x of a word (none for x < 0, all for x >= 31)
__device__ __forceinline__ uint32_t bits_upto(int x) { return x < 0 ? 0u : 0xffffffffu >> (31 - min(x, 31)); }

// A part of a packed item is done: O (unnormalised), maximum and sum of this thread's row go to the workspace; the warpgroup that
// draws the item's last ticket adds the parts up in order and writes the output rows.  False when a wait ran out.
__device__ __forceinline__ bool split_epilogue(const Cta &c, const TcArgs &a, const PackArgs &pk, int t, int r, int row, uint32_t tO, float m, float l,
                                               uint32_t &phase)
{
    const bool valid = row < c.q_end;
    float4 *o = pk.acc_o + ((size_t)c.acc * 2 + t) * 32 * BM + r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t x[32];
        tc_ld32(tO + q * 32, x);
        tc_wait_ld();
        if (valid) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                o[(8 * q + e) * BM] = make_float4(__uint_as_float(x[4 * e]), __uint_as_float(x[4 * e + 1]), __uint_as_float(x[4 * e + 2]),
                                                  __uint_as_float(x[4 * e + 3]));
        }
    }
    if (valid) pk.acc_ml[((size_t)c.acc * 2 + t) * BM + r] = make_float2(m, l);
    // the warpgroup meets at an mbarrier, whose wait is bounded like every other
    auto meet = [&]() {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(c.bar(BAR_GROUP + t));
        const bool ok = c.wait(BAR_GROUP + t, phase & 1);
        ++phase;
        return ok;
    };
    volatile int *last = c.abort_flag + (OFF_LAST - OFF_ABORT) / 4 + t;
    if (!meet()) return false;
    if (r == 0) {
        unsigned seen;
        uint32_t *ticket = pk.tickets + 2 * c.ticket + t;
        asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(seen) : "l"(ticket) : "memory");
        *last = seen == (unsigned)(c.parts - 1);
        if (seen == (unsigned)(c.parts - 1)) *ticket = 0u;
    }
    if (!meet()) return false;
    if (!*last) return true;
    const int n_valid = c.q_end - (row - r);             // rows of this tile that exist
    if (n_valid <= min(4 * c.parts, 48)) {
        // Few rows: a thread takes a channel quad of a row, every part's share of it asked for at once, four rows a round; neighbouring
        // threads take neighbouring rows, which lie side by side.  A thread per row (below) waits for one part after the
        // other, 0.6 us each, with most threads idle.  Whole call, 8/2 heads, this / the other way: 8 rows over 1024 keys (2 parts)
        // 15.4 / 16.1 us, 24 rows 18.1 / 16.2; 32 rows over 8192 (16 parts) 25.0 / 29.4, 64 rows 34.4 / 29.7.
        for (int z = r; z < n_valid * 32; z += kSoftmaxThreads) {
            const int quad = z / n_valid, zr = z - quad * n_valid;
            const float2 *ml = pk.acc_ml + ((size_t)c.ticket * 2 + t) * BM + zr;
            const float4 *po = pk.acc_o + (((size_t)c.ticket * 2 + t) * 32 + quad) * BM + zr;
            float4 v[kMaxParts];
            float2 x[kMaxParts];
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int i = 0; i < kMaxParts; ++i) {
                x[i] = make_float2(-INFINITY, 0.f);
                v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (i < c.parts) {
                    x[i] = __ldcg(ml + (size_t)i * 2 * BM);
                    v[i] = __ldcg(po + (size_t)i * 2 * 32 * BM);
                }
            }
#pragma unroll
            for (int i = 0; i < kMaxParts; ++i) top = fmaxf(top, x[i].x);
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < kMaxParts; ++i) {
                const float w = fast_exp2(x[i].x - top); // 0 for a part that keeps none of the row's keys
                sum = fmaf(x[i].y, w, sum);
                s.x = fmaf(v[i].x, w, s.x);
                s.y = fmaf(v[i].y, w, s.y);
                s.z = fmaf(v[i].z, w, s.z);
                s.w = fmaf(v[i].w, w, s.w);
            }
            const float inv = 1.0f / sum;
            uint2 y = make_uint2(pack_bf16(s.x * inv, s.y * inv), pack_bf16(s.z * inv, s.w * inv));
            *reinterpret_cast<uint2 *>(a.out + ((size_t)(c.q_row + row - r + zr - c.q_start) * a.Hq + c.head(t)) * kHeadDim + 4 * quad) = y;
        }
        return true;
    }
    if (!valid) return true;
    const float2 *ml = pk.acc_ml + ((size_t)c.ticket * 2 + t) * BM + r;
    const float4 *po = pk.acc_o + ((size_t)c.ticket * 2 + t) * 32 * BM + r;
    float top = -INFINITY, sum = 0.f;
    for (int i = 0; i < c.parts; ++i) top = fmaxf(top, __ldcg(ml + (size_t)i * 2 * BM).x);
    float4 s[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) s[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int i = 0; i < c.parts; ++i) {
        const float2 x = __ldcg(ml + (size_t)i * 2 * BM);
        const float w = fast_exp2(x.x - top);            // 0 for a part that keeps none of the row's keys
        sum = fmaf(x.y, w, sum);
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            const float4 v = __ldcg(po + (size_t)i * 2 * 32 * BM + e * BM);
            s[e].x = fmaf(v.x, w, s[e].x);
            s[e].y = fmaf(v.y, w, s[e].y);
            s[e].z = fmaf(v.z, w, s[e].z);
            s[e].w = fmaf(v.w, w, s[e].w);
        }
    }
    const float inv = 1.0f / sum;
    __nv_bfloat16 *dst = a.out + ((size_t)(c.q_row + row - c.q_start) * a.Hq + c.head(t)) * kHeadDim;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        uint32_t y[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[2 * e] = pack_bf16(s[4 * q + e].x * inv, s[4 * q + e].y * inv);
            y[2 * e + 1] = pack_bf16(s[4 * q + e].z * inv, s[4 * q + e].w * inv);
        }
        st_global_32B(dst + q * 16, y);
    }
    return true;
}

// ================= softmax of query tile t (one thread per query row) =================
template <int kMode>
__device__ __forceinline__ void role_softmax(Cta &c, const TcArgs &a, const typename PackOf<kMode>::type &pk, int t, int warp, int lane)
{
    const int r = (warp & 3) * 32 + lane;            // row of the tile = TMEM lane
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = c.tmem + lane_base + TM_S + t * 128;
    const uint32_t tO = c.tmem + lane_base + TM_O + t * 128;
    const int S = a.S, W = a.W;
    const float scale_log2 = a.scale_log2;
    int tiles = 0, items = 0;                        // KV tiles and items this slot has done (barrier phases)
    uint32_t group_phase = 0;
    for (int k = 0;; ++k) {
        if (!next_item(a, pk, k, c)) break;
        if (t >= c.nslots) continue;                 // this item has a single query tile
        const int i0 = c.i0(t);                      // first absolute position of this query tile
        const int row = i0 + r;                      // absolute position of this query
        float m_used = -INFINITY;                    // running maximum in use, scaled log2 units
        float2 lsum = make_float2(0.f, 0.f);
        TileWalk<kMode> walk(c);
        int jt;
        uint32_t pat;
        while (walk.next(jt, pat)) {
            if (!c.wait(BAR_S_FULL + t, (uint32_t)(tiles & 1))) return;
            const bool first = walk.it == (kMode == kPacked ? c.t_begin : 0) + 1;   // first KV tile of this item: O holds nothing yet
            ++tiles;
            tc_fence_after();
            uint32_t sr[4][32];
#pragma unroll
            for (int q = 0; q < 4; ++q) tc_ld32(tS + q * 32, sr[q]);
            tc_wait_ld();
            const int j0 = jt * BN;
            const int jmax = j0 + BN - 1;
            // this row's two block bits of the tile (block-mask mode): keys [j0, j0+64) and [j0+64, j0+128)
            const uint32_t mine = pat >> (4 * t + 2 * (r >> 6));
            const bool full = kMode == kBlocks ? (jmax <= i0 && ((pat >> (4 * t)) & 0xfu) == 0xfu)
                                     : ((jmax <= i0) && (c.fa || jmax < S || j0 > i0 + BM - 1 - W));
            if (!full) {
                // The keys this row keeps as one bit each, 32 to a word: positions up to its own, of those the window's and the
                // sink's.  (The comparisons written out per element became branches: 4.8 us a tile instead of 0.5.)
                const int hi = row - j0, lo = c.fa ? INT_MIN / 2 : hi - W, sk = S - 1 - j0;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t word = bits_upto(hi - 32 * q);
                    if (kMode == kBlocks) {
                        if (((mine >> (q >> 1)) & 1u) == 0u) word = 0u;
                    } else {
                        word &= ~bits_upto(lo - 32 * q) | bits_upto(sk - 32 * q);
                    }
                    if (__all_sync(0xffffffffu, word == 0xffffffffu)) continue;
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if ((word & (1u << e)) == 0u) sr[q][e] = 0xff800000u;   // -inf
                }
            }
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int e = 0; e < 32; e += 2)
                    mx[q] = fmax3(mx[q], __uint_as_float(sr[q][e]), __uint_as_float(sr[q][e + 1]));
            const float mxs = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale_log2;
            const bool need = mxs > m_used + kRescaleThreshold;
            if (__any_sync(0xffffffffu, need)) {
                const float alpha = need ? fast_exp2(m_used - mxs) : 1.0f;   // 0 when nothing was kept so far
                if (need) m_used = mxs;
                lsum.x *= alpha;
                lsum.y *= alpha;
                if (!first) {                                                // PV of the previous tile is complete
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t o[32];
                        tc_ld32(tO + q * 32, o);
                        tc_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                        tc_st32(tO + q * 32, o);
                    }
                }
            }
            if constexpr (kMode == kPacked) {
                // Keys past the end of the request: their weights are 0, but V there belongs to another request (or to
                // nobody), and 0 x inf would be NaN.  Tile 0's four warps clear those rows before they hand over P (the
                // issuer waits for all four); PV of tile 0 is issued first, so this covers tile 1 too.
                if (t == 0 && jmax >= c.q_end) {
                    const int vi = 2 * tiles - 1;                  // place of this tile's V in the ring's sequence
                    if (!c.wait(BAR_KV_FULL + vi % kKvSlots, (uint32_t)((vi / kKvSlots) & 1))) return;
                    const uint32_t vb = c.sb + OFF_KV + (vi % kKvSlots) * kTileBytes;
                    for (int z = (c.q_end - j0) * 8 + r; z < BN * 8; z += kSoftmaxThreads)      // 16-byte pieces of both halves
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vb + h * kHalfBytes + z * 16), "r"(0u) : "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
            }
            const float neg_m = (m_used == -INFINITY) ? 0.f : -m_used;
            const float2 sc2 = make_float2(scale_log2, scale_log2), nm2 = make_float2(neg_m, neg_m);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t p[32];
                float2 acc2 = make_float2(0.f, 0.f);
#pragma unroll
                for (int qq = 0; qq < 2; ++qq)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float2 x = ffma2(make_float2(__uint_as_float(sr[2 * half + qq][2 * e]),
                                                     __uint_as_float(sr[2 * half + qq][2 * e + 1])), sc2, nm2);
                        x.x = fast_exp2(x.x);
                        x.y = fast_exp2(x.y);
                        if (qq == 0) lsum = fadd2(lsum, x); else acc2 = fadd2(acc2, x);
                        p[16 * qq + e] = pack_bf16(x.x, x.y);
                    }
                lsum = fadd2(lsum, acc2);
                tc_st32(tS + half * 32, p);                  // P columns [32 half, 32 half + 32) = keys [64 half, 64 half + 64)
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(c.bar(BAR_P_FULL + 2 * t + half));
            }
        }
        // ---- epilogue of the item: O / l -> bf16 -> global ----
        if (!c.wait(BAR_O_FULL + t, (uint32_t)(items & 1))) return;
        ++items;
        tc_fence_after();
        const float lrow = lsum.x + lsum.y;
        if constexpr (kMode == kPacked) {
            if (c.parts > 1) {
                if (!split_epilogue(c, a, pk, t, r, row, tO, m_used, lrow, group_phase)) return;
                continue;
            }
        }
        // (block-mask mode) a row whose mask keeps no key: zero output row, flagged
        const bool empty = kMode == kBlocks && !(lrow > 0.f);
        if (empty && row < c.q_end) atomicOr(c.status, FLUX_STATUS_BAD_MASK);
        const float inv = empty ? 0.f : 1.0f / lrow;
        const bool valid = row < c.q_end;
        __nv_bfloat16 *dst = a.out + ((size_t)(!valid ? 0 : kMode == kPacked ? c.q_row + row - c.q_start : row - a.q_start) * a.Hq + c.head(t)) * kHeadDim;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t o[32];
            tc_ld32(tO + q * 32, o);
            tc_wait_ld();
            if (valid) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint32_t w[8];
#pragma unroll
                    for (int z = 0; z < 8; ++z)
                        w[z] = empty ? 0u   // O holds nothing meaningful
                                     : pack_bf16(__uint_as_float(o[16 * e + 2 * z]) * inv, __uint_as_float(o[16 * e + 2 * z + 1]) * inv);
                    st_global_32B(dst + q * 32 + e * 16, w);
                }
            }
        }
        // The next item's first P_t is published by these same warps only after this point, and its
        // first PV (which overwrites O_t) waits for that P_t: O_t needs no hand-over barrier of its own.
    }
}

template <int kMode>
__global__ void __launch_bounds__(kThreads, 1)
prefill_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                  const __grid_constant__ CUtensorMap tm_v, TcArgs a, const __grid_constant__ typename PackOf<kMode>::type pk)
{
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    Cta c;
    c.sb = (raw + 1023u) & ~1023u;
    unsigned char *sm = smem_raw + (c.sb - raw);
    c.abort_flag = reinterpret_cast<volatile int *>(sm + OFF_ABORT);
    c.status = a.status;
    c.bar0 = c.sb + OFF_BAR;
    volatile uint32_t *tmem_ptr_smem = reinterpret_cast<volatile uint32_t *>(sm + OFF_TMEM_PTR);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // a CTA that starts after a wait has run out anywhere does nothing (packed prompts: it draws no item)
    if (kMode == kPacked) {
        if (tid == 0) *c.abort_flag = 0;
        if (tid < 3) asm volatile("prefetch.tensormap [%0];" ::"l"(tid == 0 ? &tm_q : tid == 1 ? &tm_k : &tm_v) : "memory");
    } else {
        if (tid == 0) *c.abort_flag = (*reinterpret_cast<volatile uint32_t *>(a.status) & FLUX_STATUS_WAIT_EXPIRED) ? 1 : 0;
        __syncthreads();
        if (*c.abort_flag) return;
    }

    const int bid = blockIdx.x;
    c.q_end = a.q_start + a.Nq;                           // KV rows present
    const uint8_t mode_raw = kMode != kRouted ? (uint8_t)1 : a.mask[a.req * a.L + a.layer];
    if (mode_raw > 1 && tid == 0) atomicOr(a.status, FLUX_STATUS_BAD_MASK);
    c.fa = mode_raw != 0;
    c.bm = a.bm;
    c.n_kb = a.n_kb;

    if (kMode == kRouted && bid == 0 && tid == 0) {
        const int n = c.q_end;
        const bool two = !c.fa && n > a.S + a.W;
        int32_t *d = a.debug;
        d[0] = c.fa ? 1 : 0; d[1] = a.layer; d[2] = a.req; d[3] = n;
        d[4] = 0; d[5] = two ? a.S : n; d[6] = two ? n - a.W : 0; d[7] = two ? n : 0;
    }

    // ---- set-up: barriers, TMEM ----
    if (tid == 0) {
        mbar_init(c.bar(BAR_Q_FULL), 1);
        for (int s = 0; s < kKvSlots; ++s) {
            mbar_init(c.bar(BAR_KV_FULL + s), 1);
            mbar_init(c.bar(BAR_KV_EMPTY + s), 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(c.bar(BAR_S_FULL + t), 1);
            mbar_init(c.bar(BAR_P_FULL + 2 * t), 4);       // one elected lane per softmax warp
            mbar_init(c.bar(BAR_P_FULL + 2 * t + 1), 4);
            mbar_init(c.bar(BAR_O_FULL + t), 1);
        }
        mbar_init(c.bar(BAR_Q_EMPTY), 1);
        mbar_init(c.bar(BAR_DRAIN), 1);
        if (kMode == kPacked)
            for (int s = 0; s < 2; ++s) {
                mbar_init(c.bar(BAR_ITEM_FULL + s), 1);
                mbar_init(c.bar(BAR_ITEM_EMPTY + s), kItemReaders);
                mbar_init(c.bar(BAR_GROUP + s), 4);            // one lane per softmax warp
            }
        if (kMode == kPacked) mbar_init(c.bar(BAR_ITEM_WANT), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(c.sb + OFF_TMEM_PTR), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    c.tmem = *tmem_ptr_smem;
    // packed prompts are launched with programmatic stream serialisation: the set-up above, and the scheduler's reading of the
    // argument table, run while the kernel before drains
    if (kMode == kPacked && warp != 10) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    }

    // Each warpgroup executes one setmaxnreg, all four of its warps the same one.
    int kv_requested = 0, q_requested = 0;               // the producer warp's counters (see the teardown)
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == 8) {
            role_load<kMode>(c, a, pk, &tm_q, &tm_k, &tm_v, kv_requested, q_requested);
        } else if (warp == 9) {
            role_mma<kMode>(c, a, pk);
        } else if (warp == 10) {
            if constexpr (kMode == kPacked) role_schedule(c, a, pk);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        role_softmax<kMode>(c, a, pk, warp >> 2, warp, lane);
    }

    // ---- teardown ----
    tc_fence_before();
    __syncthreads();
    if (*c.abort_flag) {
        // A wait gave up somewhere: copies and MMAs that were already issued must land before the shared memory and
        // TMEM go away.  The producer waits for the last copy it requested into each ring slot and for the last Q
        // tiles (their barriers complete when the bytes have arrived, whoever was to consume them); the issuer commits
        // once more and waits for that commit, which follows every MMA it issued.  These waits are bounded too.
        auto drain = [&](int bar, uint32_t parity) {
            for (int i = 0; i < 200 && !mbar_try(c.bar(bar), parity); ++i) __nanosleep(1000);
        };
        if (warp == 8) {
            for (int s = 0; s < kKvSlots; ++s) {
                const int last = kv_requested - 1 - ((kv_requested - 1 - s) % kKvSlots + kKvSlots) % kKvSlots;   // latest request into slot s
                if (kv_requested > 0 && last >= 0) drain(BAR_KV_FULL + s, (uint32_t)((last / kKvSlots) & 1));
            }
            if (q_requested > 0) drain(BAR_Q_FULL, (uint32_t)((q_requested - 1) & 1));
        }
        if (warp == 9) {
            if (elect_one()) tc_commit(c.bar(BAR_DRAIN));
            drain(BAR_DRAIN, 0u);
        }
        __syncthreads();
    }
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(c.tmem), "r"(kTmemCols) : "memory");
    }
}

// One warp waits, with the bounded wait the prefill kernel uses, on an mbarrier nothing ever
// arrives at: the wait runs out after `limit` cycles, raises FLUX_STATUS_WAIT_EXPIRED and the
// kernel returns normally.  Exists so that the give-up path can be exercised without a fault.
__global__ void wait_probe_kernel(uint32_t *status, long long limit)
{
    __shared__ __align__(8) unsigned long long bar_storage;
    __shared__ int abort_flag;
    const uint32_t bar = smem_u32(&bar_storage);
    if (threadIdx.x == 0) {
        abort_flag = 0;
        mbar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    mbar_wait(bar, 0, &abort_flag, status, limit);
}

// Dispatch records of requests without new tokens, for which no launch of the kernel above has work.
__global__ void skipped_records_kernel(int32_t *debug, int layer, int b0, int n)
{
    for (int b = b0 + threadIdx.x; b < b0 + n; b += blockDim.x) {
        int32_t *d = debug + (size_t)b * 8;
        d[0] = -1; d[1] = layer; d[2] = b;
        for (int i = 3; i < 8; ++i) d[i] = 0;
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn g_encode = nullptr;

// [rows][heads][128] bf16 tensor viewed as (d, head, row); box = 64 columns x 1 head x 128 rows
int make_map(CUtensorMap *tm, const void *base, int heads, int rows, int64_t row_stride = 0 /* elements; 0: contiguous rows */)
{
    cuuint64_t dims[3] = {(cuuint64_t)kHeadDim, (cuuint64_t)heads, (cuuint64_t)rows};
    cuuint64_t strides[2] = {(cuuint64_t)kRowBytes, row_stride ? (cuuint64_t)row_stride * 2 : (cuuint64_t)kRowBytes * (cuuint64_t)heads};
    cuuint32_t box[3] = {64, 1, (cuuint32_t)BM};
    cuuint32_t estr[3] = {1, 1, 1};
    CUresult r = g_encode(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(FLUX_E_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
    return FLUX_OK;
}

}  // namespace

int prefill_tc_setup()
{
    if (!g_encode) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        int rc = check_cuda(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &qres),
                            "cudaGetDriverEntryPointByVersion(cuTensorMapEncodeTiled)");
        if (rc) return rc;
        if (qres != cudaDriverEntryPointSuccess || !fn)
            return fail(FLUX_E_CUDA, "the driver does not export cuTensorMapEncodeTiled");
        g_encode = (EncodeTiledFn)fn;
    }
    // setmaxnreg moves registers inside the CTA's own allocation (registers per thread at launch x
    // threads); a request beyond it would block for ever, so refuse to run rather than launch that.
    const void *fns[3] = {(const void *)prefill_tc_kernel<kRouted>, (const void *)prefill_tc_kernel<kBlocks>,
                          (const void *)prefill_tc_kernel<kPacked>};
    for (const void *fn : fns) {
        cudaFuncAttributes fa;
        int rc = check_cuda(cudaFuncGetAttributes(&fa, fn), "cudaFuncGetAttributes(prefill_tc_kernel)");
        if (rc) return rc;
        if (fa.numRegs * kThreads < 2 * kSoftmaxThreads * kSoftmaxRegs + (kThreads - 2 * kSoftmaxThreads) * kOtherRegs)
            return fail(FLUX_E_CUDA, "prefill kernel was built with %d registers per thread: too few for its register rebalancing",
                        fa.numRegs);
        rc = check_cuda(cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes),
                        "cudaFuncSetAttribute(prefill_tc_kernel)");
        if (rc) return rc;
    }
    return FLUX_OK;
}

int launch_wait_probe(flux_plan *p, long long limit_cycles, cudaStream_t st)
{
    wait_probe_kernel<<<1, 32, 0, st>>>((uint32_t *)((char *)p->ws + p->lay.status), limit_cycles);
    p->launches++;
    return check_cuda(cudaGetLastError(), "wait probe launch");
}

// block_mask == NULL: a routed layer (FA or SA by the cached routing bit); else block-mask mode
int launch_prefill_tc(flux_plan *p, int layer, int req, const void *q, const void *k, const void *v, int q_start,
                      int Nq, void *out, cudaStream_t st, const uint8_t *block_mask, int n_kv_blocks)
{
    const flux_config &c = p->cfg;
    char *ws = (char *)p->ws;
    CUtensorMap tq, tk, tv;
    int rc = make_map(&tq, q, c.n_q_heads, Nq);
    if (!rc) rc = make_map(&tk, k, c.n_kv_heads, q_start + Nq);
    if (!rc) rc = make_map(&tv, v, c.n_kv_heads, q_start + Nq);
    if (rc) return rc;
    TcArgs a;
    a.out = (__nv_bfloat16 *)out;
    a.mask = p->d_mask;
    a.L = c.n_layers; a.layer = layer; a.req = req; a.Hq = c.n_q_heads; a.G = p->G;
    a.S = c.sink; a.W = c.window; a.q_start = q_start; a.Nq = Nq;
    a.n_qt = (Nq + BM - 1) / BM;
    a.n_kv = c.n_kv_heads;
    a.P = p->G / 2;
    a.odd = p->G & 1;
    a.n_items = a.n_qt * a.n_kv * a.P + a.odd * a.n_kv * ((a.n_qt + 1) / 2);
    const int n_ctas = a.n_items < p->dev.n_sms ? a.n_items : p->dev.n_sms;   // persistent: one CTA per SM
    a.scale_log2 = p->scale_log2;
    a.debug = (int32_t *)(ws + p->lay.debug);
    a.status = (uint32_t *)(ws + p->lay.status);
    a.bm = block_mask;
    a.n_kb = n_kv_blocks;
    a.touch = p->touch;
    const int rec = prof_begin(p, FLUX_KERNEL_PREFILL, st);
    if (block_mask)
        prefill_tc_kernel<kBlocks><<<n_ctas, kThreads, kSmemBytes, st>>>(tq, tk, tv, a, NoPack());
    else
        prefill_tc_kernel<kRouted><<<n_ctas, kThreads, kSmemBytes, st>>>(tq, tk, tv, a, NoPack());
    prof_end(p, rec, st);
    p->launches++;
    if (!block_mask) p->debug_records = 1;
    return check_cuda(cudaGetLastError(), "prefill tensor-core kernel launch");
}

int launch_prefill_packed_nothing(flux_plan *p, int layer, int b0, int n, cudaStream_t st)
{
    skipped_records_kernel<<<1, 128, 0, st>>>((int32_t *)((char *)p->ws + p->lay.debug), layer, b0, n);
    p->launches++;
    return check_cuda(cudaGetLastError(), "skipped records launch");
}

int launch_prefill_packed(flux_plan *p, int layer, int B, const void *q, const void *k, const void *v, int64_t q_stride,
                          int64_t k_stride, int64_t v_stride, const int32_t *q_rows, const int32_t *k_rows, void *out, cudaStream_t st)
{
    const flux_config &c = p->cfg;
    char *ws = (char *)p->ws;
    CUtensorMap tq, tk, tv;
    int rc = make_map(&tq, q, c.n_q_heads, q_rows[B], q_stride);
    if (!rc) rc = make_map(&tk, k, c.n_kv_heads, k_rows[B], k_stride);
    if (!rc) rc = make_map(&tv, v, c.n_kv_heads, k_rows[B], v_stride);
    if (rc) return rc;
    TcArgs a = {};
    a.out = (__nv_bfloat16 *)out;
    a.mask = p->d_mask;
    a.L = c.n_layers; a.layer = layer; a.Hq = c.n_q_heads; a.G = p->G;
    a.S = c.sink; a.W = c.window;
    a.n_kv = c.n_kv_heads;
    a.P = p->G / 2;
    a.odd = p->G & 1;
    a.scale_log2 = p->scale_log2;
    a.debug = (int32_t *)(ws + p->lay.debug);
    a.status = (uint32_t *)(ws + p->lay.status);
    a.touch = p->touch;
    const int per2 = a.n_kv * (2 * a.P + a.odd);
    // Key tiles to walk in all if every request is dense, in units of items (the modes are on the device), and a CTA's share of them.
    // A request whose items are longer than the share is cut into parts of about that length, while there are accumulators.
    double work = 0;
    for (int b = 0; b < B; ++b) {
        const int nq = q_rows[b + 1] - q_rows[b];
        if (nq == 0) continue;
        const int n_qt = (nq + BM - 1) / BM, pairs = (n_qt + 1) / 2, tiles = (k_rows[b + 1] - k_rows[b] + BN - 1) / BN;
        work += (double)(pairs * per2 - (n_qt & 1) * a.n_kv * a.P) * (tiles - pairs + 1);
    }
    const double share = work / p->dev.n_sms;
    const int most_acc = p->dev.n_sms < kPackAccs ? p->dev.n_sms : kPackAccs;     // one wave of parts: a second would cost more than cutting saves
    for (int b = 0; b < B;) {
        PackArgs pk;
        const int b0 = b;
        pk.n = 0;
        int acc = 0;
        int64_t items = 0;
        for (; b < B && pk.n < kPackReqs; ++b) {
            const int nq = q_rows[b + 1] - q_rows[b], nk = nq ? k_rows[b + 1] - k_rows[b] : 0;
            const int n_qt = (nq + BM - 1) / BM, pairs = (n_qt + 1) / 2, tiles = (nk + BN - 1) / BN;
            const int n_acc = pairs * per2 - (n_qt & 1) * a.n_kv * a.P;        // the last pair may lack its second rank
            int parts = nq == 0 ? 1 : parts_of(share * kMaxParts < tiles ? kMaxParts : (int)(tiles / share), tiles, nq);
            if (parts > 1 && (int64_t)acc + (int64_t)n_acc * parts > most_acc) parts = (most_acc - acc) / n_acc;
            if (parts > kPackReqs - pk.n) parts = kPackReqs - pk.n;
            if (parts < 2) parts = 1;
            for (int i = 0; i < parts; ++i) pk.r[pk.n++] = {b, q_rows[b], k_rows[b], nq, nk, i, parts, acc};
            if (parts > 1) acc += n_acc * parts;
            items += (int64_t)n_acc * parts;
        }
        if (items == 0) {
            rc = launch_prefill_packed_nothing(p, layer, b0, b - b0, st);
            if (rc) return rc;
            continue;
        }
        if (items >= (1ll << 30)) return fail(FLUX_E_CAPACITY, "too many query tiles for one call");
        a.n_items = (int)items;
        pk.touch_words = p->touch_words;
        pk.counter = (uint32_t *)(ws + p->lay.pack_counter);
        pk.tickets = pk.counter + 8;
        pk.acc_o = (float4 *)(ws + p->lay.pack_acc);
        pk.acc_ml = (float2 *)(ws + p->lay.pack_acc + (size_t)kPackAccs * 2 * BM * kHeadDim * sizeof(float));
        const int n_ctas = a.n_items < p->dev.n_sms ? a.n_items : p->dev.n_sms;
        const int rec = prof_begin(p, FLUX_KERNEL_PREFILL, st);
        cudaLaunchConfig_t lc = {};
        lc.gridDim = dim3((unsigned)n_ctas);
        lc.blockDim = dim3(kThreads);
        lc.dynamicSmemBytes = kSmemBytes;
        lc.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        lc.attrs = attr;
        lc.numAttrs = 1;
        rc = check_cuda(cudaLaunchKernelEx(&lc, prefill_tc_kernel<kPacked>, tq, tk, tv, a, pk), "packed prefill kernel launch");
        prof_end(p, rec, st);
        p->launches++;
        if (rc) return rc;
    }
    p->debug_records = B;
    return FLUX_OK;
}

}  // namespace flux
