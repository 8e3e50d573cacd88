// Norm of a head and rotation by its position, shared by the kernel over rows (flux_paged.cu) and the decode step
// (flux_decode_paged.cu), so that both give the same bits.
//
//   y = x w / sqrt(mean(x^2) + eps) over the 128 channels of a head (w: weight + offset; left out without a weight), then
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t) scale for the pairs of the first `rot` channels, t = 2 pi (pos f mod 1).
//
// f is held as a 64-bit fraction of a turn per position, so pos f mod 1 is one integer product that wraps: no angle ever has to be
// brought back into range, and position 10^6 is as exact as position 1 (of a turn, below 2^-34 from f at up to 2^31 positions and 2^-32
// from leaving out the product's low word; the rounding of the fraction to fp32, 2^-25 of half a turn, is what counts).
//
// Eight lanes take a head, each with eight pairs as two pieces of eight channels: of halves (i, i + rot / 2), of neighbours
// (2 i, 2 i + 1), and of what is not rotated any two.  So a pair never leaves its lane, whatever rot is (a multiple of 16), a
// piece is one 16-byte load, and the norm takes three shuffles.  Arithmetic in fp32, rounded once to bf16.  (Sixteen lanes with
// pieces of four channels: 150 instructions for two heads, issue slots 67 % used at 77 % of the copy bandwidth.  Two products an
// instruction, fma.rn.f32x2: 91 us instead of 87.6 for 24K rows, the pairs of registers cost more than they save.)
#pragma once

#include "flux_internal.h"
#include "flux_mma_util.h"

namespace flux {

constexpr int kHeadLanes = 8;        // lanes that share a head

struct RopeArgs {
    const __nv_bfloat16 *weight[2];  // of query and key heads, NULL: no norm
    const uint64_t *freqs;           // [rot / 2]
    float eps, offset, scale;
    int rot, pairs;                  // pairs: of neighbouring channels
};

// two pairs at a time
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return make_float2(a.x * b.x, a.y * b.y); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }

// Two pieces of a lane, and its eight pairs (a of pairs 2 j, 2 j + 1 in a[j]).
struct Pieces {
    uint4 a, b;
};
struct Pairs {
    float2 a[4], b[4];
};
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ Pairs to_pairs(const Pieces &p, bool neighbours)
{
    Pairs x;
    if (neighbours) {
        x.a[0] = make_float2(low(p.a.x), low(p.a.y)); x.b[0] = make_float2(high(p.a.x), high(p.a.y));
        x.a[1] = make_float2(low(p.a.z), low(p.a.w)); x.b[1] = make_float2(high(p.a.z), high(p.a.w));
        x.a[2] = make_float2(low(p.b.x), low(p.b.y)); x.b[2] = make_float2(high(p.b.x), high(p.b.y));
        x.a[3] = make_float2(low(p.b.z), low(p.b.w)); x.b[3] = make_float2(high(p.b.z), high(p.b.w));
    } else {
        x.a[0] = make_float2(low(p.a.x), high(p.a.x)); x.b[0] = make_float2(low(p.b.x), high(p.b.x));
        x.a[1] = make_float2(low(p.a.y), high(p.a.y)); x.b[1] = make_float2(low(p.b.y), high(p.b.y));
        x.a[2] = make_float2(low(p.a.z), high(p.a.z)); x.b[2] = make_float2(low(p.b.z), high(p.b.z));
        x.a[3] = make_float2(low(p.a.w), high(p.a.w)); x.b[3] = make_float2(low(p.b.w), high(p.b.w));
    }
    return x;
}
__device__ __forceinline__ Pieces to_pieces(const Pairs &y, bool neighbours)
{
    if (neighbours)
        return {make_uint4(pack_bf16(y.a[0].x, y.b[0].x), pack_bf16(y.a[0].y, y.b[0].y), pack_bf16(y.a[1].x, y.b[1].x), pack_bf16(y.a[1].y, y.b[1].y)),
                make_uint4(pack_bf16(y.a[2].x, y.b[2].x), pack_bf16(y.a[2].y, y.b[2].y), pack_bf16(y.a[3].x, y.b[3].x), pack_bf16(y.a[3].y, y.b[3].y))};
    return {make_uint4(pack_bf16(y.a[0].x, y.a[0].y), pack_bf16(y.a[1].x, y.a[1].y), pack_bf16(y.a[2].x, y.a[2].y), pack_bf16(y.a[3].x, y.a[3].y)),
            make_uint4(pack_bf16(y.b[0].x, y.b[0].y), pack_bf16(y.b[1].x, y.b[1].y), pack_bf16(y.b[2].x, y.b[2].y), pack_bf16(y.b[3].x, y.b[3].y))};
}

// Where a lane's two pieces are in a head, and the sines of its pairs.
struct RopeLane {
    int a, b;                        // first channel of either piece
    bool still;                      // they lie behind the rotated channels
    float2 c[4], s[4];
    __device__ __forceinline__ void place(const RopeArgs &r, int lane)
    {
        const int h = lane & (kHeadLanes - 1), half = r.rot / 2;
        still = 8 * h >= half;
        if (r.pairs) {
            a = 16 * h;
            b = a + 8;
        } else if (!still) {
            a = 8 * h;
            b = a + half;
        } else {
            a = half + 8 * h;
            b = a + kHeadDim / 2 - half;
        }
    }
    // The four heads of a warp have the same sines: each of the four lanes that need a pair's finds two of its eight.
    __device__ __forceinline__ void sines(const RopeArgs &r, const struct RopeFreqs &k, int lane, int pos);
    __device__ __forceinline__ Pieces load(const unsigned char *head) const
    {
        return {*reinterpret_cast<const uint4 *>(head + a * 2), *reinterpret_cast<const uint4 *>(head + b * 2)};
    }
    __device__ __forceinline__ void store(unsigned char *head, const Pieces &p) const
    {
        *reinterpret_cast<uint4 *>(head + a * 2) = p.a;
        *reinterpret_cast<uint4 *>(head + b * 2) = p.b;
    }
};

// What a lane needs of the arguments whatever the row: its two frequencies, and its weights.
struct RopeFreqs {
    uint64_t f[2];
    __device__ __forceinline__ void read(const RopeArgs &r, int lane)
    {
        const int i = 8 * (lane & (kHeadLanes - 1)) + 2 * (lane / kHeadLanes);
        f[0] = f[1] = 0;
        if (i < r.rot / 2) {
            f[0] = r.freqs[i];
            f[1] = r.freqs[i + 1];
        }
    }
};
__device__ __forceinline__ Pieces rope_weights(const __nv_bfloat16 *weight, const RopeLane &l)
{
    return weight != nullptr ? l.load(reinterpret_cast<const unsigned char *>(weight)) : Pieces{};
}

__device__ __forceinline__ void RopeLane::sines(const RopeArgs &r, const RopeFreqs &k, int lane, int pos)
{
    const int i = 8 * (lane & (kHeadLanes - 1)) + 2 * (lane / kHeadLanes);
    float cos[2] = {1.f, 1.f}, sin[2] = {0.f, 0.f};
    if (i < r.rot / 2) {
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            const uint64_t part = (uint64_t)(int64_t)pos * k.f[z];
            sincospif((float)(int32_t)(part >> 32) * 0x1p-31f, &sin[z], &cos[z]);
            sin[z] *= r.scale;
            cos[z] *= r.scale;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int from = (lane & (kHeadLanes - 1)) + kHeadLanes * j;
        c[j] = make_float2(__shfl_sync(0xffffffffu, cos[0], from), __shfl_sync(0xffffffffu, cos[1], from));
        s[j] = make_float2(__shfl_sync(0xffffffffu, sin[0], from), __shfl_sync(0xffffffffu, sin[1], from));
    }
}

// What turns the pairs of a lane, weights folded in: y_a = (x_a ca + x_b sb) inv, y_b = (x_b cb + x_a sa) inv.  Behind the rotated channels
// y_a = x_a ca inv, y_b = x_b cb inv: two of them are no pair, and a zero times an infinity or a NaN would carry it into the other one.
// (The selects cost 24K rows of 128 rotated channels 2 us of 83, so those go without; of 64 rotated ones, 85.7 us instead of 83.2.)
struct RopeFactors {
    float2 ca[4], sb[4], cb[4], sa[4];
    bool whole, still;               // the same in all lanes: every channel is rotated; this lane's are not
    // weights: this lane's pieces of them, if there are any
    __device__ __forceinline__ void fold(const RopeArgs &r, const RopeLane &l, bool weighted, const Pieces &weights)
    {
        whole = r.rot == kHeadDim;
        still = l.still;
        Pairs w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w.a[j] = w.b[j] = make_float2(1.f, 1.f);
        if (weighted) {
            w = to_pairs(weights, r.pairs != 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w.a[j].x += r.offset; w.a[j].y += r.offset;
                w.b[j].x += r.offset; w.b[j].y += r.offset;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            ca[j] = mul2(l.c[j], w.a[j]);
            sb[j] = mul2(make_float2(-l.s[j].x, -l.s[j].y), w.b[j]);
            cb[j] = mul2(l.c[j], w.b[j]);
            sa[j] = mul2(l.s[j], w.a[j]);
        }
    }
    // One head over its eight lanes (every lane of the warp takes part).
    __device__ __forceinline__ Pairs turn(const Pieces &p, bool neighbours, bool norm, float eps) const
    {
        const Pairs x = to_pairs(p, neighbours);
        float inv = 1.f;
        if (norm) {
            float2 two = mul2(x.a[0], x.a[0]);
#pragma unroll
            for (int j = 1; j < 4; ++j) two = fma2(x.a[j], x.a[j], two);
#pragma unroll
            for (int j = 0; j < 4; ++j) two = fma2(x.b[j], x.b[j], two);
            float sum = two.x + two.y;
#pragma unroll
            for (int d = kHeadLanes / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            inv = rsqrtf(fmaf(sum, 1.f / kHeadDim, eps));
        }
        const float2 both = make_float2(inv, inv);
        Pairs y;
        if (whole) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y.a[j] = mul2(fma2(x.a[j], ca[j], mul2(x.b[j], sb[j])), both);
                y.b[j] = mul2(fma2(x.b[j], cb[j], mul2(x.a[j], sa[j])), both);
            }
            return y;
        }
        auto other = [&](float2 v, float2 f) { return still ? make_float2(0.f, 0.f) : mul2(v, f); };
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            y.a[j] = mul2(fma2(x.a[j], ca[j], other(x.b[j], sb[j])), both);
            y.b[j] = mul2(fma2(x.b[j], cb[j], other(x.a[j], sa[j])), both);
        }
        return y;
    }
};

}  // namespace flux
