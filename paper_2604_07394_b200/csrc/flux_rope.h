// Norm of a head and rotation by its position, shared by the kernel over rows (flux_paged.cu) and the decode step
// (flux_decode_paged.cu), so that both give the same bits.
//
//   y = x w / sqrt(mean(x^2) + eps) over the 128 channels of a head (w: weight + offset; left out without a weight), then
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t) scale for the pairs of the first `rot` channels, t = 2 pi (pos f mod 1).
//
// f is held as a 64-bit fraction of a turn per position, so pos f mod 1 is one integer product that wraps: no angle ever has to be
// brought back into range, and position 10^6 is as exact as position 1 (error below 2^-33 of a turn up to 2^31 positions; the
// rounding of the fraction to fp32, 2^-25 of half a turn, is what remains).
//
// Sixteen lanes take a head, each with four pairs as two pieces of four channels: of halves (i, i + rot / 2), of neighbours
// (2 i, 2 i + 1), and of what is not rotated any two.  So a pair never leaves its lane, whatever rot is (a multiple of 8),
// and a piece is one 8-byte load.  All in fp32, rounded once to bf16.
#pragma once

#include "flux_internal.h"
#include "flux_mma_util.h"

namespace flux {

struct RopeArgs {
    const __nv_bfloat16 *weight[2];  // of query and key heads, NULL: no norm
    const uint64_t *freqs;           // [rot / 2]
    float eps, offset, scale;
    int rot, pairs;                  // pairs: of neighbouring channels
};

// Where a lane's two pieces are in a head, and what turns them: with the weights folded in,
// y_a = (x_a ca - x_b sb) inv, y_b = (x_b cb + x_a sa) inv.
struct RopeLane {
    int a, b;                        // first channel of either piece
    float c[4], s[4];
    __device__ __forceinline__ void place(const RopeArgs &r, int lane)
    {
        const int h = lane & 15, half = r.rot / 2;
        if (r.pairs) {
            a = 8 * h;
            b = a + 4;
        } else if (4 * h < half) {
            a = 4 * h;
            b = a + half;
        } else {                     // behind the rotated channels
            a = half + 4 * h;
            b = a + kHeadDim / 2 - half;
        }
    }
    __device__ __forceinline__ void turn(const RopeArgs &r, int lane, int pos)
    {
        const int i = 4 * (lane & 15);
        const bool live = i < r.rot / 2;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            c[k] = 1.f;
            s[k] = 0.f;
            if (live) {
                const uint64_t part = (uint64_t)(int64_t)pos * r.freqs[i + k];
                sincospif((float)(int32_t)(part >> 32) * 0x1p-31f, &s[k], &c[k]);
                s[k] *= r.scale;
                c[k] *= r.scale;
            }
        }
    }
};

struct RopeFactors {
    float ca[4], sb[4], cb[4], sa[4];
    __device__ __forceinline__ void fold(const RopeArgs &r, const RopeLane &l, int which)
    {
        float wa[4] = {1.f, 1.f, 1.f, 1.f}, wb[4] = {1.f, 1.f, 1.f, 1.f};
        if (r.weight[which] != nullptr) {
            const uint2 pa = *reinterpret_cast<const uint2 *>(r.weight[which] + l.a), pb = *reinterpret_cast<const uint2 *>(r.weight[which] + l.b);
            spread(pa, pb, r.pairs, wa, wb);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                wa[k] += r.offset;
                wb[k] += r.offset;
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            ca[k] = l.c[k] * wa[k];
            sb[k] = l.s[k] * wb[k];
            cb[k] = l.c[k] * wb[k];
            sa[k] = l.s[k] * wa[k];
        }
    }
    // the four pairs of two pieces
    static __device__ __forceinline__ void spread(uint2 pa, uint2 pb, int pairs, float (&xa)[4], float (&xb)[4])
    {
        const uint32_t lo0 = pairs ? __byte_perm(pa.x, pa.y, 0x5410) : pa.x, lo1 = pairs ? __byte_perm(pb.x, pb.y, 0x5410) : pa.y;
        const uint32_t hi0 = pairs ? __byte_perm(pa.x, pa.y, 0x7632) : pb.x, hi1 = pairs ? __byte_perm(pb.x, pb.y, 0x7632) : pb.y;
        xa[0] = __uint_as_float(lo0 << 16); xa[1] = __uint_as_float(lo0 & 0xffff0000u);
        xa[2] = __uint_as_float(lo1 << 16); xa[3] = __uint_as_float(lo1 & 0xffff0000u);
        xb[0] = __uint_as_float(hi0 << 16); xb[1] = __uint_as_float(hi0 & 0xffff0000u);
        xb[2] = __uint_as_float(hi1 << 16); xb[3] = __uint_as_float(hi1 & 0xffff0000u);
    }
    // One head over its sixteen lanes (every lane of the warp takes part): its four pairs, fp32.
    __device__ __forceinline__ void turn(uint2 pa, uint2 pb, int pairs, bool norm, float eps, float (&ya)[4], float (&yb)[4]) const
    {
        float xa[4], xb[4];
        spread(pa, pb, pairs, xa, xb);
        float inv = 1.f;
        if (norm) {
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) sum = fmaf(xa[k], xa[k], fmaf(xb[k], xb[k], sum));
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            inv = rsqrtf(fmaf(sum, 1.f / kHeadDim, eps));
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            ya[k] = (xa[k] * ca[k] - xb[k] * sb[k]) * inv;
            yb[k] = (xb[k] * cb[k] + xa[k] * sa[k]) * inv;
        }
    }
    // Pairs back into pieces.  rest: what the rounding leaves over, for a second call with what it leaves.
    static __device__ __forceinline__ void gather(float (&ya)[4], float (&yb)[4], int pairs, uint2 &pa, uint2 &pb, bool rest = false)
    {
        uint32_t y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            y[k] = pack_bf16(ya[k], yb[k]);
            if (rest) {
                ya[k] -= __uint_as_float(y[k] << 16);
                yb[k] -= __uint_as_float(y[k] & 0xffff0000u);
            }
        }
        if (pairs) {
            pa = make_uint2(y[0], y[1]);
            pb = make_uint2(y[2], y[3]);
        } else {
            pa = make_uint2(__byte_perm(y[0], y[1], 0x5410), __byte_perm(y[2], y[3], 0x5410));
            pb = make_uint2(__byte_perm(y[0], y[1], 0x7632), __byte_perm(y[2], y[3], 0x7632));
        }
    }
    // pieces in, pieces out
    __device__ __forceinline__ void apply(uint2 &pa, uint2 &pb, int pairs, bool norm, float eps) const
    {
        float ya[4], yb[4];
        turn(pa, pb, pairs, norm, eps, ya, yb);
        gather(ya, yb, pairs, pa, pb);
    }
};

}  // namespace flux
