// The 8-bit KV cache: layout, block scales and the two code types.  Shared by the kernels that fill and read
// it (flux_kvq.cu) and the decode kernel that attends over it (flux_decode_kvq.cu).
//
// A cache of one (layer, request) -- K and V each have one -- is a tail followed by tiles:
//   tail   bf16 [Hkv][16][128]: the rows of the newest block while it is incomplete (row = position mod 16)
//   tile t 64 positions: [Hkv][2 strips], padded to 128 bytes; a strip is 32 positions of one head: codes of its 2 blocks
//          (2048 bytes each), their 2 fp32 scales, 8 bytes unused -- one piece for one bulk copy
// A block is 16 positions of one head with one scale; code x scale is the value.  Codes lie in the order in which
// the lanes of an m16n8k16 product take them as the A operand (K: keys x channels, V: channels x keys), so a lane
// of the decode kernel reads its share of a block as 16-byte pieces at lane * 16, piece after piece 512 bytes apart:
// no bank conflicts, no transposition.  With lane = 4 g + t:
//   K block: byte ((2 p + h) * 8 + g) * 64 + 16 t + e   = key g + 8 h, channel 64 p + 16 t + e
//   V block: byte (8 q + g) * 64 + 16 t + 4 e + 2 h + b = channel 32 q + 4 g + e, key 8 h + 2 t + b
// A compact sparse cache (FLUX_KV_COMPACT_SA) keeps its sink tiles in place and the later tiles in a ring of as many tiles as
// a window can touch, the one the newest position is in among them.  A tile is overwritten from the moment the first block of the
// tile one ring later is complete; the window reaches back from there to the tile behind it at most.
#pragma once

#include <cuda_fp16.h>
#include <math_constants.h>

#include "flux_internal.h"

namespace flux {

constexpr int kKvqBlock = 16;                                  // positions per scale
constexpr int kKvqTile = 64;                                   // positions per tile
constexpr int kKvqBlockBytes = kKvqBlock * kHeadDim;           // codes of a block of one head
constexpr int kKvqStrip = 32;                                  // positions of a strip
constexpr int kKvqStripCodes = kKvqStrip * kHeadDim;           // its codes
constexpr int kKvqStripBytes = kKvqStripCodes + 16;            // codes and scales of a strip of one head
constexpr int kKvqTailHeadBytes = kKvqBlock * kRowBytes;       // tail of one head
constexpr float kKvqMinScale = 7.888609052210118e-31f;         // 2^-100: keeps every scale and its inverse a normal number

__host__ __device__ __forceinline__ size_t kvq_tail_bytes(int Hkv) { return (size_t)Hkv * kKvqTailHeadBytes; }
__host__ __device__ __forceinline__ size_t kvq_tile_stride(int Hkv)
{
    return ((size_t)Hkv * 2 * kKvqStripBytes + 127) / 128 * 128;
}
// Strip j / 2 of a head, which holds block j, inside its tile
__host__ __device__ __forceinline__ size_t kvq_strip_at(int head, int j) { return (size_t)(2 * head + (j / 2 & 1)) * kKvqStripBytes; }
__host__ __device__ __forceinline__ int kvq_sink_tiles(int S) { return (S + kKvqTile - 1) / kKvqTile; }
__host__ __device__ __forceinline__ int kvq_ring_tiles(int W) { return (W + kKvqTile - 2) / kKvqTile + 1; }

// Place of tile `tile` in the cache.
__device__ __forceinline__ int kvq_slot(int tile, bool compact, int S, int W)
{
    const int s = kvq_sink_tiles(S);
    return !compact || tile < s ? tile : s + (tile - s) % kvq_ring_tiles(W);
}

// Whether the complete block j of a request of n tokens is still held.
__device__ __forceinline__ bool kvq_held(int j, int n, bool compact, int S, int W)
{
    return !compact || j / 4 < kvq_sink_tiles(S) || j * kKvqBlock + kKvqBlock - 1 >= n - W;
}

// Scale of a block from its largest magnitude (finite, >= 0).
//   e4m3: the smallest power of two that brings amax to 448 or below.  The codes keep four significant bits at every
//         magnitude, so nothing is lost to the power of two, and x / scale is exact: code = x / scale rounded once.  At most 2^119,
//         so that every value stays finite: entries beyond 448 * 2^119 (the top eighth of the largest binade) become that.
//   int8: amax / 127 rounded to fp32, so the largest value gets the largest code (a power of two would cost up to one bit).
// At least 2^-100, which is what a block of zeros is held with: its values are zeros under any scale, but the scale enters the decode's
// weights, and one of 1 would put it far above blocks of small values (V of size 2^-30 behind such a block came out as zeros).
template <int kFmt>
__device__ __forceinline__ float kvq_scale(float amax)
{
    if (kFmt == FLUX_KVQ_INT8) return fmaxf(__fdiv_rn(amax, 127.f), kKvqMinScale);
    // amax = 1.f * 2^x; 448 = 1.75 * 2^8
    const uint32_t u = __float_as_uint(amax);
    int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < -100 ? -100 : e > 119 ? 119 : e;
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Four bf16 values (channels 0, 1 in w01, 2, 3 in w23) to four codes.  inv = 1 / s (exact for e4m3).
template <int kFmt>
__device__ __forceinline__ uint32_t kvq_encode4(uint32_t w01, uint32_t w23, float s, float inv)
{
    if (kFmt == FLUX_KVQ_INT8) {
        const float x[4] = {__uint_as_float(w01 << 16), __uint_as_float(w01 & 0xffff0000u), __uint_as_float(w23 << 16),
                            __uint_as_float(w23 & 0xffff0000u)};
        // x * inv is within 2^-23 of the quotient, relatively (127 * 2^-23 = 2^-16 at most): adding 1.5 * 2^23 rounds it to the
        // nearest integer (ties to even), which stands in the low bits, unless it is that near the middle of two
        constexpr float kMagic = 12582912.f;
        uint32_t t[4];
        bool near = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float y = fmaf(x[i], inv, kMagic);
            t[i] = __float_as_uint(y);
            near = near || fabsf(fmaf(x[i], inv, -(y - kMagic))) > 0.5f - 6.2e-5f;      // 2^-14
        }
        if (near) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float y = __fdiv_rn(x[i], s);
                float r = rintf(y);
                if (fabsf(y - truncf(y)) == 0.5f) {       // rounded onto the middle: the remainder says on which side the quotient lies
                    const float rem = fmaf(-y, s, x[i]);
                    if (rem > 0.f) r = ceilf(y);
                    if (rem < 0.f) r = floorf(y);
                }
                t[i] = (uint32_t)(int)r;
            }
        }
        // |x| <= amax and s >= amax (1 - 2^-24) / 127: the codes are within +-127.  Held with an offset of 128.
        const uint32_t lo = __byte_perm(t[0], t[1], 0x0040), hi = __byte_perm(t[2], t[3], 0x0040);
        return __byte_perm(lo, hi, 0x5410) ^ 0x80808080u;
    }
    // the product with a power of two is exact in bf16 but below 2^-126, where the code is 0 either way
    const __nv_bfloat162 f = __float2bfloat162_rn(inv);
    __nv_bfloat162 a = __hmul2(*reinterpret_cast<__nv_bfloat162 *>(&w01), f), b = __hmul2(*reinterpret_cast<__nv_bfloat162 *>(&w23), f);
    const uint32_t ua = *reinterpret_cast<uint32_t *>(&a), ub = *reinterpret_cast<uint32_t *>(&b);
    uint32_t w;
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(w) : "f"(__uint_as_float(ua << 16)), "f"(__uint_as_float(ua & 0xffff0000u)), "f"(__uint_as_float(ub << 16)),
                    "f"(__uint_as_float(ub & 0xffff0000u)));
    return w;
}

// NaN and infinities become 0: one of them must not reach the other positions of its block, nor (as 0 x inf) rows that mask it.
__device__ __forceinline__ uint32_t kvq_finite2(uint32_t w, bool &bad)
{
    if ((w & 0x7f80u) == 0x7f80u) {
        bad = true;
        w &= 0xffff0000u;
    }
    if ((w & 0x7f800000u) == 0x7f800000u) {
        bad = true;
        w &= 0x0000ffffu;
    }
    return w;
}

// Byte c of the four words becomes word c (a 4 x 4 byte transposition).
__device__ __forceinline__ uint4 transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint32_t ab0 = __byte_perm(a, b, 0x5140), ab1 = __byte_perm(a, b, 0x7362);   // a0 b0 a1 b1 | a2 b2 a3 b3
    const uint32_t cd0 = __byte_perm(c, d, 0x5140), cd1 = __byte_perm(c, d, 0x7362);
    return make_uint4(__byte_perm(ab0, cd0, 0x5410), __byte_perm(ab0, cd0, 0x7632), __byte_perm(ab1, cd1, 0x5410),
                      __byte_perm(ab1, cd1, 0x7632));
}

// The lane's share of a block (channels 4 lane .. + 3 of 16 rows) with NaN and infinities cleared; true if there were any in
// the warp's block.  Largest magnitude: two bf16 bit patterns at a time (0x7f80 and above: infinite or NaN).
__device__ __forceinline__ uint32_t kvq_largest(const uint2 (&x)[kKvqBlock])
{
    uint32_t two = 0;
#pragma unroll
    for (int i = 0; i < kKvqBlock; ++i) two = __vmaxu2(two, __vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu));
    return __reduce_max_sync(0xffffffffu, max(two & 0xffffu, two >> 16));
}
__device__ __forceinline__ bool kvq_finite(uint2 (&x)[kKvqBlock])
{
    if (kvq_largest(x) < 0x7f80u) return false;
    bool bad = true;
#pragma unroll
    for (int i = 0; i < kKvqBlock; ++i) {
        x[i].x = kvq_finite2(x[i].x, bad);
        x[i].y = kvq_finite2(x[i].y, bad);
    }
    return true;
}

// Scale and codes of the warp's block (finite values): w[i] holds the lane's four channels of row i.
template <int kFmt>
__device__ __forceinline__ float kvq_encode_block(const uint2 (&x)[kKvqBlock], uint32_t (&w)[kKvqBlock])
{
    const float s = kvq_scale<kFmt>(__uint_as_float(kvq_largest(x) << 16)), inv = __fdiv_rn(1.f, s);
#pragma unroll
    for (int i = 0; i < kKvqBlock; ++i) w[i] = kvq_encode4<kFmt>(x[i].x, x[i].y, s, inv);
    return s;
}

// The warp's codes to a block's place (global or shared memory), in the order of K (kv 0) or V (kv 1).
__device__ __forceinline__ void kvq_put_block(unsigned char *blk, const uint32_t (&w)[kKvqBlock], int kv, int lane)
{
    if (kv == 0) {
#pragma unroll
        for (int i = 0; i < kKvqBlock; ++i)      // key i = g + 8 h
            *reinterpret_cast<uint32_t *>(blk + ((2 * (lane >> 4) + (i >> 3)) * 8 + (i & 7)) * 64 + (lane & 15) * 4) = w[i];
    } else {
#pragma unroll
        for (int t = 0; t < 4; ++t)              // channels 4 lane .. + 3, keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
            *reinterpret_cast<uint4 *>(blk + lane * 64 + t * 16) = transpose4(w[2 * t], w[2 * t + 1], w[2 * t + 8], w[2 * t + 9]);
    }
}

// Four codes to two pairs of fp16 (both types are exact in fp16): bytes 0, 1 -> lo, bytes 2, 3 -> hi.
template <int kFmt>
__device__ __forceinline__ void kvq_decode4(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    if (kFmt == FLUX_KVQ_INT8) {
        // 0x64uu is 1024 + u in fp16; the code is u - 128
        const __half2 off = __floats2half2_rn(1152.f, 1152.f);
        uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
        __half2 ha = __hsub2(*reinterpret_cast<__half2 *>(&a), off), hb = __hsub2(*reinterpret_cast<__half2 *>(&b), off);
        lo = *reinterpret_cast<uint32_t *>(&ha);
        hi = *reinterpret_cast<uint32_t *>(&hb);
    } else {
        asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
            : "=r"(lo), "=r"(hi) : "r"(w));
    }
}

// Four codes under scale s to two words of bf16 pairs (code x s in fp32, rounded once).
template <int kFmt>
__device__ __forceinline__ uint2 kvq_values4(uint32_t w, float s)
{
    float x[4];
    if (kFmt == FLUX_KVQ_INT8) {
        // 0x4b0000uu is 2^23 + u
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 + i)) - 8388736.f) * s;
    } else {
        uint32_t lo, hi;
        kvq_decode4<kFmt>(w, lo, hi);
        const float2 fl = __half22float2(*reinterpret_cast<__half2 *>(&lo)), fh = __half22float2(*reinterpret_cast<__half2 *>(&hi));
        x[0] = fl.x * s; x[1] = fl.y * s; x[2] = fh.x * s; x[3] = fh.y * s;
    }
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    return make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}

}  // namespace flux
