// What lies between the QKV projection and the cache: RMS norms of queries and keys for each head, the position rotation, and
// the append of the rotated keys and the values to the BF16 or the 4-bit paged cache; and the read-back of the 4-bit cache.
//
//     y = x rsqrt(mean_i x_i^2 + eps) w                      per head, where a weight is given
//     (a, b) -> A (a cos t - b sin t, b cos t + a sin t)     t = position * inv_freq, in binary64
//     4 bits: zero = bf16(min), scale = bf16((max - zero) * (1/15)), code = clamp(rint((x - zero) / scale), 0, 15) per 64 channels
//
// Every call moves each element once, so it is bound by memory where it is long and by latency where it is short.  A row (one
// head of one token) belongs to D / 16 lanes with two units of 8 channels each (two 16-byte loads); with rotation by halves the
// two units are a unit and its partner, so that no value crosses lanes but in the sums and minima.  A warp takes the rows of one
// token (few tokens: several warps a part of them each): every row of a lane then meets the same eight angles, which stay in
// registers, and nothing waits for another warp.
//
// B200, of 6.56 TB/s of measured copy bandwidth: norms and rotation alone, 16384 tokens, 64 / 8 heads, d = 64, 51.5 us, 89 %; append of 8191
// tokens to the BF16 cache 33 us, 77 % (two waves of blocks); one token 2.0 us behind another call; read-back of 24575 rows of 8 heads,
// d = 128, 25.8 us, 76 %.  Registers are what occupancy hangs on: seven blocks of 128 threads (five with the 4-bit quantiser) beat
// six and eight, and a block of four tokens with tables in shared memory took 61 us for the first of these.
#include <math_constants.h>

#include "novakv_int4.cuh"
#include "novakv_ops.cuh"

namespace {

constexpr int ROT_THREADS = 128;
enum { DST_ROWS, DST_BF16, DST_INT4 };       // k goes to rows, to the BF16 pool, to the 4-bit pool

struct RotateArgs {
    const __nv_bfloat16 *q, *k, *v;
    long long q_stride, k_stride, v_stride, q_out_stride, k_out_stride;    // elements from token to token
    __nv_bfloat16 *q_out, *k_out;
    const int32_t *tok_seq, *tok_pos;
    int n_tokens, hq, hkv, parts;            // parts: warps of a token
    const float* inv_freq;
    const __nv_bfloat16 *q_weight, *k_weight;
    float eps, amplitude;
    int rot_dim;
    uint8_t *k_pages, *v_pages;              // (the BF16 pools too)
    int n_pages, max_pages_per_seq, n_seq;
    const int32_t* page_table;
    int32_t* seq_lens;
    uint32_t* dev_status;
};

template <bool VEC>
__device__ __forceinline__ uint4 load_unit(const __nv_bfloat16* p) {
    uint4 r;
    if (VEC) {
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    } else {
        const unsigned short* s = reinterpret_cast<const unsigned short*>(p);
        r.x = s[0] | (uint32_t)s[1] << 16; r.y = s[2] | (uint32_t)s[3] << 16;
        r.z = s[4] | (uint32_t)s[5] << 16; r.w = s[6] | (uint32_t)s[7] << 16;
    }
    return r;
}
template <bool VEC>
__device__ __forceinline__ void store_unit(__nv_bfloat16* p, uint4 r) {
    if (VEC) {
        *reinterpret_cast<uint4*>(p) = r;
    } else {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
        unsigned short* s = reinterpret_cast<unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = (unsigned short)(w[i / 2] >> (16 * (i & 1)));
    }
}
__device__ __forceinline__ void unpack_unit(uint4 r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint4 pack_unit(const float (&x)[8]) {
    return make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
}
// two binary32 numbers side by side: one instruction does both (the append is bound by their number)
struct Two {
    uint64_t v;
    __device__ __forceinline__ Two() = default;
    __device__ __forceinline__ Two(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); }
    __device__ __forceinline__ void get(float& lo, float& hi) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
};
__device__ __forceinline__ Two operator+(Two a, Two b) { Two d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v)); return d; }
__device__ __forceinline__ Two operator-(Two a, Two b) { Two d; asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v)); return d; }
__device__ __forceinline__ Two operator*(Two a, Two b) { Two d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v)); return d; }
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) { Two d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return d; }

// minimum and maximum that keep a NaN: a group that holds one gets it as its zero
__device__ __forceinline__ float min_nan(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float min_nan(float a, float b, float c) { float r; asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
__device__ __forceinline__ float max_nan(float a, float b, float c) { float r; asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }

// What a lane knows of its token and layer: (cos, sin) of its eight pairs - (x_i, y_i), or neighbours (IL) x_2i, x_2i+1 for i < 4
// and y_2i-8, y_2i-7 - and its channels' weights as they are given.  (The weights taken into the cosines would save an eighth of
// the instructions, and cost the registers of two more blocks an SM: a prompt of 16384 tokens, d = 64, 51.5 against 56 us.)
struct Turn {
    float c[8], s[8];
    uint4 wx, wy;
    bool norm;
};
// the angle of a lane's pair i
template <bool IL>
__device__ __forceinline__ int angle_of(int i, int ua, int ub) { return !IL ? 8 * ua + i : i < 4 ? 4 * ua + i : 4 * ub + i - 4; }
template <bool IL>
__device__ __forceinline__ float& first_of(int i, float (&x)[8], float (&y)[8]) { return !IL ? x[i] : i < 4 ? x[2 * i] : y[2 * i - 8]; }
template <bool IL>
__device__ __forceinline__ float& second_of(int i, float (&x)[8], float (&y)[8]) { return !IL ? y[i] : i < 4 ? x[2 * i + 1] : y[2 * i - 7]; }

// norm and rotation of a row's two units.  All lanes of the warp take part.  False (PACKED alone) where the sum of squares leaves
// the range in which its roundings are relative ones.
// PACKED: two numbers an instruction, for the kernel that is bound by instructions; where memory is the bound its registers cost
// more than it saves (16384 tokens, d = 64: 51.4 against 53.8 us).
template <int D, bool IL, bool PACKED>
__device__ __forceinline__ bool transform_row(const RotateArgs& a, const Turn& turn, int ua, int ub, float (&x)[8], float (&y)[8]) {
    constexpr int LANES = D / 16;
    bool fine = true;
    if constexpr (PACKED) {
        Two p[4], q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { p[i] = Two(x[2 * i], x[2 * i + 1]); q[i] = Two(y[2 * i], y[2 * i + 1]); }
        if (turn.norm) {
            Two s0(0.f, 0.f), s1(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) { s0 = fma2(p[i], p[i], s0); s1 = fma2(q[i], q[i], s1); }
            float ss, st;
            (s0 + s1).get(ss, st);
            ss += st;
#pragma unroll
            for (int s = 1; s < LANES; s <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, s);
            const float r = rsqrtf(fmaf(ss, 1.f / D, a.eps));
            fine = ss > 1e-30f && ss < 1e30f;
            const Two rr(r, r);
            float w[8];
            unpack_unit(turn.wx, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = p[i] * (rr * Two(w[2 * i], w[2 * i + 1]));
            unpack_unit(turn.wy, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = q[i] * (rr * Two(w[2 * i], w[2 * i + 1]));
        }
        // (what is not rotated is left alone: infinity times 0 would be NaN)
        if (!IL && 8 * ua < a.rot_dim) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Two c(turn.c[2 * i], turn.c[2 * i + 1]), s(turn.s[2 * i], turn.s[2 * i + 1]);
                const Two u = p[i] * c - q[i] * s;
                q[i] = fma2(p[i], s, q[i] * c);
                p[i] = u;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) { p[i].get(x[2 * i], x[2 * i + 1]); q[i].get(y[2 * i], y[2 * i + 1]); }
    } else if (turn.norm) {
        float ss = 0.f, st = 0.f, w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) { ss = fmaf(x[i], x[i], ss); st = fmaf(y[i], y[i], st); }
        ss += st;
#pragma unroll
        for (int s = 1; s < LANES; s <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, s);
        const float r = rsqrtf(fmaf(ss, 1.f / D, a.eps));
        unpack_unit(turn.wx, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= r * w[i];
        unpack_unit(turn.wy, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] *= r * w[i];
    }
    if (IL || !PACKED) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (8 * (IL && i >= 4 ? ub : ua) >= a.rot_dim) continue;
            float &e = first_of<IL>(i, x, y), &f = second_of<IL>(i, x, y);
            const float u = e * turn.c[i] - f * turn.s[i];
            f = f * turn.c[i] + e * turn.s[i];
            e = u;
        }
    }
    return fine;
}

// Quotients by one scale.  With r the nearest number to 1 / s and q0 = x r, q0 + (x - q0 s) r with fused multiply-adds is the
// nearest number to x / s (P. Markstein, 1990) while nothing overflows or underflows; groups out of that range are divided.
struct Divisor {
    float s, r;
    __device__ __forceinline__ explicit Divisor(float scale) : s(scale), r(1.f / scale) {}
    __device__ __forceinline__ Two quotient(Two x) const {
        const Two rr(r, r), q0 = x * rr;
        return fma2(fma2(q0, Two(-s, -s), x), rr, q0);
    }
};
constexpr float ROUND = 12582912.f;          // 1.5 2^23: added and taken away again it leaves the nearest integer, ties to even

// Codes and pairs of a row.  All lanes of the warp take part.
// A value row is given exactly.  A key (KEY) is defined by binary64, but formed in binary32 first: each element is off by less
// than 2^-19 (|a| + |b|) of the pair it comes from (a mean of D squares and its root 14 roundings of 2^-24, cos and sin 5, far
// positions 4, the root's product with weight and element 2, two products and a sum 3: less than 32), which is at most sqrt(2) times that of the
// pair it gives.  Where no element, minimum or maximum can have crossed a border of its rounding by that, codes and pairs are
// those of the binary64 key; else the answer is false, and the row is formed again in binary64: 0.9 % of the rows, 3 % of the
// warps' four.  (In binary64 throughout, a prompt of 16384 tokens and 32 / 8 heads of d = 128 took 158 us where this takes 91;
// its floor is 57, what bounds it is instructions: 3700 a token, some 1400 of them for the queries.)
template <int D, bool KEY>
struct Quantised {
    uint32_t wx, wy;
    float zero[I4Layout<D>::GROUPS], scale[I4Layout<D>::GROUPS];

    // APART: the units lie in a group each (d = 64: in the one there is)
    template <bool INTERLEAVED, bool APART>
    __device__ __forceinline__ bool form(int ua, int ub, const float (&x)[8], const float (&y)[8]) {
        constexpr int G = I4Layout<D>::GROUPS, LANES = D / 16;
        constexpr float OFF = 2.75e-6f;                           // sqrt(2) 2^-19 = 2.70e-6
        bool sure = true, ranged = true;
        float dx[8], dy[8];
        float xl, xh, yl, yh, xl2 = 0.f, xh2 = 0.f, yl2 = 0.f, yh2 = 0.f;
        if (!KEY) {
            extremes(x, xl, xh);
            extremes(y, yl, yh);
        } else {
            float ux[8], uy[8], lx[8], ly[8];                     // upper and lower ends
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dx[i] = OFF * (fabsf(x[i]) + fabsf(INTERLEAVED ? x[i ^ 1] : y[i]));
                dy[i] = INTERLEAVED ? OFF * (fabsf(y[i]) + fabsf(y[i ^ 1])) : dx[i];
            }
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const Two x2(x[i], x[i + 1]), y2(y[i], y[i + 1]), dx2(dx[i], dx[i + 1]), dy2(dy[i], dy[i + 1]);
                (x2 + dx2).get(ux[i], ux[i + 1]); (y2 + dy2).get(uy[i], uy[i + 1]);
                (x2 - dx2).get(lx[i], lx[i + 1]); (y2 - dy2).get(ly[i], ly[i + 1]);
            }
            extremes(ux, xl, xh); extremes(uy, yl, yh);
            extremes(lx, xl2, xh2); extremes(ly, yl2, yh2);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const bool xin = G == 1 || (APART ? g == 0 : ua / 8 == g), yin = G == 1 || (APART ? g == 1 : ub / 8 == g);
            float lo = min_nan(xin ? xl : CUDART_INF_F, yin ? yl : CUDART_INF_F), hi = max_nan(xin ? xh : -CUDART_INF_F, yin ? yh : -CUDART_INF_F);
            if (!KEY) {
#pragma unroll
                for (int s = 1; s < LANES; s <<= 1) {
                    lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, s));
                    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, s));
                }
                zero[g] = __bfloat162float(__float2bfloat16_rn(lo));
                scale[g] = scale_of(hi, zero[g]);
                ranged = ranged && zero[g] > -1e28f && hi < 1e28f && scale[g] > 1e-28f;
            } else {
                const float lo2 = min_nan(xin ? xl2 : CUDART_INF_F, yin ? yl2 : CUDART_INF_F);
                float hi2 = max_nan(xin ? xh2 : -CUDART_INF_F, yin ? yh2 : -CUDART_INF_F);
                __nv_bfloat162 both = __floats2bfloat162_rn(lo, lo2);   // (rounding keeps the order)
#pragma unroll
                for (int s = 1; s < LANES; s <<= 1) {
                    const uint32_t o = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<const uint32_t*>(&both), s);
                    both = __hmin2_nan(both, *reinterpret_cast<const __nv_bfloat162*>(&o));
                    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, s));
                    hi2 = max_nan(hi2, __shfl_xor_sync(0xffffffffu, hi2, s));
                }
                zero[g] = __low2float(both);
                scale[g] = scale_of(hi, zero[g]);
                sure = sure && zero[g] == __high2float(both) && scale[g] == scale_of(hi2, zero[g]) && scale[g] > 1e-28f && zero[g] > -1e28f && hi < 1e28f;
            }
        }
        const int ga = G == 1 || APART ? 0 : ua / 8, gb = G == 1 ? 0 : APART ? 1 : ub / 8;
        const float zx = ga ? zero[G - 1] : zero[0], zy = gb ? zero[G - 1] : zero[0];
        const Divisor qx(ga ? scale[G - 1] : scale[0]), qy(gb ? scale[G - 1] : scale[0]);
        if (KEY) {
            float worst = 0.f;
            wx = unit_near(x, dx, zx, qx.r, worst);
            wy = unit_near(y, dy, zy, qy.r, worst);
            return sure && worst < 0.5f;
        }
        wx = unit(x, zx, qx);
        wy = unit(y, zy, qy);
        if (!ranged) {
            wx = unit_divided(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7], zx, qx.s);
            wy = unit_divided(y[0], y[1], y[2], y[3], y[4], y[5], y[6], y[7], zy, qy.s);
        }
        return true;
    }
    // eight codes, given as -code: four as a number of 16 bits, twice
    static __device__ __forceinline__ uint32_t pack_codes(const float (&c)[8]) {
        float half[2];
#pragma unroll
        for (int i = 7; i >= 0; --i) half[i / 4] = i % 4 == 3 ? c[i] : fmaf(half[i / 4], 16.f, c[i]);
        return __byte_perm(__float_as_uint(8388608.f - half[0]), __float_as_uint(8388608.f - half[1]), 0x5410);
    }
    static __device__ __forceinline__ void extremes(const float (&x)[8], float& lo, float& hi) {
        lo = min_nan(min_nan(x[0], x[1], x[2]), min_nan(x[3], x[4], x[5]), min_nan(x[6], x[7]));
        hi = max_nan(max_nan(x[0], x[1], x[2]), max_nan(x[3], x[4], x[5]), max_nan(x[6], x[7]));
    }
    // the code word of a unit
    static __device__ __forceinline__ uint32_t unit(const float (&x)[8], float zero, const Divisor& by) {
        const Two z(zero, zero), up(ROUND, ROUND);
        float c[8];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            float t0, t1;
            by.quotient(Two(x[i], x[i + 1]) - z).get(t0, t1);
            t0 = fminf(fmaxf(t0, 0.f), 15.f); t1 = fminf(fmaxf(t1, 0.f), 15.f);       // (a NaN gets code 0)
            (up - (Two(t0, t1) + up)).get(c[i], c[i + 1]);
        }
        return pack_codes(c);
    }
    // The same of a key, not to the last bit: t = (x - zero) r / 15 in [0, 1] by one multiply-add that saturates, and how far
    // 15 t can be from its code at most: the element's own error, roundings of 1 / s, 1 / 15, their product and the zero's, at most
    // 2^-24 (7 |zero| / s + 63), and what difference and quotient are off by where the code is defined, 2^-24 31.
    static __device__ __forceinline__ uint32_t unit_near(const float (&x)[8], const float (&d)[8], float zero, float r, float& worst) {
        const float r15 = r * (1.f / 15.f), z15 = -zero * r15, off = fmaf(fabsf(z15), 7e-6f, 7e-6f);
        const Two fifteen(15.f, 15.f), up(ROUND, ROUND);
        float c[8], far = 0.f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const Two t(__saturatef(fmaf(x[i], r15, z15)), __saturatef(fmaf(x[i + 1], r15, z15))), minus = up - fma2(t, fifteen, up);
            minus.get(c[i], c[i + 1]);
            float e0, e1;
            fma2(t, fifteen, minus).get(e0, e1);
            far = fmaxf(far, fmaxf(fmaf(d[i], r, fabsf(e0)), fmaf(d[i + 1], r, fabsf(e1))));
        }
        worst = fmaxf(worst, far + off);
        return pack_codes(c);
    }
    static __device__ __noinline__ uint32_t unit_divided(float x0, float x1, float x2, float x3, float x4, float x5, float x6, float x7, float zero, float scale) {
        const float x[8] = {x0, x1, x2, x3, x4, x5, x6, x7};
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= (uint32_t)__float2int_rn(fminf(fmaxf(__fdiv_rn(x[i] - zero, scale), 0.f), 15.f)) << (4 * i);
        return w;
    }
    static __device__ __forceinline__ float scale_of(float hi, float zero) {
        const float s = __bfloat162float(__float2bfloat16_rn(__fmul_rn(hi - zero, 1.f / 15.f)));
        return s > 0.f && s < CUDART_INF_F ? s : 1.f;
    }
    __device__ __forceinline__ void store(uint8_t* chunk, int slot, int l, int ua, int ub) const {
        using Lay = I4Layout<D>;
        uint8_t* tile = chunk + (slot / I4_TILE) * Lay::TILE_BYTES;
        const int t = slot % I4_TILE;
        *reinterpret_cast<uint32_t*>(tile + Lay::word(t, ua)) = wx;
        *reinterpret_cast<uint32_t*>(tile + Lay::word(t, ub)) = wy;
        if (l < Lay::GROUPS)                                      // (both numbers are bfloat16: the upper half of their bits)
            *reinterpret_cast<uint32_t*>(tile + Lay::pair(t, l)) =
                __float_as_uint(l ? scale[Lay::GROUPS - 1] : scale[0]) >> 16 | (__float_as_uint(l ? zero[Lay::GROUPS - 1] : zero[0]) & 0xffff0000u);
    }
};

// A key row in binary64, from the row as it was given, to its slot: what its codes are defined by.  (A call, and by value: the
// rows of the binary32 path stay in registers.)
template <int D, bool IL>
__device__ __noinline__ void store_row64(const RotateArgs& a, int pos, int l, int ua, int ub, uint4 ra, uint4 rb, uint8_t* chunk, bool live) {
    constexpr int LANES = D / 16;
    float xo[8], yo[8];
    double x[8], y[8];
    unpack_unit(ra, xo);
    unpack_unit(rb, yo);
#pragma unroll
    for (int i = 0; i < 8; ++i) { x[i] = xo[i]; y[i] = yo[i]; }
    if (a.k_weight != nullptr) {
        double ss = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += x[i] * x[i] + y[i] * y[i];
#pragma unroll
        for (int s = 1; s < LANES; s <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, s);
        const double r = 1.0 / sqrt(ss / D + (double)a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] *= r * (double)__bfloat162float(a.k_weight[8 * ua + i]);
            y[i] *= r * (double)__bfloat162float(a.k_weight[8 * ub + i]);
        }
    }
    // (the lanes of a unit form its angles together here, too)
    constexpr int RPW = 32 / LANES, EACH = 8 / RPW;
    const int sub = (threadIdx.x & 31) / LANES;
    double c[EACH], s[EACH];
#pragma unroll 1
    for (int e = 0; e < EACH; ++e) {
        const int i = sub * EACH + e;
        double se = 0.0, ce = 1.0;
        if (8 * (IL && i >= 4 ? ub : ua) < a.rot_dim) {
            sincos((double)pos * (double)a.inv_freq[angle_of<IL>(i, ua, ub)], &se, &ce);
            ce *= (double)a.amplitude; se *= (double)a.amplitude;
        }
        if (e == 0) { c[0] = ce; s[0] = se; } else { c[EACH - 1] = ce; s[EACH - 1] = se; }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double ci = __shfl_sync(0xffffffffu, c[i % EACH], i / EACH * LANES + l), si = __shfl_sync(0xffffffffu, s[i % EACH], i / EACH * LANES + l);
        if (8 * (IL && i >= 4 ? ub : ua) >= a.rot_dim) continue;
        double &p = !IL ? x[i] : i < 4 ? x[2 * i] : y[2 * i - 8], &q = !IL ? y[i] : i < 4 ? x[2 * i + 1] : y[2 * i - 7];
        const double v = p * ci - q * si;
        q = q * ci + p * si;
        p = v;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) { xo[i] = (float)x[i]; yo[i] = (float)y[i]; }
    Quantised<D, false> code;
    code.template form<false, false>(ua, ub, xo, yo);
    if (live) code.store(chunk, pos % NOVAKV_PAGE_TOKENS, l, ua, ub);
}

template <int D, int DST, bool VEC, bool IL>
__global__ void __launch_bounds__(ROT_THREADS, DST == DST_INT4 ? 5 : 7)
novakv_rotate_kernel(const __grid_constant__ RotateArgs a) {
    constexpr int LANES = D / 16, RPW = 32 / LANES, WARPS = ROT_THREADS / 32;
    const int lane = threadIdx.x & 31, sub = lane / LANES, l = lane % LANES;
    const int warp = blockIdx.x * WARPS + threadIdx.x / 32, token = warp / a.parts, part = warp - token * a.parts;
    // rotation by halves pairs units u and u + rot / 16; what does not turn is dealt out in order
    const int ru = IL ? 0 : a.rot_dim / 16;
    const int ka = ru == 0 || l < ru ? l : 2 * l, kb = ru == 0 ? l + LANES : l < ru ? l + ru : 2 * l + 1;
    novakv_grid_dependency_wait();
    if (token >= a.n_tokens) return;

    const int pos = a.tok_pos[token], seq = DST == DST_ROWS ? 0 : a.tok_seq[token];
    const int step = a.parts * RPW, h0 = part * RPW;              // heads: a warp takes RPW at a time
    struct Row { uint4 x, y; };
    // (lanes behind the last head read it too: they take part, and write nothing)
    auto fetch = [&](const __nv_bfloat16* rows, int h, int heads, int ua, int ub) {
        const __nv_bfloat16* src = rows + min(h + sub, heads - 1) * D;
        return Row{load_unit<VEC>(src + 8 * ua), load_unit<VEC>(src + 8 * ub)};
    };
    // q, then k, then v, counted through; a role's first rows are on their way while the angles, or the role before, are formed
    const __nv_bfloat16 *q = a.q + token * a.q_stride, *k = a.k + token * a.k_stride, *v = a.v + token * a.v_stride;
    const int nq = (a.hq + RPW - 1) / RPW * RPW, nk = (a.hkv + RPW - 1) / RPW * RPW;
    auto first_k = [&](int h) { Row r = {}; if (h < nk) r = fetch(k, h, a.hkv, ka, kb); return r; };
    auto first_v = [&](int h) { Row r = {}; if (DST != DST_ROWS && h < nk) r = fetch(v, h, a.hkv, l, l + LANES); return r; };
    int h = h0;
    Row next = h < nq ? fetch(q, h, a.hq, ka, kb) : h - nq < nk ? first_k(h - nq) : first_v(h - nq - nk);

    int page = -1, slot = 0;                                      // -1: the token is skipped
    if (DST != DST_ROWS && seq != -1) {
        slot = pos % NOVAKV_PAGE_TOKENS;
        if (seq < 0 || seq >= a.n_seq || pos < 0 || pos / NOVAKV_PAGE_TOKENS >= a.max_pages_per_seq) {
            if (part == 0 && lane == 0) atomicOr(a.dev_status, NOVAKV_DEV_BAD_TOKEN);
        } else {
            page = a.page_table[(size_t)seq * a.max_pages_per_seq + pos / NOVAKV_PAGE_TOKENS];
            if (page < 0 || page >= a.n_pages) {
                if (part == 0 && lane == 0) atomicOr(a.dev_status, NOVAKV_DEV_BAD_PAGE);
                page = -1;
            } else if (part == 0 && lane == 0 && a.seq_lens[seq] <= pos) {     // (lengths only grow: a stale one costs an atomic)
                atomicMax(&a.seq_lens[seq], pos + 1);
            }
        }
    }
    if (DST != DST_ROWS && page < 0) return;

    // the lanes of a unit form its eight angles together: turns in binary64 (a far position keeps its angle), what is left of
    // them in binary32
    Turn turn;
    {
        constexpr int EACH = 8 / RPW;
        float c[EACH], s[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int i = sub * EACH + e;
            c[e] = 1.f; s[e] = 0.f;
            if (8 * (IL && i >= 4 ? kb : ka) < a.rot_dim) {
                double turns = (double)pos * (double)a.inv_freq[angle_of<IL>(i, ka, kb)] * 0.15915494309189533577;
                turns -= rint(turns);
                sincospif(2.f * (float)turns, &s[e], &c[e]);
                c[e] *= a.amplitude; s[e] *= a.amplitude;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            turn.c[i] = __shfl_sync(0xffffffffu, c[i % EACH], i / EACH * LANES + l);
            turn.s[i] = __shfl_sync(0xffffffffu, s[i % EACH], i / EACH * LANES + l);
        }
    }
    auto weights_of = [&](const __nv_bfloat16* w) {
        turn.norm = w != nullptr;
        if (turn.norm) { turn.wx = load_unit<false>(w + 8 * ka); turn.wy = load_unit<false>(w + 8 * kb); }
    };
    if (h < nq) {
        weights_of(a.q_weight);
        __nv_bfloat16* out = a.q_out + token * a.q_out_stride + sub * D;
#pragma unroll 1
        for (; h < nq; h += step) {
            const Row r = next;
            next = h + step < nq ? fetch(q, h + step, a.hq, ka, kb) : first_k(h + step - nq);
            float x[8], y[8];
            unpack_unit(r.x, x);
            unpack_unit(r.y, y);
            transform_row<D, IL, DST == DST_INT4>(a, turn, ka, kb, x, y);
            if (h + sub < a.hq) {
                store_unit<VEC>(out + h * D + 8 * ka, pack_unit(x));
                store_unit<VEC>(out + h * D + 8 * kb, pack_unit(y));
            }
        }
        if (h - nq >= nk) next = first_v(h - nq - nk);
    }
    h -= nq;
    if (h < nk) {
        weights_of(a.k_weight);
        const bool apart = D == 64 || IL || a.rot_dim == 0 || a.rot_dim == D;
#pragma unroll 1
        for (; h < nk; h += step) {
            const Row r = next;
            next = h + step < nk ? fetch(k, h + step, a.hkv, ka, kb) : first_v(h + step - nk);
            const bool live = h + sub < a.hkv;
            float x[8], y[8];
            unpack_unit(r.x, x);
            unpack_unit(r.y, y);
            bool sure = transform_row<D, IL, DST == DST_INT4>(a, turn, ka, kb, x, y);
            if constexpr (DST == DST_INT4) {
                uint8_t* chunk = a.k_pages + ((size_t)page * a.hkv + h + sub) * I4Layout<D>::CHUNK_BYTES;
                Quantised<D, true> code;
                sure = (apart ? code.template form<IL, true>(ka, kb, x, y) : code.template form<IL, false>(ka, kb, x, y)) && sure;
                if (__any_sync(0xffffffffu, live && !sure)) store_row64<D, IL>(a, pos, l, ka, kb, r.x, r.y, chunk, live);
                else if (live) code.store(chunk, slot, l, ka, kb);
            } else if (live) {
                __nv_bfloat16* dst = DST == DST_ROWS ? a.k_out + token * a.k_out_stride + (h + sub) * D
                                                     : reinterpret_cast<__nv_bfloat16*>(a.k_pages) + (((size_t)page * a.hkv + h + sub) * NOVAKV_PAGE_TOKENS + slot) * D;
                store_unit<VEC>(dst + 8 * ka, pack_unit(x));
                store_unit<VEC>(dst + 8 * kb, pack_unit(y));
            }
        }
    }
    if (DST == DST_ROWS) return;
    h -= nk;
#pragma unroll 1
    for (; h < nk; h += step) {
        const Row r = next;
        next = first_v(h + step);
        const bool live = h + sub < a.hkv;
        if constexpr (DST == DST_INT4) {
            float x[8], y[8];
            unpack_unit(r.x, x);
            unpack_unit(r.y, y);
            Quantised<D, false> code;
            code.template form<false, true>(l, l + LANES, x, y);
            if (live) code.store(a.v_pages + ((size_t)page * a.hkv + h + sub) * I4Layout<D>::CHUNK_BYTES, slot, l, l, l + LANES);
        } else if (live) {
            __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(a.v_pages) + (((size_t)page * a.hkv + h + sub) * NOVAKV_PAGE_TOKENS + slot) * D;
            store_unit<VEC>(dst + 8 * l, r.x);
            store_unit<VEC>(dst + 8 * (l + LANES), r.y);
        }
    }
}

// Read-back of the 4-bit cache: a row belongs to D / 16 lanes, and what they store at a time lies side by side.
struct GatherArgs {
    const int32_t *tok_seq, *tok_pos, *page_table;
    int n_tokens, hkv, n_pages, max_pages_per_seq, n_seq, parts;     // parts: warps of a token
    const uint8_t *k_pages, *v_pages;
    void *k_out, *v_out;
    uint32_t* dev_status;
};

// Values of the code word of 8 channels, as four pairs of bf16: 128 + code is a bfloat16 number that one OR makes, 128 is taken off
// exactly, and zero + scale code is rounded once.
__device__ __forceinline__ uint4 word_values(uint32_t w, __nv_bfloat162 scale, __nv_bfloat162 zero) {
    uint32_t v[4];                                                // channels (i, i + 4)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = (w >> (4 * i) & 0x000f000fu) | 0x43004300u;
        const __nv_bfloat162 x = __hfma2(scale, __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&c), __float2bfloat162_rn(128.f)), zero);
        v[i] = *reinterpret_cast<const uint32_t*>(&x);
    }
    return make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632));
}

// A warp takes the heads of a token, 2 x 32 / (D / 16) rows of keys and of values at a time.
template <int D, bool FP32>
__global__ void __launch_bounds__(ROT_THREADS)
novakv_int4_gather_kernel(const GatherArgs a) {
    using Lay = I4Layout<D>;
    constexpr int LANES = D / 16, RPW = 32 / LANES, AT_ONCE = 2;
    novakv_grid_dependency_wait();
    const int lane = threadIdx.x & 31, sub = lane / LANES, l = lane % LANES;
    const int warp = blockIdx.x * (ROT_THREADS / 32) + threadIdx.x / 32, t = warp / a.parts, part = warp - t * a.parts;
    if (t >= a.n_tokens) return;
    const int seq = a.tok_seq[t], pos = a.tok_pos[t];
    if (seq == -1) return;
    if (seq < 0 || seq >= a.n_seq || pos < 0 || pos / NOVAKV_PAGE_TOKENS >= a.max_pages_per_seq) {
        if (part == 0 && lane == 0) atomicOr(a.dev_status, NOVAKV_DEV_BAD_TOKEN);
        return;
    }
    const int page = a.page_table[(size_t)seq * a.max_pages_per_seq + pos / NOVAKV_PAGE_TOKENS];
    if (page < 0 || page >= a.n_pages) {
        if (part == 0 && lane == 0) atomicOr(a.dev_status, NOVAKV_DEV_BAD_PAGE);
        return;
    }
    // 16 bytes of a row at a time: 8 channels of bf16 or 4 of binary32
    constexpr int CH = FP32 ? 4 : 8, N = D / (LANES * CH);
    const int slot = pos % I4_TILE;
    const size_t tile = (size_t)page * a.hkv * Lay::CHUNK_BYTES + (pos % NOVAKV_PAGE_TOKENS / I4_TILE) * Lay::TILE_BYTES;
#pragma unroll 1
    for (int h0 = part * AT_ONCE * RPW; h0 < a.hkv; h0 += a.parts * AT_ONCE * RPW) {
        uint32_t code[AT_ONCE][2][N], meta[AT_ONCE][2][Lay::GROUPS];
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) {
            const int h = min(h0 + e * RPW + sub, a.hkv - 1);     // (rows behind the last head are read again, and not written)
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const uint8_t* src = (side ? a.v_pages : a.k_pages) + tile + (size_t)h * Lay::CHUNK_BYTES;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int c = (i * LANES + l) * CH;
                    const uint8_t* at = src + Lay::word(slot, c / 8) + c % 8 / 2;
                    code[e][side][i] = FP32 ? *reinterpret_cast<const uint16_t*>(at) : *reinterpret_cast<const uint32_t*>(at);
                }
#pragma unroll
                for (int g = 0; g < Lay::GROUPS; ++g) meta[e][side][g] = *reinterpret_cast<const uint32_t*>(src + Lay::pair(slot, g));
            }
        }
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) {
            const int h = h0 + e * RPW + sub;
            if (h >= a.hkv) break;
#pragma unroll
            for (int side = 0; side < 2; ++side)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int c = (i * LANES + l) * CH;
                    const uint32_t m = Lay::GROUPS == 1 || c < I4_GROUP ? meta[e][side][0] : meta[e][side][Lay::GROUPS - 1];
                    const size_t o = ((size_t)t * a.hkv + h) * D + c;
                    if constexpr (FP32) {
                        const float scale = __uint_as_float(m << 16), zero = __uint_as_float(m & 0xffff0000u);
                        float x[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)               // (2^23 + code is a number that one OR makes)
                            x[k] = fmaf(scale, __uint_as_float((code[e][side][i] >> (4 * k) & 15u) | 0x4b000000u) - 8388608.f, zero);
                        *reinterpret_cast<float4*>(reinterpret_cast<float*>(side ? a.v_out : a.k_out) + o) = make_float4(x[0], x[1], x[2], x[3]);
                    } else {
                        const uint32_t s2 = __byte_perm(m, 0, 0x1010), z2 = __byte_perm(m, 0, 0x3232);
                        *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(side ? a.v_out : a.k_out) + o) =
                            word_values(code[e][side][i], *reinterpret_cast<const __nv_bfloat162*>(&s2), *reinterpret_cast<const __nv_bfloat162*>(&z2));
                    }
                }
        }
    }
}

template <int D, int DST, bool IL>
novakv_status launch_rotate_t(novakv_ctx* ctx, RotateArgs& a, bool vec, cudaStream_t stream) {
    constexpr int RPW = 512 / D, WARPS = ROT_THREADS / 32;
    const int nq = (a.hq + RPW - 1) / RPW, nk = (a.hkv + RPW - 1) / RPW, tasks = nq + (DST == DST_ROWS ? 1 : 2) * nk;
    // a warp for each token, and several where there are fewer than some two waves of warps
    a.parts = min(tasks, max(1, (64 * ctx->n_sm + a.n_tokens - 1) / a.n_tokens));
    const long long blocks = ((long long)a.n_tokens * a.parts + WARPS - 1) / WARPS;
    auto* kern = vec ? novakv_rotate_kernel<D, DST, true, IL> : novakv_rotate_kernel<D, DST, false, IL>;
    if (novakv_launch_pdl(kern, dim3((unsigned)blocks), dim3(ROT_THREADS), 0, stream, a) != cudaSuccess) return NOVAKV_ECUDA;
    if (DST == DST_ROWS || a.hq > 0) novakv_queries_written(stream);       // (rows of either role: with as many heads they are alike)
    ctx->launches++;
    return NOVAKV_OK;
}
template <int D, int DST>
novakv_status launch_rotate(novakv_ctx* ctx, RotateArgs& a, bool interleaved, bool vec, cudaStream_t stream) {
    return interleaved ? launch_rotate_t<D, DST, true>(ctx, a, vec, stream) : launch_rotate_t<D, DST, false>(ctx, a, vec, stream);
}

// what all calls with a transform check of it
novakv_status check_transform(const novakv_ctx* ctx, const novakv_qk_transform* tr) {
    if (!tr) return NOVAKV_OK;
    const int d = ctx->cfg.head_dim;
    if (tr->rot_dim < 0 || tr->rot_dim > d || tr->rot_dim % 16 != 0) return NOVAKV_ESHAPE;
    if (tr->rot_dim > 0 && (!tr->inv_freq || ((uintptr_t)tr->inv_freq & 3))) return NOVAKV_EINVAL;
    if (tr->interleaved != 0 && tr->interleaved != 1) return NOVAKV_EINVAL;
    if (!(tr->eps >= 0.f) || !(tr->amplitude == tr->amplitude)) return NOVAKV_EINVAL;
    if (((uintptr_t)tr->q_weight | (uintptr_t)tr->k_weight) & 1) return NOVAKV_EINVAL;
    return NOVAKV_OK;
}
void set_transform(RotateArgs& a, const novakv_qk_transform* tr) {
    if (!tr) return;
    a.inv_freq = tr->inv_freq;
    a.rot_dim = tr->rot_dim;
    a.amplitude = tr->amplitude;
    a.q_weight = (const __nv_bfloat16*)tr->q_weight;
    a.k_weight = (const __nv_bfloat16*)tr->k_weight;
    a.eps = tr->eps;
}
// rows [n][heads][d] with `stride` elements from token to token: they must not overlap
bool rows_ok(const void* p, long long stride, int heads, int d) { return ((uintptr_t)p & 1) == 0 && stride >= (long long)heads * d; }
bool rows_vec(const void* p, long long stride) { return ((uintptr_t)p & 15) == 0 && stride % 8 == 0; }

novakv_status append(novakv_ctx* ctx, const novakv_qk_transform* tr, const void* k_new, long long k_stride, const void* v_new,
                     long long v_stride, const int32_t* tok_seq, const int32_t* tok_pos, int n_tokens, void* k_pages, void* v_pages,
                     int n_pages, const int32_t* page_table, int max_pages_per_seq, int n_seq, int32_t* seq_lens, const void* q,
                     long long q_stride, void* q_out, long long q_out_stride, novakv_stream stream, bool int4) {
    if (!ctx || n_tokens < 0) return NOVAKV_EINVAL;
    const int hq = ctx->cfg.n_q_heads, hkv = ctx->cfg.n_kv_heads, d = ctx->cfg.head_dim;
    const novakv_status st = check_transform(ctx, tr);
    if (st != NOVAKV_OK) return st;
    if (n_tokens == 0) return NOVAKV_OK;
    if (!k_new || !v_new || !tok_seq || !tok_pos || !k_pages || !v_pages || !page_table || !seq_lens) return NOVAKV_EINVAL;
    if ((q == nullptr) != (q_out == nullptr)) return NOVAKV_EINVAL;
    if (n_pages <= 0 || max_pages_per_seq <= 0 || n_seq <= 0) return NOVAKV_EPAGE;
    if (!rows_ok(k_new, k_stride, hkv, d) || !rows_ok(v_new, v_stride, hkv, d)) return NOVAKV_EINVAL;
    if (q && (!rows_ok(q, q_stride, hq, d) || !rows_ok(q_out, q_out_stride, hq, d))) return NOVAKV_EINVAL;
    if (((uintptr_t)k_pages | (uintptr_t)v_pages) & 15) return NOVAKV_EINVAL;
    if (((uintptr_t)tok_seq | (uintptr_t)tok_pos | (uintptr_t)page_table | (uintptr_t)seq_lens) & 3) return NOVAKV_EINVAL;
    const novakv_device_guard guard(ctx);
    if (!guard.ok) return NOVAKV_ECUDA;
    RotateArgs a = {};
    a.q = (const __nv_bfloat16*)q; a.k = (const __nv_bfloat16*)k_new; a.v = (const __nv_bfloat16*)v_new;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
    a.q_out = (__nv_bfloat16*)q_out;
    a.tok_seq = tok_seq; a.tok_pos = tok_pos;
    a.n_tokens = n_tokens; a.hq = q ? hq : 0; a.hkv = hkv;
    set_transform(a, tr);
    a.k_pages = (uint8_t*)k_pages; a.v_pages = (uint8_t*)v_pages;
    a.n_pages = n_pages; a.max_pages_per_seq = max_pages_per_seq; a.n_seq = n_seq;
    a.page_table = page_table; a.seq_lens = seq_lens; a.dev_status = ctx->dev_status;
    const bool il = tr && tr->interleaved && tr->rot_dim > 0;
    const bool vec = rows_vec(k_new, k_stride) && rows_vec(v_new, v_stride) && (!q || (rows_vec(q, q_stride) && rows_vec(q_out, q_out_stride)));
    if (int4)
        return d == 128 ? launch_rotate<128, DST_INT4>(ctx, a, il, vec, (cudaStream_t)stream) : launch_rotate<64, DST_INT4>(ctx, a, il, vec, (cudaStream_t)stream);
    return d == 128 ? launch_rotate<128, DST_BF16>(ctx, a, il, vec, (cudaStream_t)stream) : launch_rotate<64, DST_BF16>(ctx, a, il, vec, (cudaStream_t)stream);
}

}  // namespace

extern "C" novakv_status novakv_qk_norm_rope(novakv_ctx* ctx, const novakv_qk_transform* tr, const void* q, long long q_stride,
    const void* k, long long k_stride, const int32_t* tok_pos, int n_tokens, void* q_out, long long q_out_stride, void* k_out,
    long long k_out_stride, novakv_stream stream) {
    if (!ctx || !tr || n_tokens < 0) return NOVAKV_EINVAL;
    const int hq = ctx->cfg.n_q_heads, hkv = ctx->cfg.n_kv_heads, d = ctx->cfg.head_dim;
    const novakv_status st = check_transform(ctx, tr);
    if (st != NOVAKV_OK) return st;
    if (n_tokens == 0) return NOVAKV_OK;
    if ((!q && !k) || (q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr)) return NOVAKV_EINVAL;
    if (!tok_pos || ((uintptr_t)tok_pos & 3)) return NOVAKV_EINVAL;
    if (q && (!rows_ok(q, q_stride, hq, d) || !rows_ok(q_out, q_out_stride, hq, d))) return NOVAKV_EINVAL;
    if (k && (!rows_ok(k, k_stride, hkv, d) || !rows_ok(k_out, k_out_stride, hkv, d))) return NOVAKV_EINVAL;
    const novakv_device_guard guard(ctx);
    if (!guard.ok) return NOVAKV_ECUDA;
    RotateArgs a = {};
    a.q = (const __nv_bfloat16*)q; a.k = (const __nv_bfloat16*)k;
    a.q_stride = q_stride; a.k_stride = k_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
    a.q_out = (__nv_bfloat16*)q_out; a.k_out = (__nv_bfloat16*)k_out;
    a.tok_pos = tok_pos;
    a.n_tokens = n_tokens; a.hq = q ? hq : 0; a.hkv = k ? hkv : 0;
    set_transform(a, tr);
    const bool il = tr->interleaved && tr->rot_dim > 0;
    const bool vec = (!q || (rows_vec(q, q_stride) && rows_vec(q_out, q_out_stride))) && (!k || (rows_vec(k, k_stride) && rows_vec(k_out, k_out_stride)));
    return d == 128 ? launch_rotate<128, DST_ROWS>(ctx, a, il, vec, (cudaStream_t)stream) : launch_rotate<64, DST_ROWS>(ctx, a, il, vec, (cudaStream_t)stream);
}

extern "C" novakv_status novakv_bf16_append(novakv_ctx* ctx, const novakv_qk_transform* tr, const void* k_new, long long k_stride,
    const void* v_new, long long v_stride, const int32_t* tok_seq, const int32_t* tok_pos, int n_tokens, void* k_pages_bf16,
    void* v_pages_bf16, int n_pages, const int32_t* page_table, int max_pages_per_seq, int n_seq, int32_t* seq_lens, const void* q,
    long long q_stride, void* q_out, long long q_out_stride, novakv_stream stream) {
    return append(ctx, tr, k_new, k_stride, v_new, v_stride, tok_seq, tok_pos, n_tokens, k_pages_bf16, v_pages_bf16, n_pages, page_table,
                  max_pages_per_seq, n_seq, seq_lens, q, q_stride, q_out, q_out_stride, stream, false);
}

extern "C" novakv_status novakv_int4_append(novakv_ctx* ctx, const novakv_qk_transform* tr, const void* k_new, long long k_stride,
    const void* v_new, long long v_stride, const int32_t* tok_seq, const int32_t* tok_pos, int n_tokens, uint8_t* k_pages, uint8_t* v_pages,
    int n_pages, const int32_t* page_table, int max_pages_per_seq, int n_seq, int32_t* seq_lens, const void* q, long long q_stride,
    void* q_out, long long q_out_stride, novakv_stream stream) {
    return append(ctx, tr, k_new, k_stride, v_new, v_stride, tok_seq, tok_pos, n_tokens, k_pages, v_pages, n_pages, page_table,
                  max_pages_per_seq, n_seq, seq_lens, q, q_stride, q_out, q_out_stride, stream, true);
}

extern "C" size_t novakv_int4_page_bytes(const novakv_ctx* ctx) {
    if (!ctx) return 0;
    return (size_t)ctx->cfg.n_kv_heads * (ctx->cfg.head_dim == 128 ? I4Layout<128>::CHUNK_BYTES : I4Layout<64>::CHUNK_BYTES);
}

extern "C" novakv_status novakv_int4_gather(novakv_ctx* ctx, const int32_t* tok_seq, const int32_t* tok_pos, int n_tokens,
    const uint8_t* k_pages, const uint8_t* v_pages, int n_pages, const int32_t* page_table, int max_pages_per_seq, int n_seq, void* k_out,
    void* v_out, int out_is_fp32, novakv_stream stream) {
    if (!ctx || n_tokens < 0) return NOVAKV_EINVAL;
    if (n_tokens == 0) return NOVAKV_OK;
    if (!tok_seq || !tok_pos || !k_pages || !v_pages || !page_table || !k_out || !v_out) return NOVAKV_EINVAL;
    if (n_pages <= 0 || max_pages_per_seq <= 0 || n_seq <= 0) return NOVAKV_EPAGE;
    if (((uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)k_out | (uintptr_t)v_out) & 15) return NOVAKV_EINVAL;
    if (((uintptr_t)tok_seq | (uintptr_t)tok_pos | (uintptr_t)page_table) & 3) return NOVAKV_EINVAL;
    const int d = ctx->cfg.head_dim;
    const int rounds = (ctx->cfg.n_kv_heads + 1024 / d - 1) / (1024 / d);
    const int parts = min(rounds, max(1, (64 * ctx->n_sm + n_tokens - 1) / n_tokens));
    const long long blocks = ((long long)n_tokens * parts + ROT_THREADS / 32 - 1) / (ROT_THREADS / 32);
    const novakv_device_guard guard(ctx);
    if (!guard.ok) return NOVAKV_ECUDA;
    const GatherArgs a = {tok_seq, tok_pos, page_table, n_tokens, ctx->cfg.n_kv_heads, n_pages, max_pages_per_seq, n_seq, parts,
                          k_pages, v_pages, k_out, v_out, ctx->dev_status};
    auto* kern = d == 128 ? (out_is_fp32 ? novakv_int4_gather_kernel<128, true> : novakv_int4_gather_kernel<128, false>)
                          : (out_is_fp32 ? novakv_int4_gather_kernel<64, true> : novakv_int4_gather_kernel<64, false>);
    if (novakv_launch_pdl(kern, dim3((unsigned)blocks), dim3(ROT_THREADS), 0, (cudaStream_t)stream, a) != cudaSuccess) return NOVAKV_ECUDA;
    ctx->launches++;
    return NOVAKV_OK;
}
