// What lies between the QKV projection and the cache: RMS norms of queries and keys for each head, the position rotation, and
// the append of the rotated keys and the values to the BF16 or the 4-bit paged cache; and the read-back of the 4-bit cache.
//
//     y = x rsqrt(mean_i x_i^2 + eps) w                      per head, where a weight is given
//     (a, b) -> A (a cos t - b sin t, b cos t + a sin t)     t = position * inv_freq, in binary64
//     4 bits: zero = bf16(min), scale = bf16((max - zero) / 15), code = clamp(rint((x - zero) / scale), 0, 15) per 64 channels
//
// Every call moves each element once, so it is bound by memory where it is long and by latency where it is short.  A row (one
// head of one token) belongs to D / 16 lanes with two units of 8 channels each (two 16-byte loads); with rotation by halves the
// two units are a unit and its partner, so that no value crosses lanes but in the sums and minima.  A block takes a few tokens
// with all of their heads, q, k and v: the angles are formed once for them, while the first rows are on their way.
#include <math_constants.h>

#include "novakv_int4.cuh"
#include "novakv_ops.cuh"

namespace {

constexpr int ROT_THREADS = 256;
enum { DST_ROWS, DST_BF16, DST_INT4 };       // k goes to rows, to the BF16 pool, to the 4-bit pool

struct RotateArgs {
    const __nv_bfloat16 *q, *k, *v;
    long long q_stride, k_stride, v_stride, q_out_stride, k_out_stride;    // elements from token to token
    __nv_bfloat16 *q_out, *k_out;
    const int32_t *tok_seq, *tok_pos;
    int n_tokens, hq, hkv, tokens_per_block;
    const float* inv_freq;
    const __nv_bfloat16 *q_weight, *k_weight;
    float eps, amplitude;
    int rot_dim, interleaved;
    uint8_t *k_pages, *v_pages;              // (the BF16 pools too)
    int n_pages, max_pages_per_seq, n_seq;
    const int32_t* page_table;
    int32_t* seq_lens;
    uint32_t* dev_status;
};

// The key of the 4-bit cache is formed in binary64: the definition's codes and bfloat16 pairs are those of the exact number
// rounded to binary32, and a key formed in binary32 would now and then fall to the other side of a border.
__device__ __forceinline__ float rsqrt_of(float mean, float eps) { return rsqrtf(mean + eps); }
__device__ __forceinline__ double rsqrt_of(double mean, float eps) { return 1.0 / sqrt(mean + (double)eps); }

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
template <typename T>
__device__ __forceinline__ uint4 pack_unit(const T (&x)[8]) {
    return make_uint4(pack2((float)x[0], (float)x[1]), pack2((float)x[2], (float)x[3]), pack2((float)x[4], (float)x[5]),
                      pack2((float)x[6], (float)x[7]));
}
// minimum and maximum that keep a NaN: a group that holds one gets it as its zero
__device__ __forceinline__ float min_nan(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// norm and rotation of a row's two units; cs: (cos, sin) of the token's angles.  All lanes of the warp take part.
template <int D, typename T, typename T2>
__device__ __forceinline__ void transform_row(const RotateArgs& a, const __nv_bfloat16* weight, const T2* cs, int ua, int ub, T (&x)[8], T (&y)[8]) {
    constexpr int LANES = D / 16;
    if (weight != nullptr) {
        T ss = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) { ss += x[i] * x[i]; ss += y[i] * y[i]; }
#pragma unroll
        for (int s = 1; s < LANES; s <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, s);
        const T r = rsqrt_of(ss / D, a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = x[i] * r * (T)__bfloat162float(weight[8 * ua + i]);
            y[i] = y[i] * r * (T)__bfloat162float(weight[8 * ub + i]);
        }
    }
    if (8 * ua >= a.rot_dim) return;                              // (without rotation rot_dim is 0)
    if (!a.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const T2 c = cs[8 * ua + i];
            const T u = x[i] * c.x - y[i] * c.y;
            y[i] = y[i] * c.x + x[i] * c.y;
            x[i] = u;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            T2 c = cs[4 * ua + i / 2];
            T u = x[i] * c.x - x[i + 1] * c.y;
            x[i + 1] = x[i + 1] * c.x + x[i] * c.y;
            x[i] = u;
            if (8 * ub < a.rot_dim) {
                c = cs[4 * ub + i / 2];
                u = y[i] * c.x - y[i + 1] * c.y;
                y[i + 1] = y[i + 1] * c.x + y[i] * c.y;
                y[i] = u;
            }
        }
    }
}

__device__ __forceinline__ uint32_t code_word(const float (&x)[8], float zero, float scale) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)                                   // (a NaN gets code 0)
        w |= (uint32_t)__float2int_rn(fminf(fmaxf(__fdiv_rn(x[i] - zero, scale), 0.f), 15.f)) << (4 * i);
    return w;
}

// a row into the 4-bit chunk of its (page, KV head).  All lanes of the warp take part; `live` ones write.
template <int D>
__device__ __forceinline__ void store_row4(uint8_t* chunk, int slot, int l, int ua, int ub, const float (&x)[8], const float (&y)[8], bool live) {
    using Lay = I4Layout<D>;
    constexpr int LANES = D / 16;
    float lo[Lay::GROUPS], hi[Lay::GROUPS];
    {
        float xl = x[0], xh = x[0], yl = y[0], yh = y[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) {
            xl = min_nan(xl, x[i]); xh = max_nan(xh, x[i]);
            yl = min_nan(yl, y[i]); yh = max_nan(yh, y[i]);
        }
#pragma unroll
        for (int g = 0; g < Lay::GROUPS; ++g) {
            const bool xin = Lay::GROUPS == 1 || ua / 8 == g, yin = Lay::GROUPS == 1 || ub / 8 == g;
            lo[g] = min_nan(xin ? xl : CUDART_INF_F, yin ? yl : CUDART_INF_F);
            hi[g] = max_nan(xin ? xh : -CUDART_INF_F, yin ? yh : -CUDART_INF_F);
#pragma unroll
            for (int s = 1; s < LANES; s <<= 1) {
                lo[g] = min_nan(lo[g], __shfl_xor_sync(0xffffffffu, lo[g], s));
                hi[g] = max_nan(hi[g], __shfl_xor_sync(0xffffffffu, hi[g], s));
            }
        }
    }
    if (!live) return;
    float zero[Lay::GROUPS], scale[Lay::GROUPS];
#pragma unroll
    for (int g = 0; g < Lay::GROUPS; ++g) {
        zero[g] = __bfloat162float(__float2bfloat16_rn(lo[g]));
        scale[g] = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(hi[g] - zero[g], 15.f)));
        if (!(scale[g] > 0.f && scale[g] < CUDART_INF_F)) scale[g] = 1.f;
    }
    const int ga = Lay::GROUPS == 1 ? 0 : ua / 8, gb = Lay::GROUPS == 1 ? 0 : ub / 8;
    uint8_t* tile = chunk + (slot / I4_TILE) * Lay::TILE_BYTES;
    const int t = slot % I4_TILE;
    *reinterpret_cast<uint32_t*>(tile + Lay::word(t, ua)) = code_word(x, ga ? zero[Lay::GROUPS - 1] : zero[0], ga ? scale[Lay::GROUPS - 1] : scale[0]);
    *reinterpret_cast<uint32_t*>(tile + Lay::word(t, ub)) = code_word(y, gb ? zero[Lay::GROUPS - 1] : zero[0], gb ? scale[Lay::GROUPS - 1] : scale[0]);
    if (l < Lay::GROUPS)                                          // (both numbers are bfloat16: the upper half of their bits)
        *reinterpret_cast<uint32_t*>(tile + Lay::pair(t, l)) =
            __float_as_uint(l ? scale[Lay::GROUPS - 1] : scale[0]) >> 16 | (__float_as_uint(l ? zero[Lay::GROUPS - 1] : zero[0]) & 0xffff0000u);
}

template <int D, int DST, bool VEC>
__global__ void __launch_bounds__(ROT_THREADS)
novakv_rotate_kernel(const RotateArgs a) {
    constexpr int LANES = D / 16, RPW = 32 / LANES, WARPS = ROT_THREADS / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    const int tpb = a.tokens_per_block, half = a.rot_dim / 2;
    float2* cs = reinterpret_cast<float2*>(smem);                 // [tokens][half]
    double2* cd = reinterpret_cast<double2*>(smem + (((size_t)tpb * half * 8 + 15) & ~(size_t)15));
    int2* where = reinterpret_cast<int2*>(smem + (((size_t)tpb * half * 8 + 15) & ~(size_t)15) + (DST == DST_INT4 ? (size_t)tpb * half * 16 : 0));
    novakv_grid_dependency_wait();
    const int tok0 = blockIdx.x * tpb, n_tok = min(tpb, a.n_tokens - tok0);
    for (int i = threadIdx.x; i < n_tok * half; i += ROT_THREADS) {
        const int t = i / half, f = i - t * half;
        const double angle = (double)a.tok_pos[tok0 + t] * (double)a.inv_freq[f];
        if (DST == DST_INT4) {
            double s, c;
            sincos(angle, &s, &c);
            c *= (double)a.amplitude; s *= (double)a.amplitude;
            cd[i] = make_double2(c, s);
            cs[i] = make_float2((float)c, (float)s);
        } else {
            // turns in binary64 (a far position keeps its angle), what is left of them in binary32
            double turns = angle * 0.15915494309189533577;
            turns -= rint(turns);
            float s, c;
            sincospif(2.f * (float)turns, &s, &c);
            cs[i] = make_float2(c * a.amplitude, s * a.amplitude);
        }
    }
    if (DST != DST_ROWS) {                                        // slot of every token: (page, slot), page -1: skipped
        for (int t = threadIdx.x; t < n_tok; t += ROT_THREADS) {
            const int seq = a.tok_seq[tok0 + t], pos = a.tok_pos[tok0 + t];
            int page = -1;
            if (seq != -1) {
                if (seq < 0 || seq >= a.n_seq || pos < 0 || pos / NOVAKV_PAGE_TOKENS >= a.max_pages_per_seq) {
                    atomicOr(a.dev_status, NOVAKV_DEV_BAD_TOKEN);
                } else {
                    page = a.page_table[(size_t)seq * a.max_pages_per_seq + pos / NOVAKV_PAGE_TOKENS];
                    if (page < 0 || page >= a.n_pages) {
                        atomicOr(a.dev_status, NOVAKV_DEV_BAD_PAGE);
                        page = -1;
                    } else if (a.seq_lens[seq] <= pos) {          // (lengths only grow: a stale one costs an atomic)
                        atomicMax(&a.seq_lens[seq], pos + 1);
                    }
                }
            }
            where[t] = make_int2(page, pos % NOVAKV_PAGE_TOKENS);
        }
    }
    __syncthreads();

    const int lane = threadIdx.x & 31, sub = lane / LANES, l = lane % LANES;
    const int wq = (n_tok * a.hq + RPW - 1) / RPW, wk = (n_tok * a.hkv + RPW - 1) / RPW;
    const int tasks = wq + wk + (DST == DST_ROWS ? 0 : wk);
    // rotation by halves pairs units u and u + rot / 16; what does not turn is dealt out in order
    const int ru = a.interleaved ? 0 : a.rot_dim / 16;
    const int ka = a.interleaved || ru == 0 ? l : l < ru ? l : 2 * l, kb = a.interleaved || ru == 0 ? l + LANES : l < ru ? l + ru : 2 * l + 1;
    for (int task = blockIdx.y * WARPS + threadIdx.x / 32; task < tasks; task += WARPS * gridDim.y) {
        const int role = task < wq ? 0 : task < wq + wk ? 1 : 2;
        const int heads = role == 0 ? a.hq : a.hkv;
        const int row = (task - (role == 0 ? 0 : role == 1 ? wq : wq + wk)) * RPW + sub;
        bool live = row < n_tok * heads;
        const int t = live ? row / heads : 0, h = live ? row - t * heads : 0;
        if (DST != DST_ROWS) live = live && where[t].x >= 0;
        const int ua = role == 2 ? l : ka, ub = role == 2 ? l + LANES : kb;
        const __nv_bfloat16* src = role == 0 ? a.q + (tok0 + t) * a.q_stride : role == 1 ? a.k + (tok0 + t) * a.k_stride : a.v + (tok0 + t) * a.v_stride;
        src += h * D;
        uint4 ra = make_uint4(0, 0, 0, 0), rb = ra;
        if (live) { ra = load_unit<VEC>(src + 8 * ua); rb = load_unit<VEC>(src + 8 * ub); }
        float x[8], y[8];
        unpack_unit(ra, x);
        unpack_unit(rb, y);
        if (role == 0) {
            transform_row<D, float, float2>(a, a.q_weight, cs + t * half, ua, ub, x, y);
            if (live) {
                __nv_bfloat16* dst = a.q_out + (tok0 + t) * a.q_out_stride + h * D;
                store_unit<VEC>(dst + 8 * ua, pack_unit(x));
                store_unit<VEC>(dst + 8 * ub, pack_unit(y));
            }
            continue;
        }
        if constexpr (DST == DST_INT4) {
            if (role == 1) {
                double u[8], w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) { u[i] = x[i]; w[i] = y[i]; }
                transform_row<D, double, double2>(a, a.k_weight, cd + t * half, ua, ub, u, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) { x[i] = (float)u[i]; y[i] = (float)w[i]; }
            }
            uint8_t* chunk = (role == 1 ? a.k_pages : a.v_pages) + ((size_t)max(where[t].x, 0) * a.hkv + h) * I4Layout<D>::CHUNK_BYTES;
            store_row4<D>(chunk, where[t].y, l, ua, ub, x, y, live);
            continue;
        }
        if (role == 1) transform_row<D, float, float2>(a, a.k_weight, cs + t * half, ua, ub, x, y);
        if (live) {
            __nv_bfloat16* dst;
            if (DST == DST_ROWS) dst = a.k_out + (tok0 + t) * a.k_out_stride + h * D;
            else
                dst = reinterpret_cast<__nv_bfloat16*>(role == 1 ? a.k_pages : a.v_pages) +
                      (((size_t)where[t].x * a.hkv + h) * NOVAKV_PAGE_TOKENS + where[t].y) * D;
            store_unit<VEC>(dst + 8 * ua, role == 1 ? pack_unit(x) : ra);
            store_unit<VEC>(dst + 8 * ub, role == 1 ? pack_unit(y) : rb);
        }
    }
}

// Read-back of the 4-bit cache: a row belongs to D / 16 lanes of 16 channels (8 code bytes) each.
struct GatherArgs {
    const int32_t *tok_seq, *tok_pos, *page_table;
    int n_tokens, hkv, n_pages, max_pages_per_seq, n_seq;
    const uint8_t *k_pages, *v_pages;
    void *k_out, *v_out;
    uint32_t* dev_status;
};

template <int D, bool FP32>
__global__ void __launch_bounds__(ROT_THREADS)
novakv_int4_gather_kernel(const GatherArgs a) {
    using Lay = I4Layout<D>;
    constexpr int LANES = D / 16;
    novakv_grid_dependency_wait();
    const long long row = ((long long)blockIdx.x * ROT_THREADS + threadIdx.x) / LANES;
    const int l = threadIdx.x % LANES;
    if (row >= (long long)a.n_tokens * a.hkv) return;
    const int t = (int)(row / a.hkv), h = (int)(row - (long long)t * a.hkv);
    const int seq = a.tok_seq[t], pos = a.tok_pos[t];
    if (seq == -1) return;
    if (seq < 0 || seq >= a.n_seq || pos < 0 || pos / NOVAKV_PAGE_TOKENS >= a.max_pages_per_seq) {
        if (h == 0 && l == 0) atomicOr(a.dev_status, NOVAKV_DEV_BAD_TOKEN);
        return;
    }
    const int page = a.page_table[(size_t)seq * a.max_pages_per_seq + pos / NOVAKV_PAGE_TOKENS];
    if (page < 0 || page >= a.n_pages) {
        if (h == 0 && l == 0) atomicOr(a.dev_status, NOVAKV_DEV_BAD_PAGE);
        return;
    }
    const size_t tile = ((size_t)page * a.hkv + h) * Lay::CHUNK_BYTES + (pos % NOVAKV_PAGE_TOKENS / I4_TILE) * Lay::TILE_BYTES;
    const int slot = pos % I4_TILE, at = Lay::word(slot, 2 * l), pair = Lay::pair(slot, l / 4);
    uint2 code[2];
    uint32_t meta[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const uint8_t* src = (side ? a.v_pages : a.k_pages) + tile;
        code[side] = *reinterpret_cast<const uint2*>(src + at);
        meta[side] = *reinterpret_cast<const uint32_t*>(src + pair);
    }
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const float scale = __uint_as_float(meta[side] << 16), zero = __uint_as_float(meta[side] & 0xffff0000u);
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
            x[i] = fmaf(scale, (float)((i < 8 ? code[side].x >> (4 * i) : code[side].y >> (4 * i - 32)) & 15u), zero);
        const size_t o = (size_t)row * D + 16 * l;
        if (FP32) {
            float4* dst = reinterpret_cast<float4*>(reinterpret_cast<float*>(side ? a.v_out : a.k_out) + o);
#pragma unroll
            for (int i = 0; i < 4; ++i) dst[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
        } else {
            uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(side ? a.v_out : a.k_out) + o);
            dst[0] = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
            dst[1] = make_uint4(pack2(x[8], x[9]), pack2(x[10], x[11]), pack2(x[12], x[13]), pack2(x[14], x[15]));
        }
    }
}

template <int D, int DST>
novakv_status launch_rotate(novakv_ctx* ctx, RotateArgs& a, bool vec, cudaStream_t stream) {
    const int half = a.rot_dim / 2;
    a.tokens_per_block = a.n_tokens >= 8 * ctx->n_sm ? 4 : 1;
    const size_t smem = (((size_t)a.tokens_per_block * half * 8 + 15) & ~(size_t)15) + (DST == DST_INT4 ? (size_t)a.tokens_per_block * half * 16 : 0) +
                        a.tokens_per_block * sizeof(int2);
    const dim3 grid((a.n_tokens + a.tokens_per_block - 1) / a.tokens_per_block);
    const cudaError_t e = vec ? novakv_launch_pdl(novakv_rotate_kernel<D, DST, true>, grid, dim3(ROT_THREADS), smem, stream, a)
                              : novakv_launch_pdl(novakv_rotate_kernel<D, DST, false>, grid, dim3(ROT_THREADS), smem, stream, a);
    if (e != cudaSuccess) return NOVAKV_ECUDA;
    ctx->launches++;
    return NOVAKV_OK;
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
    a.interleaved = tr->interleaved;
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
    const bool vec = rows_vec(k_new, k_stride) && rows_vec(v_new, v_stride) && (!q || (rows_vec(q, q_stride) && rows_vec(q_out, q_out_stride)));
    if (int4)
        return d == 128 ? launch_rotate<128, DST_INT4>(ctx, a, vec, (cudaStream_t)stream) : launch_rotate<64, DST_INT4>(ctx, a, vec, (cudaStream_t)stream);
    return d == 128 ? launch_rotate<128, DST_BF16>(ctx, a, vec, (cudaStream_t)stream) : launch_rotate<64, DST_BF16>(ctx, a, vec, (cudaStream_t)stream);
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
    const bool vec = (!q || (rows_vec(q, q_stride) && rows_vec(q_out, q_out_stride))) && (!k || (rows_vec(k, k_stride) && rows_vec(k_out, k_out_stride)));
    return d == 128 ? launch_rotate<128, DST_ROWS>(ctx, a, vec, (cudaStream_t)stream) : launch_rotate<64, DST_ROWS>(ctx, a, vec, (cudaStream_t)stream);
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
    const long long blocks = ((long long)n_tokens * ctx->cfg.n_kv_heads * (d / 16) + ROT_THREADS - 1) / ROT_THREADS;
    if (blocks > 0x7fffffffll) return NOVAKV_ESHAPE;
    const novakv_device_guard guard(ctx);
    if (!guard.ok) return NOVAKV_ECUDA;
    const GatherArgs a = {tok_seq, tok_pos, page_table, n_tokens, ctx->cfg.n_kv_heads, n_pages, max_pages_per_seq, n_seq,
                          k_pages, v_pages, k_out, v_out, ctx->dev_status};
    auto* kern = d == 128 ? (out_is_fp32 ? novakv_int4_gather_kernel<128, true> : novakv_int4_gather_kernel<128, false>)
                          : (out_is_fp32 ? novakv_int4_gather_kernel<64, true> : novakv_int4_gather_kernel<64, false>);
    if (novakv_launch_pdl(kern, dim3((unsigned)blocks), dim3(ROT_THREADS), 0, (cudaStream_t)stream, a) != cudaSuccess) return NOVAKV_ECUDA;
    ctx->launches++;
    return NOVAKV_OK;
}
