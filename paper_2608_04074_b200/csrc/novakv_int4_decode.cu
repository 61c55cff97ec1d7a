// Decode attention over the 4-bit cache: one query token per sequence,
//
//     z_j = sm_scale q . k^_j,   p = softmax(z) over the positions in sight,   o = sum_j p_j v^_j,   x^ = zero + scale code
//
// per 64 channels, so that z_j = sm_scale sum_g (scale_jg q_g . c_jg + zero_jg sum q_g) and likewise for the values: both
// products run on the codes themselves.  d / 2 + d / 16 bytes per token, head and side are read once (144 at d = 128); the
// multiplications are four per byte and query head, so HBM is the bound and instructions are what has to be kept few.
//
//  * Tensor cores, mma.sync m16n8k16 with the codes as the 16-row operand and the query heads of the KV head as the 8 columns
//    (tcgen05 wants its operands as 16-bit tiles in shared memory: the unpacked codes would have to be written there first,
//    four times the bytes of the cache).  A code c is the binary16 subnormal c 2^-24, which the tensor core multiplies exactly:
//    one AND of a word gives two operands, no conversion.  Codes in bits 4..7 are 16 c; what they meet carries a 1/16.
//  * Exactness: q is a bfloat16 number, exact in binary16 after a power of two per head; the weights are carried as binary16
//    pairs hi + lo (22 bits).  With four heads the lo parts are the unused four columns of the same product; with eight they
//    take a second one.  Accumulation, softmax statistics and the zeros' share are binary32.
//  * Streaming: the walk over (sequence, KV head, tile of 32 tokens) is cut evenly among the CTAs (one per SM) and again among
//    their 16 warps; each warp copies its tiles' keys and values (one bulk copy each) into a ring of its own, five tiles at
//    d = 128, and no warp waits for another before the end.
//  * Join: what a warp has of a (sequence, KV head) pair that it does not hold whole goes to shared memory; the CTA joins these
//    pieces, and a second kernel joins the at most two per CTA that reach over its ends.
#include <math_constants.h>

#include "novakv_int4.cuh"
#include "novakv_ops.cuh"
#include "novakv_tcgen05.cuh"

namespace {

constexpr int WARPS = 16, THREADS = WARPS * 32;
constexpr int HEADROOM = 4;                  // a new maximum is set this many bits high: the next records need no rescaling
constexpr float W_ONE = 32768.f;             // the weight 1 in binary16: what underflows is 2^-39 of the largest

template <int D, int HG>
struct Plan {
    using Lay = I4Layout<D>;
    static constexpr int SLOTS = D == 128 ? 5 : 10;                // ring of a warp, in tiles of one side
    static constexpr int PIECE = HG * (D + 2);                     // floats of a partial: per head maximum, sum, accumulators
    static constexpr int RING = WARPS * SLOTS * Lay::TILE_BYTES;
    static constexpr int BARS = RING;
    static constexpr int HEADS = BARS + WARPS * SLOTS * 8;         // first pieces of the warps (the last ones lie in their rings)
    static constexpr int PREFIX = HEADS + WARPS * PIECE * 4;       // int [THREADS + 1]
    static constexpr int MISC = (PREFIX + (THREADS + 1) * 4 + 15) & ~15;
    static constexpr int TOTAL = MISC + 512;
    static_assert(SLOTS * Lay::TILE_BYTES >= PIECE * 4, "a warp's last piece fits into its ring");
    static_assert(TOTAL <= 227 * 1024, "shared memory");
};

struct DecodeArgs {
    const __nv_bfloat16* q;
    const uint8_t *k_pages, *v_pages;
    int n_pages;
    const int32_t *page_table, *seq_lens;
    int max_pages_per_seq, batch, hkv, window, out_is_fp32;
    float scale_log2;
    const float* sink;
    void* out;
    int* info;                               // [CTAs][2] pair of the piece that reaches over the CTA's front / back end, or -1
    float* part;                             // [CTAs][2][PIECE]
    uint32_t* dev_status;
    long wait_clocks;
};

__device__ __forceinline__ float ex2f(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t movmatrix_t(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// A warp's wait for a slot of its ring: all lanes come to the same answer.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
    return __all_sync(0xffffffffu, mbar_wait_slow<0>(bar, parity, abort_flag));
}

// Sequence b's tiles in sight and its first one.
struct Sight { int len, start, t0, tiles; };
__device__ __forceinline__ Sight sight_of(const DecodeArgs& a, int b) {
    Sight s;
    s.len = min(max(a.seq_lens[b], 0), a.max_pages_per_seq * NOVAKV_PAGE_TOKENS);
    s.start = a.window > 0 ? max(0, s.len - a.window) : 0;
    s.t0 = s.start / I4_TILE;
    s.tiles = s.len > 0 ? (s.len + I4_TILE - 1) / I4_TILE - s.t0 : 0;
    return s;
}
// Where unit u of the walk lies: sequence, KV head, tile of the pair.
struct Place { int b, kvh, tile; Sight s; };
__device__ __forceinline__ Place locate(const DecodeArgs& a, const int* prefix, int chunk, long long u) {
    int lo = 0, hi = THREADS;                                     // prefix[lo] hkv <= u < prefix[hi] hkv
#pragma unroll 1
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((long long)prefix[mid] * a.hkv <= u) lo = mid;
        else hi = mid;
    }
    Place p;
    p.b = lo * chunk;
    long long r = u - (long long)prefix[lo] * a.hkv;
    p.s = sight_of(a, p.b);
#pragma unroll 1
    while (r >= (long long)p.s.tiles * a.hkv && p.b + 1 < a.batch) {
        r -= (long long)p.s.tiles * a.hkv;
        p.s = sight_of(a, ++p.b);
    }
    const int tiles = max(p.s.tiles, 1);
    p.kvh = min((int)r / tiles, a.hkv - 1);
    p.tile = (int)r - p.kvh * tiles;
    return p;
}

template <int D, int HG>
__device__ __forceinline__ void write_out(const DecodeArgs& a, int pair, int i, float o) {
    const size_t oi = (size_t)pair * HG * D + i;                  // [batch][Hkv][Hg][D]
    if (a.out_is_fp32) reinterpret_cast<float*>(a.out)[oi] = o;
    else reinterpret_cast<__nv_bfloat16*>(a.out)[oi] = __float2bfloat16_rn(o);
}
// the sink's share of a head's sum, relative to its maximum m
__device__ __forceinline__ float sink_mass(const DecodeArgs& a, int head, float m) {
    return a.sink != nullptr ? ex2f(fmaf(a.sink[head], 1.44269504f, -m)) : 0.f;
}

template <int D, int HG>
__global__ void __launch_bounds__(THREADS, 1)
novakv_int4_decode_kernel(const DecodeArgs a) {
    using Lay = I4Layout<D>;
    using P = Plan<D, HG>;
    constexpr int G = Lay::GROUPS, NP = Lay::PIECES, SLOTS = P::SLOTS, TB = Lay::TILE_BYTES;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, j = lane & 3;
    int* prefix = reinterpret_cast<int*>(smem + P::PREFIX);
    int* misc = reinterpret_cast<int*>(smem + P::MISC);           // 1 abort flag, 8..9 wait limit, 16..31 warp sums, 32..63 pieces' pairs, 64..95 their ends
    volatile int* abort_flag = misc + 1;
    const uint32_t ring = smem_u32(smem) + warp * SLOTS * TB, bars = smem_u32(smem + P::BARS) + warp * SLOTS * 8;
    if (lane < SLOTS) mbar_init(bars + 8 * lane, 1);
    if (threadIdx.x == 0) {
        misc[1] = 0;
        *reinterpret_cast<long long*>(misc + 1 + MBAR_LIMIT) = a.wait_clocks;
    }
    if (threadIdx.x < 2 * WARPS) misc[32 + threadIdx.x] = -1;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    novakv_grid_dependency_wait();

    // ---- the walk: prefix of the tiles by runs of `chunk` sequences -------------------------------------------------
    const int chunk = (a.batch + THREADS - 1) / THREADS;
    {
        int sum = 0;
        for (int b = threadIdx.x * chunk; b < min(a.batch, ((int)threadIdx.x + 1) * chunk); ++b) {
            sum += sight_of(a, b).tiles;
            if (blockIdx.x == 0 && a.seq_lens[b] > a.max_pages_per_seq * NOVAKV_PAGE_TOKENS) atomicOr(a.dev_status, NOVAKV_DEV_BAD_LENGTH);
        }
        int inc = sum;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, inc, s);
            if (lane >= s) inc += o;
        }
        if (lane == 31) misc[16 + warp] = inc;
        __syncthreads();
        int base = 0;
        for (int w = 0; w < warp; ++w) base += misc[16 + w];
        prefix[threadIdx.x + 1] = base + inc;
        if (threadIdx.x == 0) prefix[0] = 0;
        __syncthreads();
    }
    const long long units = (long long)prefix[THREADS] * a.hkv;
    // (no CTA in between without a unit: the join goes by the CTAs' order)
    const long long ctas = max(1ll, min((long long)gridDim.x, units)), cta = min((long long)blockIdx.x, ctas);
    const long long cu0 = units * cta / ctas, cu1 = units * min(cta + 1, ctas) / ctas;
    const long long wu0 = cu0 + (cu1 - cu0) * warp / WARPS, wu1 = cu0 + (cu1 - cu0) * (warp + 1) / WARPS;
    const int n = (int)(wu1 - wu0);

    // ---- producer: the tiles' chunks 32 at a time, the next batch always on its way ---------------------------------
    auto chunk_of = [&](int i) -> int {                           // (page, KV head, half) of the warp's i-th tile
        if (i >= n) return 0;
        const Place p = locate(a, prefix, chunk, wu0 + i);
        const int tile = p.s.t0 + p.tile;
        int page = a.page_table[(size_t)p.b * a.max_pages_per_seq + tile / 2];
        if (page < 0 || page >= a.n_pages) {
            atomicOr(a.dev_status, NOVAKV_DEV_BAD_PAGE);
            page = 0;
        }
        return (page * a.hkv + p.kvh) * 2 + (tile & 1);
    };
    int batch_now = 0, chunks = 0, chunks_next = 0;
    if (n > 0) { chunks = chunk_of(lane); if (n > 32) chunks_next = chunk_of(32 + lane); }
    int put_slot = 0;
    auto issue = [&](int item) {                                  // item 2 t: keys of tile t, 2 t + 1: its values
        const int t = item >> 1;
        if (t >> 5 != batch_now) {
            batch_now = t >> 5;
            chunks = chunks_next;
            chunks_next = chunk_of(((batch_now + 1) << 5) + lane);
        }
        const size_t at = (size_t)__shfl_sync(0xffffffffu, chunks, t & 31) * TB;
        if (lane == 0) {
            mbar_expect_tx(bars + 8 * put_slot, TB);
            bulk_copy(ring + put_slot * TB, ((item & 1) ? a.v_pages : a.k_pages) + at, TB, bars + 8 * put_slot);
        }
        put_slot = put_slot + 1 == SLOTS ? 0 : put_slot + 1;
    };
    __syncwarp();
    for (int i = 0; i < min(SLOTS, 2 * n); ++i) issue(i);
    int issued = min(SLOTS, 2 * n), taken = 0, get_slot = 0, parity = 0;
    bool given_up = false;
    auto next_slot = [&]() {
        if (++get_slot == SLOTS) { get_slot = 0; parity ^= 1; }
        ++taken;
    };

    // ---- consumer ---------------------------------------------------------------------------------------------------
    // the lane's columns 2 j, 2 j + 1 of the products: column c is head c % HG, its hi (c / HG = 0) or lo part (1)
    const int head0 = 2 * j % HG, head1 = (2 * j + 1) % HG;
    Place at = {};
    if (n > 0) at = locate(a, prefix, chunk, wu0);
    uint32_t qf[NP][2][2];
    float qfac0 = 0.f, qfac1 = 0.f, qz0[G], qz1[G];
    float m0, m1, l0, l1, zs0[G], zs1[G], vbound, vfac;
    float o[NP][2][4];
    bool fresh = true;
    int seg_first = 0;

#pragma unroll 1
    for (int t = 0; t < n && !given_up; ++t) {
        if (fresh) {                                              // ---- a new (sequence, KV head) pair
            fresh = false;
            seg_first = at.tile;
            const __nv_bfloat16* qp = a.q + (((size_t)at.b * a.hkv + at.kvh) * HG + gr % HG) * D + 8 * j;
            uint4 w[NP];
            float mx = 0.f;
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                w[p] = *reinterpret_cast<const uint4*>(qp + 32 * p);
                const uint32_t* ww = reinterpret_cast<const uint32_t*>(&w[p]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    mx = fmaxf(mx, fmaxf(fabsf(__uint_as_float(ww[i] << 16)), fabsf(__uint_as_float(ww[i] & 0xffff0000u))));
            }
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            // 2^up brings the head's largest coordinate just below 2^15
            const int up = min(max(15 - ((int)(__float_as_uint(mx) >> 23) - 126), -100), 120);
            const float f = __uint_as_float((uint32_t)(up + 127) << 23);
            float sum[G];
#pragma unroll
            for (int g = 0; g < G; ++g) sum[g] = 0.f;
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const uint32_t ww[4] = {w[p].x, w[p].y, w[p].z, w[p].w};
                float x[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(ww[i] << 16); x[2 * i + 1] = __uint_as_float(ww[i] & 0xffff0000u); }
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[p / 2] += x[i];
#pragma unroll
                for (int s = 0; s < 2; ++s) {                     // channels 8 j + 2 s + {0, 4} in the low bits, + {1, 5} in bits 4..7
                    qf[p][s][0] = pack_half(x[2 * s] * f, x[2 * s + 4] * f);
                    qf[p][s][1] = pack_half(x[2 * s + 1] * f * 0.0625f, x[2 * s + 5] * f * 0.0625f);
                }
            }
            const float fac = a.scale_log2 * __uint_as_float((uint32_t)(24 - up + 127) << 23);
            qfac0 = __shfl_sync(0xffffffffu, fac, 8 * j);
            qfac1 = __shfl_sync(0xffffffffu, fac, 8 * j + 4);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 1);
                sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 2);
                qz0[g] = a.scale_log2 * __shfl_sync(0xffffffffu, sum[g], 8 * j);
                qz1[g] = a.scale_log2 * __shfl_sync(0xffffffffu, sum[g], 8 * j + 4);
                zs0[g] = zs1[g] = 0.f;
            }
            m0 = m1 = -CUDART_INF_F;
            l0 = l1 = 0.f;
            vbound = 0.f; vfac = 0.f;
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[p][s][i] = 0.f;
        }

        // ---- logits of the tile's 32 tokens: z[s][0..1] of token 16 s + gr, z[s][2..3] of token 16 s + 8 + gr ---------
        float z[2][4];
        {
            if (!warp_wait(bars + 8 * get_slot, parity, abort_flag)) { given_up = true; break; }
            const uint32_t base = ring + get_slot * TB;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float acc[G][4];
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[g][i] = 0.f;
                const int row = 16 * s + (lane & 15);
#pragma unroll
                for (int pp = 0; pp < NP; pp += 2) {
                    uint32_t r[4];
                    ldmatrix4(base + row * Lay::ROW + (((pp + (lane >> 4)) ^ Lay::swizzle(row)) << 4), r);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t x = r[2 * h], y = r[2 * h + 1];
                        mma16816(acc[(pp + h) / 2], x & 0x000f000fu, y & 0x000f000fu, x & 0x00f000f0u, y & 0x00f000f0u, qf[pp + h][0][0], qf[pp + h][0][1]);
                        mma16816(acc[(pp + h) / 2], x >> 8 & 0x000f000fu, y >> 8 & 0x000f000fu, x >> 8 & 0x00f000f0u, y >> 8 & 0x00f000f0u,
                                 qf[pp + h][1][0], qf[pp + h][1][1]);
                    }
                }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t meta = base + Lay::pair(16 * s + 8 * half + gr, 0);
                    uint32_t w[2];
                    if (G == 2) { const uint2 v = lds64(meta); w[0] = v.x; w[1] = v.y; }
                    else w[0] = w[1] = lds32(meta);
                    float d0 = 0.f, d1 = 0.f, e0 = 0.f, e1 = 0.f;
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const float scale = __uint_as_float(w[g] << 16), zero = __uint_as_float(w[g] & 0xffff0000u);
                        d0 = fmaf(scale, acc[g][2 * half], d0); d1 = fmaf(scale, acc[g][2 * half + 1], d1);
                        e0 = fmaf(zero, qz0[g], e0); e1 = fmaf(zero, qz1[g], e1);
                    }
                    z[s][2 * half] = fmaf(d0, qfac0, e0);
                    z[s][2 * half + 1] = fmaf(d1, qfac1, e1);
                }
            }
            next_slot();
            __syncwarp();
            if (issued < 2 * n) { issue(issued); ++issued; }
        }

        // ---- scales and zeros of the values, tokens out of sight, running maximum --------------------------------------
        if (!warp_wait(bars + 8 * get_slot, parity, abort_flag)) { given_up = true; break; }
        const uint32_t vbase = ring + get_slot * TB;
        float vs[2][2][G], vz[2][2][G];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t meta = vbase + Lay::pair(16 * s + 8 * half + gr, 0);
                uint32_t w[2];
                if (G == 2) { const uint2 v = lds64(meta); w[0] = v.x; w[1] = v.y; }
                else w[0] = w[1] = lds32(meta);
#pragma unroll
                for (int g = 0; g < G; ++g) { vs[s][half][g] = __uint_as_float(w[g] << 16); vz[s][half][g] = __uint_as_float(w[g] & 0xffff0000u); }
            }
        const int tok0 = (at.s.t0 + at.tile) * I4_TILE;
        if (tok0 < at.s.start || tok0 + I4_TILE > at.s.len) {     // (what lies out of sight is arbitrary bytes: nothing of it may count)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int tok = tok0 + 16 * s + 8 * half + gr;
                    if (tok < at.s.start || tok >= at.s.len) {
                        z[s][2 * half] = z[s][2 * half + 1] = -CUDART_INF_F;
#pragma unroll
                        for (int g = 0; g < G; ++g) vs[s][half][g] = vz[s][half][g] = 0.f;
                    }
                }
        }
        {
            const float x0 = fmaxf(fmaxf(z[0][0], z[0][2]), fmaxf(z[1][0], z[1][2])), x1 = fmaxf(fmaxf(z[0][1], z[0][3]), fmaxf(z[1][1], z[1][3]));
            float vm = 0.f;
#pragma unroll
            for (int g = 0; g < G; ++g) vm = fmaxf(vm, fmaxf(fmaxf(vs[0][0][g], vs[0][1][g]), fmaxf(vs[1][0][g], vs[1][1][g])));
            if (__any_sync(0xffffffffu, x0 > m0 || x1 > m1 || vm > vbound)) {
                float y0 = x0, y1 = x1;
#pragma unroll
                for (int s = 4; s < 32; s <<= 1) {
                    y0 = fmaxf(y0, __shfl_xor_sync(0xffffffffu, y0, s));
                    y1 = fmaxf(y1, __shfl_xor_sync(0xffffffffu, y1, s));
                    vm = fmaxf(vm, __shfl_xor_sync(0xffffffffu, vm, s));
                }
                const float n0 = y0 > m0 ? y0 + HEADROOM : m0, n1 = y1 > m1 ? y1 + HEADROOM : m1;
                float a0 = n0 > m0 ? ex2f(m0 - n0) : 1.f, a1 = n1 > m1 ? ex2f(m1 - n1) : 1.f;
                m0 = n0; m1 = n1;
                l0 *= a0; l1 *= a1;
#pragma unroll
                for (int g = 0; g < G; ++g) { zs0[g] *= a0; zs1[g] *= a1; }
                if (vm > vbound) {                                // power of two above the largest scale so far, with room
                    const float nb = __uint_as_float(min(max((__float_as_uint(vm) >> 23) + 2u, 27u), 254u) << 23);
                    const float r = vbound / nb;
                    a0 *= r; a1 *= r;
                    vbound = nb;
                    vfac = W_ONE / nb;
                }
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int s = 0; s < 2; ++s) { o[p][s][0] *= a0; o[p][s][1] *= a1; o[p][s][2] *= a0; o[p][s][3] *= a1; }
            }
        }

        // ---- weights and values --------------------------------------------------------------------------------------
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            uint32_t b_hi[G][2], b_lo[G][2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const float p0 = ex2f(z[s][2 * half] - m0), p1 = ex2f(z[s][2 * half + 1] - m1);
                l0 += p0; l1 += p1;
                const float f0 = p0 * vfac, f1 = p1 * vfac;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    zs0[g] = fmaf(p0, vz[s][half][g], zs0[g]);
                    zs1[g] = fmaf(p1, vz[s][half][g], zs1[g]);
                    const float w0 = f0 * vs[s][half][g], w1 = f1 * vs[s][half][g];
                    const uint32_t hi = pack_half(w0, w1);
                    const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hi));
                    const uint32_t lo = pack_half(w0 - back.x, w1 - back.y);
                    if (HG == 8) {
                        b_hi[g][half] = movmatrix_t(hi);
                        b_lo[g][half] = movmatrix_t(lo);
                    } else {
                        const uint32_t mine = HG == 4 ? (j < 2 ? hi : lo) : HG == 2 ? (j == 0 ? hi : j == 1 ? lo : 0u) : (j == 0 ? (hi & 0xffffu) | (lo & 0xffff0000u) : 0u);
                        b_hi[g][half] = movmatrix_t(mine);
                    }
                }
            }
            const int row = 16 * s + (lane & 15);
#pragma unroll
            for (int pp = 0; pp < NP; pp += 2) {
                uint32_t r[4];
                ldmatrix4t(vbase + row * Lay::ROW + (((pp + (lane >> 4)) ^ Lay::swizzle(row)) << 4), r);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t x = r[2 * h], y = r[2 * h + 1];
                    const int p = pp + h, g = p / 2;
#pragma unroll
                    for (int sh = 0; sh < 2; ++sh) {
                        const uint32_t a0 = (sh ? x >> 8 : x) & 0x000f000fu, a1 = (sh ? x >> 8 : x) & 0x00f000f0u;
                        const uint32_t a2 = (sh ? y >> 8 : y) & 0x000f000fu, a3 = (sh ? y >> 8 : y) & 0x00f000f0u;
                        mma16816(o[p][sh], a0, a1, a2, a3, b_hi[g][0], b_hi[g][1]);
                        if (HG == 8) mma16816(o[p][sh], a0, a1, a2, a3, b_lo[g][0], b_lo[g][1]);
                    }
                }
            }
        }
        next_slot();
        __syncwarp();
        if (issued < 2 * n) { issue(issued); ++issued; }

        // ---- end of the pair, or of the warp's share -------------------------------------------------------------------
        const bool ends = at.tile + 1 == at.s.tiles;
        if (ends || t + 1 == n) {
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) {
                l0 += __shfl_xor_sync(0xffffffffu, l0, s);
                l1 += __shfl_xor_sync(0xffffffffu, l1, s);
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    zs0[g] += __shfl_xor_sync(0xffffffffu, zs0[g], s);
                    zs1[g] += __shfl_xor_sync(0xffffffffu, zs1[g], s);
                }
            }
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float v = o[p][s][i];
                        if (HG == 4) v += __shfl_xor_sync(0xffffffffu, v, 2);
                        if (HG == 2) v += __shfl_xor_sync(0xffffffffu, v, 1);
                        o[p][s][i] = v * (16777216.f / W_ONE * (i < 2 ? 1.f : 0.0625f)) * vbound;
                    }
            if (HG == 1)
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int s = 0; s < 2; ++s) { o[p][s][0] += o[p][s][1]; o[p][s][2] += o[p][s][3]; }
            const int pair = at.b * a.hkv + at.kvh;
            const bool whole = ends && seg_first == 0;
            // the pieces of a warp that are not whole: one at its front, one at its back
            const bool front = !whole && seg_first != 0;
            float* dst = front ? reinterpret_cast<float*>(smem + P::HEADS) + warp * P::PIECE : reinterpret_cast<float*>(smem + warp * SLOTS * TB);
            if (2 * j < (HG == 1 ? 2 : HG)) {                     // lane (gr, j): heads 2 j, 2 j + 1, channels 32 p + 4 gr + 0..3
                float inv0 = 1.f, inv1 = 1.f;
                if (whole) {
                    inv0 = 1.f / (l0 + sink_mass(a, at.kvh * HG + head0, m0));
                    inv1 = 1.f / (l1 + sink_mass(a, at.kvh * HG + head1, m1));
                }
#pragma unroll
                for (int c = 0; c < (HG == 1 ? 1 : 2); ++c) {
                    const int h = c ? head1 : head0;
                    if (!whole && gr == 0) { dst[h * (D + 2)] = c ? m1 : m0; dst[h * (D + 2) + 1] = c ? l1 : l0; }
#pragma unroll
                    for (int p = 0; p < NP; ++p)
#pragma unroll
                        for (int s = 0; s < 2; ++s)
#pragma unroll
                            for (int hf = 0; hf < 2; ++hf) {
                                const int ch = 32 * p + 4 * gr + 2 * s + hf;
                                const float v = o[p][s][2 * hf + c] + (c ? zs1[p / 2] : zs0[p / 2]);
                                if (whole) write_out<D, HG>(a, pair, h * D + ch, v * (c ? inv1 : inv0));
                                else dst[h * (D + 2) + 2 + ch] = v;
                            }
                }
            }
            if (!whole && lane == 0) {
                misc[32 + 2 * warp + !front] = pair;
                misc[64 + 2 * warp + !front] = (seg_first == 0) | ends << 1;
            }
            fresh = true;
        }
        // ---- next tile
        if (++at.tile == at.s.tiles) {
            at.tile = 0;
            if (++at.kvh == a.hkv && t + 1 < n) {
                at.kvh = 0;
                do at.s = sight_of(a, ++at.b);
                while (at.s.tiles == 0 && at.b + 1 < a.batch);
            }
        }
    }
    if (given_up) {                                               // the copies in flight end before the shared memory does
        for (; taken < issued; next_slot()) mbar_wait_mma(bars + 8 * get_slot, parity, abort_flag);
        if (lane == 0) atomicOr(a.dev_status, NOVAKV_DEV_WAIT_TIMEOUT);
    }
    for (int b = blockIdx.x; b < a.batch; b += gridDim.x)         // sequences without a token
        if (sight_of(a, b).tiles == 0)
            for (int i = threadIdx.x; i < a.hkv * HG * D; i += THREADS) write_out<D, HG>(a, b * a.hkv, i, 0.f);

    // ---- join the warps' pieces --------------------------------------------------------------------------------------
    __syncthreads();
    int reach[2] = {-1, -1};
    for (int i0 = 0; i0 < 2 * WARPS;) {
        const int pair = misc[32 + i0];
        if (pair < 0) { ++i0; continue; }
        int i1 = i0, last = i0;
        for (; i1 < 2 * WARPS && (misc[32 + i1] == pair || misc[32 + i1] < 0); ++i1)
            if (misc[32 + i1] == pair) last = i1;
        const bool begins = misc[64 + i0] & 1, ends = misc[64 + last] >> 1;
        const int side = begins ? 1 : 0;
        if (!(begins && ends)) reach[side] = pair;
        float* to = a.part + ((size_t)blockIdx.x * 2 + side) * P::PIECE;
        for (int i = threadIdx.x; i < HG * D; i += THREADS) {
            const int h = i / D, c = i % D;
            float m = -CUDART_INF_F;
            for (int k = i0; k <= last; ++k)
                if (misc[32 + k] == pair)
                    m = fmaxf(m, ((k & 1) ? reinterpret_cast<const float*>(smem + (k >> 1) * SLOTS * TB) : reinterpret_cast<const float*>(smem + P::HEADS) + (k >> 1) * P::PIECE)[h * (D + 2)]);
            float acc = 0.f, l = 0.f;
            for (int k = i0; k <= last; ++k)
                if (misc[32 + k] == pair) {
                    const float* src = ((k & 1) ? reinterpret_cast<const float*>(smem + (k >> 1) * SLOTS * TB) : reinterpret_cast<const float*>(smem + P::HEADS) + (k >> 1) * P::PIECE) + h * (D + 2);
                    const float f = src[0] == -CUDART_INF_F ? 0.f : ex2f(src[0] - m);
                    acc = fmaf(f, src[2 + c], acc);
                    l = fmaf(f, src[1], l);
                }
            if (begins && ends) {
                write_out<D, HG>(a, pair, i, acc / (l + sink_mass(a, pair % a.hkv * HG + h, m)));
            } else {
                to[h * (D + 2) + 2 + c] = acc;
                if (c == 0) { to[h * (D + 2)] = m; to[h * (D + 2) + 1] = l; }
            }
        }
        i0 = last + 1;
    }
    if (threadIdx.x < 2) a.info[2 * blockIdx.x + threadIdx.x] = threadIdx.x ? reach[1] : reach[0];
}

// One block per CTA of the scan: joins the pair that begins in it and reaches over its back end, with the front pieces of the
// CTAs behind it.
constexpr int MERGE_THREADS = 512;
template <int D, int HG>
__global__ void __launch_bounds__(MERGE_THREADS)
novakv_int4_merge_kernel(const DecodeArgs a) {
    constexpr int PIECE = Plan<D, HG>::PIECE;
    novakv_grid_dependency_wait();
    const int c0 = blockIdx.x, pair = a.info[2 * c0 + 1];
    if (pair < 0) return;
    const int parts = 1 + __syncthreads_count(c0 + 1 + threadIdx.x < gridDim.x && a.info[2 * (c0 + 1 + threadIdx.x)] == pair);
    for (int i = threadIdx.x; i < HG * D; i += MERGE_THREADS) {
        const int h = i / D, c = i % D;
        float m = -CUDART_INF_F;
        for (int k = 0; k < parts; ++k) m = fmaxf(m, a.part[((size_t)(c0 + k) * 2 + (k == 0)) * PIECE + h * (D + 2)]);
        float acc = 0.f, l = 0.f;
        for (int k = 0; k < parts; ++k) {
            const float* src = a.part + ((size_t)(c0 + k) * 2 + (k == 0)) * PIECE + h * (D + 2);
            const float f = src[0] == -CUDART_INF_F ? 0.f : ex2f(src[0] - m);
            acc = fmaf(f, src[2 + c], acc);
            l = fmaf(f, src[1], l);
        }
        write_out<D, HG>(a, pair, i, acc / (l + sink_mass(a, pair % a.hkv * HG + h, m)));
    }
}

int scan_ctas(const novakv_ctx* ctx) { return ctx->scan_ctas > 0 && ctx->scan_ctas < ctx->n_sm ? ctx->scan_ctas : ctx->n_sm; }
size_t info_bytes(const novakv_ctx* ctx) { return ((size_t)ctx->n_sm * 2 * sizeof(int) + 255) & ~(size_t)255; }

template <int D, int HG>
novakv_status launch(novakv_ctx* ctx, DecodeArgs& a, void* workspace, cudaStream_t stream) {
    using P = Plan<D, HG>;
    auto* kern = novakv_int4_decode_kernel<D, HG>;
    const unsigned bit = 1u << (__builtin_ctz(HG) + (D == 128 ? 4 : 0));
    if (!(ctx->int4_opt_in & bit)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, P::TOTAL) != cudaSuccess) return NOVAKV_ECUDA;
        ctx->int4_opt_in |= bit;
    }
    a.info = (int*)workspace;
    a.part = (float*)((char*)workspace + info_bytes(ctx));
    const dim3 grid(scan_ctas(ctx));
    if (novakv_launch_pdl(kern, grid, dim3(THREADS), P::TOTAL, stream, a) != cudaSuccess) return NOVAKV_ECUDA;
    ctx->launches++;
    if (novakv_launch_pdl(novakv_int4_merge_kernel<D, HG>, grid, dim3(MERGE_THREADS), 0, stream, a) != cudaSuccess) return NOVAKV_ECUDA;
    ctx->launches++;
    return NOVAKV_OK;
}

}  // namespace

extern "C" size_t novakv_int4_workspace_bytes(const novakv_ctx* ctx, int batch) {
    if (!ctx || batch <= 0) return 0;
    return info_bytes(ctx) + (size_t)ctx->n_sm * 2 * ctx->hg * (ctx->cfg.head_dim + 2) * sizeof(float);
}

extern "C" novakv_status novakv_int4_decode_attention(novakv_ctx* ctx, const void* q, const uint8_t* k_pages, const uint8_t* v_pages,
    int n_pages, const int32_t* page_table, int max_pages_per_seq, const int32_t* seq_lens, int batch, float sm_scale, int window,
    const float* sink_logits, void* out, int out_is_fp32, void* workspace, size_t workspace_bytes, novakv_stream stream) {
    if (!ctx || batch < 0 || window < 0) return NOVAKV_EINVAL;
    if (batch == 0) return NOVAKV_OK;
    if (!q || !k_pages || !v_pages || !page_table || !seq_lens || !out) return NOVAKV_EINVAL;
    if (n_pages <= 0 || max_pages_per_seq <= 0) return NOVAKV_EPAGE;
    if (((uintptr_t)q | (uintptr_t)k_pages | (uintptr_t)v_pages) & 15) return NOVAKV_EINVAL;
    if (((uintptr_t)page_table | (uintptr_t)seq_lens | (uintptr_t)sink_logits) & 3) return NOVAKV_EINVAL;
    if ((uintptr_t)out & (out_is_fp32 ? 3 : 1)) return NOVAKV_EINVAL;
    if (!(sm_scale == sm_scale)) return NOVAKV_EINVAL;
    const long long hkv = ctx->cfg.n_kv_heads;
    // (tiles of the pools and of the batch are counted in 32 bits)
    if (n_pages * hkv * 2 > 0x7fffffffll || (long long)batch * max_pages_per_seq * 2 > 0x7fffffffll || batch * hkv > 0x7fffffffll || max_pages_per_seq * hkv * 2 > 0x7fffffffll ||
        max_pages_per_seq > 0x7fffffff / NOVAKV_PAGE_TOKENS) return NOVAKV_ESHAPE;
    if (!workspace || workspace_bytes < novakv_int4_workspace_bytes(ctx, batch) || ((uintptr_t)workspace & 255)) return NOVAKV_EWORKSPACE;
    const novakv_device_guard guard(ctx);
    if (!guard.ok) return NOVAKV_ECUDA;
    DecodeArgs a = {};
    a.q = (const __nv_bfloat16*)q;
    a.k_pages = k_pages; a.v_pages = v_pages; a.n_pages = n_pages;
    a.page_table = page_table; a.seq_lens = seq_lens; a.max_pages_per_seq = max_pages_per_seq; a.batch = batch; a.hkv = (int)hkv;
    a.window = window; a.out_is_fp32 = out_is_fp32; a.scale_log2 = sm_scale * 1.4426950408889634f; a.sink = sink_logits; a.out = out;
    a.dev_status = ctx->dev_status; a.wait_clocks = ctx->wait_clocks;
    cudaStream_t s = (cudaStream_t)stream;
    if (ctx->cfg.head_dim == 128)
        return ctx->hg == 1 ? launch<128, 1>(ctx, a, workspace, s) : ctx->hg == 2 ? launch<128, 2>(ctx, a, workspace, s) : launch<128, 4>(ctx, a, workspace, s);
    return ctx->hg == 1 ? launch<64, 1>(ctx, a, workspace, s) : ctx->hg == 2 ? launch<64, 2>(ctx, a, workspace, s)
         : ctx->hg == 4 ? launch<64, 4>(ctx, a, workspace, s) : launch<64, 8>(ctx, a, workspace, s);
}
