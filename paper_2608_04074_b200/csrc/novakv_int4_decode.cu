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
//  * Exactness: q is a bfloat16 number, exact in binary16 after a power of two (but for what is 2^-27 of the KV head's largest);
//    accumulators, softmax statistics and the zeros' share are binary32.  What the weights are rounded to goes by the output's type (FINE below).
//  * Streaming: the walk over (sequence, KV head, unit of 32 tokens at d = 128, 64 at d = 64) is cut evenly among the CTAs (one
//    per SM) and again among their 16 warps; each warp copies its units' keys and values (a bulk copy each) into a ring of its
//    own, a unit ahead of the one it works on, and no warp waits for another before the end.  (A page, 64 tokens, is 4.6 KB of a
//    side at d = 128; 16 warps x 2 units are 147 KB in flight or at work, three times what the latency of HBM asks for.)
//  * Join: what a warp has of a (sequence, KV head) pair that it does not hold whole goes to shared memory; the CTA joins these
//    pieces, and a second kernel joins the at most two per CTA that reach over its ends.
//
// B200, bf16 output, 6.56 TB/s of measured copy bandwidth: 64 x 16384 tokens (32 / 8 heads, d = 128) 193 to 197 us, 94 to 96 % of it; 8 x 16384
// 37 us, 62 %, of which launches, the look-up of the first units and the join are 8; 16 x 65536 (64 / 8 heads, d = 64) 115 us, 80 %, and
// 134 where it runs for seconds and the board's power limit takes the clock from 1.96 to 1.67 GHz: what is left is instructions (680 a unit,
// set-up and join included; 580 at d = 128).
#include <math_constants.h>

#include "novakv_int4.cuh"
#include "novakv_ops.cuh"
#include "novakv_tcgen05.cuh"

namespace {

constexpr int WARPS = 16, THREADS = WARPS * 32;
constexpr int SLOTS = 2;                     // ring of a warp, in units (keys and values)
// What setting up and writing out a (sequence, KV head) pair weighs in units, when the walk is cut.  32 sequences of 163 to 32768
// tokens (d = 128, 8 KV heads): 60.3 us at 0, 55.3 at 1, 51.6 at 2, 50.6 at 3, 50.9 at 5; 8 x 16384 tokens 37.4, 36.6, 36.3, 36.2, 36.2.
constexpr int PAIR_COST = 3;
constexpr int HEADROOM = 4;                  // a new maximum is set this many bits high: the next records need no rescaling
// The weight 1 at the largest scale so far, in binary16, once that scale is a quarter to a half of its power of two: what lies below
// 2^-34 of the largest weight (HEADROOM below 1) times that scale is cut off.
constexpr float W_ONE = 32768.f;

template <int D, int HG>
struct Plan {
    using Lay = I4Layout<D>;
    static constexpr int TILES = 128 / D;                          // tiles of a unit: what a warp copies, waits for and weighs at a time
    static constexpr int TOKENS = TILES * I4_TILE;
    static constexpr int HEAD = D + 4;                             // floats of a head's partial: maximum, sum, two unused, accumulators
    static constexpr int PIECE = HG * HEAD;
    static constexpr int SLOT = 2 * TILES * Lay::TILE_BYTES;
    static constexpr int RING = WARPS * SLOTS * SLOT;
    static constexpr int BARS = RING;
    static constexpr int FRONT = BARS + WARPS * SLOTS * 8;         // first pieces of the warps (the last ones lie in their rings)
    static constexpr int PREFIX = FRONT + WARPS * PIECE * 4;       // int [THREADS + 1]
    static constexpr int SEQS = PREFIX + (THREADS + 1) * 4;        // int [THREADS + 1]
    static constexpr int LENS = SEQS + (THREADS + 1) * 4;          // int [THREADS]
    static constexpr int MISC = (LENS + THREADS * 4 + 15) & ~15;
    static constexpr int TOTAL = MISC + 512;
    static_assert(SLOTS * SLOT >= PIECE * 4, "a warp's last piece fits into its ring");
    static_assert(TOTAL <= 227 * 1024, "shared memory");
};

struct DecodeArgs {
    const __nv_bfloat16* q;
    const uint8_t *k_pages, *v_pages;
    int n_pages;
    const int32_t *page_table, *seq_lens;
    int max_pages_per_seq, batch, hkv, window, out_is_fp32, one, few;   // one: a CTA for each pair, which joins all of it; few: at most 32 sequences, the cost fits 32 bits
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
// (x, y) += (a, b), (x, y) -= (a, b): one instruction for both
__device__ __forceinline__ void add2(float& x, float& y, float a, float b) {
    asm("{.reg .b64 u, v; mov.b64 u, {%0, %1}; mov.b64 v, {%2, %3}; add.rn.f32x2 u, u, v; mov.b64 {%0, %1}, u;}" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
__device__ __forceinline__ void sub2(float& x, float& y, float a, float b) {
    asm("{.reg .b64 u, v; mov.b64 u, {%0, %1}; mov.b64 v, {%2, %3}; sub.rn.f32x2 u, u, v; mov.b64 {%0, %1}, u;}" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
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

// Sequence b's units in sight and its first one.
struct Sight { int len, start, t0, units; };
template <int TOKENS>
__device__ __forceinline__ Sight sight_of(const DecodeArgs& a, int len) {
    Sight s;
    s.len = min(max(len, 0), a.max_pages_per_seq * NOVAKV_PAGE_TOKENS);
    s.start = a.window > 0 ? max(0, s.len - a.window) : 0;
    s.t0 = s.start / TOKENS;
    s.units = s.len > 0 ? (s.len + TOKENS - 1) / TOKENS - s.t0 : 0;
    return s;
}
// Where a unit of the walk lies: sequence, KV head, unit of the pair.
struct Place { int b, kvh, unit; Sight s; };
// The walk over all pairs: prefix[i] units (of one KV head) and seqs[i] sequences with a token lie before sequence i chunk.  It is
// cut where the cost is even: units, and PAIR_COST in front of each pair.
struct Walk {
    const int *prefix, *seqs, *lens;
    int chunk;
    __device__ __forceinline__ int len(const DecodeArgs& a, int b) const { return chunk == 1 ? lens[b] : a.seq_lens[b]; }
    __device__ __forceinline__ long long cost(const DecodeArgs& a, int i) const { return (prefix[i] + (long long)PAIR_COST * seqs[i]) * a.hkv; }
    // A sequence that is met on the way: cost and units before it.
    struct Stop { long long cost, units; int b; Sight s; };
    // The sequence in which cost x lies (x < the total), by a warp: 32 entries, then the 16 between two of them, then one by one.
    template <int TOKENS>
    __device__ __forceinline__ Stop find(const DecodeArgs& a, long long x, int lane) const {
        constexpr int STEP = THREADS / 32;
        int i = (31 - __clz(__ballot_sync(0xffffffffu, cost(a, lane * STEP) <= x))) * STEP;
        i += 31 - __clz(__ballot_sync(0xffffffffu, lane < STEP && cost(a, i + lane % STEP) <= x));
        Stop w = {cost(a, i), (long long)prefix[i] * a.hkv, i * chunk, {}};
        for (;; ++w.b) {
            w.s = sight_of<TOKENS>(a, len(a, w.b));
            const long long own = w.s.units > 0 ? (long long)(w.s.units + PAIR_COST) * a.hkv : 0;
            if (x < w.cost + own || w.b + 1 >= a.batch) return w;
            w.cost += own;
            w.units += (long long)w.s.units * a.hkv;
        }
    }
    // The first unit that is not before cost x, in the sequence where x lies; the units of the whole walk before it.
    __device__ __forceinline__ long long enter(const Stop& w, long long x, Place& p) const {
        const unsigned left = (unsigned)(x - w.cost), per = w.s.units + PAIR_COST, pair = left / per;
        p.b = w.b;
        p.s = w.s;
        p.kvh = (int)pair;
        p.unit = max((int)(left - pair * per) - PAIR_COST, 0);
        return w.units + (long long)pair * w.s.units + p.unit;
    }
    // to the pair that a unit counted from this one's first lies in
    template <int TOKENS>
    __device__ __forceinline__ void settle(const DecodeArgs& a, Place& p) const {
#pragma unroll 1
        while (p.unit >= p.s.units) {
            p.unit -= p.s.units;
            if (++p.kvh < a.hkv) continue;
            p.kvh = 0;
            do p.s = sight_of<TOKENS>(a, len(a, ++p.b));
            while (p.s.units == 0 && p.b + 1 < a.batch);
        }
    }
};

// two neighbouring channels of the output [batch][Hkv][Hg][D], i counted from the pair's first
template <int D, int HG>
__device__ __forceinline__ void write_out2(const DecodeArgs& a, int pair, int i, float x, float y) {
    const size_t oi = (size_t)pair * HG * D + i;
    if (a.out_is_fp32) *reinterpret_cast<float2*>(reinterpret_cast<float*>(a.out) + oi) = make_float2(x, y);
    else *reinterpret_cast<__nv_bfloat162*>(reinterpret_cast<__nv_bfloat16*>(a.out) + oi) = __floats2bfloat162_rn(x, y);
}
// the sink's share of a head's sum, relative to its maximum m
__device__ __forceinline__ float sink_mass(const DecodeArgs& a, int head, float m) {
    return a.sink != nullptr ? ex2f(fmaf(a.sink[head], 1.44269504f, -m)) : 0.f;
}

// Four codes of a word's 16-bit halves as binary16 numbers.  Plain: codes 0, 2 are c 2^-24, codes 1, 3 are 16 c 2^-24, five
// instructions.  FINE: all four in the upper bits of the mantissa, c 2^-18, eight instructions: the tensor core aligns products by
// the operands' exponents and cuts off what lies 2^-24 below, which for a subnormal number is counted from 2^-14 on, not from its
// first bit, so that small ones lose up to ten of the product's bits.
template <bool FINE>
__device__ __forceinline__ void unpack_codes(uint32_t x, uint32_t (&c)[4]) {
    if (FINE) {
        c[0] = x << 6 & 0x03c003c0u; c[1] = x << 2 & 0x03c003c0u; c[2] = x >> 2 & 0x03c003c0u; c[3] = x >> 6 & 0x03c003c0u;
    } else {
        const uint32_t y = x >> 8;
        c[0] = x & 0x000f000fu; c[1] = x & 0x00f000f0u; c[2] = y & 0x000f000fu; c[3] = y & 0x00f000f0u;
    }
}

// For the values, whose sums are taken apart every 32 tokens, four instructions: rows of codes c0 + 16 c1 (a byte) and of 16 c1 above
// them, from which the sums over c0 and c1 follow; likewise c2, c3.
__device__ __forceinline__ void unpack_bytes(uint32_t x, uint32_t (&c)[4]) {
    c[0] = x & 0x00ff00ffu; c[1] = x & 0x00f000f0u;
    c[2] = __byte_perm(x, 0, 0x4341); c[3] = c[2] & 0x00f000f0u;
}

// FINE: for binary32 outputs.  The products keep the bits that they would lose (unpack_codes) and the weights meet the codes as
// binary16 pairs hi + lo, in two products (8 x 16384 tokens: 46.9 us against 36.8).  Without, each product of a logit is cut off at 2^-15
// of what one step of its key's code moves it by in the query's largest channel (136 cuts at most, some 2^-11 in all as measured),
// and weight times scale is a binary16 number, 11 bits: off by 2^-11 of itself at most, an eighth of a bfloat16 output's own rounding.
// The codes that it meets count from their middle, 7.5 (wsum below), so that errors which agree - weights nearly alike over a long
// sequence - stay a part of the result and do not meet the zeros, whose sum is exact: at 16 x 65536 tokens, d = 64, and logits of a
// standard deviation of 3e-4 the output is then off by 1.66e-3 of its size, what its own rounding leaves, and by 3.6e-3 without.
template <int D, int HG, bool FINE>
__global__ void __launch_bounds__(THREADS, 1)
novakv_int4_decode_kernel(const DecodeArgs a) {
    using Lay = I4Layout<D>;
    using P = Plan<D, HG>;
    constexpr int G = Lay::GROUPS, NP = Lay::PIECES, TB = Lay::TILE_BYTES, UB = P::TILES * TB, S = P::TOKENS / 16;
    // Columns of the products.  Eight heads fill the eight columns, and a lane holds two tokens of 16 for two heads.  With fewer
    // heads columns 4..7 repeat columns 0..3, and the lanes that hold them take the other token: one token for two heads each.
    constexpr bool SPLIT = HG < 8;
    constexpr int R = SPLIT ? 1 : 2, COLS = SPLIT ? 4 : 8;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, j = lane & 3, up = SPLIT ? j >> 1 : 0, jj = SPLIT ? j & 1 : j;
    int *prefix = reinterpret_cast<int*>(smem + P::PREFIX), *lens = reinterpret_cast<int*>(smem + P::LENS);
    int* misc = reinterpret_cast<int*>(smem + P::MISC);           // 1 abort flag, 8..9 wait limit, 16..31 warp sums, 32..63 pieces' pairs, 64..95 their ends, 96..111 warp sums
    volatile int* abort_flag = misc + 1;
    const uint32_t ring = smem_u32(smem) + warp * SLOTS * P::SLOT, bars = smem_u32(smem + P::BARS) + warp * SLOTS * 8;
    if (lane < SLOTS) mbar_init(bars + 8 * lane, 1);
    if (threadIdx.x == 0) {
        misc[1] = 0;
        *reinterpret_cast<long long*>(misc + 1 + MBAR_LIMIT) = a.wait_clocks;
    }
    if (threadIdx.x < 2 * WARPS) misc[32 + threadIdx.x] = -1;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    novakv_grid_dependency_wait();

    // ---- the walk over (sequence, KV head, unit), and this warp's share of it
    int* seqs = reinterpret_cast<int*>(smem + P::SEQS);
    const Walk walk = {prefix, seqs, a.few ? a.seq_lens : lens, (a.batch + THREADS - 1) / THREADS};
    Place at = {};                                                // the warp's first unit
    int n = 0;
    bool idle = false;                                            // some sequence has no token
    if (a.one) {
        at.b = blockIdx.x / a.hkv;
        at.kvh = blockIdx.x - at.b * a.hkv;
        const int len = a.seq_lens[at.b];
        at.s = sight_of<P::TOKENS>(a, len);
        if (threadIdx.x == 0 && at.kvh == 0 && len > a.max_pages_per_seq * NOVAKV_PAGE_TOKENS) atomicOr(a.dev_status, NOVAKV_DEV_BAD_LENGTH);
        at.unit = at.s.units * warp / WARPS;
        n = at.s.units * (warp + 1) / WARPS - at.unit;
        idle = at.s.units == 0;
        __syncthreads();
    } else if (a.few) {
        // Up to 32 sequences, a lane each: every warp forms the walk itself, and nothing of it waits for another.  (3000 cycles
        // to a warp's first unit where the general way below takes 4600: code that runs once runs at the pace of its fetches.)
        const int len = lane < a.batch ? a.seq_lens[lane] : 0;
        if (blockIdx.x == 0 && warp == 0 && len > a.max_pages_per_seq * NOVAKV_PAGE_TOKENS) atomicOr(a.dev_status, NOVAKV_DEV_BAD_LENGTH);
        const int units = sight_of<P::TOKENS>(a, len).units, own = units > 0 ? (units + PAIR_COST) * a.hkv : 0;
        int cost = own, before = units;
#pragma unroll 1
        for (int s = 1; s < 32; s <<= 1) {
            const int c = __shfl_up_sync(0xffffffffu, cost, s), u = __shfl_up_sync(0xffffffffu, before, s);
            if (lane >= s) { cost += c; before += u; }
        }
        const unsigned total = __shfl_sync(0xffffffffu, cost, 31), all = __shfl_sync(0xffffffffu, before, 31) * a.hkv;
        cost -= own;
        before = (before - units) * a.hkv;
        idle = __any_sync(0xffffffffu, lane < a.batch && units == 0);
        const unsigned ctas = max(1u, min(gridDim.x, total / (PAIR_COST + 1))), cta = min(blockIdx.x, ctas), each = total / ctas, more = total - each * ctas;
        const unsigned c0 = each * cta + min(cta, more), share = cta < ctas ? each + (cta < more) : 0;
        const unsigned x[2] = {c0 + (share * warp >> 4), c0 + (share * (warp + 1) >> 4)};
        unsigned units_at[2] = {all, all};
        if (x[0] < x[1]) {
#pragma unroll 1
            for (int e = 1; e >= 0; --e) {
                const unsigned xe = e ? x[1] : x[0];
                if (xe >= total) continue;
                const int b = 31 - __clz(__ballot_sync(0xffffffffu, own > 0 && (unsigned)cost <= xe));
                at.b = b;
                at.s = sight_of<P::TOKENS>(a, __shfl_sync(0xffffffffu, len, b));
                const unsigned left = xe - __shfl_sync(0xffffffffu, cost, b), per = at.s.units + PAIR_COST;
                at.kvh = left / per;
                at.unit = max((int)(left - at.kvh * per) - PAIR_COST, 0);
                const unsigned u = __shfl_sync(0xffffffffu, before, b) + at.kvh * at.s.units + at.unit;
                if (e) units_at[1] = u; else units_at[0] = u;
            }
            n = units_at[1] - units_at[0];
        }
        __syncthreads();
    } else {
        int sum = 0, used = 0;
        for (int b = threadIdx.x * walk.chunk; b < min(a.batch, ((int)threadIdx.x + 1) * walk.chunk); ++b) {
            const int len = a.seq_lens[b], units = sight_of<P::TOKENS>(a, len).units;
            sum += units;
            used += units > 0;
            if (walk.chunk == 1) lens[b] = len;
            if (blockIdx.x == 0 && len > a.max_pages_per_seq * NOVAKV_PAGE_TOKENS) atomicOr(a.dev_status, NOVAKV_DEV_BAD_LENGTH);
            idle |= units == 0;
        }
        int inc = sum, inc_used = used;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, inc, s), u = __shfl_up_sync(0xffffffffu, inc_used, s);
            if (lane >= s) { inc += o; inc_used += u; }
        }
        if (lane == 31) { misc[16 + warp] = inc; misc[96 + warp] = inc_used; }
        __syncthreads();
        int base = lane < warp ? misc[16 + (lane & (WARPS - 1))] : 0, base_used = lane < warp ? misc[96 + (lane & (WARPS - 1))] : 0;
#pragma unroll
        for (int s = 1; s < WARPS; s <<= 1) {                     // (lanes from WARPS on hold 0)
            base += __shfl_xor_sync(0xffffffffu, base, s);
            base_used += __shfl_xor_sync(0xffffffffu, base_used, s);
        }
        prefix[threadIdx.x + 1] = __shfl_sync(0xffffffffu, base, 0) + inc;
        seqs[threadIdx.x + 1] = __shfl_sync(0xffffffffu, base_used, 0) + inc_used;
        if (threadIdx.x == 0) prefix[0] = seqs[0] = 0;
        idle = __syncthreads_or(idle);
        const long long total = walk.cost(a, THREADS);
        // (no CTA in between without a unit, since the join goes by the CTAs' order: a CTA takes more cost than a pair's own)
        const unsigned ctas = (unsigned)max(1ll, min((long long)gridDim.x, total / (PAIR_COST + 1))), cta = min(blockIdx.x, ctas);
        const long long each = total >> 32 ? total / ctas : (long long)((unsigned)total / ctas);
        const unsigned more = (unsigned)(total - each * ctas);    // (the first so many take one more)
        const long long c0 = each * cta + min(cta, more), c1 = cta < ctas ? each * (cta + 1) + min(cta + 1, more) : c0;
        const long long x0 = c0 + ((c1 - c0) * warp >> 4), x1 = c0 + ((c1 - c0) * (warp + 1) >> 4);
        static_assert(WARPS == 16, "a sixteenth of a CTA's share");
        if (x0 < x1) {
            auto stop = walk.find<P::TOKENS>(a, x0, lane);
            const long long first = walk.enter(stop, x0, at);
            long long behind = (long long)prefix[THREADS] * a.hkv;
            if (x1 < total) {
                if (x1 >= stop.cost + (long long)(stop.s.units + PAIR_COST) * a.hkv) stop = walk.find<P::TOKENS>(a, x1, lane);
                Place unused;
                behind = walk.enter(stop, x1, unused);
            }
            n = (int)(behind - first);
        }
    }

    // ---- producer: the units' chunks 32 at a time, the next batch always on its way
    const Place begin = at;
    auto chunk_of = [&](int i) -> int {                           // (page, KV head, part of the page) of the warp's i-th unit
        if (i >= n) return 0;
        Place p = begin;
        p.unit += i;
        walk.settle<P::TOKENS>(a, p);
        const int unit = p.s.t0 + p.unit;
        int page = a.page_table[(size_t)p.b * a.max_pages_per_seq + unit * P::TOKENS / NOVAKV_PAGE_TOKENS];
        if (page < 0 || page >= a.n_pages) {
            atomicOr(a.dev_status, NOVAKV_DEV_BAD_PAGE);
            page = 0;
        }
        return (page * a.hkv + p.kvh) * (NOVAKV_PAGE_TOKENS / P::TOKENS) + unit % (NOVAKV_PAGE_TOKENS / P::TOKENS);
    };
    int chunks = 0, chunks_next = 0;
    auto issue = [&](int t) {                                     // unit t into slot t % SLOTS
        if ((t & 31) == 0 && t > 0) {
            chunks = chunks_next;
            chunks_next = chunk_of(t + 32 + lane);
        }
        const size_t at = (size_t)__shfl_sync(0xffffffffu, chunks, t & 31) * UB;
        if (lane == 0) {
            const uint32_t bar = bars + 8 * (t % SLOTS), dst = ring + (t % SLOTS) * P::SLOT;
            mbar_expect_tx(bar, 2 * UB);
            bulk_copy(dst, a.k_pages + at, UB, bar);
            bulk_copy(dst + UB, a.v_pages + at, UB, bar);
        }
    };
    if (n > 0) {
        chunks = chunk_of(lane);
        __syncwarp();
        for (int t = 0; t < min(SLOTS, n); ++t) issue(t);
        if (n > 32) chunks_next = chunk_of(32 + lane);
        __syncwarp();
    }

    // ---- consumer ---------------------------------------------------------------------------------------------------
    // the lane's columns 2 jj, 2 jj + 1: with fewer heads than columns some repeat, and are not looked at in the end
    const int head0 = 2 * jj % HG, head1 = (2 * jj + 1) % HG;
    // lane's row of the matrix loads: token lane % 16 (of 16), piece lane / 16 (of two)
    const uint32_t mat = (lane & 15) * Lay::ROW + (((lane >> 4) ^ Lay::swizzle(lane & 15)) << 4);
    const uint32_t pairs = Lay::pair(8 * up + gr, 0);
    bool given_up = n > 0 && a.wait_clocks == 0;                  // (a limit of 0: before the first look)
    int t = 0;
#pragma unroll 1
    while (t < n && !given_up) {
        // ---- a (sequence, KV head) pair: its queries as the products' columns
        const int seg_first = at.unit, seg_n = min(at.s.units - at.unit, n - t);
        uint32_t qf[NP][2][2];
        float qfac, qz0[G], qz1[G], mid0[G], mid1[G];                // (mid: FINE alone, -8 times the sums of q as the products have it)
        {
            const __nv_bfloat16* qp = a.q + (((size_t)at.b * a.hkv + at.kvh) * HG + gr % COLS % HG) * D + 8 * j;
            uint4 w[NP];
            float mx = 0.f;
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                w[p] = *reinterpret_cast<const uint4*>(qp + 32 * p);
                const uint32_t ww[4] = {w[p].x, w[p].y, w[p].z, w[p].w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    mx = fmaxf(mx, fmaxf(fabsf(__uint_as_float(ww[i] << 16)), fabsf(__uint_as_float(ww[i] & 0xffff0000u))));
            }
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            if (!(mx < CUDART_INF_F)) mx = 0.f;                   // (a head with an infinity does not decide for the others)
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
            // 2^e brings the heads' largest coordinate just below 2^15: their eight bits fit down to 2^-31 of it, 2^-27
            // where a sixteenth of them is taken
            const int e = min(15 - ((int)(__float_as_uint(mx) >> 23) - 126), 120);
            const float f = __uint_as_float((uint32_t)(e + 127) << 23), odd = FINE ? f : f * 0.0625f;
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
                for (int s = 0; s < 2; ++s) {                     // codes 2 s, 2 s + 1 of a half: channels 8 j + 2 s + {0, 4}, + {1, 5}
                    qf[p][s][0] = pack_half(x[2 * s] * f, x[2 * s + 4] * f);
                    qf[p][s][1] = pack_half(x[2 * s + 1] * odd, x[2 * s + 5] * odd);
                }
            }
            const int back = (FINE ? 18 : 24) - e;                 // (-102 to 137: in two steps)
            qfac = a.scale_log2 * __uint_as_float((uint32_t)(back / 2 + 127) << 23) * __uint_as_float((uint32_t)(back - back / 2 + 127) << 23);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 1);
                sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 2);
                if (FINE) {                                       // codes are counted from the middle, 8: what is taken off is small
                    const float u = sum[g] * f * -0x1p-15f;
                    mid0[g] = __shfl_sync(0xffffffffu, u, 8 * jj);
                    mid1[g] = __shfl_sync(0xffffffffu, u, 8 * jj + 4);
                }
                qz0[g] = a.scale_log2 * __shfl_sync(0xffffffffu, sum[g], 8 * jj);     // (lane 4 c holds column c)
                qz1[g] = a.scale_log2 * __shfl_sync(0xffffffffu, sum[g], 8 * jj + 4);
            }
        }
        float m0 = -CUDART_INF_F, m1 = m0, l0 = 0.f, l1 = 0.f, zs0[G], zs1[G], vbound = 0.f, vfac = 0.f;
        float o[NP][2][4], wsum0[G], wsum1[G];                       // (wsum: bf16 outputs alone, the sums of the weights that met the codes)
#pragma unroll
        for (int g = 0; g < G; ++g) zs0[g] = zs1[g] = wsum0[g] = wsum1[g] = 0.f;
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[p][s][i] = 0.f;
        // tokens in sight, counted from the unit's first one
        int lo = at.s.start - (at.s.t0 + at.unit) * P::TOKENS, hi = at.s.len - (at.s.t0 + at.unit) * P::TOKENS;

#pragma unroll 1
        for (const int end = t + seg_n; t < end; ++t, lo -= P::TOKENS, hi -= P::TOKENS) {
            const uint32_t kbase = ring + (t % SLOTS) * P::SLOT, vbase = kbase + UB;
            if (!warp_wait(bars + 8 * (t % SLOTS), t / SLOTS & 1, abort_flag)) { given_up = true; break; }

            // ---- logits: z[s][r] of token 16 s + 8 (SPLIT ? up : r) + gr
            float z0[S][R], z1[S][R];
#pragma unroll
            for (int s = 0; s < S; ++s) {
                float acc[G][4];
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[g][i] = !FINE ? 0.f : (i & 1) ? mid1[g] : mid0[g];
#pragma unroll
                for (int pp = 0; pp < NP; pp += 2) {
                    uint32_t r[4];
                    ldmatrix4((kbase + mat ^ pp << 4) + s / 2 * TB + s % 2 * 16 * Lay::ROW, r);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t x[4], y[4];
                        unpack_codes<FINE>(r[2 * h], x);
                        unpack_codes<FINE>(r[2 * h + 1], y);
                        mma16816(acc[(pp + h) / 2], x[0], y[0], x[1], y[1], qf[pp + h][0][0], qf[pp + h][0][1]);
                        mma16816(acc[(pp + h) / 2], x[2], y[2], x[3], y[3], qf[pp + h][1][0], qf[pp + h][1][1]);
                    }
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const uint32_t meta = kbase + pairs + s / 2 * TB + (s % 2 * 16 + 8 * r) * G * 4;
                    uint32_t w[2];
                    if (G == 2) { const uint2 v = lds64(meta); w[0] = v.x; w[1] = v.y; }
                    else w[0] = w[1] = lds32(meta);
                    float d0 = 0.f, d1 = 0.f;
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const float step = __uint_as_float(w[g] << 16), scale = step * qfac;
                        const float zero = FINE ? fmaf(8.f, step, __uint_as_float(w[g] & 0xffff0000u)) : __uint_as_float(w[g] & 0xffff0000u);
                        const float c0 = SPLIT ? (up ? acc[g][2] : acc[g][0]) : acc[g][2 * r], c1 = SPLIT ? (up ? acc[g][3] : acc[g][1]) : acc[g][2 * r + 1];
                        d0 = fmaf(scale, c0, g ? fmaf(zero, qz0[g], d0) : zero * qz0[g]);
                        d1 = fmaf(scale, c1, g ? fmaf(zero, qz1[g], d1) : zero * qz1[g]);
                    }
                    z0[s][r] = d0;
                    z1[s][r] = d1;
                }
            }

            // ---- scales and zeros of the values, tokens out of sight, running maximum
            float vs[S][R][G], vz[S][R][G];
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const uint32_t meta = vbase + pairs + s / 2 * TB + (s % 2 * 16 + 8 * r) * G * 4;
                    uint32_t w[2];
                    if (G == 2) { const uint2 v = lds64(meta); w[0] = v.x; w[1] = v.y; }
                    else w[0] = w[1] = lds32(meta);
#pragma unroll
                    for (int g = 0; g < G; ++g) { vs[s][r][g] = __uint_as_float(w[g] << 16); vz[s][r][g] = __uint_as_float(w[g] & 0xffff0000u); }
                }
            if (lo > 0 || hi < P::TOKENS) {                       // (what lies out of sight is arbitrary bytes: nothing of it may count)
#pragma unroll
                for (int s = 0; s < S; ++s)
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const int tok = 16 * s + 8 * (SPLIT ? up : r) + gr;
                        if (tok < lo || tok >= hi) {
                            z0[s][r] = z1[s][r] = -CUDART_INF_F;
#pragma unroll
                            for (int g = 0; g < G; ++g) vs[s][r][g] = vz[s][r][g] = 0.f;
                        }
                    }
            }
            {
                float x0 = z0[0][0], x1 = z1[0][0], vm = 0.f;
#pragma unroll
                for (int s = 0; s < S; ++s)
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        x0 = fmaxf(x0, z0[s][r]);
                        x1 = fmaxf(x1, z1[s][r]);
#pragma unroll
                        for (int g = 0; g < G; ++g) vm = fmaxf(vm, vs[s][r][g]);
                    }
                if (__any_sync(0xffffffffu, x0 > m0 || x1 > m1 || vm > vbound)) {
#pragma unroll
                    for (int s = SPLIT ? 2 : 4; s < 32; s <<= 1) {
                        x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, s));
                        x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, s));
                    }
#pragma unroll
                    for (int s = 1; s < 32; s <<= 1) vm = fmaxf(vm, __shfl_xor_sync(0xffffffffu, vm, s));
                    const float n0 = x0 > m0 ? x0 + HEADROOM : m0, n1 = x1 > m1 ? x1 + HEADROOM : m1;
                    float a0 = n0 > m0 ? ex2f(m0 - n0) : 1.f, a1 = n1 > m1 ? ex2f(m1 - n1) : 1.f;
                    m0 = n0; m1 = n1;
                    l0 *= a0; l1 *= a1;
#pragma unroll
                    for (int g = 0; g < G; ++g) { zs0[g] *= a0; zs1[g] *= a1; }
                    if (vm > vbound) {                            // power of two above the largest scale so far, with room
                        const float nb = __uint_as_float(min(max((__float_as_uint(vm) >> 23) + 2u, 27u), 254u) << 23);
                        const float r = vbound / nb;
                        a0 *= r; a1 *= r;
                        vbound = nb;
                        vfac = W_ONE / nb;
                    }
#pragma unroll
                    for (int g = 0; g < G; ++g) { wsum0[g] *= a0; wsum1[g] *= a1; }
#pragma unroll
                    for (int p = 0; p < NP; ++p)
#pragma unroll
                        for (int s = 0; s < 2; ++s) { o[p][s][0] *= a0; o[p][s][1] *= a1; o[p][s][2] *= a0; o[p][s][3] *= a1; }
                }
            }

            // ---- weights and values, in sums of 32 tokens that are added in binary32: the tensor core cuts sums off instead of
            // rounding them, which over a long sequence of like weights would add up against a result that is small beside them (one
            // accumulator over a warp's 3500 tokens of a flat attention, 16 x 65536, d = 64: 14 % of the result; so 2^-10 of it).
            // The codes count from their middle, 7.5, since a sum from 0 would be 4 to 1000 times the result: FINE by a product with the
            // constant -7.5 of all of them, bf16 outputs by the weights' sum afterwards (a product there, as well: 197 against 193 us).
            // FINE: hi and lo parts apart.  Sums over hi parts are exact (15 bits a product) while the weights of 32 tokens lie within
            // 2^10 of one another; with lo parts in the same sum each of these was cut off at 2^-20 of a code's step, always towards
            // zero: 4e-5 of a flat output over 32768 tokens, 2e-7 so, which is a binary32 evaluation's.
            constexpr int SB = 2;
#pragma unroll
            for (int sb = 0; sb < S; sb += SB) {
                float p0[SB][R], p1[SB][R];
#pragma unroll
                for (int e = 0; e < SB; ++e)
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        p0[e][r] = ex2f(z0[sb + e][r] - m0); p1[e][r] = ex2f(z1[sb + e][r] - m1);
                        l0 += p0[e][r]; l1 += p1[e][r];
                    }
#pragma unroll
                for (int g = 0; g < G; ++g) {                     // (a group's weights, then its two pieces: few registers at a time)
                    uint32_t b_hi[SB][2], b_lo[SB][2];
#pragma unroll
                    for (int e = 0; e < SB; ++e)
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            const int s = sb + e;
                            const float zero = fmaf(7.5f, vs[s][r][g], vz[s][r][g]);
                            zs0[g] = fmaf(p0[e][r], zero, zs0[g]);
                            zs1[g] = fmaf(p1[e][r], zero, zs1[g]);
                            const float f = vfac * vs[s][r][g], w0 = p0[e][r] * f, w1 = p1[e][r] * f;
                            const uint32_t hi16 = pack_half(w0, w1), x = movmatrix_t(hi16);
                            const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hi16));
                            if (!FINE) add2(wsum0[g], wsum1[g], back.x, back.y);
                            // SPLIT: columns 0..3 take the lower eight tokens, columns 4..7 the upper ones
                            if (SPLIT) { b_hi[e][0] = gr < 4 ? x : 0u; b_hi[e][1] = gr < 4 ? 0u : x; }
                            else b_hi[e][r] = x;
                            if (FINE) {
                                const uint32_t y = movmatrix_t(pack_half(w0 - back.x, w1 - back.y));
                                if (SPLIT) { b_lo[e][0] = gr < 4 ? y : 0u; b_lo[e][1] = gr < 4 ? 0u : y; }
                                else b_lo[e][r] = y;
                            }
                        }
                    float mid[4] = {0.f, 0.f, 0.f, 0.f}, mid_lo[4] = {0.f, 0.f, 0.f, 0.f};
                    if (FINE) {
                        constexpr uint32_t M = 0x81e081e0u;       // -7.5 2^-18 twice
#pragma unroll
                        for (int e = 0; e < SB; ++e) {
                            mma16816(mid, M, M, M, M, b_hi[e][0], b_hi[e][1]);
                            mma16816(mid_lo, M, M, M, M, b_lo[e][0], b_lo[e][1]);
                        }
                    }
                    uint32_t r[SB][4];
#pragma unroll
                    for (int e = 0; e < SB; ++e) ldmatrix4t((vbase + mat ^ 2 * g << 4) + (sb + e) / 2 * TB + (sb + e) % 2 * 16 * Lay::ROW, r[e]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int p = 2 * g + h;
                        uint32_t x[SB][4], y[SB][4];
#pragma unroll
                        for (int e = 0; e < SB; ++e) {
                            if (!FINE) { unpack_bytes(r[e][2 * h], x[e]); unpack_bytes(r[e][2 * h + 1], y[e]); }
                            else { unpack_codes<FINE>(r[e][2 * h], x[e]); unpack_codes<FINE>(r[e][2 * h + 1], y[e]); }
                        }
#pragma unroll
                        for (int sh = 0; sh < 2; ++sh) {
                            float sum[4] = {mid[0], mid[1], mid[2], mid[3]}, sum_lo[4] = {mid_lo[0], mid_lo[1], mid_lo[2], mid_lo[3]};
#pragma unroll
                            for (int e = 0; e < SB; ++e) {
                                mma16816(sum, x[e][2 * sh], x[e][2 * sh + 1], y[e][2 * sh], y[e][2 * sh + 1], b_hi[e][0], b_hi[e][1]);
                                if (FINE) mma16816(sum_lo, x[e][2 * sh], x[e][2 * sh + 1], y[e][2 * sh], y[e][2 * sh + 1], b_lo[e][0], b_lo[e][1]);
                            }
                            if (FINE) {
                                add2(sum[0], sum[1], sum_lo[0], sum_lo[1]);
                                add2(sum[2], sum[3], sum_lo[2], sum_lo[3]);
                            } else {                              // (c0 + 16 c1 and 16 c1)
                                sub2(sum[0], sum[1], sum[2], sum[3]);
                            }
                            add2(o[p][sh][0], o[p][sh][1], sum[0], sum[1]);
                            add2(o[p][sh][2], o[p][sh][3], sum[2], sum[3]);
                        }
                    }
                }
            }
            __syncwarp();
            if (t + SLOTS < n) issue(t + SLOTS);
        }
        if (given_up) break;

        // ---- end of the pair, or of the warp's share
#pragma unroll
        for (int s = SPLIT ? 2 : 4; s < 32; s <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, s);
            l1 += __shfl_xor_sync(0xffffffffu, l1, s);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                zs0[g] += __shfl_xor_sync(0xffffffffu, zs0[g], s);
                zs1[g] += __shfl_xor_sync(0xffffffffu, zs1[g], s);
                if (FINE) continue;
                wsum0[g] += __shfl_xor_sync(0xffffffffu, wsum0[g], s);
                wsum1[g] += __shfl_xor_sync(0xffffffffu, wsum1[g], s);
            }
        }
        if (!FINE) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                zs0[g] = fmaf(wsum0[g] * (-7.5f / W_ONE), vbound, zs0[g]);
                zs1[g] = fmaf(wsum1[g] * (-7.5f / W_ONE), vbound, zs1[g]);
            }
        }
        const bool ends = seg_first + seg_n == at.s.units, whole = ends && seg_first == 0;
        const int pair = at.b * a.hkv + at.kvh;
        // the pieces of a warp that are not whole: one at its front (it does not begin its pair), one at its back
        const bool front = seg_first != 0;
        float* dst = reinterpret_cast<float*>(front ? smem + P::FRONT + warp * P::PIECE * 4 : smem + warp * SLOTS * P::SLOT);
        float inv0 = 1.f, inv1 = 1.f;
        if (whole) {
            inv0 = 1.f / (l0 + sink_mass(a, at.kvh * HG + head0, m0));
            inv1 = 1.f / (l1 + sink_mass(a, at.kvh * HG + head1, m1));
        } else if (gr == 0 && up == 0) {
            *reinterpret_cast<float2*>(dst + head0 * P::HEAD) = make_float2(m0, l0);
            if (HG > 1) *reinterpret_cast<float2*>(dst + head1 * P::HEAD) = make_float2(m1, l1);
        }
        constexpr float UNIT = (FINE ? 262144.f : 16777216.f) / W_ONE;
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int s = 0; s < 2; ++s) {                         // channels 32 p + 4 gr + 2 s, + 1 of the lane's two heads
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = o[p][s][i];
                    if (SPLIT) v[i] += __shfl_xor_sync(0xffffffffu, v[i], 2);
                    v[i] = fmaf(v[i] * (i < 2 || FINE ? UNIT : UNIT * 0.0625f), vbound, (i & 1) ? zs1[p / 2] : zs0[p / 2]);
                }
                if (2 * jj >= HG || (SPLIT && s != up)) continue; // (both halves hold the sums: each writes one s)
                const int ch = 32 * p + 4 * gr + 2 * s;
                if (whole) {
                    write_out2<D, HG>(a, pair, head0 * D + ch, v[0] * inv0, v[2] * inv0);
                    if (HG > 1) write_out2<D, HG>(a, pair, head1 * D + ch, v[1] * inv1, v[3] * inv1);
                } else {
                    *reinterpret_cast<float2*>(dst + head0 * P::HEAD + 4 + ch) = make_float2(v[0], v[2]);
                    if (HG > 1) *reinterpret_cast<float2*>(dst + head1 * P::HEAD + 4 + ch) = make_float2(v[1], v[3]);
                }
            }
        if (!whole && lane == 0) {
            misc[32 + 2 * warp + !front] = pair;
            misc[64 + 2 * warp + !front] = (seg_first == 0) | ends << 1;
        }
        // ---- next pair
        if (t < n) {
            at.unit = 0;
            if (++at.kvh == a.hkv) {
                at.kvh = 0;
                do at.s = sight_of<P::TOKENS>(a, walk.len(a, ++at.b));
                while (at.s.units == 0 && at.b + 1 < a.batch);
            }
        }
    }
    if (given_up) {                                               // the copies in flight end before the shared memory does
        for (const int end = min(t + SLOTS, n); t < end; ++t) mbar_wait_mma(bars + 8 * (t % SLOTS), t / SLOTS & 1, abort_flag);
        if (lane == 0) atomicOr(a.dev_status, NOVAKV_DEV_WAIT_TIMEOUT);
    }
    if (idle) {                                                   // sequences without a token
        if (a.one) {
            for (int i = 2 * threadIdx.x; i < HG * D; i += 2 * THREADS) write_out2<D, HG>(a, blockIdx.x, i, 0.f, 0.f);
            return;
        }
        for (int b = blockIdx.x; b < a.batch; b += gridDim.x)
            if (sight_of<P::TOKENS>(a, walk.len(a, b)).units == 0)
                for (int i = 2 * threadIdx.x; i < a.hkv * HG * D; i += 2 * THREADS) write_out2<D, HG>(a, b * a.hkv, i, 0.f, 0.f);
    }

    // ---- join the warps' pieces: they lie in the order of the walk, those of a pair side by side; a warp takes a head of a pair
    __syncthreads();
    const int mine = misc[32 + lane], ends_of = mine >= 0 ? misc[64 + lane] : 0;
    const uint32_t valid = __ballot_sync(0xffffffffu, mine >= 0), below = valid & ((1u << lane) - 1);
    const int before = __shfl_sync(0xffffffffu, mine, below ? 31 - __clz(below) : 0);
    uint32_t starts = __ballot_sync(0xffffffffu, mine >= 0 && (below == 0 || before != mine));
    int reach_front = -1, reach_back = -1, task = 0;
    while (starts) {
        const int first = __ffs(starts) - 1, pair = __shfl_sync(0xffffffffu, mine, first);
        starts &= starts - 1;
        const uint32_t pieces = __ballot_sync(0xffffffffu, mine == pair);
        const bool begins = __shfl_sync(0xffffffffu, ends_of, first) & 1, ends = __shfl_sync(0xffffffffu, ends_of, 31 - __clz(pieces)) >> 1;
        if (!begins) reach_front = pair;
        else if (!ends) reach_back = pair;
        for (int h = 0; h < HG; ++h) {
            if ((task++ & (WARPS - 1)) != warp) continue;
            auto piece = [&](int k) { return reinterpret_cast<const float*>(k & 1 ? smem + (k >> 1) * SLOTS * P::SLOT : smem + P::FRONT + (k >> 1) * P::PIECE * 4) + h * P::HEAD; };
            const float2 ml = mine == pair ? *reinterpret_cast<const float2*>(piece(lane)) : make_float2(-CUDART_INF_F, 0.f);
            float m = ml.x;
#pragma unroll
            for (int s = 1; s < 32; s <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
            const float f = ml.x == -CUDART_INF_F ? 0.f : ex2f(ml.x - m);
            float l = f * ml.y;
#pragma unroll
            for (int s = 1; s < 32; s <<= 1) l += __shfl_xor_sync(0xffffffffu, l, s);
            float acc[D / 32];
#pragma unroll
            for (int i = 0; i < D / 32; ++i) acc[i] = 0.f;
#pragma unroll 1
            for (int k0 = 0; k0 < 2 * WARPS; k0 += 8) {           // eight slots' loads in flight together
                if (!(pieces >> k0 & 255u)) continue;
                float v[8][D / 32];
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) v[e][i] = pieces >> (k0 + e) & 1 ? piece(k0 + e)[4 + lane * (D / 32) + i] : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float fk = __shfl_sync(0xffffffffu, f, k0 + e);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) acc[i] = fmaf(fk, v[e][i], acc[i]);
                }
            }
            if (begins && ends) {
                const float inv = 1.f / (l + sink_mass(a, pair % a.hkv * HG + h, m));
#pragma unroll
                for (int i = 0; i < D / 32; i += 2) write_out2<D, HG>(a, pair, h * D + lane * (D / 32) + i, acc[i] * inv, acc[i + 1] * inv);
            } else {
                float* to = a.part + ((size_t)blockIdx.x * 2 + begins) * P::PIECE + h * P::HEAD;
                if (lane == 0) *reinterpret_cast<float2*>(to) = make_float2(m, l);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) to[4 + lane * (D / 32) + i] = acc[i];
            }
        }
    }
    if (!a.one && threadIdx.x < 2) a.info[2 * blockIdx.x + threadIdx.x] = threadIdx.x ? reach_back : reach_front;
}

// One block per CTA of the scan: joins the pair that begins in the CTA and reaches over its back end with the front pieces of the
// CTAs behind it.  A warp takes a head and every GROUPS-th piece; what it loads hangs on two loads in a row, the pairs' numbers
// and the pieces (one sequence of 16384 tokens, 19 CTAs a pair: 16.4 us with a chain of four loads and a warp per head, 14.1 so).
constexpr int MERGE_WARPS = 16;
template <int D, int HG>
__global__ void __launch_bounds__(MERGE_WARPS * 32)
novakv_int4_merge_kernel(const DecodeArgs a) {
    using P = Plan<D, HG>;
    constexpr int N = D / 32, GROUPS = MERGE_WARPS / HG, BATCH = 4;
    __shared__ float s_ml[MERGE_WARPS][2], s_acc[MERGE_WARPS][D];
    novakv_grid_dependency_wait();
    const int c0 = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x & 31, h = warp % HG, g = warp / HG, left = gridDim.x - c0;
    const int pair = a.info[2 * c0 + 1], behind = lane > 0 && lane < left ? a.info[2 * (c0 + lane)] : -1;
    if (pair < 0) return;
    // pieces lie side by side: k = 0 is the back piece of this CTA, k > 0 the front piece of CTA c0 + k
    int parts = __popc(__ballot_sync(0xffffffffu, lane == 0 || behind == pair));
    for (int k0 = 32; parts == k0; k0 += 32) parts += __popc(__ballot_sync(0xffffffffu, k0 + lane < left && a.info[2 * (c0 + k0 + lane)] == pair));
    float m = -CUDART_INF_F, l = 0.f, acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.f;
    for (int k0 = g; k0 < parts; k0 += BATCH * GROUPS) {
        float2 ml[BATCH];
        float v[BATCH][N];
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
            const int k = min(k0 + e * GROUPS, parts - 1);
            const float* src = a.part + ((size_t)(c0 + k) * 2 + (k == 0)) * P::PIECE + h * P::HEAD;
            ml[e] = *reinterpret_cast<const float2*>(src);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const float2 x = *reinterpret_cast<const float2*>(src + 4 + lane * N + i);
                v[e][i] = x.x; v[e][i + 1] = x.y;
            }
        }
        float mx = m;
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
            if (k0 + e * GROUPS >= parts) ml[e] = make_float2(-CUDART_INF_F, 0.f);
            mx = fmaxf(mx, ml[e].x);
        }
        const float old = m == -CUDART_INF_F ? 0.f : ex2f(m - mx);
        m = mx;
        l *= old;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] *= old;
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
            const float f = ml[e].x == -CUDART_INF_F ? 0.f : ex2f(ml[e].x - m);
            l = fmaf(f, ml[e].y, l);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = k0 + e * GROUPS < parts ? fmaf(f, v[e][i], acc[i]) : acc[i];
        }
    }
    if (GROUPS > 1) {
        if (lane == 0) { s_ml[warp][0] = m; s_ml[warp][1] = l; }
#pragma unroll
        for (int i = 0; i < N; ++i) s_acc[warp][lane * N + i] = acc[i];
        __syncthreads();
        if (g > 0) return;
        float mx = m;
#pragma unroll
        for (int e = 1; e < GROUPS; ++e) mx = fmaxf(mx, s_ml[e * HG + h][0]);
        const float old = m == -CUDART_INF_F ? 0.f : ex2f(m - mx);
        m = mx;
        l *= old;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] *= old;
#pragma unroll
        for (int e = 1; e < GROUPS; ++e) {
            const float me = s_ml[e * HG + h][0], f = me == -CUDART_INF_F ? 0.f : ex2f(me - m);
            l = fmaf(f, s_ml[e * HG + h][1], l);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = fmaf(f, s_acc[e * HG + h][lane * N + i], acc[i]);
        }
    }
    const float inv = 1.f / (l + sink_mass(a, pair % a.hkv * HG + h, m));
#pragma unroll
    for (int i = 0; i < N; i += 2) write_out2<D, HG>(a, pair, h * D + lane * N + i, acc[i] * inv, acc[i + 1] * inv);
}

// Units of a warp up to which a CTA keeps a pair to itself.  One sequence, 8 pairs, one CTA each / split over all and joined:
// d = 128, 777 tokens (2 units a warp) 9.0 / 10.9 us, 1500 (3) 11.2 / 11.0, 2048 (4) 12.9 / 11.7, 4096 (8) 19.4 / 11.2;
// d = 64, 700 tokens (1) 6.0 / 9.4, 2000 (2) 8.7 / 10.0, 4000 (4) 12.5 / 10.8.  (The host goes by what a sequence can have: the table's width
// and the window.  A short sequence behind a wide table takes the second form.)
constexpr int ONE_UNITS = 3;
int scan_ctas(const novakv_ctx* ctx) { return ctx->scan_ctas > 0 && ctx->scan_ctas < ctx->n_sm ? ctx->scan_ctas : ctx->n_sm; }
size_t info_bytes(const novakv_ctx* ctx) { return ((size_t)ctx->n_sm * 2 * sizeof(int) + 255) & ~(size_t)255; }

template <int D, int HG, bool FINE>
novakv_status launch_t(novakv_ctx* ctx, DecodeArgs& a, void* workspace, cudaStream_t stream) {
    using P = Plan<D, HG>;
    auto* kern = novakv_int4_decode_kernel<D, HG, FINE>;
    const unsigned bit = 1u << (__builtin_ctz(HG) + (D == 128 ? 4 : 0) + (FINE ? 8 : 0));
    if (!(ctx->int4_opt_in & bit)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, P::TOTAL) != cudaSuccess) return NOVAKV_ECUDA;
        ctx->int4_opt_in |= bit;
    }
    a.info = (int*)workspace;
    a.part = (float*)((char*)workspace + info_bytes(ctx));
    // One CTA for each pair, and no second kernel, where every pair has an SM to itself and its warps few units each.
    const long long pairs = (long long)a.batch * a.hkv;
    const int seen = a.window > 0 ? min(a.window / P::TOKENS + 2, a.max_pages_per_seq * (NOVAKV_PAGE_TOKENS / P::TOKENS))
                                  : a.max_pages_per_seq * (NOVAKV_PAGE_TOKENS / P::TOKENS);
    a.one = pairs <= scan_ctas(ctx) && seen <= ONE_UNITS * WARPS;
    a.few = !a.one && a.batch <= 32 && pairs * ((long long)a.max_pages_per_seq * (NOVAKV_PAGE_TOKENS / P::TOKENS) + PAIR_COST) < (1ll << 27);
    const dim3 grid(a.one ? (int)pairs : scan_ctas(ctx));
    if (novakv_launch_pdl(kern, grid, dim3(THREADS), P::TOTAL, stream, a) != cudaSuccess) return NOVAKV_ECUDA;
    ctx->launches++;
    if (a.one) return NOVAKV_OK;
    if (novakv_launch_pdl(novakv_int4_merge_kernel<D, HG>, grid, dim3(MERGE_WARPS * 32), 0, stream, a) != cudaSuccess) return NOVAKV_ECUDA;
    ctx->launches++;
    return NOVAKV_OK;
}
template <int D, int HG>
novakv_status launch(novakv_ctx* ctx, DecodeArgs& a, void* workspace, cudaStream_t stream) {
    return a.out_is_fp32 ? launch_t<D, HG, true>(ctx, a, workspace, stream) : launch_t<D, HG, false>(ctx, a, workspace, stream);
}

}  // namespace

extern "C" size_t novakv_int4_workspace_bytes(const novakv_ctx* ctx, int batch) {
    if (!ctx || batch <= 0) return 0;
    return info_bytes(ctx) + (size_t)ctx->n_sm * 2 * ctx->hg * (ctx->cfg.head_dim + 4) * sizeof(float);
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
    if ((uintptr_t)out & (out_is_fp32 ? 7 : 3)) return NOVAKV_EINVAL;
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
