// Attention of many query rows over the rows of one KV head, on the fifth-generation tensor cores: the part that
// santapp_prefix_decode_attn (prefix.cu) and santapp_prompt_attn (prompt.cu) share.
//
// The query heads of a KV head are rows of one matrix (row t * G + g: head g of token t), so keys and values are
// fetched once for the whole group. A block works on two accumulators ("streams") of 128 query rows; keys come in
// tiles of 128:
//   S = Q K^T        128 x 128 x 128, both operands in shared memory (128-byte swizzle, as TMA leaves them)
//   P = exp2(S ...)  a thread per row: tcgen05.ld of its 128 scores, running maximum and sum in fp32, weights
//                    written back over the scores as 16-bit values (tensor memory)
//   O += P V         P from tensor memory, V as it lies in memory (N-major)
// While the tensor core does stream 0's O += P V and its next S, the other stream's warps take their exponentials.
// With more than 128 query rows the streams are two row tiles over the same keys (a tile of keys is fetched
// once for both); with fewer they take the key tiles of the same rows in turn and are joined at the end. Rows that fill
// half or a quarter of a tile are in it two or four times (fold), each time with weights for one half or quarter of the keys and
// zeros for the others: a thread has 64 or 32 exponentials to take where the tensor core has idle rows anyway.
//
// Weights: kTwo splits a weight into two 16-bit terms, p = hi + lo (off by at most 2^-16 of it, bf16), two products with V:
// outputs good to fp32. Without, a weight is rounded once (2^-8, bf16), for outputs that are 16 bits wide anyway.
// The running maximum is renewed only when a score passes it by 2^slack: until then weights are at most that, and O need not be scaled, which
// takes a warp 1200 cycles and is due as soon as one of its 32 rows asks for it (with 2^8, in every second tile of rows whose best key stands
// out by e^9). Sums, O and bf16 weights have the range of fp32: 2^24 (values of V to 2^80 stay finite). fp16 weights end at 2^16:
// they carry a factor 2^shift, which cancels in O / l, and slack + shift = 15: 11 + 4, or 8 + 7 for the two terms, whose second
// loses nothing above 2^-31 of the reference. Statistics and sums are fp32.
//
// Every wait is bounded: one that runs out makes all roles of the block stop, waits for its own copies and products, and the
// results are NaN (and bit 2 of the status word).
#pragma once
#include <cuda.h>
#include <math_constants.h>

#include "common.cuh"
#include "santapp_serve.h"
#include "tc.cuh"

namespace santapp {

constexpr int kTaThreads = 384;           // warps 0-3, 4-7: a row per thread of streams 0, 1; warp 8: copies; warp 9: products; warp 10: the
                                          // last tile's values that are somebody else's; warp 11: its keys, where scores are capped
// Registers a thread at launch, at most what kTaThreads leave each (and what the compiler gives them), and after the split: the softmax warps take
// what the other four leave.
constexpr int kTaRegs = 168, kTaRegsSoftmax = 192, kTaRegsOther = 120;
static_assert(8 * kTaRegsSoftmax + 4 * kTaRegsOther <= 12 * kTaRegs, "the split draws on the registers at launch");
constexpr int kTaTile = 128;              // query rows of a stream, keys of a tile
constexpr int kTaTileBytes = kTaTile * kHeadDim * 2;
constexpr int kTaRing = 5;                // tiles of keys or values under way
template <bool kHalf, bool kTwo> constexpr float kTaSlack = !kHalf ? 24.f : (kTwo ? 8.f : 11.f);
template <bool kHalf, bool kTwo> constexpr float kTaShift = !kHalf ? 0.f : (kTwo ? 7.f : 4.f);

struct TaSmem {
    alignas(1024) unsigned char q[2][kTaTileBytes];
    unsigned char ring[kTaRing][kTaTileBytes];
    uint64_t full[4], left[4];                // a group of tiles has landed; the products have left it. By group % 4
    uint64_t q_ready, s_ready[2], p_ready[2][2], done[2];      // p_ready: weights of keys 0-95, 96-127
    uint64_t pos_ready[2][2], tail[2];        // tail: the last tile of keys (0), of values (1) has landed, with somebody else's rows behind it
    alignas(16) float pos[2][2][kTaTile];                 // positions of the keys of a stream's tile, less n_keys; by tile parity
    uint32_t tmem;
    int failed;
};
constexpr int kTaSmemBytes = sizeof(TaSmem);
static_assert(kTaSmemBytes <= 227 * 1024, "shared memory budget");

// row / group and row % group for rows below 2^29 and groups up to 8: by_group is 2^32 / group rounded up to a whole number above it
__host__ __device__ __forceinline__ uint32_t ta_by_group(int group) { return group == 1 ? 0u : (uint32_t)((0x100000000ull) / (uint32_t)group) + 1u; }
__device__ __forceinline__ int ta_token(int row, uint32_t by_group) { return by_group ? (int)__umulhi((uint32_t)row, by_group) : row; }

// What a block works on.
struct TaItem {
    int head0;                // first query head of the KV head
    int group, n_q;
    uint32_t by_group;        // ta_by_group(group)
    const uint16_t *q;        // row r is q + ((r / group) * n_q + head0 + r % group) * 128
    int n_rows;               // query rows from r = row0 on that are real
    int row0;
    int plane;                // KV head: the third coordinate of the planes
    int key0;                 // plane row of key 0
    int n_keys;               // rows behind this belong to somebody else
    int tile0;                // first key tile
    int count0, count1;       // key tiles of each stream
    bool shared;              // the streams are two row tiles over the same keys
    int fold;                 // not shared: the 128 lanes hold the rows 1, 2 or 4 times, each time for another part of a tile's keys
    bool fix_tail;            // the planes hold rows behind n_keys: they are zeroed in V's last tile (0 times NaN is no 0), and with a cap
                              // in K's (how the warp takes its tanh goes by the largest score of the tile, seen or not)
};
struct TaScore {
    float scale_log2;         // scale * log2 e
    float cap_in, cap_log2;   // scale / cap, cap * log2 e
    const float *slopes;
    int32_t *status;
};

__device__ __forceinline__ uint32_t ta_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ int ta_byte(int r, int ch)   // 16-byte piece ch of row r: two blocks of 64 values, pieces XOR-swizzled
{
    return (ch >> 3) * (kTaTile * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
}
__device__ __forceinline__ float ta_ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <bool kHalf>
__device__ __forceinline__ uint32_t ta_pack(float lo, float hi)
{
    uint32_t r;
    if constexpr (kHalf) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else                 asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Products whose descriptors differ in their lower words alone (addresses): between two of them the issuing lane has two additions to
// make. (With 64-bit descriptors and a predicate computed for each, 16 of them took 90 to 99 cycles each beside nothing, 64 this way.)
__device__ __forceinline__ void ta_mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t upper, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}\n" ::"r"(d), "r"(a), "r"(b), "r"(upper), "r"(idesc), "r"(accumulate)
                 : "memory");
}
// A in tensor memory
__device__ __forceinline__ void ta_mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t upper, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 b, {%2, %3};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}\n" ::"r"(d), "r"(a), "r"(b), "r"(upper), "r"(idesc), "r"(accumulate)
                 : "memory");
}
// 32 columns, on their way until ta_ld_wait
__device__ __forceinline__ void ta_ld32(uint32_t taddr, float *v)
{
    uint32_t *u = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
                   "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]),
                   "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]),
                   "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
                 : "r"(taddr));
}
__device__ __forceinline__ void ta_tie(float *v)         // nothing computed from these 32 values moves ahead of this point
{
    uint32_t *u = reinterpret_cast<uint32_t *>(v);
    asm volatile("" : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]), "+r"(u[8]),
                      "+r"(u[9]), "+r"(u[10]), "+r"(u[11]), "+r"(u[12]), "+r"(u[13]), "+r"(u[14]), "+r"(u[15]), "+r"(u[16]), "+r"(u[17]),
                      "+r"(u[18]), "+r"(u[19]), "+r"(u[20]), "+r"(u[21]), "+r"(u[22]), "+r"(u[23]), "+r"(u[24]), "+r"(u[25]), "+r"(u[26]),
                      "+r"(u[27]), "+r"(u[28]), "+r"(u[29]), "+r"(u[30]), "+r"(u[31]));
}
__device__ __forceinline__ void ta_ld16(uint32_t taddr, float (&f)[16])      // 16 columns, there when it returns
{
    uint32_t *u = reinterpret_cast<uint32_t *>(f);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
                   "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void ta_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void ta_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void ta_st16(uint32_t taddr, const uint32_t *v)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 :: "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
                   "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr) : "memory");
}
// 64 values (128 bytes) x 128 rows of plane `z` from row y on
__device__ __forceinline__ void ta_copy(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void ta_named_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// A wait returns false once any of the block's waits has run out.
__device__ __forceinline__ bool ta_wait(TaSmem &sm, uint64_t *bar, uint32_t parity)
{
    const uint32_t b = ta_addr(bar);
    for (int i = 0; i < (1 << 20); ++i) {
        uint32_t over;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}\n"
                     : "=r"(over) : "r"(b), "r"(parity) : "memory");
        if (over) return true;
        if (*reinterpret_cast<volatile int *>(&sm.failed)) return false;
    }
    *reinterpret_cast<volatile int *>(&sm.failed) = 1;
    return false;
}
// The same for a whole warp, whose lanes agree on the answer.
__device__ __forceinline__ bool ta_wait_warp(TaSmem &sm, uint64_t *bar, uint32_t parity)
{
    return __all_sync(0xFFFFFFFFu, ta_wait(sm, bar, parity));
}
// One arrival for the warp, behind everything its lanes did.
__device__ __forceinline__ void ta_arrive_warp(uint64_t *bar)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(ta_addr(bar));
}
__device__ __forceinline__ bool ta_elect()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// ---- pairs of fp32 values in one instruction ----
__device__ __forceinline__ uint64_t ta_two(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void ta_split(uint64_t x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ uint64_t ta_fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t ta_add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t ta_mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
template <int kStream> struct TaStream { static constexpr int value = kStream; };
// The ring is filled in the order of first use, and in groups that land and are left together (a wait and a commit each, which cost the
// issuing lane a hundred or two hundred cycles apiece): where both streams use a tile, K_0 | V_0 K_1 | V_1 K_2 | ..., where they take
// tiles in turn, K_0 K_1 | V_0 K_2 | V_1 K_3 | ... Slot: place % kTaRing.
__device__ __forceinline__ int ta_tiles(const TaItem &it) { return it.shared ? it.count1 : it.count0 + it.count1; }
__device__ __forceinline__ int ta_key_place(const TaItem &it, int tile) { return it.shared ? 2 * tile : max(2 * tile - 1, 0); }
__device__ __forceinline__ int ta_value_place(const TaItem &it, int tile)
{
    return it.shared ? 2 * tile + 1 : min(2 * tile + 2, 2 * ta_tiles(it) - 1);
}
// (of a place that is not the last)
__device__ __forceinline__ int ta_group(const TaItem &it, int place) { return it.shared ? (place + 1) / 2 : place / 2; }
__device__ __forceinline__ bool ta_cut(const TaItem &it) { return it.fix_tail && it.n_keys < (it.tile0 + ta_tiles(it)) * kTaTile; }

// cap * tanh(x cap_in) * log2 e of a thread's products: tanh(y) = y P(y^2) with the P of kN coefficients that has the smallest largest relative
// error on [0, 1/2] (kWide: [0, 1]), cap * log2 e folded into them: 5e-7 of 4 coefficients, 1e-8 of 5 (kWide 6e-7 of 6, 5e-8 of 7). On
// [0, 1/2] the powers of cap_in are folded into them too, which leaves the squares of the products themselves: one multiplication less.
template <int kN>
__device__ __forceinline__ constexpr float ta_tanh_term(int k)
{
    constexpr float kP[4][7] = {{0.9999994557709386f, -0.33326317935941724f, 0.13190296603213952f, -0.04440222612781058f},
                                {0.9999999868718333f, -0.33333069394022213f, 0.1332477931761862f, -0.05298607529180707f, 0.0171350066346453f},
                                {0.9999994135992578f, -0.3332904237853047f, 0.13281433880736535f, -0.05160567400212715f, 0.016743115063748693f,
                                 -0.0030670603265534825f},
                                {0.9999999502407364f, -0.3333283915307065f, 0.1332520407582405f, -0.0534570295681808f, 0.02028998042301148f,
                                 -0.006203379104680566f, 0.0010410226337084262f}};
    return kP[kN - 4][k];
}
// cap_log2 * tanh(y) of one value: the polynomial up to 1, beyond it from e = exp(-2 |y|) as (1 - e) / (1 + e), which would cancel for small y (its error
// is 2^-22 of the cap, whatever the score: a cap of 1e6 left scores of 1 nothing).
template <int kN>
__device__ __forceinline__ float ta_cap_one(float y, float cap_log2)
{
    const float u = y * y, e = ta_ex2(-2.885390082f * fabsf(y));
    float r = ta_tanh_term<kN>(kN - 1);
#pragma unroll
    for (int k = kN - 2; k >= 0; --k) r = fmaf(r, u, ta_tanh_term<kN>(k));
    return (fabsf(y) <= 1.f ? r * y : copysignf(__fdividef(1.f - e, 1.f + e), y)) * cap_log2;
}
template <bool kWide, int kN, int kCols>
__device__ __forceinline__ void ta_cap_poly(const TaScore &sc, float (&v)[kCols])
{
    static_assert(kWide ? kN == 6 || kN == 7 : kN == 4 || kN == 5, "a row of the table");
    uint64_t c[kN];
    float by = kWide ? sc.cap_log2 : sc.cap_log2 * sc.cap_in;
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        c[k] = ta_two(ta_tanh_term<kN>(k) * by, ta_tanh_term<kN>(k) * by);
        if (!kWide) by *= sc.cap_in * sc.cap_in;
    }
    const uint64_t in = ta_two(sc.cap_in, sc.cap_in);
#pragma unroll
    for (int i = 0; i < kCols; i += 8) {                    // four pairs side by side: one alone waits for each of its products
        uint64_t y[4], u[4], r[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            y[x] = ta_two(v[i + 2 * x], v[i + 2 * x + 1]);
            if (kWide) y[x] = ta_mul2(y[x], in);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) u[x] = ta_mul2(y[x], y[x]);
#pragma unroll
        for (int x = 0; x < 4; ++x) r[x] = ta_fma2(c[kN - 1], u[x], c[kN - 2]);
#pragma unroll
        for (int k = kN - 3; k >= 0; --k)
#pragma unroll
            for (int x = 0; x < 4; ++x) r[x] = ta_fma2(r[x], u[x], c[k]);
#pragma unroll
        for (int x = 0; x < 4; ++x) ta_split(ta_mul2(r[x], y[x]), v[i + 2 * x], v[i + 2 * x + 1]);
    }
}
// The same where scores reach beyond the cap: the polynomial (of kN coefficients) up to |y| = 1/2, and from there on (1 - e) / (1 + e) with
// e = exp(-2 |y|), two uses of the special-function unit, good to 2^-21 there. (Below, it cancels: 2^-22 of the cap would be left of small
// scores that stand beside large ones.)
template <int kN>
__device__ __forceinline__ void ta_cap_far(const TaScore &sc, float (&v)[16])
{
    static_assert(kN == 4 || kN == 5, "a row of the table");
    const uint64_t in = ta_two(sc.cap_in, sc.cap_in);
    uint64_t c[kN];
#pragma unroll
    for (int k = 0; k < kN; ++k) c[k] = ta_two(ta_tanh_term<kN>(k) * sc.cap_log2, ta_tanh_term<kN>(k) * sc.cap_log2);
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const uint64_t y = ta_mul2(ta_two(v[i], v[i + 1]), in), u = ta_mul2(y, y);
        uint64_t r = c[kN - 1];
#pragma unroll
        for (int k = kN - 2; k >= 0; --k) r = ta_fma2(r, u, c[k]);
        float near[2], at[2];
        ta_split(ta_mul2(r, y), near[0], near[1]);
        ta_split(y, at[0], at[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float e = ta_ex2(-2.885390082f * fabsf(at[h])), far = copysignf(__fdividef(1.f - e, 1.f + e), at[h]) * sc.cap_log2;
            v[i + h] = fabsf(at[h]) <= 0.5f ? near[h] : far;
        }
    }
}
// By a polynomial where the warp's |x cap_in| are at most 1, the usual case. Otherwise 16 of the thread's columns (from t_v on in tensor memory) at a time,
// there and back, which keeps that path's code short: unrolled over all of them it cost the others 3 to 10 %, 32 at a time one of them 2 %.
template <bool kTwo, int kCols>
__device__ __forceinline__ void ta_cap(const TaScore &sc, uint32_t t_v, float (&v)[kCols])
{
    float most[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kCols; i += 8)
#pragma unroll
        for (int x = 0; x < 4; ++x) most[x] = fmaxf(fmaxf(most[x], fabsf(v[i + x])), fabsf(v[i + 4 + x]));
    const float far = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * sc.cap_in;
    // (cap_in within 2^-12 and 2^12: its eighth power is a normal number)
    if (sc.cap_in >= 0x1p-12f && sc.cap_in <= 0x1p12f && __all_sync(0xFFFFFFFFu, far <= 0.5f)) {
        ta_cap_poly<false, kTwo ? 5 : 4>(sc, v);
    } else if (__all_sync(0xFFFFFFFFu, far <= 1.f)) {
        ta_cap_poly<true, kTwo ? 7 : 6>(sc, v);
    } else {
#pragma unroll 1
        for (int q = 0; q < kCols / 16; ++q) {
            float w[16];
            ta_ld16(t_v + 16 * q, w);
            ta_cap_far<kTwo ? 5 : 4>(sc, w);
            ta_st16(t_v + 16 * q, reinterpret_cast<const uint32_t *>(w));
        }
        ta_st_wait();
#pragma unroll
        for (int q = 0; q < kCols / 32; ++q) ta_ld32(t_v + 32 * q, v + 32 * q);
        ta_ld_wait();
#pragma unroll
        for (int q = 0; q < kCols / 32; ++q) ta_tie(v + 32 * q);
    }
}

// One stream's rows: thread t of 128 owns row t. `vis`: keys [0, vis) are seen by the row; q_pos its position; key_pos
// the positions of the plane's keys (null: their index). Leaves the statistics (maximum in log2 units, sum).
//
// What a tile takes between its scores and its weights decides the pace (the products of the other stream are shorter), so the first quarter of the
// exponentials is taken against the maximum of the tiles before, beside the search for this tile's; where a score passes it by
// more than the slack, and in the first tile, that quarter is taken again. The last quarter of the weights is handed over on its own: only
// its product remains to be done when the last weight is there.
template <bool kHalf, bool kTwo, bool kCap, bool kBias, int kCols>
__device__ __forceinline__ bool ta_softmax(TaSmem &sm, const TaItem &it, const TaScore &sc, int s, bool live, int vis, int q_pos,
                                           float slope_log2, const int32_t *key_pos, float &m, float &l)
{
    constexpr float kShift = kTaShift<kHalf, kTwo>;
    constexpr bool kRaw = !kCap && !kBias;                  // scores stay in units of the product, not yet scaled
    const int t = threadIdx.x & 127;
    const uint32_t lanes = (uint32_t)((threadIdx.x >> 5) & 3) << 21;
    const uint32_t t_s = sm.tmem + lanes + 128u * s, t_o = sm.tmem + lanes + 256u + 128u * s;
    const int col0 = t / kCols * kCols;      // first of the keys of a tile that this thread weighs
    const bool warp_live = __any_sync(0xFFFFFFFFu, live);
    m = -CUDART_INF_F;
    l = 0.f;
    const int count = s ? it.count1 : it.count0;
    if (kBias && key_pos == nullptr) {
        sm.pos[s][0][t] = (float)t;
        ta_named_barrier(2 + s, 128);
    }
    for (int c = 0; c < count; ++c) {
        const int tile = (it.tile0 + (it.shared ? c : 2 * c + s)) * kTaTile, kb = tile + col0;
        if (kBias && key_pos != nullptr) {
            // (relative to n_keys, so that near keys of a very long prompt keep whole distances in fp32; who writes here has
            // seen all 128 threads at the tile before this one, that is behind the reading of the tile before that)
            sm.pos[s][c & 1][t] = tile + t < it.n_keys ? (float)(key_pos[tile + t] - it.n_keys) : 0.f;
            mbar_arrive(ta_addr(&sm.pos_ready[s][c & 1]));
            if (!ta_wait_warp(sm, &sm.pos_ready[s][c & 1], (uint32_t)(c >> 1) & 1u)) return false;
        }
        if (!ta_wait_warp(sm, &sm.s_ready[s], c & 1)) return false;
        if (warp_live) {
            tc_fence_after();
            float v[kCols];
#pragma unroll
            for (int q = 0; q < kCols / 32; ++q) ta_ld32(t_s + col0 + 32 * q, v + 32 * q);
            ta_ld_wait();
#pragma unroll
            for (int q = 0; q < kCols / 32; ++q) ta_tie(v + 32 * q);
            if constexpr (kCap) ta_cap<kTwo>(sc, t_s + col0, v);
            if constexpr (kBias) {
                // linear in the key's position as long as no key is behind the query
                const bool table = key_pos != nullptr;
                const float *pos = sm.pos[s][table ? c & 1 : 0] + (table ? col0 : 0);
                const uint64_t slope2 = ta_two(slope_log2, slope_log2), mul2 = kCap ? ta_two(1.f, 1.f) : ta_two(sc.scale_log2, sc.scale_log2);
                const float d = (float)(table ? q_pos - it.n_keys : q_pos - kb);
                if (table || !__any_sync(0xFFFFFFFFu, live && min(vis, kb + kCols) - 1 > q_pos)) {
                    const uint64_t base = ta_two(-slope_log2 * d, -slope_log2 * d);
#pragma unroll
                    for (int i = 0; i < kCols; i += 4) {
                        const ulonglong2 p = *reinterpret_cast<const ulonglong2 *>(pos + i);
                        ta_split(ta_fma2(slope2, p.x, ta_fma2(ta_two(v[i], v[i + 1]), mul2, base)), v[i], v[i + 1]);
                        ta_split(ta_fma2(slope2, p.y, ta_fma2(ta_two(v[i + 2], v[i + 3]), mul2, base)), v[i + 2], v[i + 3]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < kCols; ++i) v[i] = fmaf(-slope_log2, fabsf(d - (float)i), kCap ? v[i] : v[i] * sc.scale_log2);
                }
            }
            const int seen = vis - kb;
            if (__any_sync(0xFFFFFFFFu, seen < kCols)) {
#pragma unroll
                for (int i = 0; i < kCols; ++i) v[i] = i < seen ? v[i] : -CUDART_INF_F;
            }
            const float mul = kRaw ? sc.scale_log2 : 1.f;
            const uint64_t mul2 = ta_two(mul, mul);
            uint64_t sum[2];
            uint32_t hi[16], lo[16];
            const auto weights = [&](int q, uint64_t shift2) {          // of keys 32 q .. 32 q + 31
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint64_t two = ta_two(v[32 * q + 2 * i], v[32 * q + 2 * i + 1]), x = kRaw ? ta_fma2(two, mul2, shift2) : ta_add2(two, shift2);
                    float p0, p1;
                    ta_split(x, p0, p1);
                    p0 = ta_ex2(p0);
                    p1 = ta_ex2(p1);
                    const uint64_t pp = ta_two(p0, p1);
                    sum[i & 1] = ta_add2(sum[i & 1], pp);
                    hi[i] = ta_pack<kHalf>(p0, p1);
                    if constexpr (kTwo) {
                        float d0, d1;
                        ta_split(ta_fma2(ta_two(elem_lo<kHalf>(hi[i]), elem_hi<kHalf>(hi[i])), ta_two(-1.f, -1.f), pp), d0, d1);
                        lo[i] = ta_pack<kHalf>(d0, d1);
                    }
                }
            };
            const auto store = [&](int q) {
                ta_st16(t_s + col0 / 2 + 16 * q, hi);
                if constexpr (kTwo) ta_st16(t_s + 64 + col0 / 2 + 16 * q, lo);
            };
            float shift = kShift - (m == -CUDART_INF_F ? 0.f : m);
            sum[0] = sum[1] = 0;
            weights(0, ta_two(shift, shift));
            float top[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
            for (int i = 4; i < kCols; i += 8)
#pragma unroll
                for (int x = 0; x < 4; ++x) top[x] = i + 4 + x < kCols ? fmaxf(fmaxf(top[x], v[i + x]), v[i + 4 + x]) : fmaxf(top[x], v[i + x]);
            const float m_new = fmaxf(m, mul * fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
            if (__any_sync(0xFFFFFFFFu, m_new > m + (c == 0 ? 0.f : kTaSlack<kHalf, kTwo>))) {
                if (c > 0) {
                    const float f = m_new == -CUDART_INF_F ? 1.f : ta_ex2(m - m_new);
                    float o[16];
#pragma unroll 1
                    for (int q = 0; q < 8; ++q) {
                        ta_ld16(t_o + 16 * q, o);
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] *= f;
                        ta_st16(t_o + 16 * q, reinterpret_cast<const uint32_t *>(o));
                    }
                    l *= f;
                }
                m = m_new;
                shift = kShift - (m == -CUDART_INF_F ? 0.f : m);
                sum[0] = sum[1] = 0;
                weights(0, ta_two(shift, shift));
            }
            const uint64_t shift2 = ta_two(shift, shift);
            store(0);
            if constexpr (kCols == kTaTile) {
                weights(1, shift2);
                store(1);
                weights(2, shift2);
                store(2);
                ta_st_wait();
                tc_fence_before();
                ta_arrive_warp(&sm.p_ready[s][0]);
                weights(3, shift2);
                store(3);
            } else {
                if constexpr (kCols == 64) {
                    weights(1, shift2);
                    store(1);
                }
                // nothing for the keys that other lanes of this row weigh
#pragma unroll
                for (int i = 0; i < 16; ++i) hi[i] = 0u;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (32 * q < col0 || 32 * q >= col0 + kCols) {
                        ta_st16(t_s + 16 * q, hi);
                        if constexpr (kTwo) ta_st16(t_s + 64 + 16 * q, hi);
                    }
            }
            float s0, s1;
            ta_split(ta_add2(sum[0], sum[1]), s0, s1);
            l += s0 + s1;
            ta_st_wait();
            tc_fence_before();
            if constexpr (kCols != kTaTile) ta_arrive_warp(&sm.p_ready[s][0]);
            ta_arrive_warp(&sm.p_ready[s][1]);
        } else {
            ta_arrive_warp(&sm.p_ready[s][0]);
            ta_arrive_warp(&sm.p_ready[s][1]);
        }
    }
    m -= kShift;                                           // the factor of the weights is the sum's too
    if (count > 0) {
        if (!ta_wait_warp(sm, &sm.done[s], 0)) return false;
        tc_fence_after();
    }
    return true;
}

// The block: set-up, copies, products. `rows(row, vis, q_pos)` tells how many keys a row sees and its position; `finish(ok, s, live, m, l)`
// gets the statistics of the thread's row and takes O out of tensor memory (ta_rows). kCols: keys of a tile that a thread weighs, 128 / fold.
template <bool kHalf, bool kTwo, bool kCap, bool kBias, int kCols, typename Rows, typename Finish>
__device__ __forceinline__ void ta_block(TaSmem &sm, const TaItem &it, const TaScore &sc, const CUtensorMap *k_map, const CUtensorMap *v_map,
                                         const int32_t *key_pos, Rows rows, Finish finish)
{
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (warp < 8) {                                         // the queries, on their way while the rest is set up
        const int tiles = it.shared ? 2 : 1;
#pragma unroll 8
        for (int e = tid; e < tiles * kTaTile * 16; e += 256) {
            const int r = e >> 4, ch = e & 15, lr = it.shared ? r : r % (kTaTile / it.fold), row = it.row0 + min(lr, it.n_rows - 1);
            const int token = ta_token(row, it.by_group);
            const uint16_t *src = it.q + ((int64_t)token * it.n_q + it.head0 + row - token * it.group) * kHeadDim + 8 * ch;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ta_addr(sm.q[r >> 7] + ta_byte(r & 127, ch))), "l"(src),
                         "r"(lr < it.n_rows ? 16 : 0) : "memory");
        }
    } else if (tid == 256) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(k_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(v_map) : "memory");
    }
    if (tid == 288) {
        sm.failed = 0;
        for (int i = 0; i < 4; ++i) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(ta_addr(&sm.full[i])), "r"(2));
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(ta_addr(&sm.left[i])), "r"(1));
        }
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(ta_addr(&sm.q_ready)), "r"(256));
        for (int i = 0; i < 2; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(ta_addr(&sm.tail[i])), "r"(1));
        for (int s = 0; s < 2; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(ta_addr(&sm.s_ready[s])), "r"(1));
            for (int i = 0; i < 2; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(ta_addr(&sm.p_ready[s][i])), "r"(4));
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(ta_addr(&sm.done[s])), "r"(1));
            for (int i = 0; i < 2; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(ta_addr(&sm.pos_ready[s][i])), "r"(128));
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 10) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(ta_addr(&sm.tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTaRegsSoftmax));
        // ---- a row of scores per thread ----
        asm volatile("cp.async.wait_all;" ::: "memory");
        proxy_fence();
        mbar_arrive(ta_addr(&sm.q_ready));
        const int s = warp >> 2, r = it.shared ? (tid & 127) + kTaTile * s : (tid & 127) % (kTaTile / it.fold);
        bool live = r < it.n_rows;
        int vis = it.n_keys;
        int q_pos = 0;
        float slope = 0.f, m, l;
        if (live) rows(it.row0 + r, vis, q_pos);
        if (kBias && live) slope = 1.4426950409f * sc.slopes[it.head0 + (it.row0 + r) % it.group];
        const bool ok = ta_softmax<kHalf, kTwo, kCap, kBias, kCols>(sm, it, sc, s, live, vis, q_pos, slope, key_pos, m, l);
        finish(ok, s, live, m, l);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTaRegsOther));
        if (warp == 8) {
            // ---- copies ----
            if (ta_elect()) {
                int n = 0, waited = -1;                    // tiles asked for; the last group known to be left
                const int n_tiles = ta_tiles(it);
                const bool cut = ta_cut(it);
                const auto ask = [&](bool value, int tile, int group) {
                    if (n >= kTaRing) {
                        const int g = ta_group(it, n - kTaRing);
                        if (g > waited && !ta_wait(sm, &sm.left[g & 3], (uint32_t)(g >> 2) & 1u)) return false;
                        waited = g;
                    }
                    // (warps 10 and 11 hand on tiles that end in somebody else's rows)
                    const bool fixed = cut && tile == n_tiles - 1 && (value || kCap);
                    const uint32_t bar = ta_addr(fixed ? &sm.tail[value] : &sm.full[group & 3]), dst = ta_addr(sm.ring[n % kTaRing]);
                    const int y = it.key0 + (it.tile0 + tile) * kTaTile;
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(kTaTileBytes) : "memory");
                    const CUtensorMap *map = value ? v_map : k_map;
                    ta_copy(dst, map, 0, y, it.plane, bar);
                    ta_copy(dst + kTaTileBytes / 2, map, 64, y, it.plane, bar);
                    ++n;
                    return true;
                };
                const auto alone = [&](int group) { mbar_arrive(ta_addr(&sm.full[group & 3])); };      // a group of one tile
                const int ahead = it.shared ? 1 : 2;       // keys are so many tiles ahead of the values
                int groups = 0;
                bool ok = ask(false, 0, 0);
                if (ok && ahead == 2 && n_tiles > 1) ok = ask(false, 1, 0);
                else alone(0);
                for (int i = 0; ok && i < n_tiles; ++i) {
                    groups = i + 1;
                    ok = ask(true, i, groups);
                    if (ok && i + ahead < n_tiles) ok = ask(false, i + ahead, groups);
                    else if (ok) alone(groups);
                }
                // nothing leaves while a copy is under way (in the normal course the products have waited for all of them)
                if (!ok)
                    for (int g = max(0, groups - 3); g <= groups; ++g) tc_wait(ta_addr(&sm.full[g & 3]), (uint32_t)(g >> 2) & 1u);
            }
            __syncwarp();
        } else if (warp == 9) {
            // ---- products: one lane. Strictly in turn, stream 0's weights with its values and its next scores, then stream 1's: when both
            // streams' weights are there at once, one still gets its scores a thousand cycles before the other, and its exponentials
            // are taken while the other's products run (a warp per stream left both waiting for one another's halves: 515 us for 442) ----
            const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, sm.tmem, 0);
            if (ta_elect()) {
                const uint32_t idesc_s = tc_idesc(kTaTile, kTaTile, 0, 0, kHalf), idesc_o = tc_idesc(kTaTile, kHeadDim, 0, 1, kHalf);
                // (lower words: address / 16, leading offset)
                const uint32_t q_low = (uint32_t)tc_desc_sw128(ta_addr(sm.q[0]), 16, 1024), k_low = (uint32_t)tc_desc_sw128(ta_addr(sm.ring[0]), 16, 1024);
                const uint32_t v_low = (uint32_t)tc_desc_sw128(ta_addr(sm.ring[0]), kTaTileBytes / 2, 1024), upper = (uint32_t)(tc_desc_sw128(0, 16, 1024) >> 32);
                const uint32_t q1_low = q_low + (it.shared ? kTaTileBytes >> 4 : 0);
                const int n_tiles = ta_tiles(it);
                const auto landed = [&](int g) { return ta_wait(sm, &sm.full[g & 3], (uint32_t)(g >> 2) & 1u); };
                const auto scores = [&](auto stream, int tile) {
                    constexpr int s = decltype(stream)::value;
                    const uint32_t a = s ? q1_low : q_low, b = k_low + (uint32_t)(ta_key_place(it, tile) % kTaRing * (kTaTileBytes >> 4));
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        const uint32_t at = ((x >> 2) * (kTaTileBytes / 2) + (x & 3) * 32) >> 4;
                        ta_mma_ss(tmem + 128u * s, a + at, b + at, upper, idesc_s, x > 0 ? 1u : 0u);
                    }
                    tc_commit(ta_addr(&sm.s_ready[s]));
                };
                // the stream's c-th tile of weights
                const auto values = [&](auto stream, int c, int tile) {
                    constexpr int s = decltype(stream)::value;
                    const uint32_t b = v_low + (uint32_t)(ta_value_place(it, tile) % kTaRing * (kTaTileBytes >> 4));
#pragma unroll
                    for (int part = 0; part < 2; ++part) {                  // keys 0 .. 95, 96 .. 127
                        if (!ta_wait(sm, &sm.p_ready[s][part], c & 1)) return false;
                        tc_fence_after();
#pragma unroll
                        for (int x = 6 * part; x < (part ? 8 : 6); ++x)
#pragma unroll
                            for (int term = 0; term < (kTwo ? 2 : 1); ++term)
                                ta_mma_ts(tmem + 256u + 128u * s, tmem + 128u * s + 64u * term + 8u * x, b + ((x * 2048) >> 4), upper, idesc_o,
                                          x > 0 || term > 0 ? 1u : (c > 0 ? 1u : 0u));
                    }
                    if (c + 1 == (s ? it.count1 : it.count0)) tc_commit(ta_addr(&sm.done[s]));
                    return true;
                };
                bool ok = ta_wait(sm, &sm.q_ready, 0) && landed(0);
                if (ok) {
                    tc_fence_after();
                    scores(TaStream<0>{}, 0);
                    if (it.count1 > 0) scores(TaStream<1>{}, it.shared ? 0 : 1);
                    tc_commit(ta_addr(&sm.left[0]));
                }
                const int rounds = it.shared ? n_tiles : it.count0;
                for (int c = 0; ok && c < rounds; ++c) {
                    const int t0 = it.shared ? c : 2 * c, t1 = it.shared ? c : 2 * c + 1, step = it.shared ? 1 : 2;
                    if (!(ok = landed(t0 + 1))) break;
                    if (c < it.count0) {
                        if (!(ok = values(TaStream<0>{}, c, t0))) break;
                        if (c + 1 < it.count0) scores(TaStream<0>{}, t0 + step);
                    }
                    if (!it.shared) {
                        tc_commit(ta_addr(&sm.left[(t0 + 1) & 3]));
                        if (c < it.count1 && !(ok = landed(t1 + 1))) break;
                    }
                    if (c < it.count1) {
                        if (!(ok = values(TaStream<1>{}, c, t1))) break;
                        if (c + 1 < it.count1) scores(TaStream<1>{}, t1 + step);
                        tc_commit(ta_addr(&sm.left[(t1 + 1) & 3]));
                    }
                }
                ok = ok && ta_wait(sm, &sm.left[n_tiles & 3], (uint32_t)(n_tiles >> 2) & 1u);      // (its own last arrival)
                if (!ok) {                                 // products under way finish before their memory goes
                    for (int i = 0; i < 4096; ++i) __nanosleep(256);
                    if (sc.status != nullptr) atomicOr(sc.status, 4);
                }
            }
            __syncwarp();
        } else if (ta_cut(it) && (warp == 10 || kCap)) {
            // ---- the rows behind the last one, in the last tile of values (warp 10) and of keys ----
            const bool value = warp == 10;
            const int last = ta_tiles(it) - 1, valid = it.n_keys - (it.tile0 + last) * kTaTile;
            const int place = value ? 2 * last + 1 : ta_key_place(it, last), group = value ? last + 1 : ta_group(it, place);
            if (ta_wait_warp(sm, &sm.tail[value], 0)) {
                for (int e = max(valid, 0) * 16 + lane; e < kTaTile * 16; e += 32)
                    *reinterpret_cast<uint4 *>(sm.ring[place % kTaRing] + ta_byte(e >> 4, e & 15)) = make_uint4(0, 0, 0, 0);
                proxy_fence();
                ta_arrive_warp(&sm.full[group & 3]);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 10) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sm.tmem), "r"(512));
}

__device__ __forceinline__ void *ta_shfl(void *p, int lane)
{
    const unsigned long long v = reinterpret_cast<unsigned long long>(p);
    const uint32_t a = __shfl_sync(0xFFFFFFFFu, (uint32_t)v, lane), b = __shfl_sync(0xFFFFFFFFu, (uint32_t)(v >> 32), lane);
    return reinterpret_cast<void *>((unsigned long long)b << 32 | a);
}

// O of the rows, out of tensor memory and through shared memory, so that a row leaves in pieces of 256 bytes: fp32 as it is (kOut32) or
// 16-bit values of O / l. row_at(r) says where row r of the item goes, stats(r, m, l) takes its statistics. All 256 softmax threads
// come here, whatever their waits said; where one ran out l is NaN, and with it the row.
// Two row tiles: a warp's 32 rows pass through the warp's own quarter of its stream's queries, which are done with.
// One: parts of a row (of the two streams, and of its copies in the tile) are joined; each thread scales its own, and they are added
// up where the key and value tiles were.
constexpr int kTaPitch = kHeadDim + 4;
static_assert(2 * kTaTile * kTaPitch * 4 <= kTaRing * kTaTileBytes, "O of both streams fits the ring");
template <bool kHalf, bool kOut32, typename RowAt, typename Stats>
__device__ __forceinline__ void ta_rows(TaSmem &sm, const TaItem &it, bool ok, int s, bool live, float m, float l, RowAt row_at, Stats stats)
{
    const int t = threadIdx.x & 127, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t t_o = sm.tmem + ((uint32_t)(warp & 3) << 21) + 256u + 128u * s;
    const bool warp_live = __any_sync(0xFFFFFFFFu, live);
    if (!ok) m = 0.f, l = CUDART_NAN_F;
    float o[32];
    if (it.shared) {
        if (!warp_live) return;
        const int r0 = kTaTile * s + 32 * (warp & 3), mine = r0 + lane;
        if (live) stats(mine, m, l);
        const float by = kOut32 ? (ok ? 1.f : l) : (l == 0.f ? 0.f : __fdividef(1.f, l));
        void *dst = row_at(min(mine, it.n_rows - 1));
        unsigned char *stage = sm.q[s] + 8192 * (warp & 3);
        constexpr int kCols = kOut32 ? 64 : 128;           // columns in 256 bytes
#pragma unroll
        for (int pass = 0; pass < kHeadDim / kCols; ++pass) {
#pragma unroll
            for (int q = 0; q < kCols / 32; ++q) {
                ta_ld32(t_o + kCols * pass + 32 * q, o);
                ta_ld_wait();
                ta_tie(o);
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] *= by;
#pragma unroll
                for (int i = 0; i < (kOut32 ? 8 : 4); ++i) {
                    const int ch = q * (kOut32 ? 8 : 4) + i;
                    uint4 x;
                    if constexpr (kOut32)
                        x = make_uint4(__float_as_uint(o[4 * i]), __float_as_uint(o[4 * i + 1]), __float_as_uint(o[4 * i + 2]), __float_as_uint(o[4 * i + 3]));
                    else
                        x = make_uint4(ta_pack<kHalf>(o[8 * i], o[8 * i + 1]), ta_pack<kHalf>(o[8 * i + 2], o[8 * i + 3]),
                                       ta_pack<kHalf>(o[8 * i + 4], o[8 * i + 5]), ta_pack<kHalf>(o[8 * i + 6], o[8 * i + 7]));
                    *reinterpret_cast<uint4 *>(stage + lane * 256 + ((ch ^ (lane & 7)) << 4)) = x;
                }
            }
            __syncwarp();
#pragma unroll 8
            for (int i = 0; i < 16; ++i) {
                const int r = 2 * i + (lane >> 4), ch = lane & 15;
                uint4 *to = reinterpret_cast<uint4 *>(ta_shfl(dst, r)) + 16 * pass + ch;
                if (r0 + r < it.n_rows) *to = *reinterpret_cast<const uint4 *>(stage + r * 256 + ((ch ^ (r & 7)) << 4));
            }
            __syncwarp();
        }
        return;
    }
    float *rows = reinterpret_cast<float *>(sm.ring[0]);
    float2 *stat = reinterpret_cast<float2 *>(sm.q[1]);    // (no queries there)
    const int copy = kTaTile / it.fold, r = t % copy;
    stat[kTaTile * s + t] = make_float2(m, l);
    ta_named_barrier(1, 256);                              // both streams' products are over
    float top = -CUDART_INF_F, sum = 0.f;
    for (int e = r; e < 2 * kTaTile; e += copy) top = fmaxf(top, stat[e].x);
    const float ref = top == -CUDART_INF_F ? 0.f : top;
    for (int e = r; e < 2 * kTaTile; e += copy) sum = fmaf(stat[e].y, ta_ex2(stat[e].x - ref), sum);
    if (live && s == 0 && t < copy) stats(r, top, sum);
    {
        float by = ta_ex2(m - ref);
        if (sum != sum) by = sum;
        else if constexpr (!kOut32) by = sum == 0.f ? 0.f : __fdividef(by, sum);
        float *dst = rows + (kTaTile * s + t) * kTaPitch;
        if ((s ? it.count1 : it.count0) > 0 && warp_live) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                ta_ld32(t_o + 32 * q, o);
                ta_ld_wait();
                ta_tie(o);
#pragma unroll
                for (int i = 0; i < 32; i += 4)
                    *reinterpret_cast<float4 *>(dst + 32 * q + i) = make_float4(o[i] * by, o[i + 1] * by, o[i + 2] * by, o[i + 3] * by);
            }
        }
    }
    ta_named_barrier(1, 256);
    const int streams = it.count1 > 0 ? 2 : 1;             // (a stream without a tile has left nothing)
    void *dst = row_at(min(8 * (lane & 15) + warp, it.n_rows - 1));
#pragma unroll 4
    for (int i = 0; i < kTaTile / 8; ++i) {
        const int row = 8 * i + warp;
        void *to = ta_shfl(dst, i);
        if (row >= it.n_rows) break;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int e = row; e < streams * kTaTile; e += copy) {
            const float4 y = reinterpret_cast<const float4 *>(rows + e * kTaPitch)[lane];
            x.x += y.x;
            x.y += y.y;
            x.z += y.z;
            x.w += y.w;
        }
        if constexpr (kOut32) reinterpret_cast<float4 *>(to)[lane] = x;
        else                  reinterpret_cast<uint2 *>(to)[lane] = make_uint2(ta_pack<kHalf>(x.x, x.y), ta_pack<kHalf>(x.z, x.w));
    }
}

// Planes [n_planes][rows][128] of 16-bit values, plane_rows rows apart, as a tensor map with boxes of 64 values x 128 rows;
// rows behind `rows` read as zeros. Returns false where the driver refuses.
bool ta_tensor_map(CUtensorMap *map, const void *base, int64_t rows, int64_t plane_rows, int n_planes, bool half);
int ta_score(const santapp_attn_opts *opts, TaScore *score);     // a santapp_status
// What a kernel on this file needs once per device. One that was built with fewer registers than its split asks for would wait for them for
// ever: it is not launched.
inline cudaError_t ta_prepare(const void *kernel, std::atomic<unsigned long long> &done)
{
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    if (dev >= 64 || !(done.load(std::memory_order_acquire) >> dev & 1)) {
        cudaFuncAttributes a;
        if ((err = cudaFuncGetAttributes(&a, kernel)) != cudaSuccess) return err;
        if (a.numRegs < kTaRegs) return cudaErrorInvalidKernelImage;
    }
    return ensure_dynamic_smem(kernel, kTaSmemBytes, done);
}

}  // namespace santapp
