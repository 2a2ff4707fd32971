// Decode attention of a batch that shares one long prompt (santapp_prefix_decode_attn).
//
// prefix_kernel   the shared prompt, on attn_tc.cuh: the query heads of a KV head of ALL sequences are the rows of one matrix, so
//                 the prompt's rows are read once for the batch. The key tiles are cut into parts; a block takes up to 256
//                 rows over one part and leaves a partial (maximum, sum, O) per row.
// finish_kernel   one cluster per (sequence, KV head): exact attention over the sequence's own suffix (mma.sync: a pair has at
//                 most eight query rows), and the log-sum-exp merge with the pair's partials.
//
// Up to 128 rows (18 sequences of 7 heads) the prompt's bytes bound the first kernel, 512 per row and KV head: 5 sequences of 32 heads over
// 131071 rows, 541 MB, take 93 us in it (5.8 TB/s, 0.90 of the copy rate). Beyond, its products and weights: 4 d per row and key, half again
// for the weights' second term (the outputs are fp32); 64 sequences of 28 heads over 32768 rows with a cap, 68 us, the tensor core busy 43 %.
// The merge: 3 us for a pair's suffix and 2 for its partials, another 2 where a cluster shares it (two cluster barriers).
#include <algorithm>
#include <math.h>
#include <string.h>

#include "attn_tc.cuh"
#include "santapp_serve.h"

namespace santapp {

namespace {

constexpr int kFinishWarps = 4;
constexpr int kFinishThreads = kFinishWarps * 32;
constexpr int kFinishStages = 3;          // blocks of 16 suffix rows a warp has under way
constexpr int kFinishBlock = 16;
constexpr int kFinishStageBytes = 2 * kFinishBlock * kHeadDim * 2;
constexpr int kEntryFloats = 132;         // O of a head, maximum, sum
constexpr int kMaxCluster = 8;

struct PrefixParams {
    const uint16_t *q;
    int n_q, n_kv, group, n_seqs, rows;   // rows: n_seqs * group, of each KV head
    int n_keys, n_tiles, parts, row_items;
    int64_t plane_rows;
    const int32_t *key_pos;               // nullable
    const int32_t *suffix_len;            // nullable
    int suffix_cap;
    const uint16_t *k_suffix, *v_suffix;
    TaScore score;
    float *part_o;                        // [n_kv][parts][rows][128]
    float2 *part_ml;                      // [n_kv][parts][rows] maximum (log2 units), sum
    float *out;
};

__device__ __forceinline__ int suffix_rows(const PrefixParams &p, int b)
{
    return p.suffix_len != nullptr ? min(max(p.suffix_len[b], 0), p.suffix_cap) : 0;
}

template <bool kHalf, bool kCap, bool kBias, int kFold>
__global__ void __launch_bounds__(kTaThreads, 1)
prefix_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ PrefixParams p)
{
    step_wait();
    // (finish_kernel's blocks may come as this one's leave: they begin with the suffixes, which nothing here writes)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    extern __shared__ __align__(1024) unsigned char smem_prefix[];
    TaSmem &sm = *reinterpret_cast<TaSmem *>(smem_prefix);
    const int part = blockIdx.x, j = blockIdx.y % p.n_kv, pair = blockIdx.y / p.n_kv;
    const int t0 = (int)((int64_t)p.n_tiles * part / p.parts), t1 = (int)((int64_t)p.n_tiles * (part + 1) / p.parts);
    TaItem it;
    it.head0 = j * p.group;
    it.group = p.group;
    it.by_group = ta_by_group(p.group);
    it.n_q = p.n_q;
    it.q = p.q;
    it.row0 = pair * 2 * kTaTile;
    it.n_rows = min(2 * kTaTile, p.rows - it.row0);
    it.plane = j;
    it.key0 = 0;
    it.n_keys = p.n_keys;
    it.tile0 = t0;
    it.shared = kFold == 1 && it.n_rows > kTaTile;
    it.fold = kFold;
    it.fix_tail = false;                                    // (the tensor map ends at the last row)
    it.count0 = it.shared ? t1 - t0 : (t1 - t0 + 1) / 2;
    it.count1 = it.shared ? t1 - t0 : (t1 - t0) / 2;
    const int32_t *key_pos = kBias && p.key_pos != nullptr ? p.key_pos + (int64_t)j * p.plane_rows : nullptr;
    ta_block<kHalf, true, kCap, kBias, kTaTile / kFold>(
        sm, it, p.score, &k_map, &v_map, key_pos,
        [&](int row, int &, int &q_pos) {
            if (kBias) q_pos = p.n_keys + suffix_rows(p, row / p.group) - 1;
        },
        [&](bool ok, int s, bool live, float m, float l) {
            const int64_t slot = ((int64_t)j * p.parts + part) * p.rows + it.row0;
            ta_rows<kHalf, true>(
                sm, it, ok, s, live, m, l, [&](int r) { return static_cast<void *>(p.part_o + (slot + r) * kHeadDim); },
                [&](int r, float top, float sum) { p.part_ml[slot + r] = make_float2(top, sum); });
        });
}

// ---- the suffix and the merge ----
__device__ __forceinline__ void fin_copy16(uint32_t dst, const void *src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void fin_ldmatrix(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void fin_ldmatrix_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
template <bool kHalf>
__device__ __forceinline__ void fin_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (kHalf)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t fin_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t fin_size()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void fin_cluster_sync()
{
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ float fin_remote(const float *local, uint32_t rank)
{
    uint32_t a;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(ta_addr(local)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

using Entry = float[kMaxGroup][kEntryFloats];
struct FinishSmem {
    unsigned char ring[kFinishWarps][kFinishStages][kFinishStageBytes];
    Entry block;                                                 // the block's
    // sums over warp w's suffix rows (e = w) and its partials (kFinishWarps + w), where its rows were
    __device__ __forceinline__ Entry &entry(int e) { return reinterpret_cast<Entry *>(ring[e % kFinishWarps])[e / kFinishWarps]; }
};
static_assert(2 * sizeof(Entry) <= kFinishStages * kFinishStageBytes, "the entries of a warp fit its ring");

template <bool kHalf, bool kCap, bool kBias>
__global__ void __launch_bounds__(kFinishThreads)
finish_kernel(const __grid_constant__ PrefixParams p)
{
    // The prefix kernel asks for this one once it has begun itself, behind everything before it on the stream: what it does not write is
    // there. Without a prefix kernel this is the call's first.
    if (p.parts == 0) step_wait();
    extern __shared__ __align__(1024) unsigned char smem_finish[];
    FinishSmem &sm = *reinterpret_cast<FinishSmem *>(smem_finish);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)fin_rank(), n_blocks = (int)fin_size();
    const int pair = blockIdx.y, b = pair / p.n_kv, j = pair % p.n_kv, G = p.group;
    const int share = rank * kFinishWarps + warp, shares = n_blocks * kFinishWarps;
    const int len = suffix_rows(p, b), n_blk = (len + kFinishBlock - 1) / kFinishBlock;
    constexpr float kShift = kHalf ? 15.f : 0.f;             // fp16 weights: 2^15 of the running maximum's, see attend.cu

    // ---- suffix: blocks share, share + shares, ... of 16 rows ----
    const uint32_t ring = ta_addr(sm.ring[warp][0]);
    const int64_t plane = ((int64_t)b * p.n_kv + j) * p.suffix_cap;
    const auto fetch = [&](int blk, int stage) {
        if (blk < n_blk) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = 2 * i + (lane >> 4), ch = lane & 15, row = blk * kFinishBlock + r;
                const int64_t at = (plane + min(row, len - 1)) * 16 + ch;
                const uint32_t dst = ring + stage * kFinishStageBytes + r * 256 + ((ch ^ (r & 7)) << 4);
                fin_copy16(dst, reinterpret_cast<const uint4 *>(p.k_suffix) + at, row < len);
                fin_copy16(dst + kFinishStageBytes / 2, reinterpret_cast<const uint4 *>(p.v_suffix) + at, row < len);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < kFinishStages - 1; ++s) fetch(share + s * shares, s);

    const int g = lane >> 2, kc = (lane & 3) * 2;             // this lane's head, first of its columns
    uint32_t qa[8][2];
    {
        const uint16_t *q = p.q + ((int64_t)b * p.n_q + j * G + min(g, G - 1)) * kHeadDim;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            qa[x][0] = g < G ? *reinterpret_cast<const uint32_t *>(q + 16 * x + kc) : 0u;
            qa[x][1] = g < G ? *reinterpret_cast<const uint32_t *>(q + 16 * x + kc + 8) : 0u;
        }
    }
    float slope = 0.f;
    if (kBias && g < G) slope = 1.4426950409f * p.score.slopes[j * G + g];
    float m = -CUDART_INF_F, l = 0.f, o[16][4];
#pragma unroll
    for (int x = 0; x < 16; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[x][i] = 0.f;
    int stage = 0;
    for (int blk = share; blk < n_blk; blk += shares) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kFinishStages - 2) : "memory");
        __syncwarp();
        fetch(blk + (kFinishStages - 1) * shares, (stage + kFinishStages - 1) % kFinishStages);
        const uint32_t kb = ring + stage * kFinishStageBytes, vb = kb + kFinishStageBytes / 2;
        stage = (stage + 1) % kFinishStages;
        float c0[4] = {0.f, 0.f, 0.f, 0.f}, c1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            uint32_t k4[4];
            const int r = (lane & 7) + ((lane >> 4) & 1) * 8, ch = 2 * x + ((lane >> 3) & 1);
            fin_ldmatrix(k4, kb + r * 256 + ((ch ^ (r & 7)) << 4));
            fin_mma<kHalf>(c0, qa[x][0], 0u, qa[x][1], 0u, k4[0], k4[1]);
            fin_mma<kHalf>(c1, qa[x][0], 0u, qa[x][1], 0u, k4[2], k4[3]);
        }
        float v[4] = {c0[0], c0[1], c1[0], c1[1]};           // keys kc, kc + 1, kc + 8, kc + 9 of head g
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = blk * kFinishBlock + kc + (i & 1) + (i >> 1) * 8;
            if constexpr (kCap) {
                v[i] = ta_cap_one<7>(v[i] * p.score.cap_in, p.score.cap_log2);
            } else {
                v[i] *= p.score.scale_log2;
            }
            if constexpr (kBias) v[i] = fmaf(-slope, (float)(len - 1 - key), v[i]);
            if (key >= len) v[i] = -CUDART_INF_F;
        }
        float mx = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 2));
        const float m_new = fmaxf(m, mx), ref = m_new == -CUDART_INF_F ? 0.f : m_new;
        const float f = ta_ex2(m - ref);
        m = m_new;
        l *= f;
        float pw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            pw[i] = ta_ex2(v[i] - ref + kShift);
            l += pw[i];
        }
        const uint32_t h0 = ta_pack<kHalf>(pw[0], pw[1]), h1 = ta_pack<kHalf>(pw[2], pw[3]);
        const uint32_t l0 = ta_pack<kHalf>(pw[0] - elem_lo<kHalf>(h0), pw[1] - elem_hi<kHalf>(h0));
        const uint32_t l1 = ta_pack<kHalf>(pw[2] - elem_lo<kHalf>(h1), pw[3] - elem_hi<kHalf>(h1));
#pragma unroll
        for (int x = 0; x < 16; x += 2) {
            uint32_t v4[4];
            const int r = (lane & 7) + ((lane >> 3) & 1) * 8, ch = x + (lane >> 4);
            fin_ldmatrix_trans(v4, vb + r * 256 + ((ch ^ (r & 7)) << 4));
#pragma unroll
            for (int i = 0; i < 4; ++i) { o[x][i] *= f; o[x + 1][i] *= f; }
            // the weights' second terms are rows 8 .. 15 of the same product
            fin_mma<kHalf>(o[x], h0, l0, h1, l1, v4[0], v4[1]);
            fin_mma<kHalf>(o[x + 1], h0, l0, h1, l1, v4[2], v4[3]);
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();                                            // every lane has read the last rows
    l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
    l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
    {
        float *e = sm.entry(warp)[g];
#pragma unroll
        for (int x = 0; x < 16; ++x) *reinterpret_cast<float2 *>(e + 8 * x + kc) = make_float2(o[x][0] + o[x][2], o[x][1] + o[x][3]);
        if ((lane & 3) == 0) *reinterpret_cast<float2 *>(e + kHeadDim) = make_float2(m == -CUDART_INF_F ? m : m - kShift, l);
    }

    // ---- partials share, share + shares, ... of the pair's rows, the next one's on its way ----
    if (p.parts > 0) step_wait();
    {
        const int64_t first = (int64_t)j * p.parts * p.rows + (int64_t)b * G;
        float top[kMaxGroup], sum[kMaxGroup];
        float4 acc[kMaxGroup], x[kMaxGroup];
        float2 ml = make_float2(-CUDART_INF_F, 0.f);
        const auto fetch_part = [&](int i) {
            if (i >= p.parts) return;
            const int64_t slot = first + (int64_t)i * p.rows;
            ml = p.part_ml[slot + min(lane, G - 1)];
#pragma unroll
            for (int h = 0; h < kMaxGroup; ++h)
                if (h < G) x[h] = reinterpret_cast<const float4 *>(p.part_o + (slot + h) * kHeadDim)[lane];
        };
#pragma unroll
        for (int h = 0; h < kMaxGroup; ++h) {
            top[h] = -CUDART_INF_F;
            sum[h] = 0.f;
            acc[h] = x[h] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        fetch_part(share);
        for (int i = share; i < p.parts; i += shares) {
            const float2 ml_now = ml;
            float4 now[kMaxGroup];
#pragma unroll
            for (int h = 0; h < kMaxGroup; ++h) now[h] = x[h];
            fetch_part(i + shares);
#pragma unroll
            for (int h = 0; h < kMaxGroup; ++h) {
                const float mm = __shfl_sync(0xFFFFFFFFu, ml_now.x, h), ll = __shfl_sync(0xFFFFFFFFu, ml_now.y, h);
                // (a part whose scores are all no numbers has no maximum either, but its sum is none: it is taken, and the factors
                // exp2(-inf - -inf), or 0 times it, leave no number)
                if (h >= G || (mm == -CUDART_INF_F && ll == 0.f)) continue;
                const float t = fmaxf(top[h], mm), a = ta_ex2(top[h] - t), w = ta_ex2(mm - t);
                top[h] = t;
                sum[h] = fmaf(w, ll, sum[h] * a);
                acc[h].x = fmaf(w, now[h].x, acc[h].x * a);
                acc[h].y = fmaf(w, now[h].y, acc[h].y * a);
                acc[h].z = fmaf(w, now[h].z, acc[h].z * a);
                acc[h].w = fmaf(w, now[h].w, acc[h].w * a);
            }
        }
#pragma unroll
        for (int h = 0; h < kMaxGroup; ++h) {
            if (h >= G) continue;
            float *e = sm.entry(kFinishWarps + warp)[h];
            reinterpret_cast<float4 *>(e)[lane] = acc[h];
            if (lane == 0) *reinterpret_cast<float2 *>(e + kHeadDim) = make_float2(top[h], sum[h]);
        }
    }
    __syncthreads();

    // ---- the block's, then the cluster's ----
    for (int h = warp; h < G; h += kFinishWarps) {
        float top = -CUDART_INF_F, sum = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int e = 0; e < 2 * kFinishWarps; ++e) top = fmaxf(top, sm.entry(e)[h][kHeadDim]);
        const float ref = top == -CUDART_INF_F ? 0.f : top;
#pragma unroll
        for (int e = 0; e < 2 * kFinishWarps; ++e) {
            const float w = ta_ex2(sm.entry(e)[h][kHeadDim] - ref);
            const float4 x = reinterpret_cast<const float4 *>(sm.entry(e)[h])[lane];
            sum = fmaf(w, sm.entry(e)[h][kHeadDim + 1], sum);
            acc.x = fmaf(w, x.x, acc.x);
            acc.y = fmaf(w, x.y, acc.y);
            acc.z = fmaf(w, x.z, acc.z);
            acc.w = fmaf(w, x.w, acc.w);
        }
        if (n_blocks == 1) {
            const float by = sum == 0.f ? 0.f : 1.f / sum;
            reinterpret_cast<float4 *>(p.out + ((int64_t)b * p.n_q + j * G + h) * kHeadDim)[lane] =
                make_float4(acc.x * by, acc.y * by, acc.z * by, acc.w * by);
        } else {
            reinterpret_cast<float4 *>(sm.block[h])[lane] = acc;
            if (lane == 0) *reinterpret_cast<float2 *>(sm.block[h] + kHeadDim) = make_float2(top, sum);
        }
    }
    if (n_blocks == 1) return;
    fin_cluster_sync();
    for (int h = rank; h < G; h += n_blocks) {              // a thread per value
        float tops[kMaxCluster], top = -CUDART_INF_F, sum = 0.f, acc = 0.f;
#pragma unroll
        for (int c = 0; c < kMaxCluster; ++c) {
            tops[c] = c < n_blocks ? fin_remote(&sm.block[h][kHeadDim], c) : -CUDART_INF_F;
            top = fmaxf(top, tops[c]);
        }
        const float ref = top == -CUDART_INF_F ? 0.f : top;
#pragma unroll
        for (int c = 0; c < kMaxCluster; ++c) {
            if (c >= n_blocks) continue;
            const float w = ta_ex2(tops[c] - ref);
            sum = fmaf(w, fin_remote(&sm.block[h][kHeadDim + 1], c), sum);
            acc = fmaf(w, fin_remote(&sm.block[h][tid], c), acc);
        }
        p.out[((int64_t)b * p.n_q + j * G + h) * kHeadDim + tid] = sum == 0.f ? 0.f : acc / sum;
    }
    fin_cluster_sync();                                     // nobody leaves while its memory is read
}

// How the prompt is cut: parts of its key tiles such that the blocks fill the SMs. A block costs its tiles (two units
// each where its two streams are row tiles, one where they take tiles in turn) and about four units to fill and drain.
struct PrefixPlan {
    int row_items, parts, n_tiles;
    size_t part_o, part_ml, total;
};
size_t up256(size_t x) { return (x + 255) / 256 * 256; }
PrefixPlan prefix_plan(const santapp_geom *g, int64_t n_keys)
{
    PrefixPlan L;
    const int64_t rows = (int64_t)g->n_seqs * (g->n_q_heads / g->n_kv_heads);
    const int sms = attend_grid_size();
    L.row_items = (int)((rows + 2 * kTaTile - 1) / (2 * kTaTile));
    L.n_tiles = (int)((n_keys + kTaTile - 1) / kTaTile);
    const int64_t items = (int64_t)L.row_items * g->n_kv_heads;
    const int unit = rows > kTaTile ? 2 : 1;
    L.parts = L.n_tiles ? 1 : 0;
    double best = 1e300;
    for (int c = 1; c <= L.n_tiles && c <= 2 * sms; ++c) {
        const int64_t waves = (items * c + sms - 1) / sms;
        const double cost = (double)waves * ((double)((L.n_tiles + c - 1) / c) * unit + 4.0) + 0.02 * c;
        if (cost < best) best = cost, L.parts = c;
    }
    L.part_o = 0;
    L.part_ml = up256(sizeof(float) * (size_t)g->n_kv_heads * L.parts * (size_t)rows * kHeadDim);
    L.total = std::max<size_t>(256, L.part_ml + up256(sizeof(float2) * (size_t)g->n_kv_heads * L.parts * (size_t)rows));
    return L;
}

bool misaligned(const void *p, size_t a) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) % a) != 0; }

int check_prefix(const santapp_geom *geom, int64_t n_keys, int suffix_cap)
{
    const int rc = check_geometry(geom);
    if (rc != SANTAPP_OK) return rc;
    if (n_keys < 0 || suffix_cap < 0) return SANTAPP_ERR_INVALID_ARG;
    if (n_keys >= (int64_t)1 << 30) return SANTAPP_ERR_UNSUPPORTED;
    if ((int64_t)geom->n_seqs * geom->n_kv_heads > 65535) return SANTAPP_ERR_UNSUPPORTED;       // a grid dimension
    if ((int64_t)geom->n_seqs * geom->n_kv_heads * (int64_t)suffix_cap >= (int64_t)1 << 31) return SANTAPP_ERR_UNSUPPORTED;
    return SANTAPP_OK;
}

using PrefixKernel = void (*)(const CUtensorMap, const CUtensorMap, const PrefixParams);
using FinishKernel = void (*)(const PrefixParams);
template <bool kHalf, bool kCap, bool kBias>
void kernels_of(int fold, PrefixKernel *a, FinishKernel *b)
{
    *a = fold == 4 ? prefix_kernel<kHalf, kCap, kBias, 4> : (fold == 2 ? prefix_kernel<kHalf, kCap, kBias, 2> : prefix_kernel<kHalf, kCap, kBias, 1>);
    *b = finish_kernel<kHalf, kCap, kBias>;
}
template <bool kHalf>
void kernels_of(bool cap, bool bias, int fold, PrefixKernel *a, FinishKernel *b)
{
    if (cap && bias) kernels_of<kHalf, true, true>(fold, a, b);
    else if (cap)    kernels_of<kHalf, true, false>(fold, a, b);
    else if (bias)   kernels_of<kHalf, false, true>(fold, a, b);
    else             kernels_of<kHalf, false, false>(fold, a, b);
}

}  // namespace

// ---- what prompt.cu uses too ----
bool ta_tensor_map(CUtensorMap *map, const void *base, int64_t rows, int64_t plane_rows, int n_planes, bool half)
{
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<void *> entry{nullptr};
    void *fn = entry.load(std::memory_order_acquire);
    if (fn == nullptr) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess
            || found != cudaDriverEntryPointSuccess || fn == nullptr)
            return false;
        entry.store(fn, std::memory_order_release);
    }
    const cuuint64_t dims[3] = {kHeadDim, (cuuint64_t)rows, (cuuint64_t)n_planes};
    const cuuint64_t strides[2] = {kHeadDim * 2, (cuuint64_t)plane_rows * kHeadDim * 2};
    const cuuint32_t box[3] = {64, kTaTile, 1}, step[3] = {1, 1, 1};
    return reinterpret_cast<Encode>(fn)(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims,
                                        strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int ta_score(const santapp_attn_opts *opts, TaScore *score)
{
    const float given = opts ? opts->scale : 0.f, cap = opts ? opts->cap : 0.f;
    if (!(given >= 0.f) || isinf(given) || !(cap >= 0.f) || isinf(cap)) return SANTAPP_ERR_INVALID_ARG;
    if (opts && (misaligned(opts->slopes, 4) || misaligned(opts->status, 4))) return SANTAPP_ERR_INVALID_ARG;
    const double scale = given == 0.f ? 1.0 / sqrt((double)kHeadDim) : (double)given, log2e = 1.4426950408889634;
    score->scale_log2 = (float)(scale * log2e);
    score->cap_in = cap > 0.f ? (float)(scale / cap) : 0.f;
    score->cap_log2 = (float)(cap * log2e);
    // (0 times an infinite factor would be no number, and a subnormal quotient has lost its lower bits)
    if (isinf(score->scale_log2) || isinf(score->cap_log2) || (cap > 0.f && !isnormal(score->cap_in))) return SANTAPP_ERR_INVALID_ARG;
    score->slopes = opts ? opts->slopes : nullptr;
    score->status = opts ? opts->status : nullptr;
    return SANTAPP_OK;
}

}  // namespace santapp

using namespace santapp;

extern "C" {

size_t santapp_prefix_decode_workspace_bytes(const santapp_geom *geom, int64_t prefix_len, int32_t suffix_cap)
{
    if (check_prefix(geom, prefix_len, suffix_cap) != SANTAPP_OK) return 0;
    return prefix_plan(geom, prefix_len).total;
}

int santapp_prefix_decode_attn(const santapp_geom *geom, const void *k_prefix, const void *v_prefix, int64_t prefix_len,
                               int64_t plane_rows, const int32_t *prefix_token, const void *q, const void *k_suffix,
                               const void *v_suffix, const int32_t *suffix_len_dev, int32_t suffix_cap,
                               const santapp_attn_opts *opts, float *out, void *workspace, size_t workspace_bytes,
                               santapp_stream stream)
{
    int rc = check_prefix(geom, prefix_len, suffix_cap);
    if (rc != SANTAPP_OK) return rc;
    PrefixParams p;
    memset(&p, 0, sizeof(p));
    if ((rc = ta_score(opts, &p.score)) != SANTAPP_OK) return rc;
    if (!q || !out || !workspace || (prefix_len > 0 && (!k_prefix || !v_prefix))) return SANTAPP_ERR_INVALID_ARG;
    if (prefix_len > 0 && plane_rows < prefix_len) return SANTAPP_ERR_INVALID_ARG;
    if (plane_rows >= (int64_t)1 << 31) return SANTAPP_ERR_UNSUPPORTED;
    if (misaligned(q, 16) || misaligned(out, 16) || misaligned(workspace, 16) || misaligned(k_prefix, 16) || misaligned(v_prefix, 16)
        || misaligned(k_suffix, 16) || misaligned(v_suffix, 16) || misaligned(suffix_len_dev, 4) || misaligned(prefix_token, 4))
        return SANTAPP_ERR_INVALID_ARG;
    if (suffix_cap > 0 && suffix_len_dev && (!k_suffix || !v_suffix)) return SANTAPP_ERR_INVALID_ARG;
    const PrefixPlan L = prefix_plan(geom, prefix_len);
    if (workspace_bytes < L.total) return SANTAPP_ERR_WORKSPACE_TOO_SMALL;
    begin_call();
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    p.q = static_cast<const uint16_t *>(q);
    p.n_q = geom->n_q_heads;
    p.n_kv = geom->n_kv_heads;
    p.group = p.n_q / p.n_kv;
    p.n_seqs = geom->n_seqs;
    p.rows = p.n_seqs * p.group;
    p.n_keys = (int)prefix_len;
    p.n_tiles = L.n_tiles;
    p.parts = L.parts;
    p.row_items = L.row_items;
    p.plane_rows = plane_rows;
    p.key_pos = p.score.slopes ? prefix_token : nullptr;
    p.suffix_len = suffix_cap > 0 ? suffix_len_dev : nullptr;
    p.suffix_cap = suffix_cap;
    p.k_suffix = static_cast<const uint16_t *>(k_suffix);
    p.v_suffix = static_cast<const uint16_t *>(v_suffix);
    p.part_o = reinterpret_cast<float *>(static_cast<char *>(workspace) + L.part_o);
    p.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + L.part_ml);
    p.out = out;

    const bool cap = p.score.cap_log2 > 0.f, bias = p.score.slopes != nullptr, half = geom->elem_type != 0;
    PrefixKernel prefix;
    FinishKernel finish;
    const int fold = p.rows <= kTaTile / 4 ? 4 : (p.rows <= kTaTile / 2 ? 2 : 1);
    if (half) kernels_of<true>(cap, bias, fold, &prefix, &finish);
    else      kernels_of<false>(cap, bias, fold, &prefix, &finish);
    static std::atomic<unsigned long long> opted[4][8];
    const int which = (half ? 4 : 0) + (cap ? 2 : 0) + (bias ? 1 : 0);
    cudaError_t err = ta_prepare(reinterpret_cast<const void *>(prefix), opted[fold == 4 ? 2 : fold - 1][which]);
    if (err == cudaSuccess) err = ensure_dynamic_smem(reinterpret_cast<const void *>(finish), (int)sizeof(FinishSmem), opted[3][which]);
    if (err != cudaSuccess) return note_cuda_failure(err, "prefix attention set-up");
    int launches = 0;
    if (L.parts > 0) {
        CUtensorMap k_map, v_map;
        if (!ta_tensor_map(&k_map, k_prefix, prefix_len, plane_rows, p.n_kv, half) || !ta_tensor_map(&v_map, v_prefix, prefix_len, plane_rows, p.n_kv, half))
            return note_cuda_failure(cudaErrorInvalidValue, "tensor maps");
        err = launch_step(prefix, dim3((unsigned)L.parts, (unsigned)(L.row_items * p.n_kv)), dim3(kTaThreads), kTaSmemBytes, s, k_map, v_map, p);
        if (err != cudaSuccess) return note_cuda_failure(err, "prefix attention launch");
        ++launches;
    }
    // blocks of a cluster: no more than there is work for, and all clusters about one block an SM (of eight pairs' worth more, some
    // clusters find no room beside the others and come second: 12.5 us in place of 8)
    const int pairs = p.n_seqs * p.n_kv, work = std::max((suffix_cap + kFinishBlock - 1) / kFinishBlock, L.parts);
    int blocks = 1;
    while (blocks < kMaxCluster && 2 * blocks * pairs <= attend_grid_size() * 9 / 8 && blocks * kFinishWarps < work) blocks *= 2;
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = (unsigned)blocks;
    attrs[1].val.clusterDim.y = 1;
    attrs[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks, (unsigned)pairs);
    cfg.blockDim = dim3(kFinishThreads);
    cfg.dynamicSmemBytes = sizeof(FinishSmem);
    cfg.stream = s;
    cfg.attrs = attrs;
    cfg.numAttrs = 2;
    err = cudaLaunchKernelEx(&cfg, finish, p);
    if (err != cudaSuccess) return note_cuda_failure(err, "prefix merge launch");
    note_launch_count(launches + 1);
    return SANTAPP_OK;
}

}  // extern "C"
