// Attention of the prompts of a ragged batch (santapp_prompt_attn) on attn_tc.cuh.
//
// A block takes 256 query rows (a KV head's query heads of 256 / group tokens) of one sequence and every key tile that one of them sees:
// 4 d operations per query head and visible pair, far more than the bytes, so tensor cores and exponentials bound
// it: 8192 rows of 28 heads over 4 KV heads, 0.48 TFLOP, take 380 to 450 us inside a graph (1.07 to 1.27 PFLOP/s, 0.64 to 0.76 of the library
// product's burst rate; tensor core busy 59 %, special-function unit 59 %, the card at its power limit when it is repeated). Blocks run from the longest sequence's last rows (which see most keys) down, so that the last ones are short. Where 256 rows a
// block leave SMs idle or the longest block alone (item_rows), a block takes 128, whose two streams share the keys.
// The sequences' tables travel in the kernel's arguments, kPromptSeqs at a launch.
#include <algorithm>
#include <math.h>
#include <string.h>

#include "attn_tc.cuh"
#include "santapp_serve.h"

namespace santapp {

namespace {

constexpr int kPromptSeqs = 96;

struct PromptSeq {
    int key0, n_keys, token0, n_new, both, item0;
};
struct PromptParams {
    const uint16_t *q;
    uint16_t *out;
    int n_q, n_kv, group, n_seqs, item_rows;
    uint32_t by_group;
    TaScore score;
    PromptSeq seq[kPromptSeqs];
};

template <bool kHalf, bool kCap, bool kBias>
__global__ void __launch_bounds__(kTaThreads, 1)
prompt_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ PromptParams p)
{
    step_wait();
    extern __shared__ __align__(1024) unsigned char smem_prompt[];
    TaSmem &sm = *reinterpret_cast<TaSmem *>(smem_prompt);
    int lo = 0, hi = p.n_seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (p.seq[mid].item0 <= (int)blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const PromptSeq sq = p.seq[lo];
    const int local = (int)blockIdx.x - sq.item0, n_rows = sq.n_new * p.group, j = local % p.n_kv;
    TaItem it;
    it.head0 = j * p.group;
    it.group = p.group;
    it.by_group = p.by_group;
    it.n_q = p.n_q;
    it.q = p.q + (int64_t)sq.token0 * p.n_q * kHeadDim;
    it.row0 = ((n_rows + p.item_rows - 1) / p.item_rows - 1 - local / p.n_kv) * p.item_rows;
    it.n_rows = min(p.item_rows, n_rows - it.row0);
    it.plane = j;
    it.key0 = sq.key0;
    it.n_keys = sq.n_keys;
    it.tile0 = 0;
    it.shared = it.n_rows > kTaTile;
    it.fold = 1;
    it.fix_tail = true;
    const auto seen = [&](int row) { return max(sq.n_keys - sq.n_new + ta_token(row, p.by_group) + 1, sq.both); };
    const auto tiles = [&](int rows) { return (seen(it.row0 + rows - 1) + kTaTile - 1) / kTaTile; };
    if (it.shared) {
        it.count0 = tiles(kTaTile);
        it.count1 = tiles(it.n_rows);
    } else {
        const int n = tiles(it.n_rows);
        it.count0 = (n + 1) / 2;
        it.count1 = n / 2;
    }
    ta_block<kHalf, false, kCap, kBias, kTaTile>(
        sm, it, p.score, &k_map, &v_map, nullptr,
        [&](int row, int &vis, int &q_pos) {
            q_pos = sq.n_keys - sq.n_new + ta_token(row, p.by_group);
            vis = seen(row);
        },
        [&](bool ok, int s, bool live, float m, float l) {
            ta_rows<kHalf, false>(
                sm, it, ok, s, live, m, l,
                [&](int r) {
                    const int row = it.row0 + r, token = ta_token(row, p.by_group);
                    return static_cast<void *>(p.out + ((int64_t)(sq.token0 + token) * p.n_q + it.head0 + row - token * p.group) * kHeadDim);
                },
                [](int, float, float) {});
        });
}

// Query rows a block takes: what ends first when blocks are dealt out from the longest down. A tile of keys costs a block of 256 rows a
// step, one of 128 half a step (its streams take tiles in turn), either kOverhead steps to begin and end.
int item_rows(const PromptSeq *seq, int n, int group, int n_kv)
{
    constexpr double kOverhead = 4.0;
    double best = 1e300;
    int rows = 2 * kTaTile;
    for (int size = 2 * kTaTile; size >= kTaTile; size /= 2) {
        const double step = size == kTaTile ? 0.5 : 1.0;
        double total = 0.0, longest = 0.0;
        for (int i = 0; i < n; ++i) {
            const double items = (double)(((int64_t)seq[i].n_new * group + size - 1) / size);
            const double last = std::max((double)seq[i].n_keys, (double)seq[i].both) / kTaTile, first = std::max(last - (double)seq[i].n_new / kTaTile, (double)seq[i].both / kTaTile);
            total += items * n_kv * (step * 0.5 * (first + last + 1.0) + kOverhead);
            longest = std::max(longest, step * (last + 0.5) + kOverhead);
        }
        const double cost = std::max(longest, total / attend_grid_size() + 0.5 * longest);
        if (cost < best) best = cost, rows = size;
    }
    return rows;
}

bool misaligned(const void *p, size_t a) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) % a) != 0; }

using PromptKernel = void (*)(const CUtensorMap, const CUtensorMap, const PromptParams);
template <bool kHalf>
PromptKernel prompt_kernel_of(bool cap, bool bias)
{
    return cap ? (bias ? prompt_kernel<kHalf, true, true> : prompt_kernel<kHalf, true, false>)
               : (bias ? prompt_kernel<kHalf, false, true> : prompt_kernel<kHalf, false, false>);
}

}  // namespace

}  // namespace santapp

using namespace santapp;

extern "C" int santapp_prompt_attn(const santapp_geom *geom, const int32_t *prompt_len_host, const int32_t *new_len_host,
                                   const int32_t *prefix_len_host, const void *q, const void *k_prompt, const void *v_prompt,
                                   const santapp_attn_opts *opts, void *out, santapp_stream stream)
{
    int rc = check_geometry(geom);
    if (rc != SANTAPP_OK) return rc;
    TaScore score;
    if ((rc = ta_score(opts, &score)) != SANTAPP_OK) return rc;
    if (!prompt_len_host || !k_prompt || !v_prompt) return SANTAPP_ERR_INVALID_ARG;
    if (misaligned(q, 16) || misaligned(k_prompt, 16) || misaligned(v_prompt, 16) || misaligned(out, 16)) return SANTAPP_ERR_INVALID_ARG;
    const int B = geom->n_seqs, group = geom->n_q_heads / geom->n_kv_heads;
    int64_t keys = 0, tokens = 0;
    for (int b = 0; b < B; ++b) {
        const int n = prompt_len_host[b], m = new_len_host ? new_len_host[b] : n, both = prefix_len_host ? prefix_len_host[b] : 0;
        if (n < 1 || m < 0 || m > n || both < 0 || both > n) return SANTAPP_ERR_INVALID_ARG;
        keys += n;
        tokens += m;
    }
    if (tokens > 0 && (!q || !out)) return SANTAPP_ERR_INVALID_ARG;
    if (keys >= (int64_t)1 << 30 || tokens * group >= (int64_t)1 << 29) return SANTAPP_ERR_UNSUPPORTED;
    if ((tokens * group / kTaTile + B) * geom->n_kv_heads >= (int64_t)1 << 31) return SANTAPP_ERR_UNSUPPORTED;
    begin_call();
    if (tokens == 0) return SANTAPP_OK;
    CUtensorMap k_map, v_map;
    if (!ta_tensor_map(&k_map, k_prompt, keys, keys, geom->n_kv_heads, geom->elem_type != 0)
        || !ta_tensor_map(&v_map, v_prompt, keys, keys, geom->n_kv_heads, geom->elem_type != 0))
        return note_cuda_failure(cudaErrorInvalidValue, "tensor maps");

    PromptParams p;
    memset(&p, 0, sizeof(p));
    p.q = static_cast<const uint16_t *>(q);
    p.out = static_cast<uint16_t *>(out);
    p.n_q = geom->n_q_heads;
    p.n_kv = geom->n_kv_heads;
    p.group = group;
    p.by_group = ta_by_group(group);
    p.score = score;
    const PromptKernel kernel = geom->elem_type ? prompt_kernel_of<true>(score.cap_log2 > 0.f, score.slopes != nullptr)
                                                : prompt_kernel_of<false>(score.cap_log2 > 0.f, score.slopes != nullptr);
    static std::atomic<unsigned long long> opted[8];
    const int which = (geom->elem_type ? 4 : 0) + (score.cap_log2 > 0.f ? 2 : 0) + (score.slopes != nullptr ? 1 : 0);
    cudaError_t err = ta_prepare(reinterpret_cast<const void *>(kernel), opted[which]);
    if (err != cudaSuccess) return note_cuda_failure(err, "prompt attention set-up");
    int launches = 0, key0 = 0, token0 = 0;
    for (int first = 0; first < B;) {
        int n = 0, b = first;
        for (; b < B && n < kPromptSeqs; ++b) {
            const int m = new_len_host ? new_len_host[b] : prompt_len_host[b];
            if (m > 0) p.seq[n++] = {key0, prompt_len_host[b], token0, m, prefix_len_host ? prefix_len_host[b] : 0, 0};
            key0 += prompt_len_host[b];
            token0 += m;
        }
        first = b;
        if (n == 0) continue;
        std::sort(p.seq, p.seq + n, [](const PromptSeq &x, const PromptSeq &y) { return x.n_keys != y.n_keys ? x.n_keys > y.n_keys : x.key0 < y.key0; });
        int items = 0;
        p.item_rows = item_rows(p.seq, n, group, geom->n_kv_heads);
        for (int i = 0; i < n; ++i) {
            p.seq[i].item0 = items;
            items += (p.seq[i].n_new * group + p.item_rows - 1) / p.item_rows * geom->n_kv_heads;
        }
        p.n_seqs = n;
        err = launch_step(kernel, dim3((unsigned)items), dim3(kTaThreads), kTaSmemBytes, static_cast<cudaStream_t>(stream), k_map, v_map, p);
        if (err != cudaSuccess) return note_cuda_failure(err, "prompt attention launch");
        ++launches;
    }
    note_launch_count(launches);
    return SANTAPP_OK;
}
