// Suffixes of a batch whose answers fork, move or end (santapp_suffix_fork).
//
// Row r of KV head j of slot b becomes that of slot src[b], for r below src[b]'s length, in place. Slots may form chains
// and cycles (a permutation of the batch), so no order of whole-slot copies is safe. A block takes the same rows
// of one head of ALL slots: it reads every row that moves into shared memory, and writes when it has them all; no other
// block touches these rows, so one launch does it without a second buffer.
//
// Bound by memory: each moved row is read and written once. Rows of slots that stay are not touched: the block's threads go through a list of
// the slots that move. 16 of 32 slots of up to 1024 rows (26.5 MB, 4.1 us at the copy rate) take 7.4 us.
#include "common.cuh"
#include "santapp_serve.h"

namespace santapp {

namespace {

constexpr int kForkThreads = 256;
// Bytes of rows a block stages at most, while one row of every slot is no more: a block waits for memory twice (its table, its rows), so
// what hides that is blocks beside it, six of this size an SM (that case, when these were compared: 7.7 us; 16, 24 and 64 KB 9.1, 9.0 and 8.2)
constexpr int kForkStage = 32 * 1024;
constexpr int kForkMaxSeqs = 4096;

struct ForkParams {
    int n_seqs, n_kv, cap;
    int row_bits;                         // a block takes 2^row_bits rows of every slot
    int piece_bits;                       // 2^piece_bits 16-byte pieces of them (4: whole rows)
    const int32_t *src, *len;
    uint4 *k, *v;
    int32_t *len_out;
};

__global__ void __launch_bounds__(kForkThreads)
fork_kernel(ForkParams p)
{
    step_wait();
    extern __shared__ __align__(16) unsigned char smem_fork[];
    __shared__ int n_moved;
    const int tid = threadIdx.x, B = p.n_seqs, bits = p.row_bits + p.piece_bits, rows = 1 << p.row_bits;
    uint4 *stage = reinterpret_cast<uint4 *>(smem_fork);                              // [moved slot][row][piece]
    int2 *tab = reinterpret_cast<int2 *>(stage + ((size_t)B << bits));                 // slot and its source, rows of this block that move
    const int r0 = (blockIdx.x >> (4 - p.piece_bits)) << p.row_bits, c0 = (blockIdx.x & ((16 >> p.piece_bits) - 1)) << p.piece_bits;
    const int j = blockIdx.y;
    uint4 *buf = blockIdx.z ? p.v : p.k;
    const bool writes_len = p.len_out != nullptr && blockIdx.x == 0 && j == 0 && blockIdx.z == 0;
    if (tid == 0) n_moved = 0;
    __syncthreads();
    for (int b = tid; b < B; b += kForkThreads) {
        const int a = p.src[b];
        const int n = a >= 0 && a < B ? min(max(p.len[a], 0), p.cap) : 0;
        const int move = a != b ? min(n - r0, rows) : 0;
        if (move > 0) tab[atomicAdd(&n_moved, 1)] = make_int2(b << 16 | a, move);
        if (writes_len) p.len_out[b] = n;
    }
    __syncthreads();
    const int total = n_moved << bits;
    const auto at = [&](int b, int e) {
        return (((int64_t)b * p.n_kv + j) * p.cap + r0 + (e >> p.piece_bits)) * 16 + c0 + (e & ((1 << p.piece_bits) - 1));
    };
#pragma unroll 4
    for (int i = tid; i < total; i += kForkThreads) {
        const int2 t = tab[i >> bits];
        const int e = i & ((1 << bits) - 1);
        if ((e >> p.piece_bits) < t.y)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(stage + i)), "l"(buf + at(t.x & 0xFFFF, e)) : "memory");
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
#pragma unroll 4
    for (int i = tid; i < total; i += kForkThreads) {
        const int2 t = tab[i >> bits];
        const int e = i & ((1 << bits) - 1);
        if ((e >> p.piece_bits) < t.y) buf[at(t.x >> 16, e)] = stage[i];
    }
}

}  // namespace

}  // namespace santapp

using namespace santapp;

extern "C" int santapp_suffix_fork(const santapp_geom *geom, const int32_t *src, const int32_t *suffix_len, void *k_suffix,
                                   void *v_suffix, int32_t suffix_cap, int32_t *suffix_len_out, santapp_stream stream)
{
    const int rc = check_geometry(geom);
    if (rc != SANTAPP_OK) return rc;
    if (!src || !suffix_len || !k_suffix || !v_suffix || suffix_cap < 1 || k_suffix == v_suffix) return SANTAPP_ERR_INVALID_ARG;
    const auto off = [](const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; };
    if (off(src, 4) || off(suffix_len, 4) || off(k_suffix, 16) || off(v_suffix, 16) || off(suffix_len_out, 4))
        return SANTAPP_ERR_INVALID_ARG;
    if (geom->n_seqs > kForkMaxSeqs) return SANTAPP_ERR_UNSUPPORTED;
    if (geom->n_kv_heads > 65535) return SANTAPP_ERR_UNSUPPORTED;
    if ((int64_t)geom->n_seqs * geom->n_kv_heads * (int64_t)suffix_cap >= (int64_t)1 << 31) return SANTAPP_ERR_UNSUPPORTED;
    if (suffix_len_out) {                                       // other blocks still read the lengths when one writes the new ones
        const uintptr_t bytes = sizeof(int32_t) * (uintptr_t)geom->n_seqs, o = reinterpret_cast<uintptr_t>(suffix_len_out);
        for (const int32_t *in : {src, suffix_len}) {
            const uintptr_t i = reinterpret_cast<uintptr_t>(in);
            if (o < i + bytes && i < o + bytes) return SANTAPP_ERR_INVALID_ARG;
        }
    }
    ForkParams p;
    p.n_seqs = geom->n_seqs;
    p.n_kv = geom->n_kv_heads;
    p.cap = suffix_cap;
    p.piece_bits = 4;
    while (p.piece_bits > 1 && p.n_seqs << (p.piece_bits + 4) > 128 * 1024) --p.piece_bits;     // (32 bytes: a sector of memory; 128 KB at 4096 slots)
    p.row_bits = 0;
    while (p.row_bits < 4 && p.n_seqs << (p.piece_bits + p.row_bits + 5) <= kForkStage) ++p.row_bits;
    p.src = src;
    p.len = suffix_len;
    p.k = static_cast<uint4 *>(k_suffix);
    p.v = static_cast<uint4 *>(v_suffix);
    p.len_out = suffix_len_out;
    begin_call();
    const size_t smem = ((size_t)p.n_seqs << (p.row_bits + p.piece_bits + 4)) + sizeof(int2) * (size_t)p.n_seqs;
    static std::atomic<unsigned long long> opted{0};
    cudaError_t err = ensure_dynamic_smem(reinterpret_cast<const void *>(fork_kernel), 200 * 1024, opted);
    if (err != cudaSuccess) return note_cuda_failure(err, "fork set-up");
    const dim3 grid((unsigned)(((suffix_cap + (1 << p.row_bits) - 1) >> p.row_bits) << (4 - p.piece_bits)), (unsigned)p.n_kv, 2);
    err = launch_step(fork_kernel, grid, dim3(kForkThreads), smem, static_cast<cudaStream_t>(stream), p);
    if (err != cudaSuccess) return note_cuda_failure(err, "fork launch");
    note_launch_count(1);
    return SANTAPP_OK;
}
