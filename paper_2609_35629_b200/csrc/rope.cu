// Rotary positions (santapp_rope_append, santapp_rope_prompt).
//
// A pair (a, b) of a head at position p turns by p w: (a cos - b sin, b cos + a sin), times an amplitude.
// Angles are kept in turns: w / 2 pi in fp64, p times that less its nearest integer in fp64, so what reaches the
// fp32 sine and cosine is below half a turn at any position (fp32 throughout would be 0.008 rad off at 131072).
//
// Bound by memory: every value is read once and written once (18.4 KB each way for a token of 28 + 4 + 4 heads). All heads of
// a token share its 64 angles: a block computes them once, a pair per thread, into shared memory, behind the loads
// of its rows, which are under way before.
#include <math.h>
#include <string.h>

#include "common.cuh"
#include "santapp_serve.h"

namespace santapp {

namespace {

constexpr int kRopeThreads = 256;
// Many rows: four tokens a block, two units of 32 bytes a thread under way and six blocks an SM. A 32K prompt's 28 + 4 + 4 heads (604 MB)
// take 100 us inside a graph, 6.0 TB/s (93 % of the copy rate), 109 eagerly; five units and three blocks 117, one token a block 114, eight blocks 99 to 109.
constexpr int kMany = 4, kManyAhead = 2, kManyBlocks = 6;
constexpr int kUnits = 8;                 // units of a head: two 16-byte pieces that hold both values of eight pairs

struct RopeParams {
    int n_q, n_kv, rot, interleaved;
    int64_t n_rows;
    const uint4 *q, *k, *v;               // 16-byte pieces
    int64_t q_stride, k_stride, v_stride; // pieces from token to token
    const int32_t *positions;             // nullable: the row's index. Append: base_pos
    const int32_t *rows;                  // append: suffix_len; else dst_row, nullable: the row's index
    int64_t row_limit;                    // append: suffix_cap; else plane rows
    int append;
    uint4 *q_out, *k_out, *v_out;
    int32_t *len_out;                     // append, nullable
    float amplitude;
    double turns[64];                     // inv_freq / 2 pi
};

// Eight pairs: first values in a, second in b (16-bit), cos and sin of each.
template <bool kHalf>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    uint32_t r;
    if constexpr (kHalf) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else                 asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <bool kHalf>
__device__ __forceinline__ void turn_halves(uint4 &x, uint4 &y, const float2 *cs)
{
    uint32_t *a = reinterpret_cast<uint32_t *>(&x), *b = reinterpret_cast<uint32_t *>(&y);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 c = *reinterpret_cast<const float4 *>(cs + 2 * i);          // cos, sin, cos, sin
        const float a0 = elem_lo<kHalf>(a[i]), a1 = elem_hi<kHalf>(a[i]), b0 = elem_lo<kHalf>(b[i]), b1 = elem_hi<kHalf>(b[i]);
        a[i] = pack2<kHalf>(a0 * c.x - b0 * c.y, a1 * c.z - b1 * c.w);
        b[i] = pack2<kHalf>(b0 * c.x + a0 * c.y, b1 * c.z + a1 * c.w);
    }
}
// The same for neighbouring values: a word is a pair.
template <bool kHalf>
__device__ __forceinline__ void turn_neighbours(uint4 &x, uint4 &y, const float2 *cs)
{
    uint32_t *w[2] = {reinterpret_cast<uint32_t *>(&x), reinterpret_cast<uint32_t *>(&y)};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 c = cs[i];
        uint32_t &v = w[i >> 2][i & 3];
        const float a = elem_lo<kHalf>(v), b = elem_hi<kHalf>(v);
        v = pack2<kHalf>(a * c.x - b * c.y, b * c.x + a * c.y);
    }
}

// kTokens tokens a block, kAhead units a thread under way.
template <bool kHalf, int kTokens, int kAhead, int kBlocks>
__global__ void __launch_bounds__(kRopeThreads, kBlocks)
rope_kernel(const __grid_constant__ RopeParams p)
{
    step_wait();
    __shared__ __align__(16) float2 table[kTokens][64];
    __shared__ int64_t dst[kTokens];                        // row each token's key and value go to; negative: none
    const int tid = threadIdx.x;
    const int64_t row0 = (int64_t)blockIdx.x * kTokens;
    const int n_tok = (int)min((int64_t)kTokens, p.n_rows - row0);
    const int heads = p.n_q + 2 * p.n_kv, half = p.rot / 2, n_units = n_tok * heads * kUnits;

    // pieces of unit u of a head: rotated ones hold pairs 8 u .. 8 u + 7
    auto first_piece = [&](int u) { return u < p.rot / 16 && !p.interleaved ? u : 2 * u; };
    auto second_piece = [&](int u) { return u < p.rot / 16 && !p.interleaved ? u + p.rot / 16 : 2 * u + 1; };
    // token and row of heads of unit e
    const auto token_of = [&](int e) {
        int t = 0;
#pragma unroll
        for (int x = 1; x < kTokens; ++x) t += e >= x * heads * kUnits;
        return t;
    };
    uint4 x[kAhead], y[kAhead];
    auto load = [&](int base) {
#pragma unroll
        for (int m = 0; m < kAhead; ++m) {
            const int e = base + m * kRopeThreads + tid;
            if (e >= n_units) break;
            const int u = e & (kUnits - 1), t = token_of(e), h = e / kUnits - t * heads;
            const int64_t row = row0 + t;
            const uint4 *src = h < p.n_q ? p.q + row * p.q_stride + h * 16
                                         : (h < p.n_q + p.n_kv ? p.k + row * p.k_stride + (h - p.n_q) * 16
                                                               : p.v + row * p.v_stride + (h - p.n_q - p.n_kv) * 16);
            x[m] = src[first_piece(u)];
            y[m] = src[second_piece(u)];
        }
    };
    load(0);
    int len = 0;
    if (tid < kTokens * 64 && (tid >> 6) < n_tok) {
        const int t = tid >> 6, i = tid & 63;
        const int64_t row = row0 + t;
        len = p.rows != nullptr ? p.rows[row] : (int)row;
        const double pos = p.positions != nullptr ? (double)p.positions[row] + (p.append ? (double)len : 0.0) : (double)row;
        if (i < half) {
            const double turns = pos * p.turns[i];
            float s, c;
            sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
            table[t][i] = make_float2(c * p.amplitude, s * p.amplitude);
        }
        if (i == 0) dst[t] = p.rows == nullptr ? row : (len >= 0 && len < p.row_limit ? (int64_t)len : (int64_t)-1);
    }
    __syncthreads();
    if (p.append && p.len_out != nullptr && tid < kTokens * 64 && (tid & 63) == 0 && (tid >> 6) < n_tok)
        p.len_out[row0 + (tid >> 6)] = dst[tid >> 6] >= 0 ? len + 1 : len;
    for (int base = 0; base < n_units; base += kAhead * kRopeThreads) {
        if (base > 0) load(base);
#pragma unroll
        for (int m = 0; m < kAhead; ++m) {
            const int e = base + m * kRopeThreads + tid;
            if (e >= n_units) break;
            const int u = e & (kUnits - 1), t = token_of(e), h = e / kUnits - t * heads;
            const int64_t row = row0 + t, to = dst[t];
            if (h < p.n_q + p.n_kv && u < p.rot / 16) {
                if (p.interleaved) turn_neighbours<kHalf>(x[m], y[m], &table[t][8 * u]);
                else turn_halves<kHalf>(x[m], y[m], &table[t][8 * u]);
            }
            uint4 *out;
            if (h < p.n_q) {
                if (p.append && to < 0) continue;
                out = p.q_out + (row * p.n_q + h) * 16;
            } else {
                if (to < 0) continue;
                const int j = h < p.n_q + p.n_kv ? h - p.n_q : h - p.n_q - p.n_kv;
                const int64_t plane = p.append ? row * p.n_kv + j : j;
                out = (h < p.n_q + p.n_kv ? p.k_out : p.v_out) + (plane * p.row_limit + to) * 16;
            }
            out[first_piece(u)] = x[m];
            out[second_piece(u)] = y[m];
        }
    }
}

bool misaligned(const void *p, size_t a) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) % a) != 0; }

int check_rope(const santapp_geom *geom, const santapp_rope *r, const void *const (&rows)[6], int64_t q_stride, int64_t k_stride,
               int64_t v_stride)
{
    const int rc = check_geometry(geom);
    if (rc != SANTAPP_OK) return rc;
    if (!r) return SANTAPP_ERR_INVALID_ARG;
    if (r->interleaved != 0 && r->interleaved != 1) return SANTAPP_ERR_INVALID_ARG;
    if (r->rot_dim < 2 || r->rot_dim > kHeadDim || !isfinite((float)r->amplitude)) return SANTAPP_ERR_INVALID_ARG;
    if (r->rot_dim % 16 != 0) return SANTAPP_ERR_UNSUPPORTED;
    for (int i = 0; i < r->rot_dim / 2; ++i)
        if (!isfinite(r->inv_freq[i]) || fabs(r->inv_freq[i]) > 1e6) return SANTAPP_ERR_INVALID_ARG;
    for (const void *x : rows)
        if (x == nullptr || misaligned(x, 16)) return SANTAPP_ERR_INVALID_ARG;
    const int64_t q_row = (int64_t)geom->n_q_heads * kHeadDim, kv_row = (int64_t)geom->n_kv_heads * kHeadDim;
    if (q_stride < q_row || k_stride < kv_row || v_stride < kv_row || q_stride % 8 || k_stride % 8 || v_stride % 8)
        return SANTAPP_ERR_INVALID_ARG;
    if (rows[3] == rows[0] && q_stride != q_row) return SANTAPP_ERR_INVALID_ARG;          // q_out is dense
    return SANTAPP_OK;
}

int run_rope(RopeParams &p, const santapp_geom *geom, const santapp_rope *r, santapp_stream stream)
{
    p.n_q = geom->n_q_heads;
    p.n_kv = geom->n_kv_heads;
    p.rot = r->rot_dim;
    p.interleaved = r->interleaved;
    p.amplitude = (float)r->amplitude;
    for (int i = 0; i < 64; ++i) p.turns[i] = i < r->rot_dim / 2 ? r->inv_freq[i] / 6.283185307179586476925 : 0.0;
    begin_call();
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool many = p.n_rows >= 4 * 4 * (int64_t)attend_grid_size();
    const dim3 grid((unsigned)(many ? (p.n_rows + kMany - 1) / kMany : p.n_rows));
    cudaError_t err;
    if (many) err = launch_step(geom->elem_type ? rope_kernel<true, kMany, kManyAhead, kManyBlocks> : rope_kernel<false, kMany, kManyAhead, kManyBlocks>, grid, dim3(kRopeThreads), 0, s, p);
    else      err = launch_step(geom->elem_type ? rope_kernel<true, 1, 5, 1> : rope_kernel<false, 1, 5, 1>, grid, dim3(kRopeThreads), 0, s, p);
    if (err != cudaSuccess) return note_cuda_failure(err, "rope launch");
    note_launch_count(1);
    return SANTAPP_OK;
}

RopeParams rope_params(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride, void *q_out,
                       void *k_out, void *v_out)
{
    RopeParams p;
    memset(&p, 0, sizeof(p));
    p.q = static_cast<const uint4 *>(q);
    p.k = static_cast<const uint4 *>(k);
    p.v = static_cast<const uint4 *>(v);
    p.q_stride = q_stride / 8;
    p.k_stride = k_stride / 8;
    p.v_stride = v_stride / 8;
    p.q_out = static_cast<uint4 *>(q_out);
    p.k_out = static_cast<uint4 *>(k_out);
    p.v_out = static_cast<uint4 *>(v_out);
    return p;
}

}  // namespace

}  // namespace santapp

using namespace santapp;

extern "C" {

int santapp_rope_frequencies(santapp_rope *rope, double theta, double factor, double low, double high, double original_len)
{
    if (!rope || rope->rot_dim < 2 || rope->rot_dim > kHeadDim || rope->rot_dim % 2 != 0) return SANTAPP_ERR_INVALID_ARG;
    if (!(theta > 1.0) || !(factor >= 1.0) || !(original_len >= 0.0) || !isfinite(theta) || !isfinite(factor) || !isfinite(original_len))
        return SANTAPP_ERR_INVALID_ARG;
    if (original_len > 0.0 && (!(high > low) || !isfinite(low) || !isfinite(high))) return SANTAPP_ERR_INVALID_ARG;
    for (int i = 0; i < rope->rot_dim / 2; ++i) {
        const double f = pow(theta, -2.0 * i / rope->rot_dim);
        double keep = 0.0;
        if (original_len > 0.0) {
            keep = (original_len * f / 6.283185307179586476925 - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
        }
        rope->inv_freq[i] = f * (keep + (1.0 - keep) / factor);
    }
    return SANTAPP_OK;
}

int santapp_rope_append(const santapp_geom *geom, const santapp_rope *rope, const void *q, int64_t q_stride, const void *k,
                        int64_t k_stride, const void *v, int64_t v_stride, const int32_t *base_pos, const int32_t *suffix_len,
                        void *q_out, void *k_suffix, void *v_suffix, int32_t suffix_cap, int32_t *suffix_len_out,
                        santapp_stream stream)
{
    const int rc = check_rope(geom, rope, {q, k, v, q_out, k_suffix, v_suffix}, q_stride, k_stride, v_stride);
    if (rc != SANTAPP_OK) return rc;
    if (!base_pos || !suffix_len || suffix_cap < 1) return SANTAPP_ERR_INVALID_ARG;
    if (misaligned(base_pos, 4) || misaligned(suffix_len, 4) || misaligned(suffix_len_out, 4)) return SANTAPP_ERR_INVALID_ARG;
    if ((int64_t)geom->n_seqs * geom->n_kv_heads * (int64_t)suffix_cap >= (int64_t)1 << 31) return SANTAPP_ERR_UNSUPPORTED;
    if (suffix_len_out) {                                       // other blocks still read lengths and positions when one writes its new length
        const uintptr_t bytes = sizeof(int32_t) * (uintptr_t)geom->n_seqs, o = reinterpret_cast<uintptr_t>(suffix_len_out);
        for (const int32_t *in : {base_pos, suffix_len}) {
            const uintptr_t i = reinterpret_cast<uintptr_t>(in);
            if (o < i + bytes && i < o + bytes && !(in == suffix_len && o == i)) return SANTAPP_ERR_INVALID_ARG;
        }
    }
    RopeParams p = rope_params(q, q_stride, k, k_stride, v, v_stride, q_out, k_suffix, v_suffix);
    p.n_rows = geom->n_seqs;
    p.positions = base_pos;
    p.rows = suffix_len;
    p.row_limit = suffix_cap;
    p.append = 1;
    p.len_out = suffix_len_out;
    return run_rope(p, geom, rope, stream);
}

int santapp_rope_prompt(const santapp_geom *geom, const santapp_rope *rope, int64_t n_rows, const void *q, int64_t q_stride,
                        const void *k, int64_t k_stride, const void *v, int64_t v_stride, const int32_t *positions,
                        const int32_t *dst_row, void *q_out, void *k_prompt, void *v_prompt, int64_t plane_rows,
                        santapp_stream stream)
{
    const int rc = check_rope(geom, rope, {q, k, v, q_out, k_prompt, v_prompt}, q_stride, k_stride, v_stride);
    if (rc != SANTAPP_OK) return rc;
    if (n_rows < 1 || plane_rows < 1 || (dst_row == nullptr && plane_rows < n_rows)) return SANTAPP_ERR_INVALID_ARG;
    if (misaligned(positions, 4) || misaligned(dst_row, 4)) return SANTAPP_ERR_INVALID_ARG;
    if (n_rows >= (int64_t)1 << 31 || plane_rows >= (int64_t)1 << 31) return SANTAPP_ERR_UNSUPPORTED;
    RopeParams p = rope_params(q, q_stride, k, k_stride, v, v_stride, q_out, k_prompt, v_prompt);
    p.n_rows = n_rows;
    p.positions = positions;
    p.rows = dst_row;
    p.row_limit = plane_rows;
    return run_rope(p, geom, rope, stream);
}

}  // extern "C"
