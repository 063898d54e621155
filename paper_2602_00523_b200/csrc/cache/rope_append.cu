// Rotary positions with up to three axes, and the way of new keys and values into the paged cache, sm_100a.
//
// Element pair (i, i + 64) of a query or key row turns by a_i = pos[axis_i] * inv_freq_i:
//   x'[i] = x[i] cos a_i - x[i + 64] sin a_i,  x'[i + 64] = x[i + 64] cos a_i + x[i] sin a_i.
// Bound by memory: every row is read once and written once.  A block takes one token of one layer (all heads, so that
// the 64 angles are worked out once for 20 KB of rows) and asks for its rows before it works them out.
// The angle is a number of turns in 64 bits, of which only the fraction counts: a position of 2^20 times a frequency of 1
// has 0.06 radians of rounding in 32 bits.  The fraction, at most half a turn, then goes through sincospif in 32 bits.
#include "sage_common.cuh"

namespace sage {
namespace rope {

constexpr int kUnits = 768;             // units of a token that are asked for at once: 80 heads (64 + 8 + 8) have 640

struct Params {
    const __nv_bfloat16 *q, *k, *v;
    int64_t q_layer, q_token, k_layer, k_token, v_layer, v_token;      // elements between layers and between tokens
    __nv_bfloat16 *out, *k_pool, *v_pool;
    int64_t layer_stride;
    int n_pages, max_pages, batch, sum_tokens, Hq, Hkv;
    const int32_t *pos, *parent, *next_pos;     // pos [3][sum_tokens], or the tree and each sequence's next position
    const int32_t *page_table, *seq_len, *node_offsets;
    int32_t* status;
    double turns[64];                   // inv_freq / (2 pi)
    uint8_t axis[64];
    float scale;
};

__device__ __forceinline__ void turn2(uint32_t lo, uint32_t hi, float2 c, float2 s, uint32_t& out_lo, uint32_t& out_hi) {
    const float l0 = __uint_as_float(lo << 16), l1 = __uint_as_float(lo & 0xffff0000u), h0 = __uint_as_float(hi << 16),
                h1 = __uint_as_float(hi & 0xffff0000u);
    __nv_bfloat162 a = __floats2bfloat162_rn(l0 * c.x - h0 * s.x, l1 * c.y - h1 * s.y);
    __nv_bfloat162 b = __floats2bfloat162_rn(h0 * c.x + l0 * s.x, h1 * c.y + l1 * s.y);
    out_lo = *reinterpret_cast<uint32_t*>(&a);
    out_hi = *reinterpret_cast<uint32_t*>(&b);
}

// kThreads: of a block.  256 spread a token's rows over more warps, 128 leave more blocks on an SM: 16384 tokens of 64 + 8 + 8 heads 117 / 109.5 us,
// 3000 tokens 28.4 / 28.7, 672 tokens 7.5 / 8.8.  (The chain in front of the stores is short on purpose: positions are asked for beside the rows, the page id is
// not waited for before the angles are there, 130 -> 117 us.  Two or four tokens a block, the next one's rows asked for early: 146, 153.)
template <int kThreads>
__global__ void __launch_bounds__(kThreads) rope_append_kernel(const __grid_constant__ Params p) {
    __shared__ float2 s_cs[64];         // (cos, sin)
    __shared__ int s_b, s_parent[SAGE_MAX_NODES];
    const int tid = threadIdx.x, tok = blockIdx.x, layer = blockIdx.y;
    if (tid == 0) s_b = -1;
    after_previous_kernel();
    __syncthreads();
    for (int b = tid; b < p.batch; b += kThreads) {
        const int a = p.node_offsets[b], z = p.node_offsets[b + 1];
        if (a <= tok && tok < z) s_b = b;
        if (tok == 0 && layer == 0 && (a < 0 || z < a || z > p.sum_tokens)) report_status(p.status, SAGE_STATUS_BAD_TREE);
    }
    // A unit is 16 bytes of either half of a query or key head, or 32 bytes of a value head.
    const int turned = (p.Hq + p.Hkv) * 8, units = turned + p.Hkv * 8;
    auto source = [&](int u) {
        const int h = u >> 3, c = (u & 7) * 8;
        if (h < p.Hq) return p.q + layer * p.q_layer + tok * p.q_token + h * kHeadDim + c;
        if (h < p.Hq + p.Hkv) return p.k + layer * p.k_layer + tok * p.k_token + (h - p.Hq) * kHeadDim + c;
        return p.v + layer * p.v_layer + tok * p.v_token + (h - p.Hq - p.Hkv) * kHeadDim + c;
    };
    constexpr int kRounds = kUnits / kThreads;
    uint4 lo[kRounds], hi[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int u = tid + i * kThreads;
        if (u < units) {
            const __nv_bfloat16* x = source(u);
            lo[i] = *reinterpret_cast<const uint4*>(x);
            hi[i] = *reinterpret_cast<const uint4*>(x + 64);
        }
    }
    int pos = 0;
    if (p.pos && tid < 64) pos = p.pos[(size_t)p.axis[tid] * p.sum_tokens + tok];     // (asked for beside the rows)
    __syncthreads();
    const int b = s_b;
    if (b < 0) return;                  // (a row behind the last sequence: left as it is)
    const int n0 = p.node_offsets[b], N = p.node_offsets[b + 1] - n0, L = p.seq_len[b];
    if (n0 < 0 || n0 + (long long)N > p.sum_tokens) return;     // (reported above)
    if (L < 0 || (long long)L + N > (long long)p.max_pages * kPageSize) {
        if (tid == 0) report_status(p.status, SAGE_STATUS_BAD_PAGE);
        return;
    }
    const int at = L + tok - n0;        // logical position in the cache
    const int page_id = p.page_table[(size_t)b * p.max_pages + at / kPageSize];
    int depth = 0;
    if (!p.pos) {
        if (N > SAGE_MAX_NODES) {
            if (tid == 0) report_status(p.status, SAGE_STATUS_BAD_TREE);
            return;
        }
        if (tid < N) s_parent[tid] = p.parent[n0 + tid];
        __syncthreads();
        bool bad = s_parent[0] != -1;
        for (int i = tok - n0; i > 0; ++depth) {            // (parents lie in front of their children)
            const int up = s_parent[i];
            if (up < 0 || up >= i) { bad = true; break; }
            i = up;
        }
        if (bad) {                      // uniform
            if (tid == 0) report_status(p.status, SAGE_STATUS_BAD_TREE);
            return;
        }
    }
    if (tid < 64) {
        if (!p.pos) pos = p.next_pos[b] + depth;
        const double t = (double)pos * p.turns[tid];
        float s, c;
        sincospif(2.f * (float)(t - rint(t)), &s, &c);
        s_cs[tid] = make_float2(c * p.scale, s * p.scale);
    }
    int page = page_id;                 // (looked at only now: the angles need not wait for it)
    if (page < 0 || page >= p.n_pages) {
        if (tid == 0) report_status(p.status, SAGE_STATUS_BAD_PAGE);
        page = -1;
    }
    __syncthreads();
    auto finish = [&](int u, const uint4& l, const uint4& h) {
        const int head = u >> 3, c = (u & 7) * 8;
        uint4 a = l, z = h;
        if (u < turned) {
            const float4* cs = reinterpret_cast<const float4*>(s_cs + c);
            const float4 w0 = cs[0], w1 = cs[1], w2 = cs[2], w3 = cs[3];       // (cos, sin) of two elements each
            turn2(l.x, h.x, make_float2(w0.x, w0.z), make_float2(w0.y, w0.w), a.x, z.x);
            turn2(l.y, h.y, make_float2(w1.x, w1.z), make_float2(w1.y, w1.w), a.y, z.y);
            turn2(l.z, h.z, make_float2(w2.x, w2.z), make_float2(w2.y, w2.w), a.z, z.z);
            turn2(l.w, h.w, make_float2(w3.x, w3.z), make_float2(w3.y, w3.w), a.w, z.w);
        }
        __nv_bfloat16* dst;
        if (head < p.Hq) {
            dst = p.out + (((size_t)layer * p.sum_tokens + tok) * p.Hq + head) * kHeadDim + c;
        } else {
            if (page < 0) return;
            const bool key = head < p.Hq + p.Hkv;
            const int g = head - p.Hq - (key ? 0 : p.Hkv);
            dst = (key ? p.k_pool : p.v_pool) + layer * p.layer_stride + (((size_t)page * p.Hkv + g) * kPageSize + at % kPageSize) * kHeadDim + c;
        }
        *reinterpret_cast<uint4*>(dst) = a;
        *reinterpret_cast<uint4*>(dst + 64) = z;
    };
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int u = tid + i * kThreads;
        if (u < units) finish(u, lo[i], hi[i]);
    }
    for (int u = tid + kRounds * kThreads; u < units; u += kThreads) {
        const __nv_bfloat16* x = source(u);
        finish(u, *reinterpret_cast<const uint4*>(x), *reinterpret_cast<const uint4*>(x + 64));
    }
}

}  // namespace rope
}  // namespace sage

using namespace sage;

extern "C" int sage_rope_append(const sage_rope_rows* rows, const sage_rope_policy* policy, int n_layers, int sum_tokens, int n_q_heads,
                                int n_kv_heads, int head_dim, const int32_t* pos, const int32_t* parent, const int32_t* next_pos,
                                void* q_out, void* k_pool, void* v_pool, int64_t layer_stride_elems, int n_pages, int page_size,
                                const int32_t* page_table, int max_pages_per_seq, const int32_t* seq_len, const int32_t* node_offsets,
                                int batch, int32_t* status, void* stream) {
    if (!rows || !policy || !rows->q || !rows->k || !rows->v || !q_out || !k_pool || !v_pool || !page_table || !seq_len || !node_offsets)
        return SAGE_ERR_INVALID_ARG;
    if (pos ? (parent || next_pos) : (!parent || !next_pos)) return SAGE_ERR_INVALID_ARG;      // positions are given, or follow from the tree
    if (n_layers < 1 || sum_tokens < 0 || n_q_heads < 1 || n_kv_heads < 1 || n_pages < 1 || max_pages_per_seq < 1 || batch < 0 ||
        layer_stride_elems < 0)
        return SAGE_ERR_INVALID_ARG;
    if (head_dim != kHeadDim || page_size != kPageSize || n_layers > 65535 || max_pages_per_seq > (1 << 24) ||
        n_q_heads > 65536 || n_kv_heads > 65536)
        return SAGE_ERR_UNSUPPORTED;
    const uintptr_t at = (uintptr_t)rows->q | (uintptr_t)rows->k | (uintptr_t)rows->v | (uintptr_t)q_out | (uintptr_t)k_pool | (uintptr_t)v_pool;
    const int64_t strides[6] = {rows->q_layer_stride, rows->q_token_stride, rows->k_layer_stride, rows->k_token_stride, rows->v_layer_stride,
                                rows->v_token_stride};
    if ((at & 15) || (layer_stride_elems & 7)) return SAGE_ERR_INVALID_ARG;
    for (int64_t s : strides)
        if (s < 0 || (s & 7)) return SAGE_ERR_INVALID_ARG;
    if (n_layers > 1 && layer_stride_elems < (int64_t)n_pages * n_kv_heads * kPageSize * kHeadDim) return SAGE_ERR_INVALID_ARG;
    rope::Params p{};
    for (int i = 0; i < 64; ++i) {
        if (policy->axis[i] > 2 || !(policy->inv_freq[i] >= -1e6 && policy->inv_freq[i] <= 1e6)) return SAGE_ERR_INVALID_ARG;
        p.turns[i] = policy->inv_freq[i] * 0.15915494309189533577;      // 1 / (2 pi)
        p.axis[i] = policy->axis[i];
    }
    if (batch == 0 || sum_tokens == 0) return SAGE_OK;
    p.q = (const __nv_bfloat16*)rows->q; p.k = (const __nv_bfloat16*)rows->k; p.v = (const __nv_bfloat16*)rows->v;
    p.q_layer = strides[0]; p.q_token = strides[1]; p.k_layer = strides[2]; p.k_token = strides[3]; p.v_layer = strides[4]; p.v_token = strides[5];
    p.out = (__nv_bfloat16*)q_out; p.k_pool = (__nv_bfloat16*)k_pool; p.v_pool = (__nv_bfloat16*)v_pool;
    p.layer_stride = layer_stride_elems;
    p.n_pages = n_pages; p.max_pages = max_pages_per_seq; p.batch = batch; p.sum_tokens = sum_tokens; p.Hq = n_q_heads; p.Hkv = n_kv_heads;
    p.pos = pos; p.parent = parent; p.next_pos = next_pos;
    p.page_table = page_table; p.seq_len = seq_len; p.node_offsets = node_offsets;
    p.status = status;
    p.scale = policy->scale;
    const dim3 grid(sum_tokens, n_layers);
    if ((int64_t)sum_tokens * n_layers >= 4096) return launch_status(launch(rope::rope_append_kernel<128>, grid, 128, 0, as_stream(stream), 0, p));
    return launch_status(launch(rope::rope_append_kernel<256>, grid, 256, 0, as_stream(stream), 0, p));
}
