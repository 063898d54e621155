// Tree attention over part of a cache or over a cache in two forms, sm_100a:
//   sage_tree_attention_window : the last `window` positions and the first `sink` ones of a bf16 cache
//   sage_tree_attention_sealed : every position; full pages are e4m3 with a power-of-two scale for each page and KV head
//                                (see seal_kv.cu), the rest (the page that is not full, the tree's rows) is bf16
// For query row i (a node and one of the G query heads that share a KV head), out = sum_t p_t V[t] / sum_t p_t with
// p_t = exp(sm_scale q K[t]), t over what the row sees.
//
// A block owns one tile of 128 query rows and one slice of the pages that its item (layer, sequence, KV head) has to
// read; two blocks are resident on an SM (96 KB to 113 KB of shared memory, 256 columns of tensor memory each), so the chain
// scores -> softmax -> P V of one runs while the other's waits.  The pages to read are counted without the gap between sinks and
// window (Walk); the sealed ones come first in that order, and a block walks it backwards: bf16 pages, then sealed ones.
//   TMA     : query rows; K and V pages -> 128B-swizzled shared memory, a ring of five 16 KB slots: a bf16 page takes two
//             (K, V), a sealed one takes one for both
//   tcgen05 : S = Q K^T (128 x 64 fp32, two buffers), O += P V with P as the TMEM operand, V MN-major
//   softmax : one thread per row, online, fp32, log2 domain
// What is sealed is multiplied as it is, in kind::f8f6f4, without a way through registers and back: each bf16 query row is
// the sum of two e4m3 rows (split_queries: exact down to 2^-9 of the row's largest element, off by 2^-17 of it below), and each
// probability the sum of an e4m3 and an e5m2 number (pack_e4m3: 2^-7 of its value at most, where bf16 has 2^-8; 2^-23 of the
// row's reference at least).  Two products of 8 bits cost the tensor pipe what one of 16 does, and HBM half.
// The scales are powers of two: the key's goes into the row's factor of the scores, the value's into the exponent of the
// probabilities (against the largest of the pages so far, `v_ref`, to which the accumulator is scaled).
// All waits are bounded: on expiry the block records SAGE_STATUS_TIMEOUT, drains its copies and MMAs, frees its TMEM and returns.
#include <cuda_fp16.h>

#include "attention_stream.cuh"
#include "paged.cuh"

namespace sage {
namespace paged {

using namespace stream;

constexpr int kSlots = 5;                                   // ring of 16 KB slots
constexpr int kSlotBytes = kPageSize * kHeadDim * 2;        // a bf16 K or V page of a head, or both of a sealed one
constexpr int kSealedBytes = kPageSize * kHeadDim;          // a sealed K or V page of a head
constexpr int kThreads = 192;                               // a softmax warpgroup, the TMA warp, the MMA warp
constexpr int kTmemColumns = 256;                           // S 2 x 64, O 128
constexpr uint32_t kIdescPage = idesc_f16(kPageSize);       // S = Q K^T, bf16
// kind::f8f6f4: D fp32, M = 128; types of A: 0 e4m3, 1 e5m2; B e4m3
constexpr uint32_t idesc_f8(uint32_t n, uint32_t a_type) { return (1u << 4) | (a_type << 7) | ((n >> 3) << 17) | ((128u >> 4) << 24); }
constexpr uint32_t kIdescSealedQK = idesc_f8(kPageSize, 0);
constexpr uint32_t kIdescSealedPVHigh = idesc_f8(kHeadDim, 0) | (1u << 16);     // B (= V) MN-major
constexpr uint32_t kIdescSealedPVLow = idesc_f8(kHeadDim, 1) | (1u << 16);
// Probabilities are taken against a reference 2^kHeadroom below the maximum that set it, and may reach 448 = 2^8.807 (e4m3's
// largest): a row's maximum may grow by 2.8 (in log2; 1.9 in the scores) before the accumulator is scaled again.
constexpr float kHeadroom = 6.f, kMostLog2 = 8.807f;
// Exponents of sealed scales (sage_seal_kv writes no others; a byte outside is read as the nearest).
constexpr int kExpLo = 127 - 60, kExpHi = 127 + 60;

struct __align__(8) Shared {
    uint64_t full[kSlots], empty[kSlots];
    uint64_t s_full[2];        // [page parity]: scores of a page are in TMEM
    uint64_t p_full[2];        // [page parity]: probabilities of a page are in TMEM (an arrival per warp that has rows)
    uint64_t pv_done;          // completes once per page, when its P V product has finished
    uint64_t o_full;           // every MMA has finished
    uint64_t q_ready;          // the query rows are in shared memory
    uint64_t q_split;          // ... as two e4m3 rows each
    uint32_t tmem_base;
    volatile int abort;
    float k_scale[kSlots];     // of the sealed page in a slot
    int v_exp[kSlots];
    int parent[SAGE_MAX_NODES];
};
constexpr int kSmemBytes = kQTileBytes + kSlots * kSlotBytes + 1024;
static_assert(sizeof(Shared) <= 1024 && 2 * (kSmemBytes + 1024) <= 233472, "two blocks have to fit on an SM");

// D[tmem] (+)= A[smem desc] * B[smem desc], 8-bit operands (see mma_ss)
template <uint32_t kHi, uint32_t kIdesc>
__device__ __forceinline__ void mma_ss_f8(uint32_t leader, uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
                 "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %4, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "n"(kHi), "n"(kIdesc), "r"(acc), "r"(leader) : "memory");
}
template <uint32_t kHi, uint32_t kIdesc>
__device__ __forceinline__ void mma_ts_f8(uint32_t leader, uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
                 "mov.b64 db, {%2, %3};\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], db, %4, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "n"(kHi), "n"(kIdesc), "r"(acc), "r"(leader) : "memory");
}

// Two fp16 numbers (each exactly the sum of what comes back, as far as the formats reach) as a pair of e4m3 and the pair that is
// left over, in e4m3 or e5m2.
template <bool kLowE5M2>
__device__ __forceinline__ void split_pair(uint32_t x, uint32_t& high, uint32_t& low) {
    uint16_t h, l;
    uint32_t back, rest;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(h) : "r"(x));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(back) : "h"(h));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(rest) : "r"(x), "r"(back));
    if constexpr (kLowE5M2) asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;" : "=h"(l) : "r"(rest));
    else asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(l) : "r"(rest));
    high = h;
    low = l;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }      // -126 <= e <= 127
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// The pages that a row tile reads, counted without the gap between sinks and window.
struct Walk {
    int n_sink;     // pages with sinks, in front of the window's first
    int w0;         // the window's first page
    int n_sealed;   // of all that are read; the others follow
    int n;          // pages
    __device__ __forceinline__ int page(int w) const { return w < n_sink ? w : w - n_sink + w0; }
};
__device__ __forceinline__ Walk make_walk(int L, int N, int sealed, int window, int sink) {
    Walk k;
    k.w0 = max(0, L - window + 1) / kPageSize;              // the root sees furthest back
    k.n_sink = min((sink + kPageSize - 1) / kPageSize, k.w0);
    k.n_sealed = min(k.n_sink, sealed) + max(0, sealed - k.w0);
    k.n = k.n_sink + (L + N + kPageSize - 1) / kPageSize - k.w0;
    return k;
}

// What a row sees: the slots of the tree, and where its window begins.
struct Sight {
    uint64_t tree;      // tree slots, one bit each
    int begin, end;     // prefix positions [begin, end) are out of sight
};
// Bits of the 64 keys of the page at position t0 that a row sees.
__device__ __forceinline__ uint64_t visible_page(const Sight& s, int t0, int L) {
    uint64_t vis = (uint64_t)visible_keys(t0 - L, s.tree) | ((uint64_t)visible_keys(t0 - L + 32, s.tree) << 32);
    const int a = max(s.begin - t0, 0), b = min(s.end - t0, 64);
    if (b > a) vis &= ~((b - a == 64 ? ~0ull : (1ull << (b - a)) - 1) << a);
    return vis;
}

// Probabilities of 64 keys as e4m3 (16 words, four keys each) and what is left over as e5m2 (16 words).
__device__ __forceinline__ void pack_e4m3(const float* pr, uint32_t* out) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        uint32_t h0, l0, h1, l1;
        split_pair<true>(pack_f16(pr[4 * i], pr[4 * i + 1]), h0, l0);
        split_pair<true>(pack_f16(pr[4 * i + 2], pr[4 * i + 3]), h1, l1);
        out[i] = h0 | (h1 << 16);
        out[16 + i] = l0 | (l1 << 16);
    }
}

// One page for one query row per thread: scores -> probabilities over the first 32 columns of the S buffer, running reference
// and sum.  scale: of this row and page; dv: exponent by which the page's values exceed the accumulator's; o_factor: what the accumulator
// is to be multiplied by because of the values' scales (1: nothing).  parity: of the P V product of the page before.
template <bool kSealedPage>
__device__ __forceinline__ bool softmax_page(const Params& p, Shared* sh, uint32_t parity, uint32_t s_taddr, uint32_t o_taddr, float scale,
                                             int dv, float o_factor, bool row_ok, bool first, bool masked, uint64_t vis,
                                             float& m_ref, float& l_sum) {
    uint32_t sr[64];
    tmem_ld32(s_taddr, *reinterpret_cast<uint32_t(*)[32]>(&sr[0]));
    tmem_ld32(s_taddr + 32, *reinterpret_cast<uint32_t(*)[32]>(&sr[32]));
    tmem_wait_ld();
    if (masked) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if (!((uint32_t)vis & (1u << i))) sr[i] = 0xff800000u;      // -inf
            if (!((uint32_t)(vis >> 32) & (1u << i))) sr[32 + i] = 0xff800000u;
        }
    }
    float mx = -INFINITY;
    max_chunk(sr, mx);
    max_chunk(sr + 32, mx);
    const float m_cand = mx * scale;
    const bool grow = row_ok && m_cand > m_ref + kMostLog2;
    float alpha = 1.f;
    if (grow) {
        alpha = fast_exp2(m_ref - (m_cand - kHeadroom));    // 0 when m_ref was -inf
        m_ref = m_cand - kHeadroom;
    }
    if (!first && __any_sync(0xffffffffu, grow || o_factor != 1.f)) {
        // O *= alpha, once the P V product of the page before has finished
        if (!__all_sync(0xffffffffu, mbar_wait(&sh->pv_done, parity, sh, p))) return false;
        tc_fence_after();
        rescale_o_rows(o_taddr, alpha * o_factor);
    }
    const float base = (m_ref == -INFINITY ? 0.f : -m_ref) + (float)dv;
    uint64_t acc[2] = {0ull, 0ull};
    if constexpr (kSealedPage) {
        const uint64_t scale2 = f2_pack(scale, scale), base2 = f2_pack(base, base);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            float x0, x1;
            f2_unpack(f2_fma(f2_pack(__uint_as_float(sr[2 * i]), __uint_as_float(sr[2 * i + 1])), scale2, base2), x0, x1);
            x0 = fast_exp2(x0);
            x1 = fast_exp2(x1);
            acc[i & 1] = f2_add(acc[i & 1], f2_pack(x0, x1));
            sr[2 * i] = __float_as_uint(x0);
            sr[2 * i + 1] = __float_as_uint(x1);
        }
        uint32_t packed[32];
        pack_e4m3(reinterpret_cast<const float*>(sr), packed);
        tmem_st32(s_taddr, packed);
    } else {
#pragma unroll
        for (int c = 0; c < 2; ++c) exp_chunk<0>(sr + 32 * c, scale, base, sr + 16 * c, acc);   // may hold -inf
        tmem_st32(s_taddr, sr);
    }
    float sum_a, sum_b;
    f2_unpack(f2_add(acc[0], acc[1]), sum_a, sum_b);
    l_sum = l_sum * alpha + (sum_a + sum_b) * pow2(-dv);
    tmem_wait_st();
    tc_fence_before();
    return true;
}

// A bf16 query row in shared memory (two swizzled rows of 128 bytes, one per 64-wide half) becomes two e4m3 rows in the same
// places: x 2^e = high + low, e such that the row's largest element lies in [128, 256).  Returns 2^-e (NaN for a row that is not finite).
__device__ __forceinline__ float split_queries(uint8_t* sQ, int r) {
    uint4 v[16];
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        v[c] = *reinterpret_cast<const uint4*>(sQ + (c >> 3) * kQHalfBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4));
        most = __vmaxu2(most, __vmaxu2(__vmaxu2(v[c].x & 0x7fff7fffu, v[c].y & 0x7fff7fffu), __vmaxu2(v[c].z & 0x7fff7fffu, v[c].w & 0x7fff7fffu)));
    }
    const int exponent = max(8, (int)(max(most & 0xffffu, most >> 16) >> 7));       // biased; below 8 the row is as good as zero
    if (exponent == 255) return __uint_as_float(0x7fffffffu);
    const float up = __uint_as_float((uint32_t)(261 - exponent) << 23);
#pragma unroll
    for (int c = 0; c < 8; ++c) {                           // 16 elements: 16 bytes of either row
        uint32_t h[4], l[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint4& s = v[2 * c + (k >> 1)];
            const uint32_t a = k & 1 ? s.z : s.x, b = k & 1 ? s.w : s.y;
            uint32_t h0, l0, h1, l1;
            split_pair<false>(pack_f16(__uint_as_float(a << 16) * up, __uint_as_float(a & 0xffff0000u) * up), h0, l0);
            split_pair<false>(pack_f16(__uint_as_float(b << 16) * up, __uint_as_float(b & 0xffff0000u) * up), h1, l1);
            h[k] = h0 | (h1 << 16);
            l[k] = l0 | (l1 << 16);
        }
        uint8_t* at = sQ + r * 128 + ((c ^ (r & 7)) << 4);
        *reinterpret_cast<uint4*>(at) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(at + kQHalfBytes) = make_uint4(l[0], l[1], l[2], l[3]);
    }
    return __uint_as_float((uint32_t)(exponent - 7) << 23);
}

__global__ void __launch_bounds__(kThreads, 2)
tree_attention_paged_kernel(const Params p, const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                            const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CUtensorMap k8map,
                            const __grid_constant__ CUtensorMap v8map) {
    // (the swizzle's pattern repeats every 1024 bytes of address; with no static shared memory the dynamic part begins on such a boundary)
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* sQ = smem;                                     // [2 halves][128 rows][128 B]
    uint8_t* sRing = smem + kQTileBytes;                    // [kSlots][16 KB]
    Shared* sh = reinterpret_cast<Shared*>(sRing + kSlots * kSlotBytes);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rtile = blockIdx.x % p.row_tiles;
    const int slice = blockIdx.x / p.row_tiles % p.n_splits;
    const int item = blockIdx.x / (p.row_tiles * p.n_splits);
    const int g = item % p.Hkv, b = item / p.Hkv % p.batch, layer = item / (p.Hkv * p.batch);
    if (warp == 4 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&qmap) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&kmap) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&vmap) : "memory");
        if (p.sealed) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&k8map) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&v8map) : "memory");
        }
    }
    after_previous_kernel();
    const int n0 = p.node_offsets[b];
    const int N = p.node_offsets[b + 1] - n0;
    const int L = p.seq_len[b];
    const int sealed = p.sealed ? p.sealed[b] : 0;
    const bool bad_tree = N < 1 || N > SAGE_MAX_NODES || n0 < 0 || n0 + N > p.sum_nodes;
    const bool bad_page = !bad_tree && (L < 0 || (long long)L + N > (long long)p.max_pages * kPageSize || sealed < 0 ||
                                        sealed > L / kPageSize || sealed > p.max_pages8 || (smem_u32(smem) & 1023));
    const int T = L + N, M = N * p.G, row0 = rtile * kRowTile;
    if (bad_tree || bad_page) {                             // uniform
        if (tid == 0) report_status(p.status, bad_tree ? SAGE_STATUS_BAD_TREE : SAGE_STATUS_BAD_PAGE);
        return;
    }
    if (row0 >= M) return;
    // this block's slice [w_lo, w_hi) of the pages to read; it walks them from the last to the first
    const Walk walk = make_walk(L, N, sealed, p.window, p.sink);
    const int per_slice = (walk.n + p.n_splits - 1) / p.n_splits;
    const int w_lo = min(walk.n, slice * per_slice), w_hi = min(walk.n, w_lo + per_slice);
    const int ns = w_hi - w_lo;
    const int nb = max(0, w_hi - max(w_lo, walk.n_sealed));      // bf16 pages; the others are sealed
    const int live_warps = min(4, (M - row0 + 31) / 32);
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&sh->tmem_base)), "r"(kTmemColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else if (tid == 0) {
        for (int i = 0; i < kSlots; ++i) { mbar_init(&sh->full[i], 1); mbar_init(&sh->empty[i], 1); }
        for (int x = 0; x < 2; ++x) { mbar_init(&sh->s_full[x], 1); mbar_init(&sh->p_full[x], live_warps); }
        mbar_init(&sh->pv_done, 1);
        mbar_init(&sh->o_full, 1);
        mbar_init(&sh->q_ready, 1);
        mbar_init(&sh->q_split, live_warps);
        sh->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem_base;
    // ring positions of a page: a bf16 page takes two slots in a row, a sealed one takes one
    auto k_seq = [&](int j) { return j < nb ? 2 * j : nb + j; };
    auto v_seq = [&](int j) { return j < nb ? 2 * j + 1 : nb + j; };

    if (warp == 4) {
        // =========================== TMA producer ===========================
        // Page ids (and scales) of 32 pages at a time, one per lane; each lane then hands its own out.
        struct Page { int id, ke, ve; };
        auto look_up = [&](int j) {
            Page e{0, 127, 127};
            if (j >= ns) return e;
            const int w = w_hi - 1 - j, pg = walk.page(w);
            const bool is8 = j >= nb;
            e.id = is8 ? p.page_table8[(size_t)b * p.max_pages8 + pg] : p.page_table[(size_t)b * p.max_pages + pg];
            if (e.id < 0 || e.id >= (is8 ? p.n_pages8 : p.n_pages)) {       // (checked: it becomes a TMA coordinate)
                report_status(p.status, SAGE_STATUS_BAD_PAGE);
                e.id = 0;
            }
            if (is8) {
                const size_t at = ((size_t)layer * p.n_pages8 + e.id) * p.Hkv + g;
                e.ke = p.k_exp[at];
                e.ve = p.v_exp[at];
            }
            return e;
        };
        const bool on = ns > 0 && !p.producer_off;
        int issued = 0;
        if (on) {
            if (lane == 0) {
                mbar_expect_tx(&sh->q_ready, kQTileBytes);
                for (int h = 0; h < 2; ++h)
                    tma_load_5d(smem_u32(sQ + h * kQHalfBytes), &qmap, h * 64, 0, g, n0 + (row0 >> p.g_shift), layer, &sh->q_ready);
            }
            Page now = look_up(lane);
            bool ok = true;
            for (int j0 = 0; ok && j0 < ns; j0 += 32) {
                const Page next = look_up(j0 + 32 + lane);
                const int n = min(32, ns - j0);
                for (int i = 0; ok && i < n; ++i) {
                    const int j = j0 + i;
                    const bool is8 = j >= nb;
                    const int id = __shfl_sync(0xffffffffu, now.id, i), ke = __shfl_sync(0xffffffffu, now.ke, i),
                              ve = __shfl_sync(0xffffffffu, now.ve, i);
                    const int c2 = id * p.Hkv + g;
                    for (int part = 0; part < (is8 ? 1 : 2); ++part) {
                        const int s = issued % kSlots, use = issued / kSlots;
                        if (use > 0) ok = mbar_wait_warp(&sh->empty[s], (use - 1) & 1, sh, p);
                        if (!ok) break;
                        if (lane == 0) {
                            uint8_t* dst = sRing + s * kSlotBytes;
                            if (is8) {
                                sh->k_scale[s] = __uint_as_float((uint32_t)min(max(ke, kExpLo), kExpHi) << 23);
                                sh->v_exp[s] = min(max(ve, kExpLo), kExpHi) - 127;
                            }
                            mbar_expect_tx(&sh->full[s], kSlotBytes);
                            if (is8) {
                                tma_load_4d(smem_u32(dst), &k8map, 0, 0, c2, layer, &sh->full[s]);
                                tma_load_4d(smem_u32(dst + kSealedBytes), &v8map, 0, 0, c2, layer, &sh->full[s]);
                            } else {
                                const CUtensorMap* map = part == 0 ? &kmap : &vmap;
                                for (int h = 0; h < 2; ++h)
                                    tma_load_4d(smem_u32(dst + h * kPageHalfBytes), map, h * 64, 0, c2, layer, &sh->full[s]);
                            }
                        }
                        ++issued;
                    }
                }
                now = next;
            }
            if (sh->abort && lane == 0) {
                // drain: every issued copy must land before the block may exit
                mbar_wait_quiet(&sh->q_ready, 0, p.wait_cycles);
                for (int n = max(0, issued - kSlots); n < issued; ++n)
                    mbar_wait_quiet(&sh->full[n % kSlots], (n / kSlots) & 1, p.wait_cycles);
            }
            __syncwarp();
        }
    } else if (warp == 5) {
        // =========================== MMA issuer ===========================
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        const int n = __shfl_sync(0xffffffffu, ns, 0);
        const uint32_t leader = elect_one() ? 1u : 0u;
        auto wait_all = [&](uint64_t* bar, uint32_t parity) { return mbar_wait_warp(bar, parity, sh, p); };
        const uint32_t dq = desc_lo(smem_u32(sQ), 16);
        const uint32_t dring = desc_lo(smem_u32(sRing), 16);
        const uint32_t dring_mn = desc_lo(smem_u32(sRing), kPageHalfBytes);
        const uint32_t o_tmem = tm + 128;
        auto wait_slot = [&](int seq) { return wait_all(&sh->full[seq % kSlots], (seq / kSlots) & 1); };
        auto issue_qk = [&](int j) {
            const int s = k_seq(j) % kSlots;
            const uint32_t d = tm + (j & 1) * 64, dk = dring + ((s * kSlotBytes) >> 4);
            if (j < nb) {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)              // slices of K = 16 over d = 128 (4 per 64-wide half)
                    mma_ss<kDescHi, kIdescPage>(leader, d, dq + (((ks >> 2) * kQHalfBytes + (ks & 3) * 32) >> 4),
                                                dk + (((ks >> 2) * kPageHalfBytes + (ks & 3) * 32) >> 4), ks > 0 ? 1u : 0u);
            } else {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)              // slices of K = 32: 4 of the high rows, 4 of the low ones
                    mma_ss_f8<kDescHi, kIdescSealedQK>(leader, d, dq + (((ks >> 2) * kQHalfBytes + (ks & 3) * 32) >> 4),
                                                       dk + (((ks & 3) * 32) >> 4), ks > 0 ? 1u : 0u);
            }
            tc_commit(leader, &sh->s_full[j & 1]);
            if (j < nb) tc_commit(leader, &sh->empty[s]);
        };
        auto issue_pv = [&](int j) {
            const int s = v_seq(j) % kSlots;
            const uint32_t a = tm + (j & 1) * 64, acc = j > 0 ? 1u : 0u;
            if (j < nb) {
                const uint32_t dv = dring_mn + ((s * kSlotBytes) >> 4);
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)              // 16 keys; P in TMEM (8 columns per slice), V MN-major
                    mma_ts<kDescHi, kIdescPV>(leader, o_tmem, a + ks * 8, dv + ((ks * 2048) >> 4), ks > 0 ? 1u : acc);
            } else {
                const uint32_t dv = dring_mn + ((s * kSlotBytes + kSealedBytes) >> 4);
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)              // 32 keys
                    mma_ts_f8<kDescHi, kIdescSealedPVHigh>(leader, o_tmem, a + ks * 8, dv + ((ks * 4096) >> 4), ks > 0 ? 1u : acc);
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
                    mma_ts_f8<kDescHi, kIdescSealedPVLow>(leader, o_tmem, a + 16 + ks * 8, dv + ((ks * 4096) >> 4), 1u);
            }
            tc_commit(leader, &sh->pv_done);
            tc_commit(leader, &sh->empty[s]);
        };
        // Keys of page j are there, and the query rows in the form that they need.
        auto keys_ready = [&](int j) {
            if (j >= n) return true;
            if (!wait_slot(k_seq(j))) return false;
            return j != nb || wait_all(&sh->q_split, 0);
        };
        auto values_ready = [&](int j) {
            if (j >= n) return true;
            if (j >= nb) return true;                       // (with its keys)
            if (!wait_slot(v_seq(j))) return false;
            const int valid = T - walk.page(w_hi - 1 - j) * kPageSize;
            if (valid < kPageSize) {
                // rows past the end of the sequence may hold anything: zero them so that 0 * V stays 0
                uint8_t* vb = sRing + v_seq(j) % kSlots * kSlotBytes;
                for (int c = lane; c < (kPageSize - valid) * 16; c += 32) {
                    const int r = valid + c / 16, ch = c % 16;
                    *reinterpret_cast<uint4*>(vb + (ch >> 3) * kPageHalfBytes + r * 128 + ((ch & 7) << 4)) = make_uint4(0, 0, 0, 0);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            return true;
        };
        bool ok = n > 0;
        if (ok) ok = wait_all(&sh->q_ready, 0);
        for (int j = 0; ok && j < min(2, n); ++j) {
            ok = keys_ready(j);
            if (!ok) break;
            tc_fence_after();
            issue_qk(j);
        }
        if (ok) ok = values_ready(0) && keys_ready(2);
        for (int j = 0; ok && j < n; ++j) {
            ok = wait_all(&sh->p_full[j & 1], (j >> 1) & 1);
            if (!ok) break;
            tc_fence_after();
            issue_pv(j);
            if (j + 2 < n) issue_qk(j + 2);                 // reuses this page's S buffer: in pipe order behind its P V
            ok = values_ready(j + 1) && keys_ready(j + 3);
        }
        tc_commit(leader, &sh->o_full);                     // arrives when every MMA has completed
        // abort: everything issued must retire before the TMEM and the tiles go away
        if (!ok && lane == 0) mbar_wait_quiet(&sh->o_full, 0, p.wait_cycles);
        __syncwarp();
    } else {
        // =========================== softmax ===========================
        const int r = tid;                                  // row inside the tile == TMEM lane
        const uint32_t lane_base = (uint32_t)(warp * 32) << 16;
        const uint32_t s_taddr = tmem + lane_base, o_taddr = tmem + lane_base + 128;
        const int R = row0 + r;
        const bool row_ok = R < M, warp_live = row0 + warp * 32 < M;
        const int node = row_ok ? R >> p.g_shift : 0;
        const int cut = L + N - p.window;                   // some row does not see the prefix positions in front of this one
        Sight sight{1ull << node, p.sink, 0};
        if (nb > 0 || cut > 0) {                            // some page is masked (all of them are bf16 without a window)
            for (int i = r; i < N; i += 128) sh->parent[i] = p.parent[n0 + i];
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (row_ok) {
                int depth = 0, at = node;
                bool bad = false;
                while (at > 0) {                            // (parents lie in front of their children: at most N - 1 turns)
                    const int up = sh->parent[at];
                    if (up < 0 || up >= at) { bad = true; break; }
                    at = up;
                    ++depth;
                    if (depth < p.window) sight.tree |= 1ull << at;
                }
                if (bad || sh->parent[0] != -1) {
                    report_status(p.status, SAGE_STATUS_BAD_TREE);
                    sight.tree = 1ull << node;
                } else if (L < p.sink && depth >= p.window) {       // sinks among the tree's own positions
                    at = node;
                    for (int d = depth; d >= 0; --d) {
                        if (L + d < p.sink) sight.tree |= 1ull << at;
                        at = sh->parent[at];
                    }
                }
                sight.end = min(L + depth - p.window + 1, L);
            }
        }
        float m_ref = -INFINITY, l_sum = 0.f;
        float row_scale = 0.f;                              // for sealed pages
        int v_ref = 0;                                      // exponent of the accumulator: at first that of the first sealed page, if there is one
        if (nb < ns) {
            int id = p.page_table8[(size_t)b * p.max_pages8 + walk.page(w_hi - 1 - nb)];
            if (id < 0 || id >= p.n_pages8) id = 0;
            v_ref = min(max((int)p.v_exp[((size_t)layer * p.n_pages8 + id) * p.Hkv + g], kExpLo), kExpHi) - 127;
        }
        bool ok = warp_live;
        if (ok && ns > 0 && nb == 0) {
            ok = mbar_wait_warp(&sh->q_ready, 0, sh, p);
            if (ok) {
                row_scale = split_queries(sQ, r) * p.scale_log2;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->q_split);
            }
        }
        for (int j = 0; ok && j < ns; ++j) {
            const int x = j & 1, seq = k_seq(j), s = seq % kSlots;
            ok = mbar_wait_warp(&sh->s_full[x], (j >> 1) & 1, sh, p);
            // A sealed page: the copy warp's own barrier too, which orders the scales that it has left beside the page.  (The slot is not filled
            // again before this warp has been through the page.  That of a bf16 page's keys may be by now: its barrier is not to be asked.)
            if (ok && j >= nb) ok = mbar_wait_warp(&sh->full[s], (seq / kSlots) & 1, sh, p);
            if (!ok) break;
            tc_fence_after();
            if (j == nb - 1 && nb < ns) {                   // the last bf16 scores are there: the query rows change their form
                row_scale = split_queries(sQ, r) * p.scale_log2;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->q_split);
            }
            const int t0 = walk.page(w_hi - 1 - j) * kPageSize;
            const bool masked = t0 + kPageSize > L || (t0 < cut && t0 + kPageSize > p.sink);
            const uint64_t vis = masked ? visible_page(sight, t0, L) : ~0ull;
            if (j < nb) {
                ok = softmax_page<false>(p, sh, (j - 1) & 1, s_taddr + x * 64, o_taddr, p.scale_log2, -v_ref, 1.f, row_ok, j == 0, masked, vis,
                                         m_ref, l_sum);
            } else {
                float o_factor = 1.f;
                const int ve = sh->v_exp[s];
                if (ve > v_ref) {
                    o_factor = pow2(v_ref - ve);
                    v_ref = ve;
                }
                ok = softmax_page<true>(p, sh, (j - 1) & 1, s_taddr + x * 64, o_taddr, row_scale * sh->k_scale[s], ve - v_ref, o_factor,
                                        row_ok, j == 0, masked, vis, m_ref, l_sum);
            }
            if (!ok) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->p_full[x]);
        }
        // ---- epilogue: O / l -> bf16 output, or unnormalised partials for the merge
        if (ok && ns > 0) ok = mbar_wait_warp(&sh->o_full, 0, sh, p);
        if (ok) {
            tc_fence_after();
            const size_t rows_total = (size_t)p.sum_nodes * p.Hq;
            const size_t row = (size_t)(n0 + node) * p.Hq + g * p.G + (row_ok ? R & (p.G - 1) : 0);
            const size_t part = (size_t)layer * p.n_splits + slice;
            const float unit = pow2(v_ref);     // of the accumulator
            const float inv = (l_sum > 0.f) ? unit / l_sum : 0.f;
            if (p.n_splits > 1 && row_ok) p.part_ml[part * rows_total + row] = make_float2(m_ref, l_sum);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t o[32];
                if (ns == 0) break;                         // (an empty slice: its l = 0 keeps the merge from reading more)
                tmem_ld32(o_taddr + c * 32, o);
                tmem_wait_ld();
                if (p.n_splits == 1) {
                    uint4 v[4];
                    pack_rows(o, inv, v);
                    transpose4(v, lane);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int Ri = R - lane + (lane & ~3) + i;
                        if (Ri < M) {
                            const size_t orow = (size_t)(n0 + (Ri >> p.g_shift)) * p.Hq + g * p.G + (Ri & (p.G - 1));
                            reinterpret_cast<uint4*>(p.out + ((size_t)layer * rows_total + orow) * kHeadDim + c * 32)[lane & 3] = v[i];
                        }
                    }
                } else if (row_ok) {
                    float4* po = p.part_o + (part * (kHeadDim / 4) + c * 8) * rows_total + row;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        po[i * rows_total] = make_float4(__uint_as_float(o[4 * i]) * unit, __uint_as_float(o[4 * i + 1]) * unit,
                                                         __uint_as_float(o[4 * i + 2]) * unit, __uint_as_float(o[4 * i + 3]) * unit);
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemColumns) : "memory");
    }
}

// ---- host side ------------------------------------------------------------------------------
static int row_tiles_for(int sum_nodes, int G) {
    const int n = sum_nodes < SAGE_MAX_NODES ? sum_nodes : SAGE_MAX_NODES;      // a tree has at most that many nodes
    return (n * G + kRowTile - 1) / kRowTile;
}
// Pages that a row tile reads at most.
static int most_pages(int max_pages, int window, int sink) {
    const long long w = ((long long)window - 1 + SAGE_MAX_NODES + kPageSize - 1) / kPageSize + 1 + ((long long)sink + kPageSize - 1) / kPageSize;
    return w < max_pages ? (int)w : max_pages;
}
// Slices of the context: two blocks are resident per SM; a wave of them takes what its pages take plus a fixed part (set-up,
// first copies, drain), worth about six pages, and every slice costs the merge a little.
static int pick_splits(int n_sms, int n_layers, int batch, int n_kv_heads, int G, int pages, int sum_nodes) {
    const int nodes = (sum_nodes + batch - 1) / batch;
    const long long base = (long long)n_layers * batch * n_kv_heads * row_tiles_for(nodes, G), slots = 2ll * n_sms;
    const int s_max = pages < split::kMaxSplits ? pages : split::kMaxSplits;
    int best = 1;
    double best_cost = 0.0;
    for (int s = 1; s <= s_max; ++s) {
        const long long waves = (base * s + slots - 1) / slots;
        if (s > 1 && waves > 6) break;
        const double cost = (double)waves * (6 + (pages + s - 1) / s) + (s > 1 ? 4.0 + 0.25 * s : 0.0);
        if (s == 1 || cost < best_cost - 1e-9) { best_cost = cost; best = s; }
    }
    return best;
}
static size_t workspace_size(int n_layers, int batch, int sum_nodes, int n_q_heads, int n_kv_heads, int pages) {
    const int S = pick_splits(resident_ctas(), n_layers, batch, n_kv_heads, n_q_heads / n_kv_heads, pages, sum_nodes);
    return S == 1 ? 16 : (size_t)n_layers * S * sum_nodes * n_q_heads * (kHeadDim + 2) * sizeof(float);
}
static bool sizes_ok(int n_layers, int batch, int sum_nodes, int n_q_heads, int n_kv_heads, int max_pages) {
    return n_layers >= 1 && batch >= 1 && sum_nodes >= 1 && n_q_heads >= 1 && n_kv_heads >= 1 && max_pages >= 1 && n_q_heads % n_kv_heads == 0;
}

struct Pools {
    const void *k, *v;
    int64_t layer_stride;       // elements
    int n_pages;
};
struct SealedPools {
    const void *k, *v;
    int64_t layer_stride;
    const uint8_t *k_exp, *v_exp;
    int n_pages;
    const int32_t* page_table;
    int max_pages;
    const int32_t* sealed;
};

static int run(const void* q, const Pools& pools, const SealedPools* s8, int n_layers, const int32_t* page_table, int max_pages,
               const int32_t* seq_len, const int32_t* parent, const int32_t* node_offsets, int batch, int sum_nodes, int n_q_heads,
               int n_kv_heads, int head_dim, int page_size, float sm_scale, int window, int sink, void* out, void* ws, size_t ws_bytes,
               int32_t* status, void* stream) {
    if (!q || !pools.k || !pools.v || !page_table || !seq_len || !parent || !node_offsets || !out) return SAGE_ERR_INVALID_ARG;
    if (n_layers < 1 || pools.n_pages < 1 || max_pages < 1 || batch < 0 || sum_nodes < 1 || n_q_heads < 1 || n_kv_heads < 1 ||
        pools.layer_stride < 0 || !(sm_scale > 0.f) || window < 1 || sink < 0)
        return SAGE_ERR_INVALID_ARG;
    if (head_dim != kHeadDim || page_size != kPageSize || n_q_heads % n_kv_heads) return SAGE_ERR_UNSUPPORTED;
    const int G = n_q_heads / n_kv_heads;
    if (G != 1 && G != 2 && G != 4 && G != 8) return SAGE_ERR_UNSUPPORTED;
    if (max_pages > (1 << 24)) return SAGE_ERR_UNSUPPORTED;
    if ((((uintptr_t)q | (uintptr_t)pools.k | (uintptr_t)pools.v | (uintptr_t)out) & 15) || (pools.layer_stride & 7)) return SAGE_ERR_INVALID_ARG;
    if (n_layers > 1 && pools.layer_stride < (int64_t)pools.n_pages * n_kv_heads * kPageSize * kHeadDim) return SAGE_ERR_INVALID_ARG;
    if (s8) {
        if (!s8->k || !s8->v || !s8->k_exp || !s8->v_exp || !s8->page_table || !s8->sealed) return SAGE_ERR_INVALID_ARG;
        if (s8->n_pages < 1 || s8->max_pages < 1 || s8->layer_stride < 0) return SAGE_ERR_INVALID_ARG;
        if (s8->max_pages > (1 << 24)) return SAGE_ERR_UNSUPPORTED;
        if ((((uintptr_t)s8->k | (uintptr_t)s8->v) & 15) || (s8->layer_stride & 15)) return SAGE_ERR_INVALID_ARG;
        if (n_layers > 1 && s8->layer_stride < (int64_t)s8->n_pages * n_kv_heads * kPageSize * kHeadDim) return SAGE_ERR_INVALID_ARG;
    }
    if (batch == 0) return SAGE_OK;
    // (no position lies beyond the page table: larger ones say the same)
    window = window < max_pages * kPageSize ? window : max_pages * kPageSize;
    sink = sink < max_pages * kPageSize ? sink : max_pages * kPageSize;
    const int pages = most_pages(max_pages, window, sink);
    const int S = pick_splits(resident_ctas(), n_layers, batch, n_kv_heads, G, pages, sum_nodes), tiles = row_tiles_for(sum_nodes, G);
    const double blocks = (double)n_layers * batch * n_kv_heads * tiles * S;
    if (blocks > 2147483647.0 || (S > 1 && n_layers > 65535)) return SAGE_ERR_UNSUPPORTED;
    if (!ws || ws_bytes < workspace_size(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, pages) || ((uintptr_t)ws & 15)) return SAGE_ERR_WORKSPACE;
    CUtensorMap qmap, kmap, vmap, k8map, v8map;
    if (!make_pool_map(&kmap, pools.k, n_layers, pools.n_pages, n_kv_heads, pools.layer_stride) ||
        !make_pool_map(&vmap, pools.v, n_layers, pools.n_pages, n_kv_heads, pools.layer_stride) ||
        !make_q_map(&qmap, q, n_layers, sum_nodes, n_kv_heads, G))
        return SAGE_ERR_CUDA;
    if (!s8) {
        k8map = kmap;           // (not used)
        v8map = vmap;
    } else if (!make_sealed_map(&k8map, s8->k, n_layers, s8->n_pages, n_kv_heads, s8->layer_stride) ||
               !make_sealed_map(&v8map, s8->v, n_layers, s8->n_pages, n_kv_heads, s8->layer_stride)) {
        return SAGE_ERR_CUDA;
    }
    Params p{};
    p.out = (__nv_bfloat16*)out;
    p.part_o = (float4*)ws;
    p.part_ml = S > 1 ? (float2*)((float*)ws + (size_t)n_layers * S * sum_nodes * n_q_heads * kHeadDim) : nullptr;
    p.page_table = page_table; p.seq_len = seq_len; p.parent = parent; p.node_offsets = node_offsets; p.status = status;
    if (s8) {
        p.page_table8 = s8->page_table; p.sealed = s8->sealed; p.k_exp = s8->k_exp; p.v_exp = s8->v_exp;
        p.n_pages8 = s8->n_pages; p.max_pages8 = s8->max_pages;
    }
    p.n_layers = n_layers; p.batch = batch; p.sum_nodes = sum_nodes; p.n_pages = pools.n_pages; p.max_pages = max_pages;
    p.Hq = n_q_heads; p.Hkv = n_kv_heads; p.G = G; p.g_shift = __builtin_ctz(G); p.n_splits = S; p.row_tiles = tiles;
    p.window = window; p.sink = sink;
    p.scale_log2 = sm_scale * 1.4426950408889634f;
    p.wait_cycles = attention_wait_cycles();
    p.producer_off = attention_producer_off();
    if (!allow_shared_memory<kSmemBytes>(tree_attention_paged_kernel) ||
        !succeeded(sage::launch(tree_attention_paged_kernel, dim3((unsigned)blocks), kThreads, kSmemBytes, as_stream(stream), 0, p, qmap, kmap, vmap,
                                k8map, v8map)))
        return SAGE_ERR_CUDA;
    if (S == 1) return SAGE_OK;
    return split::launch_merge(n_layers, node_offsets, batch, sum_nodes, n_q_heads, S, p.part_o, p.part_ml, out, true, as_stream(stream));
}

}  // namespace paged
}  // namespace sage

using namespace sage;

extern "C" size_t sage_tree_attention_window_workspace_size(int n_layers, int batch, int sum_nodes, int n_q_heads, int n_kv_heads,
                                                            int head_dim, int max_pages_per_seq, int window, int n_sink) {
    (void)head_dim;
    if (!paged::sizes_ok(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, max_pages_per_seq) || window < 1 || n_sink < 0) return 0;
    return paged::workspace_size(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, paged::most_pages(max_pages_per_seq, window, n_sink));
}

extern "C" size_t sage_tree_attention_sealed_workspace_size(int n_layers, int batch, int sum_nodes, int n_q_heads, int n_kv_heads,
                                                            int head_dim, int max_pages_per_seq) {
    (void)head_dim;
    if (!paged::sizes_ok(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, max_pages_per_seq)) return 0;
    return paged::workspace_size(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, max_pages_per_seq);
}

extern "C" int sage_tree_attention_window(const void* q, const void* k_pool, const void* v_pool, int64_t layer_stride_elems, int n_layers,
                                          int n_pages, const int32_t* page_table, int max_pages_per_seq, const int32_t* seq_len,
                                          const int32_t* parent, const int32_t* node_offsets, int batch, int sum_nodes, int n_q_heads,
                                          int n_kv_heads, int head_dim, int page_size, float sm_scale, int window, int n_sink, void* out,
                                          void* ws, size_t ws_bytes, int32_t* status, void* stream) {
    return paged::run(q, paged::Pools{k_pool, v_pool, layer_stride_elems, n_pages}, nullptr, n_layers, page_table, max_pages_per_seq, seq_len,
                      parent, node_offsets, batch, sum_nodes, n_q_heads, n_kv_heads, head_dim, page_size, sm_scale, window, n_sink, out, ws,
                      ws_bytes, status, stream);
}

extern "C" int sage_tree_attention_sealed(const void* q, const void* k_pool, const void* v_pool, int64_t layer_stride_elems, int n_layers,
                                          int n_pages, const int32_t* page_table, int max_pages_per_seq, const sage_sealed_cache* cache,
                                          const int32_t* sealed, const int32_t* seq_len, const int32_t* parent, const int32_t* node_offsets,
                                          int batch, int sum_nodes, int n_q_heads, int n_kv_heads, int head_dim, int page_size,
                                          float sm_scale, void* out, void* ws, size_t ws_bytes, int32_t* status, void* stream) {
    if (!cache) return SAGE_ERR_INVALID_ARG;
    const paged::SealedPools s8{cache->k, cache->v, cache->layer_stride, cache->k_exp, cache->v_exp, cache->n_pages, cache->page_table,
                                cache->max_pages_per_seq, sealed};
    return paged::run(q, paged::Pools{k_pool, v_pool, layer_stride_elems, n_pages}, &s8, n_layers, page_table, max_pages_per_seq, seq_len,
                      parent, node_offsets, batch, sum_nodes, n_q_heads, n_kv_heads, head_dim, page_size, sm_scale, 0x7fffffff, 0, out, ws,
                      ws_bytes, status, stream);
}
