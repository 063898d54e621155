// Tree attention over part of a cache or over a cache in two forms, sm_100a:
//   sage_tree_attention_window : the last `window` positions and the first `sink` ones of a bf16 cache
//   sage_tree_attention_sealed : every position; full pages are e4m3 with a power-of-two scale for each page and KV head
//                                (see seal_kv.cu), the rest (the page that is not full, the tree's rows) is bf16
// For query row i (a node and one of the G query heads that share a KV head), out = sum_t p_t V[t] / sum_t p_t with
// p_t = exp(sm_scale q K[t]), t over what the row sees.
//
// A block owns one tile of 128 query rows and one slice of the pages that its item (layer, sequence, KV head) has to
// read; two blocks are resident on an SM (113 KB of shared memory, 256 columns of tensor memory each), so that one's chain
// scores -> softmax -> P V runs while the other's waits.  The pages to read are counted without the gap between sinks and
// window (Walk); the sealed ones come first in that order, and a block walks it backwards: bf16 pages, then sealed ones.
//   TMA     : query rows; K and V pages -> 128B-swizzled shared memory, a ring of five 16 KB slots: a bf16 page takes two
//             (K, V), a sealed one takes one for both
//   tcgen05 : S = Q K^T (128 x 64 fp32, two buffers), O += P V with P as the TMEM operand, V MN-major
//   softmax : one thread per row, online, fp32, log2 domain
// What is sealed is multiplied as it is, in kind::f8f6f4, without a way through registers and back: each bf16 query row is
// the sum of two e4m3 rows (split_queries: exact down to 2^-9 of the row's largest element, off by 2^-17 of it below), and each
// probability the sum of three e5m2 numbers (split_three: with the rounding to fp16 ahead of it off by less than 2^-8 of its value, which is what bf16 has, for
// values from 2^-8 on against a reference that lies 2^10 or more below the row's maximum, and by 2^-17 below).  An e4m3 and an e5m2 number, one product less, have
// 2^-7.9 near the maximum, but 2^-3 from 2^-13 of it on: 2 to 5 % of an output whose row has a key 9 to 11 ahead of thousands (80 layers x 16k x 9 nodes, in
// bursts, 670 us with two terms, 740 with three; one layer, 60 nodes 47 / 49).  Two e5m2 numbers (662 us) would be off by 2^-7, 2.5e-3 in the mean of squares, where three have
// 0.5e-3 and bf16 1.7e-3.
// Two products of 8 bits cost the tensor pipe what one of 16 does: the scores cost the same as those of bf16 keys, P V half as much again, and HBM half.
// The scales are powers of two: the key's goes into the row's factor of the scores, the value's into the exponent of the
// probabilities (against the largest of the pages so far, `v_ref`, to which the accumulator is scaled).
// All waits are bounded: on expiry the block records SAGE_STATUS_TIMEOUT, drains its copies and MMAs, frees its TMEM and returns.
//
// What bounds it.  One row tile: HBM and, in long launches, the board's power limit (28 layers x 4 sequences, window of 4096: 305 us in a burst, the copy
// rate; 80 layers x 16k x 9 nodes sealed: 740 to 780 us in a burst, 885 in a loop, where 415 us of traffic are the floor).  More row tiles: the chain
// of a page, scores, probabilities, product, which the SM's other block fills in part: 1 150 clocks a page and tile, of which the tensor pipe works 640 for a sealed one
// (256 for the scores, 128 for each term of P V) and 512 for a bf16 one (one layer, 60 nodes, 16k keys: 49 us, tensor pipe at 47 %).  Short launches: some 4 000 clocks before
// the first scores (offsets, page ids, pages, query rows), 1 150 to 1 650 a page, 5 000 for partial results and merge (one token at 2k keys 11.2 us).
// Tried and slower: steps of 128 keys in one S buffer (the softmax waits 2 000 clocks a step for the products of its own block; 80 layers 735 us where
// pages took 690); a maximum in every page (2 300 clocks a page instead of 1 100 to 1 500); one exponential pair in eight or four on the FMA pipe (+0.5, +3 %).
#include <cuda_fp16.h>

#include "attention_stream.cuh"
#include "paged.cuh"

namespace sage {
namespace paged {

using namespace stream;

constexpr int kSlots = 5;                                   // ring of 16 KB slots
constexpr int kSlotBytes = kPageSize * kHeadDim * 2;        // a bf16 K or V page of a head, or both of a sealed one
constexpr int kSealedBytes = kPageSize * kHeadDim;          // a sealed K or V page of a head
constexpr int kMostSplits = 32, kMostInCluster = 16;        // slices of an item; as one cluster
constexpr int kThreads = 256;                               // a softmax warpgroup; the TMA warp, the MMA warp and two idle ones
constexpr int kTmemColumns = 256;                           // S 2 x 64, O 128
constexpr uint32_t kIdescPage = idesc_f16(kPageSize);       // S = Q K^T, bf16
// kind::f8f6f4: D fp32, M = 128; types of A: 0 e4m3, 1 e5m2; B e4m3
constexpr uint32_t idesc_f8(uint32_t n, uint32_t a_type) { return (1u << 4) | (a_type << 7) | ((n >> 3) << 17) | ((128u >> 4) << 24); }
constexpr uint32_t kIdescSealedQK = idesc_f8(kPageSize, 0);
constexpr uint32_t kIdescSealedPV = idesc_f8(kHeadDim, 1) | (1u << 16);         // B (= V) MN-major
// Probabilities are taken against a reference 2^headroom below the maximum that set it, and may reach 2^15.999 (fp16's largest): a
// row's maximum may grow by 2^(15.9 - headroom) before the accumulator is scaled again.  At first, when most of the growth is still to come, a headroom
// of 10 (a page's maximum may lie 4 below the row's in the scores), later 12: a row's largest probability is at least 2^10, and what
// the formats keep of small ones is counted from there.
constexpr float kHeadroomFirst = 10.f, kHeadroom = 12.f, kMostLog2 = 15.9f;
constexpr uint32_t kMostF16 = 0x7bff;       // fp16's largest number
constexpr float kMostSum = 4096.f * kMaxSum;    // bf16 pages: what the probabilities of a page may sum to (kMaxSum is against the maximum itself)
constexpr long long kDrainCycles = 4000000000ll;    // for what is in flight when a wait has run out (whatever the waits' own budget)
constexpr int kTerms = 3;                   // e5m2 numbers that a probability over sealed pages is the sum of
template <bool kSealed>
constexpr int kWords = kSealed ? 8 * kTerms : 16;   // of the probabilities of 32 keys: 8 for each term; bf16 16
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
    int issued;                // slots that copies have been asked for (-1: nor the query rows)
    int parent[SAGE_MAX_NODES];
};
constexpr int kSmemBytes = kQTileBytes + kSlots * kSlotBytes + 1024;
static_assert(sizeof(Shared) <= 1024 && 2 * (kSmemBytes + 1024) <= 233472, "two blocks have to fit on an SM");

// mbar_wait_warp with its loop apart: a dozen waits in line are a fifth of the kernel's code, and what the warps of an SM run at the same time has to
// fit its instruction caches.
static __device__ __noinline__ bool wait_longer(uint64_t* bar, uint32_t parity, Shared* sh, long long wait_cycles, int32_t* status) {
    struct Limits { long long wait_cycles; int32_t* status; };
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, sh, Limits{wait_cycles, status}));
}
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, Shared* sh, const Params& p) {
    if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
    return wait_longer(bar, parity, sh, p.wait_cycles, p.status);
}

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

// Four fp16 numbers (two words) as a word of e4m3 and one of what is left over, in e4m3 too.  (The first word is put together
// before it is read again: with the 16-bit halves used for both, the compiler of CUDA 12.9 subtracts the wrong one.)
__device__ __forceinline__ void split_four(uint32_t x0, uint32_t x1, uint32_t& high, uint32_t& low) {
    uint32_t b0, b1;
    asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e4m3x2.f16x2 a, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 b, %2;\n\tmov.b32 %0, {a, b};\n\t}"
        : "=r"(high) : "r"(x0), "r"(x1));
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=&r"(b0), "=r"(b1) : "r"(high));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(b0) : "r"(x0), "r"(b0));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(b1) : "r"(x1), "r"(b1));
    asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e4m3x2.f16x2 a, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 b, %2;\n\tmov.b32 %0, {a, b};\n\t}"
        : "=r"(low) : "r"(b0), "r"(b1));
}
// Four fp16 numbers that are not negative (two words) as the sum of three e5m2 numbers each.  e5m2 is the upper byte of an fp16 number, so the first term is that
// byte, the second that of what is left over (both differences are exact), the third the nearest e5m2 number to the rest: three
// significant bits twice, and then half a step of three more, 2^-9 of the number's binade.  Steps stop at 2^-16: 2^-17 for numbers below 2^-8.
__device__ __forceinline__ void split_three(uint32_t x0, uint32_t x1, uint32_t& first, uint32_t& second, uint32_t& third) {
    first = __byte_perm(x0, x1, 0x7531);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(x0) : "r"(x0), "r"(x0 & 0xff00ff00u));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(x1) : "r"(x1), "r"(x1 & 0xff00ff00u));
    second = __byte_perm(x0, x1, 0x7531);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(x0) : "r"(x0), "r"(x0 & 0xff00ff00u));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(x1) : "r"(x1), "r"(x1 & 0xff00ff00u));
    asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e5m2x2.f16x2 a, %1;\n\tcvt.rn.satfinite.e5m2x2.f16x2 b, %2;\n\tmov.b32 %0, {a, b};\n\t}"
        : "=r"(third) : "r"(x0), "r"(x1));
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
    int n_sealed;   // of all that are read (with sealed pages the window takes nothing away); the others follow
    int n;          // pages
    __device__ __forceinline__ int page(int w) const { return w < n_sink ? w : w - n_sink + w0; }
};
__device__ __forceinline__ Walk make_walk(int L, int N, int sealed, int window, int sink) {
    Walk k;
    k.w0 = max(0, L - window + 1) / kPageSize;              // the root sees furthest back
    k.n_sink = min((sink + kPageSize - 1) / kPageSize, k.w0);
    k.n_sealed = sealed;
    k.n = k.n_sink + (L + N + kPageSize - 1) / kPageSize - k.w0;
    return k;
}

// What is wrong with a sequence; 0: nothing.  One with an error is left out, by the merge too.
__device__ __forceinline__ int sequence_error(const Params& p, int n0, int N, int L, int sealed) {
    if (N < 1 || N > SAGE_MAX_NODES || n0 < 0 || n0 > p.sum_nodes - N) return SAGE_STATUS_BAD_TREE;
    if (L < 0 || (long long)L + N > (long long)p.max_pages * kPageSize || sealed < 0 || sealed > L / kPageSize || sealed > p.max_pages8)
        return SAGE_STATUS_BAD_PAGE;
    return 0;
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

// exp2(s * scale + base) of 32 columns.  Probabilities for the products in kWords words at pk (sealed: 8 of
// each term, see split_three; else bf16), their fp32 sums in acc, sealed: the largest so far, as
// fp16 bits, in either half of `most`.
template <bool kSealed>
__device__ __forceinline__ void exp_pack(const uint32_t* sr, float scale, float base, uint32_t* pk, uint64_t (&acc)[2], uint32_t& most) {
    if constexpr (!kSealed) {
        exp_chunk<0>(sr, scale, base, pk, acc);
    } else {
        const uint64_t scale2 = f2_pack(scale, scale), base2 = f2_pack(base, base);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint64_t x2[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x2[i] = f2_fma(f2_pack(__uint_as_float(sr[16 * h + 2 * i]), __uint_as_float(sr[16 * h + 2 * i + 1])), scale2, base2);
            uint32_t f16[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float x0, x1;
                f2_unpack(x2[i], x0, x1);
                x0 = fast_exp2(x0);
                x1 = fast_exp2(x1);
                x2[i] = f2_pack(x0, x1);
                f16[i] = pack_f16(x0, x1);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i & 1] = f2_add(acc[i & 1], x2[i]);
#pragma unroll
            for (int i = 0; i < 8; i += 2) most = __vimax3_u16x2(most, f16[i], f16[i + 1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) split_three(f16[2 * i], f16[2 * i + 1], pk[4 * h + i], pk[8 + 4 * h + i], pk[16 + 4 * h + i]);
        }
    }
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
template <bool kSealed>
__device__ __forceinline__ void tmem_st_words(uint32_t taddr, const uint32_t* r) {
    tmem_st16(taddr, r);
    if constexpr (kSealed)
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     ::"r"(taddr + 16), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]) : "memory");
}

// A page for one query row per thread: 64 scores -> probabilities over the first 16 columns of each 32, running reference m
// and sum l.  scale: of the scores; dv: exponent by which the page's values exceed the accumulator's.
//
// A page that needs care: the first one, one with keys out of sight (bf16: a sealed page lies within the prefix, and that call has no window), one whose values have a larger scale than those so far (o_factor: what the
// accumulator is to be multiplied by), one whose probabilities outgrew the reference.  Goes through the maximum.
struct Running { float m, l; };
template <bool kSealed>
static __device__ __noinline__ Running careful_page(const Params& p, Shared* sh, int pv_parity, uint32_t s_taddr, uint32_t o_taddr, float scale, int dv,
                                                    float o_factor, bool row_ok, bool first, float headroom, uint64_t vis, float m, float l) {
    uint32_t sr[2][32];
    tmem_ld32(s_taddr, sr[0]);
    tmem_ld32(s_taddr + 32, sr[1]);
    tmem_wait_ld();
    if (!kSealed && __any_sync(0xffffffffu, vis != ~0ull)) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if (!((uint32_t)vis & (1u << i))) sr[0][i] = 0xff800000u;      // -inf
            if (!((uint32_t)(vis >> 32) & (1u << i))) sr[1][i] = 0xff800000u;
        }
    }
    float mx = -INFINITY;
    max_chunk(sr[0], mx);
    max_chunk(sr[1], mx);
    const float m_cand = mx * scale;
    // (where one row of the warp has to move its reference, all those move that have found a larger score: they would be next)
    const bool move = __any_sync(0xffffffffu, row_ok && m_cand > m + kMostLog2);
    const bool grow = move && m_cand > m + headroom;
    float alpha = 1.f;
    if (grow) {
        alpha = fast_exp2(m - (m_cand - headroom));         // 0 when m was -inf
        m = m_cand - headroom;
    }
    if (!first && (move || o_factor != 1.f)) {
        // O *= alpha, once the P V product of the page before has finished (a wait that runs out ends the block at its next one)
        mbar_wait_warp(&sh->pv_done, pv_parity, sh, p);
        tc_fence_after();
        rescale_o_rows(o_taddr, alpha * o_factor);
    }
    const float base = (m == -INFINITY ? 0.f : -m) + (float)dv;
    uint64_t acc[2] = {};
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        uint32_t pk[kWords<kSealed>];
        exp_pack<kSealed>(sr[c], scale, base, pk, acc, most);      // may hold -inf
        tmem_st_words<kSealed>(s_taddr + 32 * c, pk);
    }
    float sum_a, sum_b;
    f2_unpack(f2_add(acc[0], acc[1]), sum_a, sum_b);
    tmem_wait_st();
    tc_fence_before();
    return Running{m, l * alpha + (sum_a + sum_b) * pow2(-dv)};
}

// Any other page: probabilities are taken against the reference of the pages before, and it shows in them whether it still serves (sealed:
// none above what fp16 holds; bf16: by their sum, see kMaxSum).  Returns false, with the scores as they were, where it does not.
template <bool kSealed>
__device__ __forceinline__ bool plain_page(uint32_t s_taddr, float scale, int dv, bool row_ok, float m, float& l) {
    uint32_t sa[32], sb[32], pa[kWords<kSealed>], pb[kWords<kSealed>], most = 0;
    uint64_t acc[2] = {};
    tmem_ld32(s_taddr, sa);
    tmem_wait_ld_of(sa);
    tmem_ld32(s_taddr + 32, sb);
    const float base = (float)dv - m;
    exp_pack<kSealed>(sa, scale, base, pa, acc, most);
    tmem_wait_ld_of(sb);
    exp_pack<kSealed>(sb, scale, base, pb, acc, most);
    float sum_a, sum_b;
    f2_unpack(f2_add(acc[0], acc[1]), sum_a, sum_b);
    const float sum = (sum_a + sum_b) * pow2(-dv);
    const bool outgrown = kSealed ? max(most & 0xffffu, most >> 16) > kMostF16 : !(sum < kMostSum);
    if (__any_sync(0xffffffffu, row_ok && outgrown)) return false;
    l += sum;
    tmem_st_words<kSealed>(s_taddr, pa);
    tmem_st_words<kSealed>(s_taddr + 32, pb);
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
            split_four(pack_f16(__uint_as_float(a << 16) * up, __uint_as_float(a & 0xffff0000u) * up),
                              pack_f16(__uint_as_float(b << 16) * up, __uint_as_float(b & 0xffff0000u) * up), h[k], l[k]);
        }
        uint8_t* at = sQ + r * 128 + ((c ^ (r & 7)) << 4);
        *reinterpret_cast<uint4*>(at) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(at + kQHalfBytes) = make_uint4(l[0], l[1], l[2], l[3]);
    }
    return __uint_as_float((uint32_t)(exponent - 7) << 23);
}

// ---- slices of a row tile as one cluster: partial results stay in shared memory, where the pages were -------------------
// [128 rows][32 column quads, padded to 33: rows of neighbouring lanes in different banks], then (reference, sum) of each row
__device__ __forceinline__ float4& part_o(uint8_t* smem, int r, int quad) { return reinterpret_cast<float4*>(smem)[r * 33 + quad]; }
__device__ __forceinline__ float2& part_ml(uint8_t* smem, int r) { return reinterpret_cast<float2*>(smem + kRowTile * 33 * 16)[r]; }
static_assert(kRowTile * (33 * 16 + 8) <= kQTileBytes + kSlots * kSlotBytes, "partial results have to fit where queries and pages were");
__device__ __forceinline__ void cluster_sync() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// its two halves, each by a whole warp
__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t of_block(uint32_t saddr, int rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(saddr), "r"(rank));
    return a;
}
// Each block merges an equal part of the tile's rows x 32 column quads, read from all blocks' shared memory, one output a thread at a time.  A warp
// lets the others go (they may not leave before their memory has been read) as soon as it has its last values.  (As a launch of its own behind the
// slices, the merge costs some 2.5 us more for few rows, and no more for 128.  The code is run once and cold, so it is kept short: unrolled
// for sixteen slices, or several outputs at a time, it is slower by up to a microsecond where there are few rows.)
__device__ __forceinline__ void merge_in_cluster(const Params& p, uint8_t* smem, int layer, int g, int n0, int row0, int rows, int rank, int tid) {
    constexpr int kAhead = 8;
    const int S = p.n_splits, total = rows * 32, end = total * (rank + 1) / S;
    // (the same number of turns for all lanes of a warp, which arrives as a whole)
    int left = (end - (total * rank / S + (tid & ~31)) + kRowTile - 1) / kRowTile;
    if (left <= 0) cluster_arrive();
    for (int at = total * rank / S + tid; left > 0; at += kRowTile, --left) {
        const int e = min(at, end - 1), r = e >> 5, quad = e & 31;
        const uint32_t at_o = smem_u32(&part_o(smem, r, quad)), at_ml = smem_u32(&part_ml(smem, r));
        float m = -INFINITY, l = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int s0 = 0; s0 < S; s0 += kAhead) {
            float2 ml[kAhead];
            float4 v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                ml[u] = make_float2(-INFINITY, 0.f);
                if (s0 + u < S) {
                    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(ml[u].x), "=f"(ml[u].y) : "r"(of_block(at_ml, s0 + u)));
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                 : "=f"(v[u].x), "=f"(v[u].y), "=f"(v[u].z), "=f"(v[u].w) : "r"(of_block(at_o, s0 + u)) : "memory");
                }
            }
            float top = m;
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (ml[u].y > 0.f) top = fmaxf(top, ml[u].x);
            if (s0 + kAhead >= S && left == 1) cluster_arrive();
            const float old = top == -INFINITY ? 0.f : fast_exp2(m - top);
            m = top;
            l *= old;
            acc.x *= old; acc.y *= old; acc.z *= old; acc.w *= old;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const float w = ml[u].y > 0.f ? fast_exp2(ml[u].x - top) : 0.f;
                l = fmaf(ml[u].y, w, l);                    // (NaN stays NaN)
                if (w > 0.f) {                              // (else an empty slice, or one that holds nothing for the row)
                    acc.x = fmaf(w, v[u].x, acc.x); acc.y = fmaf(w, v[u].y, acc.y);
                    acc.z = fmaf(w, v[u].z, acc.z); acc.w = fmaf(w, v[u].w, acc.w);
                }
            }
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int R = row0 + r;
        const size_t row = (size_t)(n0 + (R >> p.g_shift)) * p.Hq + g * p.G + (R & (p.G - 1));
        if (at < end)
            *reinterpret_cast<uint2*>(p.out + ((size_t)layer * p.sum_nodes * p.Hq + row) * kHeadDim + quad * 4) =
                make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    }
    cluster_wait();
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
    // Which item, row tile and slice: the first items are worked on whole, the others in slices; or all in slices, those of a row tile
    // side by side as one cluster.
    int rtile, n_slices, slice, item;
    if (p.in_cluster) {
        n_slices = p.n_splits;
        slice = blockIdx.x % p.n_splits;
        rtile = blockIdx.x / p.n_splits % p.row_tiles;
        item = blockIdx.x / (p.n_splits * p.row_tiles);
    } else {
        const int unit = blockIdx.x / p.row_tiles;
        rtile = blockIdx.x % p.row_tiles;
        n_slices = unit < p.n_whole ? 1 : p.n_splits;
        slice = unit < p.n_whole ? 0 : (unit - p.n_whole) % p.n_splits;
        item = unit < p.n_whole ? unit : p.n_whole + (unit - p.n_whole) / p.n_splits;
    }
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
    const int error = sequence_error(p, n0, N, L, sealed);
    const int T = L + N, M = N * p.G, row0 = rtile * kRowTile;
    if (error) {                                            // uniform
        if (tid == 0) report_status(p.status, error);
        return;
    }
    if (row0 >= M) return;
    // this block's slice [w_lo, w_hi) of the pages to read; it walks them from the last to the first
    const Walk walk = make_walk(L, N, sealed, p.window, p.sink);
    const int per_slice = (walk.n + n_slices - 1) / n_slices;
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
        sh->issued = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem_base;
    // ring positions of a page: a bf16 page takes two slots in a row, a sealed one takes one
    auto k_seq = [&](int j) { return j < nb ? 2 * j : nb + j; };
    auto v_seq = [&](int j) { return j < nb ? 2 * j + 1 : nb + j; };

    // Registers move to the softmax warps: 128 + 128 a thread become 192 + 64.
    if (warp >= 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 4) {
            // =========================== TMA producer ===========================
            // page ids of 32 pages at a time, one per lane
            auto look_up = [&](int j) {
                if (j >= ns) return 0;
                const bool is8 = j >= nb;
                const int pg = walk.page(w_hi - 1 - j);
                int id = is8 ? p.page_table8[(size_t)b * p.max_pages8 + pg] : p.page_table[(size_t)b * p.max_pages + pg];
                if (id < 0 || id >= (is8 ? p.n_pages8 : p.n_pages)) {           // (checked: it becomes a TMA coordinate)
                    report_status(p.status, SAGE_STATUS_BAD_PAGE);
                    id = 0;
                }
                return id;
            };
            const bool on = ns > 0 && !p.producer_off;
            int issued = 0;
            if (on) {
                if (lane == 0) {
                    mbar_expect_tx(&sh->q_ready, kQTileBytes);
                    for (int h = 0; h < 2; ++h)
                        tma_load_5d(smem_u32(sQ + h * kQHalfBytes), &qmap, h * 64, 0, g, n0 + (row0 >> p.g_shift), layer, &sh->q_ready);
                }
                int now = look_up(lane);
                bool ok = true;
                for (int j0 = 0; ok && j0 < ns; j0 += 32) {
                    const int next = look_up(j0 + 32 + lane);
                    const int n = min(32, ns - j0);
                    for (int i = 0; ok && i < n; ++i) {
                        const bool is8 = j0 + i >= nb;
                        const int id = __shfl_sync(0xffffffffu, now, i);
                        const int c2 = id * p.Hkv + g;
                        for (int part = 0; part < (is8 ? 1 : 2); ++part) {
                            const int s = issued % kSlots, use = issued / kSlots;
                            if (use > 0) ok = wait_warp(&sh->empty[s], (use - 1) & 1, sh, p);
                            if (!ok) break;
                            if (lane == 0) {
                                uint8_t* dst = sRing + s * kSlotBytes;
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
                if (lane == 0) sh->issued = issued;
                __syncwarp();
            }
        } else if (warp == 5) {
            // =========================== MMA issuer ===========================
            const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
            const int n = __shfl_sync(0xffffffffu, ns, 0);
            const uint32_t leader = elect_one() ? 1u : 0u;
            auto wait_all = [&](uint64_t* bar, uint32_t parity) { return wait_warp(bar, parity, sh, p); };
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
                        mma_ts<kDescHi, kIdescPV>(leader, o_tmem, a + 32 * (ks >> 1) + 8 * (ks & 1), dv + ((ks * 2048) >> 4), ks > 0 ? 1u : acc);
                } else {
                    const uint32_t dv = dring_mn + ((s * kSlotBytes + kSealedBytes) >> 4);
#pragma unroll
                    for (int ks = 0; ks < 2 * kTerms; ++ks)     // 32 keys; one term of their probabilities after the other
                        mma_ts_f8<kDescHi, kIdescSealedPV>(leader, o_tmem, a + (ks & 1) * 32 + (ks >> 1) * 8, dv + (((ks & 1) * 4096) >> 4),
                                                           ks > 0 ? 1u : acc);
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
            // (Keys of page j + 2 are waited for behind the product of page j: a bf16 page's slot is free only once the values of page j - 1 have been read, and a
            // wait for page j + 3 ahead of the probabilities of page j + 1 held those up by a copy's latency.)
            if (ok) ok = values_ready(0);
            for (int j = 0; ok && j < n; ++j) {
                ok = wait_all(&sh->p_full[j & 1], (j >> 1) & 1);
                if (!ok) break;
                tc_fence_after();
                issue_pv(j);
                if (j + 2 < n) {                                // reuses this page's S buffer: in pipe order behind its P V
                    ok = keys_ready(j + 2);
                    if (!ok) break;
                    tc_fence_after();
                    issue_qk(j + 2);
                }
                ok = values_ready(j + 1);
            }
            tc_commit(leader, &sh->o_full);                     // arrives when every MMA has completed
            __syncwarp();
        }
        if (p.in_cluster) {
            cluster_sync();
            cluster_sync();
        }
    } else {
        // =========================== softmax ===========================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        const int r = tid;                                  // row inside the tile == TMEM lane
        const uint32_t lane_base = (uint32_t)(warp * 32) << 16;
        const uint32_t s_taddr = tmem + lane_base, o_taddr = tmem + lane_base + 128;
        const int R = row0 + r;
        const bool row_ok = R < M, warp_live = row0 + warp * 32 < M;
        const int node = row_ok ? R >> p.g_shift : 0;
        const int cut = L + N - p.window;                   // some row does not see the prefix positions in front of this one
        Sight sight{1ull << node, p.sink, 0};
        // scales of 32 sealed pages at a time, one pair of exponent bytes per lane
        auto sealed_id = [&](int i) { return nb + i < ns ? p.page_table8[(size_t)b * p.max_pages8 + walk.page(w_hi - 1 - nb - i)] : 0; };
        struct Raw { uint32_t k, v; };                      // (as they come: packed and limited only once they are needed)
        auto scales_of = [&](int i, int id) {
            Raw e{127u, 127u};
            if (nb + i < ns) {
                if (id < 0 || id >= p.n_pages8) id = 0;     // (reported by the copy warp)
                const size_t at = ((size_t)layer * p.n_pages8 + id) * p.Hkv + g;
                e.k = p.k_exp[at];
                e.v = p.v_exp[at];
            }
            return e;
        };
        auto packed = [](const Raw& e) { return min(max(e.k, (uint32_t)kExpLo), (uint32_t)kExpHi) | (min(max(e.v, (uint32_t)kExpLo), (uint32_t)kExpHi) << 8); };
        const bool tree = nb > 0;                           // some page may be masked
        const int first_id = sealed_id(lane), next_id = sealed_id(32 + lane);      // (asked for at once: the set-up is a chain of loads)
        if (tree && r < N) sh->parent[r] = p.parent[n0 + r];
        const Raw first_scales = scales_of(lane, first_id);
        Raw next_scales = scales_of(32 + lane, next_id);
        uint32_t scales = 0;
        if (tree) {
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
        float m_ref = row_ok ? -INFINITY : INFINITY, l_sum = 0.f;     // (rows that are not the tree's: probabilities of zero, which cost the tensor cores less power)
        float row_scale = 0.f;                              // for sealed pages
        int v_ref = 0;                                      // exponent of the accumulator: at first that of the first sealed page, if there is one
        bool ok = warp_live;
        auto split = [&]() {                                // the query rows change their form
            row_scale = split_queries(sQ, r) * p.scale_log2;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->q_split);
            __syncwarp();
        };
        if (ok && ns > 0 && nb == 0) {
            ok = mbar_wait_warp(&sh->q_ready, 0, sh, p);
            if (ok) split();
        }
        if (ok && nb < ns) {
            scales = packed(first_scales);
            v_ref = (int)(__shfl_sync(0xffffffffu, scales, 0) >> 8) - 127;
        }
        for (int j = 0; ok && j < nb; ++j) {                // bf16 pages
            const int x = j & 1;
            ok = mbar_wait_warp(&sh->s_full[x], (j >> 1) & 1, sh, p);
            if (!ok) break;
            tc_fence_after();
            if (j == nb - 1 && nb < ns) split();            // (the last bf16 scores are there)
            const int t0 = walk.page(w_hi - 1 - j) * kPageSize;
            const bool masked = t0 + kPageSize > L || (t0 < cut && t0 + kPageSize > p.sink);
            if (j == 0 || masked || !plain_page<false>(s_taddr + x * 64, p.scale_log2, -v_ref, row_ok, m_ref, l_sum)) {
                const float room = j < 2 ? kHeadroomFirst : kHeadroom;
                const Running u = careful_page<false>(p, sh, (j - 1) & 1, s_taddr + x * 64, o_taddr, p.scale_log2, -v_ref, 1.f, row_ok, j == 0, room,
                                                      masked ? visible_page(sight, t0, L) : ~0ull, m_ref, l_sum);
                m_ref = u.m;
                l_sum = u.l;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->p_full[x]);
        }
        for (int j = nb; ok && j < ns; ++j) {               // sealed pages
            const int x = j & 1, i = j - nb;
            ok = mbar_wait_warp(&sh->s_full[x], (j >> 1) & 1, sh, p);
            if (!ok) break;
            tc_fence_after();
            if (i > 0 && i % 32 == 0) {
                scales = packed(next_scales);
                next_scales = scales_of(i + 32 + lane, sealed_id(i + 32 + lane));
            }
            const uint32_t e = __shfl_sync(0xffffffffu, scales, i & 31);
            const int ve = (int)(e >> 8) - 127;
            const float scale = row_scale * __uint_as_float((e & 0xffu) << 23);
            if (j == 0 || ve > v_ref || !plain_page<true>(s_taddr + x * 64, scale, ve - v_ref, row_ok, m_ref, l_sum)) {
                const int v_max = max(v_ref, ve);
                const float room = j < 2 ? kHeadroomFirst : kHeadroom;
                const Running u = careful_page<true>(p, sh, (j - 1) & 1, s_taddr + x * 64, o_taddr, scale, ve - v_max, pow2(v_ref - v_max), row_ok, j == 0, room,
                                                     ~0ull, m_ref, l_sum);
                v_ref = v_max;
                m_ref = u.m;
                l_sum = u.l;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->p_full[x]);
        }
        // ---- epilogue: O / l -> bf16 output, or unnormalised partials for the merge
        if (ok && ns > 0) ok = mbar_wait_warp(&sh->o_full, 0, sh, p);
        if (ok) {
            tc_fence_after();
            const size_t rows_total = (size_t)p.sum_nodes * p.Hq;
            const size_t rows = (size_t)p.row_tiles * kRowTile;       // of an item in the workspace
            const size_t part = (size_t)(item - p.n_whole) * p.n_splits + slice;
            const float o_unit = pow2(v_ref);   // of the accumulator
            const float inv = (l_sum > 0.f) ? o_unit / l_sum : 0.f;
            if (p.in_cluster) part_ml(smem, r) = make_float2(m_ref, l_sum);
            else if (n_slices > 1 && row_ok) p.part_ml[part * rows + R] = make_float2(m_ref, l_sum);
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                uint32_t o[32];
                if (ns == 0) break;                         // (an empty slice: its l = 0 keeps the merge from reading more)
                tmem_ld32(o_taddr + c * 32, o);
                tmem_wait_ld();
                if (n_slices == 1) {
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
                } else if (p.in_cluster) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        part_o(smem, r, c * 8 + i) = make_float4(__uint_as_float(o[4 * i]) * o_unit, __uint_as_float(o[4 * i + 1]) * o_unit,
                                                                 __uint_as_float(o[4 * i + 2]) * o_unit, __uint_as_float(o[4 * i + 3]) * o_unit);
                } else if (row_ok) {
                    float4* po = p.part_o + (part * (kHeadDim / 4) + c * 8) * rows + R;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        po[i * rows] = make_float4(__uint_as_float(o[4 * i]) * o_unit, __uint_as_float(o[4 * i + 1]) * o_unit,
                                                   __uint_as_float(o[4 * i + 2]) * o_unit, __uint_as_float(o[4 * i + 3]) * o_unit);
                }
            }
        }
        if (p.in_cluster) {
            cluster_sync();                                 // (every block of the cluster comes here, whatever its waits came to)
            merge_in_cluster(p, smem, layer, g, n0, row0, min(kRowTile, M - row0), slice, r);
            __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (sh->abort) {
        // Whichever wait ran out: every copy has to land, and every MMA to retire, before the tiles and the tensor memory go away.
        if (tid == 0) {
            for (int n = max(0, sh->issued - kSlots); n < sh->issued; ++n)
                mbar_wait_quiet(&sh->full[n % kSlots], (n / kSlots) & 1, kDrainCycles);
            if (sh->issued >= 0) mbar_wait_quiet(&sh->q_ready, 0, kDrainCycles);
            mbar_wait_quiet(&sh->o_full, 0, kDrainCycles);
        }
        __syncthreads();
    }
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemColumns) : "memory");
    }
}

// Merge of the items that were worked on in slices.  A block owns 32 rows of an item (one per lane) and 32 of the 128 columns (four per
// warp): enough warps to keep the loads of a few hundred rows in flight on the whole chip.  The weights of the slices are shared among
// the warps; the first partial results are asked for before they are known.
__global__ void __launch_bounds__(256) paged_merge_kernel(const Params p) {
    after_previous_kernel();
    constexpr int kAhead = 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, S = p.n_splits, quad = blockIdx.z * 8 + warp;
    const int item = p.n_whole + blockIdx.y, g = item % p.Hkv, b = item / p.Hkv % p.batch, layer = item / (p.Hkv * p.batch);
    const int n0 = p.node_offsets[b], N = p.node_offsets[b + 1] - n0, M = N * p.G;
    if (sequence_error(p, n0, N, p.seq_len[b], p.sealed ? p.sealed[b] : 0) || blockIdx.x * 32 >= M) return;      // (not worked on)
    const int R = blockIdx.x * 32 + lane;
    const bool ok = R < M;
    const size_t rows = (size_t)p.row_tiles * kRowTile, r = ok ? R : blockIdx.x * 32;
    const float2* ml = p.part_ml + (size_t)blockIdx.y * S * rows + r;
    const float4* po = p.part_o + ((size_t)blockIdx.y * S * (kHeadDim / 4) + quad) * rows + r;
    const size_t slice = (kHeadDim / 4) * rows;
    __shared__ float s_m[kMostSplits][32], s_l[kMostSplits][32], s_w[kMostSplits][32];
    float4 v[kAhead];
    for (int s = warp; s < S; s += 8) {
        const float2 x = ml[(size_t)s * rows];
        s_m[s][lane] = x.y > 0.f ? x.x : -INFINITY;
        s_l[s][lane] = x.y;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
        if (u < S) v[u] = po[u * slice];
    __syncthreads();
    float mx = -INFINITY, lsum = 0.f;
    for (int s = 0; s < S; ++s) mx = fmaxf(mx, s_m[s][lane]);
    for (int s = warp; s < S; s += 8) s_w[s][lane] = s_m[s][lane] == -INFINITY ? 0.f : exp2f(s_m[s][lane] - mx);
    __syncthreads();
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < S; s0 += kAhead) {
        if (s0 > 0) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (s0 + u < S) v[u] = po[(s0 + u) * slice];
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (s0 + u >= S) break;
            const float w = s_w[s0 + u][lane];
            lsum = fmaf(s_l[s0 + u][lane], w, lsum);        // (NaN stays NaN)
            if (w > 0.f) {                                  // (else an empty slice: nothing was written; or one that holds nothing for the row)
                acc.x = fmaf(w, v[u].x, acc.x); acc.y = fmaf(w, v[u].y, acc.y);
                acc.z = fmaf(w, v[u].z, acc.z); acc.w = fmaf(w, v[u].w, acc.w);
            }
        }
    }
    if (!ok) return;
    const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
    const size_t row = (size_t)(n0 + (R >> p.g_shift)) * p.Hq + g * p.G + (R & (p.G - 1));
    *reinterpret_cast<uint2*>(p.out + ((size_t)layer * p.sum_nodes * p.Hq + row) * kHeadDim + quad * 4) =
        make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
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
// Per device: shared memory beyond 48 KB, clusters of more than eight blocks.
static bool allow_paged() {
    static std::atomic<bool> done[64];
    int dev = 0;
    if (!allow_shared_memory<kSmemBytes>(tree_attention_paged_kernel) || !succeeded(cudaGetDevice(&dev)) || dev < 0 || dev >= 64) return false;
    if (!done[dev].load(std::memory_order_acquire)) {
        if (!succeeded(cudaFuncSetAttribute(tree_attention_paged_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1))) return false;
        done[dev].store(true, std::memory_order_release);
    }
    return true;
}
// How a launch is cut: items [0, whole) are worked on by a block per row tile, the others by `splits` of them, merged by a kernel of its own.
// Or all items are cut and the slices of a row tile are one cluster, which merges them itself; clusters of S blocks fit the chip
// `clusters(S)` times at once.
struct Cut { int whole, splits; bool in_cluster; };
// Bytes of partial results: of the items that are cut and not merged by a cluster.
static size_t partial_bytes(const Cut& cut, int n_layers, int batch, int sum_nodes, int n_q_heads, int n_kv_heads) {
    const size_t rest = (size_t)n_layers * batch * n_kv_heads - cut.whole;
    if (rest == 0 || cut.in_cluster) return 16;
    return rest * cut.splits * row_tiles_for(sum_nodes, n_q_heads / n_kv_heads) * kRowTile * (kHeadDim + 2) * sizeof(float);
}
static int clusters(int S) {
    static std::atomic<int> known[64][kMostInCluster + 1];      // + 1; 0: not asked yet
    int dev = 0;
    if (!succeeded(cudaGetDevice(&dev)) || dev < 0 || dev >= 64) return 0;      // (a size query without a device asks for what any plan needs)
    int n = known[dev][S].load(std::memory_order_relaxed);
    if (n == 0) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)S);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = kSmemBytes;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = (unsigned)S;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        if (!allow_paged() || !succeeded(cudaOccupancyMaxActiveClusters(&n, tree_attention_paged_kernel, &cfg))) return 0;
        known[dev][S].store(++n, std::memory_order_relaxed);
    }
    return n - 1;
}
// The costs, in us, fitted to launches of one to 63 pages a sequence, 8 to 480 rows, forced to one to sixteen slices:
//   a wave of blocks, one per SM           2.5 + 0.67 a page (a lone token 7.5 + 0.67 P with the launch's 5: 8.6 / 9.9 / 12.5 / 18.2 / 49.7 for 2 / 4 / 8 / 16 / 63)
//   ... two per SM                         4.5 + 1.05 a page
//   the merge as a kernel                  1.7, 2 more beyond eight slices (another round of reads), and the partial results, written and read
//   the merge in a cluster                 0.3, and 0.42 for each of a thread's outputs (128 rows: 6.7 us with two slices, 1.5 with eight), 0.55 beyond eight slices;
//                                          several clusters of more than ten blocks 1.6 more (one token at 2k keys, 8 / 10 / 11 / 16 slices 11.1 / 10.7 / 11.9 / 11.8)
// Full waves are left whole and what is left over fills the last one: 640 items of 257 pages are two waves and a sixth.  Cut only for a clear gain, since
// trees and lengths of a batch differ and blocks without rows leave at once: four sequences of 200 to 800 keys, 24 to 60 nodes, 18.6 us whole, 24 to 28 cut.
// room: of the workspace; no cut is taken whose partial results it does not hold (a size query asks with all the room there is, and more nodes
// may need less than fewer: what was allocated for one call has to do for another).
static Cut pick_cut(int n_sms, int n_layers, int batch, int n_kv_heads, int G, int pages, int sum_nodes, size_t room) {
    const int nodes = (sum_nodes + batch - 1) / batch, limit = nodes < SAGE_MAX_NODES ? nodes : SAGE_MAX_NODES;
    const long long items = (long long)n_layers * batch * n_kv_heads, tiles = row_tiles_for(nodes, G), slots = 2ll * n_sms;
    const double rows = (double)limit * G / (double)tiles;              // of a tile
    auto last_wave = [&](long long blocks, int per_block) {
        double cost = 0.0;
        for (; blocks > slots; blocks -= slots) cost += 4.5 + 1.05 * per_block;
        return cost + (blocks <= 0 ? 0.0 : blocks <= n_sms ? 2.5 + 0.67 * per_block : 4.5 + 1.05 * per_block);
    };
    const long long full = items * tiles / slots;
    Cut best{(int)items, 1, false};
    double best_cost = full * (4.5 + 1.05 * pages) + last_wave(items * tiles - full * slots, pages);
    best_cost *= 0.92;
    for (long long waves = full; waves >= 0 && waves >= full - 1; --waves) {
        const long long whole = waves * slots / tiles, rest = items - whole;
        if (rest < 1) continue;
        for (int s = 2; s <= kMostSplits && s <= pages && rest * tiles * s <= 4 * slots; ++s) {
            const double cost = waves * (4.5 + 1.05 * pages) + last_wave(rest * tiles * s, (pages + s - 1) / s) + 1.7 + (s > 8 ? 2.0 : 0.0) +
                                1.2e-6 / 6.5 * rest * tiles * s * rows * (kHeadDim + 2) * 4;
            const Cut cut{(int)whole, s, false};
            if (cost < best_cost && partial_bytes(cut, n_layers, batch, sum_nodes, n_kv_heads * G, n_kv_heads) <= room) {
                best_cost = cost;
                best = cut;
            }
        }
    }
    for (int s = 2; full == 0 && s <= kMostInCluster && s <= pages; ++s) {
        if (items * tiles > clusters(s)) continue;                      // (one wave of them)
        const double turns = (int)((rows * 32 / s + kRowTile - 1) / kRowTile);
        const double cost = last_wave(items * tiles * s, (pages + s - 1) / s) + 0.3 + (s > 8 ? 0.55 : 0.42) * turns + (s > 10 && items * tiles > 4 ? 1.6 : 0.0);
        if (cost < best_cost) {
            best_cost = cost;
            best = Cut{0, s, true};
        }
    }
    return best;
}
static size_t workspace_size(int n_layers, int batch, int sum_nodes, int n_q_heads, int n_kv_heads, int pages) {
    const Cut cut = pick_cut(resident_ctas(), n_layers, batch, n_kv_heads, n_q_heads / n_kv_heads, pages, sum_nodes, SIZE_MAX);
    return partial_bytes(cut, n_layers, batch, sum_nodes, n_q_heads, n_kv_heads);
}
static bool sizes_ok(int n_layers, int batch, int sum_nodes, int n_q_heads, int n_kv_heads, int max_pages) {
    return n_layers >= 1 && batch >= 1 && sum_nodes >= 1 && n_q_heads >= 1 && n_kv_heads >= 1 && max_pages >= 1 && n_q_heads % n_kv_heads == 0 &&
           (double)n_layers * batch * n_kv_heads <= 2147483647.0;
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
    if (!sizes_ok(n_layers, batch, sum_nodes, n_q_heads, n_kv_heads, max_pages)) return SAGE_ERR_UNSUPPORTED;
    if (!ws || ws_bytes < 16 || ((uintptr_t)ws & 15)) return SAGE_ERR_WORKSPACE;
    const Cut cut = pick_cut(resident_ctas(), n_layers, batch, n_kv_heads, G, pages, sum_nodes, ws_bytes);
    const int tiles = row_tiles_for(sum_nodes, G), rest = n_layers * batch * n_kv_heads - cut.whole;
    const double blocks = ((double)cut.whole + (double)rest * cut.splits) * tiles;
    if (blocks > 2147483647.0) return SAGE_ERR_UNSUPPORTED;
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
    if (!cut.in_cluster) p.part_ml = (float2*)((float*)ws + (size_t)rest * cut.splits * tiles * kRowTile * kHeadDim);
    p.page_table = page_table; p.seq_len = seq_len; p.parent = parent; p.node_offsets = node_offsets; p.status = status;
    if (s8) {
        p.page_table8 = s8->page_table; p.sealed = s8->sealed; p.k_exp = s8->k_exp; p.v_exp = s8->v_exp;
        p.n_pages8 = s8->n_pages; p.max_pages8 = s8->max_pages;
    }
    p.n_layers = n_layers; p.batch = batch; p.sum_nodes = sum_nodes; p.n_pages = pools.n_pages; p.max_pages = max_pages;
    p.Hq = n_q_heads; p.Hkv = n_kv_heads; p.G = G; p.g_shift = __builtin_ctz(G); p.n_whole = cut.whole; p.n_splits = cut.splits; p.in_cluster = cut.in_cluster; p.row_tiles = tiles;
    p.window = window; p.sink = sink;
    p.scale_log2 = sm_scale * 1.4426950408889634f;
    p.wait_cycles = attention_wait_cycles();
    p.producer_off = attention_producer_off();
    if (!allow_paged() || !succeeded(sage::launch(tree_attention_paged_kernel, dim3((unsigned)blocks), kThreads, kSmemBytes, as_stream(stream),
                                                  cut.in_cluster ? cut.splits : 0, p, qmap, kmap, vmap, k8map, v8map)))
        return SAGE_ERR_CUDA;
    if (rest == 0 || cut.in_cluster) return SAGE_OK;
    return launch_status(sage::launch(paged_merge_kernel, dim3(tiles * (kRowTile / 32), rest, 4), 256, 0, as_stream(stream), 0, p));
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
