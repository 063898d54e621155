// Full pages of the bf16 cache move into an 8-bit one ("sealed"), sm_100a.
//
// A tile is the 64 x 128 values of one page, KV head and layer, of K or of V.  Its scale is the smallest power of two 2^e with
// max |x| <= 448 * 2^e (e in [-60, 60]; the byte e + 127 is kept), its values are the nearest e4m3 numbers to x / 2^e.
// A power of two costs a format with an exponent nothing but, at the lower end, one of its 18 binades, and lets the attention
// kernel apply scales in exponents.  Whole pages only: every value is rounded once, when its page is complete, and no page changes its scale.
// Bound by memory (2 bytes read, 1 written per value): a block takes K and V of one (layer, page, head), 128 threads each, which
// hold the tile in registers between its maximum and its values, so it is read once.
#include "paged.cuh"

namespace sage {
namespace seal {

constexpr int kThreads = 256;
constexpr int kChunks = kPageSize * kHeadDim / 8 / 128;     // of 8 values, per thread
constexpr int kExpLo = -60, kExpHi = 60;

struct Params {
    const __nv_bfloat16 *k_pool, *v_pool;
    uint8_t *k8, *v8, *k_exp, *v_exp;
    int64_t layer_stride, layer_stride8;
    int n_layers, n_pages, max_pages, n_pages8, max_pages8, batch, Hkv;
    const int32_t *page_table, *page_table8, *seq_len;
    int32_t *sealed, *status;
};

// Pages [first, last) of sequence b are to be sealed.
struct Range { int first, last; };
__device__ __forceinline__ Range range_of(const Params& p, int b, bool* bad) {
    Range r{p.sealed[b], p.seq_len[b] / kPageSize};
    if (p.seq_len[b] < 0 || r.first < 0 || r.first > r.last || r.last > p.max_pages || r.last > p.max_pages8) {
        *bad = true;
        r.last = r.first;
    }
    return r;
}

__global__ void __launch_bounds__(kThreads) seal_pages_kernel(const __grid_constant__ Params p) {
    __shared__ uint32_t s_most[2][2][4];        // [parity][K, V][warp]
    __shared__ long long s_total;
    __shared__ int s_page[2];
    after_previous_kernel();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, side = tid >> 7, t = tid & 127;
    // pages of the launch; work = pages x layers x heads, this block's share of it in one piece (pages change least often)
    if (warp == 0) {
        long long total = 0;
        for (int b = lane; b < p.batch; b += 32) {
            bool bad = false;
            const Range r = range_of(p, b, &bad);
            total += r.last - r.first;
        }
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        if (lane == 0) s_total = total;
    }
    __syncthreads();
    const long long per_page = (long long)p.n_layers * p.Hkv, work = s_total * per_page;
    const long long begin = work * blockIdx.x / gridDim.x, end = work * (blockIdx.x + 1) / gridDim.x;
    long long page_no = -1;
    int src = -1, dst = -1, parity = 0;
    for (long long w = begin; w < end; ++w) {
        const long long u = w / per_page;
        const int rest = (int)(w - u * per_page), layer = rest / p.Hkv, g = rest % p.Hkv;
        if (u != page_no) {                     // uniform
            page_no = u;
            __syncthreads();
            if (warp == 0) {
                long long run = 0;
                for (int b0 = 0; b0 < p.batch; b0 += 32) {
                    bool bad = false;
                    Range r{0, 0};
                    if (b0 + lane < p.batch) r = range_of(p, b0 + lane, &bad);
                    int inc = r.last - r.first;
                    const int n = inc;
                    for (int o = 1; o < 32; o <<= 1) {
                        const int v = __shfl_up_sync(0xffffffffu, inc, o);
                        if (lane >= o) inc += v;
                    }
                    const bool mine = u >= run + inc - n && u < run + inc;
                    if (mine) {
                        const size_t at = r.first + (size_t)(u - (run + inc - n));
                        s_page[0] = p.page_table[(size_t)(b0 + lane) * p.max_pages + at];
                        s_page[1] = p.page_table8[(size_t)(b0 + lane) * p.max_pages8 + at];
                    }
                    if (__any_sync(0xffffffffu, mine)) break;
                    run += __shfl_sync(0xffffffffu, inc, 31);
                }
            }
            __syncthreads();
            src = s_page[0];
            dst = s_page[1];
            if (src < 0 || src >= p.n_pages || dst < 0 || dst >= p.n_pages8) src = -1;     // (reported by the other kernel)
        }
        if (src < 0) continue;                  // uniform
        const size_t head8 = (size_t)dst * p.Hkv + g;
        const uint4* x = reinterpret_cast<const uint4*>((side ? p.v_pool : p.k_pool) + layer * p.layer_stride +
                                                        ((size_t)src * p.Hkv + g) * kPageSize * kHeadDim);
        uint4 v[kChunks];                       // neighbours in a pair of chunks: 32 bytes in, 16 out
#pragma unroll
        for (int i = 0; i < kChunks / 2; ++i) {
            v[2 * i] = x[(i * 128 + t) * 2];
            v[2 * i + 1] = x[(i * 128 + t) * 2 + 1];
        }
        uint32_t most = 0;                      // largest magnitude bits: NaN above infinity above all others
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
            most = __vmaxu2(most, __vmaxu2(__vmaxu2(v[i].x & 0x7fff7fffu, v[i].y & 0x7fff7fffu), __vmaxu2(v[i].z & 0x7fff7fffu, v[i].w & 0x7fff7fffu)));
        most = __reduce_max_sync(0xffffffffu, max(most & 0xffffu, most >> 16));
        if (lane == 0) s_most[parity][side][warp & 3] = most;
        __syncthreads();
        most = max(max(s_most[parity][side][0], s_most[parity][side][1]), max(s_most[parity][side][2], s_most[parity][side][3]));
        parity ^= 1;
        // |x| = m 2^E, m in [1, 2): 448 2^e = 1.75 2^(8 + e) holds it for e = E - 8, or E - 7 where m > 1.75
        int e = (int)(most >> 7) - 127 - 8 + ((most & 0x7f) > 0x60 ? 1 : 0);
        e = min(max(e, kExpLo), kExpHi);
        const float down = __uint_as_float((uint32_t)(127 - e) << 23);
        uint4* y = reinterpret_cast<uint4*>((side ? p.v8 : p.k8) + layer * p.layer_stride8 + head8 * kPageSize * kHeadDim);
#pragma unroll
        for (int i = 0; i < kChunks / 2; ++i) {
            uint32_t o[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const uint4& c = v[2 * i + (h >> 1)];
                const uint32_t a = h & 1 ? c.z : c.x, b = h & 1 ? c.w : c.y;
                uint16_t lo, hi;
                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(__uint_as_float(a & 0xffff0000u) * down), "f"(__uint_as_float(a << 16) * down));
                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(__uint_as_float(b & 0xffff0000u) * down), "f"(__uint_as_float(b << 16) * down));
                o[h] = lo | ((uint32_t)hi << 16);
            }
            y[i * 128 + t] = make_uint4(o[0], o[1], o[2], o[3]);
        }
        if (t == 0) (side ? p.v_exp : p.k_exp)[((size_t)layer * p.n_pages8 + dst) * p.Hkv + g] = (uint8_t)(e + 127);
    }
}

// Behind it: the sequences whose pages were all there count them as sealed (a block per sequence).
__global__ void __launch_bounds__(128) count_sealed_kernel(const __grid_constant__ Params p) {
    after_previous_kernel();
    const int b = blockIdx.x;
    bool bad = false;
    const Range r = range_of(p, b, &bad);
    for (int i = r.first + threadIdx.x; i < r.last; i += 128) {
        const int src = p.page_table[(size_t)b * p.max_pages + i], dst = p.page_table8[(size_t)b * p.max_pages8 + i];
        bad |= src < 0 || src >= p.n_pages || dst < 0 || dst >= p.n_pages8;
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
        if (bad) report_status(p.status, SAGE_STATUS_BAD_PAGE);
        else p.sealed[b] = r.last;
    }
}

}  // namespace seal
}  // namespace sage

using namespace sage;

extern "C" int sage_seal_kv(const void* k_pool, const void* v_pool, int64_t layer_stride_elems, int n_layers, int n_pages,
                            const int32_t* page_table, int max_pages_per_seq, const int32_t* seq_len, const sage_sealed_cache* cache,
                            int32_t* sealed, int batch, int n_kv_heads, int head_dim, int page_size, int32_t* status, void* stream) {
    if (!k_pool || !v_pool || !page_table || !seq_len || !cache || !sealed) return SAGE_ERR_INVALID_ARG;
    if (!cache->k || !cache->v || !cache->k_exp || !cache->v_exp || !cache->page_table) return SAGE_ERR_INVALID_ARG;
    if (n_layers < 1 || n_pages < 1 || max_pages_per_seq < 1 || batch < 0 || n_kv_heads < 1 || layer_stride_elems < 0 || cache->n_pages < 1 ||
        cache->max_pages_per_seq < 1 || cache->layer_stride < 0)
        return SAGE_ERR_INVALID_ARG;
    if (head_dim != kHeadDim || page_size != kPageSize) return SAGE_ERR_UNSUPPORTED;
    if ((((uintptr_t)k_pool | (uintptr_t)v_pool | (uintptr_t)cache->k | (uintptr_t)cache->v) & 15) || (layer_stride_elems & 7) ||
        (cache->layer_stride & 15))
        return SAGE_ERR_INVALID_ARG;
    if (n_layers > 1 && (layer_stride_elems < (int64_t)n_pages * n_kv_heads * kPageSize * kHeadDim ||
                         cache->layer_stride < (int64_t)cache->n_pages * n_kv_heads * kPageSize * kHeadDim))
        return SAGE_ERR_INVALID_ARG;
    if ((int64_t)n_layers * n_kv_heads > 0x7fffffff) return SAGE_ERR_UNSUPPORTED;
    if (batch == 0) return SAGE_OK;
    seal::Params p{};
    p.k_pool = (const __nv_bfloat16*)k_pool; p.v_pool = (const __nv_bfloat16*)v_pool;
    p.k8 = (uint8_t*)cache->k; p.v8 = (uint8_t*)cache->v; p.k_exp = cache->k_exp; p.v_exp = cache->v_exp;
    p.layer_stride = n_layers > 1 ? layer_stride_elems : 0;
    p.layer_stride8 = n_layers > 1 ? cache->layer_stride : 0;
    p.n_layers = n_layers; p.n_pages = n_pages; p.max_pages = max_pages_per_seq; p.n_pages8 = cache->n_pages; p.max_pages8 = cache->max_pages_per_seq;
    p.batch = batch; p.Hkv = n_kv_heads;
    p.page_table = page_table; p.page_table8 = cache->page_table; p.seq_len = seq_len;
    p.sealed = sealed; p.status = status;
    // What may have to be sealed is known on the device only: as many blocks as are resident (three per SM), or as there can be tiles.  (One page of each of
    // sixteen sequences, 4 layers / 80 layers / a prefill of 16k, 28 layers: 8.5 / 83.7 / 428 us; with four, of which one waits, 9.5 / 101 / 524; with six
    // 10.1 / 85 / 432; four resident, in 64 registers, 7.8 / 90 / 473.)
    const double most = (double)batch * max_pages_per_seq * n_layers * n_kv_heads;
    const int resident = resident_ctas() * 3, blocks = most < resident ? (int)most : resident;
    const int code = launch_status(launch(seal::seal_pages_kernel, dim3(blocks), seal::kThreads, 0, as_stream(stream), 0, p));
    if (code != SAGE_OK) return code;
    return launch_status(launch(seal::count_sealed_kernel, dim3(batch), 128, 0, as_stream(stream), 0, p));
}
