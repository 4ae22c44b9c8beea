// na_cache.hip -- the paged cache's tables, built on the GPU from request lengths, and the
// writes of new keys and values into its pages (gfx950).
#include "na_launch.h"
#include "na_seq_kernels.h"

namespace na {

namespace {

constexpr int kTabThreads = 256;
constexpr int kTabPer = 4;                          // requests per thread and pass
constexpr int kTabPass = kTabThreads * kTabPer;     // requests per pass
constexpr int kTabTokens = 1024;                    // tokens per workgroup

// Inclusive sum over the wave.
__device__ __forceinline__ int64_t wave_scan(int64_t x, int lane) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int64_t y = __shfl_up(x, d, kWave);
        x += lane >= d ? y : 0;
    }
    return x;
}

// One launch: every workgroup sums the lengths of all requests up to its own range of tokens
// (two int32 a request from L2, a pass of 1024 requests at a time) instead of waiting for
// another launch's sums, then finds the request of each of its tokens in the sums it holds in
// LDS.  A new page's id follows from the free list by index alone (request by request, page
// by page), so a token needs no table entry that this launch writes; the token that begins a
// page writes its entry.  Bound by its chain of loads and LDS steps: 64 requests of one token
// 4.2 us, 256 prompts of 0 to 511 tokens 8.4 us.
__global__ __launch_bounds__(kTabThreads) void cache_tables_kernel(
    int R, int tokens, int lgps, int max_pages, int num_free, const int* __restrict__ context,
    const int* __restrict__ fresh, const int* __restrict__ free_pages, const int* __restrict__ head,
    int* __restrict__ table, int* __restrict__ cu, int64_t* __restrict__ slots,
    int* __restrict__ positions, int* __restrict__ new_head) {
    __shared__ int64_t s_cu[kTabPass + 1];   // offset of each request of the pass
    __shared__ int64_t s_page[kTabPass];     // pages taken before it
    __shared__ int s_ctx[kTabPass];
    __shared__ int64_t s_n[kTabThreads / kWave], s_p[kTabThreads / kWave];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t t0 = (int64_t)blockIdx.x * kTabTokens;
    const int64_t t1 = min(t0 + kTabTokens, (int64_t)tokens);
    const int page = 1 << lgps;
    const int64_t h0 = head ? *head : 0;
    int64_t total = 0, taken = 0;  // of the passes before
    for (int base = 0; base < R; base += kTabPass) {
        if (blockIdx.x != 0 && total >= t1) return;
        int n[kTabPer], need[kTabPer];
        int64_t sn = 0, sp = 0;
#pragma unroll
        for (int i = 0; i < kTabPer; ++i) {
            const int r = base + tid * kTabPer + i;
            n[i] = need[i] = 0;
            if (r < R) {
                const int c = min(max(context[r], 0), 1 << 30);
                n[i] = min(max(fresh[r], 0), 1 << 30);
                const int held = (int)(((int64_t)c + page - 1) >> lgps);
                const int after = (int)(((int64_t)c + n[i] + page - 1) >> lgps);
                need[i] = min(after, max_pages) - min(held, max_pages);
                s_ctx[tid * kTabPer + i] = c;
            }
            sn += n[i];
            sp += need[i];
        }
        const int64_t in_n = wave_scan(sn, lane), in_p = wave_scan(sp, lane);
        if (lane == 63) {
            s_n[wave] = in_n;
            s_p[wave] = in_p;
        }
        __syncthreads();
        int64_t an = total + in_n - sn, ap = taken + in_p - sp, all_n = 0, all_p = 0;
#pragma unroll
        for (int w = 0; w < kTabThreads / kWave; ++w) {
            an += w < wave ? s_n[w] : 0;
            ap += w < wave ? s_p[w] : 0;
            all_n += s_n[w];
            all_p += s_p[w];
        }
#pragma unroll
        for (int i = 0; i < kTabPer; ++i) {
            const int x = tid * kTabPer + i;
            s_cu[x] = an;
            s_page[x] = ap;
            if (blockIdx.x == 0 && base + x < R) cu[base + x] = (int)min(an, (int64_t)INT32_MAX);
            an += n[i];
            ap += need[i];
        }
        if (tid == kTabThreads - 1) s_cu[kTabPass] = an;
        __syncthreads();
        const int64_t end = min(t1, total + all_n);
        for (int64_t tok = max(t0, total) + tid; tok < end; tok += kTabThreads) {
            int lo = 0, hi = kTabPass;  // the last request with s_cu <= tok
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_cu[mid] <= tok) lo = mid;
                else hi = mid;
            }
            const int c = s_ctx[lo];
            const int pos = c + (int)(tok - s_cu[lo]);
            const int idx = pos >> lgps, held = (int)(((int64_t)c + page - 1) >> lgps);
            int* entry = table + (int64_t)(base + lo) * max_pages + idx;
            int id = -1;
            if (idx < max_pages) {
                if (idx < held) {
                    id = *entry;
                } else {
                    const int64_t f = h0 + s_page[lo] + (idx - held);
                    if (f >= 0 && f < num_free) id = free_pages[f];
                    if ((pos & (page - 1)) == 0) *entry = id;
                }
            }
            slots[tok] = id < 0 ? -1 : ((int64_t)id << lgps) + (pos & (page - 1));
            positions[tok] = pos;
        }
        total += all_n;
        taken += all_p;
        __syncthreads();
    }
    for (int64_t tok = max(t0, total) + tid; tok < t1; tok += kTabThreads) {
        slots[tok] = -1;
        positions[tok] = -1;
    }
    if (blockIdx.x == 0 && tid == 0) {
        cu[R] = (int)min(total, (int64_t)INT32_MAX);
        *new_head = (int)min(h0 + taken, (int64_t)INT32_MAX);
    }
}

// A thread per 16 bytes of a key row and its value row; consecutive threads run along a row,
// so loads and stores are whole rows.  Bound by memory: 32k tokens of 8 heads, bf16 D = 128,
// 258 MB in 49 us a call on changing buffers (5.2 TB/s; 41 us of kernel time on the same ones
// again, part of which caches may hold); 64 tokens 2.6 us.
__global__ __launch_bounds__(256) void cache_write_kernel(
    uint32_t units, int lgseg, int Hkv, FastDiv fd_kv, int lgps, int64_t slots_end, int64_t kt,
    int64_t kh, int64_t vt, int64_t vh, const unsigned char* __restrict__ k,
    const unsigned char* __restrict__ v, const int64_t* __restrict__ slots,
    unsigned char* __restrict__ k_pages, unsigned char* __restrict__ v_pages) {
    for (uint32_t u = blockIdx.x * 256 + threadIdx.x; u < units; u += gridDim.x * 256) {
        const int seg = (int)(u & ((1u << lgseg) - 1)) << 4;
        const int rest = (int)(u >> lgseg);
        const int tok = fd_kv.div(rest), h = rest - tok * Hkv;
        const int64_t slot = slots[tok];
        if (slot < 0 || slot >= slots_end) continue;
        const int64_t row = ((((slot >> lgps) * Hkv + h) << lgps) + (slot & ((1 << lgps) - 1)));
        const int64_t to = (row << (lgseg + 4)) + seg;
        const i32x4 a = ld16<i32x4>(k + tok * kt + h * kh + seg);
        const i32x4 b = ld16<i32x4>(v + tok * vt + h * vh + seg);
        st16(k_pages + to, a);
        st16(v_pages + to, b);
    }
}

}  // namespace

hipError_t launch_cache_tables(int R, int tokens, int lgps, int max_pages, int num_free,
                               const int32_t* context, const int32_t* fresh,
                               const int32_t* free_pages, const int32_t* head, int32_t* table,
                               int32_t* cu, int64_t* slots, int32_t* positions, int32_t* new_head,
                               hipStream_t s) {
    const int grid = tokens > kTabTokens ? (int)(((int64_t)tokens + kTabTokens - 1) / kTabTokens) : 1;
    hipLaunchKernelGGL(cache_tables_kernel, dim3(grid), dim3(kTabThreads), 0, s, R, tokens, lgps,
                       max_pages, num_free, context, fresh, free_pages, head, table, cu, slots,
                       positions, new_head);
    return hipGetLastError();
}

hipError_t launch_cache_write(int tokens, int Hkv, int row_bytes, int lgps, int64_t slots_end,
                              int64_t kt, int64_t kh, int64_t vt, int64_t vh, const void* k,
                              const void* v, const int64_t* slots, void* k_pages, void* v_pages,
                              hipStream_t s) {
    const int lgseg = 31 - __builtin_clz((unsigned)row_bytes >> 4);
    const uint32_t units = ((uint32_t)tokens * (uint32_t)Hkv) << lgseg;
    FastDiv fd;
    fd.init(Hkv);
    const uint32_t grid = std::min<uint32_t>((units + 255) / 256, 1u << 16);
    hipLaunchKernelGGL(cache_write_kernel, dim3(grid), dim3(256), 0, s, units, lgseg, Hkv, fd, lgps,
                       slots_end, kt, kh, vt, vh, static_cast<const unsigned char*>(k),
                       static_cast<const unsigned char*>(v), slots,
                       static_cast<unsigned char*>(k_pages), static_cast<unsigned char*>(v_pages));
    return hipGetLastError();
}

}  // namespace na
