// The life of pages outside the boundary step: requests get them from the free
// stack (gp_pages_reserve), share them with the requests that continue them
// (gp_pages_fork; App. E.2, reference-counted blocks) and give them back
// (gp_pages_release).
//
// The stack is one sequence, so whatever pops or pushes it is one workgroup, and
// the order of pages follows from prefix sums over the requests (pops) or from
// the page ids (pushes), never from which thread came first.  Bound: latency, a
// chain of dependent reads (list, request, table, count) and the launch.
#include <algorithm>

#include "gp_internal.h"

namespace gp {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// Inclusive sums over the workgroup's threads; *total: of all.
__device__ inline int block_sums(int x, int *s_wave, int *total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    __syncthreads();                                  // s_wave may still be read from the last call
    if (lane == 63) s_wave[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int n = s_wave[w];
        before += w < wave ? n : 0;
        all += n;
    }
    *total = all;
    return before + x;
}

// Which of n ascending ends is the first behind x (the last is).
__device__ inline int first_behind(const int *s_end, int n, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (s_end[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Pages in flight per thread, of whatever requests they are.
constexpr int kBatch = 8;

// ---------------------------------------------------------------- reserve --

__global__ __launch_bounds__(kThreads) void reserve_kernel(PagesArgs a) {
    __shared__ int s_wave[kWaves];
    __shared__ int s_end[kThreads], s_held[kThreads];  // pages granted up to a request; pages that it had
    const int tid = threadIdx.x;
    const int height = min(max(*a.free_count, 0), a.pool_pages);
    int64_t asked = 0;                                // pages asked for by the requests so far
    int taken = 0;
    for (int r0 = 0; r0 < a.R; r0 += kThreads) {
        const int r = r0 + tid;
        int P = 0, need = 0;
        bool fits = false;
        if (r < a.R) {
            const int m = a.seq_lens[r];
            P = a.num_pages[r];
            const int64_t want = ((int64_t)m + max(a.tokens[r], 0) + kPage - 1) / kPage;
            fits = m >= 0 && P >= 0 && P <= a.max_pages && want <= a.max_pages;
            need = fits ? max((int)want - P, 0) : 0;
        }
        int all, got;
        const int upto = block_sums(need, s_wave, &all);
        const bool ok = fits && (need == 0 || asked + upto <= height - a.keep_free);
        if (r < a.R) a.flags[r] = ok;
        // (requests are served until one cannot be: what is granted is asked for without a gap)
        s_end[tid] = block_sums(ok ? need : 0, s_wave, &got);
        s_held[tid] = P;
        if (ok && need) a.num_pages[r] = P + need;
        __syncthreads();
        for (int x0 = tid; x0 < got; x0 += kThreads * kBatch) {
            int page[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) page[k] = a.free_list[height - 1 - taken - min(x0 + k * kThreads, got - 1)];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int x = x0 + k * kThreads;
                if (x >= got) break;
                const int i = first_behind(s_end, kThreads, x);
                a.page_table[(size_t)(r0 + i) * a.max_pages + s_held[i] + x - (i ? s_end[i - 1] : 0)] = page[k];
                if (page[k] >= 0 && page[k] < a.pool_pages) a.refcount[page[k]] = 1;
            }
        }
        __syncthreads();
        asked += all;
        taken += got;
    }
    if (tid == 0 && taken) *a.free_count = height - taken;
}

// ---------------------------------------------------------------- release --

constexpr int kReleaseList = 2048;                    // requests whose pages are walked at a time
constexpr int kBitWords = 32768;                      // pages of pools up to 2^20 are marked in LDS

// The pages marked in s_bits onto the stack from `height` on, in ascending order: their number.
// A wave has a run of words, a lane one of 64 at a time, so that a wave's ids go to a few
// lines of the stack; a barrier between stores would wait for them (16 us for 6000 pages).
__device__ inline int push_marked(const PagesArgs &a, const uint32_t *s_bits, int *s_wave, int height) {
    const int words = cdiv(a.pool_pages, 32), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = cdiv(cdiv(words, kWaves), 64) * 64, w0 = min(wave * per, words), w1 = min(w0 + per, words);
    int mine = 0;
    for (int w = w0 + lane; w < w1; w += 64) mine += __popc(s_bits[w]);
    int pushed;
    int at = block_sums(mine, s_wave, &pushed);
    at = height + __shfl(at - mine, 0, 64);           // the wave's first place
    for (int w = w0; w < w1; w += 64) {
        uint32_t u = w + lane < w1 ? s_bits[w + lane] : 0;
        const int n = __popc(u);
        int upto = n;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int y = __shfl_up(upto, o, 64);
            if (lane >= o) upto += y;
        }
        int to = at + upto - n;
        for (; u; u &= u - 1, ++to)
            if (to < a.pool_pages) a.free_list[to] = 32 * (w + lane) + __ffs(u) - 1;
        at += __shfl(upto, 63, 64);
    }
    return pushed;
}

// All in one launch.  MARKS: larger pools: a page whose last reference goes is marked by a count of -1.
template <bool MARKS>
__global__ __launch_bounds__(kThreads) void release_kernel(PagesArgs a) {
    __shared__ int s_wave[kWaves];
    __shared__ int s_req[kReleaseList], s_end[kReleaseList];
    __shared__ uint32_t s_bits[MARKS ? 1 : kBitWords];
    const int tid = threadIdx.x;
    if (!MARKS)
        for (int i = tid; i < cdiv(a.pool_pages, 32); i += kThreads) s_bits[i] = 0;
    const int height = min(max(*a.free_count, 0), a.pool_pages);
    for (int i0 = 0; i0 < a.n; i0 += kReleaseList) {
        const int n = min(a.n - i0, kReleaseList);
        // each request once, however often it is listed: whoever takes its page count
        int sum = 0;
        for (int b = 0; b < n; b += kThreads) {
            const int i = b + tid;
            int r = -1, P = 0;
            if (i < n) {
                r = a.reqs[i0 + i];
                if (r >= 0 && r < a.R && a.seq_lens[r] >= 0) {
                    P = min(max(atomicExch(&a.num_pages[r], 0), 0), a.max_pages);
                    a.seq_lens[r] = 0;
                }
            }
            int all;
            const int upto = block_sums(P, s_wave, &all);
            if (i < n) {
                s_req[i] = r;
                s_end[i] = sum + upto;
            }
            sum += all;
        }
        __syncthreads();
        for (int base = 0; base < sum; base += kThreads * kBatch) {
            int page[kBatch], old[kBatch];
            // (base + k * kThreads < sum: none of the threads has the page otherwise)
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                page[k] = -1;
                if (base + k * kThreads >= sum) continue;
                const int x = base + k * kThreads + tid, i = first_behind(s_end, n, x);
                if (x < sum) page[k] = a.page_table[(size_t)s_req[i] * a.max_pages + (x - (i ? s_end[i - 1] : 0))];
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (base + k * kThreads >= sum) continue;
                old[k] = 0;
                if (page[k] >= 0 && page[k] < a.pool_pages) old[k] = atomicSub(&a.refcount[page[k]], 1);
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (base + k * kThreads >= sum || old[k] != 1) continue;
                if (MARKS) atomicExch(&a.refcount[page[k]], -1);
                else atomicOr(&s_bits[page[k] >> 5], 1u << (page[k] & 31));
            }
        }
        __syncthreads();
    }
    int pushed = 0;
    if (MARKS) {
        for (int p0 = 0; p0 < a.pool_pages; p0 += kThreads * kBatch) {
            int count[kBatch], mine = 0;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) count[k] = a.refcount[min(p0 + tid * kBatch + k, a.pool_pages - 1)];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) mine += p0 + tid * kBatch + k < a.pool_pages && count[k] == -1;
            int all;
            int at = height + pushed + block_sums(mine, s_wave, &all) - mine;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int p = p0 + tid * kBatch + k;
                if (p >= a.pool_pages || count[k] != -1) continue;
                a.refcount[p] = 0;
                if (at < a.pool_pages) a.free_list[at] = p;
                ++at;
            }
            pushed += all;
        }
    } else {
        pushed = push_marked(a, s_bits, s_wave, height);
    }
    if (tid == 0 && pushed) *a.free_count = min(height + pushed, a.pool_pages);
}

// Many pages in two launches: one workgroup's references to scattered counts take 2-3 ns each.  First a workgroup per request, which
// puts the pages that go onto the stack in any order and leaves -2 - (their number) as the
// request's page count; whoever takes the count away first works, so a request listed
// twice counts once.
constexpr int kRowThreads = 256, kOneReleaseLaunch = 32768;
__global__ __launch_bounds__(kRowThreads) void release_rows_kernel(PagesArgs a) {
    __shared__ int s_pages, s_freed;
    const int tid = threadIdx.x, r = a.reqs[blockIdx.x];
    if (r < 0 || r >= a.R || a.seq_lens[r] < 0) return;
    if (tid == 0) {
        const int P = a.num_pages[r];
        s_pages = P > 0 && atomicCAS(&a.num_pages[r], P, -1) == P ? min(P, a.max_pages) : 0;
        s_freed = 0;
    }
    __syncthreads();
    const int P = s_pages;
    if (P == 0) return;
    for (int base = 0; base < P; base += kRowThreads * kBatch) {
        int page[kBatch], old[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int j = base + k * kRowThreads + tid;
            page[k] = j < P ? a.page_table[(size_t)r * a.max_pages + j] : -1;
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            old[k] = 0;
            if (page[k] >= 0 && page[k] < a.pool_pages) old[k] = atomicSub(&a.refcount[page[k]], 1);
        }
        int mine = 0;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) mine += old[k] == 1;
        // places for the wave's pages, and in them for the lane's
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int y = __shfl_up(upto, o, 64);
            if ((tid & 63) >= o) upto += y;
        }
        int at = 0;
        if ((tid & 63) == 63 && upto) {
            at = atomicAdd(a.free_count, upto);
            atomicAdd(&s_freed, upto);
        }
        at = __shfl(at, 63, 64) + upto - mine;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (old[k] != 1) continue;
            if (at >= 0 && at < a.pool_pages) a.free_list[at] = page[k];
            ++at;
        }
    }
    __syncthreads();
    if (tid == 0) a.num_pages[r] = -2 - s_freed;
}

// Then the stack's new part in order, and the rows empty.
__global__ __launch_bounds__(kThreads) void release_order_kernel(PagesArgs a) {
    __shared__ int s_wave[kWaves];
    __shared__ int s_total;
    __shared__ uint32_t s_bits[kBitWords];
    const int tid = threadIdx.x, words = cdiv(a.pool_pages, 32);
    for (int i = tid; i < words; i += kThreads) s_bits[i] = 0;
    if (tid == 0) s_total = 0;
    const int end = *a.free_count;
    __syncthreads();
    for (int i = tid; i < a.n; i += kThreads) {
        const int r = a.reqs[i];
        if (r < 0 || r >= a.R || a.seq_lens[r] < 0) continue;
        const int x = atomicExch(&a.num_pages[r], 0);
        if (x <= -2) atomicAdd(&s_total, -2 - x);
        a.seq_lens[r] = 0;
    }
    __syncthreads();
    const int top = min(end, a.pool_pages), height = max(end - s_total, 0);
    for (int j = height + tid; j < top; j += kThreads) {
        const int page = a.free_list[j];
        if (page >= 0 && page < a.pool_pages) atomicOr(&s_bits[page >> 5], 1u << (page & 31));
    }
    __syncthreads();
    push_marked(a, s_bits, s_wave, height);
    if (tid == 0 && end > top) *a.free_count = top;
}

// ------------------------------------------------------------------- fork --

// Decisions, fresh pages and the children's lengths.  Everything is judged on the
// state as the call starts: all reads lie before the barriers of the sums, all
// writes behind them.  A fork's child then holds its last page already, so the
// second launch finds what to copy in the page state.
__global__ __launch_bounds__(kThreads) void fork_kernel(PagesArgs a) {
    __shared__ int s_wave[kWaves];
    __shared__ int s_child[kMaxForks];
    const int tid = threadIdx.x;
    for (int i = tid; i < a.n; i += kThreads) s_child[i] = a.children[i];
    const int height = min(max(*a.free_count, 0), a.pool_pages);
    __syncthreads();
    int p[2], c[2], L[2], pos[2];
    bool ok[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = tid + k * kThreads;
        ok[k] = false;
        p[k] = c[k] = -1;
        L[k] = pos[k] = 0;
        if (i >= a.n) continue;
        p[k] = a.reqs[i];
        c[k] = s_child[i];
        if (p[k] < 0 || p[k] >= a.R || c[k] < 0 || c[k] >= a.R) continue;
        const int m = a.seq_lens[p[k]], P = a.num_pages[p[k]];
        const bool empty = a.num_pages[c[k]] == 0 && a.seq_lens[c[k]] == 0;
        ok[k] = empty && m >= 0 && P >= 0 && P <= a.max_pages;
        L[k] = min(m, P * kPage);
        if (a.lengths) L[k] = min(L[k], max(a.lengths[i], 0));
        if (a.positions) pos[k] = a.positions[p[k]] - (m - L[k]);
        for (int j = 0; j < i && ok[k]; ++j) ok[k] = s_child[j] != c[k];
    }
    int taken = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = tid + k * kThreads;
        const bool need = ok[k] && L[k] % kPage;
        int all;
        const int rank = taken + block_sums(need, s_wave, &all) - 1;
        const bool got = need && rank < height;
        if (need && !got) ok[k] = false;
        if (i < a.n) a.flags[i] = ok[k];
        if (ok[k]) {
            const int full = L[k] / kPage;
            if (got) {
                const int page = a.free_list[height - 1 - rank];
                a.page_table[(size_t)c[k] * a.max_pages + full] = page;
                if (page >= 0 && page < a.pool_pages) a.refcount[page] = 1;
            }
            a.num_pages[c[k]] = full + got;
            a.seq_lens[c[k]] = L[k];
            if (a.positions) a.positions[c[k]] = pos[k];
        }
        taken += min(all, height - taken);
        if (k == 0 && a.n <= kThreads) break;
    }
    if (tid == 0 && taken) *a.free_count = height - taken;
}

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// blockIdx.y < n_layers: the rows of the page that the child cannot share, one layer, in
// 16-byte units; the last blockIdx.y: the references to those it shares.
constexpr int kCopyThreads = 256, kCopyBatch = 4;
__global__ __launch_bounds__(kCopyThreads) void fork_copy_kernel(PagesArgs a, PageLayers layers) {
    const int i = blockIdx.x, l = blockIdx.y, tid = threadIdx.x;
    if (!a.flags[i]) return;
    const int p = a.reqs[i], c = a.children[i], L = a.seq_lens[c];
    const int full = L / kPage, rows = L % kPage;
    const int32_t *from = a.page_table + (size_t)p * a.max_pages;
    int32_t *to = a.page_table + (size_t)c * a.max_pages;
    if (l == a.n_layers) {
        for (int j0 = tid; j0 < full; j0 += kCopyThreads * kCopyBatch) {
            int page[kCopyBatch];
#pragma unroll
            for (int k = 0; k < kCopyBatch; ++k) page[k] = from[min(j0 + k * kCopyThreads, full - 1)];
#pragma unroll
            for (int k = 0; k < kCopyBatch; ++k) {
                const int j = j0 + k * kCopyThreads;
                if (j >= full) break;
                to[j] = page[k];
                if (page[k] >= 0 && page[k] < a.pool_pages) atomicAdd(&a.refcount[page[k]], 1);
            }
        }
        return;
    }
    if (rows == 0) return;
    const int src = from[full], dst = to[full];
    if (src < 0 || src >= a.pool_pages || dst < 0 || dst >= a.pool_pages) return;
    const int per = rows * a.row_bytes / 16, slice = kPage * a.row_bytes / 16;        // units of one head's rows, of its page
    const int total = 2 * a.Hkv * per;
    for (int x0 = tid; x0 < total; x0 += kCopyThreads * kCopyBatch) {
        u32x4_t u[kCopyBatch];
        u32x4_t *at[kCopyBatch];
#pragma unroll
        for (int k = 0; k < kCopyBatch; ++k) {
            const int x = min(x0 + k * kCopyThreads, total - 1);
            const int head = x / per, unit = x - head * per;
            const bool isv = head >= a.Hkv;
            const int h = isv ? head - a.Hkv : head;
            u32x4_t *pool = static_cast<u32x4_t *>(isv ? layers.v[l] : layers.k[l]);
            u[k] = pool[((size_t)src * a.Hkv + h) * slice + unit];
            at[k] = pool + ((size_t)dst * a.Hkv + h) * slice + unit;
        }
#pragma unroll
        for (int k = 0; k < kCopyBatch; ++k)
            if (x0 + k * kCopyThreads < total) *at[k] = u[k];
    }
    if (layers.k_scale[l])
        for (int x = tid; x < 2 * a.Hkv; x += kCopyThreads) {
            float *s = x < a.Hkv ? layers.k_scale[l] : layers.v_scale[l];
            const int h = x < a.Hkv ? x : x - a.Hkv;
            s[(size_t)dst * a.Hkv + h] = s[(size_t)src * a.Hkv + h];
        }
}

}  // namespace

hipError_t launch_reserve(const PagesArgs &a, hipStream_t s) {
    reserve_kernel<<<1, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_pages_release(const PagesArgs &a, hipStream_t s) {
    // (the table's width is all that is known of the rows' pages: 32 rows of up to 1026, 6200 in all, take 19.6
    // us in one launch, 5.2 and 12.7 in two; fewer less in one, more in two)
    if (a.pool_pages <= 32 * kBitWords && a.n > 1 && (int64_t)a.n * a.max_pages > kOneReleaseLaunch) {
        release_rows_kernel<<<a.n, kRowThreads, 0, s>>>(a);
        release_order_kernel<<<1, kThreads, 0, s>>>(a);
    } else if (a.pool_pages <= 32 * kBitWords) release_kernel<false><<<1, kThreads, 0, s>>>(a);
    else release_kernel<true><<<1, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_fork(const PagesArgs &args, const PageLayers *layers, int n_layers, hipStream_t s) {
    PagesArgs a = args;
    fork_kernel<<<1, kThreads, 0, s>>>(a);
    for (int l = 0; l < n_layers; l += kMaxLayers, ++layers) {
        a.n_layers = std::min(n_layers - l, kMaxLayers);
        // (references once, with the first layers)
        fork_copy_kernel<<<dim3(a.n, a.n_layers + (l == 0)), kCopyThreads, 0, s>>>(a, *layers);
    }
    return hipGetLastError();
}

}  // namespace gp
