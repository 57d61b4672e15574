// Attention over a selection of the pages: the bounds of each page's keys
// (gp_page_bounds) and the choice of the pages by them (gp_select_pages).
//
// For a query head q and a page whose keys lie in the box [lo, hi], no logit of
// the page exceeds sum_d max(q_d lo_d, q_d hi_d).  The sum over the query heads of
// a KV head is linear in the box, sum_d (hi_d Q+_d + lo_d Q-_d) with Q+ (Q-) the sum
// of the heads' positive (negative) parts, so a page's score costs 2 d products
// whatever the number of heads.  Products of bfloat16 bounds with Q+- are exact in
// 64 bits and their sum almost always is, so that the choice does not hang on the
// order of a sum; it is rounded once to float32 and the ties go to the lower page.
//
// Bound: HBM.  The bounds of a page and head are 2 d elements, a sixteenth of the
// page's keys and values.  Scores: 226 MB of boxes in 40.8 us, 5.5 TB/s, of the 6.9 that
// a stream of reads reaches; bounds: 337 MB (float32, d 64) in 63.7 us, 5.3 TB/s, 304 MB
// (bfloat16, d 128) in 64.5, 4.7, 156 MB (8 bits, d 128) in 48.8, 3.2.  The choice itself
// reads a few numbers a page and waits on its own barriers: 6.4 us, 7.8 for 384 lists
// out of up to 2048 pages.
#include <algorithm>
#include <type_traits>

#include "gp_internal.h"

namespace gp {

namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef u32x4_t u32x4_e2_t __attribute__((aligned(2)));
typedef u32x4_t u32x4_e4_t __attribute__((aligned(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef f32x4_t f32x4_e4_t __attribute__((aligned(4)));
__device__ inline u32x4_t load16(const uint16_t *p) { return *reinterpret_cast<const u32x4_e2_t *>(p); }
__device__ inline u32x4_t load16(const float *p) { return *reinterpret_cast<const u32x4_e4_t *>(p); }
__device__ inline void store16(uint16_t *p, const u32x4_t &x) { *reinterpret_cast<u32x4_e2_t *>(p) = x; }
__device__ inline void store16(float *p, const u32x4_t &x) { *reinterpret_cast<u32x4_e4_t *>(p) = x; }

// ... of data that is read once: the caches keep what others reuse, and the reads
// themselves are faster (scores of 226 MB of boxes 48.1 -> 40.5 us, bounds 71 -> 63.5)
__device__ inline u32x4_t load16_once(const uint16_t *p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_e2_t *>(p)); }
__device__ inline u32x4_t load16_once(const float *p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_e4_t *>(p)); }

template <typename T>
struct Unit;                                          // 16 bytes of T, widened
template <>
struct Unit<uint16_t> {
    static constexpr int N = 8;
    __device__ static inline float at(const u32x4_t &u, int e) { return e & 1 ? bf16_hi(u[e / 2]) : bf16_lo(u[e / 2]); }
};
template <>
struct Unit<float> {
    static constexpr int N = 4;
    __device__ static inline float at(const u32x4_t &u, int e) { return __uint_as_float(u[e]); }
};

// ------------------------------------------------------------------ bounds --
// Minimum and maximum that keep a NaN.
__device__ inline float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ inline float greatest(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// f over the lanes l ^ 32, l ^ 16 (and l ^ 8): the partners' values exchanged in the
// vector ALU
template <typename F>
__device__ inline float fold32(float x, F f) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <typename F>
__device__ inline float fold16(float x, F f) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <typename F>
__device__ inline float fold8(float x, F f) {
    return f(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x128, 0xf, 0xf, false)));
}

// A wave per (page, KV head) slice, the heads of a page side by side.  Lane (u, g)
// takes elements EU u .. of rows g, g + RG, ..: every load instruction is one
// contiguous run of the slice.  CACHE: bytes of a pool element.  16 requests of 300-16384
// tokens, 8 KV heads, float32, d 64 (337 MB): 63.5 us; with two or four slices in flight
// per wave 61-63, but a step's 64 pages 4.8 and 6.7 us instead of 3.5.
constexpr int kBoundWaves = 4;
template <int CACHE, int D>
__global__ __launch_bounds__(64 * kBoundWaves) void bounds_kernel(BoundsArgs a) {
    using E = typename std::conditional<CACHE == 4, float, uint16_t>::type;     // of the bounds
    constexpr int EU = CACHE == 4 ? 4 : 8;            // elements per lane and row
    constexpr int UPR = D / EU, RG = 64 / UPR, RPL = kPage / RG;
    const int r = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int u = lane % UPR, g = lane / UPR;
    const int P = min(max(a.num_pages[r], 0), a.max_pages), m = min(a.seq_lens[r], P * kPage);
    if (m <= 0) return;                               // nothing resident, or held
    const int from = a.from ? max(a.from[r], 0) : 0;
    if (from >= m) return;
    const int p0 = from / kPage, count = min(cdiv(m, kPage) - p0, a.max_update);
    const int tasks = count * a.Hkv;
    for (int task = blockIdx.x * kBoundWaves + wave; task < tasks; task += gridDim.x * kBoundWaves) {
        const int p = p0 + task / a.Hkv, h = task % a.Hkv;
        const int pid = a.page_table[(size_t)r * a.max_pages + p];
        if (pid < 0 || pid >= a.pool_pages) continue;
        const int ntok = min(kPage, m - p * kPage);
        const size_t slice = (size_t)pid * a.Hkv + h;
        float x[RPL][EU], scale = 1.0f;               // (8 bits: codes; the scale is positive and meets the bounds)
        if constexpr (CACHE == 1) {
            const uint8_t *src = reinterpret_cast<const uint8_t *>(a.k) + slice * kPage * D + u * EU;
            scale = a.k_scale[slice];
            u32x2_t w[RPL];
#pragma unroll
            for (int i = 0; i < RPL; ++i) w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t *>(src + (i * RG + g) * D));
#pragma unroll
            for (int i = 0; i < RPL; ++i)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const auto y0 = __builtin_amdgcn_cvt_pk_f32_fp8(w[i][c], false), y1 = __builtin_amdgcn_cvt_pk_f32_fp8(w[i][c], true);
                    x[i][4 * c] = y0[0];
                    x[i][4 * c + 1] = y0[1];
                    x[i][4 * c + 2] = y1[0];
                    x[i][4 * c + 3] = y1[1];
                }
        } else {
            const E *src = reinterpret_cast<const E *>(a.k) + slice * kPage * D + u * EU;
            u32x4_t w[RPL];
#pragma unroll
            for (int i = 0; i < RPL; ++i) w[i] = load16_once(src + (i * RG + g) * D);
#pragma unroll
            for (int i = 0; i < RPL; ++i)
#pragma unroll
                for (int e = 0; e < EU; ++e) x[i][e] = Unit<E>::at(w[i], e);
        }
        u32x4_t out_lo, out_hi;
        float lo[EU], hi[EU];
#pragma unroll
        for (int e = 0; e < EU; ++e) {
            lo[e] = __builtin_huge_valf();
            hi[e] = -__builtin_huge_valf();
#pragma unroll
            for (int i = 0; i < RPL; ++i) {
                const bool in = i * RG + g < ntok;
                lo[e] = in ? least(lo[e], x[i][e]) : lo[e];
                hi[e] = in ? greatest(hi[e], x[i][e]) : hi[e];
            }
            lo[e] = fold32(lo[e], least);
            hi[e] = fold32(hi[e], greatest);
            if constexpr (RG >= 4) {
                lo[e] = fold16(lo[e], least);
                hi[e] = fold16(hi[e], greatest);
            }
            if constexpr (RG >= 8) {
                lo[e] = fold8(lo[e], least);
                hi[e] = fold8(hi[e], greatest);
            }
        }
        if constexpr (CACHE == 1) {                   // (the lanes that write them: g = 0 the least, 1 the greatest)
#pragma unroll
            for (int e = 0; e < EU; ++e) lo[e] = hi[e] = odd_product(g == 1 ? hi[e] : lo[e], scale);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (CACHE == 4) {
                out_lo[e] = __float_as_uint(lo[e]);
                out_hi[e] = __float_as_uint(hi[e]);
            } else {
                out_lo[e] = f32_to_bf16(lo[2 * e]) | (uint32_t)f32_to_bf16(lo[2 * e + 1]) << 16;
                out_hi[e] = f32_to_bf16(hi[2 * e]) | (uint32_t)f32_to_bf16(hi[2 * e + 1]) << 16;
            }
        }
        E *to = reinterpret_cast<E *>(a.bounds) + slice * 2 * D + u * EU;
        if (g == 0) store16(to, out_lo);
        if (g == 1) store16(to + D, out_hi);
    }
}

// ------------------------------------------------------------------ scores --
// Pages resident of request r (0: none, or held).
__device__ inline int resident_pages(const SelectArgs &a, int r) {
    const int P = min(max(a.num_pages[r], 0), a.max_pages);
    return cdiv(min(max(a.seq_lens[r], 0), P * kPage), kPage);
}

// x of the lane that DPP control CTRL names
template <int CTRL>
__device__ inline double from_lane(double x) {
    const long long b = __builtin_bit_cast(long long, x);
    const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xf, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xf, 0xf, false);
    return __builtin_bit_cast(double, (long long)hi << 32 | (unsigned)lo);
}
// the sum over a lane's group of eight, in all of them: xor 1, xor 2 (quad
// permutations), then the mirrored half row, which has the other quad's
__device__ inline double sum8(double x) {
    x += from_lane<0xb1>(x);
    x += from_lane<0x4e>(x);
    return x + from_lane<0x141>(x);
}
// Two sums over lanes l and l ^ BIT for one addition: a's in the lanes where BIT is
// clear, b's where it is set.  The halves (rows) trade places in the vector ALU.
template <int BIT>
__device__ inline double pair_sum(double a, double b) {
    const long long x = __builtin_bit_cast(long long, a), y = __builtin_bit_cast(long long, b);
    if constexpr (BIT == 8) {
        const bool set = __lane_id() & 8;
        const double keep = set ? b : a, give = set ? a : b;
        return keep + from_lane<0x128>(give);         // row rotated by 8
    } else {
        auto swap = [](unsigned u, unsigned v) {
            if constexpr (BIT == 32) return __builtin_amdgcn_permlane32_swap(u, v, false, false);
            else return __builtin_amdgcn_permlane16_swap(u, v, false, false);
        };
        const auto lo = swap((unsigned)x, (unsigned)y), hi = swap((unsigned)(x >> 32), (unsigned)(y >> 32));
        return __builtin_bit_cast(double, (long long)hi[0] << 32 | lo[0]) +
               __builtin_bit_cast(double, (long long)hi[1] << 32 | lo[1]);
    }
}

// A lane holds one 16-byte unit of a page's box (least, then greatest values), so a
// load instruction reads PPI whole boxes of LPP lanes each, and a lane needs its own
// N dims of Q- or Q+ only.  kScoreLoads instructions are in flight per wave; their
// sums meet pairwise over the lanes (pair_sum), then over groups of eight.  (Eight
// lanes per page, with 32 dims each, took 64 registers for Q+- and left half as many
// bytes in flight: 57 us for 227 MB; with float32 sums no less.)
// The waves of a workgroup take the heads of the same pages side by side.  Grid
// (items of one KV head and wave_pages pages, kScoreWaves a workgroup; request).
constexpr int kScoreWaves = 4, kScorePages = 64;      // waves, and pages per wave at most
constexpr int kScoreLoads = 8;
template <typename T, int D>
struct Box {
    static constexpr int N = Unit<T>::N, LPP = 2 * D / N, PPI = 64 / LPP, STEP = kScoreLoads * PPI;   // STEP: pages per step
};
template <typename T, int D, int G>
__global__ __launch_bounds__(64 * kScoreWaves) void score_kernel(SelectArgs a) {
    using B = Box<T, D>;
    constexpr int N = B::N, LPP = B::LPP, PPI = B::PPI, U = kScoreLoads;
    const int r = blockIdx.y;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int item = blockIdx.x * kScoreWaves + wave, h = item % a.Hkv;
    const int u = lane % LPP, group = lane / LPP;
    const bool upper = u >= LPP / 2;                  // of the greatest values
    const int n = resident_pages(a, r);
    const int p0 = item / a.Hkv * a.wave_pages;
    if (n <= a.budget || p0 >= n) return;             // all pages are selected; none for this wave
    const int count = min(a.wave_pages, n - p0);
    int id = lane < count ? a.page_table[(size_t)r * a.max_pages + p0 + lane] : -1;
    if (id >= a.pool_pages) id = -1;
    const T *boxes = reinterpret_cast<const T *>(a.bounds) + (size_t)h * 2 * D + u * N;
    float *scores = a.scores + ((size_t)r * a.Hkv + h) * a.max_pages + p0;
    u32x4_t box[U];
    auto request = [&](int s) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int pid = __shfl(id, min(s * B::STEP + j * PPI + group, 63), 64);
            box[j] = load16_once(boxes + (size_t)max(pid, 0) * a.Hkv * 2 * D);
        }
    };
    // this lane's dims of the group's queries: requested before the boxes, as loads are
    // waited for in order
    u32x4_t qx[G];
    const T *q = reinterpret_cast<const T *>(a.q) + ((size_t)r * a.Hkv + h) * G * D + u % (LPP / 2) * N;
#pragma unroll
    for (int g = 0; g < G; ++g) qx[g] = load16(q + g * D);
    request(0);
    double w[N];
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = 0.0;
#pragma unroll
    for (int g = 0; g < G; ++g) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float y = Unit<T>::at(qx[g], e);
            w[e] += (upper ? y < 0.0f : y >= 0.0f) ? 0.0f : y;                   // (a NaN counts in both)
            __asm__ volatile("" : "+v"(w[e]));
        }
    }
    for (int s = 0; s * B::STEP < count; ++s) {
        double v[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            v[j] = 0.0;
#pragma unroll
            for (int e = 0; e < N; ++e) v[j] = __builtin_fma((double)Unit<T>::at(box[j], e), w[e], v[j]);
            // (a value of its own: the compiler would make vectors of the boxes' chains, with
            // four copies of w, 130 registers instead of 84)
            __asm__ volatile("" : "+v"(v[j]));
        }
        bool bad = false;
#pragma unroll
        for (int j = 0; j < U; ++j) bad |= v[j] != v[j];
        if (__any(bad)) {                             // rare: a zero factor meets an infinite bound, and adds nothing
#pragma unroll
            for (int j = 0; j < U; ++j) {
                __asm__ volatile("" : "+v"(box[j]));  // (widened again, not kept from above)
                v[j] = 0.0;
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (w[e] != 0.0) v[j] = __builtin_fma((double)Unit<T>::at(box[j], e), w[e], v[j]);
                __asm__ volatile("" : "+v"(v[j]));
            }
        }
        if ((s + 1) * B::STEP < count) request(s + 1);
        // sums over the LPP lanes of a page; value i of a lane is then that of load j(i)
        constexpr int LEFT = LPP == 64 ? U / 8 : LPP == 32 ? U / 4 : U / 2;
        double x[U / 2];
        if constexpr (LPP == 64) {
#pragma unroll
            for (int i = 0; i < U / 2; ++i) x[i] = pair_sum<32>(v[2 * i], v[2 * i + 1]);
#pragma unroll
            for (int i = 0; i < U / 4; ++i) x[i] = pair_sum<16>(x[2 * i], x[2 * i + 1]);
#pragma unroll
            for (int i = 0; i < U / 8; ++i) x[i] = pair_sum<8>(x[2 * i], x[2 * i + 1]);
        } else if constexpr (LPP == 32) {
#pragma unroll
            for (int i = 0; i < U / 2; ++i) x[i] = pair_sum<16>(v[2 * i], v[2 * i + 1]);
#pragma unroll
            for (int i = 0; i < U / 4; ++i) x[i] = pair_sum<8>(x[2 * i], x[2 * i + 1]);
        } else {
#pragma unroll
            for (int i = 0; i < U / 2; ++i) x[i] = pair_sum<8>(v[2 * i], v[2 * i + 1]);
        }
        const int b3 = lane >> 3 & 1, b4 = lane >> 4 & 1, b5 = lane >> 5;
#pragma unroll
        for (int i = 0; i < LEFT; ++i) {
            const double sum = sum8(x[i]);
            const int j = LPP == 64 ? 2 * (2 * (2 * i + b3) + b4) + b5 : LPP == 32 ? 2 * (2 * i + b3) + b4 : 2 * i + b3;
            const int p = s * B::STEP + j * PPI + group;
            const int pid = __shfl(id, min(p, 63), 64);
            if ((lane & 7) == i && p < count) scores[p] = pid >= 0 ? (float)sum : -__builtin_huge_valf();
        }
    }
}

// --------------------------------------------------------------- selection --
__device__ inline int wave_scan(int x) {              // inclusive, over the wave
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// the sum over the first 16 lanes, to all
__device__ inline int row_total(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    return __builtin_amdgcn_readlane(x, 15);
}

constexpr int kBins = 1024;           // bins of the scores' range
constexpr int kRanked = 256;          // keys of one bin that are ranked one against the other

// A workgroup per (KV head, request).  Thread t holds the keys of pages C t .. C t + C
// - 1 (the scores' bits in an order that unsigned comparison follows), so that a
// prefix sum over the threads is one over the pages.
//  1. The scores between the least and the greatest finite one are counted in kBins
//     equal bins (LDS atomics; whole numbers, so their order does not show; equal
//     widths of the value spread the atomics, while the top bits of the keys, sign and
//     exponent, are nearly all alike).  NaN and infinities count in the end bins.
//  2. From the top bin down: the bin in which the need-th score lies.  The pages of the
//     bins above are taken.
//  3. That bin's pages, a handful, are ranked one against the other by (key, page).
//     Should it hold more than kRanked (many equal scores), its need-th key is found
//     from the top bits down instead, two bits a round by three counts of ballots, and
//     ties are taken in order.
//  4. The pages taken are written in order.
// (The search by bits over all keys took 11-16 us a call: 16 rounds of 0.8 us.)
template <int NT, int C>
__global__ __launch_bounds__(NT) void select_kernel(SelectArgs a) {
    constexpr int NW = NT / 64;
    __shared__ uint32_t s_bins[kBins];
    __shared__ uint2 s_count[2][NW];                  // search by bits: per wave c1 | c2 << 16, c3
    __shared__ float2 s_range[NW];
    __shared__ uint2 s_cand[kRanked];                 // key, page
    __shared__ uint32_t s_taken[NT * C / 32];         // a bit per page of the bin: ranked high enough
    __shared__ int s_sum[NW], s_found[3], s_cands;
    const int h = blockIdx.x, r = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (a.seq_lens[r] < 0) return;                    // held
    const int n = resident_pages(a, r);
    int32_t *out = a.selected + ((size_t)r * a.Hkv + h) * a.budget;
    if (n <= a.budget) {
        for (int i = tid; i < a.budget; i += NT) out[i] = i < n ? i : -1;
        return;
    }
    const float *scores = a.scores + ((size_t)r * a.Hkv + h) * a.max_pages;
    // (all loads first: the compiler would put each behind its branch, and wait there.
    // A thread's last ones may lie past the row, in the next or in the workspace's end.)
    f32x4_t at[C / 4];
#pragma unroll
    for (int c = 0; c < C / 4; ++c) at[c] = *reinterpret_cast<const f32x4_e4_t *>(scores + min(C * tid, n - 1) + 4 * c);
    for (int i = tid; i < kBins; i += NT) s_bins[i] = 0;
    for (int i = tid; i < NT * C / 32; i += NT) s_taken[i] = 0;
    if (tid == 0) s_cands = 0;
#pragma unroll
    for (int c = 0; c < C / 4; ++c) __asm__ volatile("" : "+v"(at[c]));
    uint32_t kept = 0, cand = 0;                      // bit c: page C tid + c is taken whatever its score; has a score that counts
    constexpr float kInf = __builtin_huge_valf();
    float least = kInf, greatest = -kInf;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int p = C * tid + c;
        const float s = at[c / 4][c % 4];
        if (p < n) {
            if (p < a.keep_first || p >= n - a.keep_last) {
                kept |= 1u << c;
            } else {
                cand |= 1u << c;
                if (fabsf(s) < kInf) {
                    least = fminf(least, s);
                    greatest = fmaxf(greatest, s);
                }
            }
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        least = fminf(least, __shfl_xor(least, o, 64));
        greatest = fmaxf(greatest, __shfl_xor(greatest, o, 64));
    }
    if (lane == 0) s_range[wave] = make_float2(least, greatest);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        least = fminf(least, s_range[w].x);
        greatest = fmaxf(greatest, s_range[w].y);
    }
    // (a range past the largest float: its halves; every step below is monotonic in the score)
    const float scale = (kBins - 1) * 0.5f / fmaxf(0.5f * greatest - 0.5f * least, 1e-30f);
    auto bin_of = [&](float s) {
        if (s != s) return kBins - 1;
        return (int)fminf(fmaxf((0.5f * s - 0.5f * least) * (2.0f * scale), 0.0f), (float)(kBins - 1));
    };
    auto key_of = [&](float s) {
        const uint32_t u = __float_as_uint(s + 0.0f);     // (-0, what a small negative sum rounds to, ties with 0)
        return s != s ? 0xffffffffu : u ^ ((int)u < 0 ? 0xffffffffu : 0x80000000u);
    };
    int bin[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        bin[c] = bin_of(at[c / 4][c % 4]);
        if (cand >> c & 1) atomicAdd(&s_bins[bin[c]], 1u);
    }
    __syncthreads();
    const int need = a.budget - a.keep_first - a.keep_last;
    if (wave == 0 && need > 0) {                      // lane l: bins 16 l .. + 15
        static_assert(kBins == 1024, "sixteen bins per lane");
        int sum = 0, part[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            part[i] = s_bins[16 * lane + i];
            sum += part[i];
        }
        const int incl = wave_scan(sum), above = __builtin_amdgcn_readlane(incl, 63) - incl;   // in the bins of later lanes
        if (above < need && need <= above + sum) {    // (one lane: the candidates are more than need)
            int b = 0, over = above, acc = above;
            bool found = false;
#pragma unroll
            for (int i = 15; i >= 0; --i) {
                if (!found && acc + part[i] >= need) {
                    found = true;
                    b = 16 * lane + i;
                    over = acc;
                }
                acc += part[i];
            }
            s_found[0] = b;
            s_found[1] = over;
            s_found[2] = s_bins[b];
        }
    }
    __syncthreads();
    if (need > 0) {
        const int b = s_found[0], rest = need - s_found[1], members = s_found[2];   // rest: pages to take from bin b
        if (members <= kRanked) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (!(cand >> c & 1)) continue;
                if (bin[c] > b) kept |= 1u << c;
                if (bin[c] == b) s_cand[atomicAdd(&s_cands, 1)] = make_uint2(key_of(at[c / 4][c % 4]), C * tid + c);
            }
            __syncthreads();
            for (int i = tid; i < members; i += NT) {
                const uint2 x = s_cand[i];
                int rank = 0;
                for (int k = 0; k < members; ++k) {
                    const uint2 y = s_cand[k];
                    rank += y.x > x.x || (y.x == x.x && y.y < x.y) ? 1 : 0;
                }
                if (rank < rest) atomicOr(&s_taken[x.y / 32], 1u << x.y % 32);
            }
            __syncthreads();
            kept |= s_taken[C * tid / 32] >> C * tid % 32 & ((1u << C) - 1);
        } else {
            uint32_t key[C];                          // of the bin's pages; others 0, below every key
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if ((cand >> c & 1) && bin[c] > b) kept |= 1u << c;
                key[c] = (cand >> c & 1) && bin[c] == b ? key_of(at[c / 4][c % 4]) : 0u;
            }
            uint32_t T = 0;
            int above = 0;                            // keys above T
            for (int s = 30; s >= 0; s -= 2) {
                int c1 = 0, c2 = 0, c3 = 0;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    c1 += __popcll(__ballot(key[c] >= (T | 1u << s)));
                    c2 += __popcll(__ballot(key[c] >= (T | 2u << s)));
                    c3 += __popcll(__ballot(key[c] >= (T | 3u << s)));
                }
                if (lane == 0) s_count[s / 2 & 1][wave] = make_uint2(c1 | c2 << 16, c3);
                __syncthreads();
                const uint2 x = lane < NW ? s_count[s / 2 & 1][lane] : make_uint2(0, 0);
                const int lo = row_total(x.x);
                c1 = lo & 0xffff;
                c2 = (uint32_t)lo >> 16;
                c3 = row_total(x.y);
                // the digit of the rest-th key, and the keys above it
                if (c3 >= rest) {
                    T |= 3u << s;
                } else if (c2 >= rest) {
                    T |= 2u << s;
                    above = c3;
                } else if (c1 >= rest) {
                    T |= 1u << s;
                    above = c2;
                } else {
                    above = c1;
                }
            }
            // the pages above T, and the first of those equal to it
            int eq = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (key[c] > T) kept |= 1u << c;
                eq += key[c] == T ? 1 : 0;
            }
            const int incl = wave_scan(eq);
            if (lane == 63) s_sum[wave] = incl;
            __syncthreads();
            int tied = incl - eq;
            for (int w = 0; w < wave; ++w) tied += s_sum[w];
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (key[c] == T && tied++ < rest - above) kept |= 1u << c;
            __syncthreads();                          // s_sum is used again
        }
    }
    const int mine = __popc(kept), incl = wave_scan(mine);
    if (lane == 63) s_sum[wave] = incl;
    __syncthreads();
    int to = incl - mine;
    for (int w = 0; w < wave; ++w) to += s_sum[w];
#pragma unroll
    for (int c = 0; c < C; ++c)
        if ((kept >> c & 1) && to < a.budget) out[to++] = C * tid + c;
}

template <typename T, int D>
hipError_t launch_td(int G, SelectArgs a, hipStream_t s) {
    // two steps a wave, so that a long batch is several rounds of waves (48 requests of
    // 4096-32768 tokens, 32/8 heads, d 128: 46.9 us, four steps 49.6, one 48.8), but one
    // where that leaves less than a wave per slot of the chip (4096)
    a.wave_pages = std::min(kScorePages, 2 * Box<T, D>::STEP);
    if ((int64_t)a.R * a.Hkv * cdiv(a.max_pages, a.wave_pages) < 4096) a.wave_pages = Box<T, D>::STEP;
    // tables no wider than the budget: every page is selected
    if (a.max_pages > a.budget) {
        const dim3 grid((uint32_t)(((int64_t)a.Hkv * cdiv(a.max_pages, a.wave_pages) + kScoreWaves - 1) / kScoreWaves), a.R);
        switch (G) {
            case 1: score_kernel<T, D, 1><<<grid, 64 * kScoreWaves, 0, s>>>(a); break;
            case 2: score_kernel<T, D, 2><<<grid, 64 * kScoreWaves, 0, s>>>(a); break;
            case 4: score_kernel<T, D, 4><<<grid, 64 * kScoreWaves, 0, s>>>(a); break;
            case 8: score_kernel<T, D, 8><<<grid, 64 * kScoreWaves, 0, s>>>(a); break;
            default: return hipErrorInvalidValue;
        }
    }
    const dim3 grid(a.Hkv, a.R);
    if (a.max_pages <= 1024) select_kernel<256, 4><<<grid, 256, 0, s>>>(a);
    else if (a.max_pages <= 4096) select_kernel<512, 8><<<grid, 512, 0, s>>>(a);
    else select_kernel<1024, 8><<<grid, 1024, 0, s>>>(a);
    return hipGetLastError();
}

template <int CACHE, int D>
hipError_t launch_bounds_cd(const BoundsArgs &a, hipStream_t s) {
    // every workgroup walks its share of a request's pages: no more of them than
    // the widest request could use, and about 16384 in all
    const int64_t tasks = (int64_t)a.max_update * a.Hkv;
    const int64_t most = (tasks + kBoundWaves - 1) / kBoundWaves, fair = cdiv(16384, a.R);
    const dim3 grid((uint32_t)(most < fair ? most : fair), a.R);
    bounds_kernel<CACHE, D><<<grid, 64 * kBoundWaves, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_bounds(int cache, int D, const BoundsArgs &a, hipStream_t s) {
    if (cache == 1) return D == 128 ? launch_bounds_cd<1, 128>(a, s) : launch_bounds_cd<1, 64>(a, s);
    if (cache == 2) return D == 128 ? launch_bounds_cd<2, 128>(a, s) : launch_bounds_cd<2, 64>(a, s);
    return D == 128 ? launch_bounds_cd<4, 128>(a, s) : launch_bounds_cd<4, 64>(a, s);
}

hipError_t launch_select(gp_dtype_t dt, int D, int G, const SelectArgs &a, hipStream_t s) {
    if (dt == GP_BF16) return D == 128 ? launch_td<uint16_t, 128>(G, a, s) : launch_td<uint16_t, 64>(G, a, s);
    return D == 128 ? launch_td<float, 128>(G, a, s) : launch_td<float, 64>(G, a, s);
}

}  // namespace gp
