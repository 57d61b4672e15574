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
// page's keys and values.
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
// contiguous run of the slice.  CACHE: bytes of a pool element.
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
        float x[RPL][EU];
        if constexpr (CACHE == 1) {
            const uint8_t *src = reinterpret_cast<const uint8_t *>(a.k) + slice * kPage * D + u * EU;
            const float scale = a.k_scale[slice];
            u32x2_t w[RPL];
#pragma unroll
            for (int i = 0; i < RPL; ++i) w[i] = *reinterpret_cast<const u32x2_t *>(src + (i * RG + g) * D);
#pragma unroll
            for (int i = 0; i < RPL; ++i)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const auto y0 = __builtin_amdgcn_cvt_pk_f32_fp8(w[i][c], false), y1 = __builtin_amdgcn_cvt_pk_f32_fp8(w[i][c], true);
                    x[i][4 * c] = y0[0] * scale;
                    x[i][4 * c + 1] = y0[1] * scale;
                    x[i][4 * c + 2] = y1[0] * scale;
                    x[i][4 * c + 3] = y1[1] * scale;
                }
        } else {
            const E *src = reinterpret_cast<const E *>(a.k) + slice * kPage * D + u * EU;
            u32x4_t w[RPL];
#pragma unroll
            for (int i = 0; i < RPL; ++i) w[i] = load16(src + (i * RG + g) * D);
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

template <int CTRL>
__device__ inline double add_from(double x) {
    const long long b = __builtin_bit_cast(long long, x);
    const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xf, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xf, 0xf, false);
    return x + __builtin_bit_cast(double, (long long)hi << 32 | (unsigned)lo);
}
// the sum over a lane's group of eight, in all of them: xor 1, xor 2 (quad
// permutations), then the mirrored half row, which has the other quad's
__device__ inline double sum8(double x) { return add_from<0x141>(add_from<0x4e>(add_from<0xb1>(x))); }

// Eight lanes per page, eight pages per wave and step: lane l of a group takes the
// 16-byte units l, l + 8, .. of the page's box (least, then greatest values), so
// that a load instruction reads 128 bytes of each of eight pages and the sums meet in
// three exchanges.  The units' dims are the lane's own, so its part of Q+- stays in
// registers.  Grid (KV head and block of kScoreWaves x 64 pages, request).
constexpr int kScoreWaves = 4, kScorePages = 64;      // waves, and pages per wave
template <typename T, int D, int G>
__global__ __launch_bounds__(64 * kScoreWaves) void score_kernel(SelectArgs a) {
    constexpr int N = Unit<T>::N, UPL = D / N / 8;    // units of half a box per lane
    const int h = blockIdx.x % a.Hkv, r = blockIdx.y;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l = lane & 7, at = lane >> 3;
    const int n = resident_pages(a, r);
    const int p0 = ((int)(blockIdx.x / a.Hkv) * kScoreWaves + wave) * kScorePages;
    if (n <= a.budget || p0 >= n) return;             // all pages are selected; none for this wave
    int id = p0 + lane < n ? a.page_table[(size_t)r * a.max_pages + p0 + lane] : -1;
    if (id >= a.pool_pages) id = -1;
    double wn[UPL][N], wp[UPL][N];
#pragma unroll
    for (int i = 0; i < UPL; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) wn[i][e] = wp[i][e] = 0.0;
    const T *q = reinterpret_cast<const T *>(a.q) + ((size_t)r * a.Hkv + h) * G * D + l * N;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < UPL; ++i) {
            const u32x4_t x = load16(q + g * D + i * 8 * N);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const double y = Unit<T>::at(x, e);
                if (y < 0.0) wn[i][e] += y;
                else wp[i][e] += y;                   // (a NaN counts here)
            }
        }
    const T *boxes = reinterpret_cast<const T *>(a.bounds) + (size_t)h * 2 * D + l * N;
    float *scores = a.scores + ((size_t)r * a.Hkv + h) * a.max_pages + p0;
    const int steps = cdiv(min(kScorePages, n - p0), 8);
    for (int s = 0; s < steps; ++s) {
        const int pid = __shfl(id, s * 8 + at, 64);
        const T *box = boxes + (size_t)max(pid, 0) * a.Hkv * 2 * D;
        u32x4_t lo[UPL], hi[UPL];
#pragma unroll
        for (int i = 0; i < UPL; ++i) {
            lo[i] = load16(box + i * 8 * N);
            hi[i] = load16(box + D + i * 8 * N);
        }
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < UPL; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                sum = __builtin_fma((double)Unit<T>::at(lo[i], e), wn[i][e], sum);
                sum = __builtin_fma((double)Unit<T>::at(hi[i], e), wp[i][e], sum);
            }
        sum = sum8(sum);
        if (__any(sum != sum)) {                      // rare: a zero factor meets an infinite bound, and adds nothing
            double t = 0.0;
#pragma unroll
            for (int i = 0; i < UPL; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (wn[i][e] != 0.0) t = __builtin_fma((double)Unit<T>::at(lo[i], e), wn[i][e], t);
                    if (wp[i][e] != 0.0) t = __builtin_fma((double)Unit<T>::at(hi[i], e), wp[i][e], t);
                }
            sum = sum8(t);
        }
        if (l == 0 && p0 + s * 8 + at < n) scores[s * 8 + at] = pid < 0 ? -__builtin_huge_valf() : (float)sum;
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

// A workgroup per (KV head, request).  Thread t holds the keys of pages C t .. C t + C
// - 1 (the scores' bits in an order that unsigned comparison follows), so that a
// prefix sum over the threads is one over the pages.  The need-th largest key is
// found from its top bits down, two bits a round: three counts of keys at or above a
// threshold, by ballots (a histogram in LDS would take nearly all pages in one bin:
// scores share their sign and exponent).  Then those above it and the first of those
// equal to it are written in order.
template <int NT, int C>
__global__ __launch_bounds__(NT) void select_kernel(SelectArgs a) {
    constexpr int NW = NT / 64;
    __shared__ int s_count[2][NW][3];
    __shared__ int s_sum[NW];
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
    uint32_t key[C];
    uint32_t kept = 0;                                // bit c: page C tid + c is taken whatever its score
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int p = C * tid + c;
        key[c] = 0;
        if (p < n) {
            if (p < a.keep_first || p >= n - a.keep_last) {
                kept |= 1u << c;
            } else {
                const float s = scores[p];
                const uint32_t u = __float_as_uint(s);
                key[c] = s != s ? 0xfffffffeu : u ^ ((int)u < 0 ? 0xffffffffu : 0x80000000u);
            }
        }
    }
    const int need = a.budget - a.keep_first - a.keep_last;
    uint32_t T = 0;
    int above = 0;                                    // keys above T
    if (need == 0) {
        T = 0xffffffffu;
    } else {
        for (int s = 30; s >= 0; s -= 2) {
            int c1 = 0, c2 = 0, c3 = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                c1 += __popcll(__ballot(key[c] >= (T | 1u << s)));
                c2 += __popcll(__ballot(key[c] >= (T | 2u << s)));
                c3 += __popcll(__ballot(key[c] >= (T | 3u << s)));
            }
            int(&cnt)[NW][3] = s_count[s / 2 & 1];
            if (lane == 0) {
                cnt[wave][0] = c1;
                cnt[wave][1] = c2;
                cnt[wave][2] = c3;
            }
            __syncthreads();
            c1 = c2 = c3 = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                c1 += cnt[w][0];
                c2 += cnt[w][1];
                c3 += cnt[w][2];
            }
            // the keys above the digit taken
            if (c3 >= need) {
                T |= 3u << s;
            } else if (c2 >= need) {
                T |= 2u << s;
                above = c3;
            } else if (c1 >= need) {
                T |= 1u << s;
                above = c2;
            } else {
                above = c1;
            }
        }
    }
    const int ties = need - above;                    // pages of key T that are taken
    int gt = 0, eq = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        gt += (kept >> c & 1) || key[c] > T ? 1 : 0;
        eq += key[c] == T && !(kept >> c & 1) ? 1 : 0;
    }
    const int both = gt | eq << 16, incl = wave_scan(both);
    if (lane == 63) s_sum[wave] = incl;
    __syncthreads();
    int before = incl - both;
    for (int w = 0; w < wave; ++w) before += s_sum[w];
    int taken = before & 0xffff, tied = before >> 16;
    taken += min(tied, ties);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        bool in = (kept >> c & 1) || key[c] > T;
        if (!in && key[c] == T && C * tid + c < n) {
            in = tied < ties;
            ++tied;
        }
        if (in && taken < a.budget) out[taken++] = C * tid + c;
    }
}

template <typename T, int D>
hipError_t launch_td(int G, const SelectArgs &a, hipStream_t s) {
    // tables no wider than the budget: every page is selected
    if (a.max_pages > a.budget) {
        const dim3 grid(a.Hkv * cdiv(a.max_pages, kScoreWaves * kScorePages), a.R);
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
