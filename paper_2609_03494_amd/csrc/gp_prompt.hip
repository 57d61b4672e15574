// Attention of new tokens over the paged cache (gp_prompt_attention; Sec. 3.1
// attention-output equation with a causal limit): whole prompts, chunks behind a
// context, drafted tokens.
//
// Work item: one KV head and kRows rows of one request, a row being a (new token, query
// head of that KV head) pair: the G heads of a token read the same keys, so they lie
// side by side and the causal border of an item is kRows / G tokens wide.  A wave has 32
// rows.  Keys and values come in tiles of Tile::TOK tokens through two LDS stages, one
// filled (from registers, so that the loads of a tile are in flight during the one
// before) while the other is read.
//
// Products, both transposed: S^T = K Q^T, then O^T += V^T P^T, on 32 x 32 matrix
// instructions.  A lane then holds scores of one row only (its column), so maxima and
// sums are in-lane but for one exchange with lane ^ 32, the rescaling of O^T is in-lane
// as well, and the scores become the second product's operand without moving: lane half
// h has tokens 8 k + 4 h + 0..3 of every 16, and V^T is read in that order.
#include <float.h>

#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "gp_internal.h"

namespace gp {

namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef short s16x4_t __attribute__((ext_vector_type(4)));
// as a caller's buffers may lie: at any multiple of the element
typedef u32x4_t u32x4_e2_t __attribute__((aligned(2)));
typedef u32x4_t u32x4_e4_t __attribute__((aligned(4)));
typedef u32x2_t u32x2_e2_t __attribute__((aligned(2)));

constexpr float kNegInf = -__builtin_huge_valf();
constexpr int kWaves = 4, kThreads = 64 * kWaves;
static_assert(kPromptRows == 32 * kWaves, "rows of an item");

__device__ inline int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int scalar_load(const int32_t *p, int64_t i) {
    return ((const __attribute__((address_space(4))) int32_t *)p)[i];
}
__device__ inline float scalar_load(const float *p, int64_t i) {
    return ((const __attribute__((address_space(4))) float *)p)[i];
}
__device__ inline u32x4_t load16(const uint16_t *p) { return *reinterpret_cast<const u32x4_e2_t *>(p); }
__device__ inline u32x4_t load16(const float *p) { return *reinterpret_cast<const u32x4_e4_t *>(p); }
__device__ inline float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// x where at < 0, else -inf (in vector registers alone: 32 compares would take 64 scalar ones)
__device__ inline float masked(float x, int at) {
    const uint32_t keep = (uint32_t)(at >> 31);
    return __uint_as_float((__float_as_uint(x) & keep) | (0xff800000u & ~keep));
}
__device__ inline uint32_t pack_bf16(float a, float b) {             // to nearest even
    const bf16x2_t x = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, x);
}

// 16 bytes a lane from base + off to LDS, `to` + 16 lane, past the registers.  Written as
// assembly since the compiler makes every LDS read wait for all such loads in flight,
// those into the other stage included; here the wave waits for them (kWaitVm0) before
// the barrier that hands the stage over.  No register is written.
__device__ inline void load_lds(const void *base, uint32_t off, uint32_t to) {
    __asm__ volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(to) : "memory");
}
__device__ inline uint32_t lds_addr(const void *p) {
    return (uint32_t)(size_t)(__attribute__((address_space(3))) const char *)p;
}
constexpr int kWaitVm0 = 0x0F70;                                     // s_waitcnt vmcnt(0)

// CACHE: bytes of a pool element (1: e4m3 codes, as bfloat16 in LDS).
template <int CACHE, int D>
struct Tile {
    static constexpr int LB = CACHE == 4 ? 4 : 2;                    // bytes of an element in LDS
    static constexpr int TOK = CACHE == 4 && D == 128 ? 32 : 64;     // tokens of a tile
    static constexpr int ROWB = D * LB, UPR = ROWB / 16;             // bytes and 16-byte units of a token
    static constexpr int BYTES = TOK * ROWB;                         // of the keys, or the values
    static constexpr int PAGES = TOK / kPage;
    static constexpr int PU = D * CACHE;                             // 16-byte units of a page in the pool
    static constexpr int LOADS = PAGES * PU / kThreads;              // units of a thread
    static constexpr int PUR = PU / kPage;                           // units of a token in the pool
    static_assert(PU % 64 == 0 && LOADS * kThreads == PAGES * PU, "a wave's unit lies in one page");
    // XOR-swizzle of a token's units.  Keys: 32 lanes read one unit of 32 tokens.  Values,
    // 16 bits: 32 lanes read 64 bytes of each of four tokens (transposed); 32 bits: 32 lanes
    // 128 bytes of one token, the other lanes of the fourth after it.
    __device__ static int key_swizzle(int t) { return UPR >= 16 ? t & 15 : (t >> 1) & 7; }
    __device__ static int value_swizzle(int t) {
        if (CACHE == 4) return ((t >> 2) & 1) * 8;
        return UPR >= 16 ? (t & 3) * 4 : ((t >> 1) & 1) * 4;
    }
};

// What a request brings to the call.
struct Asked {
    int ts, n, before;        // first token's row, tokens, resident tokens that precede them
    bool in;                  // the request takes part
};
__device__ inline Asked asked(const PromptArgs &a, int r) {
    Asked q;
    q.ts = r;
    int te = r + 1;
    if (a.start) {
        q.ts = min(max(a.start[r], 0), a.T);
        te = min(max(a.start[r + 1], q.ts), a.T);
    }
    q.n = te - q.ts;
    const int m = a.seq_lens[r], P = min(max(a.num_pages[r], 0), a.max_pages);
    q.in = m >= 0;
    q.before = min(m, P * kPage) - (a.advanced ? q.n : 0);
    // without room for all of them none went in: no keys
    if (!a.advanced && q.n > P * kPage - m) q.before = INT_MIN / 2;
    return q;
}

// the last request whose first place is at or before i (every lane the same)
__device__ inline int request_at(const PromptArgs &a, int i, int lane) {
    int lo = 0, hi = a.R;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, r = lo + lane * step;
        const bool at = r < hi && max(a.start[min(r, a.R)], 0) / a.tokens + r <= i;
        const int n = max(__popcll(__ballot(at)), 1);
        lo += (n - 1) * step;
        hi = min(hi, lo + step);
    }
    return uni(lo);
}

template <int CACHE, int D>
__global__ __launch_bounds__(kThreads, 2) void prompt_kernel(PromptArgs a) {
    using TL = Tile<CACHE, D>;
    using E = typename std::conditional<CACHE == 4, float, uint16_t>::type;
    constexpr int TOK = TL::TOK, TB = TOK / 32, DB = D / 32, LOADS = TL::LOADS;
    constexpr int QS = CACHE == 4 ? D / 8 : D / 16;                  // 16-byte pieces of a row per lane
    __shared__ __attribute__((aligned(16))) unsigned char s_k[2][TL::BYTES];
    __shared__ __attribute__((aligned(16))) unsigned char s_v[2][TL::BYTES];
    __shared__ int s_odd[2];                                         // the tile whose values are not all finite
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int h = blockIdx.x % a.Hkv, place = blockIdx.x / a.Hkv;
    int r = place, j0 = 0;
    if (a.start) {
        r = request_at(a, place, lane);
        j0 = (place - (max(scalar_load(a.start, r), 0) / a.tokens + r)) * a.tokens;
    }
    const Asked rq = asked(a, r);
    if (!rq.in || j0 < 0 || j0 >= rq.n) return;
    const int rows = min(a.tokens, rq.n - j0) << a.lg;               // of this item
    const int first = rq.before + j0 + 1, last = rq.before + j0 + (rows >> a.lg);   // tokens that its first and last row see
    const int tiles = last > 0 ? (last + TOK - 1) / TOK : 0;
    const int last_page = max(last - 1, 0) / kPage;

    // the wave's rows: a lane's row is its column of S^T and O^T
    const int col = lane & 31, half = lane >> 5;
    const int row = wave * 32 + col, at = min(row, rows - 1);
    const int sees = rq.before + j0 + (at >> a.lg) + 1;
    const int wave_first = rq.before + j0 + (min(wave * 32, rows - 1) >> a.lg) + 1;
    const int wave_last = wave * 32 < rows ? rq.before + j0 + (min(wave * 32 + 31, rows - 1) >> a.lg) + 1 : 0;
    const int64_t token = rq.ts + j0 + (at >> a.lg);
    const int head = h * a.G + (at & (a.G - 1));
    u32x4_t q[QS];
    {
        const E *src = reinterpret_cast<const E *>(a.q) + token * a.q_stride + (int64_t)head * D + half * (16 / (int)sizeof(E));
#pragma unroll
        for (int s = 0; s < QS; ++s) q[s] = load16(src + s * (32 / (int)sizeof(E)));
    }

    // a tile's way from the pools to LDS: a wave takes LOADS pieces of 1024 bytes each of
    // the keys and the values, 8-bit ones through registers, where they are widened
    const int32_t *table = a.page_table + (size_t)r * a.max_pages;
    const size_t slice = (size_t)h * kPage * D * CACHE, page_bytes = (size_t)a.Hkv * kPage * D * CACHE;
    u32x4_t kr[CACHE == 1 ? LOADS : 1], vr[CACHE == 1 ? LOADS : 1];
    float ks[2][TL::PAGES], vs[2][TL::PAGES];                        // 8-bit: scales, of the tile in work and the next
    int ids[LOADS], pids[TL::PAGES];                                 // pages of the next pieces; 8-bit: of the next tile
    auto page_of = [&](int tile, int pg) { return scalar_load(table, min(tile * TL::PAGES + pg, last_page)); };
    auto inside = [&](int id) { return min(max(id, 0), a.pool_pages - 1); };
    auto request = [&](int tile) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) ids[i] = page_of(tile, (i * kThreads + wave * 64) / TL::PU);
        if constexpr (CACHE == 1)
#pragma unroll
            for (int p = 0; p < TL::PAGES; ++p) pids[p] = page_of(tile, p);
    };
    auto load = [&](int buf) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int piece = i * kWaves + wave;
            const size_t from = inside(ids[i]) * page_bytes + slice + (size_t)(piece * 64 % TL::PU) * 16;
            const char *kp = static_cast<const char *>(a.k) + from, *vp = static_cast<const char *>(a.v) + from;
            if constexpr (CACHE == 1) {
                kr[i] = reinterpret_cast<const u32x4_t *>(kp)[lane];
                vr[i] = reinterpret_cast<const u32x4_t *>(vp)[lane];
            } else {
                // the unit that belongs at the lane's place in LDS
                const int t = (piece * 64 + lane) / TL::UPR, c = lane % TL::UPR;
                const int ku = (lane & ~(TL::UPR - 1)) + (c ^ TL::key_swizzle(t)), vu = (lane & ~(TL::UPR - 1)) + (c ^ TL::value_swizzle(t));
                load_lds(kp, ku * 16, lds_addr(s_k[buf] + piece * 1024));
                load_lds(vp, vu * 16, lds_addr(s_v[buf] + piece * 1024));
            }
        }
        if constexpr (CACHE == 1) {
#pragma unroll
            for (int p = 0; p < TL::PAGES; ++p) {
                const int64_t sc = (int64_t)inside(pids[p]) * a.Hkv + h;
                ks[1][p] = scalar_load(a.k_scale, sc);
                vs[1][p] = scalar_load(a.v_scale, sc);
            }
        }
    };
    auto widen = [](uint32_t x0, uint32_t x1, float scale) {
        const bf16x2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x0, scale, false), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x0, scale, true);
        const bf16x2_t p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x1, scale, false), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x1, scale, true);
        return u32x4_t{__builtin_bit_cast(uint32_t, p0), __builtin_bit_cast(uint32_t, p1), __builtin_bit_cast(uint32_t, p2), __builtin_bit_cast(uint32_t, p3)};
    };
    auto odd = [](const u32x4_t &x) {                                // infinite or NaN among the elements
        bool is = false;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (CACHE == 4) is |= (x[c] & 0x7f800000u) == 0x7f800000u;
            else is |= (x[c] & 0x7f80u) == 0x7f80u || (x[c] & 0x7f800000u) == 0x7f800000u;
        }
        return is;
    };
    // the loaded tile stands in LDS after this and a barrier.  border: some row does not see
    // all of its tokens: values behind the request's tokens become zero (whatever lies there),
    // and a tile is marked that has infinite values or NaN among the others
    auto settle = [&](int tile, int buf, bool border) {
        bool found = false;
        if constexpr (CACHE == 1) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int u = i * kThreads + tid, t = u / TL::PUR, c = u % TL::PUR;
                u32x4_t *kt = reinterpret_cast<u32x4_t *>(s_k[buf] + t * TL::ROWB), *vt = reinterpret_cast<u32x4_t *>(s_v[buf] + t * TL::ROWB);
                const int sk = TL::key_swizzle(t), sv = TL::value_swizzle(t);
                if (border && tile * TOK + t >= last) vr[i] = u32x4_t{};
                constexpr float unit = 1.0f / kQ8KeyScale;           // (see Page<E4m3>::kKeyUnit of the decode kernel)
                const u32x4_t v0 = widen(vr[i][0], vr[i][1], 1.0f), v1 = widen(vr[i][2], vr[i][3], 1.0f);
                kt[(2 * c) ^ sk] = widen(kr[i][0], kr[i][1], unit);
                kt[(2 * c + 1) ^ sk] = widen(kr[i][2], kr[i][3], unit);
                vt[(2 * c) ^ sv] = v0;
                vt[(2 * c + 1) ^ sv] = v1;
                if (border) found |= odd(v0) || odd(v1);
            }
        } else {
            __builtin_amdgcn_s_waitcnt(kWaitVm0);
            if (border) {
                __asm__ volatile("" ::: "memory");
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    const int u = (i * kWaves + wave) * 64 + lane;
                    u32x4_t *at = reinterpret_cast<u32x4_t *>(s_v[buf]) + u;
                    if (tile * TOK + u / TL::UPR >= last) *at = u32x4_t{};
                    else found |= odd(*at);
                }
            }
        }
        if (border && __any(found) && lane == 0) s_odd[buf] = tile;
    };
    auto on_border = [&](int tile) { return (tile + 1) * TOK > first; };

    f32x16_t o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = f32x16_t{};
    float m = kNegInf, l = 0.0f;                                     // the row's maximum (both halves the same), this half's sum
    if (tid < 2) s_odd[tid] = -1;
    if (tiles > 0) {
        request(0);
        load(0);
        request(1);
    }
    __syncthreads();
    if (tiles > 0) settle(0, 0, on_border(0));
    __syncthreads();
    for (int tile = 0; tile < tiles; ++tile) {
        const int buf = tile & 1;
        if constexpr (CACHE == 1) {
#pragma unroll
            for (int p = 0; p < TL::PAGES; ++p) {
                ks[0][p] = ks[1][p];
                vs[0][p] = vs[1][p];
            }
        }
        if (tile + 1 < tiles) {
            load(buf ^ 1);
            request(tile + 2);
        }
        if (tile * TOK < wave_last) {
            // S^T
            f32x16_t st[TB];
            const unsigned char *kb = s_k[buf] + col * TL::ROWB;
            const int sw = TL::key_swizzle(col);
#pragma unroll
            for (int tb = 0; tb < TB; ++tb) {
                st[tb] = f32x16_t{};
#pragma unroll
                for (int s = 0; s < QS; ++s) {
                    const u32x4_t x = *reinterpret_cast<const u32x4_t *>(kb + tb * 32 * TL::ROWB + (((2 * s + half) ^ sw) << 4));
                    if constexpr (CACHE == 4) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            st[tb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[e]), __uint_as_float(q[s][e]), st[tb], 0, 0, 0);
                    } else {
                        st[tb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x), __builtin_bit_cast(bf16x8_t, q[s]), st[tb], 0, 0, 0);
                    }
                }
            }
            // (8-bit: in units of log2, with the page's scale; the others' scale comes with the difference)
            if constexpr (CACHE == 1) {
#pragma unroll
                for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) st[tb][i] *= __builtin_amdgcn_fmed3f(a.qscale * ks[0][2 * tb + i / 8], FLT_TRUE_MIN, FLT_MAX);
            }
            const float unit = CACHE == 1 ? 1.0f : a.qscale;
            if ((tile + 1) * TOK > wave_first) {
                const int left = sees - tile * TOK - 4 * half;       // tokens of the tile that the row sees, from this half's first on
#pragma unroll
                for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        st[tb][i] = masked(st[tb][i], tb * 32 + 8 * (i / 4) + i % 4 - left);
            }
            float top = st[0][0];
#pragma unroll
            for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, st[tb][i]);
            top = max_halves(top);
            // (a maximum may lag by 8 in log2: weights up to 2^8, relative errors as they are)
            if (__any(top * unit > m * unit + 8.0f)) {
                const float up = fmaxf(m, top), f = m == kNegInf ? 0.0f : __builtin_amdgcn_exp2f((m - up) * unit);
                l *= f;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= f;
                m = up;
            }
            const float from = m == kNegInf ? 0.0f : m * unit;       // (a row that sees nothing yet)
#pragma unroll
            for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    st[tb][i] = __builtin_amdgcn_exp2f(fmaf(st[tb][i], unit, -from));
                    l += st[tb][i];
                }
            if constexpr (CACHE == 1) {
#pragma unroll
                for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) st[tb][i] *= vs[0][2 * tb + i / 8];
            }
            // O^T
            const bool odd_values = uni(s_odd[buf]) == tile;
            const unsigned char *vb = s_v[buf];
            if constexpr (CACHE == 4) {
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    auto value = [&](int tb, int i) {
                        const int t = tb * 32 + 8 * (i / 4) + 4 * half + i % 4, u = (d * 32 + col) / 4;
                        return *reinterpret_cast<const float *>(vb + t * TL::ROWB + ((u ^ TL::value_swizzle(t)) << 4) + (col & 3) * 4);
                    };
                    if (odd_values) {
                        for (int part = 0; part < 3; ++part) {       // finite values; where +inf or NaN, where -inf or NaN
                            f32x16_t y = {};
#pragma unroll
                            for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    const float x = value(tb, i);
                                    const bool mine = x != x || x == (part == 1 ? __builtin_huge_valf() : kNegInf);
                                    const float z = part == 0 ? (fabsf(x) < __builtin_huge_valf() ? x : 0.0f) : mine ? 1.0f : 0.0f;
                                    y = __builtin_amdgcn_mfma_f32_32x32x2f32(z, st[tb][i], y, 0, 0, 0);
                                }
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[d][i] += part == 0 ? y[i] : y[i] > 0.0f ? (part == 1 ? __builtin_huge_valf() : kNegInf) : 0.0f;
                        }
                    } else {
#pragma unroll
                        for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(value(tb, i), st[tb][i], o[d], 0, 0, 0);
                    }
                }
            } else {
                u32x4_t p[2 * TB];
#pragma unroll
                for (int k = 0; k < 2 * TB; ++k)
#pragma unroll
                    for (int c = 0; c < 4; ++c) p[k][c] = pack_bf16(st[k / 2][8 * (k % 2) + 2 * c], st[k / 2][8 * (k % 2) + 2 * c + 1]);
                // lane j of a group of 16 names four dims of token j / 4 and receives dim j of the four tokens
                const int g = (lane >> 4) & 1, tt = 4 * half + ((lane & 15) >> 2), cc = 2 * g + ((lane & 3) >> 1);
                const uint32_t v0 = (uint32_t)(tt * TL::ROWB + ((cc ^ TL::value_swizzle(tt)) << 4) + (lane & 1) * 8);
                typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;
                auto read = [&](int k, int d) {                      // values of k-step k, dims 32 d ..: V^T's operand
                    // (units 4 d of a token: the swizzle flips units of 4, which 4 d xors with)
                    const unsigned char *x = vb + (v0 ^ (uint32_t)(d << 6)) + k * 16 * TL::ROWB;
                    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(x));
                    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(x + 8 * TL::ROWB));
                    const u32x2_t y0 = __builtin_bit_cast(u32x2_t, lo), y1 = __builtin_bit_cast(u32x2_t, hi);
                    return u32x4_t{y0[0], y0[1], y1[0], y1[1]};
                };
                if (odd_values) {
#pragma unroll
                    for (int d = 0; d < DB; ++d)
                        for (int part = 0; part < 3; ++part) {       // finite values; where +inf or NaN, where -inf or NaN
                            f32x16_t y = {};
#pragma unroll
                            for (int k = 0; k < 2 * TB; ++k) {
                                u32x4_t x = read(k, d);
#pragma unroll
                                for (int c = 0; c < 4; ++c) {
                                    uint32_t z = 0;
#pragma unroll
                                    for (int s = 0; s < 32; s += 16) {
                                        const uint32_t e = (x[c] >> s) & 0xffff, size = e & 0x7fff;
                                        const bool mine = size > 0x7f80 || e == (part == 1 ? 0x7f80u : 0xff80u);
                                        z |= part == 0 ? (size < 0x7f80 ? e << s : 0u) : mine ? 0x3f80u << s : 0u;
                                    }
                                    x[c] = z;
                                }
                                y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x), __builtin_bit_cast(bf16x8_t, p[k]), y, 0, 0, 0);
                            }
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[d][i] += part == 0 ? y[i] : y[i] > 0.0f ? (part == 1 ? __builtin_huge_valf() : kNegInf) : 0.0f;
                        }
                } else {
#pragma unroll
                    for (int k = 0; k < 2 * TB; ++k)
#pragma unroll
                        for (int d = 0; d < DB; ++d)
                            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, read(k, d)), __builtin_bit_cast(bf16x8_t, p[k]), o[d], 0, 0, 0);
                }
            }
        }
        if (tile + 1 < tiles) settle(tile + 1, buf ^ 1, on_border(tile + 1));
        __syncthreads();
    }
    l = sum_halves(l);
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    if (row < rows) {
        E *to = reinterpret_cast<E *>(a.out) + (token * a.Hkv * a.G + head) * D + 4 * half;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) x[c] = l > 0.0f ? o[d][4 * i + c] * inv : 0.0f;
                if constexpr (CACHE == 4)
                    *reinterpret_cast<u32x4_e4_t *>(to + 32 * d + 8 * i) = u32x4_t{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
                else
                    *reinterpret_cast<u32x2_e2_t *>(to + 32 * d + 8 * i) = u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
            }
    }
}

}  // namespace

hipError_t launch_prompt(int cache, int D, const PromptArgs &a, hipStream_t s) {
    const int grid = a.places * a.Hkv;
    if (cache == 1) D == 128 ? prompt_kernel<1, 128><<<grid, kThreads, 0, s>>>(a) : prompt_kernel<1, 64><<<grid, kThreads, 0, s>>>(a);
    else if (cache == 2) D == 128 ? prompt_kernel<2, 128><<<grid, kThreads, 0, s>>>(a) : prompt_kernel<2, 64><<<grid, kThreads, 0, s>>>(a);
    else D == 128 ? prompt_kernel<4, 128><<<grid, kThreads, 0, s>>>(a) : prompt_kernel<4, 64><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace gp
