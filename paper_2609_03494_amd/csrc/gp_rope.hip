// New tokens into the paged cache with the position rotation on the way
// (gp_append_rope; Sec. 3.1 paged cache): the decode step's tokens as well as
// whole prompts, into bfloat16, float32 and 8-bit pools.
//
// Rotation.  Pair (x_i, x_{i + d/2}) turns by t theta^(-2 i / d).  The angle is
// kept as a number of turns in 64 bits, t * (theta^(-2 i / d) / 2 pi) less its
// nearest integer, so that far positions lose nothing, and its cosine and sine are
// taken in 64 bits and rounded once to float32; the products are rounded one at
// a time, as a plain float32 evaluation rounds them.
//
// Work item: a page's worth of one request's new tokens (those that fall into
// one page of 16 slots), so that the 16 x d/2 cosines and sines are made once per
// workgroup, in LDS, for all query and key heads, and an 8-bit page's scale is
// found where all of its rows are at hand.  Request r's items are the grid's
// places start_r / 16 + 2 r and on: its n_r tokens touch at most n_r / 16 + 2 pages
// (integer division), which is no more than to the next request's first place, so
// a workgroup finds its request by a search over `start` alone and the lengths
// never visit the host.  blockIdx.y splits the heads of an item where there are few
// items.
//
// Bound: HBM for prompts (every row read once and written once): 42 k tokens of 64/8
// heads, d 128, bfloat16 take 339 us for 1.73 GB, 5.1 TB/s (a device copy of 2 GiB
// reaches 4.9); 42 k of 32/8 in float32 365 us for 1.81 GB, 5.0 TB/s; 8-bit chunks 135 us
// for 0.70 GB, 5.2 TB/s.  Latency for the tokens of a step: 3.6 us, 8 bits 6.2 (load, the
// page's maximum, old codes, store); advancing the lengths is a launch of its own, 1.4 us.
#include <algorithm>
#include <type_traits>

#include "gp_internal.h"

namespace gp {

namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef u32x4_t u32x4_e2_t __attribute__((aligned(2)));
typedef u32x4_t u32x4_e4_t __attribute__((aligned(4)));
template <typename E>
using Piece = typename std::conditional<sizeof(E) == 4, u32x4_e4_t, u32x4_e2_t>::type;
// 16 bytes; STREAM: past the caches
template <bool STREAM, typename E>
__device__ inline u32x4_t load16(const E *p) {
    if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const Piece<E> *>(p));
    else return *reinterpret_cast<const Piece<E> *>(p);
}
template <bool STREAM, typename E>
__device__ inline void store16(E *p, const u32x4_t &x) {
    if constexpr (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<Piece<E> *>(p));
    else *reinterpret_cast<Piece<E> *>(p) = x;
}

// the elements of 16 bytes, widened, and back
__device__ inline void widen(const u32x4_t &u, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(u[i]);
        x[2 * i + 1] = bf16_hi(u[i]);
    }
}
__device__ inline void widen(const u32x4_t &u, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(u[i]);
}
__device__ inline u32x4_t narrow(const float (&x)[8]) {
    u32x4_t u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __bf16 lo = (__bf16)x[2 * i], hi = (__bf16)x[2 * i + 1];     // round to nearest even
        u[i] = __builtin_bit_cast(uint16_t, lo) | (uint32_t)__builtin_bit_cast(uint16_t, hi) << 16;
    }
    return u;
}
__device__ inline u32x4_t narrow(const float (&x)[4]) {
    u32x4_t u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(x[i]);
    return u;
}

// one rotary pair, products and sums rounded one at a time
__device__ inline void rotate(float &a, float &b, const float2 &cs) {
#pragma clang fp contract(off)
    const float x = a * cs.x - b * cs.y, y = b * cs.x + a * cs.y;
    a = x;
    b = y;
}

// What a request brings: tokens [ts, ts + n), its resident length m (< 0: held),
// and whether they go into the cache.
struct Brought {
    int ts, n, m;
    bool room;
};
__device__ inline Brought brought(const RopeArgs &a, int r) {
    Brought b;
    b.ts = r;
    int te = r + 1;
    if (a.start) {
        b.ts = min(max(a.start[r], 0), a.T);
        te = min(max(a.start[r + 1], b.ts), a.T);
    }
    b.n = te - b.ts;
    b.m = a.seq_lens[r];
    const int P = a.num_pages[r];
    b.room = b.m >= 0 && P > 0 && P <= a.max_pages && b.m <= P * kPage && b.n <= P * kPage - b.m;
    return b;
}

// the last request whose first place is at or before i (every lane the same)
__device__ inline int request_at(const RopeArgs &a, int i, int lane) {
    int lo = 0, hi = a.R;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, r = lo + lane * step;
        const bool at = r < hi && (a.start[min(r, a.R)] >> 4) + 2 * r <= i;
        const int n = max(__popcll(__ballot(at)), 1);
        lo += (n - 1) * step;
        hi = min(hi, lo + step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

__device__ inline float wave_max(float x) {
#pragma unroll
    for (int o = 32; o > 0; o /= 2) x = fmaxf(x, __shfl_xor(x, o, 64));
    return x;
}

// 2^e with the least e >= -100 for which amax <= 448 2^e; 448 = 1.75 2^8
__device__ inline float scale_for(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffff) > 0x600000 ? 1 : 0);
    return __uint_as_float((uint32_t)(max(e, -100) + 127) << 23);
}
// the least power of two that is no less than a page's older scale (at most 2^127)
__device__ inline float power_from(float old) {
    const uint32_t u = __float_as_uint(old);
    return __uint_as_float(u & 0x7fffff ? min((u & 0x7f800000u) + 0x800000u, 0x7f000000u) : u);
}
__device__ inline uint32_t codes(float a, float b, float c, float d) {
    int u = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);              // round to nearest even
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, u, true);
}

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kBatch = 4;                             // row pieces in flight per thread

// CACHE: bytes of a pool element.  STREAM: the call moves more than the last-level
// cache holds (see launch_cd).
template <int CACHE, int D, bool STREAM>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
    using E = typename std::conditional<CACHE == 4, float, uint16_t>::type;
    constexpr int EPU = 16 / (int)sizeof(E);          // elements per 16 bytes
    constexpr int H = D / 2, UPH = H / EPU;           // rotary pairs; 16-byte units of half a row
    __shared__ float2 s_cs[kPage][H];                 // cosine, sine
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int item = blockIdx.x;
    int r = item, j = 0;
    if (a.start) {
        r = request_at(a, item, lane);
        j = item - ((a.start[r] >> 4) + 2 * r);
        if (j < 0 || j > a.T / kPage + 2) return;     // (starts that break the contract)
    }
    const Brought b = brought(a, r);
    if (b.m < 0) return;                              // held
    const int in_page = b.m % kPage;
    const int lo = j == 0 ? in_page : 0, first = j == 0 ? 0 : j * kPage - in_page;   // first slot, first token
    const int rows = min(kPage - lo, b.n - first);
    if (rows <= 0) return;
    const int64_t tok = b.ts + first;
    int pid = -1;
    if (b.room) {
        pid = a.page_table[(size_t)r * a.max_pages + b.m / kPage + j];
        if (pid < 0 || pid >= a.pool_pages) pid = -1;
    }
    const double pos = (double)a.positions[r] + 1.0 + first;
    for (int i = tid; i < rows * H; i += kThreads) {
        const double t = (pos + i / H) * a.turns[i % H];
        double s, c;
        sincospi(2.0 * (t - rint(t)), &s, &c);
        s_cs[i / H][i % H] = make_float2((float)c, (float)s);
    }
    __syncthreads();

    // rows that go out in their own type, in pieces of two 16-byte units that
    // rotate into each other: the queries, and the keys and values of such a pool
    {
        const int kv = CACHE == 1 || pid < 0 ? 0 : a.Hkv;
        const int heads = a.Hq + 2 * kv, total = rows * heads;
        constexpr int GROUPS = kThreads / UPH;        // threads of one row and head
        const int u = tid % UPH;
        for (int x0 = tid / UPH + GROUPS * kBatch * (int)blockIdx.y; x0 < total; x0 += GROUPS * kBatch * (int)gridDim.y) {
            u32x4_t p[kBatch], q[kBatch];
            E *to[kBatch];
            int row[kBatch];
            bool turn[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int x = min(x0 + k * GROUPS, total - 1);
                row[k] = x / heads;
                const int hh = x - row[k] * heads;
                const int64_t t = tok + row[k];
                const E *src;
                turn[k] = true;
                if (hh < a.Hq) {
                    src = reinterpret_cast<const E *>(a.q) + t * a.q_stride + (int64_t)hh * D;
                    to[k] = reinterpret_cast<E *>(a.q_out) + (t * a.Hq + hh) * D;
                } else {
                    const bool isv = hh >= a.Hq + kv;
                    const int h = hh - a.Hq - (isv ? kv : 0);
                    src = reinterpret_cast<const E *>(isv ? a.v_new : a.k_new) + t * (isv ? a.v_stride : a.k_stride) + (int64_t)h * D;
                    to[k] = reinterpret_cast<E *>(isv ? a.v : a.k) + (((size_t)pid * a.Hkv + h) * kPage + lo + row[k]) * D;
                    turn[k] = !isv;
                }
                p[k] = load16<STREAM>(src + u * EPU);
                q[k] = load16<STREAM>(src + H + u * EPU);
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (x0 + k * GROUPS >= total) break;
                if (turn[k]) {
                    float xa[EPU], xb[EPU];
                    widen(p[k], xa);
                    widen(q[k], xb);
#pragma unroll
                    for (int e = 0; e < EPU; ++e) rotate(xa[e], xb[e], s_cs[row[k]][u * EPU + e]);
                    p[k] = narrow(xa);
                    q[k] = narrow(xb);
                }
                store16<STREAM>(to[k] + u * EPU, p[k]);
                store16<STREAM>(to[k] + H + u * EPU, q[k]);
            }
        }
    }

    // 8-bit pools: a wave per KV head and pool takes the page's rows, four lanes a
    // row, finds the scale and writes the codes
    if constexpr (CACHE == 1) {
        if (pid < 0) return;
        constexpr int EH = H / 4;                     // elements per lane of each half row: 16 or 8
        const int slot = lane / 4, sub = lane % 4, row = slot - lo;
        const bool mine = row >= 0 && row < rows;
        const int rr = min(max(row, 0), rows - 1);
        for (int job = wave + kWaves * (int)blockIdx.y; job < 2 * a.Hkv; job += kWaves * (int)gridDim.y) {
            const int h = job >> 1;
            const bool isv = job & 1;
            const uint16_t *src = reinterpret_cast<const uint16_t *>(isv ? a.v_new : a.k_new) +
                                  (tok + rr) * (isv ? a.v_stride : a.k_stride) + (int64_t)h * D + sub * EH;
            float x[2][EH];
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int c = 0; c < EH; c += 8)
                    widen(load16<STREAM>(src + half * H + c), reinterpret_cast<float(&)[8]>(x[half][c]));
            if (!isv) {
#pragma unroll
                for (int e = 0; e < EH; ++e) rotate(x[0][e], x[1][e], s_cs[rr][sub * EH + e]);
            }
            float *sp = (isv ? a.v_scale : a.k_scale) + (size_t)pid * a.Hkv + h;
            float old = lo > 0 ? *sp : 0.0f;          // the page held tokens before (wave-uniform; requested with the rows)
            float amax = 0.0f;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int e = 0; e < EH; ++e) {
                    const float y = fabsf(x[half][e]);
                    if (y < __builtin_huge_valf()) amax = fmaxf(amax, y);
                    else x[half][e] = __builtin_nanf("");
                }
            amax = wave_max(mine ? amax : 0.0f);
            float scale = scale_for(amax);
            uint8_t *page = reinterpret_cast<uint8_t *>(isv ? a.v : a.k) + ((size_t)pid * a.Hkv + h) * kPage * D + slot * D + sub * EH;
            if (lo > 0) {
                scale = fmaxf(scale, power_from(old));
                if (scale > old && slot < lo) {       // their codes under the new scale
                    const float f = old / scale;          // exact, as inv
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int c = 0; c < EH; c += 4) {
                            uint32_t *w = reinterpret_cast<uint32_t *>(page + half * H + c);
                            const uint32_t u = *w;
                            const auto x0 = __builtin_amdgcn_cvt_pk_f32_fp8(u, false), x1 = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
                            *w = codes(odd_product(x0[0], f), odd_product(x0[1], f), odd_product(x1[0], f), odd_product(x1[1], f));
                        }
                }
            }
            const float inv = 1.0f / scale;           // exact: a power of two
            if (mine) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t w[EH / 4];
#pragma unroll
                    for (int c = 0; c < EH / 4; ++c) {
                        const float *y = x[half] + 4 * c;
                        w[c] = codes(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
                    }
                    if constexpr (EH == 16) *reinterpret_cast<u32x4_t *>(page + half * H) = u32x4_t{w[0], w[1], w[2], w[3]};
                    else *reinterpret_cast<u32x2_t *>(page + half * H) = u32x2_t{w[0], w[1]};
                }
            }
            if (lane == 0) *sp = scale;
        }
    }
}

// lengths and positions of the requests that took their tokens, once every read of
// them by the first launch is done
__global__ __launch_bounds__(256) void rope_advance_kernel(RopeArgs a) {
    const int r = blockIdx.x * 256 + threadIdx.x;
    if (r >= a.R) return;
    const Brought b = brought(a, r);
    if (!b.room) return;
    a.seq_lens[r] = b.m + b.n;
    a.positions[r] += b.n;
}

template <int CACHE, int D>
void launch_cd(const RopeArgs &a, hipStream_t s) {
    const int items = a.start ? a.T / kPage + 2 * a.R : a.R;
    // heads split so that about 1024 workgroups are there, as long as each has a batch of
    // pieces per thread or, in 8 bits, one job per wave
    const int pieces = (a.start ? kPage : 1) * (a.Hq + 2 * a.Hkv) * (D / 2) / (CACHE == 4 ? 4 : 8);
    const int most = CACHE == 1 ? cdiv(2 * a.Hkv, kWaves) : cdiv(pieces, kThreads * kBatch);
    const int split = std::max(1, std::min(most, cdiv(1024, items)));
    // rows past the caches where the call would only displace what others keep there (256
    // MB): 42 k tokens of 64/8 heads, d 128, 1.7 GB, 349 -> 338 us; chunks in 8 bits, 0.7 GB,
    // 146 -> 135.  Smaller calls leave the queries there for the attention that follows.
    const int64_t row = (int64_t)D * (CACHE == 4 ? 4 : 2), bytes = a.T * row * (2 * a.Hq + 3 * a.Hkv);
    const dim3 grid(items, split);
    if (bytes > (int64_t)256 << 20) rope_kernel<CACHE, D, true><<<grid, kThreads, 0, s>>>(a);
    else rope_kernel<CACHE, D, false><<<grid, kThreads, 0, s>>>(a);
}

}  // namespace

hipError_t launch_rope(int cache, int D, const RopeArgs &a, bool advance, hipStream_t s) {
    if (cache == 1) D == 128 ? launch_cd<1, 128>(a, s) : launch_cd<1, 64>(a, s);
    else if (cache == 2) D == 128 ? launch_cd<2, 128>(a, s) : launch_cd<2, 64>(a, s);
    else D == 128 ? launch_cd<4, 128>(a, s) : launch_cd<4, 64>(a, s);
    if (advance) rope_advance_kernel<<<cdiv(a.R, 256), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace gp
