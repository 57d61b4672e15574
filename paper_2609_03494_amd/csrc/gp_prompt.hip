// Attention of new tokens over the paged cache (gp_prompt_attention; Sec. 3.1
// attention-output equation with a causal limit): whole prompts, chunks behind a
// context, drafted tokens, single tokens.
//
// Work item: one KV head and kPromptRows rows of one request, a row being a (new token, query
// head of that KV head) pair: the G heads of a token read the same keys, so they lie
// side by side and the causal border of an item is kPromptRows / G tokens wide.  A wave has 32
// rows; keys and values come in blocks of 32 tokens, two pages, through LDS.
//
// Products, both transposed: S^T = K Q^T, then O^T += V^T P^T, on 32 x 32 matrix
// instructions.  A lane then holds scores of one row only (its column), so maxima and
// sums are in-lane but for one exchange with lane ^ 32, the rescaling of O^T is in-lane
// as well, and the scores become the second product's operand without moving: lane half
// h has tokens 8 k + 4 h + 0..3 of every 16, and V^T is read in that order (16 bits: by
// transposing LDS reads).  Softmax in one pass, weights in units of log2; the maximum may
// lag behind by 2^8, so that O^T is rescaled in few blocks.  Scores, statistics and outputs are
// float32.  The weights (of 8 bits: times the values' scales) go to the second product of 16- and 8-bit caches as bfloat16, the
// only form in which the matrix instruction takes them beside such values.  Items of up to 32 rows have them in two terms, as
// the decode step does (2^-16 of a weight at most): they wait for the cache, and 64 single tokens take 235 us with one
// term or two, five behind 6001 15.0 (60 single tokens of 8 heads per KV head at d 64, where little is read: 127.2 and 128.3).  Items of
// more rows have one (half a step, 2^-8 of a weight): three products for two cost them a third and more (8 chunks of 1024 behind
// 8192, see below, in turn on one card: 1072 and 1469 us, d 64 636 and 880, 8 bits 1197 and 1605), for a relative error (2-norm, random values) of
// 0.00166 in place of 0.00183, where the output's own rounding is 0.00166.
//
// Two paths, by an item's rows.  More than 32 (wide): the four waves share the blocks, and a wave works
// on the scores of block b + 1 and the weights of block b at once, independent work for the
// matrix unit and the others; up to four blocks are on their way straight into LDS.  Up to 32 (narrow:
// drafted and single tokens, ends of requests): bound by reading the cache, so every wave has blocks of its own
// and no barrier, and the waves' results meet in LDS at the end.
//
// Bound (8 chunks of 1024 tokens behind 8192, 32/8 heads; cards differ by 10 %, a library's product of two 8192 x 8192
// matrices with them; this one's reaches 1094 TFLOP/s): the matrix unit and with it the chip's power at head_dim 128, 1155 us, 1011 TFLOP/s; head_dim
// 64 has half of the products per weight and is bound by the vector instructions of the softmax (16 exponentials of
// 16 cycles are half of them): 681 us, 858 TFLOP/s.  8-bit: each code is widened once a workgroup, 1284 us and 910
// TFLOP/s, 803 and 727.  float32: its matrix instructions' rate, 1062 us for 4 of 512 behind 4096,
// 137 TFLOP/s of 154.  64 single tokens behind 1024 to 8143: the read of the cache, 5.1 TB/s.
// Tried and slower: the sum of weights by the matrix unit as well (bf16, head_dim 64: 5 %), keys widened by two waves
// and values by the others (8 bits, head_dim 64: 1 %), the merge by whoever ends an item last (5 tokens behind 6001:
// 24 us against 15).
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
// those into the other stage included; here the wave waits for them (wait_loads) before
// the barrier that hands the stage over.  No vector register is written; m0, the place in LDS, is.
__device__ inline void load_lds(const void *base, uint32_t off, uint32_t to) {
    __asm__ volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(to) : "m0", "memory");
}
__device__ inline uint32_t lds_addr(const void *p) {
    return (uint32_t)(size_t)(__attribute__((address_space(3))) const char *)p;
}
// all but the newest N vector memory operations; all LDS reads
template <int N>
__device__ inline void wait_loads() { __asm__ volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }
__device__ inline void wait_lds() { __asm__ volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

// CACHE: bytes of a pool element (1: e4m3 codes, as bfloat16 in LDS).  Keys and values go
// through LDS in blocks of 32 tokens.
template <int CACHE, int D>
struct Block {
    static constexpr int LB = CACHE == 4 ? 4 : 2;                    // bytes of an element in LDS
    static constexpr int ROWB = D * LB, UPR = ROWB / 16;             // bytes and 16-byte units of a token
    static constexpr int BYTES = 32 * ROWB;                          // of the keys, or the values
    static constexpr int PU = D * CACHE, PUR = PU / kPage;           // 16-byte units of a page in the pool, of a token
    static constexpr int STAGES = CACHE == 4 && D == 128 ? 2 : 4;    // blocks of keys, and of values, in LDS
    static constexpr int LOADS = CACHE == 1 ? 2 * PU / kThreads : BYTES / 1024 / kWaves;   // pieces of 1024 bytes of a wave
    static constexpr int NARROW = CACHE == 4 && D == 128 ? 2 : kWaves;   // waves with a block of their own, see prompt_kernel
    static constexpr int MEM = 2 * BYTES * (STAGES > NARROW ? STAGES : NARROW);
    static_assert(LOADS >= 1 || CACHE == 1, "each wave has a piece");
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

// --------------------------------------------------------------- division --
//
// One workgroup divides the batch into pieces: an item is up to a.tokens new tokens of a
// request, its cost the tokens that its last row sees (an item of up to 32 rows reads as many
// bytes in the time that 128 rows take to multiply them); where items are fewer or longer than the
// chip has places, an item's tokens are split into pieces of about the batch's share per place, each
// with a partial result of its own.  Pieces go out longest first (of many items request by
// request), sorted by cost in kBuckets steps; their order within a step is whoever came first and
// has no bearing on any result.
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64, kBuckets = 256;

// What a part takes of the workspace, in units of 32 rows.
__device__ inline int part_units(const PromptArgs &a, int rows) { return rows <= 32 ? 1 : a.part_rows / 32; }

__device__ inline int wave_sums(int x, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    return x;
}

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PromptArgs a) {
    constexpr int kFew = 4;                           // a thread takes requests of up to so many items, a wave the others
    __shared__ Asked s_asked[kPlanThreads];
    __shared__ int s_many[kPlanThreads];
    __shared__ unsigned long long s_cost, s_tokens;
    __shared__ int s_most, s_items, s_slots, s_merges, s_nmany, s_hist[kBuckets], s_wave[kBuckets / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    if (tid < kBuckets) s_hist[tid] = 0;
    if (tid == 0) {
        s_cost = s_tokens = 0;
        s_most = s_items = s_slots = s_merges = s_nmany = 0;
    }
    __syncthreads();
    // the sum of costs, the largest, all items and tokens
    {
        unsigned long long sum = 0, all = 0;
        int most = 0, items_ = 0;
        for (int r = tid; r < a.R; r += kPlanThreads) {
            const Asked q = asked(a, r);
            if (r < kPlanThreads) s_asked[r] = q;
            if (!q.in || q.n == 0) continue;
            const int items = (q.n + a.tokens - 1) / a.tokens;
            sum += (unsigned long long)items * max(q.before, 0) + (unsigned long long)items * (items - 1) / 2 * a.tokens + q.n;
            all += q.n;
            items_ += items;
            most = max(most, q.before + q.n);
        }
#pragma unroll
        for (int o = 32; o > 0; o /= 2) {
            sum += __shfl_xor(sum, o, 64);
            all += __shfl_xor(all, o, 64);
            items_ += __shfl_xor(items_, o, 64);
            most = max(most, __shfl_xor(most, o, 64));
        }
        if (lane == 0 && all) {
            atomicAdd(&s_cost, sum);
            atomicAdd(&s_tokens, all);
            atomicAdd(&s_items, items_);
            atomicMax(&s_most, most);
        }
    }
    __syncthreads();
    if (s_tokens > (unsigned long long)a.T) {         // (starts that decrease: more than the workspace is made for)
        if (tid < 2) a.counts[tid] = 0;
        return;
    }
    const int share = share_of(s_cost, a.slots);
    const float scale = (float)(kBuckets - 1) / (float)max(s_most, 1);
    // pass 1: pieces per bucket; 2: pieces to their places.  Few items all start at once: any order
    const bool sorted = s_items > a.slots / 2;
    // Of many items a request's go out one after the other, longest first, requests by their longest: workgroups that run
    // at the same time then read the same keys and values, from the XCD's L2 (60 prompts of 150 to 2330 tokens 1242 us,
    // 1117 so; two batches of 12 of 200 to 6000 1145 and 1124, 1096 and 1084; 8 chunks of 1024 behind 8192 1096 and 1058, at head_dim 64 620 and 625).  Of few, each by its own
    // length: the last ones should be short (six prompts of 300 to 1900 tokens in float32: 207 us, request by request 245)
    const bool grouped = s_items >= 3 * a.slots;
    for (int pass = sorted ? 1 : 2; pass < 3; ++pass) {
        auto item = [&](const Asked &q, int i, int &n, int &seen) {
            n = min(a.tokens, q.n - i * a.tokens);
            seen = max(q.before + i * a.tokens + n, 0);
            return split_of(seen, n << a.lg, share, a.fine);
        };
        auto bucket = [&](int longest) { return sorted ? max(kBuckets - 1 - (int)((float)longest * scale), 0) : 0; };
        // a request's step: by its longest piece (one of its last two items')
        auto bucket_of = [&](const Asked &q, int items) {
            int longest = 0;
            for (int i = items - 1; i >= max(items - 2, 0); --i) {
                int n, seen;
                const Split x = item(q, i, n, seen);
                longest = max(longest, min(x.per, seen));
            }
            return bucket(longest);
        };
        // item i to places `at` and on (the bounds hold for any batch, see PromptWs)
        auto put = [&](int r, const Asked &q, int i, int n, int seen, const Split &x, int at) {
            int slot = -1;
            const int units = part_units(a, n << a.lg), j0 = i * a.tokens;
            if (x.parts > 1) {
                slot = atomicAdd(&s_slots, x.parts * units);
                const int to = atomicAdd(&s_merges, 1);
                if (to < a.max_merges) a.merges[to] = make_int4(slot, x.parts, q.ts + j0, n);
            }
            for (int p = 0; p < x.parts; ++p, ++at) {
                if (at >= a.max_pieces) break;
                a.pieces[2 * at] = make_int4(r, slot < 0 ? -1 : slot + p * units, p * x.per, min((p + 1) * x.per, seen));
                a.pieces[2 * at + 1] = make_int4(q.ts + j0, n, q.before + j0, 0);
            }
        };
        for (int r0 = 0; r0 < a.R; r0 += kPlanThreads) {
            const int r = r0 + tid;
            Asked q = {};
            if (r < a.R) q = r0 == 0 ? s_asked[tid] : asked(a, r);
            const int items = q.in ? (q.n + a.tokens - 1) / a.tokens : 0;
            if (items > kFew) {
                const int at = atomicAdd(&s_nmany, 1);
                s_many[at] = r;
            } else if (items) {
                int at = 0, n, seen;
                if (grouped) {
                    int all = 0;
                    for (int i = 0; i < items; ++i) all += item(q, i, n, seen).parts;
                    at = atomicAdd(&s_hist[bucket_of(q, items)], all);
                }
                for (int i = items - 1; i >= 0; --i) {
                    const Split x = item(q, i, n, seen);
                    if (!grouped) at = atomicAdd(&s_hist[bucket(min(x.per, seen))], x.parts);
                    if (pass == 2) put(r, q, i, n, seen, x, at);
                    at += x.parts;
                }
            }
            __syncthreads();
            for (int k = wave; k < s_nmany; k += kPlanWaves) {
                const int rr = uni(s_many[k]);
                const Asked big = r0 == 0 ? s_asked[rr] : asked(a, rr);
                const int count = (big.n + a.tokens - 1) / a.tokens, of_all = grouped ? bucket_of(big, count) : 0;
                for (int i0 = count - 1; i0 >= 0; i0 -= 64) {
                    const int i = i0 - lane;
                    int n = 0, seen = 0, at = 0;
                    Split x = {0, 0};
                    if (i >= 0) x = item(big, i, n, seen);
                    if (grouped) {
                        const int upto = wave_sums(x.parts, lane);
                        if (lane == 63) at = atomicAdd(&s_hist[of_all], upto);
                        at = __shfl(at, 63, 64) + upto - x.parts;
                    } else if (i >= 0) {
                        at = atomicAdd(&s_hist[bucket(min(x.per, seen))], x.parts);
                    }
                    if (pass == 2 && i >= 0) put(rr, big, i, n, seen, x, at);
                }
            }
            __syncthreads();
            if (tid == 0) s_nmany = 0;
            __syncthreads();
        }
        if (pass == 1) {
            // first place of each bucket
            int n = 0, x = 0;
            if (tid < kBuckets) {
                n = x = s_hist[tid];
#pragma unroll
                for (int o = 1; o < 64; o *= 2) {
                    const int y = __shfl_up(x, o, 64);
                    if (lane >= o) x += y;
                }
                if (lane == 63) s_wave[wave] = x;
            }
            __syncthreads();
            if (tid < kBuckets) {
                for (int w = 0; w < wave; ++w) x += s_wave[w];
                s_hist[tid] = x - n;
            }
            __syncthreads();
        }
    }
    if (tid == 0) {
        a.counts[0] = min(s_hist[sorted ? kBuckets - 1 : 0], a.max_pieces);   // (where the last bucket's last piece ended)
        a.counts[1] = min(s_merges, a.max_merges);
    }
}

// A call of up to 64 items needs no list: every workgroup finds its piece, and every merging
// one its item, by a scan over the items, a lane each; where a request can have several, a scan over the
// requests comes before.  (The list of such a call took 6 us: one prompt of 1000 tokens 37.5 us, now 32.0.)
// piece: piece `index` (merge: split item `index`); r < 0: none.
// (A piece and a split item as the lists have them: all that a workgroup has to know, so that
// it does not look its request up first.)
struct Piece {
    int r, slot;                  // request (-1: none); partial slot (-1: a whole item)
    int from, to;                 // tokens that the piece reads
    int ts, n, before;            // the item's first row of q and out, its tokens, those that precede them
};
struct Merge { int slot, parts, ts, n; };
template <bool MERGE, bool SEVERAL>
__device__ inline typename std::conditional<MERGE, Merge, Piece>::type direct_place(const PromptArgs &a, int index, int lane) {
    Asked q = {};
    if (lane < a.R) q = asked(a, lane);
    // (starts that decrease can ask for more than T tokens: none is served)
    const bool none = __shfl(wave_sums(q.in ? q.n : 0, lane), 63, 64) > a.T;
    bool in = q.in && q.n > 0;
    int request = lane;
    if constexpr (SEVERAL) {
        const int items = in ? (q.n + a.tokens - 1) / a.tokens : 0, upto = wave_sums(items, lane);
        const int all = __shfl(upto, 63, 64), item = all - 1 - lane;      // (the last comes first: a request's longest)
        // the first request whose items end behind this one
        int r = 0;
#pragma unroll
        for (int o = 32; o > 0; o /= 2)
            if (__shfl(upto, r + o - 1, 64) <= item) r += o;
        request = r;
        in = item >= 0;
        const int j0 = (item - __shfl(upto - items, r, 64)) * a.tokens;
        q.ts = __shfl(q.ts, r, 64) + j0;
        q.before = __shfl(q.before, r, 64) + j0;
        const int left = __shfl(q.n, r, 64) - j0;             // (by all lanes: one that is not in may hold another's)
        q.n = in ? min(left, a.tokens) : 0;
    }
    const int seen = in ? max(q.before + q.n, 0) : 0;
    const int cost = __shfl(wave_sums(seen, lane), 63, 64);
    const Split x = split_of(seen, (in ? q.n : 0) << a.lg, share_of(cost, a.slots), 1);
    const int parts = in ? x.parts : 0, units = part_units(a, (in ? q.n : 0) << a.lg), split = parts > 1 ? parts * units : 0;
    const int slot_end = wave_sums(split, lane), end = MERGE ? wave_sums(split ? 1 : 0, lane) : wave_sums(parts, lane);
    const int begin = end - (MERGE ? (split ? 1 : 0) : parts);
    const uint64_t who = none ? 0 : __ballot(index >= begin && index < end);
    const int r = who ? __builtin_ctzll(who) : 0, parts_r = __shfl(parts, r, 64), units_r = __shfl(units, r, 64), slot0 = __shfl(slot_end, r, 64) - parts_r * units_r;
    const int ts = __shfl(q.ts, r, 64), n = __shfl(q.n, r, 64), before = __shfl(q.before, r, 64);
    if constexpr (MERGE) {
        return {slot0, who ? parts_r : 0, ts, n};
    } else {
        const int part = index - __shfl(begin, r, 64), per = __shfl(x.per, r, 64);
        return {who ? __shfl(request, r, 64) : -1, parts_r > 1 ? slot0 + part * units_r : -1, part * per, min(part * per + per, __shfl(seen, r, 64)), ts, n, before};
    }
}

// ---------------------------------------------------------------- products --

template <int CACHE, int D>
__global__ __launch_bounds__(kThreads, CACHE != 4 && D == 64 ? 3 : 2) void prompt_kernel(PromptArgs a) {
    using TL = Block<CACHE, D>;
    using E = typename std::conditional<CACHE == 4, float, uint16_t>::type;
    constexpr int DB = D / 32, LOADS = TL::LOADS;
    constexpr int QS = CACHE == 4 ? D / 8 : D / 16;                  // 16-byte pieces of a row per lane
    // a piece of up to 32 rows: each wave has blocks, and LDS, to itself
    constexpr int NW = TL::NARROW, NB = TL::BYTES, NL = NB / 1024;   // such waves; a block's keys, in pieces of 1024 bytes
    constexpr int QL = CACHE == 1 ? D / 32 : 1;                      // 8-bit: 16-byte units of a lane, of such a block
    __shared__ __attribute__((aligned(16))) unsigned char s_mem[TL::MEM];
    __shared__ uint32_t s_odd[4];                                    // wide: tokens of block b whose values are not all finite, b % 4; narrow: of the wave's
    static_assert(NW * 32 * D * 4 <= TL::MEM, "the waves' parts meet in LDS");
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int h = blockIdx.x % a.Hkv, at_piece = blockIdx.x / a.Hkv;
    Piece piece;
    if (a.direct) {
        piece = a.several ? direct_place<false, true>(a, at_piece, lane) : direct_place<false, false>(a, at_piece, lane);
        if (piece.r < 0) return;
    } else {
        if (at_piece >= scalar_load(a.counts, 0)) return;
        const int32_t *x = reinterpret_cast<const int32_t *>(a.pieces + 2 * (size_t)at_piece);
        piece = {scalar_load(x, 0), scalar_load(x, 1), scalar_load(x, 2), scalar_load(x, 3), scalar_load(x, 4), scalar_load(x, 5), scalar_load(x, 6)};
    }
    const int r = uni(piece.r), slot = uni(piece.slot), from_token = uni(piece.from), ts = uni(piece.ts), before = uni(piece.before);
    const int rows = uni(piece.n) << a.lg;                           // of this item
    const int first = before + 1, last = uni(piece.to);              // tokens that its first row sees, the end of the piece
    const int last_page = max(last - 1, 0) / kPage;
    const bool narrow = rows <= 32;

    // the wave's rows: a lane's row is its column of S^T and O^T
    const int col = lane & 31, half = lane >> 5;
    const int row0 = narrow ? 0 : wave * 32;
    const int row = row0 + col, at = min(row, rows - 1);
    const int sees = min(before + (at >> a.lg) + 1, last);
    const int wave_first = before + (min(row0, rows - 1) >> a.lg) + 1;
    const int wave_last = row0 < rows ? before + (min(row0 + 31, rows - 1) >> a.lg) + 1 : 0;
    const int64_t token = ts + (at >> a.lg);
    const int head = h * a.G + (at & (a.G - 1));
    u32x4_t q[QS];
    {
        const E *src = reinterpret_cast<const E *>(a.q) + token * a.q_stride + (int64_t)head * D + half * (16 / (int)sizeof(E));
#pragma unroll
        for (int s = 0; s < QS; ++s) q[s] = load16(src + s * (32 / (int)sizeof(E)));
    }
    f32x16_t o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = f32x16_t{};
    // The row's maximum (both halves the same) and this half's sum of weights 2^(score - from).  The
    // maximum may lag by 8 in log2, so that outputs are rarely rescaled: relative errors are as they are.
    // Of 8-bit caches the weights are kept below one, since they are multiplied by the values' scales.
    const float unit = CACHE == 1 ? 1.0f : a.qscale;                 // maxima to units of log2 (8-bit: in them already)
    const float lag = CACHE == 1 ? 8.0f : a.lag, offset = CACHE == 1 ? 8.0f : 0.0f;
    float m = kNegInf, l = 0.0f, above = kNegInf, from = 0.0f;       // above: the score that moves the maximum
    // the factor from one maximum to another (halves: the difference of two scores may be past float32, and come back by the unit)
    auto fall = [&](float of, float to) __attribute__((always_inline)) {
        return of == kNegInf ? 0.0f : __builtin_amdgcn_exp2f((0.5f * of - 0.5f * to) * unit * 2.0f);
    };

    // S^T of the 32 tokens whose keys lie at kb
    auto scores = [&](f32x16_t &st, const unsigned char *kb) __attribute__((always_inline)) {
        kb += col * TL::ROWB;
        const int sw = TL::key_swizzle(col);
        st = f32x16_t{};
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            const u32x4_t x = *reinterpret_cast<const u32x4_t *>(kb + (((2 * s + half) ^ sw) << 4));
            if constexpr (CACHE == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    st = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[e]), __uint_as_float(q[s][e]), st, 0, 0, 0);
            } else {
                st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x), __builtin_bit_cast(bf16x8_t, q[s]), st, 0, 0, 0);
            }
        }
    };
    // the factors of a block's two pages of scores to units of log2 (8-bit: with the pages' key scales)
    auto factor = [&](float ks) __attribute__((always_inline)) {
        return CACHE == 1 ? __builtin_amdgcn_fmed3f(a.qscale * ks, FLT_TRUE_MIN, FLT_MAX) : unit;
    };
    // scores of tokens t0 .. as far as the row sees them; the maximum, sum and outputs so far follow
    auto settle_scores = [&](f32x16_t &st, int t0, const float (&ks)[2], bool border) __attribute__((always_inline)) {
        if (border && t0 + 32 > min(wave_first, last)) {
            const int left = sees - t0 - 4 * half;                   // tokens that the row sees, from this half's first on
#pragma unroll
            for (int i = 0; i < 16; ++i) st[i] = masked(st[i], 8 * (i / 4) + i % 4 - left);
        }
        float t[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            t[p] = st[8 * p];
#pragma unroll
            for (int i = 1; i < 8; ++i) t[p] = fmaxf(t[p], st[8 * p + i]);
            if (CACHE == 1) t[p] *= factor(ks[p]);
        }
        const float top = max_halves(fmaxf(t[0], t[1]));
        if (__any(top > above)) {
            const float up = fmaxf(m, top), f = fall(m, up);
            l *= f;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
            m = up;
            above = up + lag;
            from = up == kNegInf ? 0.0f : up * unit + offset;        // (a row that sees nothing yet)
        }
    };
    // scores to weights, which the sum takes in (8-bit: then times the pages' value scales vs)
    auto weigh = [&](f32x16_t &st, const float (&ks)[2], const float (&vs)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) st[i] = __builtin_amdgcn_exp2f(fmaf(st[i], factor(ks[i / 8]), -from));
        float sum[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = (st[i] + st[i + 4]) + (st[i + 8] + st[i + 12]);
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        if constexpr (CACHE == 1) {
#pragma unroll
            for (int i = 0; i < 16; ++i) st[i] *= vs[i / 8];
        }
    };
    // O^T += V^T P^T; two: the weights in two bfloat16 terms
    auto values = [&](const f32x16_t &st, const unsigned char *vb, auto two) __attribute__((always_inline)) {
        if constexpr (CACHE == 4) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int t = 8 * (i / 4) + 4 * half + i % 4, u = (d * 32 + col) / 4;
                    const float x = *reinterpret_cast<const float *>(vb + t * TL::ROWB + ((u ^ TL::value_swizzle(t)) << 4) + (col & 3) * 4);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, st[i], o[d], 0, 0, 0);
                }
        } else {
            // lane j of a group of 16 names four dims of token j / 4 and receives dim j of the four tokens
            const int g = (lane >> 4) & 1, tt = 4 * half + ((lane & 15) >> 2), cc = 2 * g + ((lane & 3) >> 1);
            const uint32_t v0 = (uint32_t)(tt * TL::ROWB + ((cc ^ TL::value_swizzle(tt)) << 4) + (lane & 1) * 8);
            typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                u32x4_t p, rest;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float w0 = st[8 * k + 2 * c], w1 = st[8 * k + 2 * c + 1];
                    p[c] = pack_bf16(w0, w1);
                    if constexpr (two) rest[c] = pack_bf16(w0 - __uint_as_float(p[c] << 16), w1 - __uint_as_float(p[c] & 0xffff0000u));   // (exact before it is rounded)
                }
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    // (units 4 d of a token: the swizzle flips units of 4, which 4 d xors with)
                    const unsigned char *x = vb + (v0 ^ (uint32_t)(d << 6)) + k * 16 * TL::ROWB;
                    const u32x2_t y0 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)x));
                    const u32x2_t y1 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(x + 8 * TL::ROWB)));
                    const bf16x8_t v = __builtin_bit_cast(bf16x8_t, u32x4_t{y0[0], y0[1], y1[0], y1[1]});
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8_t, p), o[d], 0, 0, 0);
                    if constexpr (two) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8_t, rest), o[d], 0, 0, 0);
                }
            }
        }
    };

    const int32_t *table = a.page_table + (size_t)r * a.max_pages;
    const size_t slice = (size_t)h * kPage * D * CACHE;
    const uint32_t page_bytes = (uint32_t)a.Hkv * kPage * D * CACHE;
    auto page_of = [&](int page) __attribute__((always_inline)) { return scalar_load(table, min(page, last_page)); };
    auto inside = [&](int id) __attribute__((always_inline)) { return min(max(id, 0), a.pool_pages - 1); };
    auto page_at = [&](int id) __attribute__((always_inline)) { return (uint64_t)(uint32_t)inside(id) * page_bytes; };
    auto widen = [](uint32_t x0, uint32_t x1, float scale) __attribute__((always_inline)) {
        const bf16x2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x0, scale, false), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x0, scale, true);
        const bf16x2_t p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x1, scale, false), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x1, scale, true);
        return u32x4_t{__builtin_bit_cast(uint32_t, p0), __builtin_bit_cast(uint32_t, p1), __builtin_bit_cast(uint32_t, p2), __builtin_bit_cast(uint32_t, p3)};
    };
    // On the border, where some row does not see all of a block's tokens, a weight of zero would not
    // keep an infinite value or NaN out: 16 bytes of token t of block blk in LDS become zero if the
    // token lies behind the piece's, else its infinite values and NaN do, and the token's bit says so
    auto clean = [&](unsigned char *to, int blk, int t, uint32_t *odd) __attribute__((always_inline)) {
        u32x4_t x = *reinterpret_cast<u32x4_t *>(to);
        if (blk * 32 + t >= last) {
            x = u32x4_t{};
        } else {
            bool found = false;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if constexpr (CACHE == 4) {
                    const bool is = (x[c] & 0x7f800000u) == 0x7f800000u;
                    x[c] = is ? 0u : x[c];
                    found |= is;
                } else {
                    const bool lo = (x[c] & 0x7f80u) == 0x7f80u, hi = (x[c] & 0x7f800000u) == 0x7f800000u;
                    x[c] &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0xffffu : 0xffffffffu);
                    found |= lo || hi;
                }
            }
            if (!found) return;
            atomicOr(odd, 1u << t);
        }
        *reinterpret_cast<u32x4_t *>(to) = x;
    };
    // ... and the rows that see such a token take them in from the pool: the result is infinite or NaN at any weight, as
    // where a weight of zero meets them in the product, and stays so wherever outputs are scaled by zero
    auto add_odd = [&](int blk, uint32_t odd) __attribute__((always_inline)) {
        for (; odd; odd &= odd - 1) {
            const int t = __builtin_ctz(odd);
            const size_t at_token = page_at(page_of(2 * blk + t / kPage)) + slice + (size_t)(t % kPage) * D * CACHE;
            const unsigned char *v = static_cast<const unsigned char *>(a.v) + at_token;
            const bool seen = blk * 32 + t < sees;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int dim = 32 * d + 8 * (i / 4) + 4 * half + i % 4;
                    float x;
                    if constexpr (CACHE == 4) x = reinterpret_cast<const float *>(v)[dim];
                    else if constexpr (CACHE == 2) x = bf16_to_f32(reinterpret_cast<const uint16_t *>(v)[dim]);
                    else x = (v[dim] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f;
                    if (seen && !(fabsf(x) < __builtin_huge_valf())) o[d][i] += x;
                }
        }
    };
    constexpr float key_unit = 1.0f / kQ8KeyScale;                   // (see Page<E4m3>::kKeyUnit of the decode kernel)
    // 16 codes of unit c of token t, widened, to the rows at `to`
    auto put_codes = [&](unsigned char *to, int t, int c, int swizzle, const u32x4_t &x, float scale) __attribute__((always_inline)) {
        u32x4_t *row_ = reinterpret_cast<u32x4_t *>(to + t * TL::ROWB);
        row_[(2 * c) ^ swizzle] = widen(x[0], x[1], scale);
        row_[(2 * c + 1) ^ swizzle] = widen(x[2], x[3], scale);
    };
    u32x4_t kr[QL], vr[QL];

    if (!narrow) {
        // Blocks of keys and values have STAGES (a power of two) places each in LDS.  In step b the workgroup reads the
        // keys of block b + 1 and the values of block b, so that the scores of the one and the weights of
        // the other are independent work; on their way are later blocks, up to keys b + STAGES and
        // values b + STAGES - 1, whose places step b - 1 was the last to read.  8-bit blocks go through
        // registers, where they are widened, a step before they are read.
        constexpr int ST = TL::STAGES;
        const int b0 = from_token / 32, b1 = (last + 31) / 32, border = min(first, last);
        // the place of block b0 + i in LDS
        auto place = [&](int i) __attribute__((always_inline)) { return (uint32_t)(i & (ST - 1)) * TL::BYTES; };
        unsigned char *const s_k = s_mem, *const s_v = s_mem + ST * TL::BYTES;
        constexpr int PIECES = TL::BYTES / 1024;                     // (CACHE != 1) of a block
        const char *const kbase = static_cast<const char *>(a.k) + slice, *const vbase = static_cast<const char *>(a.v) + slice;
        // keys (which: 0) or values of two pages, to the place at `to`
        auto load = [&](int which, const int (&ids)[2], uint32_t to) __attribute__((always_inline)) {
            const char *pool = which ? vbase : kbase;
            if constexpr (CACHE == 1) {
                if (2 * TL::PU >= kThreads || tid < 2 * TL::PU)
                    (which ? vr : kr)[0] = reinterpret_cast<const u32x4_t *>(pool + page_at(ids[wave * 64 / TL::PU]) + (wave * 64 % TL::PU) * 16)[lane];
            } else {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    const int part = i * kWaves + wave;
                    // the unit that belongs at the lane's place in LDS
                    const int t = (part * 64 + lane) / TL::UPR, c = lane % TL::UPR;
                    const int u = (lane & ~(TL::UPR - 1)) + (c ^ (which ? TL::value_swizzle(t) : TL::key_swizzle(t)));
                    const int pg = LOADS == 1 ? wave / (kWaves / 2) : i / (LOADS / 2);
                    load_lds(pool + page_at(ids[pg]) + (part % (PIECES / 2)) * 1024, u * 16, lds_addr((which ? s_v : s_k) + part * 1024) + to);
                }
            }
        };
        auto ids_of = [&](int blk, int (&ids)[2]) __attribute__((always_inline)) {
            ids[0] = page_of(2 * blk);
            ids[1] = page_of(2 * blk + 1);
        };
        auto scales_of = [&](const float *scales, const int (&ids)[2], float (&x)[2]) __attribute__((always_inline)) {
            if constexpr (CACHE == 1)
#pragma unroll
                for (int p = 0; p < 2; ++p) x[p] = scalar_load(scales, (int64_t)inside(ids[p]) * a.Hkv + h);
        };
        // 8-bit: the loaded block to LDS
        auto put = [&](int which, uint32_t to) __attribute__((always_inline)) {
            if constexpr (CACHE == 1) {
                const int t = tid / TL::PUR, c = tid % TL::PUR;
                if (2 * TL::PU >= kThreads || tid < 2 * TL::PU) {
                    if (which) put_codes(s_v + to, t, c, TL::value_swizzle(t), vr[0], 1.0f);
                    else put_codes(s_k + to, t, c, TL::key_swizzle(t), kr[0], key_unit);
                }
            }
        };
        // the units of a block's values that this thread brought (see clean)
        auto settle_values = [&](int blk, uint32_t to) __attribute__((always_inline)) {
            if ((blk + 1) * 32 <= border) return;
            constexpr int UNITS = CACHE == 1 ? 2 : LOADS;
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int u = CACHE == 1 ? (tid / TL::PUR) * TL::UPR + (((tid % TL::PUR) * 2 + i) ^ TL::value_swizzle(tid / TL::PUR)) : (i * kWaves + wave) * 64 + lane;
                if (CACHE == 1 && tid >= 2 * TL::PU) continue;
                clean(s_v + to + u * 16, blk, u / TL::UPR, &s_odd[blk & 3]);
            }
        };
        if (tid < 4) s_odd[tid] = 0;
        int kid[2], vid[2];                                          // pages of the next keys and values to be loaded
        float ks[2] = {}, kn[2] = {}, vs[2] = {}, vn[2] = {};        // 8-bit: scales of the keys, values in work, and the next
        f32x16_t sa, sb;
        if (b0 < b1) {
            if constexpr (CACHE == 1) {
                ids_of(b0, kid);
                load(0, kid, 0);
                load(1, kid, 0);
                scales_of(a.k_scale, kid, ks);
                scales_of(a.v_scale, kid, vs);
                put(0, place(0));
                put(1, place(0));
                ids_of(b0 + 1, kid);
                load(0, kid, 0);
                load(1, kid, 0);
                scales_of(a.k_scale, kid, kn);
                scales_of(a.v_scale, kid, vn);
                put(0, place(1));
            } else {
#pragma unroll
                for (int i = 0; i < ST; ++i) {
                    ids_of(b0 + i, kid);
                    load(0, kid, place(i));
                    if (i < ST - 1) load(1, kid, place(i));
                }
                wait_loads<0>();
            }
        }
        __syncthreads();
        if (b0 < b1) settle_values(b0, place(0));
        __syncthreads();
        if (b0 < b1) {
            if (b0 * 32 < wave_last) {
                scores(sa, s_k + place(0));
                settle_scores(sa, b0 * 32, ks, true);
            }
            vid[0] = kid[0], vid[1] = kid[1];                        // (the last keys loaded are the next values)
            ids_of(b0 + (CACHE == 1 ? 2 : ST), kid);
        }
        __syncthreads();                                             // (the first keys' place is free)
        // what is loaded in step b, the i-th (`i` counts modulo ST).  Page ids behind the last are the last's: the
        // loads are the same number in every step
        auto fetch = [&](int b, int i) __attribute__((always_inline)) {
            if constexpr (CACHE == 1) {
                put(1, place(i + 1));
                load(0, kid, 0);
                load(1, kid, 0);
            } else {
                load(0, kid, place(i));
                load(1, vid, place(i + ST - 1));
                vid[0] = kid[0], vid[1] = kid[1];
                ids_of(b + ST + 1, kid);
            }
        };
        // ... and what step b + 1 reads, in place
        auto arrive = [&](int b, int i) __attribute__((always_inline)) {
            if constexpr (CACHE == 1) {
                put(0, place(i + 2));
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    ks[p] = kn[p];
                    vs[p] = vn[p];
                }
                scales_of(a.k_scale, kid, kn);
                scales_of(a.v_scale, kid, vn);
                ids_of(b + 3, kid);
            } else {
                wait_loads<2 * LOADS * (ST - 2)>();
            }
        };
        // step b: `st` holds the scores of block b.  Away from the border every row sees blocks b and b + 1
        auto inner = [&](int b, int i, f32x16_t &st, f32x16_t &nx) __attribute__((always_inline)) {
            fetch(b, i);
            scores(nx, s_k + place(i + 1));
            weigh(st, ks, vs);
            values(st, s_v + place(i), std::false_type{});
            settle_scores(nx, (b + 1) * 32, kn, false);
            arrive(b, i);
            __syncthreads();
        };
        auto step = [&](int b, f32x16_t &st, f32x16_t &nx) __attribute__((always_inline)) {
            const bool next = b + 1 < b1, mine = b * 32 < wave_last, more = next && (b + 1) * 32 < wave_last;
            const int i = b - b0;
            if (next) fetch(b, i);
            // (block b + 2's mark: last read two steps ago, made in the next one)
            if (tid == 0) s_odd[(b + 2) & 3] = 0;
            if (mine) {
                weigh(st, ks, vs);
                values(st, s_v + place(i), std::false_type{});
                if ((b + 1) * 32 > border) {
                    const uint32_t odd = uni(s_odd[b & 3]);
                    if (odd) add_odd(b, odd);
                }
            }
            if (more) {
                scores(nx, s_k + place(i + 1));
                settle_scores(nx, (b + 1) * 32, kn, true);
            }
            if (next) {
                arrive(b, i);
                settle_values(b + 1, place(i + 1));
            }
            __syncthreads();
        };
        // (ST steps at a time: the places are constants, and with them 12 additions of addresses a step fall away)
        int b = b0;
        if (row0 < rows) {
            for (; (b + ST + 1) * 32 <= border; b += ST)
#pragma unroll
                for (int k = 0; k < ST; k += 2) {
                    inner(b + k, k, sa, sb);
                    inner(b + k + 1, k + 1, sb, sa);
                }
        } else {
            for (; (b + ST + 1) * 32 <= border; b += ST)
#pragma unroll
                for (int k = 0; k < ST; ++k) {
                    fetch(b + k, k);
                    arrive(b + k, k);
                    __syncthreads();
                }
        }
        for (; b < b1; b += 2) {
            step(b, sa, sb);
            if (b + 1 < b1) step(b + 1, sb, sa);
        }
        if constexpr (CACHE != 1) wait_loads<0>();
        l = sum_halves(l);
    } else {
        // every wave has its own tiles of 32 tokens, NW apart, keys and values in LDS once: the next
        // keys are on their way as soon as the scores are there, the next values after the product
        unsigned char *s_k = s_mem + wave * 2 * NB, *s_v = s_k + NB;
        const int b1 = (last + 31) / 32;
        int b = wave < NW ? from_token / 32 + wave : b1;
        int ids[2];
        float ks[2], vs[2], kn[2], vn[2];
        auto request = [&](int blk) __attribute__((always_inline)) {
            ids[0] = page_of(2 * blk);
            ids[1] = page_of(2 * blk + 1);
        };
        // keys (which: 0) or values of the requested tile
        auto load = [&](int which) __attribute__((always_inline)) {
            const char *pool = static_cast<const char *>(which ? a.v : a.k);
            if constexpr (CACHE == 1) {
#pragma unroll
                for (int i = 0; i < QL; ++i) {
                    const size_t from = page_at(ids[i / (QL / 2)]) + slice + (size_t)(i % (QL / 2)) * 1024;
                    (which ? vr : kr)[i] = reinterpret_cast<const u32x4_t *>(pool + from)[lane];
                }
#pragma unroll
                for (int p = 0; p < 2; ++p) (which ? vn : kn)[p] = scalar_load(which ? a.v_scale : a.k_scale, (int64_t)inside(ids[p]) * a.Hkv + h);
            } else {
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    const int t = (i * 64 + lane) / TL::UPR, c = lane % TL::UPR;
                    const int u = (lane & ~(TL::UPR - 1)) + (c ^ (which ? TL::value_swizzle(t) : TL::key_swizzle(t)));
                    const size_t from = page_at(ids[i / (NL / 2)]) + slice + (size_t)(i % (NL / 2)) * 1024;
                    load_lds(pool + from, u * 16, lds_addr((which ? s_v : s_k) + i * 1024));
                }
            }
        };
        if (b < b1) {
            request(b);
            load(0);
            load(1);
        }
        for (; b < b1; b += NW) {
            const bool more = b + NW < b1;
            if (more) request(b + NW);
            if constexpr (CACHE == 1) {
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    ks[p] = kn[p];
                    vs[p] = vn[p];
                }
#pragma unroll
                for (int i = 0; i < QL; ++i) {
                    const int t = (i * 64 + lane) / TL::PUR, c = lane % TL::PUR;
                    put_codes(s_k, t, c, TL::key_swizzle(t), kr[i], key_unit);
                }
            } else {
                wait_loads<NL>();                                    // (the values, behind the keys, may be under way)
            }
            f32x16_t st;
            scores(st, s_k);
            wait_lds();                                              // the keys are read
            if (more) load(0);
            settle_scores(st, b * 32, ks, true);
            weigh(st, ks, vs);
            const bool border = (b + 1) * 32 > min(first, last);
            if (border && lane == 0) s_odd[wave] = 0;
            if constexpr (CACHE == 1) {
#pragma unroll
                for (int i = 0; i < QL; ++i) {
                    const int t = (i * 64 + lane) / TL::PUR, c = lane % TL::PUR;
                    put_codes(s_v, t, c, TL::value_swizzle(t), vr[i], 1.0f);
                }
            } else {
                if (more) wait_loads<NL>();
                else wait_loads<0>();
            }
            if (border)
                for (int i = 0; i < NL; ++i) clean(s_v + i * 1024 + lane * 16, b, (i * 64 + lane) / TL::UPR, &s_odd[wave]);
            values(st, s_v, std::true_type{});
            if (border) {
                const uint32_t odd = uni(s_odd[wave]);
                if (odd) add_odd(b, odd);
            }
            wait_lds();
            if (more) load(1);
        }
        l = sum_halves(l);
        // the waves' parts meet in LDS: outputs as [wave][32 rows][D], swizzled by 16-byte units
        __syncthreads();
        __shared__ float s_ml[2][NW][32];
        float *s_o = reinterpret_cast<float *>(s_mem);
        auto unit_of = [&](int rr, int u) __attribute__((always_inline)) { return rr * (D / 4) + (u ^ (rr & 15)); };
        if (wave < NW) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    reinterpret_cast<f32x4_t *>(s_o + wave * 32 * D)[unit_of(col, 8 * d + 2 * i + half)] =
                        f32x4_t{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
            if (half == 0) {
                s_ml[0][wave][col] = m;
                s_ml[1][wave][col] = l;
            }
        }
        __syncthreads();
        float mx = kNegInf, f[NW], sum = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) mx = fmaxf(mx, s_ml[0][w][col]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float mw = s_ml[0][w][col], lw = s_ml[1][w][col];
            f[w] = fall(mw, mx);
            sum += lw * f[w];                                        // (no weight: lw is 0, or NaN, which stays)
        }
        // wave w finishes a share of the units
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if ((d * 4 + i) % kWaves != wave) continue;
                f32x4_t y = {};
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const f32x4_t x = reinterpret_cast<const f32x4_t *>(s_o + w * 32 * D)[unit_of(col, 8 * d + 2 * i + half)];
#pragma unroll
                    for (int c = 0; c < 4; ++c) y[c] += x[c] * f[w];
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) o[d][4 * i + c] = y[c];
            }
        m = mx;
        l = sum;
    }

    // a whole item's outputs, or a piece's part of them (wave-uniform).  Narrow: every wave its share of the dims
    if (row >= rows) return;
    if (slot < 0) {
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        E *to = reinterpret_cast<E *>(a.out) + (token * a.Hkv * a.G + head) * D + 4 * half;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (narrow && (d * 4 + i) % kWaves != wave) continue;
                float x[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) x[c] = l > 0.0f ? o[d][4 * i + c] * inv : 0.0f;
                if constexpr (CACHE == 4)
                    *reinterpret_cast<u32x4_e4_t *>(to + 32 * d + 8 * i) = u32x4_t{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
                else
                    *reinterpret_cast<u32x2_e2_t *>(to + 32 * d + 8 * i) = u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
            }
    } else {
        const int units = part_units(a, rows), part_rows = 32 * units;
        if (slot + units > a.units) return;                          // (no batch asks for more, see prompt_ws)
        float *to = a.partial + ((size_t)slot * a.Hkv + (size_t)h * units) * 32 * (D + 2);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (narrow && (d * 4 + i) % kWaves != wave) continue;
                *reinterpret_cast<f32x4_t *>(to + (size_t)row * D + 32 * d + 8 * i + 4 * half) =
                    f32x4_t{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
            }
        if (half == 0 && (!narrow || wave == 0)) {
            float *ml = to + (size_t)part_rows * D;
            ml[row] = m * unit;
            ml[part_rows + row] = l;
        }
    }
}

// Parts of split items to outputs: ROWS rows of an item and KV head a workgroup, D / 4 threads a row,
// BATCH parts in flight.  Few rows (calls of up to 32): many parts, so eight at a time and eight rows
// a workgroup (5 tokens behind 6001: 25.6 us a call with one part after the other, 15.0 so).  Many:
// few parts, and workgroups without an item cost more than theirs take (a prompt of 2048: 80.9 us
// in that form, 72 with 32 rows and four parts).
template <typename E, int D, int RPW, int BATCH>
__global__ __launch_bounds__(256) void merge_kernel(PromptArgs a) {
    constexpr int LANES = D / 4, ROWS = 256 / LANES;
    const int h = blockIdx.x, block = blockIdx.y, at = blockIdx.z;       // (those without an item end the launch)
    Merge x;
    if (a.direct) {
        x = a.several ? direct_place<true, true>(a, at, threadIdx.x & 63) : direct_place<true, false>(a, at, threadIdx.x & 63);
        if (x.parts == 0) return;
    } else {
        if (at >= scalar_load(a.counts, 1)) return;
        const int4 y = a.merges[at];
        x = {y.x, y.y, y.z, y.w};
    }
    const int rows = x.n << a.lg;
    const int u = threadIdx.x % LANES, parts = uni(x.parts);
    if (x.slot + parts * part_units(a, rows) > a.units) return;
    for (int row = block * RPW + threadIdx.x / LANES; row < min(rows, (block + 1) * RPW); row += ROWS) {
        const int units = part_units(a, rows), part_rows = 32 * units;
        const size_t stride = (size_t)a.Hkv * part_rows * (D + 2);
        const float *p = a.partial + ((size_t)x.slot * a.Hkv + (size_t)h * units) * 32 * (D + 2);
        const float *ml = p + (size_t)part_rows * D + row;
        float m = kNegInf, l = 0.0f;
        f32x4_t o = {};
        for (int k0 = 0; k0 < parts; k0 += BATCH) {
            float mk[BATCH], lk[BATCH];
            f32x4_t ok[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                mk[k] = kNegInf;
                lk[k] = 0.0f;
                ok[k] = f32x4_t{};
                if (k0 + k >= parts) continue;            // (the same for all threads)
                const size_t part = (k0 + k) * stride;
                mk[k] = ml[part];
                lk[k] = ml[part + part_rows];
                ok[k] = *reinterpret_cast<const f32x4_t *>(p + part + (size_t)row * D + 4 * u);
            }
            float up = m;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) up = fmaxf(up, mk[k]);
            const float f = m == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m - up);
            l *= f;
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] *= f;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const float g = mk[k] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(mk[k] - up);
                l += lk[k] * g;                           // (a sum that is NaN stays so)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[c] += ok[k][c] * g;
            }
            m = up;
        }
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        float y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = l > 0.0f ? o[c] * inv : 0.0f;
        const int64_t token = x.ts + (row >> a.lg);
        E *to = reinterpret_cast<E *>(a.out) + (token * a.Hkv * a.G + h * a.G + (row & (a.G - 1))) * D + 4 * u;
        if constexpr (sizeof(E) == 4)
            *reinterpret_cast<u32x4_e4_t *>(to) = u32x4_t{__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])};
        else
            *reinterpret_cast<u32x2_e2_t *>(to) = u32x2_t{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
    }
}

template <int CACHE, int D>
void launch_cd(const PromptArgs &a, hipStream_t s) {
    if (!a.direct) plan_kernel<<<1, kPlanThreads, 0, s>>>(a);
    prompt_kernel<CACHE, D><<<a.max_pieces * a.Hkv, kThreads, 0, s>>>(a);
    using E = typename std::conditional<CACHE == 4, float, uint16_t>::type;
    if (a.part_rows <= 32) merge_kernel<E, D, 8, 8><<<dim3(a.Hkv, a.part_rows / 8, a.max_merges), 256, 0, s>>>(a);
    else merge_kernel<E, D, 32, 4><<<dim3(a.Hkv, a.part_rows / 32, a.max_merges), 256, 0, s>>>(a);
}

}  // namespace

hipError_t launch_prompt(int cache, int D, const PromptArgs &a, hipStream_t s) {
    if (cache == 1) D == 128 ? launch_cd<1, 128>(a, s) : launch_cd<1, 64>(a, s);
    else if (cache == 2) D == 128 ? launch_cd<2, 128>(a, s) : launch_cd<2, 64>(a, s);
    else D == 128 ? launch_cd<4, 128>(a, s) : launch_cd<4, 64>(a, s);
    return hipGetLastError();
}

}  // namespace gp
