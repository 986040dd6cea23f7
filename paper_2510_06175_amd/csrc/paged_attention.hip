// Decode attention over a full-precision paged cache, one new token per sequence.
//
//   s_t = scale q . k_t,   o = sum_t p_t v_t,   p = softmax(s),   L = log sum_t exp(s_t)
//
// One workgroup per (split, KV head, sequence), all G query heads of the KV head in it, so that a key or value row is
// read once.  Its wavefronts are independent: each takes every NW-th tile of 32 tokens of the split, keeps the running
// maximum and sum of its own tiles, and joins the others at the end, through LDS.
//
// A tile never leaves registers.  Both products are 16x16x32 matrix instructions with the query heads in the 16
// columns, and the tokens are dealt to the rows so that one's result is the other's operand:
//   scores   A = keys: row m of sub-tile u is token 8 (m / 4) + 4 u + m % 4; B = queries.  Lane (kg = l / 16, c = l % 16)
//            gets the scores of head c, tokens 8 kg + 4 u + r;
//   output   A = values, transposed; B = the probabilities: lane (kg, c) holds head c, tokens 8 kg .. 8 kg + 7 - which
//            are those it has.  Of the values lane (kg, c) loads D / 16 channels from channel c D / 16 of tokens
//            8 kg .. + 7, whole rows per 16 lanes, and turns the block within its own registers.  Row m of the i-th
//            product is then channel m D / 16 + i.
// What bounds it is memory: 4 D bytes per token against 32 D G / 16 matrix operations, of which the chip has 50 times
// as many per byte as are needed.  So the idle columns (G < 16) cost nothing, nor do the probabilities as two parts
// (high and low): bf16's two parts are within 2^-17 of a probability, fp16's within 2^-23 (and 2^-40 of the largest), next to
// the output's own rounding of 2^-8 and 2^-11.  The high part alone would add as much again.
#include "mfma_helpers.h"
#include "paged.h"
#include "split_merge.h"

#include <type_traits>

namespace vecinfer {

namespace {

constexpr int kTokens = 32;                               // tokens of a tile

template <typename E> struct Vec;
template <> struct Vec<f16> {
    typedef f16 v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ floatx4 mfma(v8 a, v8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    // Probabilities, and so their sums and outputs in front of the division, are held times 2^15: fp16 then has them in full
    // down to 2^-29 of the largest.  The lift goes onto a score's distance from the maximum, never onto the maximum, from
    // which fp32 cannot take 15 where it is 2^24 and more (and 2^16, as which 1 was held there, is no fp16 number).
    static constexpr float kLift = 15.f;
    static constexpr unsigned kInf = 0x7c00u;
};
template <> struct Vec<bf16> {
    typedef bf16 v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ floatx4 mfma(v8 a, v8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static constexpr float kLift = 0.f;
    static constexpr unsigned kInf = 0x7f80u;
};

// Weight of what has maximum m where the whole has maximum `all`.  Never 0, so that an infinite output stays one: with a
// maximum of -inf, or a far lower one, what it weighs is 0 or as good as that.
__device__ __forceinline__ float weight_of(float m, float all) { return fmaxf(__builtin_amdgcn_exp2f(m - all), 0x1p-126f); }

// What takes a head's scores to weights: the maximum and 1 over the sum, not one number, whose rounding would be all weights'
// (half a step of log2 of the sum is a factor of 2^0.5 at 2^23).
template <typename E>
__device__ __forceinline__ float2 norm_of(float at, float den)
{
    constexpr float lifted = Vec<E>::kLift > 0.f ? 0x1p15f : 1.f;
    static_assert(Vec<E>::kLift == 0.f || Vec<E>::kLift == 15.f, "2^15");
    return make_float2(at, den == 0.f ? 0.f : lifted / den);
}

// The infinite ones of two halves, 0 in place of the others.
template <typename E>
__device__ __forceinline__ unsigned infinite_halves(unsigned x)
{
    const unsigned low = (x & 0x7fffu) == Vec<E>::kInf ? 0xffffu : 0u, high = (x & 0x7fff0000u) == Vec<E>::kInf << 16 ? 0xffff0000u : 0u;
    return x & (low | high);
}

// sum over the four 16-lane rows of the wavefront
__device__ __forceinline__ float rows_sum(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    auto s16 = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float m = __builtin_bit_cast(float, (unsigned)s16[0]) + __builtin_bit_cast(float, (unsigned)s16[1]);
    const unsigned w = __builtin_bit_cast(unsigned, m);
    auto s32 = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return __builtin_bit_cast(float, (unsigned)s32[0]) + __builtin_bit_cast(float, (unsigned)s32[1]);
}

template <typename E>
__device__ __forceinline__ typename Vec<E>::v8 as_vec(unsigned a, unsigned b, unsigned c, unsigned d)
{
    const uintx4 u = {a, b, c, d};
    return __builtin_bit_cast(typename Vec<E>::v8, u);
}

// Called by all threads of a workgroup whose partials are stored: the last of the S workgroups of this (sequence, KV
// head) writes the output rows (split_merge.h).  The rows of the first kBatch splits travel while the weights are
// worked out, a wavefront per head.
template <typename E, int D, int KG, int NW>
__device__ __forceinline__ void merge_last(const PagedParams &p, float *lds, arrival_t *word, size_t first, int S, size_t row0)
{
    constexpr int kBlock = NW * 64, kElems = (KG * D + kBlock - 1) / kBlock, kBatch = 32 / kElems, kStep = 4;
    static_assert(kBatch >= kStep, "elements of a thread");
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), G = p.G, GD = G * D;
    unsigned *const flag = reinterpret_cast<unsigned *>(lds);
    float *const wt_s = lds + 4, *const den_s = wt_s + KG * kMergeSplits;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // this wavefront's stores are acknowledged
    __syncthreads();
    if (t == 0) {
        const arrival_t before = __hip_atomic_fetch_add(word, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *flag = (int)(before & 0xffffu) == S - 1;
    }
    __syncthreads();
    if (*flag == 0u) return;                              // (the same for the whole workgroup)
    const float *const po = p.part_o + first * GD;
    float v[kElems][kBatch];
    auto request = [&](int s0) {
#pragma unroll
        for (int j0 = 0; j0 < kBatch; j0 += kStep) {
            if (s0 + j0 >= S) break;
#pragma unroll
            for (int j = j0; j < j0 + kStep; ++j)
#pragma unroll
                for (int i = 0; i < kElems; ++i) {
                    // (behind the last split, that one again, at the least weight there is; behind the last element, the first)
                    const int e = t + i * kBlock < GD ? t + i * kBlock : 0;
                    v[i][j] = shared_load(po + (size_t)(s0 + j < S ? s0 + j : S - 1) * GD + e);
                }
        }
    };
    request(0);
    if (t == 0) __hip_atomic_store(word, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int h = wave; h < G; h += NW) {
        const float *const pm = p.part_m + first * G + h, *const pl = p.part_l + first * G + h;
        float m[kMergeSplits / 64], l[kMergeSplits / 64], M = -INFINITY, den = 0.f;
#pragma unroll
        for (int i = 0; i < kMergeSplits / 64; ++i) {
            const int s = lane + 64 * i;
            m[i] = s < S ? shared_load(pm + (size_t)s * G) : -INFINITY;
            l[i] = s < S ? shared_load(pl + (size_t)s * G) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kMergeSplits / 64; ++i) M = fmaxf(M, m[i]);
        M = wave_all(M, [](float a, float b) { return fmaxf(a, b); });
        const float at = M > -INFINITY ? M : 0.f;         // nothing to attend to: sums and outputs of 0 at any weight
#pragma unroll
        for (int i = 0; i < kMergeSplits / 64; ++i) {
            const float w = weight_of(m[i], at);
            wt_s[h * kMergeSplits + lane + 64 * i] = w;
            den = fmaf(w, l[i], den);
        }
        den = wave_all(den, [](float a, float b) { return a + b; });
        if (lane == 0) {
            const float total = den == 0.f ? -INFINITY : M + (log2f(den) - Vec<E>::kLift);
            den_s[h] = den;
            if (p.lse) p.lse[row0 + h] = natural(total);
            if (p.norm) p.norm[row0 + h] = norm_of<E>(at, den);
        }
    }
    __syncthreads();
    float acc[kElems];
#pragma unroll
    for (int i = 0; i < kElems; ++i) acc[i] = 0.f;
    for (int s0 = 0;;) {
#pragma unroll
        for (int j0 = 0; j0 < kBatch; j0 += kStep) {
            if (s0 + j0 >= S) break;
#pragma unroll
            for (int i = 0; i < kElems; ++i) {
                const int e = t + i * kBlock < GD ? t + i * kBlock : 0;
                const float4 w = *reinterpret_cast<const float4 *>(wt_s + e / D * kMergeSplits + s0 + j0);
                acc[i] = fmaf(w.x, v[i][j0], acc[i]);
                acc[i] = fmaf(w.y, v[i][j0 + 1], acc[i]);
                acc[i] = fmaf(w.z, v[i][j0 + 2], acc[i]);
                acc[i] = fmaf(w.w, v[i][j0 + 3], acc[i]);
            }
        }
        s0 += kBatch;
        if (s0 >= S) break;
        request(s0);
    }
    E *const out = static_cast<E *>(p.out) + row0 * D;
#pragma unroll
    for (int i = 0; i < kElems; ++i) {
        const int e = t + i * kBlock;
        if (e >= GD) continue;
        const float den = den_s[e / D];
        out[e] = (E)(den == 0.f ? 0.f : acc[i] / den);
    }
}

// What the way to the first page needs comes first: the command processor puts the leading 14 dwords into registers, and
// what lies behind them arrives while the length and the page travel (packed: G, the pages' shift and, dealt by length, B).
template <typename E, int D, int KG, int NW, bool SCORES, bool DEALT>
__global__ __launch_bounds__(NW * 64) void paged_attention_kernel(const int32_t *seq_lens, const int32_t *block_table, const char *q,
                                                                  const char *k_pool, const char *v_pool, int N, int max_pages,
                                                                  unsigned packed, int parts, const PagedParams p)
{
    constexpr int kSteps = D / 32;                        // matrix instructions per sub-tile of keys
    constexpr int kVE = D / 16;                           // channels of a value row that a lane loads
    constexpr int kVW = kVE / 2;                          // .. in 32-bit words
    typedef typename Vec<E>::v8 vec8;
    typedef unsigned words __attribute__((ext_vector_type(kVW)));
    constexpr int kJoin = NW * KG * (D + 2), kMerge = 4 + KG * (kMergeSplits + 1);
    __shared__ __align__(16) float lds[kJoin > kMerge ? kJoin : kMerge];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int kg = lane >> 4, c = lane & 15;
    const int G = packed & 0xff, shift = packed >> 8 & 0xff, B = packed >> 16;
    const int g = blockIdx.y;
    int b, S, n0, n1;                                     // this workgroup's sequence, its splits, the tokens [n0, n1)
    size_t first, part;                                   // partial of its split 0, and its own
    if constexpr (!DEALT) {                               // every sequence in as many splits
        const int split = blockIdx.x;
        b = blockIdx.z;
        S = parts;
        const int len = clamped_len(seq_lens, b, N);
        int chunk = (int)(((long long)len + S - 1) / S);
        chunk = (chunk + kTokens - 1) / kTokens * kTokens;
        const long long from = (long long)split * chunk;
        n0 = (int)(from < len ? from : len);
        n1 = (int)(from + chunk < len ? from + chunk : len);
        first = ((size_t)b * p.Hkv + g) * S;
        part = first + split;
    } else {
        // Splits of about as many tokens each, whatever the sequences' lengths: lane i has sequence i, in tiles of 32
        // tokens.  Every sequence's last split is shorter, so chunks are sized for a few splits less than there are
        // workgroups: a quarter of B less, or, where that makes too many, twice, three or four times that, which is enough
        // (of chunks of all / (grid - B) tiles, rounded up, there are grid - B and one more per sequence at most).
        const unsigned len = lane < B ? (unsigned)clamped_lane(seq_lens[lane], N) : 0u, own = (len + kTokens - 1) / kTokens;
        const unsigned all = __builtin_amdgcn_readlane(wave_upto(own), 63);
        unsigned pieces = 0, upto = 0;
        for (unsigned quarter = 1; quarter <= 4; ++quarter) {
            const unsigned room = (unsigned)parts - (quarter * (unsigned)B + 3) / 4;
            unsigned chunk = (all + room - 1) / room;
            chunk = chunk < (unsigned)p.least ? (unsigned)p.least : chunk;
            pieces = lane < B ? (own > chunk ? (own + chunk - 1) / chunk : 1u) : 0u;
            upto = wave_upto(pieces);
            if ((unsigned)__builtin_amdgcn_readlane(upto, 63) <= (unsigned)parts) break;
        }
        const unsigned long long mine = __ballot(blockIdx.x < upto);
        if (mine == 0) return;                            // fewer splits than workgroups
        b = __builtin_ctzll(mine);
        S = (int)__builtin_amdgcn_readlane(pieces, b);
        const unsigned before = __builtin_amdgcn_readlane(upto, b) - (unsigned)S, split = blockIdx.x - before;
        const unsigned total = __builtin_amdgcn_readlane(own, b), step = (total + S - 1) / S;
        const unsigned end = (split + 1) * step < total ? (split + 1) * step : total;
        const int n = (int)__builtin_amdgcn_readlane(len, b);
        n0 = (int)(split * step < total ? split * step : total) * kTokens;
        n1 = (int)end * kTokens < n ? (int)end * kTokens : n;
        if (n0 > n1) n0 = n1;
        first = (size_t)g * (unsigned)parts + before;
        part = first + split;
    }
    const size_t bg = (size_t)b * p.Hkv + g, row0 = (size_t)b * p.Hq + (size_t)g * G;
    arrival_t seen = 0;
    if (S > 1 && t == 0) seen = arrival_peek(p.words + bg * kWordStep);

    // The table's lines are asked for while the length travels, a lane each (2048 pages; only for the caches' sake:
    // 1000 tokens 7.7 us without it and with the merge's weights read one by one, 7.2 so).
    const int32_t *const pages = block_table + (size_t)b * max_pages;
    const int last_col = (N - 1) >> shift;
    if (!DEALT && wave == 0 && 32 * lane <= last_col) (void)*const_cast<const volatile int32_t *>(pages + 32 * lane);

    const unsigned slot_mask = (1u << shift) - 1;
    const char *const k0 = k_pool + (size_t)g * p.pages.k_head, *const v0 = v_pool + (size_t)g * p.pages.v_head;
    auto page_at = [&](int tok) {
        const int col = tok >> shift;
        return pages[col < last_col ? col : last_col];
    };

    float m, l;
    floatx4 acc[kVE];

    // The tiles of this wavefront, whose lane this is; `apart`: with infinite values taken out and added by themselves.
    auto tiles = [&](auto apart, int lane) {
        const int kg = lane >> 4, c = lane & 15;
        const int krow = 8 * (c >> 2) + (c & 3);          // this lane's key token of sub-tile 0; of sub-tile 1: + 4
        vec8 qf[kSteps];
        {
            const unsigned head = c < G ? ~0u : 0u;       // spare columns: zeros (by a mask: the request is not to wait for a branch)
            const char *const row = q + b * p.q_b + (long long)(g * G + (c < G ? c : 0)) * p.q_h;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                const uint4 x = reinterpret_cast<const uint4 *>(row)[4 * j + kg];
                qf[j] = as_vec<E>(x.x & head, x.y & head, x.z & head, x.w & head);
            }
        }
        // Keys and values of the next tile are requested as soon as this one's have been used, its pages a tile before that
        // (196608 tokens, 32 / 8 heads: 142 us with all requests at the tile's start, 139 so).  Values are not to be kept in any
        // cache: 125.  Keys are: a request takes 64 bytes of each row, half a cache line, and the next one the other half (without
        // caching 129 us, and a workgroup by itself a quarter slower).
        uint4 kr[2][kSteps];
        unsigned vr[8][kVW];
        auto load_k = [&](int t0, unsigned page) {
            const char *row = k0 + (size_t)(page < p.pages.num_pages ? page : 0u) * p.pages.k_page +
                              (size_t)((unsigned)(t0 + krow) & slot_mask) * p.pages.k_slot + 16 * kg;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int j = 0; j < kSteps; ++j) kr[u][j] = *reinterpret_cast<const uint4 *>(row + 64 * j);
                row += 4 * (size_t)p.pages.k_slot;
            }
        };
        auto load_v = [&](int t0, unsigned page) {
            const char *row = v0 + (size_t)(page < p.pages.num_pages ? page : 0u) * p.pages.v_page +
                              (size_t)((unsigned)(t0 + 8 * kg) & slot_mask) * p.pages.v_slot + 2 * kVE * c;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const words x = __builtin_nontemporal_load(reinterpret_cast<const words *>(row));
#pragma unroll
                for (int w = 0; w < kVW; ++w) vr[j][w] = x[w];
                row += p.pages.v_slot;
            }
        };
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < kVE; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
        int t0 = n0 + wave * kTokens;
        unsigned page_k = 0, page_v = 0;                  // of the tile in hand, then of the next
        if (t0 < n1) {
            page_k = (unsigned)page_at(t0 + krow);
            page_v = (unsigned)page_at(t0 + 8 * kg);
            load_k(t0, page_k);
            load_v(t0, page_v);
        }
        while (t0 < n1) {
            const bool there = page_v < p.pages.num_pages;
            const int tn = t0 + NW * kTokens;
            if (tn < n1) {
                page_k = (unsigned)page_at(tn + krow);
                page_v = (unsigned)page_at(tn + 8 * kg);
            }
            // ---- scores, in log2 units: head c, tokens t0 + 8 kg + e
            float s[8];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                floatx4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < kSteps; ++j) d = Vec<E>::mfma(__builtin_bit_cast(vec8, kr[u][j]), qf[j], d);
#pragma unroll
                for (int r = 0; r < 4; ++r) s[4 * u + r] = d[r] * p.scale2;
            }
            if (tn < n1) load_k(tn, page_k);
            // A tile with a hole, or the sequence's last: what is not there has no score, and whatever its rows hold (an
            // infinity times a probability of 0 is NaN) is taken out.
            if (t0 + kTokens > n1 || !__all(there)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool in = there && t0 + 8 * kg + e < n1;
                    s[e] = in ? s[e] : -INFINITY;
#pragma unroll
                    for (int w = 0; w < kVW; ++w) vr[e][w] = in ? vr[e][w] : 0u;
                }
            }
            if constexpr (SCORES) {
                if (c < G) {
                    float *const to = p.scores + (row0 + c) * p.n_pad + t0 + 8 * kg;
                    reinterpret_cast<float4 *>(to)[0] = make_float4(s[0], s[1], s[2], s[3]);
                    reinterpret_cast<float4 *>(to)[1] = make_float4(s[4], s[5], s[6], s[7]);
                }
            }

            // ---- softmax: every lane of a head has the same maximum, and a sum of its own tokens
            float top = s[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e]);
            top = rows_max(top);
            if (__any(top > m)) {
                const float to = fmaxf(m, top);
                const float f = weight_of(m, to);
                m = to;
                l *= f;
#pragma unroll
                for (int i = 0; i < kVE; ++i) acc[i] *= f;
            }
            const float base = m > -INFINITY ? m : 0.f;
            vec8 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float below = s[e] - base, x = __builtin_amdgcn_exp2f(Vec<E>::kLift > 0.f ? below + Vec<E>::kLift : below);
                l += x;
                hi[e] = (E)x;
                lo[e] = (E)(x - (float)hi[e]);
            }

            // ---- output
            auto turned = [&](const unsigned(&x)[8][kVW], int i) {
                const unsigned pick = i & 1 ? 0x07060302u : 0x05040100u;   // high or low halves of two rows' words
                return as_vec<E>(__builtin_amdgcn_perm(x[1][i / 2], x[0][i / 2], pick), __builtin_amdgcn_perm(x[3][i / 2], x[2][i / 2], pick),
                                 __builtin_amdgcn_perm(x[5][i / 2], x[4][i / 2], pick), __builtin_amdgcn_perm(x[7][i / 2], x[6][i / 2], pick));
            };
            if constexpr (decltype(apart)::value) {
                vec8 scored;
#pragma unroll
                for (int e = 0; e < 8; ++e) scored[e] = (E)(s[e] > -INFINITY ? 1.f : 0.f);
#pragma unroll
                for (int i = 0; i < kVE; ++i) {
                    const uintx4 a = __builtin_bit_cast(uintx4, turned(vr, i));
                    uintx4 inf;
#pragma unroll
                    for (int w = 0; w < 4; ++w) inf[w] = infinite_halves<E>(a[w]);
                    acc[i] = Vec<E>::mfma(__builtin_bit_cast(vec8, inf), scored, acc[i]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int w = 0; w < kVW; ++w) vr[e][w] &= ~infinite_halves<E>(vr[e][w]);
            }
#pragma unroll
            for (int i = 0; i < kVE; ++i) {
                const vec8 a = turned(vr, i);
                acc[i] = Vec<E>::mfma(a, hi, acc[i]);
                acc[i] = Vec<E>::mfma(a, lo, acc[i]);
            }
            if (tn < n1) load_v(tn, page_v);
            t0 = tn;
        }
    };
    tiles(std::false_type{}, lane);
    // An infinite value belongs into the output, however little it weighs, but times probabilities in two parts, of which either
    // may be 0 or negative, it makes no number.  A wavefront whose outputs are not all finite goes over its tiles once more, with
    // the infinities apart, at weight 1.  (A sum of numbers of which one is not finite is not.)
    floatx4 sum = acc[0];
#pragma unroll
    for (int i = 1; i < kVE; ++i) sum += acc[i];
    if (__builtin_expect(!__all(fabsf((sum[0] + sum[1]) + (sum[2] + sum[3])) < INFINITY), false)) {
        int again = lane;
        asm volatile("" : "+v"(again));                   // (addresses that both shared would be worked out in front of the first)
        tiles(std::true_type{}, again);
    }

    asm volatile("" : "+v"(seen));                        // (here, or the swap would wait for the partials' stores, which lie behind it in order)

    // ---- the wavefronts join
    l = rows_sum(l);
    float *const o_s = lds, *const m_s = lds + NW * KG * D, *const l_s = m_s + NW * KG;
    if (c < G) {
        float *const to = o_s + (wave * KG + c) * D;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < kVE; i += 4)
                *reinterpret_cast<float4 *>(to + (4 * kg + r) * kVE + i) = make_float4(acc[i][r], acc[i + 1][r], acc[i + 2][r], acc[i + 3][r]);
        if (kg == 0) {
            m_s[c * NW + wave] = m;
            l_s[c * NW + wave] = l;
        }
    }
    __syncthreads();
    for (int e = t; e < G * D; e += NW * 64) {
        const int h = e / D, ch = e - h * D;
        float mw[NW], lw[NW], M = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; w += 4) {
            const float4 a = *reinterpret_cast<const float4 *>(m_s + h * NW + w), b4 = *reinterpret_cast<const float4 *>(l_s + h * NW + w);
            mw[w] = a.x; mw[w + 1] = a.y; mw[w + 2] = a.z; mw[w + 3] = a.w;
            lw[w] = b4.x; lw[w + 1] = b4.y; lw[w + 2] = b4.z; lw[w + 3] = b4.w;
        }
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, mw[w]);
        const float at = M > -INFINITY ? M : 0.f;
        float den = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = weight_of(mw[w], at);
            den = fmaf(f, lw[w], den);
            o = fmaf(f, o_s[(w * KG + h) * D + ch], o);
        }
        if (S == 1) {
            static_cast<E *>(p.out)[(row0 + h) * D + ch] = (E)(den == 0.f ? 0.f : o / den);
            if (ch == 0) {
                const float total = den == 0.f ? -INFINITY : M + (log2f(den) - Vec<E>::kLift);
                if (p.lse) p.lse[row0 + h] = natural(total);
                if (p.norm) p.norm[row0 + h] = norm_of<E>(at, den);
            }
        } else {
            const size_t at_s = part * G + h;
            shared_store(p.part_o + at_s * D + ch, o);
            if (ch == 0) {
                shared_store(p.part_m + at_s, M);
                shared_store(p.part_l + at_s, den);
            }
        }
    }
    if (S == 1) return;
    if (t == 0) arrival_open(p.words + bg * kWordStep, seen, p.nonce);
    merge_last<E, D, KG, NW>(p, lds, p.words + bg * kWordStep, first, S, row0);
}

// The step's attention weights, summed over the heads of a KV head, onto the sums of its tokens.
__global__ __launch_bounds__(256) void paged_weights_kernel(const PagedParams p)
{
    const int g = blockIdx.y, b = blockIdx.z;
    const int len = clamped_len(p.seq_lens, b, p.N);
    const size_t row0 = (size_t)b * p.Hq + (size_t)g * p.G;
    const long long t = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
    if (t >= len) return;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int h = 0; h < p.G; ++h) {
        const float4 s = *reinterpret_cast<const float4 *>(p.scores + (row0 + h) * p.n_pad + t);
        const float2 n = p.norm[row0 + h];
        // (a hole weighs 0, also where the head's sum is no number)
        auto weight = [&](float score) { return score == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(score - n.x) * n.y; };
        sum.x += weight(s.x);
        sum.y += weight(s.y);
        sum.z += weight(s.z);
        sum.w += weight(s.w);
    }
    const float *const in = p.w_in ? p.w_in + ((size_t)b * p.Hkv + g) * p.w_cap + t : nullptr;
    float *const out = p.w_out + ((size_t)b * p.Hkv + g) * p.w_cap + t;
    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (t + i < len) out[i] = (in ? in[i] : 0.f) + v[i];
}

template <typename E, int D>
void start(const PagedParams &p, hipStream_t stream)
{
    constexpr int NW = 8;
    const dim3 grid((unsigned)p.S, (unsigned)p.Hkv, p.least ? 1u : (unsigned)p.B), block(NW * 64);
    const unsigned packed = (unsigned)p.G | (unsigned)p.pages.shift << 8 | (p.least ? (unsigned)p.B << 16 : 0u);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, 0, stream, p.seq_lens, p.block_table, p.q, p.pages.k, p.pages.v, p.N, (int)p.max_pages, packed, p.S, p);
    };
    // (LDS and the merge are made for up to 4, 8 or 16 query heads per KV head)
    auto heads = [&](auto scores, auto dealt) {
        constexpr bool s = decltype(scores)::value, d = decltype(dealt)::value;
        p.G <= 4 ? go(paged_attention_kernel<E, D, 4, NW, s, d>)
                 : (p.G <= 8 ? go(paged_attention_kernel<E, D, 8, NW, s, d>) : go(paged_attention_kernel<E, D, 16, NW, s, d>));
    };
    const std::true_type yes{};
    const std::false_type no{};
    if (p.scores)
        p.least ? heads(yes, yes) : heads(yes, no);
    else
        p.least ? heads(no, yes) : heads(no, no);
}

} // namespace

int launch_paged_attention(const PagedParams &p, int is_bf16, int D, hipStream_t stream)
{
    if (is_bf16)
        D == 128 ? start<bf16, 128>(p, stream) : start<bf16, 64>(p, stream);
    else
        D == 128 ? start<f16, 128>(p, stream) : start<f16, 64>(p, stream);
    return hipGetLastError() == hipSuccess ? 0 : -4;
}

int launch_paged_weights(const PagedParams &p, hipStream_t stream)
{
    const dim3 grid((unsigned)((p.N + 1023) / 1024), (unsigned)p.Hkv, (unsigned)p.B);
    hipLaunchKernelGGL(paged_weights_kernel, grid, dim3(256), 0, stream, p);
    return hipGetLastError() == hipSuccess ? 0 : -4;
}

} // namespace vecinfer
