// Eviction from a paged cache by accumulated attention weight: which tokens of a (sequence, KV head) stay, and their
// move to pages of their own, in order.
//
// The choice: every token has a 32-bit key in the order of its weight; the first and the most recent ones have the
// largest key of all, tokens of a hole have key 0 and never stay.  One workgroup per (sequence, KV head) looks for the
// key T of the last one that stays, by digits of 11, 11 and 10 bits, and reads the row three times: a histogram of the
// first digit; then, of the tokens that have T's first digit, the other bits into a list in LDS, from which the other two
// digits are found; then the tokens above T, and as many of those equal to it, lowest index first, as there is room for,
// are listed in order.  Each of the 16 wavefronts takes a stretch of the row in the second and third reading, so that
// the third knows where each has to start.  (A list that does not fit, thousands of equal weights say, stays where it is:
// the row is read again for each digit.)
// What bounds it is one compute unit's reading and counting: PLACEHOLDER_FIGURES
// The move: 16 lanes per row of a kept token, keys and values.
#include "paged.h"

namespace vecinfer {

namespace {

constexpr int kSelect = 1024, kWaves = kSelect / 64;
constexpr int kBins = 2048;
constexpr int kCopies = 4;                                // of a histogram: lanes of neighbouring tokens count apart
constexpr int kList = 24576;                              // tokens of T's first digit that LDS has room for

// Order of weights as unsigned numbers: -inf < .. < -0 = 0 < .. < inf; what is no number comes below all.
__device__ __forceinline__ unsigned weight_key(float w)
{
    if (w != w) return 1u;
    const unsigned u = __float_as_uint(w + 0.f);          // (-0 + 0 = 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct __attribute__((packed, aligned(4))) Four {
    float v[4];
};

struct Row {
    const float *w;
    const int32_t *pages;
    unsigned num_pages;
    int shift, len, first, recent_from;
};

// The keys of tokens i .. i + 3 (i a multiple of 4: they share a page); behind the end: 0.
__device__ __forceinline__ void keys4(const Row &r, int i, unsigned (&k)[4])
{
    k[0] = k[1] = k[2] = k[3] = 0u;
    if (i >= r.len) return;
    const unsigned page = (unsigned)r.pages[i >> r.shift];
    Four f;
    if (i + 3 < r.len) {
        f = *reinterpret_cast<const Four *>(r.w + i);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f.v[e] = i + e < r.len ? r.w[i + e] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        k[e] = i + e < r.first || i + e >= r.recent_from ? 0xffffffffu : weight_key(f.v[e]);
        if (page >= r.num_pages || i + e >= r.len) k[e] = 0u;
    }
}

// f(keys) for the tokens [from, to), 256 per wavefront and turn, `step` tokens apart; four turns are requested together.
template <typename F>
__device__ __forceinline__ void each(const Row &r, int from, int to, int step, F &&f)
{
    constexpr int kAhead = 4;
    for (int i = from; i < to; i += kAhead * step) {
        unsigned k[kAhead][4];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) keys4(r, i + a * step < to ? i + a * step + 4 * (int)(threadIdx.x & 63) : r.len, k[a]);
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (i + a * step < to) f(i + a * step + 4 * (int)(threadIdx.x & 63), k[a]);
    }
}

__device__ __forceinline__ unsigned wave_prefix(unsigned v, int lane)       // inclusive
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned x = __shfl_up(v, o);
        if (lane >= o) v += x;
    }
    return v;
}

struct Shared {
    unsigned hist[kBins * kCopies];
    unsigned list[kList];
    unsigned above[kWaves], equal[kWaves], sums[kWaves];
    unsigned listed, pick[3];
};

// The bin at which, counted from the top, the room ends: in pick[0]; the tokens above it in pick[1], in it in pick[2].
// pick[0] = kBins: there is room for all.  Called by all threads, histogram complete; ends behind a barrier.
__device__ __forceinline__ void find_bin(Shared &s, unsigned room)
{
    static_assert(kBins == 2 * kSelect, "two bins per thread");
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    unsigned h[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4 c = reinterpret_cast<const uint4 *>(s.hist)[kBins - 1 - (2 * t + i)];
        h[i] = c.x + c.y + c.z + c.w;
    }
    const unsigned upto = wave_prefix(h[0] + h[1], lane);
    if (lane == 63) s.sums[wave] = upto;
    if (t == 0) s.pick[0] = kBins;
    __syncthreads();
    unsigned before = upto - h[0] - h[1];
    for (int w = 0; w < wave; ++w) before += s.sums[w];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (before <= room && room < before + h[i]) {     // (one bin of all)
            s.pick[0] = kBins - 1 - (2 * t + i);
            s.pick[1] = before;
            s.pick[2] = h[i];
        }
        before += h[i];
    }
    __syncthreads();
}

__device__ __forceinline__ void clear_hist(Shared &s)
{
    static_assert(kCopies == 4, "16 bytes per bin");
    for (int i = threadIdx.x; i < kBins; i += kSelect) reinterpret_cast<uint4 *>(s.hist)[i] = make_uint4(0, 0, 0, 0);
}

__global__ __launch_bounds__(kSelect) void evict_select_kernel(const EvictParams p)
{
    __shared__ __align__(16) Shared s;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int g = blockIdx.x, b = blockIdx.y;
    const size_t bg = (size_t)b * p.Hkv + g;
    Row row;
    row.w = p.w + bg * p.w_cap;
    row.pages = p.block_table + b * p.max_pages;
    row.num_pages = p.src.num_pages;
    row.shift = p.src.shift;
    row.len = clamped_len(p.seq_lens, b, p.N);
    row.first = p.first;
    row.recent_from = row.len - p.recent;
    int32_t *const ids = p.ids + bg * (p.keep < p.N ? p.keep : p.N);
    const int copy = lane & (kCopies - 1);
    // a wavefront's stretch of the row
    const int seg = (row.len + 256 * kWaves - 1) / (256 * kWaves) * 256;
    const int from = wave * seg < row.len ? wave * seg : row.len, to = from + seg < row.len ? from + seg : row.len;

    // ---- T's first digit
    clear_hist(s);
    if (t < kWaves) s.above[t] = s.equal[t] = 0;
    if (t == 0) s.listed = 0;
    __syncthreads();
    each(row, from, to, 256, [&](int, const unsigned(&k)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (k[e]) atomicAdd(&s.hist[(k[e] >> 21) * kCopies + copy], 1u);
    });
    __syncthreads();
    unsigned room = (unsigned)p.keep;
    find_bin(s, room);
    const bool all = s.pick[0] == kBins;                  // every token that is there stays
    const unsigned d1 = s.pick[0], count = s.pick[2];
    unsigned T = 0;
    if (!all) {
        room -= s.pick[1];
        const bool fits = count <= kList;
        __syncthreads();
        // ---- the tokens of that digit, tagged with the wavefront whose stretch they are in; those above it are counted
        clear_hist(s);
        __syncthreads();
        unsigned mine = 0;
        each(row, from, to, 256, [&](int, const unsigned(&k)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned d = k[e] >> 21;
                mine += d > d1;
                const bool in = k[e] && d == d1;
                if (in) atomicAdd(&s.hist[(k[e] >> 10 & (kBins - 1)) * kCopies + copy], 1u);
                if (fits) {
                    const unsigned long long who = __ballot(in);
                    unsigned at = 0;
                    if (who && lane == 0) at = atomicAdd(&s.listed, (unsigned)__popcll(who));
                    at = __builtin_amdgcn_readfirstlane(at);
                    at += __popcll(who & ~(~0ull << lane));
                    if (in && at < kList) s.list[at] = (unsigned)wave << 21 | (k[e] & 0x1fffffu);
                }
            }
        });
        if (mine) atomicAdd(&s.above[wave], mine);
        __syncthreads();
        find_bin(s, room);
        const unsigned d2 = s.pick[0];
        room -= s.pick[1];
        __syncthreads();
        clear_hist(s);
        __syncthreads();
        const unsigned top = d1 << 11 | d2;               // the first 22 bits of T
        if (fits) {
            for (unsigned i = t; i < count; i += kSelect)
                if ((s.list[i] >> 10 & (kBins - 1)) == d2) atomicAdd(&s.hist[(s.list[i] & 1023u) * kCopies + copy], 1u);
        } else {
            each(row, from, to, 256, [&](int, const unsigned(&k)[4]) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (k[e] && k[e] >> 10 == top) atomicAdd(&s.hist[(k[e] & 1023u) * kCopies + copy], 1u);
            });
        }
        __syncthreads();
        find_bin(s, room);
        room -= s.pick[1];
        T = top << 10 | s.pick[0];
        // ---- how many tokens above T and equal to it each stretch has
        if (fits) {
            for (unsigned i = t; i < count; i += kSelect) {
                const unsigned x = s.list[i], low = x & 0x1fffffu;
                if (low > (T & 0x1fffffu)) atomicAdd(&s.above[x >> 21], 1u);
                if (low == (T & 0x1fffffu)) atomicAdd(&s.equal[x >> 21], 1u);
            }
        } else {
            unsigned more = 0, same = 0;
            each(row, from, to, 256, [&](int, const unsigned(&k)[4]) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    more += k[e] > T && k[e] >> 21 == d1;
                    same += k[e] == T;
                }
            });
            if (more) atomicAdd(&s.above[wave], more);
            if (same) atomicAdd(&s.equal[wave], same);
        }
    } else {
        unsigned mine = 0;                                // T = 0: all keys are above it
        each(row, from, to, 256, [&](int, const unsigned(&k)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) mine += k[e] != 0u;
        });
        if (mine) atomicAdd(&s.above[wave], mine);
        room = 0;
    }
    __syncthreads();

    // ---- the list: behind the tokens of the stretches before, `taken` of them, `ties` equal to T
    unsigned ties = 0, taken = 0;
    for (int w = 0; w < wave; ++w) {
        ties += s.equal[w];
        taken += s.above[w];
    }
    taken += ties < room ? ties : room;
    const unsigned long long lower = ~(~0ull << lane);
    each(row, from, to, 256, [&](int i, const unsigned(&k)[4]) {
        bool stays[4];
        unsigned long long eq[4], any = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            stays[e] = k[e] > T;
            eq[e] = room ? __ballot(k[e] == T) : 0ull;    // (room > 0: T > 0, so no key that is not there)
            any |= eq[e];
        }
        if (any && ties < room) {
            unsigned before = ties;
#pragma unroll
            for (int e = 0; e < 4; ++e) before += __popcll(eq[e] & lower);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (k[e] == T) stays[e] = before++ < room;
                ties += __popcll(eq[e]);
            }
        }
        unsigned at = taken;
        unsigned long long st[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            st[e] = __ballot(stays[e]);
            at += __popcll(st[e] & lower);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (stays[e] && at < (unsigned)p.keep) ids[at++] = i + e;     // (weights that change meanwhile may be counted otherwise)
            taken += __popcll(st[e]);
        }
    });
    if (g == 0 && wave == kWaves - 1 && lane == 0) p.dst_lens[b] = (int)(taken < (unsigned)p.keep ? taken : (unsigned)p.keep);
}

template <int D>
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams p)
{
    constexpr int kLanes = D / 8;                         // 16-byte pieces of a row
    const int t = threadIdx.x, piece = t % kLanes;
    const int j = blockIdx.x * (256 / kLanes) + t / kLanes, g = blockIdx.y, b = blockIdx.z;
    if (j >= p.dst_lens[b]) return;
    const size_t bg = (size_t)b * p.Hkv + g;
    const int i = p.ids[bg * (p.keep < p.N ? p.keep : p.N) + j];
    if (piece == 0) {
        if (p.kept) p.kept[bg * p.keep + j] = i;
        if (p.dst_w) p.dst_w[bg * p.dst_w_cap + j] = p.w[bg * p.w_cap + i];
    }
    const unsigned from = (unsigned)p.block_table[b * p.max_pages + (i >> p.src.shift)];
    const unsigned to = (unsigned)p.dst_table[b * p.dst_max_pages + (j >> p.dst.shift)];
    if (from >= p.src.num_pages || to >= p.dst.num_pages) return;
    const size_t fs = (unsigned)i & ((1u << p.src.shift) - 1), ts = (unsigned)j & ((1u << p.dst.shift) - 1);
    const uint4 k = reinterpret_cast<const uint4 *>(p.src.k + (size_t)from * p.src.k_page + (size_t)g * p.src.k_head + fs * p.src.k_slot)[piece];
    const uint4 v = reinterpret_cast<const uint4 *>(p.src.v + (size_t)from * p.src.v_page + (size_t)g * p.src.v_head + fs * p.src.v_slot)[piece];
    reinterpret_cast<uint4 *>(p.dst.k + (size_t)to * p.dst.k_page + (size_t)g * p.dst.k_head + ts * p.dst.k_slot)[piece] = k;
    reinterpret_cast<uint4 *>(p.dst.v + (size_t)to * p.dst.v_page + (size_t)g * p.dst.v_head + ts * p.dst.v_slot)[piece] = v;
}

} // namespace

int launch_evict(const EvictParams &p, hipStream_t stream)
{
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)p.Hkv, (unsigned)p.B), dim3(kSelect), 0, stream, p);
    const int rows = 256 / (p.D / 8);
    const int most = p.keep < p.N ? p.keep : p.N;
    const dim3 grid((unsigned)((most + rows - 1) / rows), (unsigned)p.Hkv, (unsigned)p.B);
    if (p.D == 128)
        hipLaunchKernelGGL(evict_move_kernel<128>, grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL(evict_move_kernel<64>, grid, dim3(256), 0, stream, p);
    return hipGetLastError() == hipSuccess ? 0 : -4;
}

} // namespace vecinfer
