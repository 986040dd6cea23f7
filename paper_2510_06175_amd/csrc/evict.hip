// Eviction from a paged cache by accumulated attention weight: which tokens of a (sequence, KV head) stay, and their
// move to pages of their own, in order.
//
// The choice: every token has a 32-bit key in the order of its weight; the first and the most recent ones have the
// largest key of all, tokens of a hole have key 0 and never stay.  The key T of the last one that stays is found by
// digits of 11, 11 and 10 bits: a histogram of the tokens that agree with T so far, and the bin at which, counted from the
// top, the room ends.  Then the tokens above T, and as many of those equal to it, lowest index first, as there is room for,
// are listed in order.
// What bounds it is issue: some 70 vector instructions per token, of which one compute unit does 64 lanes per cycle, and
// for short rows the steps themselves (500 tokens 7 us, 8192 9.8, 32000 22).  So a row of up to kHeld tokens, whose keys fit
// a workgroup's registers, is one workgroup's in one launch, and a longer one is cut into up to kMaxParts stretches, a launch
// per digit and one for the list, through a histogram per stretch: each workgroup of the next launch adds them up for
// itself, which needs no atomics, no clearing and no order of workgroups (100003 tokens: 24 us in four launches; by one
// workgroup, the row read again for each digit, 89).
// The move: 16 lanes per row of a kept token, keys and values; bound by memory (32768 of 100003 tokens, 8 KV heads, 268 MB:
// 52 us, the rate of a large copy).
#include "paged.h"

namespace vecinfer {

namespace {

constexpr int kSelect = 1024, kWaves = kSelect / 64;
constexpr int kBins = 2048;
constexpr int kCopies = 4;                                // of a histogram in LDS: neighbouring lanes count apart
// Turns of 256 tokens per wavefront whose keys are held in registers, by a workgroup that has a row for itself (1, 2, 4 or
// 8, as the row needs: 4000 tokens 14.2 us with one, 15.1 with eight) and by one that shares it: so many are read once (one
// sequence of 20000 tokens, 8 KV heads, keeping 2000: 24.2 us by a workgroup per row, 33.3 shared; 32000 30.3 and 33.6).
constexpr int kTurnsWhole = 8, kTurnsPart = 4;
constexpr int kHeld = kSelect * 4 * kTurnsWhole, kHeldPart = kSelect * 4 * kTurnsPart;
constexpr int kPart = kHeldPart / 4;                      // least tokens of a stretch
constexpr int kMaxParts = 64;
constexpr int kGroup = 32, kGroups = kBins / kGroup, kHist = kBins + kGroups;    // a stretch's histogram in memory

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

struct Shared {
    unsigned hist[kBins * kCopies];
    __align__(16) unsigned above[kWaves], equal[kWaves], sums[kWaves];
    unsigned pick[2];
    unsigned all[kWaves][kGroups], mine[kWaves][kGroups];
};

// What a workgroup knows of its tokens [from, to) of a row, of which this wavefront has [mine, mine_to).
template <int kTurns>
struct Stretch {
    const float *w;
    const int32_t *pages;
    unsigned num_pages;
    int shift, len, first, recent_from;
    int mine, mine_to;
    bool held;                                            // k has all the keys
    unsigned k[kTurns][4];

    // The keys of tokens i .. i + 3 (i a multiple of 4: they share a page); behind the end: 0.
    __device__ __forceinline__ void keys4(int i, unsigned (&key)[4]) const
    {
        key[0] = key[1] = key[2] = key[3] = 0u;
        if (i >= mine_to) return;
        const unsigned page = (unsigned)pages[i >> shift];
        Four f;
        if (i + 3 < mine_to) {
            f = *reinterpret_cast<const Four *>(w + i);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) f.v[e] = i + e < mine_to ? w[i + e] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            key[e] = i + e < first || i + e >= recent_from ? 0xffffffffu : weight_key(f.v[e]);
            if (page >= num_pages || i + e >= mine_to) key[e] = 0u;
        }
    }
    __device__ __forceinline__ void read(int from)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int a = 0; a < kTurns; ++a) keys4(from + 256 * a + 4 * lane, k[a]);
    }
    __device__ __forceinline__ void open(const EvictParams &p, int g, int b, int part, int parts)
    {
        const size_t bg = (size_t)b * p.Hkv + g;
        w = p.w + bg * p.w_cap;
        pages = p.block_table + b * p.max_pages;
        num_pages = p.src.num_pages;
        shift = p.src.shift;
        len = clamped_len(p.seq_lens, b, p.N);
        first = p.first;
        recent_from = len - p.recent;
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        const long long stretch = parts * kWaves, step = ((long long)len + 256 * stretch - 1) / (256 * stretch) * 256;
        const long long at = (part * kWaves + wave) * step;
        mine = (int)(at < len ? at : len);
        mine_to = (int)(at + step < len ? at + step : len);
        held = step <= 256 * kTurns;
        if (held) read(mine);
    }
    // f(first token, keys) for the lane's fours of this wavefront's tokens, in order
    template <typename F>
    __device__ __forceinline__ void each(F &&f)
    {
        const int lane = threadIdx.x & 63;
        for (int i = mine; i < mine_to; i += 256 * kTurns) {
            if (!held) read(i);
#pragma unroll
            for (int a = 0; a < kTurns; ++a)
                if (i + 256 * a < mine_to) f(i + 256 * a + 4 * lane, k[a]);
        }
    }
};

__device__ __forceinline__ void clear_hist(Shared &s)
{
    static_assert(kCopies == 4, "16 bytes per bin");
    for (int i = threadIdx.x; i < kBins; i += kSelect) reinterpret_cast<uint4 *>(s.hist)[i] = make_uint4(0, 0, 0, 0);
}

// Histogram of the next digit over the tokens whose digits so far are `prefix`.  Ends behind a barrier.
template <int DIGIT, int kTurns>
__device__ __forceinline__ void count_digit(Shared &s, Stretch<kTurns> &x, unsigned prefix)
{
    constexpr int kAt = DIGIT == 1 ? 21 : (DIGIT == 2 ? 10 : 0);
    constexpr unsigned kMask = DIGIT == 3 ? 1023u : 2047u;
    const int copy = threadIdx.x & (kCopies - 1);
    clear_hist(s);
    __syncthreads();
    x.each([&](int, const unsigned(&k)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (DIGIT == 1) {
                // (what is always kept comes by the wavefront, and would queue for one place)
                const unsigned long long always = __ballot(k[e] == 0xffffffffu);
                if (always && (threadIdx.x & 63) == 0) atomicAdd(&s.hist[(kBins - 1) * kCopies], (unsigned)__popcll(always));
                if (k[e] && k[e] != 0xffffffffu) atomicAdd(&s.hist[(k[e] >> kAt) * kCopies + copy], 1u);
            } else {
                if (k[e] && k[e] >> (DIGIT == 2 ? 21 : 10) == prefix) atomicAdd(&s.hist[(k[e] >> kAt & kMask) * kCopies + copy], 1u);
            }
        }
    });
    __syncthreads();
}

// This thread's two bins, the upper one first.
__device__ __forceinline__ void own_bins(const Shared &s, unsigned (&h)[2])
{
    static_assert(kBins == 2 * kSelect, "two bins per thread");
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4 c = reinterpret_cast<const uint4 *>(s.hist)[kBins - 1 - (2 * (int)threadIdx.x + i)];
        h[i] = c.x + c.y + c.z + c.w;
    }
}

// Sum of the wavefronts' counts before this one's.
__device__ __forceinline__ unsigned before_wave(const unsigned (&counts)[kWaves], int wave)
{
    unsigned sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; w += 4) {
        const uint4 c = *reinterpret_cast<const uint4 *>(counts + w);
        sum += (w < wave ? c.x : 0u) + (w + 1 < wave ? c.y : 0u) + (w + 2 < wave ? c.z : 0u) + (w + 3 < wave ? c.w : 0u);
    }
    return sum;
}

// The bin (h: this thread's two) at which, counted from the top, the room ends: returned, and the tokens above it taken
// off the room; kBins: there is room for all.  Called by all threads, ends behind a barrier.
__device__ __forceinline__ unsigned find_bin(Shared &s, const unsigned (&h)[2], unsigned &room)
{
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const unsigned upto = wave_upto(h[0] + h[1]);
    if (lane == 63) s.sums[wave] = upto;
    if (t == 0) {
        s.pick[0] = kBins;
        s.pick[1] = 0;
    }
    __syncthreads();
    unsigned before = upto - h[0] - h[1] + before_wave(s.sums, wave);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (before <= room && room < before + h[i]) {     // (one bin of all)
            s.pick[0] = kBins - 1 - (2 * t + i);
            s.pick[1] = before;
        }
        before += h[i];
    }
    __syncthreads();
    const unsigned bin = s.pick[0];
    room -= s.pick[1];
    return bin;
}

// find_bin over the sum of the stretches' histograms in memory; and of the stretches before `part`, how many tokens lie
// above the bin and in it.  First the group of bins in which the room ends, by the sums, then the bin in it, so that a
// workgroup reads 384 bytes of each stretch and not 8 KB (all bins of 13 stretches took 5 us more per launch).
__device__ __forceinline__ unsigned find_bin_of_parts(Shared &s, const unsigned *hists, int part, int parts, unsigned &room, unsigned &more,
                                                      unsigned &same)
{
    static_assert(kGroups == 64 && kGroup == 32 && kMaxParts * kGroup <= 2 * kSelect, "a lane per group; two rounds of bins");
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    // from the top: lane 0 has the highest group
    unsigned total = 0, before = 0;
    for (int q = wave; q < parts; q += kWaves) {
        const unsigned v = hists[(size_t)q * kHist + kBins + kGroups - 1 - lane];
        total += v;
        before += q < part ? v : 0u;
    }
    s.all[wave][lane] = total;
    s.mine[wave][lane] = before;
    __syncthreads();
    // (every wavefront the same, so that nobody waits for one)
    total = before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        total += s.all[w][lane];
        before += s.mine[w][lane];
    }
    const unsigned upto = wave_upto(total), from_top = upto - total, mine_upto = wave_upto(before);
    const unsigned long long here = __ballot(from_top <= room && room < upto);
    if (here == 0) {                                      // there is room for all
        more = __shfl(mine_upto, 63);
        same = 0;
        return kBins;
    }
    const int group = __builtin_ctzll(here);
    const unsigned above = __shfl(from_top, group);
    more = __shfl(mine_upto - before, group);
    __syncthreads();
    // the group's bins, the highest first: thread t has bin t % 32 of stretches t / 32 and 32 + t / 32
    const int bin = t % kGroup;
    total = before = 0;
#pragma unroll
    for (int q = t / kGroup; q < kMaxParts; q += kSelect / kGroup) {
        if (q >= parts) break;
        const unsigned v = hists[(size_t)q * kHist + (kGroups - 1 - group) * kGroup + kGroup - 1 - bin];
        total += v;
        before += q < part ? v : 0u;
    }
    total += __shfl_xor(total, 32);                       // a wavefront's two rows of bins
    before += __shfl_xor(before, 32);
    if (lane < kGroup) {
        s.all[wave][lane] = total;
        s.mine[wave][lane] = before;
    }
    __syncthreads();
    total = before = 0;
    if (lane < kGroup)
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            total += s.all[w][lane];
            before += s.mine[w][lane];
        }
    const unsigned bin_upto = above + wave_upto(total), bin_top = bin_upto - total, mine_bin = wave_upto(before);
    const int at = __builtin_ctzll(__ballot(bin_top <= room && room < bin_upto));
    more += __shfl(mine_bin - before, at);
    same = __shfl(before, at);
    room -= __shfl(bin_top, at);
    return (kGroups - 1 - group) * kGroup + kGroup - 1 - at;
}

// The list of what stays: tokens above T and, of those equal to it, the first `room` of the row.  `taken` stay and `ties`
// are equal to T in front of this workgroup's tokens (T = 0: all that are there stay, room = 0).
template <int kTurns>
__device__ __forceinline__ void list_kept(Shared &s, Stretch<kTurns> &x, const EvictParams &p, int g, int b, bool last, unsigned T, unsigned room,
                                          unsigned taken, unsigned ties)
{
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    int32_t *const ids = p.ids + ((size_t)b * p.Hkv + g) * (p.keep < p.N ? p.keep : p.N);
    unsigned above = 0, equal = 0;
    x.each([&](int, const unsigned(&k)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            above += __popcll(__ballot(k[e] > T));
            if (room) equal += __popcll(__ballot(k[e] == T));              // (room > 0: T > 0, so only tokens that are there)
        }
    });
    if (lane == 0) {
        s.above[wave] = above;
        s.equal[wave] = equal;
    }
    __syncthreads();
    taken += before_wave(s.above, wave);
    ties += before_wave(s.equal, wave);
    taken += ties < room ? ties : room;
    const unsigned long long lower = ~(~0ull << lane);
    x.each([&](int i, const unsigned(&k)[4]) {
        bool stays[4];
        unsigned long long eq[4], any = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            stays[e] = k[e] > T;
            eq[e] = room ? __ballot(k[e] == T) : 0ull;
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
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned long long st = __ballot(stays[e]);
            at += __popcll(st & lower);
            taken += __popcll(st);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (stays[e] && at < (unsigned)p.keep) ids[at++] = i + e;     // (weights that change meanwhile may be counted otherwise)
    });
    if (last && g == 0 && wave == kWaves - 1 && lane == 0) p.dst_lens[b] = (int)(taken < (unsigned)p.keep ? taken : (unsigned)p.keep);
}

// A row per workgroup: grid (KV heads, sequences).
template <int TURNS>
__global__ __launch_bounds__(kSelect) void evict_select_kernel(const EvictParams p)
{
    __shared__ __align__(16) Shared s;
    const int g = blockIdx.x, b = blockIdx.y;
    Stretch<TURNS> x;
    x.open(p, g, b, 0, 1);
    unsigned h[2], room = (unsigned)p.keep, T = 0;
    count_digit<1>(s, x, 0);
    own_bins(s, h);
    const unsigned d1 = find_bin(s, h, room);
    if (d1 == kBins) {
        room = 0;
    } else {
        count_digit<2>(s, x, d1);
        own_bins(s, h);
        const unsigned d12 = d1 << 11 | find_bin(s, h, room);
        count_digit<3>(s, x, d12);
        own_bins(s, h);
        T = d12 << 10 | find_bin(s, h, room);
    }
    list_kept(s, x, p, g, b, true, T, room, 0, 0);
}

// A stretch of a row per workgroup, grid (parts, KV heads, sequences): stage 1, 2, 3 count that digit of T, having found
// the one before, stage 4 lists.
//   p.hists   [stages 1 .. 3][rows][parts][kHist]: the bins, and behind them their sums by kGroup
//   p.states  [rows][parts][3]: the digits found, the room left behind them, and of the stretches before the tokens above
// Every workgroup of a row finds the same digits, each for itself.
template <int STAGE>
__global__ __launch_bounds__(kSelect) void evict_stage_kernel(const EvictParams p)
{
    __shared__ __align__(16) Shared s;
    const int t = threadIdx.x, part = blockIdx.x, parts = gridDim.x, g = blockIdx.y, b = blockIdx.z;
    const size_t row = (size_t)b * p.Hkv + g, rows = (size_t)p.B * p.Hkv;
    unsigned *const hists = p.hists + row * parts * kHist;
    unsigned *const state = p.states + (row * parts + part) * 3;
    Stretch<kTurnsPart> x;
    x.open(p, g, b, part, parts);
    unsigned found = 0, room = (unsigned)p.keep, taken = 0, ties = 0;
    bool all = false;
    if constexpr (STAGE > 1) {
        if constexpr (STAGE > 2) {
            found = state[0];
            room = state[1];
            taken = state[2];
            all = found == ~0u;
        }
        if (!all) {
            const unsigned *const in = hists + (STAGE - 2) * rows * parts * kHist;
            unsigned more, same;                          // tokens above and in the bin in the stretches before this one
            const unsigned d = find_bin_of_parts(s, in, part, parts, room, more, same);
            all = d == kBins;
            taken += more;
            ties = STAGE == 4 ? same : 0;
            found = all ? ~0u : found << (STAGE == 4 ? 10 : 11) | d;
            if (STAGE < 4 && t == 0) {
                state[0] = found;
                state[1] = room;
                state[2] = taken;
            }
        }
    }
    if constexpr (STAGE < 4) {
        if (all) return;
        count_digit<STAGE>(s, x, found);
        unsigned h[2];
        own_bins(s, h);
        unsigned *const out = hists + ((STAGE - 1) * rows * parts + part) * kHist;
        *reinterpret_cast<uint2 *>(out + (kBins - 2 - 2 * t)) = make_uint2(h[1], h[0]);
        unsigned sum = h[0] + h[1];                       // 16 threads have a group's bins
#pragma unroll
        for (int o = 1; o < kGroup / 2; o <<= 1) sum += __shfl_xor(sum, o);
        if (t % (kGroup / 2) == 0) out[kBins + kGroups - 1 - t / (kGroup / 2)] = sum;
    } else {
        list_kept(s, x, p, g, b, part == parts - 1, all ? 0u : found, all ? 0u : room, taken, ties);
    }
}

// from_place: the first place of this launch
template <int D, bool STREAM>
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams p, int from_place)
{
    constexpr int kLanes = D / 8;                         // 16-byte pieces of a row
    const int t = threadIdx.x, piece = t % kLanes;
    const int j = from_place + (int)blockIdx.x * (256 / kLanes) + t / kLanes, g = blockIdx.y, b = blockIdx.z;
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
    const uint4 k = load16<STREAM>(p.src.k + (size_t)from * p.src.k_page + (size_t)g * p.src.k_head + fs * p.src.k_slot, piece);
    const uint4 v = load16<STREAM>(p.src.v + (size_t)from * p.src.v_page + (size_t)g * p.src.v_head + fs * p.src.v_slot, piece);
    store16<STREAM>(p.dst.k + (size_t)to * p.dst.k_page + (size_t)g * p.dst.k_head + ts * p.dst.k_slot, piece, k);
    store16<STREAM>(p.dst.v + (size_t)to * p.dst.v_page + (size_t)g * p.dst.v_head + ts * p.dst.v_slot, piece, v);
}

} // namespace

// Workgroups that share a row in the choice: as many as fill the chip once, of 4096 tokens at least and 16384, whose keys
// are held, at most (8 rows, us of the whole call at 48000 / 100003 / 196000 tokens: stretches of 4096 35.5 / 78.4 / 47.3, of
// 8192 38.0 / 81.0 / 39.8, of 16384 44.9 / 87.1 / 45.6; at 196000 stretches of 4096 are 384 workgroups).
int evict_parts(long long rows, long long N)
{
    if (N <= kHeld) return 1;
    long long parts = num_cus() / rows;
    const long long most = (N + kPart - 1) / kPart, least = (N + kHeldPart - 1) / kHeldPart;
    if (parts > most) parts = most;
    if (parts < least) parts = least;
    return (int)(parts < kMaxParts ? parts : kMaxParts);
}

// Stretches that the workspace has room for.  More rows have fewer parts each, and fewer in all where these come in whole numbers
// (56 rows of 40000 tokens 224, 32 rows 256), so not as many as evict_parts makes, but a bound that grows with both: a
// workspace for more rows or longer ones serves fewer and shorter ones.
static size_t evict_room(long long rows, long long N)
{
    if (N <= kHeld) return 0;
    const long long most = (N + kPart - 1) / kPart, least = (N + kHeldPart - 1) / kHeldPart;
    const long long filled = rows * least > num_cus() ? rows * least : num_cus(), cut = rows * (most < kMaxParts ? most : kMaxParts);
    return (size_t)(filled < cut ? filled : cut);
}

size_t evict_hist_elems(long long rows, long long N) { return 3 * evict_room(rows, N) * kHist; }

size_t evict_state_elems(long long rows, long long N) { return 3 * evict_room(rows, N); }

int launch_evict(const EvictParams &p, hipStream_t stream)
{
    const int parts = evict_parts((long long)p.B * p.Hkv, p.N);
    if (parts == 1) {
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)p.Hkv, (unsigned)p.B), dim3(kSelect), 0, stream, p); };
        const int turns = (p.N + 4 * kSelect - 1) / (4 * kSelect);
        turns <= 1 ? go(evict_select_kernel<1>)
        : turns <= 2 ? go(evict_select_kernel<2>)
        : turns <= 4 ? go(evict_select_kernel<4>)
                     : go(evict_select_kernel<kTurnsWhole>);
    } else {
        const dim3 grid((unsigned)parts, (unsigned)p.Hkv, (unsigned)p.B);
        hipLaunchKernelGGL(evict_stage_kernel<1>, grid, dim3(kSelect), 0, stream, p);
        hipLaunchKernelGGL(evict_stage_kernel<2>, grid, dim3(kSelect), 0, stream, p);
        hipLaunchKernelGGL(evict_stage_kernel<3>, grid, dim3(kSelect), 0, stream, p);
        hipLaunchKernelGGL(evict_stage_kernel<4>, grid, dim3(kSelect), 0, stream, p);
    }
    const int rows = 256 / (p.D / 8);
    const int most = p.keep < p.N ? p.keep : p.N;
    // (up to 2^22 workgroups along the places: 2^32 threads and more are not launched)
    auto go = [&](auto kernel) {
        for (int at = 0; at < most; at += rows << 22) {
            const int left = most - at < rows << 22 ? most - at : rows << 22;
            hipLaunchKernelGGL(kernel, dim3((unsigned)((left + rows - 1) / rows), (unsigned)p.Hkv, (unsigned)p.B), dim3(256), 0, stream, p, at);
        }
    };
    const bool streams = 8ll * p.D * most * p.Hkv * p.B >= kStreamBytes;
    if (p.D == 128)
        streams ? go(evict_move_kernel<128, true>) : go(evict_move_kernel<128, false>);
    else
        streams ? go(evict_move_kernel<64, true>) : go(evict_move_kernel<64, false>);
    return hipGetLastError() == hipSuccess ? 0 : -4;
}

} // namespace vecinfer
