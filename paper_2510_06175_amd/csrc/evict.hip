// Eviction from a paged cache by accumulated attention weight: which tokens of a (sequence, KV head) stay, and their
// move to pages of their own, in order.
//
// The choice: every token has a 32-bit key in the order of its weight; the first and the most recent ones have the
// largest key of all, tokens of a hole have key 0 and never stay.  A workgroup per (sequence, KV head) finds the key
// of the last one that stays, digit by digit from the top (a histogram of 256 per digit, 4 passes over the row), and then
// lists, in order, the tokens above it and as many of those equal to it, lowest index first, as there is room for.
// The move: 16 lanes per row of a kept token, keys and values.
#include "paged.h"

namespace vecinfer {

namespace {

constexpr int kSelect = 1024;

// Order of weights as unsigned numbers: -inf < .. < -0 = 0 < .. < inf; what is no number comes below all.
__device__ __forceinline__ unsigned weight_key(float w)
{
    if (w != w) return 1u;
    const unsigned u = __float_as_uint(w + 0.f);          // (-0 + 0 = 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct Row {
    const float *w;
    const int32_t *pages;
    unsigned num_pages;
    int shift, len, first, recent_from;
    __device__ __forceinline__ unsigned key(int t) const
    {
        if ((unsigned)pages[t >> shift] >= num_pages) return 0u;
        if (t < first || t >= recent_from) return 0xffffffffu;
        return weight_key(w[t]);
    }
};

__global__ __launch_bounds__(kSelect) void evict_select_kernel(const EvictParams p)
{
    __shared__ unsigned hist[256], sums[kSelect / 64], pick[2];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
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

    // digit by digit: the tokens that agree with the digits so far, and how many of them stay
    unsigned prefix = 0, mask = 0;
    unsigned room = (unsigned)p.keep;
    bool all = false;
    for (int digit = 3; digit >= 0; --digit) {
        const int at = 8 * digit;
        if (t < 256) hist[t] = 0;
        if (t == 0) pick[0] = 256;                        // (as it stays where there are no more tokens than room)
        __syncthreads();
        for (int i = t; i < row.len; i += kSelect) {
            const unsigned k = row.key(i);
            if (k != 0u && (k & mask) == prefix) atomicAdd(&hist[k >> at & 255u], 1u);
        }
        __syncthreads();
        if (wave == 0) {                                  // from the top: the digit at which the room ends
            unsigned h[4], own = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) own += h[i] = hist[255 - (4 * lane + i)];
            unsigned before = own;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const unsigned x = __shfl_up(before, o);
                if (lane >= o) before += x;
            }
            const unsigned total = __shfl(before, 63);
            before -= own;
            if (total > room) {                           // (after the first digit always)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (before <= room && room < before + h[i]) {
                        pick[0] = 255 - (4 * lane + i);
                        pick[1] = before;
                    }
                    before += h[i];
                }
            }
        }
        __syncthreads();
        const unsigned d = pick[0];
        if (d == 256) {                                   // every token stays
            all = true;
            break;
        }
        room -= pick[1];
        prefix |= d << at;
        mask |= 255u << at;
        __syncthreads();
    }
    // stays: key & mask above prefix, or equal to it and (all, or among the first `room`)
    unsigned taken = 0, equal = 0;                        // so far, before this stretch
    for (int i0 = 0; i0 < row.len; i0 += kSelect) {
        const int i = i0 + t;
        const unsigned k = i < row.len ? row.key(i) : 0u;
        const bool eq = k != 0u && (k & mask) == prefix, above = k != 0u && (k & mask) > prefix;
        const unsigned long long beq = __ballot(eq), lower = lane ? ~0ull >> (64 - lane) : 0ull;
        if (lane == 0) sums[wave] = __popcll(beq);
        __syncthreads();
        unsigned eq_before = equal, eq_total = 0;
        for (int w = 0; w < kSelect / 64; ++w) {
            if (w < wave) eq_before += sums[w];
            eq_total += sums[w];
        }
        equal += eq_total;
        const bool stays = above || (eq && (all || eq_before + __popcll(beq & lower) < room));
        const unsigned long long bst = __ballot(stays);
        __syncthreads();
        if (lane == 0) sums[wave] = __popcll(bst);
        __syncthreads();
        unsigned before = taken, total = 0;
        for (int w = 0; w < kSelect / 64; ++w) {
            if (w < wave) before += sums[w];
            total += sums[w];
        }
        if (stays) ids[before + __popcll(bst & lower)] = i;
        taken += total;
        __syncthreads();
    }
    if (t == 0 && g == 0) p.dst_lens[b] = (int)taken;
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
