// Shared definitions of the operators around the full-precision paged cache: rotary positions, append, attention,
// eviction.
#pragma once
#include "common.h"

#include <type_traits>

namespace vecinfer {

typedef _Float16 f16;
typedef __bf16 bf16;

// A paged cache.  Row (page, KV head h, slot) of the keys is the D elements at
//   k + page * k_page + h * k_head + slot * k_slot      (bytes; every step below 2^31, a multiple of 16)
// and the page of token t of sequence b is block_table[b, t / page_size].  A page number outside
// 0 .. num_pages - 1 is a hole: its tokens are not attended to, kept or written.
struct PageSet {
    char *k, *v;
    unsigned k_page, k_head, k_slot, v_page, v_head, v_slot;
    unsigned num_pages;
    int shift;                   // log2 of the page size
};

struct RowSet {                  // rows [B, H, T, D] in memory, steps in bytes
    const char *in;
    char *out;
    long long in_b, in_h, in_t, out_b, out_h, out_t;
    int heads;
};

struct RotaryParams {
    RowSet x;                    // the tensor to turn (append: the queries; heads = 0: none)
    RowSet k, v;                 // append only: new keys and values (out_* unused)
    PageSet pages;
    const int32_t *block_table;  // [B, max_pages]
    long long max_pages;
    const int32_t *seq_lens;     // [B] lengths with the new tokens
    const int32_t *new_lens;     // [B] or nullptr: T
    const uint64_t *table;       // [R / 2] turns per position, in units of 2^-64
    const int32_t *positions;    // [B, T] or nullptr
    long long pos0;              // position of token 0 (not append)
    float *weights;              // [B, Hkv, w_cap] or nullptr: cleared for the new tokens
    long long w_cap;
    int B, T, R, interleaved;
    float sign, magnitude;
};

// Arrival words lie 256 bytes apart: the atomics of all workgroups on neighbouring words would queue for one cache line
// (1000 tokens, 8 KV heads in 32 splits: 14.6 us so, 9.7 apart).
constexpr int kWordStep = 32;

struct PagedParams {
    PageSet pages;
    const char *q;               // rows (b, h) at q + b * q_b + h * q_h bytes
    long long q_b, q_h;
    const int32_t *block_table;  // [B, max_pages]
    long long max_pages;
    const int32_t *seq_lens;     // [B] or nullptr: N
    int B, Hq, Hkv, G, N;
    int S;                       // splits of every sequence; or with `least` workgroups per KV head
    int least;                   // 0, or: splits in proportion to the lengths, of at least this many tiles; 2 <= B <= 64, B < S
    float scale2;                // softmax scale * log2(e)
    float *part_o;               // [B, Hkv, S, G, D]  partials, as in DecodeParams; with `least` [Hkv, S, G, D]
    float *part_m, *part_l;      // [B, Hkv, S, G]     or [Hkv, S, G]
    unsigned long long *words;   // [B, Hkv, kWordStep]: an arrival word (split_merge.h) each, and nothing else in its cache lines
    unsigned long long nonce;
    void *out;                   // [B, Hq, D]
    float *lse;                  // [B, Hq] or nullptr
    // sums of attention weight; scores == nullptr: none
    float *scores;               // [B, Hq, n_pad] scores in log2 units
    float2 *norm;                // [B, Hq]: weight = exp2(score - x) y, x the largest score, y 1 over the sum of these
    long long n_pad;
    const float *w_in;           // [B, Hkv, w_cap] or nullptr: 0
    float *w_out;                // [B, Hkv, w_cap]
    long long w_cap;
};

struct EvictParams {
    PageSet src, dst;
    const float *w;              // [B, Hkv, w_cap]
    long long w_cap;
    const int32_t *block_table, *dst_table;
    long long max_pages, dst_max_pages;
    const int32_t *seq_lens;     // [B] or nullptr: N
    int B, Hkv, D, N, keep, first, recent;
    int32_t *dst_lens;           // [B]
    float *dst_w;                // [B, Hkv, dst_w_cap] or nullptr
    long long dst_w_cap;
    int32_t *kept;               // [B, Hkv, keep] or nullptr
    int32_t *ids;                // [B, Hkv, min(keep, N)] in the workspace: the kept tokens, for the move
    unsigned *hists, *states;    // evict_hist_elems() and evict_state_elems() of the workspace (evict.hip)
};

__device__ __forceinline__ int clamped_lane(int v, int N) { return v < 0 ? 0 : (v > N ? N : v); }

__device__ __forceinline__ int clamped_len(const int32_t *lens, int b, int N)
{
    if (!lens) return N;
    // b is the same for the whole workgroup: a scalar load, which does not queue behind vector loads
    typedef const int32_t __attribute__((address_space(4))) *const_i32_ptr;
    const int v = ((const_i32_ptr)(uintptr_t)lens)[b];
    return clamped_lane(v, N);
}

// Sum over the lanes of the wavefront up to this one, on the vector ALU (DPP): within the rows of 16 lanes, then each
// row's last lane into the rows behind it.
__device__ __forceinline__ unsigned wave_upto(unsigned v)
{
    auto from = [&](auto ctrl, auto rows) {
        return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    };
    using std::integral_constant;
    v += from(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});      // row_shr:1
    v += from(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});      // row_shr:2
    v += from(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});      // row_shr:4
    v += from(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});      // row_shr:8
    v += from(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});      // row_bcast:15 into rows 1 and 3
    v += from(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});      // row_bcast:31 into rows 2 and 3
    return v;
}

// log2 of the sum, and the sum itself, go to natural units in one place
__device__ __forceinline__ float natural(float log2_units) { return log2_units * kLn2; }

// 16 bytes of a row.  STREAM: what goes through once need not displace anything from the caches; taken by calls that move
// 64 MB and more.  A smaller one reads what the kernel before it has left in the Infinity Cache, and writes for the next, and
// the three together are faster with the caches, where the call by itself, out of memory, is faster without (us, cached /
// streaming; left out of memory, right between a copy that writes its input and one that reads its output, in sum):
//              8 MB                      32 MB                     64 MB                     128 MB                    256 MB
//   rotary     4.4 / 4.0    9.8 / 9.9    9.1 / 9.3   21.7 / 22.9   15.4 / 14.9  39.4 / 38.9  26.9 / 24.4  71.9 / 70.9  50.3 / 46.0  160 / 135
//   append     6.1 / 5.9   11.5 / 11.2  11.4 / 10.0  21.5 / 22.6   17.4 / 15.8  34.1 / 36.1  29.8 / 27.4  60.3 / 61.9
//   eviction  12.0 / 10.8  18.8 / 19.1  20.4 / 18.4  35.4 / 37.3   31.5 / 28.4  57.6 / 60.7  54.1 / 48.7  99.8 / 106   80.7 / 75.5  191 / 178
// 64 MB is where the sum of both columns turns for the rotary kernel; by the right one alone it would be 128 to 192 MB, by the
// left one alone nothing.
constexpr long long kStreamBytes = 64ll << 20;

typedef unsigned words4 __attribute__((ext_vector_type(4)));

template <bool STREAM>
__device__ __forceinline__ uint4 load16(const char *row, int piece)
{
    const words4 *const p = reinterpret_cast<const words4 *>(row) + piece;
    return __builtin_bit_cast(uint4, STREAM ? __builtin_nontemporal_load(p) : *p);
}

template <bool STREAM>
__device__ __forceinline__ void store16(char *row, int piece, uint4 v)
{
    words4 *const p = reinterpret_cast<words4 *>(row) + piece;
    if constexpr (STREAM)
        __builtin_nontemporal_store(__builtin_bit_cast(words4, v), p);
    else
        *p = __builtin_bit_cast(words4, v);
}

int launch_rotary_table(const double *freqs, double base, int scaling, double factor, double low, double high,
                        double orig_len, int R, uint64_t *table, hipStream_t stream);
int launch_rotary(const RotaryParams &p, int bf16, int D, bool append, hipStream_t stream);
int launch_paged_attention(const PagedParams &p, int bf16, int D, hipStream_t stream);
int launch_paged_weights(const PagedParams &p, hipStream_t stream);
size_t evict_hist_elems(long long rows, long long N);
size_t evict_state_elems(long long rows, long long N);
int launch_evict(const EvictParams &p, hipStream_t stream);

} // namespace vecinfer
