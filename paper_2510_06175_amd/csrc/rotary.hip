// Rotary positions, alone and on the way into the paged cache.
//
// A pair (x1, x2) of channels at position p becomes m (x1 c - x2 s, x1 s + x2 c), c and s the cosine and sine of p f_i.
// The angle is held in turns as a 64-bit fixed-point fraction F_i = f_i / 2 pi, cut from an fp64 number: p F_i modulo 2^64 is
// the fraction of a turn exactly for the table's word, so that all that grows with the position is that number's own error,
// within 2^-50 of F_i per position (fp32 angles are off by a twentieth of a radian at 10^6).  Its upper 32 bits go through
// sincospi as an fp32 number, which is within 2^-26 turns, and moves sine and cosine by 2^-23 at most, next to the
// rows' own rounding of 2^-11 or 2^-8.  The pairs of a token are the same in all heads: a workgroup works the cosines and
// sines of its tokens out once, into LDS, a thread each.
//
// A thread owns 16 channels of a row, 8 pairs: two 16-byte pieces, in the half layout those that belong together, R / 2
// channels apart, else half of the row (or of what is only copied) apart, so that neighbouring threads' pieces are
// neighbours.
#include "paged.h"

namespace vecinfer {

namespace {

constexpr int kBlock = 256;
constexpr int kMostTokens = 4;                            // of a workgroup
constexpr unsigned kGridX = 1u << 22;                     // most workgroups of a grid's first axis: 2^32 threads and more are not launched

__global__ void rotary_table_kernel(const double *freqs, double base, int scaling, double factor, double low, double high,
                                    double orig_len, int R, uint64_t *table)
{
    const int i = threadIdx.x;
    if (i >= R / 2) return;
    constexpr double kTwoPi = 6.283185307179586476925286766559;
    double f;
    if (freqs) {
        f = freqs[i];
    } else {
        if (scaling == 2) base *= pow(factor, R / (R - 2.0));
        f = pow(base, -2.0 * i / R);
        if (scaling == 1) f /= factor;
        if (scaling == 3) {                               // by the turns of the pair within the original context
            double g = (orig_len * f / kTwoPi - low) / (high - low);
            g = g < 0 ? 0 : (g > 1 ? 1 : g);
            f = (1 - g) * f / factor + g * f;
        }
    }
    double turns = f / kTwoPi;
    turns -= floor(turns);                                // positions are whole: whole turns per position do nothing
    // (turns = 1 - 2^-54 and the like round to 2^64, which is 0; NaN and infinities, which have no fraction, give 0 too)
    const double scaled = turns * 18446744073709551616.0;
    table[i] = scaled >= 0 && scaled < 18446744073709551616.0 ? (uint64_t)scaled : 0;
}

// The pairs within a piece (cs: four of them), and those across two (cs: eight).
template <typename E>
__device__ __forceinline__ void turn_within(uint4 &piece, const float2 *cs)
{
    typedef E vec8 __attribute__((ext_vector_type(8)));
    vec8 v = __builtin_bit_cast(vec8, piece);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float x = (float)v[2 * e], y = (float)v[2 * e + 1];
        v[2 * e] = (E)fmaf(x, cs[e].x, -(y * cs[e].y));
        v[2 * e + 1] = (E)fmaf(x, cs[e].y, y * cs[e].x);
    }
    piece = __builtin_bit_cast(uint4, v);
}

template <typename E>
__device__ __forceinline__ void turn_across(uint4 &one, uint4 &two, const float2 *cs)
{
    typedef E vec8 __attribute__((ext_vector_type(8)));
    const vec8 a = __builtin_bit_cast(vec8, one), b = __builtin_bit_cast(vec8, two);
    vec8 u, v;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = (float)a[e], y = (float)b[e];
        u[e] = (E)fmaf(x, cs[e].x, -(y * cs[e].y));
        v[e] = (E)fmaf(x, cs[e].y, y * cs[e].x);
    }
    one = __builtin_bit_cast(uint4, u);
    two = __builtin_bit_cast(uint4, v);
}

// grid (tokens / TPW, head groups, kGridX of the former each); TPW tokens per workgroup, 1 << tpw_shift
template <typename E, int D, bool APPEND, bool STREAM>
__global__ __launch_bounds__(kBlock) void rotary_kernel(const RotaryParams p, int tpw_shift)
{
    constexpr int kUnits = D / 16;                        // threads per row
    constexpr int kRows = kBlock / kUnits;                // rows at a time
    __shared__ float2 cs_s[kMostTokens * (D / 2)];
    const int t = threadIdx.x, u = t % kUnits, row = t / kUnits;
    const int tpw = 1 << tpw_shift, half = p.R / 2;
    const unsigned tok0 = (blockIdx.z * kGridX + blockIdx.x) << tpw_shift, n_tok = (unsigned)p.B * (unsigned)p.T;

    for (int i = t; i < tpw * half; i += kBlock) {
        const int k = i / half, j = i - k * half;
        const unsigned tok = tok0 + k;
        if (tok >= n_tok) break;
        long long pos;
        if (p.positions) {
            pos = p.positions[tok];
        } else {
            const unsigned b = tok / (unsigned)p.T, at = tok - b * (unsigned)p.T;
            pos = p.pos0 + at;
            if constexpr (APPEND) {
                int n = p.new_lens ? p.new_lens[b] : p.T;
                n = n < 0 ? 0 : (n > p.T ? p.T : n);
                pos = (long long)p.seq_lens[b] - n + at;
            }
        }
        const int turns = (int)(((uint64_t)pos * p.table[j]) >> 32);       // fraction of a turn, -2^31 .. 2^31 - 1
        float s, c;
        sincospif((float)turns * 4.656612873077393e-10f, &s, &c);          // 2^-31: half turns
        cs_s[k * half + j] = make_float2(c * p.magnitude, s * p.magnitude * p.sign);
    }
    __syncthreads();

    const int k = row & (tpw - 1);
    const unsigned tok = tok0 + k;
    if (tok >= n_tok) return;
    const unsigned b = tok / (unsigned)p.T, at = tok - b * (unsigned)p.T;
    int c0, c1;                                           // the two pieces
    bool turn0, turn1;
    float2 cs[8];
    if (p.interleaved) {
        c0 = u;
        c1 = u + kUnits;
        turn0 = 8 * c0 < p.R;
        turn1 = 8 * c1 < p.R;
        if (turn0)
#pragma unroll
            for (int e = 0; e < 4; ++e) cs[e] = cs_s[k * half + 4 * c0 + e];
        if (turn1)
#pragma unroll
            for (int e = 0; e < 4; ++e) cs[4 + e] = cs_s[k * half + 4 * c1 + e];
    } else {
        const int pairs = p.R / 16;                       // of pieces
        turn0 = turn1 = u < pairs;
        c0 = u < pairs ? u : u + pairs;
        c1 = u < pairs ? u + pairs : u + kUnits;
        if (turn0)
#pragma unroll
            for (int e = 0; e < 8; ++e) cs[e] = cs_s[k * half + 8 * u + e];
    }

    char *k_out = nullptr, *v_out = nullptr;
    long long where = -1;
    if constexpr (APPEND) {
        int n = p.new_lens ? p.new_lens[b] : p.T;
        n = n < 0 ? 0 : (n > p.T ? p.T : n);
        if ((int)at >= n) return;
        where = (long long)p.seq_lens[b] - n + at;
        const long long col = where >> p.pages.shift;
        if (where >= 0 && col < p.max_pages) {
            const unsigned page = (unsigned)p.block_table[b * p.max_pages + col];
            const unsigned slot = (unsigned)where & ((1u << p.pages.shift) - 1);
            if (page < p.pages.num_pages) {
                k_out = p.pages.k + (unsigned long long)page * p.pages.k_page + (unsigned long long)slot * p.pages.k_slot;
                v_out = p.pages.v + (unsigned long long)page * p.pages.v_page + (unsigned long long)slot * p.pages.v_slot;
            }
        }
    }
    const int heads = APPEND ? p.x.heads + p.k.heads + p.v.heads : p.x.heads;
    const int step = kRows >> tpw_shift;
    for (int h = (row >> tpw_shift) + step * blockIdx.y; h < heads; h += step * gridDim.y) {
        const char *in;
        char *out;
        bool turn = true;
        if (!APPEND || h < p.x.heads) {
            in = p.x.in + b * p.x.in_b + h * p.x.in_h + at * p.x.in_t;
            out = p.x.out + b * p.x.out_b + h * p.x.out_h + at * p.x.out_t;
        } else if (h < p.x.heads + p.k.heads) {
            const int g = h - p.x.heads;
            if (p.weights && u == 0 && where >= 0 && where < p.w_cap) p.weights[(b * (size_t)p.k.heads + g) * p.w_cap + where] = 0.f;
            if (!k_out) continue;
            in = p.k.in + b * p.k.in_b + g * p.k.in_h + at * p.k.in_t;
            out = k_out + (unsigned long long)g * p.pages.k_head;
        } else {
            if (!v_out) continue;
            const int g = h - p.x.heads - p.k.heads;
            in = p.v.in + b * p.v.in_b + g * p.v.in_h + at * p.v.in_t;
            out = v_out + (unsigned long long)g * p.pages.v_head;
            turn = false;
        }
        uint4 one = load16<STREAM>(in, c0), two = load16<STREAM>(in, c1);
        if (turn) {
            if (p.interleaved) {
                if (turn0) turn_within<E>(one, cs);
                if (turn1) turn_within<E>(two, cs + 4);
            } else if (turn0) {
                turn_across<E>(one, two, cs);
            }
        }
        store16<STREAM>(out, c0, one);
        store16<STREAM>(out, c1, two);
    }
}

// Tokens per workgroup: 1, 2 or 4, as few as leave the fewest threads idle - its rows are then dealt to the heads of a token
// (8192 tokens, 32 heads: 24.4 us with one token, 25.5 with four; 48 heads of an append: 30.0 with two, 30.8 with four, 38
// with one; 8 heads 11.2 with four, 14.0 with one).  Where there are fewer tokens than would fill the chip, one, and a
// token's heads are dealt to several workgroups.
// Streaming: load16.
template <typename E, int D, bool APPEND>
void start(const RotaryParams &p, hipStream_t stream)
{
    constexpr int kRows = kBlock / (D / 16);
    const long long n_tok = (long long)p.B * p.T;
    const int heads = p.x.heads + (APPEND ? p.k.heads + p.v.heads : 0);
    auto rows_taken = [&](int shift) {                    // by one token's heads, idle ones included
        const int step = kRows >> shift;
        return (heads + step - 1) / step * step;
    };
    int shift = 0;
    unsigned gy = 1;
    if (n_tok >= 4 * (long long)num_cus()) {
        for (int i = 1; 1 << i <= kMostTokens; ++i)
            if (rows_taken(i) < rows_taken(shift)) shift = i;
    } else {
        const int passes = rows_taken(0) / kRows;
        gy = (unsigned)(passes < 65535 ? passes : 65535);
    }
    const unsigned groups = (unsigned)((n_tok + (1 << shift) - 1) >> shift);
    const dim3 grid(groups < kGridX ? groups : kGridX, gy, (groups + kGridX - 1) / kGridX);
    if (4 * n_tok * heads * D >= kStreamBytes)
        hipLaunchKernelGGL((rotary_kernel<E, D, APPEND, true>), grid, dim3(kBlock), 0, stream, p, shift);
    else
        hipLaunchKernelGGL((rotary_kernel<E, D, APPEND, false>), grid, dim3(kBlock), 0, stream, p, shift);
}

} // namespace

int launch_rotary_table(const double *freqs, double base, int scaling, double factor, double low, double high,
                        double orig_len, int R, uint64_t *table, hipStream_t stream)
{
    hipLaunchKernelGGL(rotary_table_kernel, dim3(1), dim3(64), 0, stream, freqs, base, scaling, factor, low, high, orig_len,
                       R, table);
    return hipGetLastError() == hipSuccess ? 0 : -4;
}

int launch_rotary(const RotaryParams &p, int is_bf16, int D, bool append, hipStream_t stream)
{
    auto by_dim = [&](auto elem) {
        typedef decltype(elem) E;
        if (append)
            D == 128 ? start<E, 128, true>(p, stream) : start<E, 64, true>(p, stream);
        else
            D == 128 ? start<E, 128, false>(p, stream) : start<E, 64, false>(p, stream);
    };
    if (is_bf16)
        by_dim(bf16{});
    else
        by_dim(f16{});
    return hipGetLastError() == hipSuccess ? 0 : -4;
}

} // namespace vecinfer
