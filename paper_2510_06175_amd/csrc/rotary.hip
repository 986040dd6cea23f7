// Rotary positions, alone and on the way into the paged cache.
//
// A pair (x1, x2) of channels at position p becomes m (x1 c - x2 s, x1 s + x2 c), c and s the cosine and sine of p f_i.
// The angle is held in turns as a 64-bit fixed-point fraction F_i = f_i / 2 pi: p F_i modulo 2^64 is the fraction of a
// turn exactly as the table has it at every position (fp32 angles are off by a twentieth of a radian at 10^6), and its
// upper 32 bits go through sincospi.  The pairs of a token are the same in all heads: a workgroup works the cosines and
// sines of its tokens out once, into LDS, a thread each.
//
// A thread owns 16 channels of a row, 8 pairs: two 16-byte pieces (half layout: R / 2 channels apart; adjacent pairs:
// side by side).
#include "paged.h"

namespace vecinfer {

namespace {

constexpr int kBlock = 256;

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

template <typename E>
__device__ __forceinline__ void turn8(uint4 &pa, uint4 &pb, const float2 (&cs)[8], bool interleaved)
{
    typedef E vec8 __attribute__((ext_vector_type(8)));
    const vec8 a = __builtin_bit_cast(vec8, pa), b = __builtin_bit_cast(vec8, pb);
    vec8 u, v;
    if (interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = (float)a[2 * e], y = (float)a[2 * e + 1];
            u[2 * e] = (E)fmaf(x, cs[e].x, -(y * cs[e].y));
            u[2 * e + 1] = (E)fmaf(x, cs[e].y, y * cs[e].x);
            x = (float)b[2 * e], y = (float)b[2 * e + 1];
            v[2 * e] = (E)fmaf(x, cs[4 + e].x, -(y * cs[4 + e].y));
            v[2 * e + 1] = (E)fmaf(x, cs[4 + e].y, y * cs[4 + e].x);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = (float)a[e], y = (float)b[e];
            u[e] = (E)fmaf(x, cs[e].x, -(y * cs[e].y));
            v[e] = (E)fmaf(x, cs[e].y, y * cs[e].x);
        }
    }
    pa = __builtin_bit_cast(uint4, u);
    pb = __builtin_bit_cast(uint4, v);
}

// grid (tokens / TPW, head groups); TPW tokens per workgroup, 1 << tpw_shift
template <typename E, int D, bool APPEND>
__global__ __launch_bounds__(kBlock) void rotary_kernel(const RotaryParams p, int tpw_shift)
{
    constexpr int kUnits = D / 16;                        // threads per row
    constexpr int kRows = kBlock / kUnits;                // rows at a time
    __shared__ float2 cs_s[4 * (D / 2)];
    const int t = threadIdx.x, u = t % kUnits, row = t / kUnits;
    const int tpw = 1 << tpw_shift, half = p.R / 2;
    const unsigned tok0 = blockIdx.x << tpw_shift, n_tok = (unsigned)p.B * (unsigned)p.T;

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
    const bool turned = u < p.R / 16;
    int c0, c1;                                           // the two 16-byte pieces
    if (turned && !p.interleaved) {
        c0 = u;
        c1 = u + p.R / 16;
    } else {
        c0 = 2 * u;                                       // (behind the turned channels as well)
        c1 = c0 + 1;
    }
    float2 cs[8];
    if (turned)
#pragma unroll
        for (int e = 0; e < 8; ++e) cs[e] = cs_s[k * half + 8 * u + e];

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
        bool turn = turned;
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
        uint4 a = reinterpret_cast<const uint4 *>(in)[c0], bb = reinterpret_cast<const uint4 *>(in)[c1];
        if (turn) turn8<E>(a, bb, cs, p.interleaved);
        reinterpret_cast<uint4 *>(out)[c0] = a;
        reinterpret_cast<uint4 *>(out)[c1] = bb;
    }
}

template <typename E, int D, bool APPEND>
void start(const RotaryParams &p, hipStream_t stream)
{
    const long long n_tok = (long long)p.B * p.T;
    const int tpw_shift = n_tok >= 4 * (long long)num_cus() ? 2 : 0;
    const int heads = p.x.heads + (APPEND ? p.k.heads + p.v.heads : 0);
    const int step = (kBlock / (D / 16)) >> tpw_shift;
    const int passes = (heads + step - 1) / step;
    const unsigned gx = (unsigned)((n_tok + (1 << tpw_shift) - 1) >> tpw_shift);
    const unsigned gy = tpw_shift ? 1 : (unsigned)(passes < 65535 ? passes : 65535);
    hipLaunchKernelGGL((rotary_kernel<E, D, APPEND>), dim3(gx, gy), dim3(kBlock), 0, stream, p, tpw_shift);
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
