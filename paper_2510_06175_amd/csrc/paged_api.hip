// C entries of the paged cache and of rotary positions: argument validation and dispatch.  See include/vecinfer.h.
#include "../../include/vecinfer.h"

#include "paged.h"

#include <math.h>

using namespace vecinfer;

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int launch_status(int rc) { return rc == 0 ? VECINFER_OK : VECINFER_ELAUNCH; }

size_t up(size_t v) { return (v + 255) / 256 * 256; }

constexpr int64_t kMaxTokens = 1 << 30;

int rotary_ok(const vecinfer_rotary_cfg *c)
{
    if (!c) return VECINFER_EINVAL;
    if (c->head_dim != 64 && c->head_dim != 128) return VECINFER_EUNSUPPORTED;
    if (c->rot_dim < 16 || c->rot_dim > c->head_dim || c->rot_dim % 16) return VECINFER_EUNSUPPORTED;
    if ((c->interleaved != 0 && c->interleaved != 1) || c->scaling < VECINFER_ROTARY_PLAIN || c->scaling > VECINFER_ROTARY_PARTS)
        return VECINFER_EINVAL;
    if (!(c->base > 0) || !isfinite(c->base) || !isfinite((float)c->magnitude)) return VECINFER_EINVAL;
    if (c->scaling != VECINFER_ROTARY_PLAIN && (!(c->factor > 0) || !isfinite(c->factor))) return VECINFER_EINVAL;
    if (c->scaling == VECINFER_ROTARY_PARTS &&
        (!(c->low_turns < c->high_turns) || !isfinite(c->low_turns) || !isfinite(c->high_turns) || c->orig_len < 1))
        return VECINFER_EINVAL;
    return VECINFER_OK;
}

// Steps of a tensor: not negative, whole 16-byte pieces.
bool strides_ok(const int64_t *s, int n, int64_t below)
{
    for (int i = 0; i < n; ++i)
        if (s[i] < 0 || s[i] % 8 || s[i] >= below) return false;
    return true;
}

constexpr int64_t kStride = (int64_t)1 << 40;

int pages_ok(const vecinfer_pages *p)
{
    if (!p || !p->k || !p->v || !aligned(p->k, 16) || !aligned(p->v, 16)) return VECINFER_EINVAL;
    if (p->dtype != VECINFER_F16 && p->dtype != VECINFER_BF16) return VECINFER_EINVAL;
    if (p->num_kv_heads < 1 || p->page_size < 1 || p->num_pages < 1) return VECINFER_EINVAL;
    if (!strides_ok(p->k_strides, 3, (int64_t)1 << 30) || !strides_ok(p->v_strides, 3, (int64_t)1 << 30)) return VECINFER_EINVAL;
    if (p->head_dim != 64 && p->head_dim != 128) return VECINFER_EUNSUPPORTED;
    if (p->page_size < 8 || p->page_size > 1024 || (p->page_size & (p->page_size - 1))) return VECINFER_EUNSUPPORTED;
    if (p->num_pages > 0x7fffffffLL || p->num_kv_heads > 65535) return VECINFER_EUNSUPPORTED;
    return VECINFER_OK;
}

PageSet page_set(const vecinfer_pages *p)
{
    PageSet s;
    s.k = static_cast<char *>(p->k);
    s.v = static_cast<char *>(p->v);
    s.k_page = (unsigned)(2 * p->k_strides[0]);
    s.k_head = (unsigned)(2 * p->k_strides[1]);
    s.k_slot = (unsigned)(2 * p->k_strides[2]);
    s.v_page = (unsigned)(2 * p->v_strides[0]);
    s.v_head = (unsigned)(2 * p->v_strides[1]);
    s.v_slot = (unsigned)(2 * p->v_strides[2]);
    s.num_pages = (unsigned)p->num_pages;
    s.shift = __builtin_ctz((unsigned)p->page_size);
    return s;
}

void rows_in(RowSet &r, const void *x, const int64_t *s, int heads)
{
    r.in = static_cast<const char *>(x);
    r.in_b = x ? 2 * s[0] : 0;
    r.in_h = x ? 2 * s[1] : 0;
    r.in_t = x ? 2 * s[2] : 0;
    r.out = nullptr;
    r.out_b = r.out_h = r.out_t = 0;
    r.heads = x ? heads : 0;
}

void rows_out(RowSet &r, void *x, const int64_t *s)
{
    if (!x) return;
    r.out = static_cast<char *>(x);
    r.out_b = 2 * s[0];
    r.out_h = 2 * s[1];
    r.out_t = 2 * s[2];
}

struct PagedLayout {
    size_t off_o, off_m, off_l, off_words, off_norm, off_scores, total;
};

// parts: partials of a (split, KV head) each
PagedLayout paged_layout(const vecinfer_pages *p, int32_t Hq, int32_t B, int64_t N, int64_t parts, bool weights)
{
    const size_t rows = (size_t)parts * (Hq / p->num_kv_heads);
    PagedLayout w;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off += up(bytes);
        return at;
    };
    w.off_o = take(sizeof(float) * rows * p->head_dim);
    w.off_m = take(sizeof(float) * rows);
    w.off_l = take(sizeof(float) * rows);
    w.off_words = take(sizeof(unsigned long long) * kWordStep * (size_t)B * p->num_kv_heads);
    w.off_norm = take(weights ? sizeof(float2) * (size_t)B * Hq : 0);
    w.off_scores = take(weights ? sizeof(float) * (size_t)B * Hq * ((N + 31) / 32 * 32) : 0);
    w.total = off;
    return w;
}

struct EvictLayout {
    size_t off_hists, off_states, total;                  // the list of kept tokens comes first
};

EvictLayout evict_layout(int64_t rows, int64_t N, int64_t keep)
{
    EvictLayout w;
    w.off_hists = up(sizeof(int32_t) * (size_t)rows * (keep < N ? keep : N));
    w.off_states = w.off_hists + up(sizeof(unsigned) * evict_hist_elems(rows, N));
    w.total = w.off_states + up(sizeof(unsigned) * evict_state_elems(rows, N));
    return w;
}

// How the tokens of a batch are dealt to workgroups: `splits` of every sequence; or, with `least`, `splits` workgroups
// per KV head, dealt by the sequences' lengths (PagedParams).
struct Cut {
    int32_t splits, least;
    int64_t parts(const vecinfer_pages *p, int32_t B) const
    {
        return least ? (int64_t)p->num_kv_heads * splits : (splits > 1 ? (int64_t)B * p->num_kv_heads * splits : 0);
    }
};

constexpr int32_t kDealt = 64;           // most sequences of a batch that is dealt by length: a lane each

// A compute unit holds one workgroup (8 wavefronts of 170 registers), and two rounds of them are slower than one where all
// are alike: a workgroup's start and end take 7 us (one sequence of 196608 tokens, 8 KV heads: 123 us in 32 splits, 136 in
// 48, 128 in 64).  So as many as fill the chip once, and
//   - no shorter than 64 tokens, two tiles, or 128 with more than eight query heads per KV head, whose merge is longer (one
//     sequence, 4 / 1 heads, 500 tokens: 6.7 us in 4, 6.4 in 8, 6.2 in 16; 1000: 6.7 in 8, 6.6 in 16 and in 32; 8 / 1, 1000:
//     7.1 in 8 and in 16, 7.8 in 32; 16 / 1, 2000: 9.9 in 16, 10.9 in 32);
//   - whole up to 256 tokens, one round of a workgroup's wavefronts (200 tokens 5.7 us whole, 6.4 to 6.7 in splits);
//   - more where one round would leave an eighth of the chip idle and splits are long (4000 tokens).
// Sequences that come with lengths of their own, 4000 tokens and up, are dealt by length to one round of workgroups, or,
// where there are more than a quarter as many as compute units per KV head, to so many rounds that each has one and there is
// one round more (N / 8 to N tokens, in the same splits / dealt: 8 KV heads, 4 x 30000 62.0 / 53.5 us, 8 x 8000 35.1 /
// 31.5, 16 x 8000 60.7 / 54.8, 64 x 6000 160 / 157; 4 KV heads, 9 x 30000 67.5 / 55.0; 32 x 8192 102 to 113, depending on which
// come first, / 102, and 32 of 8192 each 161 whole, 167 dealt.  Shorter ones not: 32 x 2000 31.7 / 35, 4 x 1000 7.8 / 8.3).
Cut even_cut(const vecinfer_pages *p, int32_t B, int64_t N, int64_t worth)
{
    const int64_t groups = (int64_t)B * p->num_kv_heads;
    int64_t s = num_cus() / groups;
    if (s < 1) s = 1;
    if (N >= 4000 * s && groups <= num_cus() && 8 * s * groups < 7 * num_cus()) s = 2 * s > 4 ? 2 * s : 4;
    if (s > worth) s = worth;
    if (s > VECINFER_MAX_SPLITS) s = VECINFER_MAX_SPLITS;
    return {s < 1 || N <= 256 ? 1 : (int32_t)s, 0};
}

Cut auto_cut(const vecinfer_pages *p, int32_t Hq, int32_t B, int64_t N, bool lengths)
{
    const int64_t G = Hq / p->num_kv_heads;
    const int64_t worth = (N + (G > 8 ? 127 : 63)) / (G > 8 ? 128 : 64);
    if (!lengths || B < 2 || B > kDealt || N < 4000) return even_cut(p, B, N, worth);
    int64_t per_head = num_cus() / p->num_kv_heads;
    if (per_head < 1) per_head = 1;
    int64_t slots = per_head >= 4 * B ? per_head : (B + 2 * per_head - 1) / per_head * per_head;
    if (slots > VECINFER_MAX_SPLITS) slots = VECINFER_MAX_SPLITS;
    return {(int32_t)slots, (int32_t)((N + 32 * worth - 1) / (32 * worth))};
}

} // namespace

extern "C" {

int vecinfer_rotary_table(const vecinfer_rotary_cfg *cfg, const double *freqs, uint64_t *table, void *stream)
{
    if (!cfg || !table || !aligned(table, 8) || !aligned(freqs, 8)) return VECINFER_EINVAL;
    const int rc = rotary_ok(cfg);
    if (rc != VECINFER_OK) return rc;
    return launch_status(launch_rotary_table(freqs, cfg->base, cfg->scaling, cfg->factor, cfg->low_turns, cfg->high_turns,
                                             (double)cfg->orig_len, cfg->rot_dim, table, static_cast<hipStream_t>(stream)));
}

int vecinfer_rotary(const vecinfer_rotary_cfg *cfg, const uint64_t *table, int32_t dtype, const void *x,
                    const int64_t x_strides[3], void *out, const int64_t out_strides[3], int32_t B, int32_t H, int64_t T,
                    const int32_t *positions, int64_t pos0, int32_t inverse, void *stream)
{
    if (!cfg || !table || !x || !out || !x_strides || !out_strides) return VECINFER_EINVAL;
    const int rc = rotary_ok(cfg);
    if (rc != VECINFER_OK) return rc;
    if (dtype != VECINFER_F16 && dtype != VECINFER_BF16) return VECINFER_EINVAL;
    if (B < 1 || H < 1 || T < 1) return VECINFER_EINVAL;
    if (!aligned(x, 16) || !aligned(out, 16) || !aligned(table, 8) || !aligned(positions, 4)) return VECINFER_EINVAL;
    if (!strides_ok(x_strides, 3, kStride) || !strides_ok(out_strides, 3, kStride)) return VECINFER_EINVAL;
    if (T > 0x7fffffffLL / B || H > 65535) return VECINFER_EUNSUPPORTED;
    RotaryParams p = {};
    rows_in(p.x, x, x_strides, H);
    rows_out(p.x, out, out_strides);
    p.table = table;
    p.positions = positions;
    p.pos0 = pos0;
    p.B = B;
    p.T = (int)T;
    p.R = cfg->rot_dim;
    p.interleaved = cfg->interleaved;
    p.sign = inverse ? -1.f : 1.f;
    p.magnitude = (float)cfg->magnitude;
    return launch_status(launch_rotary(p, dtype == VECINFER_BF16, cfg->head_dim, false, static_cast<hipStream_t>(stream)));
}

int vecinfer_paged_append(const vecinfer_pages *pages, const vecinfer_rotary_cfg *rot, const uint64_t *table,
                          const void *k_new, const int64_t k_strides[3], const void *v_new, const int64_t v_strides[3],
                          const void *q, const int64_t q_strides[3], void *q_out, const int64_t q_out_strides[3],
                          int32_t num_q_heads, const int32_t *block_table, int64_t max_pages, const int32_t *seq_lens,
                          const int32_t *new_lens, const int32_t *positions, int32_t B, int64_t T, float *weights,
                          int64_t w_cap, void *stream)
{
    if (!k_new || !v_new || !k_strides || !v_strides || !block_table || !seq_lens) return VECINFER_EINVAL;
    int rc = pages_ok(pages);
    if (rc != VECINFER_OK) return rc;
    if ((rot != nullptr) != (table != nullptr) || (q != nullptr) != (q_out != nullptr) || (q && !rot)) return VECINFER_EINVAL;
    if (rot) {
        rc = rotary_ok(rot);
        if (rc != VECINFER_OK) return rc;
        if (rot->head_dim != pages->head_dim) return VECINFER_EINVAL;
    }
    if (q && (!q_strides || !q_out_strides || num_q_heads < 1)) return VECINFER_EINVAL;
    if (B < 1 || T < 1 || max_pages < 1 || (weights && w_cap < 1)) return VECINFER_EINVAL;
    if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(q, 16) || !aligned(q_out, 16) || !aligned(table, 8)) return VECINFER_EINVAL;
    if (!aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(new_lens, 4) || !aligned(positions, 4) || !aligned(weights, 4))
        return VECINFER_EINVAL;
    if (!strides_ok(k_strides, 3, kStride) || !strides_ok(v_strides, 3, kStride)) return VECINFER_EINVAL;
    if (q && (!strides_ok(q_strides, 3, kStride) || !strides_ok(q_out_strides, 3, kStride))) return VECINFER_EINVAL;
    if (T > 0x7fffffffLL / B || num_q_heads > 65535) return VECINFER_EUNSUPPORTED;
    RotaryParams p = {};
    rows_in(p.x, q, q_strides, num_q_heads);
    rows_out(p.x, q_out, q_out_strides);
    rows_in(p.k, k_new, k_strides, pages->num_kv_heads);
    rows_in(p.v, v_new, v_strides, pages->num_kv_heads);
    p.pages = page_set(pages);
    p.block_table = block_table;
    p.max_pages = max_pages;
    p.seq_lens = seq_lens;
    p.new_lens = new_lens;
    p.table = table;
    p.positions = positions;
    p.weights = weights;
    p.w_cap = w_cap;
    p.B = B;
    p.T = (int)T;
    p.R = rot ? rot->rot_dim : 0;
    p.interleaved = rot ? rot->interleaved : 0;
    p.sign = 1.f;
    p.magnitude = rot ? (float)rot->magnitude : 1.f;
    return launch_status(launch_rotary(p, pages->dtype == VECINFER_BF16, pages->head_dim, true, static_cast<hipStream_t>(stream)));
}

size_t vecinfer_paged_workspace_bytes(const vecinfer_pages *pages, int32_t num_q_heads, int32_t B, int64_t N,
                                      int32_t num_splits, int32_t weights)
{
    if (pages_ok(pages) != VECINFER_OK || num_q_heads < 1 || num_q_heads % pages->num_kv_heads) return 0;
    if (B < 1 || N < 1 || N > kMaxTokens || num_splits < 0 || num_splits > VECINFER_MAX_SPLITS) return 0;
    const Cut fixed{num_splits, 0}, even = auto_cut(pages, num_q_heads, B, N, false), dealt = auto_cut(pages, num_q_heads, B, N, true);
    const int64_t a = even.parts(pages, B), b = dealt.parts(pages, B);
    return paged_layout(pages, num_q_heads, B, N, num_splits ? fixed.parts(pages, B) : (a > b ? a : b), weights != 0).total;
}

int vecinfer_paged_attention(const vecinfer_pages *pages, const void *q, const int64_t q_strides[2], int32_t num_q_heads,
                             const int32_t *block_table, int64_t max_pages, const int32_t *seq_lens, int32_t B, int64_t N,
                             float scale, int32_t num_splits, void *workspace, size_t workspace_bytes, void *out, float *lse,
                             const float *weights_in, float *weights_out, int64_t w_cap, void *stream)
{
    if (!q || !q_strides || !block_table || !out) return VECINFER_EINVAL;
    const int rc = pages_ok(pages);
    if (rc != VECINFER_OK) return rc;
    if (B < 1 || N < 1 || max_pages < 1 || num_q_heads < 1 || num_q_heads % pages->num_kv_heads) return VECINFER_EINVAL;
    if ((N + pages->page_size - 1) / pages->page_size > max_pages) return VECINFER_EINVAL;
    if (num_splits < 0 || num_splits > VECINFER_MAX_SPLITS || !isfinite(scale * kLog2e)) return VECINFER_EINVAL;
    if (!aligned(q, 16) || !aligned(out, 16) || !strides_ok(q_strides, 2, kStride)) return VECINFER_EINVAL;
    if (!aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(lse, 4) || !aligned(weights_in, 4) || !aligned(weights_out, 4))
        return VECINFER_EINVAL;
    if ((weights_in && !weights_out) || (weights_out && w_cap < N)) return VECINFER_EINVAL;
    const int G = num_q_heads / pages->num_kv_heads;
    if (G > 16 || B > 65535 || N > kMaxTokens || max_pages > 0x7fffffffLL) return VECINFER_EUNSUPPORTED;

    Cut cut{num_splits, 0};
    if (num_splits == 0) cut = auto_cut(pages, num_q_heads, B, N, seq_lens != nullptr);
    PagedLayout w = paged_layout(pages, num_q_heads, B, N, cut.parts(pages, B), weights_out != nullptr);
    if (num_splits == 0 && workspace_bytes < w.total) {     // fewer where the workspace has no room for that many
        if (cut.least) cut = auto_cut(pages, num_q_heads, B, N, false);
        for (;; --cut.splits) {
            w = paged_layout(pages, num_q_heads, B, N, cut.parts(pages, B), weights_out != nullptr);
            if (cut.splits == 1 || workspace_bytes >= w.total) break;
        }
    }
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < w.total) return VECINFER_EWORKSPACE;
    unsigned char *const ws = static_cast<unsigned char *>(workspace);
    PagedParams p = {};
    p.pages = page_set(pages);
    p.q = static_cast<const char *>(q);
    p.q_b = 2 * q_strides[0];
    p.q_h = 2 * q_strides[1];
    p.block_table = block_table;
    p.max_pages = max_pages;
    p.seq_lens = seq_lens;
    p.B = B;
    p.Hq = num_q_heads;
    p.Hkv = pages->num_kv_heads;
    p.G = G;
    p.N = (int)N;
    p.S = cut.splits;
    p.least = cut.least;
    p.scale2 = scale * kLog2e;
    p.part_o = reinterpret_cast<float *>(ws + w.off_o);
    p.part_m = reinterpret_cast<float *>(ws + w.off_m);
    p.part_l = reinterpret_cast<float *>(ws + w.off_l);
    p.words = reinterpret_cast<unsigned long long *>(ws + w.off_words);
    p.nonce = cut.splits > 1 ? next_nonce() : 0;
    p.out = out;
    p.lse = lse;
    if (weights_out) {
        p.scores = reinterpret_cast<float *>(ws + w.off_scores);
        p.norm = reinterpret_cast<float2 *>(ws + w.off_norm);
        p.n_pad = (N + 31) / 32 * 32;
        p.w_in = weights_in;
        p.w_out = weights_out;
        p.w_cap = w_cap;
    }
    int lr = launch_paged_attention(p, pages->dtype == VECINFER_BF16, pages->head_dim, static_cast<hipStream_t>(stream));
    if (lr == 0 && weights_out) lr = launch_paged_weights(p, static_cast<hipStream_t>(stream));
    return launch_status(lr);
}

size_t vecinfer_evict_workspace_bytes(int32_t num_kv_heads, int32_t B, int64_t N, int64_t keep)
{
    if (num_kv_heads < 1 || B < 1 || N < 1 || N > kMaxTokens || keep < 1) return 0;
    const EvictLayout w = evict_layout((int64_t)B * num_kv_heads, N, keep);
    return w.total;
}

int vecinfer_paged_evict(const vecinfer_pages *src, const float *weights, int64_t w_cap, const int32_t *block_table,
                         int64_t max_pages, const int32_t *seq_lens, int32_t B, int64_t N, int64_t keep, int64_t first,
                         int64_t recent, const vecinfer_pages *dst, const int32_t *dst_table, int64_t dst_max_pages,
                         int32_t *dst_lens, float *dst_weights, int64_t dst_w_cap, int32_t *kept, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    if (!weights || !block_table || !dst_table || !dst_lens) return VECINFER_EINVAL;
    int rc = pages_ok(src);
    if (rc == VECINFER_OK) rc = pages_ok(dst);
    if (rc != VECINFER_OK) return rc;
    if (src->dtype != dst->dtype || src->head_dim != dst->head_dim || src->num_kv_heads != dst->num_kv_heads) return VECINFER_EINVAL;
    if (B < 1 || N < 1 || max_pages < 1 || dst_max_pages < 1 || w_cap < N) return VECINFER_EINVAL;
    if ((N + src->page_size - 1) / src->page_size > max_pages) return VECINFER_EINVAL;
    if (keep < 1 || (keep + dst->page_size - 1) / dst->page_size > dst_max_pages) return VECINFER_EINVAL;
    if (first < 0 || recent < 0 || first > keep || recent > keep - first) return VECINFER_EINVAL;
    if (dst_lens == seq_lens || dst_weights == weights || (dst_weights && dst_w_cap < keep)) return VECINFER_EINVAL;
    if (!aligned(weights, 4) || !aligned(block_table, 4) || !aligned(dst_table, 4) || !aligned(seq_lens, 4) || !aligned(dst_lens, 4) ||
        !aligned(dst_weights, 4) || !aligned(kept, 4))
        return VECINFER_EINVAL;
    if (B > 65535 || N > kMaxTokens || keep > kMaxTokens) return VECINFER_EUNSUPPORTED;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < vecinfer_evict_workspace_bytes(src->num_kv_heads, B, N, keep))
        return VECINFER_EWORKSPACE;
    EvictParams p = {};
    p.src = page_set(src);
    p.dst = page_set(dst);
    p.w = weights;
    p.w_cap = w_cap;
    p.block_table = block_table;
    p.dst_table = dst_table;
    p.max_pages = max_pages;
    p.dst_max_pages = dst_max_pages;
    p.seq_lens = seq_lens;
    p.B = B;
    p.Hkv = src->num_kv_heads;
    p.D = src->head_dim;
    p.N = (int)N;
    p.keep = (int)keep;
    p.first = (int)first;
    p.recent = (int)recent;
    p.dst_lens = dst_lens;
    p.dst_w = dst_weights;
    p.dst_w_cap = dst_w_cap;
    p.kept = kept;
    const EvictLayout w = evict_layout((int64_t)B * p.Hkv, N, keep);
    unsigned char *const ws = static_cast<unsigned char *>(workspace);
    p.ids = reinterpret_cast<int32_t *>(ws);
    p.hists = reinterpret_cast<unsigned *>(ws + w.off_hists);
    p.states = reinterpret_cast<unsigned *>(ws + w.off_states);
    return launch_status(launch_evict(p, static_cast<hipStream_t>(stream)));
}

} // extern "C"
