// Host side of what a decoder does between the linears and after the output layer (include/flexq.h): argument
// checks, the handles of a paged cache and of a batch's tables, rotary frequencies.  As in fq_api.hip every check comes
// before the first HIP call.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "../../include/flexq.h"
#include "fq_internal.h"

struct fq_kv {
    uint32_t magic;
    FqKvView view;
};

struct fq_seqs {
    uint32_t magic;
    FqSeqsView view; // tokens: set by each call
};

namespace {

constexpr uint32_t KV_MAGIC = 0x46514B56u;   // "FQKV"
constexpr uint32_t SEQS_MAGIC = 0x46515351u; // "FQSQ"
constexpr size_t SAMPLE_BYTES = 256;         // asked of a caller of fq_sample; no kernel uses them (a row is one workgroup's)

inline bool aligned(const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int check_handles(const char *who, const fq_kv *kv, const fq_seqs *seqs, int tokens)
{
    if (!kv || !seqs)
        return fq_fail(FQ_ERR_NULL, "%s: a handle is NULL", who);
    if (kv->magic != KV_MAGIC || seqs->magic != SEQS_MAGIC)
        return fq_fail(FQ_ERR_NULL, "%s: a handle is not valid (destroyed or corrupted)", who);
    if (tokens < 0)
        return fq_fail(FQ_ERR_SHAPE, "%s: tokens must be >= 0 (got %d)", who, tokens);
    const long long places = ((long long)seqs->view.table_width + 1) << kv->view.page_shift;
    if (places + seqs->view.prefix_len > 0x7fff0000LL) // (a step beyond the last key still counts in 32 bits)
        return fq_fail(FQ_ERR_SHAPE, "%s: %d pages of %d tokens to a sequence and a prefix of %d pass 2^31 - 2^16 places", who,
                       seqs->view.table_width, 1 << kv->view.page_shift, seqs->view.prefix_len);
    return FQ_OK;
}

// Rows of [tokens][heads][dim] must not be shorter than a row's values, and keep every 16-byte piece aligned.
int check_rows(const char *who, const char *name, const void *p, long long stride, int heads, int dim)
{
    if (!p)
        return fq_fail(FQ_ERR_NULL, "%s: %s is NULL", who, name);
    if (stride < (long long)heads * dim)
        return fq_fail(FQ_ERR_SHAPE, "%s: rows of %s are %lld elements apart, %d heads of %d need %lld", who, name, stride,
                       heads, dim, (long long)heads * dim);
    if (!aligned(p, 16) || stride % 8 != 0)
        return fq_fail(FQ_ERR_ALIGN, "%s: %s needs 16-byte alignment and a row stride that is a multiple of 8", who, name);
    return FQ_OK;
}

// Whether two sets of as many rows, of width_a and width_b values, share one.  (Rows that lie between each other's share none.)
bool rows_overlap(const void *a, long long stride_a, long long width_a, const void *b, long long stride_b, long long width_b, int rows)
{
    typedef __int128 Place; // of a row in bytes: a stride may be any number
    Place at_a = (Place)(uintptr_t)a, at_b = (Place)(uintptr_t)b;
    const Place step_a = (Place)stride_a * 2, step_b = (Place)stride_b * 2, size_a = width_a * 2, size_b = width_b * 2;
    if (at_a + step_a * (rows - 1) + size_a <= at_b || at_b + step_b * (rows - 1) + size_b <= at_a)
        return false;
    if (step_a == step_b) { // (parts of one row) the last of a's rows to begin before a row of b ends, counted from that one's number
        const Place from = at_b - at_a - size_a, to = at_b - at_a + size_b - 1;
        Place t = to >= 0 ? to / step_a : -((step_a - 1 - to) / step_a);
        t = t < rows - 1 ? t : rows - 1;
        return t > -(Place)rows && t * step_a > from;
    }
    for (int i = 0, j = 0; i < rows && j < rows;) { // both ascend: the row that ends first meets nothing further on
        if (at_a + size_a <= at_b) {
            at_a += step_a;
            i++;
        } else if (at_b + size_b <= at_a) {
            at_b += step_b;
            j++;
        } else {
            return true;
        }
    }
    return false;
}

int check_q_heads(const char *who, int q_heads, int kv_heads)
{
    if (q_heads < 1 || q_heads > FQ_MAX_Q_HEADS || q_heads % kv_heads != 0)
        return fq_fail(FQ_ERR_SHAPE, "%s: q_heads must be a multiple of the cache's %d heads, at most %d (got %d)", who,
                       kv_heads, FQ_MAX_Q_HEADS, q_heads);
    return FQ_OK;
}

int launched(hipError_t e, const char *who)
{
    return e == hipSuccess ? FQ_OK : fq_fail(FQ_ERR_HIP, "%s launch: %s", who, hipGetErrorString(e));
}

} // namespace

extern "C" {

int fq_rope_freqs(int rot_dim, double base, int kind, double factor, double low, double high, double original,
                  double *freqs)
{
    if (!freqs)
        return fq_fail(FQ_ERR_NULL, "fq_rope_freqs: freqs is NULL");
    if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > FQ_MAX_HEAD_DIM)
        return fq_fail(FQ_ERR_SHAPE, "fq_rope_freqs: rot_dim must be even, 2..%d (got %d)", FQ_MAX_HEAD_DIM, rot_dim);
    if (!(base > 1.0) || !std::isfinite(base))
        return fq_fail(FQ_ERR_SHAPE, "fq_rope_freqs: base must be above 1 (got %g)", base);
    if (kind < FQ_ROPE_PLAIN || kind > FQ_ROPE_RAMP)
        return fq_fail(FQ_ERR_SHAPE, "fq_rope_freqs: unknown kind %d", kind);
    if (kind != FQ_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor)))
        return fq_fail(FQ_ERR_SHAPE, "fq_rope_freqs: factor must be at least 1 (got %g)", factor);
    if (kind == FQ_ROPE_BASE && rot_dim < 4)
        return fq_fail(FQ_ERR_SHAPE, "fq_rope_freqs: a scaled base needs rot_dim >= 4");
    const bool banded = kind == FQ_ROPE_WAVELENGTH || kind == FQ_ROPE_RAMP;
    if (banded && (!(low > 0.0) || !(high > low) || !(original > 0.0) || !std::isfinite(high) || !std::isfinite(original)))
        return fq_fail(FQ_ERR_SHAPE, "fq_rope_freqs: need 0 < low < high and original > 0 (got %g, %g, %g)", low, high,
                       original);
    const double two_pi = 6.283185307179586476925286766559;
    const int half = rot_dim / 2;
    const double b = kind == FQ_ROPE_BASE ? base * std::pow(factor, (double)rot_dim / (rot_dim - 2)) : base;
    double first = 0, last = 0;
    if (kind == FQ_ROPE_RAMP) {
        const double unit = rot_dim / (2.0 * std::log(base));
        first = std::fmax(std::floor(unit * std::log(original / (high * two_pi))), 0.0);
        last = std::fmin(std::ceil(unit * std::log(original / (low * two_pi))), rot_dim - 1.0);
    }
    for (int i = 0; i < half; i++) {
        const double f = std::pow(b, -2.0 * i / rot_dim);
        double keep = 1.0; // the share of the unscaled frequency
        if (kind == FQ_ROPE_LINEAR)
            keep = 0.0;
        else if (kind == FQ_ROPE_WAVELENGTH)
            keep = (original * f / two_pi - low) / (high - low);
        else if (kind == FQ_ROPE_RAMP)
            keep = 1.0 - (i - first) / std::fmax(last - first, 0.001); // (a step where the two pairs are one)
        keep = std::fmin(1.0, std::fmax(0.0, keep));
        freqs[i] = kind == FQ_ROPE_PLAIN || kind == FQ_ROPE_BASE ? f : f * (keep + (1.0 - keep) / factor);
    }
    return FQ_OK;
}

int fq_kv_create(fq_kv **out, int dtype, int kv_heads, int head_dim, int page_tokens, int n_pages, void *k, void *v,
                 long long page_stride, long long head_stride, long long token_stride)
{
    if (!out)
        return fq_fail(FQ_ERR_NULL, "fq_kv_create: out is NULL");
    *out = nullptr;
    if (dtype != FQ_F16 && dtype != FQ_BF16)
        return fq_fail(FQ_ERR_BITS, "fq_kv_create: dtype must be FQ_F16 or FQ_BF16 (got %d)", dtype);
    if (kv_heads < 1 || kv_heads > FQ_MAX_Q_HEADS || head_dim < 8 || head_dim > FQ_MAX_HEAD_DIM || head_dim % 8 != 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_kv_create: need 1..%d heads of a multiple of 8, at most %d (got %d of %d)",
                       FQ_MAX_Q_HEADS, FQ_MAX_HEAD_DIM, kv_heads, head_dim);
    if (page_tokens < 1 || page_tokens > 65536 || (page_tokens & (page_tokens - 1)) != 0 || n_pages < 1)
        return fq_fail(FQ_ERR_SHAPE, "fq_kv_create: page_tokens must be a power of two up to 65536 and n_pages >= 1 (got %d "
                                     "and %d)", page_tokens, n_pages);
    if (!k || !v)
        return fq_fail(FQ_ERR_NULL, "fq_kv_create: k or v is NULL");
    if (page_stride < 0 || head_stride < 0 || token_stride < 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_kv_create: strides must not be negative");
    if ((n_pages > 1 && page_stride < head_dim) || (kv_heads > 1 && head_stride < head_dim) ||
        (page_tokens > 1 && token_stride < head_dim))
        return fq_fail(FQ_ERR_SHAPE, "fq_kv_create: a stride is shorter than a head");
    // (far below where a sum of the three products could pass 64 bits; no card holds as much)
    const long long most = 1LL << 46;
    if (page_stride > most / n_pages || head_stride > most / kv_heads || token_stride > most / page_tokens)
        return fq_fail(FQ_ERR_SHAPE, "fq_kv_create: strides span more than 2^46 elements");
    if (!aligned(k, 16) || !aligned(v, 16) || page_stride % 8 != 0 || head_stride % 8 != 0 || token_stride % 8 != 0)
        return fq_fail(FQ_ERR_ALIGN, "fq_kv_create: k and v need 16-byte alignment, strides multiples of 8");
    fq_kv *c = new (std::nothrow) fq_kv();
    if (!c)
        return fq_fail(FQ_ERR_HIP, "fq_kv_create: out of host memory");
    c->magic = KV_MAGIC;
    c->view = FqKvView{(uint16_t *)k, (uint16_t *)v, page_stride, head_stride, token_stride, n_pages,
                       __builtin_ctz((unsigned)page_tokens), kv_heads, head_dim, dtype == FQ_BF16};
    *out = c;
    return FQ_OK;
}

int fq_kv_destroy(fq_kv *kv)
{
    if (!kv || kv->magic != KV_MAGIC)
        return fq_fail(FQ_ERR_NULL, "fq_kv_destroy: NULL or not a valid handle");
    kv->magic = 0;
    delete kv;
    return FQ_OK;
}

int fq_seqs_create(fq_seqs **out, int seqs, const int32_t *q_start, const int32_t *kv_len, const int32_t *table,
                   int table_width, const int32_t *prefix_table, int prefix_len)
{
    if (!out)
        return fq_fail(FQ_ERR_NULL, "fq_seqs_create: out is NULL");
    *out = nullptr;
    if (seqs < 1 || seqs > FQ_MAX_SEQS || table_width < 1 || prefix_len < 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_seqs_create: need seqs in 1..%d, table_width >= 1, prefix_len >= 0 (got %d, %d, %d)",
                       FQ_MAX_SEQS, seqs, table_width, prefix_len);
    if (!q_start || !kv_len || !table || (prefix_len > 0 && !prefix_table))
        return fq_fail(FQ_ERR_NULL, "fq_seqs_create: a table is NULL");
    if (!aligned(q_start, 4) || !aligned(kv_len, 4) || !aligned(table, 4) || !aligned(prefix_table, 4))
        return fq_fail(FQ_ERR_ALIGN, "fq_seqs_create: tables need 4-byte alignment");
    fq_seqs *s = new (std::nothrow) fq_seqs();
    if (!s)
        return fq_fail(FQ_ERR_HIP, "fq_seqs_create: out of host memory");
    s->magic = SEQS_MAGIC;
    s->view = FqSeqsView{q_start, kv_len, table, prefix_len ? prefix_table : nullptr, seqs, table_width, prefix_len, 0};
    *out = s;
    return FQ_OK;
}

int fq_seqs_destroy(fq_seqs *seqs)
{
    if (!seqs || seqs->magic != SEQS_MAGIC)
        return fq_fail(FQ_ERR_NULL, "fq_seqs_destroy: NULL or not a valid handle");
    seqs->magic = 0;
    delete seqs;
    return FQ_OK;
}

int fq_kv_append(const fq_kv *kv, const fq_seqs *seqs, int tokens, const void *q, long long q_stride, int q_heads,
                 void *q_out, long long q_out_stride, const void *k, long long k_stride, const void *v,
                 long long v_stride, const double *freqs, int rot_dim, int interleaved, float amplitude,
                 const int32_t *positions, void *stream)
{
    const char *who = "fq_kv_append";
    if (int rc = check_handles(who, kv, seqs, tokens))
        return rc;
    const FqKvView &c = kv->view;
    if (rot_dim < 0 || rot_dim % 2 != 0 || rot_dim > c.dim)
        return fq_fail(FQ_ERR_SHAPE, "%s: rot_dim must be even, 0..%d (got %d)", who, c.dim, rot_dim);
    if (tokens == 0)
        return FQ_OK;
    if (q_heads != 0) {
        if (int rc = check_q_heads(who, q_heads, c.kv_heads))
            return rc;
        if (int rc = check_rows(who, "q", q, q_stride, q_heads, c.dim))
            return rc;
        if (int rc = check_rows(who, "q_out", q_out, q_out_stride, q_heads, c.dim))
            return rc;
    }
    if (int rc = check_rows(who, "k", k, k_stride, c.kv_heads, c.dim))
        return rc;
    if (int rc = check_rows(who, "v", v, v_stride, c.kv_heads, c.dim))
        return rc;
    if (q_heads != 0) { // (a thread may read a value after another has written its place)
        const long long q_width = (long long)q_heads * c.dim, kv_width = (long long)c.kv_heads * c.dim;
        if (rows_overlap(q_out, q_out_stride, q_width, q, q_stride, q_width, tokens) ||
            rows_overlap(q_out, q_out_stride, q_width, k, k_stride, kv_width, tokens) ||
            rows_overlap(q_out, q_out_stride, q_width, v, v_stride, kv_width, tokens))
            return fq_fail(FQ_ERR_SHAPE, "%s: q_out may not overlap q, k or v", who);
    }
    if (rot_dim > 0 && !freqs)
        return fq_fail(FQ_ERR_NULL, "%s: freqs is NULL", who);
    if (!std::isfinite(amplitude))
        return fq_fail(FQ_ERR_SHAPE, "%s: amplitude must be finite", who);
    if (!aligned(freqs, 8) || !aligned(positions, 4))
        return fq_fail(FQ_ERR_ALIGN, "%s: freqs needs 8-byte, positions 4-byte alignment", who);
    FqAppendArgs a{c, seqs->view, (const uint16_t *)q, (const uint16_t *)k, (const uint16_t *)v, (uint16_t *)q_out, q_stride,
                   q_out_stride, k_stride, v_stride, freqs, positions, q_heads, rot_dim, amplitude};
    a.seqs.tokens = tokens;
    return launched(fq_launch_append(a, interleaved != 0, (hipStream_t)stream), who);
}

static int attend_args(const char *who, const fq_kv *kv, const fq_seqs *seqs, int tokens, int q_heads, int max_q, int max_kv,
                       FqAttendArgs *a)
{
    if (int rc = check_handles(who, kv, seqs, tokens))
        return rc;
    if (int rc = check_q_heads(who, q_heads, kv->view.kv_heads))
        return rc;
    if (tokens > 0 && (max_q < 1 || max_q > tokens || max_kv < 1))
        return fq_fail(FQ_ERR_SHAPE, "%s: need 1 <= max_q <= tokens = %d and max_kv >= 1 (got %d and %d)", who, tokens, max_q,
                       max_kv);
    if ((long long)tokens * q_heads > 0x7fffffffLL)
        return fq_fail(FQ_ERR_SHAPE, "%s: tokens * q_heads passes 2^31", who);
    *a = FqAttendArgs{};
    a->kv = kv->view;
    a->seqs = seqs->view;
    a->seqs.tokens = tokens;
    a->q_heads = q_heads;
    a->max_q = max_q;
    const long long places = (long long)seqs->view.table_width << kv->view.page_shift;
    a->max_kv = max_kv < places ? max_kv : (int)places;
    return FQ_OK;
}

size_t fq_attend_workspace_bytes(const fq_kv *kv, const fq_seqs *seqs, int tokens, int q_heads, int max_q, int max_kv)
{
    FqAttendArgs a;
    if (attend_args("fq_attend_workspace_bytes", kv, seqs, tokens, q_heads, max_q, max_kv, &a))
        return 0;
    return tokens == 0 ? 256 : fq_attend_bytes(a, true, fq_device_cus());
}

int fq_attend(const fq_kv *kv, const fq_seqs *seqs, int tokens, const void *q, long long q_stride, int q_heads, float scale,
              void *out, long long out_stride, float *lse, int max_q, int max_kv, void *workspace, size_t workspace_bytes,
              void *stream)
{
    const char *who = "fq_attend";
    FqAttendArgs a;
    if (int rc = attend_args(who, kv, seqs, tokens, q_heads, max_q, max_kv, &a))
        return rc;
    if (tokens == 0)
        return FQ_OK;
    if (int rc = check_rows(who, "q", q, q_stride, q_heads, kv->view.dim))
        return rc;
    if (int rc = check_rows(who, "out", out, out_stride, q_heads, kv->view.dim))
        return rc;
    if (!workspace)
        return fq_fail(FQ_ERR_NULL, "%s: workspace is NULL", who);
    if (!aligned(lse, 4) || !aligned(workspace, 256))
        return fq_fail(FQ_ERR_ALIGN, "%s: lse needs 4-byte, the workspace 256-byte alignment", who);
    const size_t need = fq_attend_bytes(a, false, fq_device_cus());
    if (workspace_bytes < need)
        return fq_fail(FQ_ERR_SHAPE, "%s: the workspace has %zu bytes, the call needs %zu", who,
                       workspace_bytes, need);
    // (a workgroup reads its own rows of q before it writes theirs of out, in any order with others)
    const long long width = (long long)q_heads * kv->view.dim;
    if ((q != out || q_stride != out_stride) && rows_overlap(q, q_stride, width, out, out_stride, width, tokens))
        return fq_fail(FQ_ERR_SHAPE, "%s: out may be q, row for row, but not overlap it otherwise", who);
    if (!std::isfinite(scale))
        return fq_fail(FQ_ERR_SHAPE, "%s: scale must be finite", who);
    a.q = (const uint16_t *)q;
    a.q_stride = q_stride;
    a.out = (uint16_t *)out;
    a.out_stride = out_stride;
    a.lse = lse;
    a.scale = scale;
    return launched(fq_launch_attend(a, workspace, (hipStream_t)stream), who);
}

size_t fq_sample_workspace_bytes(int R, int V)
{
    if (R < 0 || V < 1 || V > FQ_MAX_SAMPLE_V) {
        fq_fail(FQ_ERR_SHAPE, "fq_sample_workspace_bytes: need R >= 0 and V in 1..%d (got %d and %d)", FQ_MAX_SAMPLE_V, R, V);
        return 0;
    }
    return SAMPLE_BYTES;
}

static int sample_any(const char *who, bool half, const void *logits, int R, int V, long long row_stride, const float *u,
                      const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                      int32_t *token, float *prob, void *workspace, size_t workspace_bytes, void *stream)
{
    if (R < 0 || V < 1 || V > FQ_MAX_SAMPLE_V || row_stride < V || row_stride > (1LL << 40))
        return fq_fail(FQ_ERR_SHAPE, "%s: need R >= 0, V in 1..%d and row_stride >= V (got %d, %d, %lld)", who,
                       FQ_MAX_SAMPLE_V, R, V, row_stride);
    if (R == 0)
        return FQ_OK;
    if (!logits || !u || !token || !workspace)
        return fq_fail(FQ_ERR_NULL, "%s: NULL argument", who);
    if (!aligned(logits, half ? 2 : 4) || !aligned(u, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) ||
        !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(token, 4) || !aligned(prob, 4) || !aligned(workspace, 256))
        return fq_fail(FQ_ERR_ALIGN, "%s: logits need the alignment of their type, the workspace 256 bytes, the rest 4", who);
    if (workspace_bytes < SAMPLE_BYTES)
        return fq_fail(FQ_ERR_SHAPE, "%s: the workspace has %zu bytes, fq_sample_workspace_bytes asks for %zu", who,
                       workspace_bytes, SAMPLE_BYTES);
    const FqSampleArgs a{logits, u, temperature, top_p, min_p, top_k, token, prob, row_stride, R, V};
    return launched(fq_launch_sample(a, half, (hipStream_t)stream), who);
}

int fq_sample(const float *logits, int R, int V, long long row_stride, const float *u, const float *temperature,
              const int32_t *top_k, const float *top_p, const float *min_p, int32_t *token, float *prob, void *workspace,
              size_t workspace_bytes, void *stream)
{
    return sample_any("fq_sample", false, logits, R, V, row_stride, u, temperature, top_k, top_p, min_p, token, prob,
                      workspace, workspace_bytes, stream);
}

int fq_sample_f16(const void *logits, int R, int V, long long row_stride, const float *u, const float *temperature,
                  const int32_t *top_k, const float *top_p, const float *min_p, int32_t *token, float *prob, void *workspace,
                  size_t workspace_bytes, void *stream)
{
    return sample_any("fq_sample_f16", true, logits, R, V, row_stride, u, temperature, top_k, top_p, min_p, token, prob,
                      workspace, workspace_bytes, stream);
}

} // extern "C"
