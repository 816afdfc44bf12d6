// Entry points of the operators of token models: argument checks, workspace sizes, launches on the caller's stream.
//
// Nothing is kept between calls.  Every check is on the host, before anything is launched; a call that fails has launched
// nothing (an error of the HIP runtime aside).
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>

#include "ols_internal.h"

using namespace ols;

namespace {

int bad(const char* fmt, ...) {
    char text[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof(text), fmt, ap);
    va_end(ap);
    return report(OLS_EINVAL, text);
}
int done(hipError_t e, const char* what) {
    if (e == hipSuccess) return OLS_OK;
    char text[400];
    snprintf(text, sizeof(text), "%s: %s", what, hipGetErrorString(e));
    return report(OLS_EHIP, text);
}

bool is_dtype(int t) { return t == OLS_F32 || t == OLS_BF16; }
int64_t size_of(int t) { return t == OLS_F32 ? 4 : 2; }
bool element_aligned(const void* p, int t) { return ((uintptr_t)p & (uintptr_t)(size_of(t) - 1)) == 0; }
bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

constexpr int kMaxGroups = 4096;
constexpr int64_t kMaxTokens = 1 << 24, kMaxVocab = 1 << 24, kMaxWidth = 1 << 20, kMaxStride = (int64_t)1 << 40;

bool stride_ok(int64_t row, int64_t width) { return row >= width && row <= kMaxStride; }
bool group_ok(int64_t g) { return g >= 0 && g <= kMaxStride; }
// Whether the workers' matrices of rows that do not overlap lie behind each other, or side by side within a row's stride.
bool groups_apart(int groups, int64_t group, int64_t rows, int64_t row, int64_t cols) {
    return groups == 1 || group >= (rows - 1) * row + cols || (group >= cols && row >= (groups - 1) * group + cols);
}

// Bytes that a workspace needs, checked against what the caller brought.
int check_ws(const char* who, const void* ws, int64_t have, int64_t need) {
    if (need == 0) return OLS_OK;
    if (!ws || have < need) {
        char text[200];
        snprintf(text, sizeof(text), "%s: workspace of %lld bytes, %lld are needed", who, (long long)(ws ? have : 0), (long long)need);
        return report(OLS_ENOMEM, text);
    }
    if (!aligned(ws, 256)) return bad("%s: the workspace must be 256-byte aligned", who);
    return OLS_OK;
}

int check_embed(const char* who, int groups, int64_t tokens, int64_t vocab, int64_t width) {
    if (groups < 1 || groups > kMaxGroups) return bad("%s: groups must be in [1, %d], got %d", who, kMaxGroups, groups);
    if (tokens < 0 || tokens > kMaxTokens) return bad("%s: tokens must be in [0, 2^24], got %lld", who, (long long)tokens);
    if (vocab < 1 || vocab > kMaxVocab) return bad("%s: vocab must be in [1, 2^24], got %lld", who, (long long)vocab);
    if (width < 1 || width > kMaxWidth) return bad("%s: width must be in [1, 2^20], got %lld", who, (long long)width);
    return OLS_OK;
}

int check_logprob(const char* who, int dtype, int64_t rows, int64_t vocab, const void* logits, int64_t stride, const int32_t* targets) {
    if (!is_dtype(dtype)) return bad("%s: unknown type %d", who, dtype);
    if (rows < 0 || rows > 0x7fffffff) return bad("%s: rows must be in [0, 2^31), got %lld", who, (long long)rows);
    if (vocab < 1 || vocab > kMaxVocab) return bad("%s: vocab must be in [1, 2^24], got %lld", who, (long long)vocab);
    if (rows == 0) return OLS_OK;
    if (!logits || !element_aligned(logits, dtype)) return bad("%s: logits are null or not aligned to their type", who);
    if (!stride_ok(stride, vocab)) return bad("%s: rows of %lld logits cannot be %lld elements apart", who, (long long)vocab, (long long)stride);
    if (!aligned(targets, 4)) return bad("%s: targets are not aligned to their type", who);
    return OLS_OK;
}

// ---- gated feed-forward block ---------------------------------------------------------------------------------------------

int check_ffn(const char* who, const ols_ffn* f) {
    if (!f) return bad("%s: null descriptor", who);
    if (f->groups < 1 || f->groups > kMaxGroups) return bad("%s: groups must be in [1, %d], got %d", who, kMaxGroups, (int)f->groups);
    if (f->act < OLS_ACT_SILU || f->act > OLS_ACT_RELU) return bad("%s: unknown activation %d", who, (int)f->act);
    if (!is_dtype(f->dtype) || !is_dtype(f->weight_dtype) || !is_dtype(f->grad_dtype)) return bad("%s: unknown type", who);
    if (f->dtype == OLS_F32 && (f->weight_dtype != OLS_F32 || f->grad_dtype != OLS_F32)) return bad("%s: an fp32 block has fp32 weights and gradients", who);
    if (f->rows < 0 || f->rows > kMaxTokens) return bad("%s: rows must be in [0, 2^24], got %lld", who, (long long)f->rows);
    const int64_t sizes[3] = {f->width, f->hidden, f->out};
    for (int i = 0; i < 3; ++i)
        if (sizes[i] < 1 || sizes[i] > kMaxWidth)
            return bad("%s: width, hidden and out must be in [1, 2^20], got %lld, %lld, %lld", who, (long long)f->width, (long long)f->hidden, (long long)f->out);
    return OLS_OK;
}

int too_many_tiles(const char* who) { return bad("%s: a product of the workers together has 2^24 - 512 tiles of 128 x 128 results or more", who); }

int check_matrix(const char* who, const char* name, const ols_matrix& m, int64_t rows, int64_t cols, int dtype, int groups, bool written) {
    if (!m.dev || !element_aligned(m.dev, dtype)) return bad("%s: %s is null or not aligned to its type", who, name);
    if (!stride_ok(m.row, cols)) return bad("%s: rows of %s, of %lld elements, cannot be %lld apart", who, name, (long long)cols, (long long)m.row);
    if (!group_ok(m.group)) return bad("%s: the workers' stride of %s is out of range", who, name);
    if (written && !groups_apart(groups, m.group, rows, m.row, cols)) return bad("%s: the workers' %s overlap", who, name);
    return OLS_OK;
}

int check_ffn_operands(const char* who, const ols_ffn& f) {
    if (const int rc = check_matrix(who, "x", f.x, f.rows, f.width, f.dtype, f.groups, false)) return rc;
    if (const int rc = check_matrix(who, "w_gate", f.w_gate, f.width, f.hidden, f.weight_dtype, f.groups, false)) return rc;
    if (const int rc = check_matrix(who, "w_up", f.w_up, f.width, f.hidden, f.weight_dtype, f.groups, false)) return rc;
    return check_matrix(who, "w_down", f.w_down, f.hidden, f.out, f.weight_dtype, f.groups, false);
}

// ---- clipping -----------------------------------------------------------------------------------------------------------

constexpr int64_t kChunk = 16384;             // elements of a workgroup's chunk, doubled until they fill no more than kMostChunks of any group
constexpr int64_t kMostChunks = 2048;
// A tensor has a chunk of its own, however small it is.  Up to this many chunks of a group are added up by every workgroup that copies
// (some three microseconds); more by one workgroup, in a launch between.  50 000 tensors of 8 elements: 6.3 ms, 19.6 without.
constexpr int64_t kManyChunks = 2 * kMostChunks;
int check_clip(const char* who, int n, const int64_t* numel, const int32_t* group, int groups) {
    if (n < 0 || n > (1 << 20)) return bad("%s: number of tensors must be in [0, 2^20], got %d", who, n);
    if (groups < 1 || groups > kMaxGroups) return bad("%s: groups must be in [1, %d], got %d", who, kMaxGroups, groups);
    if (n > 0 && !numel) return bad("%s: null sizes", who);
    if (groups > 1 && n > 0 && !group) return bad("%s: several groups need the tensors' group numbers", who);
    int64_t total = 0;
    for (int i = 0; i < n; ++i) {
        if (numel[i] < 0 || numel[i] > kMaxStride) return bad("%s: tensor %d has %lld elements", who, i, (long long)numel[i]);
        total += numel[i];
        if (total > kMaxStride) return bad("%s: more than 2^40 elements in all", who);
        if (!group) continue;
        if (group[i] < 0 || group[i] >= groups) return bad("%s: tensor %d is of group %d of %d", who, i, (int)group[i], groups);
        if (i && group[i] < group[i - 1]) return bad("%s: the tensors must be in the order of their groups (tensor %d)", who, i);
    }
    return OLS_OK;
}

int group_of(const int32_t* group, int i) { return group ? group[i] : 0; }

int64_t clip_chunk(int n, const int64_t* numel, const int32_t* group) {
    int64_t most = 0, sum = 0;
    for (int i = 0; i < n; ++i) {
        if (i && group_of(group, i) != group_of(group, i - 1)) sum = 0;
        sum += numel[i];
        most = std::max(most, sum);
    }
    int64_t chunk = kChunk;
    while (most / chunk > kMostChunks) chunk *= 2;
    return chunk;
}

int64_t chunks_of(int64_t numel, int64_t chunk) { return (numel + chunk - 1) / chunk; }

struct ClipCall {
    int n;
    const void* const* in;
    void* const* out;
    const int64_t* numel;
    const int32_t* group;
    int64_t chunk;
    int dtype;
    float max_norm;
    float* norms;
    double* partial;
    hipStream_t stream;
};

// One stage of a call, in as many launches as its tensors fill tables.
hipError_t clip_stage(const ClipCall& c, bool copy) {
    ClipTable t = {};
    int blocks = 0, seen = -1;
    int64_t at = 0, group_first = 0, group_chunks = 0;
    for (int i = 0; i < c.n; ++i) {
        if (group_of(c.group, i) != seen) {
            seen = group_of(c.group, i);
            group_first = at, group_chunks = 0;
            for (int j = i; copy && j < c.n && group_of(c.group, j) == seen; ++j) group_chunks += chunks_of(c.numel[j], c.chunk);
            if (group_chunks > kManyChunks) group_chunks = 1;        // their sum lies in the place of the first
        }
        const int64_t chunks = chunks_of(c.numel[i], c.chunk);
        if (chunks == 0) continue;
        if (t.n == kClipTensors || blocks + chunks > 0x3fffffff) {
            const hipError_t e = launch_clip(t, c.dtype, c.chunk, blocks, copy, c.partial, c.max_norm, c.norms, c.stream);
            if (e != hipSuccess) return e;
            t.n = 0, blocks = 0;
        }
        const int k = t.n++;
        t.in[k] = c.in[i], t.out[k] = copy ? c.out[i] : nullptr, t.numel[k] = c.numel[i], t.first_sum[k] = at;
        t.group_first[k] = group_first, t.group_chunks[k] = (int)group_chunks, t.group[k] = seen, t.first_chunk[k] = blocks;
        blocks += (int)chunks, at += chunks;
    }
    return launch_clip(t, c.dtype, c.chunk, blocks, copy, c.partial, c.max_norm, c.norms, c.stream);
}

// Calls launch(table, entries) for the groups that pick(chunks) takes.
template <typename Pick, typename Launch>
hipError_t clip_groups(const ClipCall& c, int groups, Pick pick, Launch launch) {
    ClipGroups t;
    int n = 0, i = 0;
    int64_t at = 0;
    for (int g = 0; g < groups; ++g) {
        const int64_t first = at;
        for (; i < c.n && group_of(c.group, i) == g; ++i) at += chunks_of(c.numel[i], c.chunk);
        if (pick(at - first)) t.first[n] = first, t.count[n] = (int)(at - first), t.group[n] = g, ++n;
        if (n == kClipGroups || (g + 1 == groups && n)) {
            const hipError_t e = launch(t, n);
            if (e != hipSuccess) return e;
            n = 0;
        }
    }
    return hipSuccess;
}

// ---- distillation, beam search, products in 8 bits --------------------------------------------------------------------------

int check_distill(const char* who, const ols_distill* d) {
    if (!d) return bad("%s: null descriptor", who);
    if (d->k < 1 || d->k > OLS_MAX_TEACHER) return bad("%s: k must be in [1, %d], got %d", who, OLS_MAX_TEACHER, (int)d->k);
    if (!(d->temperature >= 0x1p-20f && d->temperature <= 0x1p20f)) return bad("%s: the temperature must be in [2^-20, 2^20], got %g", who, (double)d->temperature);
    if (const int rc = check_logprob(who, d->dtype, d->rows, d->vocab, d->logits, d->row_stride, d->targets)) return rc;
    if (d->rows == 0) return OLS_OK;
    if (!d->top_value || !d->top_index) return bad("%s: null list", who);
    if (!d->stats) return bad("%s: null stats", who);
    if (!aligned(d->top_value, 4) || !aligned(d->top_index, 4) || !aligned(d->loss, 4) || !aligned(d->logprob, 4) || !aligned(d->stats, 4) || !aligned(d->d_loss, 4) ||
        !aligned(d->d_logprob, 4))
        return bad("%s: a pointer is not aligned to its type", who);
    if (d->d_logits) {
        if (!element_aligned(d->d_logits, d->dtype)) return bad("%s: the gradient is not aligned to its type", who);
        if (!stride_ok(d->d_stride, d->vocab)) return bad("%s: rows of %lld gradients cannot be %lld elements apart", who, (long long)d->vocab, (long long)d->d_stride);
        if (d->d_logits == d->logits && d->d_stride != d->row_stride) return bad("%s: a gradient in place needs the logits' row stride", who);
    }
    return OLS_OK;
}
DistillParams distill_params(const ols_distill& d) {
    DistillParams p = {};
    p.dtype = d.dtype, p.k = d.k, p.rest = d.rest != 0, p.temperature = d.temperature, p.rows = d.rows, p.vocab = d.vocab, p.logits = d.logits, p.row_stride = d.row_stride;
    p.value = d.top_value, p.index = d.top_index, p.targets = d.targets, p.loss = d.loss, p.logprob = d.logprob, p.stats = d.stats;
    p.g_loss = d.d_loss, p.g_logprob = d.d_logprob, p.d_logits = d.d_logits, p.d_stride = d.d_stride;
    return p;
}

int check_beam(const char* who, int64_t batch, int in_beams, int beams, int64_t vocab, int dtype) {
    if (!is_dtype(dtype)) return bad("%s: unknown type %d", who, dtype);
    if (batch < 0 || batch > 65535) return bad("%s: batch must be in [0, 65535], got %lld", who, (long long)batch);
    if (in_beams < 1 || in_beams > OLS_MAX_TOP || beams < 1 || beams > OLS_MAX_TOP)
        return bad("%s: hypotheses must be in [1, %d], got %d and %d", who, OLS_MAX_TOP, in_beams, beams);
    if (vocab < 1 || vocab > kMaxVocab) return bad("%s: vocab must be in [1, 2^24], got %lld", who, (long long)vocab);
    return OLS_OK;
}

int too_many_parts(const char* who) { return bad("%s: 2^24 parts of 32768 bf16 or 16384 fp32 logits or more", who); }

// Rows [batch][beams] of `bytes`, as far as they reach; at least one row.
int64_t extent(int64_t batch, int64_t batch_stride, int64_t beams, int64_t beam_stride, int64_t bytes) { return (batch - 1) * batch_stride + (beams - 1) * beam_stride + bytes; }

// Whether a result of a choice lies on what the choice reads (what it takes the place of aside, if of one shape) or on another result.
bool beam_overlaps(const ols_beam& b, int64_t ws_bytes) {
    struct Span {
        const void* at;
        int64_t bytes;
    };
    const int64_t in = b.batch * b.in_beams, out = b.batch * b.beams;
    const Span reads[4] = {{b.score, 4 * in}, {b.length, 4 * in}, {b.finished, in}, {b.ws, ws_bytes}};
    const Span writes[5] = {{b.new_score, 4 * out}, {b.new_length, 4 * out}, {b.new_finished, out}, {b.token, 4 * out}, {b.parent, 4 * out}};
    auto meet = [](const Span& x, const Span& y) { return x.at && y.at && (const char*)x.at < (const char*)y.at + y.bytes && (const char*)y.at < (const char*)x.at + x.bytes; };
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < 4; ++j)
            if (meet(writes[i], reads[j]) && !(i == j && i < 3 && writes[i].at == reads[j].at && b.in_beams == b.beams)) return true;
        for (int j = 0; j < i; ++j)
            if (meet(writes[i], writes[j])) return true;
    }
    return false;
}

// Whether any of these rows shares bytes with [at, at + size).
bool rows_touch(const char* rows, int64_t batch, int64_t batch_stride, int64_t beams, int64_t beam_stride, int64_t bytes, const char* at, int64_t size) {
    if (at + size <= rows || rows + extent(batch, batch_stride, beams, beam_stride, bytes) <= at) return false;
    for (int64_t b = 0; b < batch; ++b)
        for (int64_t i = 0; i < beams; ++i) {
            const char* row = rows + b * batch_stride + i * beam_stride;
            if (row < at + size && at < row + bytes) return true;
        }
    return false;
}

constexpr int64_t kMaxInt8Width = (1 << 17) - 1;      // of whole sums in 32 bits: 2^17 - 1 products of at most 2^14

int check_int8_matrix(const char* who, const char* name, const void* q, int64_t row, int64_t group, int64_t rows, int64_t cols, int groups, bool written) {
    if (!q) return bad("%s: %s is null", who, name);
    if (!stride_ok(row, cols)) return bad("%s: rows of %s, of %lld elements, cannot be %lld apart", who, name, (long long)cols, (long long)row);
    if (!group_ok(group)) return bad("%s: the workers' stride of %s is out of range", who, name);
    if (written && !groups_apart(groups, group, rows, row, cols)) return bad("%s: the workers' %s overlap", who, name);
    return OLS_OK;
}
int check_scale(const char* who, const float* scale, int64_t group, int64_t n, int groups, bool written) {
    if (!scale || !aligned(scale, 4)) return bad("%s: scales are null or not aligned to their type", who);
    if (!group_ok(group) || (written && groups > 1 && group < n)) return bad("%s: the workers' scales overlap or are out of range", who);
    return OLS_OK;
}
int check_quantize(const char* who, int groups, int64_t rows, int64_t width, int dtype, int act) {
    if (groups < 1 || groups > kMaxGroups) return bad("%s: groups must be in [1, %d], got %d", who, kMaxGroups, groups);
    if (!is_dtype(dtype)) return bad("%s: unknown type %d", who, dtype);
    if (rows < 0 || rows > kMaxTokens) return bad("%s: rows must be in [0, 2^24], got %lld", who, (long long)rows);
    if (width < 1 || width > kMaxInt8Width) return bad("%s: width must be in [1, 2^17), got %lld", who, (long long)width);
    if (act < OLS_ACT_SILU || act > OLS_ACT_RELU) return bad("%s: unknown activation %d", who, act);
    return OLS_OK;
}
int check_int8(const char* who, const ols_int8* f) {
    if (!f) return bad("%s: null descriptor", who);
    if (const int rc = check_quantize(who, f->groups, f->rows, f->width, f->dtype == OLS_I8 ? OLS_F32 : f->dtype, f->act)) return rc;
    if (!is_dtype(f->out_dtype)) return bad("%s: unknown type %d of the result", who, (int)f->out_dtype);
    if (f->out < 1 || f->out > kMaxVocab) return bad("%s: out must be in [1, 2^24], got %lld", who, (long long)f->out);
    if (f->dtype == OLS_I8 && f->up.dev) return bad("%s: `up` is for rows that the call quantises", who);
    const int64_t tile = f->rows <= 64 ? 16 : 128;        // a launch has fewer than 2^32 threads
    if ((f->rows + tile - 1) / tile * ((f->out + tile - 1) / tile) * f->groups >= (1 << 23)) return bad("%s: 2^23 tiles of %d x %d results or more", who, (int)tile, (int)tile);
    return OLS_OK;
}

}  // namespace

extern "C" {

int ols_embed(int groups, int64_t tokens, int64_t vocab, int64_t width, const int32_t* ids_dev, int64_t ids_group, const void* table_dev, int dtype,
              int64_t table_row, int64_t table_group, float scale, void* out_dev, int out_dtype, int64_t out_row, int64_t out_group, void* stream) {
    const char* who = "ols_embed";
    if (const int rc = check_embed(who, groups, tokens, vocab, width)) return rc;
    if (!is_dtype(dtype) || !is_dtype(out_dtype)) return bad("%s: unknown type", who);
    if (tokens == 0) return OLS_OK;
    if (!ids_dev || !table_dev || !out_dev) return bad("%s: null pointer", who);
    if (!aligned(ids_dev, 4) || !element_aligned(table_dev, dtype) || !element_aligned(out_dev, out_dtype))
        return bad("%s: a pointer is not aligned to its type", who);
    if (!stride_ok(table_row, width) || !stride_ok(out_row, width)) return bad("%s: rows of %lld elements overlap at the given strides", who, (long long)width);
    if (!group_ok(ids_group) || !group_ok(table_group) || !group_ok(out_group)) return bad("%s: a worker's stride is out of range", who);
    if (!groups_apart(groups, out_group, tokens, out_row, width)) return bad("%s: the workers' outputs overlap", who);
    EmbedParams p;
    p.groups = groups, p.dtype = dtype, p.out_dtype = out_dtype, p.tokens = tokens, p.vocab = vocab, p.width = width;
    p.table = table_dev, p.table_row = table_row, p.table_group = table_group, p.ids = ids_dev, p.ids_group = ids_group, p.scale = scale;
    p.out = out_dev, p.out_row = out_row, p.out_group = out_group;
    return done(launch_embed(p, (hipStream_t)stream), who);
}

int64_t ols_embed_grad_workspace_bytes(int groups, int64_t tokens, int64_t vocab, int64_t width) {
    if (const int rc = check_embed("ols_embed_grad_workspace_bytes", groups, tokens, vocab, width)) return rc;
    return embed_grad_workspace_bytes(groups, tokens, vocab, width);
}

int ols_embed_grad(int groups, int64_t tokens, int64_t vocab, int64_t width, const int32_t* ids_dev, int64_t ids_group, const void* d_out_dev, int dtype,
                   int64_t d_out_row, int64_t d_out_group, float scale, void* grad_dev, int grad_dtype, int64_t grad_row, int64_t grad_group, int accumulate,
                   void* ws_dev, int64_t ws_bytes, void* stream) {
    const char* who = "ols_embed_grad";
    if (const int rc = check_embed(who, groups, tokens, vocab, width)) return rc;
    if (!is_dtype(dtype) || !is_dtype(grad_dtype)) return bad("%s: unknown type", who);
    if (tokens > 0 && (!ids_dev || !d_out_dev)) return bad("%s: null pointer", who);
    if (!grad_dev) return bad("%s: null gradient", who);
    if (!aligned(ids_dev, 4) || !element_aligned(d_out_dev, dtype) || !element_aligned(grad_dev, grad_dtype))
        return bad("%s: a pointer is not aligned to its type", who);
    if (!stride_ok(d_out_row, width) || !stride_ok(grad_row, width)) return bad("%s: rows of %lld elements overlap at the given strides", who, (long long)width);
    if (!group_ok(ids_group) || !group_ok(d_out_group) || !group_ok(grad_group)) return bad("%s: a worker's stride is out of range", who);
    if (!groups_apart(groups, grad_group, vocab, grad_row, width)) return bad("%s: the workers' gradients overlap", who);
    if (const int rc = check_ws(who, ws_dev, ws_bytes, embed_grad_workspace_bytes(groups, tokens, vocab, width))) return rc;
    EmbedGradParams p;
    p.groups = groups, p.dtype = dtype, p.grad_dtype = grad_dtype, p.accumulate = accumulate != 0, p.tokens = tokens, p.vocab = vocab, p.width = width;
    p.ids = ids_dev, p.ids_group = ids_group, p.dout = d_out_dev, p.dout_row = d_out_row, p.dout_group = d_out_group, p.scale = scale;
    p.grad = grad_dev, p.grad_row = grad_row, p.grad_group = grad_group;
    return done(launch_embed_grad(p, ws_dev, (hipStream_t)stream), who);
}

int64_t ols_gated_ffn_saved_bytes(const ols_ffn* f) {
    if (const int rc = check_ffn("ols_gated_ffn_saved_bytes", f)) return rc;
    return ffn_saved_bytes(*f);
}

int64_t ols_gated_ffn_workspace_bytes(const ols_ffn* f, int grad) {
    if (const int rc = check_ffn("ols_gated_ffn_workspace_bytes", f)) return rc;
    const int64_t need = ffn_workspace_bytes(*f, grad != 0);
    return need < 0 ? too_many_tiles("ols_gated_ffn_workspace_bytes") : need;
}

int ols_gated_ffn(const ols_ffn* f, void* stream) {
    const char* who = "ols_gated_ffn";
    if (const int rc = check_ffn(who, f)) return rc;
    if (f->rows == 0) return OLS_OK;
    if (const int rc = check_ffn_operands(who, *f)) return rc;
    if (const int rc = check_matrix(who, "y", f->y, f->rows, f->out, f->dtype, f->groups, true)) return rc;
    if (f->saved) {
        if (f->saved_bytes < ffn_saved_bytes(*f)) return bad("%s: `saved` of %lld bytes, %lld are needed", who, (long long)f->saved_bytes, (long long)ffn_saved_bytes(*f));
        if (!aligned(f->saved, 256)) return bad("%s: `saved` must be 256-byte aligned", who);
    }
    const int64_t need = ffn_workspace_bytes(*f, false);
    if (need < 0) return too_many_tiles(who);
    if (const int rc = check_ws(who, f->ws, f->ws_bytes, need)) return rc;
    return done(launch_ffn(*f, false, (hipStream_t)stream), who);
}

int ols_gated_ffn_grad(const ols_ffn* f, void* stream) {
    const char* who = "ols_gated_ffn_grad";
    if (const int rc = check_ffn(who, f)) return rc;
    const ols_matrix* g[3] = {&f->g_gate, &f->g_up, &f->g_down};
    const char* names[3] = {"g_gate", "g_up", "g_down"};
    for (int i = 0; i < 3; ++i)
        if (g[i]->dev)
            if (const int rc = check_matrix(who, names[i], *g[i], i < 2 ? f->width : f->hidden, i < 2 ? f->hidden : f->out, f->grad_dtype, f->groups, true)) return rc;
    if (f->rows > 0) {
        if (const int rc = check_ffn_operands(who, *f)) return rc;
        if (const int rc = check_matrix(who, "dy", f->dy, f->rows, f->out, f->dtype, f->groups, false)) return rc;
        if (f->dx.dev)
            if (const int rc = check_matrix(who, "dx", f->dx, f->rows, f->width, f->dtype, f->groups, true)) return rc;
        if (!f->saved || f->saved_bytes < ffn_saved_bytes(*f))
            return bad("%s: `saved` of %lld bytes, %lld are needed", who, (long long)(f->saved ? f->saved_bytes : 0), (long long)ffn_saved_bytes(*f));
        if (!aligned(f->saved, 256)) return bad("%s: `saved` must be 256-byte aligned", who);
        const int64_t need = ffn_workspace_bytes(*f, true);
        if (need < 0) return too_many_tiles(who);
        if (const int rc = check_ws(who, f->ws, f->ws_bytes, need)) return rc;
        if (f->dx.dev && (f->dx.dev == f->x.dev || f->dx.dev == f->dy.dev) &&
            ((f->g_gate.dev && f->g_gate.dev == f->w_gate.dev) || (f->g_up.dev && f->g_up.dev == f->w_up.dev)))
            return bad("%s: dx on x or dy and the gradients of gate or up on the weights, both at once", who);
    }
    return done(launch_ffn(*f, true, (hipStream_t)stream), who);
}

int64_t ols_token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int dtype, int top) {
    const char* who = "ols_token_logprobs_workspace_bytes";
    if (const int rc = check_logprob(who, dtype, 0, vocab, nullptr, vocab, nullptr)) return rc;
    if (rows < 0 || rows > 0x7fffffff) return bad("%s: rows must be in [0, 2^31), got %lld", who, (long long)rows);
    if (top < 0 || top > OLS_MAX_TOP || top > vocab) return bad("%s: top must be in [0, min(%d, vocab)], got %d", who, OLS_MAX_TOP, top);
    return logprob_workspace_bytes(dtype, rows, vocab, top);
}

int ols_token_logprobs(int64_t rows, int64_t vocab, const void* logits_dev, int dtype, int64_t row_stride, const int32_t* targets_dev, float* logprob_dev,
                       float* entropy_dev, float* logsumexp_dev, float* stats_dev, int top, float* top_logprob_dev, int32_t* top_index_dev, const float* d_logprob_dev,
                       const float* d_entropy_dev, void* d_logits_dev, int64_t d_stride, void* ws_dev, int64_t ws_bytes, void* stream) {
    const char* who = "ols_token_logprobs";
    if (const int rc = check_logprob(who, dtype, rows, vocab, logits_dev, row_stride, targets_dev)) return rc;
    if (top < 0 || top > OLS_MAX_TOP || top > vocab) return bad("%s: top must be in [0, min(%d, vocab)], got %d", who, OLS_MAX_TOP, top);
    if (rows == 0) return OLS_OK;
    if (!logprob_dev || !entropy_dev || !logsumexp_dev || !stats_dev) return bad("%s: null result", who);
    if (top > 0 && (!top_logprob_dev || !top_index_dev)) return bad("%s: null results for the alternatives", who);
    if (!aligned(logprob_dev, 4) || !aligned(entropy_dev, 4) || !aligned(logsumexp_dev, 4) || !aligned(stats_dev, 4) || !aligned(top_logprob_dev, 4) || !aligned(top_index_dev, 4) ||
        !aligned(d_logprob_dev, 4) || !aligned(d_entropy_dev, 4))
        return bad("%s: a pointer is not aligned to its type", who);
    if (d_logits_dev) {
        if (!element_aligned(d_logits_dev, dtype)) return bad("%s: the gradient is not aligned to its type", who);
        if (!stride_ok(d_stride, vocab)) return bad("%s: rows of %lld gradients cannot be %lld elements apart", who, (long long)vocab, (long long)d_stride);
        if (d_logits_dev == logits_dev && d_stride != row_stride) return bad("%s: a gradient in place needs the logits' row stride", who);
    }
    if (const int rc = check_ws(who, ws_dev, ws_bytes, logprob_workspace_bytes(dtype, rows, vocab, top))) return rc;
    LogprobParams p = {};
    p.dtype = dtype, p.top = top, p.rows = rows, p.vocab = vocab, p.logits = logits_dev, p.row_stride = row_stride, p.targets = targets_dev;
    p.logprob = logprob_dev, p.entropy = entropy_dev, p.lse = logsumexp_dev, p.stats = stats_dev, p.top_logprob = top_logprob_dev, p.top_index = top_index_dev;
    p.g_logprob = d_logprob_dev, p.g_entropy = d_entropy_dev, p.d_logits = d_logits_dev, p.d_stride = d_stride;
    return done(launch_logprob(p, ws_dev, (hipStream_t)stream), who);
}

int ols_token_logprobs_grad(int64_t rows, int64_t vocab, const void* logits_dev, int dtype, int64_t row_stride, const int32_t* targets_dev,
                            const float* stats_dev, const float* entropy_dev, const float* d_logprob_dev, const float* d_entropy_dev, void* d_logits_dev,
                            int64_t d_stride, void* stream) {
    const char* who = "ols_token_logprobs_grad";
    if (const int rc = check_logprob(who, dtype, rows, vocab, logits_dev, row_stride, targets_dev)) return rc;
    if (rows == 0) return OLS_OK;
    if (!stats_dev || !d_logits_dev) return bad("%s: null pointer", who);
    if (d_entropy_dev && !entropy_dev) return bad("%s: the entropy's gradient needs the entropy", who);
    if (!aligned(stats_dev, 4) || !aligned(entropy_dev, 4) || !aligned(d_logprob_dev, 4) || !aligned(d_entropy_dev, 4) || !element_aligned(d_logits_dev, dtype))
        return bad("%s: a pointer is not aligned to its type", who);
    if (!stride_ok(d_stride, vocab)) return bad("%s: rows of %lld gradients cannot be %lld elements apart", who, (long long)vocab, (long long)d_stride);
    if (d_logits_dev == logits_dev && d_stride != row_stride) return bad("%s: a gradient in place needs the logits' row stride", who);
    LogprobParams p = {};
    p.dtype = dtype, p.rows = rows, p.vocab = vocab, p.logits = logits_dev, p.row_stride = row_stride, p.targets = targets_dev;
    p.stats = const_cast<float*>(stats_dev), p.entropy = const_cast<float*>(entropy_dev), p.g_logprob = d_logprob_dev, p.g_entropy = d_entropy_dev;
    p.d_logits = d_logits_dev, p.d_stride = d_stride;
    return done(launch_logprob_grad(p, (hipStream_t)stream), who);
}

int64_t ols_clip_workspace_bytes(int n, const int64_t* numel, const int32_t* group, int groups) {
    if (const int rc = check_clip("ols_clip_workspace_bytes", n, numel, group, groups)) return rc;
    const int64_t chunk = clip_chunk(n, numel, group);
    int64_t chunks = 0;
    for (int i = 0; i < n; ++i) chunks += chunks_of(numel[i], chunk);
    return 8 * chunks;
}

int ols_clip_gradients(int n, const void* const* in_dev, void* const* out_dev, const int64_t* numel, const int32_t* group, int groups, int dtype,
                       float max_norm, float* norms_dev, void* ws_dev, int64_t ws_bytes, void* stream) {
    const char* who = "ols_clip_gradients";
    if (const int rc = check_clip(who, n, numel, group, groups)) return rc;
    if (!is_dtype(dtype)) return bad("%s: unknown type %d", who, dtype);
    if (!norms_dev || !aligned(norms_dev, 4)) return bad("%s: norms are null or not aligned to their type", who);
    if (n > 0 && !in_dev) return bad("%s: null pointers", who);
    if (out_dev && !(max_norm >= 0.0f)) return bad("%s: max_norm must not be negative", who);
    for (int i = 0; i < n; ++i) {
        if (numel[i] == 0) continue;
        if (!in_dev[i] || !element_aligned(in_dev[i], dtype)) return bad("%s: tensor %d is null or not aligned to its type", who, i);
        if (out_dev && (!out_dev[i] || !element_aligned(out_dev[i], dtype))) return bad("%s: output %d is null or not aligned to its type", who, i);
    }
    const int64_t chunk = clip_chunk(n, numel, group);
    int64_t need = 0;
    for (int i = 0; i < n; ++i) need += 8 * chunks_of(numel[i], chunk);
    if (const int rc = check_ws(who, ws_dev, ws_bytes, need)) return rc;
    const ClipCall c{n, in_dev, out_dev, numel, group, chunk, dtype, max_norm, norms_dev, (double*)ws_dev, (hipStream_t)stream};
    hipError_t e = clip_stage(c, false);
    if (e == hipSuccess && out_dev) {
        e = clip_groups(c, groups, [](int64_t chunks) { return chunks > kManyChunks; },
                        [&](const ClipGroups& t, int k) { return launch_clip_sums(t, k, c.partial, c.stream); });
        if (e == hipSuccess) e = clip_stage(c, true);
    }
    // the groups whose norm no copy has written: all without outputs, otherwise those without elements
    if (e == hipSuccess)
        e = clip_groups(c, groups, [&](int64_t chunks) { return !out_dev || chunks == 0; },
                        [&](const ClipGroups& t, int k) { return launch_clip_norms(t, k, c.partial, norms_dev, c.stream); });
    return done(e, who);
}

int64_t ols_distill_workspace_bytes(int64_t rows, int64_t vocab, int dtype, int k) {
    const char* who = "ols_distill_workspace_bytes";
    if (const int rc = check_logprob(who, dtype, 0, vocab, nullptr, vocab, nullptr)) return rc;
    if (rows < 0 || rows > 0x7fffffff) return bad("%s: rows must be in [0, 2^31), got %lld", who, (long long)rows);
    if (k < 1 || k > OLS_MAX_TEACHER) return bad("%s: k must be in [1, %d], got %d", who, OLS_MAX_TEACHER, k);
    return distill_workspace_bytes(dtype, rows, vocab, k);
}

int ols_distill_loss(const ols_distill* d, void* stream) {
    const char* who = "ols_distill_loss";
    if (const int rc = check_distill(who, d)) return rc;
    if (d->rows == 0) return OLS_OK;
    if (!d->loss || (d->targets && !d->logprob)) return bad("%s: null result", who);
    if (const int rc = check_ws(who, d->ws, d->ws_bytes, distill_workspace_bytes(d->dtype, d->rows, d->vocab, d->k))) return rc;
    DistillParams p = distill_params(*d);
    if (!d->targets) p.logprob = nullptr;
    return done(launch_distill(p, d->ws, (hipStream_t)stream), who);
}

int ols_distill_loss_grad(const ols_distill* d, void* stream) {
    const char* who = "ols_distill_loss_grad";
    if (const int rc = check_distill(who, d)) return rc;
    if (d->rows == 0) return OLS_OK;
    if (!d->d_logits) return bad("%s: null gradient", who);
    return done(launch_distill_grad(distill_params(*d), (hipStream_t)stream), who);
}

int64_t ols_beam_workspace_bytes(int64_t batch, int in_beams, int beams, int64_t vocab, int dtype) {
    if (const int rc = check_beam("ols_beam_workspace_bytes", batch, in_beams, beams, vocab, dtype)) return rc;
    const int64_t need = beam_workspace_bytes(dtype, batch, in_beams, beams, vocab);
    return need < 0 ? too_many_parts("ols_beam_workspace_bytes") : need;
}

int ols_beam_select(const ols_beam* b, void* stream) {
    const char* who = "ols_beam_select";
    if (!b) return bad("%s: null descriptor", who);
    if (const int rc = check_beam(who, b->batch, b->in_beams, b->beams, b->vocab, b->dtype)) return rc;
    if (!(b->length_penalty >= -16.0 && b->length_penalty <= 16.0)) return bad("%s: the length penalty must be in [-16, 16], got %g", who, b->length_penalty);
    if (b->length_penalty != 0.0 && !b->length) return bad("%s: a length penalty needs the lengths", who);
    if (b->new_length && !b->length) return bad("%s: new lengths need the lengths", who);
    if (b->batch == 0) return OLS_OK;
    if (!b->logits || !element_aligned(b->logits, b->dtype)) return bad("%s: logits are null or not aligned to their type", who);
    if (!group_ok(b->batch_stride) || !group_ok(b->beam_stride)) return bad("%s: a stride of the logits is out of range", who);
    if (!b->score || !b->new_score || !b->token || !b->parent || !b->new_finished) return bad("%s: null pointer", who);
    if (!aligned(b->score, 4) || !aligned(b->length, 4) || !aligned(b->new_score, 4) || !aligned(b->token, 4) || !aligned(b->parent, 4) || !aligned(b->new_length, 4))
        return bad("%s: a pointer is not aligned to its type", who);
    const int64_t need = beam_workspace_bytes(b->dtype, b->batch, b->in_beams, b->beams, b->vocab);
    if (need < 0) return too_many_parts(who);
    if (const int rc = check_ws(who, b->ws, b->ws_bytes, need)) return rc;
    if (beam_overlaps(*b, need)) return bad("%s: results overlap what is read, or each other", who);
    BeamParams p = {};
    p.dtype = b->dtype, p.in_beams = b->in_beams, p.beams = b->beams, p.eos = b->eos, p.batch = b->batch, p.vocab = b->vocab;
    p.logits = b->logits, p.batch_stride = b->batch_stride, p.beam_stride = b->beam_stride, p.score = b->score, p.finished = b->finished, p.length = b->length;
    p.penalty = b->length_penalty, p.new_score = b->new_score, p.token = b->token, p.parent = b->parent, p.new_length = b->new_length, p.new_finished = b->new_finished;
    return done(launch_beam(p, b->ws, (hipStream_t)stream), who);
}

int ols_beam_reorder(int n, const void* const* src, void* const* dst, const int64_t* row_bytes, const int64_t* src_batch, const int64_t* src_beam,
                     const int64_t* dst_batch, const int64_t* dst_beam, int64_t batch, int in_beams, int beams, const int32_t* parent, void* stream) {
    const char* who = "ols_beam_reorder";
    if (const int rc = check_beam(who, batch, in_beams, beams, 1, OLS_F32)) return rc;
    if (n < 0 || n > (1 << 20)) return bad("%s: number of tensors must be in [0, 2^20], got %d", who, n);
    if (n == 0 || batch == 0) return OLS_OK;
    if (!src || !dst || !row_bytes || !src_batch || !src_beam || !dst_batch || !dst_beam) return bad("%s: null arrays", who);
    if (!parent || !aligned(parent, 4)) return bad("%s: parents are null or not aligned to their type", who);
    for (int i = 0; i < n; ++i) {
        const int64_t bytes = row_bytes[i];
        if (bytes < 0 || bytes > (int64_t)1 << 35) return bad("%s: rows of tensor %d have %lld bytes", who, i, (long long)bytes);
        if (bytes == 0) continue;
        if (!src[i] || !dst[i]) return bad("%s: tensor %d is null", who, i);
        if (!group_ok(src_batch[i]) || !group_ok(src_beam[i]) || !group_ok(dst_batch[i]) || !group_ok(dst_beam[i])) return bad("%s: a stride of tensor %d is out of range", who, i);
        if ((beams > 1 && dst_beam[i] < bytes) || !groups_apart((int)batch, dst_batch[i], beams, beams > 1 ? dst_beam[i] : bytes, bytes))
            return bad("%s: rows of output %d overlap", who, i);
        if (src[i] == dst[i]) {
            if (in_beams != beams || (batch > 1 && src_batch[i] != dst_batch[i]) || (beams > 1 && src_beam[i] != dst_beam[i]))
                return bad("%s: tensor %d in place needs one shape and the same strides", who, i);
        } else {
            const char *s = (const char*)src[i], *d = (const char*)dst[i];
            if (s < d + extent(batch, dst_batch[i], beams, dst_beam[i], bytes) && d < s + extent(batch, src_batch[i], in_beams, src_beam[i], bytes))
                return bad("%s: output %d lies partly on its input", who, i);
        }
        if (rows_touch((const char*)dst[i], batch, dst_batch[i], beams, dst_beam[i], bytes, (const char*)parent, 4 * batch * beams))
            return bad("%s: output %d lies on the parents, which are read meanwhile", who, i);
    }
    BeamMove t;
    t.in_beams = in_beams, t.out_beams = beams, t.n = 0;
    int64_t blocks = 0;
    auto launch = [&]() {
        // a launch has fewer than 2^32 threads
        const int64_t step = std::max<int64_t>(1, std::min<int64_t>(batch, ((1 << 24) - 1) / std::max<int64_t>(1, blocks)));
        for (int64_t first = 0; first < batch; first += step) {
            BeamMove u = t;
            u.parent = parent + first * beams;
            for (int i = 0; i < t.n; ++i)
                u.src[i] = (const char*)t.src[i] + first * t.src_batch[i], u.dst[i] = (char*)t.dst[i] + first * t.dst_batch[i];
            const hipError_t e = launch_beam_move(u, (unsigned)blocks, std::min(step, batch - first), (hipStream_t)stream);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    for (int i = 0; i < n; ++i) {
        if (row_bytes[i] == 0) continue;
        const int64_t need = (row_bytes[i] + 4095) / 4096;
        if (t.n == kMoveTensors || (t.n && blocks + need >= (1 << 24))) {
            if (const hipError_t e = launch()) return done(e, who);
            t.n = 0, blocks = 0;
        }
        const int k = t.n++;
        t.src[k] = src[i], t.dst[k] = dst[i], t.row_bytes[k] = row_bytes[i], t.first_block[k] = (int)blocks;
        t.src_batch[k] = src_batch[i], t.src_beam[k] = src_beam[i], t.dst_batch[k] = dst_batch[i], t.dst_beam[k] = dst_beam[i];
        blocks += need;
    }
    return done(t.n ? launch() : hipSuccess, who);
}

int ols_quantize_rows(int groups, int64_t rows, int64_t width, const ols_matrix* x, const ols_matrix* up, int act, int dtype, int8_t* q, int64_t q_row,
                      int64_t q_group, float* scale, int64_t scale_group, void* stream) {
    const char* who = "ols_quantize_rows";
    if (const int rc = check_quantize(who, groups, rows, width, dtype, act)) return rc;
    if (rows == 0) return OLS_OK;
    if (!x) return bad("%s: null x", who);
    if (const int rc = check_matrix(who, "x", *x, rows, width, dtype, groups, false)) return rc;
    if (up && up->dev)
        if (const int rc = check_matrix(who, "up", *up, rows, width, dtype, groups, false)) return rc;
    if (const int rc = check_int8_matrix(who, "q", q, q_row, q_group, rows, width, groups, true)) return rc;
    if (const int rc = check_scale(who, scale, scale_group, rows, groups, true)) return rc;
    QuantRows p = {};
    p.groups = groups, p.dtype = dtype, p.act = act, p.rows = rows, p.width = width, p.x = *x;
    if (up) p.up = *up;
    p.q = q, p.q_row = q_row, p.q_group = q_group, p.scale = scale, p.scale_group = scale_group, p.padded = width;
    return done(launch_quantize_rows(p, (hipStream_t)stream), who);
}

int64_t ols_quantize_weight_workspace_bytes(int groups, int64_t width, int64_t out) {
    const char* who = "ols_quantize_weight_workspace_bytes";
    if (const int rc = check_quantize(who, groups, 0, width, OLS_F32, OLS_ACT_SILU)) return rc;
    if (out < 1 || out > kMaxVocab) return bad("%s: out must be in [1, 2^24], got %lld", who, (long long)out);
    return quantize_weight_workspace_bytes(groups, width, out);
}

int ols_quantize_weight(int groups, int64_t width, int64_t out, const ols_matrix* w, int dtype, int8_t* q, int64_t q_row, int64_t q_group, float* scale,
                        int64_t scale_group, void* ws_dev, int64_t ws_bytes, void* stream) {
    const char* who = "ols_quantize_weight";
    if (const int rc = check_quantize(who, groups, 0, width, dtype, OLS_ACT_SILU)) return rc;
    if (out < 1 || out > kMaxVocab) return bad("%s: out must be in [1, 2^24], got %lld", who, (long long)out);
    if ((out + 63) / 64 * ((width + 63) / 64) * groups >= (1 << 24)) return bad("%s: 2^24 tiles of 64 x 64 weights or more", who);
    if (!w) return bad("%s: null weights", who);
    if (const int rc = check_matrix(who, "w", *w, width, out, dtype, groups, false)) return rc;
    if (const int rc = check_int8_matrix(who, "q", q, q_row, q_group, out, width, groups, true)) return rc;
    if (const int rc = check_scale(who, scale, scale_group, out, groups, true)) return rc;
    if (const int rc = check_ws(who, ws_dev, ws_bytes, quantize_weight_workspace_bytes(groups, width, out))) return rc;
    QuantWeight p = {groups, dtype, width, out, *w, q, q_row, q_group, scale, scale_group};
    return done(launch_quantize_weight(p, ws_dev, (hipStream_t)stream), who);
}

int64_t ols_int8_workspace_bytes(const ols_int8* f) {
    if (const int rc = check_int8("ols_int8_workspace_bytes", f)) return rc;
    return int8_workspace_bytes(*f);
}

int ols_int8_matmul(const ols_int8* f, void* stream) {
    const char* who = "ols_int8_matmul";
    if (const int rc = check_int8(who, f)) return rc;
    if (f->rows == 0) return OLS_OK;
    if (f->dtype == OLS_I8) {
        if (const int rc = check_int8_matrix(who, "x", f->x.dev, f->x.row, f->x.group, f->rows, f->width, f->groups, false)) return rc;
        if (const int rc = check_scale(who, f->x_scale, f->x_scale_group, f->rows, f->groups, false)) return rc;
    } else {
        if (const int rc = check_matrix(who, "x", f->x, f->rows, f->width, f->dtype, f->groups, false)) return rc;
        if (f->up.dev)
            if (const int rc = check_matrix(who, "up", f->up, f->rows, f->width, f->dtype, f->groups, false)) return rc;
    }
    if (const int rc = check_int8_matrix(who, "w", f->w.dev, f->w.row, f->w.group, f->out, f->width, f->groups, false)) return rc;
    if (const int rc = check_scale(who, f->w_scale, f->w_scale_group, f->out, f->groups, false)) return rc;
    if (const int rc = check_matrix(who, "y", f->y, f->rows, f->out, f->out_dtype, f->groups, true)) return rc;
    if (const int rc = check_ws(who, f->ws, f->ws_bytes, int8_workspace_bytes(*f))) return rc;
    return done(launch_int8(*f, (hipStream_t)stream), who);
}

}  // extern "C"
