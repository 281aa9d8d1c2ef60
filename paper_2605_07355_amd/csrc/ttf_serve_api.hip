// C ABI of the entry points behind the compressed rows: argument checks and the frequencies of a rotation.
#include <cmath>
#include <cstdlib>

#include "ttf_serve.h"

namespace ttf {
namespace {

inline bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) % 16) == 0; }

ttf_status check_head(int dtype, int head_dim)
{
    if (head_dim < 1) return TTF_ERR_INVALID_ARG;
    if (dtype != TTF_BF16 && dtype != TTF_F32) return TTF_ERR_UNSUPPORTED;
    return head_dim % 8 != 0 || head_dim > kMaxHeadDim ? TTF_ERR_UNSUPPORTED : TTF_OK;
}

// A [rows, heads, D] operand: strides in steps of 16 bytes, neighbouring rows and neighbouring heads apart.
ttf_status check_rows(const void* p, int64_t row, int64_t head, int rows, int heads, int D, int dtype)
{
    const int64_t unit = dtype == TTF_BF16 ? 8 : 4, most = 1ll << 40;
    if (!p) return TTF_ERR_INVALID_ARG;
    if (row < 0 || head < 0 || row > most || head > most) return TTF_ERR_INVALID_ARG;
    if ((rows > 1 && row < D) || (heads > 1 && head < D)) return TTF_ERR_INVALID_ARG;
    return !aligned(p) || row % unit != 0 || head % unit != 0 ? TTF_ERR_UNSUPPORTED : TTF_OK;
}

// Whether two of the heads that are written share an entry: heads j apart in one direction and rows i in the other that meet.  (Strides as
// check_rows leaves them: at least D where there are two.)
bool folded(int64_t row, int64_t head, int rows, int heads, int D)
{
    if (rows < 2 || heads < 2 || (row - D) / head >= heads - 1 || (head - D) / row >= rows - 1) return false;    // (one inside the other)
    for (int64_t j = 1; j < heads; ++j)
        for (int64_t i = j * head / row, end = i + 1; i <= end && i < rows; ++i)
            if (std::llabs(j * head - i * row) < D) return true;
    return false;
}

// Whether an output that is the input itself has other strides than it.
bool crossed(const void* from, int64_t row, int64_t head, const void* to, int64_t to_row, int64_t to_head, int rows, int heads)
{
    return from == to && ((rows > 1 && row != to_row) || (heads > 1 && head != to_head));
}

// Sizes that every launch grid and every 32-bit index of the kernels has room for.
bool sizes_fit(int rows, int batch, int heads, int kv_heads)
{
    if (rows < 1 || rows > (1 << 24) || batch < 1 || batch > (1 << 20)) return false;
    if (heads < 0 || kv_heads < 0 || heads > 65536 || kv_heads > 65536) return false;
    const long long most = heads > kv_heads ? heads : kv_heads;
    return rows * most <= (1ll << 27) && batch * most <= (1ll << 22);
}

ttf_status check_cache(const ttf_kv_cache* c, int kv_heads, int D, int dtype)
{
    const int64_t unit = dtype == TTF_BF16 ? 8 : 4, most = 1ll << 40;
    if (!c || !c->k || !c->v || !c->page_table) return TTF_ERR_INVALID_ARG;
    if (c->pages < 1 || c->page_size < 1 || c->table_width < 1 || c->table_stride < c->table_width) return TTF_ERR_INVALID_ARG;
    for (const int64_t s : {c->page_stride, c->slot_stride, c->head_stride})
        if (s < 0 || s > most) return TTF_ERR_INVALID_ARG;
    if (c->page_size > (1 << 20) || c->table_stride > most) return TTF_ERR_INVALID_ARG;
    if ((c->pages > 1 && c->page_stride < D) || (c->page_size > 1 && c->slot_stride < D) || (kv_heads > 1 && c->head_stride < D))
        return TTF_ERR_INVALID_ARG;
    return !aligned(c->k) || !aligned(c->v) || c->page_stride % unit != 0 || c->slot_stride % unit != 0 || c->head_stride % unit != 0
               ? TTF_ERR_UNSUPPORTED : TTF_OK;
}

ttf_status check_qk(const ttf_qk_params* p, bool append)
{
    if (!p) return TTF_ERR_INVALID_ARG;
    if (!sizes_fit(p->rows, p->batch, p->heads, p->kv_heads)) return TTF_ERR_INVALID_ARG;
    if (p->heads + p->kv_heads < 1 || (append && p->kv_heads < 1)) return TTF_ERR_INVALID_ARG;
    if (append && (!p->row_offsets || !p->cached)) return TTF_ERR_INVALID_ARG;
    if (p->rotary_dim < 0 || p->rotary_dim % 2 != 0 || p->rotary_dim > p->head_dim) return TTF_ERR_INVALID_ARG;
    if (p->layout != TTF_ROPE_HALF && p->layout != TTF_ROPE_INTERLEAVED) return TTF_ERR_INVALID_ARG;
    if (p->rotary_dim > 0 && (!p->pos || !p->inv_freq || p->axes < 1 || p->axes > 4 || (p->axes > 1 && p->pos_stride < p->rows) ||
                              !std::isfinite(p->attention_factor)))
        return TTF_ERR_INVALID_ARG;
    if ((p->q_weight || p->k_weight) && !(p->eps >= 0.0f && std::isfinite(p->eps))) return TTF_ERR_INVALID_ARG;
    ttf_status st = check_head(p->dtype, p->head_dim);
    if (st == TTF_OK && p->heads > 0) {
        st = check_rows(p->q, p->q_row, p->q_head, p->rows, p->heads, p->head_dim, p->dtype);
        if (st == TTF_OK) st = check_rows(p->q_out, p->qo_row, p->qo_head, p->rows, p->heads, p->head_dim, p->dtype);
        if (st == TTF_OK && crossed(p->q, p->q_row, p->q_head, p->q_out, p->qo_row, p->qo_head, p->rows, p->heads)) st = TTF_ERR_INVALID_ARG;
        if (st == TTF_OK && folded(p->qo_row, p->qo_head, p->rows, p->heads, p->head_dim)) st = TTF_ERR_INVALID_ARG;
    }
    if (st == TTF_OK && p->kv_heads > 0) {
        st = check_rows(p->k, p->k_row, p->k_head, p->rows, p->kv_heads, p->head_dim, p->dtype);
        if (st == TTF_OK)
            st = append ? check_rows(p->v, p->v_row, p->v_head, p->rows, p->kv_heads, p->head_dim, p->dtype)
                        : check_rows(p->k_out, p->ko_row, p->ko_head, p->rows, p->kv_heads, p->head_dim, p->dtype);
        if (st == TTF_OK && !append && (crossed(p->k, p->k_row, p->k_head, p->k_out, p->ko_row, p->ko_head, p->rows, p->kv_heads) ||
                                        folded(p->ko_row, p->ko_head, p->rows, p->kv_heads, p->head_dim)))
            st = TTF_ERR_INVALID_ARG;
    }
    if (st == TTF_OK && (!aligned(p->q_weight) || !aligned(p->k_weight))) st = TTF_ERR_UNSUPPORTED;
    return st;
}

ttf_status check_attention(const ttf_attention_params* p)
{
    if (!p) return TTF_ERR_INVALID_ARG;
    if (!sizes_fit(p->rows, p->batch, p->heads, p->kv_heads) || p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads != 0)
        return TTF_ERR_INVALID_ARG;
    if (p->max_rows < 1 || (p->causal != 0 && p->causal != 1) || p->window < 0 || !std::isfinite(p->scale))
        return TTF_ERR_INVALID_ARG;
    return check_head(p->dtype, p->head_dim);
}

ttf_status done(hipError_t e)
{
    if (e == hipSuccess) return TTF_OK;
    set_last_hip_error(e);
    return TTF_ERR_HIP;
}

}  // namespace
}  // namespace ttf

using namespace ttf;

extern "C" {

ttf_status ttf_rope_table(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_length, double fast,
                          double slow, int32_t axes, const int32_t* sections, int32_t take_turns, double* inv_freq,
                          int32_t* axis, float* attention_factor)
{
    if (rotary_dim < 2 || rotary_dim % 2 != 0 || !(base > 1.0) || !std::isfinite(base)) return TTF_ERR_INVALID_ARG;
    if (scaling < TTF_ROPE_PLAIN || scaling > TTF_ROPE_TURNS || axes < 1 || axes > 4) return TTF_ERR_INVALID_ARG;
    if (scaling != TTF_ROPE_PLAIN && !(factor >= 1.0 && std::isfinite(factor))) return TTF_ERR_INVALID_ARG;
    const bool parts = scaling == TTF_ROPE_PARTS || scaling == TTF_ROPE_TURNS;
    if (parts && !(original_length >= 1.0 && std::isfinite(original_length) && slow > 0.0 && slow < fast && std::isfinite(fast)))
        return TTF_ERR_INVALID_ARG;
    const int half = rotary_dim / 2;
    if (sections) {
        long long sum = 0;
        for (int a = 0; a < axes; ++a) {
            if (sections[a] < 0) return TTF_ERR_INVALID_ARG;
            if (take_turns && a > 0 && sections[a] > 0 && (sections[a] - 1ll) * axes + a >= half) return TTF_ERR_INVALID_ARG;
            sum += sections[a];
        }
        if (sum != half) return TTF_ERR_INVALID_ARG;
    }
    if (scaling == TTF_ROPE_BASE && rotary_dim > 2) base *= std::pow(factor, (double)rotary_dim / (rotary_dim - 2));
    const double two_pi = 6.283185307179586477;
    // pair (not rounded) that turns n times over the original length: original_length f_j / 2 pi = n
    const auto pair_of = [&](double n) { return rotary_dim * std::log(original_length / (n * two_pi)) / (2.0 * std::log(base)); };
    double low = 0.0, high = 0.0;
    if (scaling == TTF_ROPE_PARTS) {
        low = std::fmax(std::floor(pair_of(fast)), 0.0);
        high = std::fmax(std::ceil(pair_of(slow)), 0.0);      // (beyond the last pair where that turns faster: no pair is divided whole)
    }
    for (int j = 0; j < half; ++j) {
        double f = std::pow(base, -2.0 * j / rotary_dim), g = 0.0;   // g: share that is divided
        if (scaling == TTF_ROPE_LINEAR) g = 1.0;
        else if (scaling == TTF_ROPE_PARTS) g = high > low ? std::fmin(std::fmax((j - low) / (high - low), 0.0), 1.0) : (j > low ? 1.0 : 0.0);
        else if (scaling == TTF_ROPE_TURNS)
            g = 1.0 - std::fmin(std::fmax((original_length * f / two_pi - slow) / (fast - slow), 0.0), 1.0);
        if (g > 0.0) f = f * (1.0 - g) + f / factor * g;
        if (inv_freq) inv_freq[j] = f;
        if (axis) {
            int a = 0;
            if (sections && take_turns) {
                a = j % axes;
                if (j / axes >= sections[a]) a = 0;
            } else if (sections) {
                for (int end = sections[0]; j >= end; end += sections[++a]) {}
            }
            axis[j] = a;
        }
    }
    if (attention_factor) *attention_factor = scaling == TTF_ROPE_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
    return TTF_OK;
}

ttf_status ttf_qk_norm_rope(const ttf_qk_params* params, void* hip_stream)
{
    const ttf_status st = check_qk(params, false);
    if (st != TTF_OK) return st;
    return done(launch_qk(*params, nullptr, static_cast<hipStream_t>(hip_stream)));
}

ttf_status ttf_cache_append(const ttf_qk_params* params, const ttf_kv_cache* cache, void* hip_stream)
{
    ttf_status st = check_qk(params, true);
    if (st == TTF_OK) st = check_cache(cache, params->kv_heads, params->head_dim, params->dtype);
    // (pages may share slots: which are written is the page table's to say)
    if (st == TTF_OK && folded(cache->slot_stride, cache->head_stride, cache->page_size, params->kv_heads, params->head_dim)) st = TTF_ERR_INVALID_ARG;
    if (st != TTF_OK) return st;
    return done(launch_qk(*params, cache, static_cast<hipStream_t>(hip_stream)));
}

ttf_status ttf_attention_workspace_size(const ttf_attention_params* params, size_t* bytes)
{
    if (!bytes) return TTF_ERR_INVALID_ARG;
    const ttf_status st = check_attention(params);
    if (st != TTF_OK) return st;
    *bytes = attention_workspace_bytes(*params);
    return TTF_OK;
}

ttf_status ttf_paged_attention(const ttf_attention_params* params, const ttf_kv_cache* cache, void* workspace,
                               size_t workspace_bytes, void* hip_stream)
{
    ttf_status st = check_attention(params);
    if (st != TTF_OK) return st;
    const ttf_attention_params& p = *params;
    if (!p.row_offsets || !p.cached || !workspace) return TTF_ERR_INVALID_ARG;
    st = check_rows(p.q, p.q_row, p.q_head, p.rows, p.heads, p.head_dim, p.dtype);
    if (st == TTF_OK) st = check_rows(p.out, p.o_row, p.o_head, p.rows, p.heads, p.head_dim, p.dtype);
    if (st == TTF_OK && crossed(p.q, p.q_row, p.q_head, p.out, p.o_row, p.o_head, p.rows, p.heads)) st = TTF_ERR_INVALID_ARG;
    if (st == TTF_OK && folded(p.o_row, p.o_head, p.rows, p.heads, p.head_dim)) st = TTF_ERR_INVALID_ARG;
    if (st == TTF_OK) st = check_cache(cache, p.kv_heads, p.head_dim, p.dtype);
    if (st != TTF_OK) return st;
    if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return TTF_ERR_UNSUPPORTED;
    if (workspace_bytes < attention_workspace_used(p)) return TTF_ERR_WORKSPACE_TOO_SMALL;
    return done(launch_attention(p, *cache, workspace, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
