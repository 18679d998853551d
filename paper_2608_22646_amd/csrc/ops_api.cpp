// C ABI of the stand-alone operators (see include/dllm.h): argument checks and
// launches of rotary positions, attention over documents and behind shared prompts,
// sampling, and adapters.
#include <math.h>

#include "api.h"
#include "kernels.h"

using namespace dllm;

namespace {

void check_dtype(int dtype) {
  require(dtype == DLLM_F32 || dtype == DLLM_BF16, DLLM_EINVAL, "dtype must be DLLM_F32 or DLLM_BF16");
}

// A view that is used: data there, strides not negative.
void check_view(const dllm_view* v, const char* name) {
  require(v != nullptr && v->data != nullptr, DLLM_EINVAL, std::string(name) + " is NULL");
  require(v->stride_b >= 0 && v->stride_l >= 0 && v->stride_h >= 0, DLLM_ESHAPE,
          std::string(name) + " has a negative stride");
}

RotaryRows rows_of(const dllm_view* v) { return RotaryRows{v->data, v->stride_b, v->stride_l, v->stride_h}; }

void check_rotary(const dllm_rotary_cfg* c) {
  require(c != nullptr, DLLM_EINVAL, "cfg is NULL");
  require(c->head_dim >= 2 && c->head_dim <= 512, DLLM_ESHAPE, "head_dim must be in [2, 512]");
  require(c->rot_dim >= 2 && c->rot_dim % 2 == 0 && c->rot_dim <= c->head_dim && c->rot_dim <= 256, DLLM_ESHAPE,
          "rot_dim must be even and in [2, min(head_dim, 256)]");
  require(std::isfinite(c->base) && c->base > 0, DLLM_EINVAL, "base must be positive");
  require(std::isfinite((float)c->gain), DLLM_EINVAL, "gain must be a finite float32");
  require(c->scaling >= DLLM_ROPE_PLAIN && c->scaling <= DLLM_ROPE_PARTS, DLLM_EINVAL, "unknown scaling");
  if (c->scaling != DLLM_ROPE_PLAIN)
    require(std::isfinite(c->factor) && c->factor > 0, DLLM_EINVAL, "factor must be positive");
  if (c->scaling == DLLM_ROPE_PARTS) {
    require(std::isfinite(c->orig_len) && c->orig_len > 0, DLLM_EINVAL, "orig_len must be positive");
    require(std::isfinite(c->low) && std::isfinite(c->high) && c->high > c->low, DLLM_EINVAL,
            "high must be greater than low");
  }
}

// 16-byte pieces everywhere: the address and every stride in bytes.
void check_attn_view(const dllm_view& v, int size, int hd, int64_t batches, const char* name) {
  check_view(&v, name);
  require(((uintptr_t)v.data & 15) == 0 && (v.stride_l * size) % 16 == 0 && (v.stride_h * size) % 16 == 0 &&
              (batches <= 1 || (v.stride_b * size) % 16 == 0),
          DLLM_EUNSUPPORTED, std::string(name) + ": data and strides must be multiples of 16 bytes");
  require(v.stride_l >= hd, DLLM_ESHAPE, std::string(name) + ": stride_l must be at least head_dim");
}

// The sizes of an attention call; false where there is nothing to do.
bool attn_args(const dllm_attn_args* p, AttnArgs* a) {
  require(p != nullptr, DLLM_EINVAL, "args is NULL");
  check_dtype(p->dtype);
  require(p->head_dim == 64 || p->head_dim == 128, DLLM_EUNSUPPORTED, "head_dim must be 64 or 128");
  require(p->n_heads >= 1 && p->n_kv_heads >= 1 && p->n_heads % p->n_kv_heads == 0 && p->n_heads <= 4096, DLLM_ESHAPE,
          "n_heads must be a multiple of n_kv_heads and at most 4096");
  require(p->docs >= 0 && p->docs <= 65535, DLLM_ESHAPE, "docs must be in [0, 65535]");
  require(p->max_q >= 0 && p->max_q <= p->q_tokens && p->max_kv >= 0 && p->max_kv <= p->kv_tokens, DLLM_ESHAPE,
          "max_q and max_kv must be in [0, q_tokens] and [0, kv_tokens]");
  require(p->q_tokens <= (1 << 30) && p->kv_tokens <= (1 << 30), DLLM_ESHAPE, "a slab holds at most 2^30 tokens");
  require((int64_t)p->max_q * (p->n_heads / p->n_kv_heads) <= 0x7fffff00, DLLM_ESHAPE, "too many query rows");
  require(std::isfinite(p->scale), DLLM_EINVAL, "scale must be finite");
  require(std::isfinite(p->cap) && p->cap >= 0, DLLM_EINVAL, "cap must be finite and not negative");
  require(p->block >= 0, DLLM_EINVAL, "block must not be negative");
  a->dtype = p->dtype;
  a->Hq = p->n_heads;
  a->Hkv = p->n_kv_heads;
  a->hd = p->head_dim;
  a->docs = p->docs;
  a->q_tokens = p->q_tokens;
  a->kv_tokens = p->kv_tokens;
  a->max_q = p->max_q;
  a->max_kv = p->max_kv;
  a->block = p->block;
  a->scale = p->scale;
  a->cap = p->cap;
  require(attn_docs_fits(*a), DLLM_ESHAPE, "too many documents, heads and queries for one call");
  return p->docs > 0 && p->max_q > 0;
}

AttnView attn_view(const dllm_view& v) { return AttnView{v.data, v.stride_b, v.stride_l, v.stride_h}; }

// The operands of an attention call.
void attn_operands(const dllm_attn_args* p, AttnArgs* out) {
  AttnArgs& a = *out;
  const int size = p->dtype == DLLM_F32 ? 4 : 2;
  check_attn_view(p->q, size, p->head_dim, p->docs, "q");
  check_attn_view(p->out, size, p->head_dim, p->docs, "out");
  if (p->max_kv > 0) {
    check_attn_view(p->k, size, p->head_dim, p->docs, "k");
    check_attn_view(p->v, size, p->head_dim, p->docs, "v");
    require(p->k.stride_l * size < (1 << 25) && p->v.stride_l * size < (1 << 25), DLLM_ESHAPE,
            "64 stride_l of k and v must be below 2^31 bytes");
  }
  a.q = attn_view(p->q);
  a.k = attn_view(p->k);
  a.v = attn_view(p->v);
  a.out = attn_view(p->out);
  a.q_start = p->q_start;
  a.q_len = p->q_len;
  a.kv_start = p->kv_start;
  a.kv_len = p->kv_len;
  a.q_pos = p->q_pos;
  a.prefix = p->prefix;
  a.slopes = p->slopes;
}

// The sizes of a call behind shared prompts; false where there is nothing to do.
bool shared_args(const dllm_shared_attn_args* p, SharedArgs* s) {
  require(p != nullptr, DLLM_EINVAL, "args is NULL");
  const bool some = attn_args(&p->own, &s->own);
  require(p->prompts >= 0 && p->prompts <= 65535, DLLM_ESHAPE, "prompts must be in [0, 65535]");
  require(p->max_p >= 0 && p->max_p <= p->p_tokens && p->p_tokens <= (1 << 29), DLLM_ESHAPE,
          "max_p must be in [0, p_tokens], p_tokens at most 2^29");
  require(p->own.kv_tokens <= (1 << 29), DLLM_ESHAPE, "kv_tokens must be at most 2^29");
  s->own.out.stride_b = p->own.out.stride_b;
  s->prompts = p->prompts;
  s->p_tokens = p->p_tokens;
  s->max_p = p->max_p;
  s->p_start = p->p_start;
  s->p_len = p->p_len;
  s->prompt = p->prompt;
  require(!some || attn_shared_fits(*s), DLLM_ESHAPE, "too many documents, heads and queries for one call");
  return some;
}

void check_workspace(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return;
  require(ws != nullptr, DLLM_EINVAL, "workspace is NULL");
  require(((uintptr_t)ws & 255) == 0, DLLM_EINVAL, "workspace must be 256-byte aligned");
  require(bytes >= need, DLLM_ENOMEM, "workspace too small: need " + std::to_string(need) + " bytes");
}

void check_sample_sizes(int rows, int vocab) {
  require(rows >= 0 && vocab >= 1 && vocab <= (1 << 22), DLLM_ESHAPE, "rows must be >= 0 and vocab in [1, 2^22]");
  require(sample_fits(rows, vocab), DLLM_ESHAPE, "too many rows of this vocabulary for one call");
}

// The sizes of an adapters call; false where there is nothing to do.
bool adapter_sizes(const dllm_adapter_args* p, AdaptersArgs* a) {
  require(p != nullptr, DLLM_EINVAL, "args is NULL");
  check_dtype(p->dtype);
  require(p->out_dtype == DLLM_F32 || p->out_dtype == p->dtype, DLLM_EINVAL, "out_dtype must be DLLM_F32 or dtype");
  require(p->rows >= 0 && p->rows <= (1 << 22), DLLM_ESHAPE, "rows must be in [0, 2^22]");
  require(p->d_in >= 1 && p->d_in <= (1 << 20) && p->d_out >= 1 && p->d_out <= (1 << 20), DLLM_ESHAPE,
          "d_in and d_out must be in [1, 2^20]");
  require(p->adapters >= 0 && p->adapters <= 4095, DLLM_ESHAPE, "adapters must be in [0, 4095]");
  require(p->rank >= 1 && p->rank <= 256, DLLM_ESHAPE, "rank must be in [1, 256]");
  require(p->slices >= 1 && p->slices <= DLLM_ADAPTER_SLICES, DLLM_ESHAPE, "slices must be in [1, DLLM_ADAPTER_SLICES]");
  for (int s = 0; s < p->slices; ++s)
    require(p->slice_end[s] > (s ? p->slice_end[s - 1] : 0) && (s + 1 < p->slices || p->slice_end[s] == p->d_out), DLLM_ESHAPE,
            "slice_end must rise from above 0 and end at d_out");
  a->dtype = p->dtype;
  a->out_dtype = p->out_dtype;
  a->rows = p->rows;
  a->d_in = p->d_in;
  a->d_out = p->d_out;
  a->adapters = p->adapters;
  a->rank = p->rank;
  a->slices = p->slices;
  for (int s = 0; s < p->slices; ++s) a->slice_end[s] = p->slice_end[s];
  require(p->rows == 0 || adapters_fit(*a), DLLM_ESHAPE, "too many rows and columns for one call");
  return p->rows > 0;
}

}  // namespace

extern "C" {

int dllm_rotary(const dllm_rotary_cfg* cfg, int32_t dtype, int32_t B, int32_t L, const int32_t* pos, int32_t pos0,
                const dllm_view* q, const dllm_view* q_out, int32_t n_q, const dllm_view* k, const dllm_view* k_out,
                int32_t n_k, int32_t inverse, void* stream) {
  API_BEGIN
  check_rotary(cfg);
  check_dtype(dtype);
  const bool keys = k != nullptr || k_out != nullptr;
  require(B >= 0 && L >= 0 && n_q >= 0 && (!keys || n_k >= 0), DLLM_ESHAPE, "sizes must not be negative");
  RotaryArgs a{};
  a.n_q = n_q;
  a.n_k = keys ? n_k : 0;
  require(a.n_q <= 4096 && a.n_k <= 4096, DLLM_ESHAPE, "at most 4096 heads");
  if (B == 0 || L == 0 || a.n_q + a.n_k == 0) return DLLM_OK;
  require((int64_t)B * L <= 0x7fffffff, DLLM_ESHAPE, "B * L must be below 2^31");
  if (a.n_q > 0) {
    check_view(q, "q");
    check_view(q_out, "q_out");
    a.q = rows_of(q);
    a.q_out = rows_of(q_out);
  }
  if (a.n_k > 0) {
    check_view(k, "k");
    check_view(k_out, "k_out");
    a.k = rows_of(k);
    a.k_out = rows_of(k_out);
  }
  a.dtype = dtype;
  a.B = B;
  a.L = L;
  a.hd = cfg->head_dim;
  a.rot = cfg->rot_dim;
  a.inter = cfg->interleaved != 0;
  a.scaling = cfg->scaling;
  a.inverse = inverse != 0;
  a.pos = pos;
  a.pos0 = pos0;
  a.log2_base = log2(cfg->base);
  a.factor = cfg->factor;
  a.orig_len = cfg->orig_len;
  a.low = cfg->low;
  a.high = cfg->high;
  a.gain = (float)cfg->gain;
  launch_rotary(a, (hipStream_t)stream);
  API_END
}

int dllm_attention_workspace_size(const dllm_attn_args* p, size_t* bytes) {
  API_BEGIN
  require(bytes != nullptr, DLLM_EINVAL, "bytes is NULL");
  AttnArgs a{};
  *bytes = attn_args(p, &a) ? attn_docs_bytes(a) : 0;
  API_END
}

int dllm_attention(const dllm_attn_args* p, void* ws, size_t ws_bytes, void* stream) {
  API_BEGIN
  AttnArgs a{};
  if (!attn_args(p, &a)) return DLLM_OK;
  attn_operands(p, &a);
  check_workspace(ws, ws_bytes, attn_docs_bytes(a));
  launch_attn_docs(a, ws, (hipStream_t)stream);
  API_END
}

int dllm_shared_attention_workspace_size(const dllm_shared_attn_args* p, size_t* bytes) {
  API_BEGIN
  require(bytes != nullptr, DLLM_EINVAL, "bytes is NULL");
  SharedArgs s{};
  *bytes = shared_args(p, &s) ? attn_shared_bytes(s) : 0;
  API_END
}

int dllm_shared_attention(const dllm_shared_attn_args* p, void* ws, size_t ws_bytes, void* stream) {
  API_BEGIN
  SharedArgs s{};
  if (!shared_args(p, &s)) return DLLM_OK;
  attn_operands(&p->own, &s.own);
  if (p->prompts > 0 && p->max_p > 0) {
    const int size = p->own.dtype == DLLM_F32 ? 4 : 2;
    check_attn_view(p->pk, size, p->own.head_dim, p->prompts, "pk");
    check_attn_view(p->pv, size, p->own.head_dim, p->prompts, "pv");
    require(p->pk.stride_l * size < (1 << 25) && p->pv.stride_l * size < (1 << 25), DLLM_ESHAPE,
            "64 stride_l of pk and pv must be below 2^31 bytes");
    s.pk = attn_view(p->pk);
    s.pv = attn_view(p->pv);
  }
  check_workspace(ws, ws_bytes, attn_shared_bytes(s));
  launch_attn_shared(s, ws, (hipStream_t)stream);
  API_END
}

int dllm_sample_workspace_size(int32_t rows, int32_t vocab, size_t* bytes) {
  API_BEGIN
  require(bytes != nullptr, DLLM_EINVAL, "bytes is NULL");
  check_sample_sizes(rows, vocab);
  *bytes = sample_bytes(rows, vocab);
  API_END
}

int dllm_sample(const dllm_sample_args* p, void* ws, size_t ws_bytes, void* stream) {
  API_BEGIN
  require(p != nullptr, DLLM_EINVAL, "args is NULL");
  check_dtype(p->dtype);
  check_sample_sizes(p->rows, p->vocab);
  if (p->rows == 0) return DLLM_OK;
  require(p->logits && p->u && p->token, DLLM_EINVAL, "logits, u or token is NULL");
  require(p->rows == 1 || p->row_stride >= p->vocab, DLLM_ESHAPE, "row_stride must be at least vocab");
  SampleArgs a{};
  a.logits = p->logits;
  a.row_stride = p->rows == 1 ? 0 : p->row_stride;
  a.dtype = p->dtype;
  a.rows = p->rows;
  a.vocab = p->vocab;
  a.mask_id = p->mask_id;
  a.u = p->u;
  a.temperature = p->temperature;
  a.top_k = p->top_k;
  a.top_p = p->top_p;
  a.min_p = p->min_p;
  a.token = p->token;
  a.conf = p->conf;
  a.prob = p->prob;
  check_workspace(ws, ws_bytes, sample_bytes(p->rows, p->vocab));
  launch_sample(a, ws, (hipStream_t)stream);
  API_END
}

int dllm_adapters_workspace_size(const dllm_adapter_args* p, size_t* bytes) {
  API_BEGIN
  require(bytes != nullptr, DLLM_EINVAL, "bytes is NULL");
  AdaptersArgs a{};
  *bytes = adapter_sizes(p, &a) ? adapters_bytes(a) : 0;
  API_END
}

int dllm_adapters(const dllm_adapter_args* p, void* ws, size_t ws_bytes, void* stream) {
  API_BEGIN
  AdaptersArgs a{};
  if (!adapter_sizes(p, &a)) return DLLM_OK;
  check_view(&p->out, "out");
  require(p->which != nullptr, DLLM_EINVAL, "which is NULL");
  require(p->rows == 1 || p->out.stride_l >= p->d_out, DLLM_ESHAPE, "stride_l of out must be at least d_out");
  if (p->base.data) check_view(&p->base, "base");
  if (p->adapters > 0) {
    check_view(&p->x, "x");
    check_view(&p->a, "a");
    check_view(&p->b, "b");
  }
  // strides that no element steps over, or that are not named, say nothing
  auto used = [&](const dllm_view& v, bool b, bool l, bool h) { return AttnView{v.data, b ? v.stride_b : 0, l ? v.stride_l : 0, h ? v.stride_h : 0}; };
  a.x = used(p->x, false, p->rows > 1, false);
  a.a = used(p->a, p->adapters > 1, p->rank > 1, p->slices > 1);
  a.b = used(p->b, p->adapters > 1, p->d_out > 1, false);
  a.base = used(p->base, false, p->rows > 1, false);
  a.out = used(p->out, false, p->rows > 1, false);
  require(a.base.data != a.out.data || a.base.stride_l == a.out.stride_l, DLLM_ESHAPE, "out that is base must have its stride");
  a.which = p->which;
  a.ranks = p->ranks;
  a.scales = p->scales;
  check_workspace(ws, ws_bytes, adapters_bytes(a));
  launch_adapters(a, ws, (hipStream_t)stream);
  API_END
}

}  // extern "C"
