// Host side of the cache calls of the C ABI (s2o_decode, s2o_key_weights, s2o_evict): argument validation, size
// queries and launches.  Nothing here allocates device memory or synchronises.
#include <math.h>
#include <string.h>

#include <initializer_list>

#include "../../include/s2o.h"
#include "s2o_internal.h"

namespace {

constexpr int64_t kMostRows = 1 << 30;      // of a cache, and query rows of a call: row numbers are 32-bit, with room for a block

bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// a * b * .. > limit, without overflow (factors >= 0)
bool exceeds(int64_t limit, std::initializer_list<int64_t> factors) {
  int64_t p = 1;
  for (int64_t f : factors) {
    if (f == 0) return false;
    if (p > limit / f) return true;
    p *= f;
  }
  return p > limit;
}

// Strides of a tensor of n dimensions (the last one before the D contiguous elements counts rows).  `rows`: that one is a cache's
// rows, walked with 32-bit offsets.  `out`: written to, so that two rows must not overlap.
int fill_strides(const int64_t* in, int64_t* st, const int64_t* size, int n, int D, bool rows, bool out) {
  bool packed = true;
  for (int i = 0; i < n; ++i) packed &= in[i] == 0;
  if (packed) {
    int64_t s = D;
    for (int i = n - 1; i >= 0; --i) {
      st[i] = s;
      if (s > (INT64_MAX >> 4) / (size[i] > 0 ? size[i] : 1)) return S2O_EUNSUPPORTED;
      s *= size[i];
    }
    return S2O_OK;
  }
  for (int i = 0; i < n; ++i) {
    if (size[i] <= 1) { st[i] = 0; continue; }
    if (in[i] < 0 || in[i] % 8 != 0) return S2O_EINVAL;    // 16-byte aligned rows
    if (in[i] > (INT64_MAX >> 4) / size[i]) return S2O_EINVAL;
    st[i] = in[i];
  }
  if (rows && size[n - 1] > 1) {
    if (st[n - 1] < D) return S2O_EINVAL;
    if (st[n - 1] >= (1 << 23)) return S2O_EUNSUPPORTED;
  }
  if (out) {                                               // each stride steps over all that the smaller ones reach
    int order[4];
    for (int i = 0; i < n; ++i) order[i] = i;
    for (int i = 0; i < n; ++i)
      for (int j = i + 1; j < n; ++j)
        if (st[order[j]] < st[order[i]]) { const int t = order[i]; order[i] = order[j]; order[j] = t; }
    int64_t reach = D;
    for (int i = 0; i < n; ++i) {
      if (size[order[i]] <= 1) continue;
      if (st[order[i]] < reach) return S2O_EINVAL;
      reach += st[order[i]] * (size[order[i]] - 1);
    }
  }
  return S2O_OK;
}

// Bytes from a tensor's first element to behind its last.
size_t span(const int64_t* st, const int64_t* size, int n, int D) {
  int64_t e = D;
  for (int i = 0; i < n; ++i) e += st[i] * (size[i] - 1);
  return (size_t)e * 2;
}

struct Range {
  const void* p;
  size_t bytes;
  bool meets(const Range& o) const {
    return p && o.p && bytes && o.bytes && (uintptr_t)p < (uintptr_t)o.p + o.bytes && (uintptr_t)o.p < (uintptr_t)p + bytes;
  }
};

// What is written to overlaps nothing that is read and nothing else that is written.
int check_apart(std::initializer_list<Range> outs, std::initializer_list<Range> ins) {
  for (const Range& o : outs) {
    for (const Range& i : ins) if (o.meets(i)) return S2O_EINVAL;
    for (const Range& p : outs) if (&p != &o && o.meets(p)) return S2O_EINVAL;
  }
  return S2O_OK;
}

int check_heads(int Z, int B, int H, int Hkv, int D, int T, int dtype, float scale) {
  if (Z <= 0 || B <= 0 || H <= 0 || Hkv <= 0 || D <= 0 || T <= 0) return S2O_EINVAL;
  if (H % Hkv != 0) return S2O_EINVAL;
  if (dtype != S2O_BF16 && dtype != S2O_F16) return S2O_EINVAL;
  if (!(scale >= 0.f) || isinf(scale)) return S2O_EINVAL;
  if (D != 64 && D != 128) return S2O_EUNSUPPORTED;
  if (exceeds(kMostRows, {Z, B, H, T})) return S2O_EUNSUPPORTED;
  if (exceeds(1 << 24, {Z, Hkv})) return S2O_EUNSUPPORTED;
  return S2O_OK;
}

float scale_of(float given, int D) { return given > 0.f ? given : 1.0f / sqrtf((float)D); }

#define CHECK(expr) do { const int rc_ = (expr); if (rc_ != S2O_OK) return rc_; } while (0)

int decode_args(const s2o_decode_params* p, s2o::DecodeArgs* a) {
  if (!p || p->struct_size != (int32_t)sizeof(s2o_decode_params) || p->reserved != 0) return S2O_EINVAL;
  CHECK(check_heads(p->batch, p->branches, p->q_heads, p->kv_heads, p->head_dim, p->q_len, p->dtype, p->softmax_scale));
  if (p->cache_len < 0 || p->own_len < 0 || (p->cache_len == 0 && p->own_len == 0)) return S2O_EINVAL;
  if (p->cache_len > kMostRows || p->own_len > kMostRows) return S2O_EUNSUPPORTED;
  memset(a, 0, sizeof(*a));
  a->Z = p->batch; a->B = p->branches; a->H = p->q_heads; a->Hkv = p->kv_heads; a->G = p->q_heads / p->kv_heads;
  a->D = p->head_dim; a->T = p->q_len; a->L = p->cache_len; a->Lo = p->own_len; a->f16 = p->dtype == S2O_F16;
  const int64_t q[4] = {a->Z, a->B, a->H, a->T}, k[3] = {a->Z, a->Hkv, a->L}, o[4] = {a->Z, a->B, a->Hkv, a->Lo};
  CHECK(fill_strides(p->q_stride, a->qs, q, 4, a->D, false, false));
  CHECK(fill_strides(p->o_stride, a->os, q, 4, a->D, false, true));
  if (a->L) {
    CHECK(fill_strides(p->k_stride, a->ks, k, 3, a->D, true, false));
    CHECK(fill_strides(p->v_stride, a->vs, k, 3, a->D, true, false));
  }
  if (a->Lo) {
    CHECK(fill_strides(p->own_k_stride, a->oks, o, 4, a->D, true, false));
    CHECK(fill_strides(p->own_v_stride, a->ovs, o, 4, a->D, true, false));
  }
  a->c2 = scale_of(p->softmax_scale, a->D) * 1.4426950408889634f;
  return S2O_OK;
}

int weights_args(const s2o_weights_params* p, s2o::WeightsArgs* a) {
  if (!p || p->struct_size != (int32_t)sizeof(s2o_weights_params) || p->reserved != 0) return S2O_EINVAL;
  CHECK(check_heads(p->batch, p->branches, p->q_heads, p->kv_heads, p->head_dim, p->q_len, p->dtype, p->softmax_scale));
  if (p->cache_len <= 0 || (p->causal != 0 && p->causal != 1)) return S2O_EINVAL;
  if (p->cache_len > kMostRows || exceeds(1ll << 37, {p->batch, p->kv_heads, p->cache_len})) return S2O_EUNSUPPORTED;
  memset(a, 0, sizeof(*a));
  a->Z = p->batch; a->B = p->branches; a->H = p->q_heads; a->Hkv = p->kv_heads; a->G = p->q_heads / p->kv_heads;
  a->D = p->head_dim; a->T = p->q_len; a->L = p->cache_len; a->f16 = p->dtype == S2O_F16; a->causal = p->causal;
  const int64_t q[4] = {a->Z, a->B, a->H, a->T}, k[3] = {a->Z, a->Hkv, a->L};
  CHECK(fill_strides(p->q_stride, a->qs, q, 4, a->D, false, false));
  CHECK(fill_strides(p->k_stride, a->ks, k, 3, a->D, true, false));
  const float scale = scale_of(p->softmax_scale, a->D);
  a->c2 = scale * 1.4426950408889634f;
  const double unit = (double)a->c2 / (double)scale;
  a->l2e_hi = (float)unit;
  a->l2e_lo = (float)(unit - (double)a->l2e_hi);
  return S2O_OK;
}

int evict_args(const s2o_evict_params* p, s2o::EvictArgs* a) {
  if (!p || p->struct_size != (int32_t)sizeof(s2o_evict_params) || p->reserved != 0) return S2O_EINVAL;
  CHECK(check_heads(p->batch, 1, p->kv_heads, p->kv_heads, p->head_dim, 1, p->dtype, 0.f));
  if (p->cache_len <= 0 || p->keep <= 0 || p->keep > p->cache_len || p->sink < 0 || p->recent < 0 ||
      (int64_t)p->sink + p->recent > p->keep)
    return S2O_EINVAL;
  if (p->cache_len > kMostRows || exceeds(1ll << 34, {p->batch, p->kv_heads, p->keep})) return S2O_EUNSUPPORTED;
  memset(a, 0, sizeof(*a));
  a->Z = p->batch; a->Hkv = p->kv_heads; a->D = p->head_dim; a->L = p->cache_len;
  a->keep = p->keep; a->sink = p->sink; a->recent = p->recent;
  const int64_t in[3] = {a->Z, a->Hkv, a->L}, out[3] = {a->Z, a->Hkv, a->keep};
  CHECK(fill_strides(p->k_stride, a->ks, in, 3, a->D, true, false));
  CHECK(fill_strides(p->v_stride, a->vs, in, 3, a->D, true, false));
  CHECK(fill_strides(p->out_k_stride, a->kos, out, 3, a->D, true, true));
  CHECK(fill_strides(p->out_v_stride, a->vos, out, 3, a->D, true, true));
  return S2O_OK;
}

int check_scratch(const void* scratch, size_t bytes, size_t need) {
  if (need == 0) return S2O_OK;
  return !scratch || misaligned(scratch, 256) || bytes < need ? S2O_ESCRATCH : S2O_OK;
}

// (Not supported: sizes whose launch would not fit, found before anything was launched.)
int done(hipError_t e) { return e == hipSuccess ? S2O_OK : e == hipErrorNotSupported ? S2O_EUNSUPPORTED : s2o::hip_fail(e); }

}  // namespace

extern "C" {

int s2o_decode_sizes(const s2o_decode_params* params, size_t* lse_bytes, size_t* scratch_bytes) {
  s2o::DecodeArgs a;
  CHECK(decode_args(params, &a));
  if (lse_bytes) *lse_bytes = (size_t)a.Z * a.B * a.H * a.T * 4;
  if (scratch_bytes) *scratch_bytes = s2o::decode_scratch_bytes(a);
  return S2O_OK;
}

int s2o_decode(const void* Q, const void* K, const void* V, const void* own_K, const void* own_V, const int32_t* lens,
               const int32_t* own_lens, const s2o_decode_params* params, void* O, float* lse, void* scratch, size_t scratch_bytes,
               void* stream) {
  s2o::DecodeArgs a;
  CHECK(decode_args(params, &a));
  if (!Q || !O || (a.L && (!K || !V)) || (a.Lo && (!own_K || !own_V))) return S2O_EINVAL;
  if (misaligned(Q, 16) || misaligned(O, 16) || misaligned(lse, 4) || misaligned(lens, 4) || misaligned(own_lens, 4)) return S2O_EINVAL;
  if ((a.L && (misaligned(K, 16) || misaligned(V, 16))) || (a.Lo && (misaligned(own_K, 16) || misaligned(own_V, 16)))) return S2O_EINVAL;
  const size_t need = s2o::decode_scratch_bytes(a);
  CHECK(check_scratch(scratch, scratch_bytes, need));
  const int64_t q[4] = {a.Z, a.B, a.H, a.T}, k[3] = {a.Z, a.Hkv, a.L}, o[4] = {a.Z, a.B, a.Hkv, a.Lo};
  const size_t kb = a.L ? 1 : 0, ob = a.Lo ? 1 : 0, seqs = (size_t)a.Z * a.B;
  CHECK(check_apart({{O, span(a.os, q, 4, a.D)}, {lse, seqs * a.H * a.T * 4}, {scratch, need}},
                    {{Q, span(a.qs, q, 4, a.D)}, {K, kb * span(a.ks, k, 3, a.D)}, {V, kb * span(a.vs, k, 3, a.D)}, {own_K, ob * span(a.oks, o, 4, a.D)},
                     {own_V, ob * span(a.ovs, o, 4, a.D)}, {lens, (size_t)a.Z * 4}, {own_lens, seqs * 4}}));
  a.Q = Q; a.K = K; a.V = V; a.oK = own_K; a.oV = own_V;
  a.lens = lens; a.own_lens = own_lens; a.O = O; a.lse = lse;
  return done(s2o::launch_decode(a, scratch, (hipStream_t)stream));
}

int s2o_key_weights_sizes(const s2o_weights_params* params, int with_lse, size_t* weights_bytes, size_t* scratch_bytes) {
  s2o::WeightsArgs a;
  CHECK(weights_args(params, &a));
  if (weights_bytes) *weights_bytes = (size_t)a.Z * a.Hkv * a.L * 4;
  if (scratch_bytes) *scratch_bytes = s2o::weights_scratch_bytes(a, with_lse != 0);
  return S2O_OK;
}

int s2o_key_weights(const void* Q, const void* K, const float* lse, const int32_t* lens, const s2o_weights_params* params, const float* prev,
                    float* weights, void* scratch, size_t scratch_bytes, void* stream) {
  s2o::WeightsArgs a;
  CHECK(weights_args(params, &a));
  if (!Q || !K || !weights) return S2O_EINVAL;
  if (misaligned(Q, 16) || misaligned(K, 16) || misaligned(lse, 4) || misaligned(lens, 4) || misaligned(prev, 4) || misaligned(weights, 4))
    return S2O_EINVAL;
  const size_t bytes = (size_t)a.Z * a.Hkv * a.L * 4;
  if (prev != weights && Range{prev, bytes}.meets({weights, bytes})) return S2O_EINVAL;
  const size_t need = s2o::weights_scratch_bytes(a, lse != nullptr);
  CHECK(check_scratch(scratch, scratch_bytes, need));
  const int64_t q[4] = {a.Z, a.B, a.H, a.T}, k[3] = {a.Z, a.Hkv, a.L};
  CHECK(check_apart({{weights, bytes}, {scratch, need}},
                    {{Q, span(a.qs, q, 4, a.D)}, {K, span(a.ks, k, 3, a.D)}, {lse, (size_t)a.Z * a.B * a.H * a.T * 4}, {lens, (size_t)a.Z * 4}}));
  CHECK(check_apart({{scratch, need}}, {{prev, bytes}}));
  a.Q = Q; a.K = K; a.lse = lse; a.lens = lens; a.prev = prev; a.out = weights;
  return done(s2o::launch_weights(a, scratch, (hipStream_t)stream));
}

int s2o_evict_sizes(const s2o_evict_params* params, size_t* scratch_bytes) {
  s2o::EvictArgs a;
  CHECK(evict_args(params, &a));
  if (scratch_bytes) *scratch_bytes = s2o::evict_scratch_bytes(a);
  return S2O_OK;
}

int s2o_evict(const void* K, const void* V, const float* weights, const int32_t* lens, const s2o_evict_params* params, void* K_out,
              void* V_out, float* weights_out, int32_t* kept, int32_t* lens_out, void* scratch, size_t scratch_bytes, void* stream) {
  s2o::EvictArgs a;
  CHECK(evict_args(params, &a));
  if (!weights || !kept || !K != !K_out || !V != !V_out) return S2O_EINVAL;
  if (misaligned(K, 16) || misaligned(V, 16) || misaligned(K_out, 16) || misaligned(V_out, 16)) return S2O_EINVAL;
  if (misaligned(weights, 4) || misaligned(lens, 4) || misaligned(weights_out, 4) || misaligned(kept, 4) || misaligned(lens_out, 4)) return S2O_EINVAL;
  const int64_t in[3] = {a.Z, a.Hkv, a.L}, out[3] = {a.Z, a.Hkv, a.keep};
  const size_t heads = (size_t)a.Z * a.Hkv, need = s2o::evict_scratch_bytes(a);
  CHECK(check_apart({{K_out, span(a.kos, out, 3, a.D)}, {V_out, span(a.vos, out, 3, a.D)}, {weights_out, heads * a.keep * 4}, {kept, heads * a.keep * 4},
                     {lens_out, (size_t)a.Z * 4}, {scratch, need}},
                    {{K, span(a.ks, in, 3, a.D)}, {V, span(a.vs, in, 3, a.D)}, {weights, heads * a.L * 4}, {lens, (size_t)a.Z * 4}}));
  CHECK(check_scratch(scratch, scratch_bytes, need));
  a.K = K; a.V = V; a.weights = weights; a.lens = lens;
  a.K_out = K_out; a.V_out = V_out; a.weights_out = weights_out; a.kept = kept; a.lens_out = lens_out;
  return done(s2o::launch_evict(a, scratch, (hipStream_t)stream));
}

}  // extern "C"
