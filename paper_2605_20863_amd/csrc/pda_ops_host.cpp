// Host side of include/pda_ops.h: argument checks (host code only, before any
// HIP call), the split of the work, and the launches.

#include "pda_ops.h"
#include "pda_host.h"
#include "pda_ops_internal.h"

#include <cmath>
#include <initializer_list>
#include <new>

namespace {

using pda::host_fail;

constexpr int64_t kMaxWaves = 1 << 26;  // a launch has below 2^32 threads
constexpr int64_t kHeader = 256;        // bytes of the workspace's header
static_assert(pda::kHdrWords * 4 <= kHeader, "header");

struct Ptr {
  const void* p;
  uintptr_t align;
  const char* name;
  bool required;
};

int check_pointers(std::initializer_list<Ptr> ptrs) {
  for (const Ptr& x : ptrs) {
    if (x.required && !x.p) return host_fail(PDA_EINVAL, "%s is NULL", x.name);
    if (reinterpret_cast<uintptr_t>(x.p) % x.align)
      return host_fail(PDA_EINVAL, "%s is not %d-byte aligned", x.name, (int)x.align);
  }
  return PDA_OK;
}

bool float_type(int t) { return t == PDA_DTYPE_F32 || t == PDA_DTYPE_BF16; }
int size_of(int t) { return t == PDA_DTYPE_F32 ? 4 : 2; }

// *out: the stride in elements; rows of `heads` heads must not overlap and stay 16-byte aligned.
int check_stride(const char* name, int64_t stride, int heads, int d, int type, int64_t tokens, int64_t* out) {
  const int64_t row = (int64_t)heads * d;
  if (stride == 0) stride = row;
  if (stride < row) return host_fail(PDA_EINVAL, "%s = %lld is less than a token's %lld elements", name, (long long)stride, (long long)row);
  if (stride > INT64_MAX / 8 / (tokens + 1)) return host_fail(PDA_EINVAL, "%s = %lld is too large", name, (long long)stride);
  if (stride * size_of(type) % 16) return host_fail(PDA_EINVAL, "%s = %lld elements is not a multiple of 16 bytes", name, (long long)stride);
  *out = stride;
  return PDA_OK;
}

int check_rope(const pdaops_rope_problem* pr, bool has_q_weight, bool has_k_weight, bool with_v, pda::RopeArgs* a) {
  if (!pr) return host_fail(PDA_EINVAL, "problem is NULL");
  if (pr->num_tokens < 0) return host_fail(PDA_EINVAL, "num_tokens = %d < 0", pr->num_tokens);
  if (pr->num_q_heads < 1 || pr->num_kv_heads < 1)
    return host_fail(PDA_EINVAL, "num_q_heads = %d and num_kv_heads = %d must be >= 1", pr->num_q_heads, pr->num_kv_heads);
  if (pr->num_q_heads > 65536 || pr->num_kv_heads > 65536)
    return host_fail(PDA_EINVAL, "num_q_heads = %d and num_kv_heads = %d must be <= 65536", pr->num_q_heads, pr->num_kv_heads);
  if (pr->head_dim != 64 && pr->head_dim != 128)
    return host_fail(PDA_EUNSUPPORTED, "head_dim = %d (supported: 64, 128)", pr->head_dim);
  if (pr->rotary_dim < 2 || pr->rotary_dim > pr->head_dim)
    return host_fail(PDA_EINVAL, "rotary_dim = %d (2 .. head_dim)", pr->rotary_dim);
  if (pr->rotary_dim % 16) return host_fail(PDA_EUNSUPPORTED, "rotary_dim = %d (supported: multiples of 16)", pr->rotary_dim);
  if (pr->max_positions < 1) return host_fail(PDA_EINVAL, "max_positions = %d < 1", pr->max_positions);
  if (pr->interleaved != 0 && pr->interleaved != 1) return host_fail(PDA_EINVAL, "interleaved = %d (0 or 1)", pr->interleaved);
  if (!float_type(pr->dtype)) return host_fail(PDA_EINVAL, "dtype = %d (supported: F32, BF16)", pr->dtype);
  if (!float_type(pr->out_dtype)) return host_fail(PDA_EINVAL, "out_dtype = %d (supported: F32, BF16)", pr->out_dtype);
  if (!float_type(pr->weight_dtype)) return host_fail(PDA_EINVAL, "weight_dtype = %d (supported: F32, BF16)", pr->weight_dtype);
  if (!(pr->eps >= 0.f) || !std::isfinite(pr->eps)) return host_fail(PDA_EINVAL, "eps is negative or not finite");
  if (has_q_weight != has_k_weight) return host_fail(PDA_EINVAL, "q_weight and k_weight are given both or neither");
  const int64_t T = pr->num_tokens;
  const int d = pr->head_dim, hq = pr->num_q_heads, hkv = pr->num_kv_heads;
  // a wave takes at least one row of every lane group
  if (T * ((hq + hkv) / (512 / d) + 2) > kMaxWaves)
    return host_fail(PDA_EINVAL, "num_tokens = %d of %d heads is too much for one call", pr->num_tokens, hq + hkv);
  int rc;
  if ((rc = check_stride("q_stride", pr->q_stride, hq, d, pr->dtype, T, &a->q_stride)) != PDA_OK ||
      (rc = check_stride("k_stride", pr->k_stride, hkv, d, pr->dtype, T, &a->k_stride)) != PDA_OK ||
      (rc = check_stride("v_stride", with_v ? pr->v_stride : 0, hkv, d, pr->dtype, T, &a->v_stride)) != PDA_OK ||
      (rc = check_stride("q_out_stride", pr->q_out_stride, hq, d, pr->out_dtype, T, &a->qo_stride)) != PDA_OK ||
      (rc = check_stride("k_out_stride", pr->k_out_stride, hkv, d, pr->out_dtype, T, &a->ko_stride)) != PDA_OK ||
      (rc = check_stride("grad_q_stride", pr->grad_q_stride, hq, d, pr->dtype, T, &a->dq_stride)) != PDA_OK ||
      (rc = check_stride("grad_k_stride", pr->grad_k_stride, hkv, d, pr->dtype, T, &a->dk_stride)) != PDA_OK)
    return rc;
  a->T = pr->num_tokens;
  a->Hq = hq;
  a->Hkv = hkv;
  a->D = d;
  a->R = pr->rotary_dim;
  a->P = pr->max_positions;
  a->in_bf16 = pr->dtype == PDA_DTYPE_BF16;
  a->out_bf16 = pr->out_dtype == PDA_DTYPE_BF16;
  a->w_bf16 = pr->weight_dtype == PDA_DTYPE_BF16;
  a->interleaved = pr->interleaved;
  a->eps = pr->eps;
  return PDA_OK;
}

// Arrival counts for the call, unless it is captured.
template <typename Args>
int count(hipStream_t s, const pda::HeldWorkspace& ws, Args* a) {
  pda::Counts c;
  const int rc = pda::take_counts(s, ws, &c);
  a->counts = c.words;
  a->epoch = c.epoch;
  return rc;
}

int32_t* status_word(char* base) { return reinterpret_cast<int32_t*>(base) + pda::kHdrStatus; }

int append_run(const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight,
               const float* cos_sin, const int32_t* positions, const int32_t* q_offsets, void* q_out, void* k_cache,
               void* v_cache, float* kv_scales, const int32_t* block_table, const int32_t* seq_lens,
               const pdaops_rope_problem* pr, const pdaops_cache* ca, hipStream_t stream) {
  pda::host_clear_error();
  pda::RopeArgs a = {};
  int rc = check_rope(pr, q_weight != nullptr, k_weight != nullptr, true, &a);
  if (rc != PDA_OK) return rc;
  if (!ca) return host_fail(PDA_EINVAL, "cache is NULL");
  if (ca->num_seqs < 0) return host_fail(PDA_EINVAL, "num_seqs = %d < 0", ca->num_seqs);
  if (ca->block_size != pda::kBlockSize) return host_fail(PDA_EUNSUPPORTED, "block_size = %d (supported: 16)", ca->block_size);
  if (ca->max_blocks_per_seq < 1) return host_fail(PDA_EINVAL, "max_blocks_per_seq = %d < 1", ca->max_blocks_per_seq);
  if (ca->num_blocks < 1) return host_fail(PDA_EINVAL, "num_blocks = %lld < 1", (long long)ca->num_blocks);
  const int64_t table_tokens = (int64_t)ca->max_blocks_per_seq * pda::kBlockSize;
  if (table_tokens > INT32_MAX) return host_fail(PDA_EINVAL, "max_blocks_per_seq * 16 overflows int32");
  if (ca->max_seq_len < 0 || ca->max_seq_len > table_tokens)
    return host_fail(PDA_EINVAL, "max_seq_len = %d (0 .. max_blocks_per_seq * 16 = %lld)", ca->max_seq_len, (long long)table_tokens);
  const int64_t tile = (int64_t)pda::kBlockSize * a.D * 4;
  if (ca->num_blocks > INT64_MAX / a.Hkv / tile) return host_fail(PDA_EINVAL, "num_blocks too large");
  const int kd = ca->kv_dtype;
  if (!float_type(kd) && kd != PDA_DTYPE_FP8_E4M3) return host_fail(PDA_EINVAL, "kv_dtype = %d is not a pda_dtype", kd);
  const int64_t T = a.T, B = ca->num_seqs;
  if (!q_offsets && B > 0 && T % B) return host_fail(PDA_EINVAL, "without q_offsets num_tokens = %d must be a multiple of num_seqs = %d", a.T, ca->num_seqs);
  if (!q_offsets && B == 0 && T > 0) return host_fail(PDA_EINVAL, "num_tokens = %d tokens of no sequence", a.T);
  // a sequence's n tokens touch at most (n + 30) / 16 tiles
  a.n = !q_offsets && B > 0 ? (int32_t)(T / B) : 0;
  a.tiles_per_seq = a.n > 0 ? (int32_t)(((int64_t)a.n + 14) / 16 + 1) : 0;
  const int64_t tiles = q_offsets ? T / 16 + 2 * B : B * a.tiles_per_seq;
  if (T * ((a.Hq + a.Hkv) / (512 / a.D) + 2) > kMaxWaves / 2)
    return host_fail(PDA_EINVAL, "num_tokens = %d of %d heads is too much for one call", a.T, a.Hq + a.Hkv);
  if (tiles * 2 * a.Hkv > kMaxWaves / 2)
    return host_fail(PDA_EINVAL, "%lld cache tiles of %d KV heads are too much for one call", (long long)tiles, a.Hkv);
  if (T == 0 || B == 0) return PDA_OK;
  rc = check_pointers({{q, 16, "q", true}, {k, 16, "k", true}, {v, 16, "v", true}, {q_weight, 16, "q_weight", false},
                       {k_weight, 16, "k_weight", false}, {cos_sin, 16, "cos_sin", true}, {positions, 4, "positions", false},
                       {q_offsets, 4, "q_offsets", false}, {q_out, 16, "q_out", true}, {k_cache, 16, "k_cache", true},
                       {v_cache, 16, "v_cache", true}, {kv_scales, 4, "kv_scales", kd == PDA_DTYPE_FP8_E4M3},
                       {block_table, 4, "block_table", true}, {seq_lens, 4, "seq_lens", true}});
  if (rc != PDA_OK) return rc;

  pda::HeldWorkspace ws;
  if ((rc = pda::hold_workspace(stream, kHeader, &ws)) != PDA_OK) return rc;
  a.q = q;
  a.k = k;
  a.v = v;
  a.wq = q_weight;
  a.wk = k_weight;
  a.table = cos_sin;
  a.positions = positions;
  a.q_out = q_out;
  a.status = status_word(ws.base);
  a.q_offsets = q_offsets;
  a.seq_lens = seq_lens;
  a.block_table = block_table;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.kv_scales = kv_scales;
  a.B = ca->num_seqs;
  a.max_blocks = ca->max_blocks_per_seq;
  a.len_cap = ca->max_seq_len > 0 ? ca->max_seq_len : (int32_t)table_tokens;
  a.num_blocks = ca->num_blocks;
  a.tiles = (int32_t)tiles;
  const pda::KvType kv = kd == PDA_DTYPE_F32 ? pda::KvType::F32 : kd == PDA_DTYPE_BF16 ? pda::KvType::BF16 : pda::KvType::FP8;
  const hipError_t e = pda::launch_rope_append(a, kv, stream);
  return e == hipSuccess ? PDA_OK : pda::host_fail_hip(e, "norm, rotation and append kernel launch");
}

int rope_run(const void* q, const void* k, const void* q_weight, const void* k_weight, const float* cos_sin,
             const int32_t* positions, void* q_out, void* k_out, const pdaops_rope_problem* pr, hipStream_t stream) {
  pda::host_clear_error();
  pda::RopeArgs a = {};
  int rc = check_rope(pr, q_weight != nullptr, k_weight != nullptr, false, &a);
  if (rc != PDA_OK) return rc;
  if (a.T == 0) return PDA_OK;
  rc = check_pointers({{q, 16, "q", true}, {k, 16, "k", true}, {q_weight, 16, "q_weight", false},
                       {k_weight, 16, "k_weight", false}, {cos_sin, 16, "cos_sin", true}, {positions, 4, "positions", true},
                       {q_out, 16, "q_out", true}, {k_out, 16, "k_out", true}});
  if (rc != PDA_OK) return rc;
  pda::HeldWorkspace ws;
  if ((rc = pda::hold_workspace(stream, kHeader, &ws)) != PDA_OK) return rc;
  a.q = q;
  a.k = k;
  a.wq = q_weight;
  a.wk = k_weight;
  a.table = cos_sin;
  a.positions = positions;
  a.q_out = q_out;
  a.k_out = k_out;
  a.status = status_word(ws.base);
  const hipError_t e = pda::launch_rope(a, stream);
  return e == hipSuccess ? PDA_OK : pda::host_fail_hip(e, "norm and rotation kernel launch");
}

int rope_backward_run(const void* q, const void* k, const void* q_weight, const void* k_weight, const float* cos_sin,
                      const int32_t* positions, const void* grad_q_out, const void* grad_k_out, void* grad_q,
                      void* grad_k, float* grad_q_weight, float* grad_k_weight, const pdaops_rope_problem* pr,
                      hipStream_t stream) {
  pda::host_clear_error();
  pda::RopeArgs a = {};
  int rc = check_rope(pr, q_weight != nullptr, k_weight != nullptr, false, &a);
  if (rc != PDA_OK) return rc;
  if (pr->out_dtype != pr->dtype)
    return host_fail(PDA_EINVAL, "out_dtype = %d: the gradient's tensors all have dtype = %d", pr->out_dtype, pr->dtype);
  const bool norm = q_weight != nullptr;
  if (a.T == 0 && !norm) return PDA_OK;
  const bool any = a.T > 0;
  rc = check_pointers({{q, 16, "q", norm && any}, {k, 16, "k", norm && any}, {q_weight, 16, "q_weight", false},
                       {k_weight, 16, "k_weight", false}, {cos_sin, 16, "cos_sin", any}, {positions, 4, "positions", any},
                       {grad_q_out, 16, "grad_q_out", any}, {grad_k_out, 16, "grad_k_out", any},
                       {grad_q, 16, "grad_q", any}, {grad_k, 16, "grad_k", any},
                       {grad_q_weight, 4, "grad_q_weight", norm}, {grad_k_weight, 4, "grad_k_weight", norm}});
  if (rc != PDA_OK) return rc;
  pda::HeldWorkspace ws;
  // parts of the weights' gradients: at most as many workgroups as there are tokens' parts
  constexpr int64_t kWgsPerCu = 4, kMostCus = 1024;
  const int64_t part = 2 * (int64_t)a.D * 4;
  if ((rc = pda::hold_workspace(stream, kHeader + (norm ? kWgsPerCu * kMostCus * part : 0), &ws)) != PDA_OK) return rc;
  a.q = q;
  a.k = k;
  a.wq = q_weight;
  a.wk = k_weight;
  a.table = cos_sin;
  a.positions = positions;
  a.gq = grad_q_out;
  a.gk = grad_k_out;
  a.gq_stride = a.qo_stride;
  a.gk_stride = a.ko_stride;
  a.dq = grad_q;
  a.dk = grad_k;
  a.dwq = grad_q_weight;
  a.dwk = grad_k_weight;
  a.dw_part = reinterpret_cast<float*>(ws.base + kHeader);
  a.wgs = (int32_t)kWgsPerCu * (ws.cus < kMostCus ? ws.cus : (int32_t)kMostCus);
  if (norm && (rc = count(stream, ws, &a)) != PDA_OK) return rc;
  a.status = status_word(ws.base);
  const hipError_t e = pda::launch_rope_backward(a, stream);
  return e == hipSuccess ? PDA_OK : pda::host_fail_hip(e, "norm and rotation gradient kernel launch");
}

int check_logits(const pdaops_logits_problem* pr, pda::LogitsArgs* a) {
  if (!pr) return host_fail(PDA_EINVAL, "problem is NULL");
  if (pr->num_tokens < 0) return host_fail(PDA_EINVAL, "num_tokens = %d < 0", pr->num_tokens);
  if (pr->vocab < 1 || pr->vocab > (1 << 30)) return host_fail(PDA_EINVAL, "vocab = %d (1 .. 2^30)", pr->vocab);
  if (!float_type(pr->dtype)) return host_fail(PDA_EINVAL, "dtype = %d (supported: F32, BF16)", pr->dtype);
  if (pr->targets_int64 != 0 && pr->targets_int64 != 1) return host_fail(PDA_EINVAL, "targets_int64 = %d (0 or 1)", pr->targets_int64);
  a->stride = pr->row_stride ? pr->row_stride : pr->vocab;
  if (a->stride < pr->vocab || a->stride > INT64_MAX / 8 / (pr->num_tokens + 1ll))
    return host_fail(PDA_EINVAL, "row_stride = %lld", (long long)pr->row_stride);
  if (!(pr->temperature > 0.f) || !std::isfinite(pr->temperature) || !std::isfinite(1.f / pr->temperature))
    return host_fail(PDA_EINVAL, "temperature must be positive and finite");
  a->T = pr->num_tokens;
  a->V = pr->vocab;
  a->bf16 = pr->dtype == PDA_DTYPE_BF16;
  a->targets64 = pr->targets_int64;
  a->inv_temp = 1.f / pr->temperature;
  return PDA_OK;
}

// Whole 16-byte vectors of a row.
int vectors_of(const pda::LogitsArgs& a) { return a.bf16 ? a.V / 8 : a.V / 4; }

// Parts per row: enough workgroups for the compute units, of at least 512 vectors
// (two for each thread) each. Half or twice as many workgroups, or least vectors, are
// within 10% on every size tried (1 to 3,000 rows of 8,000 to 150,000 words) but for
// rows of 8,000 words, which 256 vectors a part cut in two: 5.3 - 9.3 us per call, 4.2 - 7.1 whole.
void split_rows(pda::LogitsArgs* a) {
  constexpr int64_t kWgs = 1024, kLeast = 512;
  const int64_t v = vectors_of(*a);
  int64_t s = (kWgs + a->T - 1) / a->T;
  if (s > v / kLeast) s = v / kLeast;
  if (s > pda::kMaxSplits) s = pda::kMaxSplits;
  if (s < 1) s = 1;
  a->chunk = (int32_t)((v + s - 1) / s);
  if (a->chunk < 1) a->chunk = 1;
  a->splits = (int32_t)((v + a->chunk - 1) / a->chunk);
  if (a->splits < 1) a->splits = 1;
}

int logprobs_run(const void* logits, const void* targets, float* logprobs, float* entropy,
                 const pdaops_logits_problem* pr, hipStream_t stream) {
  pda::host_clear_error();
  pda::LogitsArgs a = {};
  int rc = check_logits(pr, &a);
  if (rc != PDA_OK) return rc;
  if (a.T == 0) return PDA_OK;
  rc = check_pointers({{logits, a.bf16 ? 2u : 4u, "logits", true}, {targets, a.targets64 ? 8u : 4u, "targets", true},
                       {logprobs, 4, "logprobs", true}, {entropy, 4, "entropy", false}});
  if (rc != PDA_OK) return rc;
  split_rows(&a);
  if ((int64_t)a.T * a.splits > kMaxWaves / 16) return host_fail(PDA_EINVAL, "num_tokens = %d is too much for one call", a.T);
  pda::HeldWorkspace ws;
  if ((rc = pda::hold_workspace(stream, kHeader + (a.splits > 1 ? (int64_t)a.T * a.splits * 16 : 0), &ws)) != PDA_OK) return rc;
  a.logits = logits;
  a.targets = targets;
  a.logp = logprobs;
  a.ent = entropy;
  a.part = reinterpret_cast<float4*>(ws.base + kHeader);
  a.status = status_word(ws.base);
  if (a.splits > 1 && a.T <= pda::kShortUnits && (rc = count(stream, ws, &a)) != PDA_OK) return rc;
  const hipError_t e = pda::launch_token_logprobs(a, stream);
  return e == hipSuccess ? PDA_OK : pda::host_fail_hip(e, "log-probability kernel launch");
}

int policy_run(const void* logits, const void* targets, const float* old_logprobs, const float* ref_logprobs,
               const float* advantages, const float* weights, float* stats, void* dlogits, float* logprobs,
               float* entropy, const pdaops_logits_problem* pr, const pdaops_policy_options* op, hipStream_t stream) {
  pda::host_clear_error();
  pda::LogitsArgs a = {};
  int rc = check_logits(pr, &a);
  if (rc != PDA_OK) return rc;
  if (!op) return host_fail(PDA_EINVAL, "options is NULL");
  if (!(op->clip_low >= 0.f && op->clip_low <= 1.f)) return host_fail(PDA_EINVAL, "clip_low must be in [0, 1]");
  if (!(op->clip_high >= 0.f) || !std::isfinite(op->clip_high)) return host_fail(PDA_EINVAL, "clip_high is negative or not finite");
  if (op->dual_clip != 0.f && !(op->dual_clip > 1.f && std::isfinite(op->dual_clip)))
    return host_fail(PDA_EINVAL, "dual_clip must be 0 or above 1");
  if (!(op->kl_coef >= 0.f) || !std::isfinite(op->kl_coef)) return host_fail(PDA_EINVAL, "kl_coef is negative or not finite");
  if (!(op->entropy_coef >= 0.f) || !std::isfinite(op->entropy_coef))
    return host_fail(PDA_EINVAL, "entropy_coef is negative or not finite");
  if (!std::isfinite(op->grad_scale)) return host_fail(PDA_EINVAL, "grad_scale is not finite");
  a.d_stride = op->dlogits_stride ? op->dlogits_stride : a.V;
  if (a.d_stride < a.V || a.d_stride > INT64_MAX / 8 / (a.T + 1ll))
    return host_fail(PDA_EINVAL, "dlogits_stride = %lld", (long long)op->dlogits_stride);
  if (op->kl_coef > 0.f && !ref_logprobs && a.T > 0) return host_fail(PDA_EINVAL, "kl_coef needs ref_logprobs");
  const bool any = a.T > 0;
  const uintptr_t e = a.bf16 ? 2 : 4;
  rc = check_pointers({{logits, e, "logits", any}, {targets, a.targets64 ? 8u : 4u, "targets", any},
                       {old_logprobs, 4, "old_logprobs", any}, {ref_logprobs, 4, "ref_logprobs", false},
                       {advantages, 4, "advantages", any}, {weights, 4, "weights", any}, {stats, 4, "stats", true},
                       {dlogits, e, "dlogits", false}, {logprobs, 4, "logprobs", false}, {entropy, 4, "entropy", false}});
  if (rc != PDA_OK) return rc;
  if (a.T > kMaxWaves / 64) return host_fail(PDA_EINVAL, "num_tokens = %d is too much for one call", a.T);
  // Rows in registers (and LDS) where they fit and either there are enough of them
  // for the compute units or they are short; otherwise in parts, read twice (us per
  // call in a HIP graph, registers / parts; bf16: 128 rows of 131,072 words 24.1 / 20.9, 192 26.0 / 33.3,
  // 512 58 / 68; 128 of 200,000 41 / 35, 192 45 / 48, 2,048 359 / 471; 64 of 32,000 11.6 / 10.6, 128 12.4 / 12.6; 1 of
  // 16,000 7.5 / 9.2, 512 13 / 17; among eager calls 8 of 20,000 9.2 / 10.7, of 32,000 10.7 / 10.6, 64 of 20,000
  // 11.2 / 12.5; f32: 64 of 50,001 14.6 / 12.5, 128 15.5 / 16.1; 128 of 110,000 31 / 34, 2,048 348 / 523).
  constexpr int kManyBf16 = 160, kManyF32 = 112, kShortVectors = 3200;
  const int v = vectors_of(a);
  if (any && ((a.T < (a.bf16 ? kManyBf16 : kManyF32) && v > kShortVectors) || v > pda::kRowVectors)) split_rows(&a);
  const int64_t terms = ((int64_t)a.T * pda::kTerms * 4 + 255) / 256 * 256;
  pda::HeldWorkspace ws;
  if ((rc = pda::hold_workspace(stream, kHeader + terms + (int64_t)a.T * a.splits * 16, &ws)) != PDA_OK) return rc;
  a.logits = logits;
  a.targets = targets;
  a.logp = logprobs;
  a.ent = entropy;
  a.old_logp = old_logprobs;
  a.ref_logp = ref_logprobs;
  a.adv = advantages;
  a.weight = weights;
  a.stats = stats;
  a.dlogits = dlogits;
  a.clip_low = op->clip_low;
  a.clip_high = op->clip_high;
  a.dual = op->dual_clip;
  a.kl = op->kl_coef;
  a.ent_coef = op->entropy_coef;
  a.grad_scale = op->grad_scale;
  a.terms = reinterpret_cast<float*>(ws.base + kHeader);
  a.part = reinterpret_cast<float4*>(ws.base + kHeader + terms);
  a.status = status_word(ws.base);
  if (any && a.T <= pda::kCountedRows && (rc = count(stream, ws, &a)) != PDA_OK) return rc;
  const hipError_t h = pda::launch_policy_loss(a, stream);
  return h == hipSuccess ? PDA_OK : pda::host_fail_hip(h, "policy loss kernel launch");
}

// A C entry: what is thrown below it (no memory for the workspace's record, a
// failed lock) becomes an error code with a text, of at most 15 characters: a
// std::string holds these without memory of its own.
template <typename F>
int entry(F run) {
  try {
    return run();
  } catch (const std::bad_alloc&) {
    return host_fail(PDA_ENOMEM, "no host memory");
  } catch (...) {
    return host_fail(PDA_EHIP, "host exception");
  }
}

}  // namespace

extern "C" {

int pdaops_paged_qk_norm_rope_append(const void* q, const void* k, const void* v, const void* q_weight,
                                     const void* k_weight, const float* cos_sin, const int32_t* positions,
                                     const int32_t* q_offsets, void* q_out, void* k_cache, void* v_cache,
                                     float* kv_scales, const int32_t* block_table, const int32_t* seq_lens,
                                     const pdaops_rope_problem* problem, const pdaops_cache* cache, hipStream_t stream) {
  return entry([&] {
    return append_run(q, k, v, q_weight, k_weight, cos_sin, positions, q_offsets, q_out, k_cache, v_cache, kv_scales,
                      block_table, seq_lens, problem, cache, stream);
  });
}

int pdaops_qk_norm_rope(const void* q, const void* k, const void* q_weight, const void* k_weight, const float* cos_sin,
                        const int32_t* positions, void* q_out, void* k_out, const pdaops_rope_problem* problem,
                        hipStream_t stream) {
  return entry([&] {
    return rope_run(q, k, q_weight, k_weight, cos_sin, positions, q_out, k_out, problem, stream);
  });
}

int pdaops_qk_norm_rope_backward(const void* q, const void* k, const void* q_weight, const void* k_weight,
                                 const float* cos_sin, const int32_t* positions, const void* grad_q_out,
                                 const void* grad_k_out, void* grad_q, void* grad_k, float* grad_q_weight,
                                 float* grad_k_weight, const pdaops_rope_problem* problem, hipStream_t stream) {
  return entry([&] {
    return rope_backward_run(q, k, q_weight, k_weight, cos_sin, positions, grad_q_out, grad_k_out, grad_q, grad_k,
                             grad_q_weight, grad_k_weight, problem, stream);
  });
}

int pdaops_token_logprobs(const void* logits, const void* targets, float* logprobs, float* entropy,
                          const pdaops_logits_problem* problem, hipStream_t stream) {
  return entry([&] {
    return logprobs_run(logits, targets, logprobs, entropy, problem, stream);
  });
}

int pdaops_policy_loss(const void* logits, const void* targets, const float* old_logprobs, const float* ref_logprobs,
                       const float* advantages, const float* weights, float* stats, void* dlogits, float* logprobs,
                       float* entropy, const pdaops_logits_problem* problem, const pdaops_policy_options* options,
                       hipStream_t stream) {
  return entry([&] {
    return policy_run(logits, targets, old_logprobs, ref_logprobs, advantages, weights, stats, dlogits, logprobs, entropy,
                      problem, options, stream);
  });
}

}  // extern "C"
