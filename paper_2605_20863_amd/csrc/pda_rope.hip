// HIP kernels for the norms of queries and keys per head with the position
// rotation in the same pass, on MI355X (gfx950): into the paged cache (decode
// steps, chunked prefill, the log-prob forward), as a training forward, and its
// gradient.
//
// For a head's row x [D] of token t at position p, with weights w:
//     r = 1 / sqrt(mean x^2 + eps),  n = x r w   (n = x without norms)
//     y_i = n_i cos(p, i) - n_j sin(p, i),  y_j = n_j cos(p, i) + n_i sin(p, i)
// over the pairs (i, j) of the first R dims: (i, i + R / 2), or (2 i, 2 i + 1)
// interleaved; dims past R stay n. With g = the gradient of y turned back by the
// same angles:
//     dw = sum over rows of g x r,   dx = r (g w - x r mean(g w x r)).
//
// A lane holds 8 neighbouring dims of a row, a row D / 8 lanes of a wave: 16-byte
// accesses (bf16), and the sums over a row are DPP adds in its lanes. All sums
// are float32 (the weights' gradient over all tokens: float32 in a wave, then
// float64); every output is rounded once.

#include "pda_arrive.h"
#include "pda_elem.h"
#include "pda_ops_internal.h"

namespace pda {
namespace {

constexpr int kWaves = 4;  // waves per workgroup
constexpr int kManyRows = 8, kFewRows = 2;  // rows of a lane group that a wave takes

__device__ __forceinline__ int lane_id() { return (int)(threadIdx.x & 63); }
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

template <int D>
struct Row {
  static constexpr int LPR = D / 8;     // lanes of a row
  static constexpr int RPI = 64 / LPR;  // rows of a wave at a time
};

// A lane's part of the rotation: y_i = n_i c_i + partner_i s_i, where dim i's
// partner is the other member of its pair and s carries the sign.
struct Angles {
  float c[8], s[8];
};
struct Turn {
  int R, half_lane;  // half_lane: lane that holds this lane's partners (half-split pairs)
  bool inter, full, on;
};

template <int D>
__device__ __forceinline__ Turn make_turn(const RopeArgs& a) {
  const int j = lane_id() % Row<D>::LPR;
  Turn t;
  t.R = a.R;
  t.inter = a.interleaved;
  t.full = a.R == D;
  t.on = 8 * j < a.R;
  t.half_lane = lane_id() + (!t.on ? 0 : 16 * j < a.R ? a.R / 16 : -(a.R / 16));
  return t;
}

__device__ __forceinline__ int clamp_position(const RopeArgs& a, int p) {
  const int q = p < 0 ? 0 : p >= a.P ? a.P - 1 : p;
  if (q != p) atomicOr(a.status, kStatusBadPosition);
  return q;
}

// Angles of table row p for this lane's 8 dims (lanes past R load row p's first and use none).
template <int D>
__device__ __forceinline__ Angles load_angles(const RopeArgs& a, const Turn& t, int p) {
  const int d0 = t.on ? 8 * (lane_id() % Row<D>::LPR) : 0, h = t.R / 2;
  const float* row = a.table + (int64_t)p * t.R;
  Angles g;
  if (t.inter) {
    const f32x4 c = *reinterpret_cast<const f32x4*>(row + d0 / 2);
    const f32x4 s = *reinterpret_cast<const f32x4*>(row + h + d0 / 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g.c[2 * i] = g.c[2 * i + 1] = c[i];
      g.s[2 * i] = -s[i];
      g.s[2 * i + 1] = s[i];
    }
  } else {
    const int f = d0 < h ? d0 : d0 - h;
    const f32x4* c = reinterpret_cast<const f32x4*>(row + f);
    const f32x4* s = reinterpret_cast<const f32x4*>(row + h + f);
    const f32x4 c0 = c[0], c1 = c[1], s0 = s[0], s1 = s[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g.c[i] = c0[i];
      g.c[4 + i] = c1[i];
      g.s[i] = d0 < h ? -s0[i] : s0[i];
      g.s[4 + i] = d0 < h ? -s1[i] : s1[i];
    }
  }
  return g;
}

// Rotates the wave's rows (all lanes active). sign -1 turns back.
template <int D>
__device__ __forceinline__ void turn(const Turn& t, const Angles& g, float sign, float (&n)[8]) {
  float o[8];
  if (t.inter) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = n[i ^ 1];
  } else if (t.full) {  // the partner's lane is half a row away
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (D == 128) o[i] = dpp<kDppRor8>(n[i]);
      else o[i] = dpp<0x1B>(dpp<kDppHalfMirror>(n[i]));  // 7 - lane, then reversed in its quad: lane ^ 4
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = __shfl(n[i], t.half_lane, 64);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = fmaf(n[i], g.c[i], o[i] * (sign * g.s[i]));
    n[i] = t.on ? y : n[i];
  }
}

// 1 / sqrt(mean x^2 + eps) of this lane's row.
template <int D>
__device__ __forceinline__ float inv_rms(const float (&x)[8], float eps) {
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) q = fmaf(x[i], x[i], q);
  return __frsqrt_rn(group_sum<Row<D>::LPR>(q) * (1.f / D) + eps);
}

template <int D>
__device__ __forceinline__ void load_weight(const void* w, bool bf16, float (&o)[8]) {
  const int d0 = 8 * (lane_id() % Row<D>::LPR);
  if (bf16) unpack(load8<false, uint16_t>(w, d0), o);
  else unpack(load8<false, float>(w, d0), o);
}

// Norm (with weights) and rotation of the wave's rows.
template <int D>
__device__ __forceinline__ void norm_turn(const RopeArgs& a, const Turn& t, const Angles& g, const float (&w)[8],
                                          float (&x)[8]) {
  if (a.wq) {
    const float r = inv_rms<D>(x, a.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
  }
  turn<D>(t, g, 1.f, x);
}

// The largest b below B with key(b) <= x for non-decreasing keys (0 where there
// is none), 64 of them a round; every read is of an index below B.
template <typename F>
__device__ __forceinline__ int wave_search(int B, int x, F key) {
  int lo = 0, size = B;
  while (size > 1) {
    const int step = (size + 63) / 64, i = lane_id() * step;
    const bool le = i < size && key(lo + i) <= x;
    const int k = __popcll(__ballot(le)) - 1;
    if (k < 0) return lo;
    lo += k * step;
    size = min(step, size - k * step);
  }
  return lo;
}

// Tokens of sequence b: rows [first, first + count) of the packed ones, at positions pos0 ..
struct Seq {
  int first, count, len, pos0;
  bool ok;
};
__device__ __forceinline__ Seq sequence(const RopeArgs& a, int b) {
  Seq s;
  if (a.q_offsets) {
    const int lo = a.q_offsets[b], hi = a.q_offsets[b + 1];
    s.first = lo;
    s.count = hi - lo;
    s.ok = 0 <= lo && lo <= hi && hi <= a.T;
  } else {
    s.first = b * a.n;
    s.count = a.n;
    s.ok = true;
  }
  const int len = a.seq_lens[b];
  s.len = len < 0 ? 0 : len > a.len_cap ? a.len_cap : len;
  s.pos0 = s.len - s.count;
  return s;
}

// The rows [row0, rows_end) of token t, heads of q, then (KROWS) of k.
template <typename T, int D, int NI, bool KROWS, bool STREAM, typename P>
__device__ __forceinline__ void token_rows(const RopeArgs& a, int t, int row0, int rows_end, P position) {
  constexpr int RPI = Row<D>::RPI, LPR = Row<D>::LPR;
  const int r = lane_id() / LPR, d0 = 8 * (lane_id() % LPR);
  Raw<T> raw[NI];
#pragma unroll
  for (int it = 0; it < NI; ++it) {
    if (row0 + it * RPI >= rows_end) break;
    const int h = min(row0 + it * RPI + r, rows_end - 1);
    const bool k = KROWS && h >= a.Hq;
    raw[it] = load8<STREAM, T>(k ? a.k : a.q, (k ? t * a.k_stride + (int64_t)(h - a.Hq) * D : t * a.q_stride + (int64_t)h * D) + d0);
  }
  float wq[8] = {}, wk[8] = {};
  if (a.wq) load_weight<D>(a.wq, a.w_bf16, wq);
  if (KROWS && a.wq) load_weight<D>(a.wk, a.w_bf16, wk);
  const int p = position();
  if (p < 0) return;
  const Turn tn = make_turn<D>(a);
  const Angles g = load_angles<D>(a, tn, p);
#pragma unroll
  for (int it = 0; it < NI; ++it) {
    if (row0 + it * RPI >= rows_end) break;
    const int h = row0 + it * RPI + r;
    const bool k = KROWS && h >= a.Hq;
    float x[8], w[8];
    unpack(raw[it], x);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = k ? wk[i] : wq[i];
    norm_turn<D>(a, tn, g, w, x);
    if (h < rows_end)
      store8<STREAM>(k ? a.k_out : a.q_out, (k ? t * a.ko_stride + (int64_t)(h - a.Hq) * D : t * a.qo_stride + (int64_t)h * D) + d0,
             a.out_bf16, x);
  }
}

// ------------------------------------------------------------- cache append

__device__ __forceinline__ uint32_t enc4(const float (&z)[4]) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = fminf(fmaxf(z[i], -kE4M3Max), kE4M3Max);
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
}
__device__ __forceinline__ uint32_t reencode4(uint32_t w, float old, const Div& d) {
  const float z[4] = {
      quotient(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * old, d), quotient(__builtin_amdgcn_cvt_f32_fp8((int)w, 1) * old, d),
      quotient(__builtin_amdgcn_cvt_f32_fp8((int)w, 2) * old, d), quotient(__builtin_amdgcn_cvt_f32_fp8((int)w, 3) * old, d)};
  return enc4(z);
}
// bytes first .. end - 1 of a 16-byte piece from y, the others from x
__device__ __forceinline__ u32x4 merge16(u32x4 x, u32x4 y, int first, int end) {
  u32x4 o;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m |= (4 * w + i >= first && 4 * w + i < end) ? 0xFFu << (8 * i) : 0u;
    o[w] = (x[w] & ~m) | (y[w] & m);
  }
  return o;
}

// Scale of an fp8 tile whose slots o .. get new values of largest size amax: as
// it was, where they fit; otherwise their own, and earlier codes are re-encoded.
__device__ __forceinline__ bool raise_scale(int o, float old, float amax, float& s) {
  s = old;
  if (o > 0 && old > 0.f && amax <= kE4M3Max * old) return false;
  s = fmaxf(__fdiv_rn(amax, kE4M3Max), kMinScale);
  return true;
}

// LDS dwords of a V tile [D][16] on its way from rows of tokens to rows of dims: 4
// spare ones after each 8 dims, so that a wave's writes (one dim of each lane's 8)
// fall on different banks.
template <KvType KV, int D>
constexpr int tile_dwords() {
  return D * 16 * (KV == KvType::F32 ? 4 : KV == KvType::BF16 ? 2 : 1) / 4 + D / 8 * 4;
}

// One wave: K or V of one KV head in one cache tile, new slots o .. e - 1.
template <typename T, KvType KV, int D, bool STREAM>
__device__ __forceinline__ void kv_tile(const RopeArgs& a, uint32_t item, uint32_t* lds) {
  constexpr int LPR = Row<D>::LPR, RPI = Row<D>::RPI, IT = 16 / RPI;
  const bool is_v = item & 1;
  const int pair = (int)(item >> 1), tile = pair / a.Hkv, h = pair - tile * a.Hkv;
  int b, jt;
  if (a.q_offsets) {
    // sequence b's tiles are at most count / 16 + 2: they are numbered from offsets[b] / 16 + 2 b
    b = __builtin_amdgcn_readfirstlane(
        wave_search(a.B, tile, [&](int i) { return (int)((uint32_t)a.q_offsets[i] / 16) + 2 * i; }));
    jt = tile - ((int)((uint32_t)a.q_offsets[b] / 16) + 2 * b);
  } else {
    b = tile / a.tiles_per_seq;
    jt = tile - b * a.tiles_per_seq;
  }
  const Seq sq = sequence(a, b);
  if (h == 0 && !is_v && jt == 0 && lane_id() == 0) {
    if (sq.len != a.seq_lens[b]) atomicOr(a.status, kStatusLenClamped);
  }
  const int start = max(sq.pos0, 0);
  if (!sq.ok || jt < 0 || jt >= (sq.len + 15) / 16 - start / 16) return;
  const int blk = start / 16 + jt;
  const int o = max(start - 16 * blk, 0), e = min(sq.len - 16 * blk, 16);
  if (o >= e) return;
  const int p = a.block_table[(int64_t)b * a.max_blocks + blk];
  const int j = lane_id() % LPR, r = lane_id() / LPR, d0 = 8 * j;
  // packed row of slot 0's token (never read below slot o)
  const int64_t t0 = (int64_t)sq.first - sq.pos0 + 16 * blk;
  const void* in = is_v ? a.v : a.k;
  const int64_t in_stride = is_v ? a.v_stride : a.k_stride;
  // K: rows of neighbouring slots; V: a lane gets both slots of a pair
  // whether the wave's rows of iteration `it` hold a new slot
  auto any = [&](int it) {
    return is_v ? 2 * RPI * (it >> 1) < e && 2 * RPI * ((it >> 1) + 1) > o : RPI * it < e && RPI * (it + 1) > o;
  };
  auto slot_of = [&](int it) { return is_v ? 2 * (r + RPI * (it >> 1)) + (it & 1) : RPI * it + r; };
  Raw<T> raw[IT];
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    if (!any(it)) continue;
    const int s = min(max(slot_of(it), o), e - 1);
    raw[it] = load8<STREAM, T>(in, (t0 + s) * in_stride + (int64_t)h * D + d0);
  }
  float y[IT][8];
  auto rows = [&]() {
#pragma unroll
    for (int it = 0; it < IT; ++it) unpack(raw[it], y[it]);
    if (is_v) return;
    const Turn tn = make_turn<D>(a);
    float w[8] = {};
    if (a.wq) load_weight<D>(a.wk, a.w_bf16, w);
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      if (!any(it)) continue;
      const int s = min(max(slot_of(it), o), e - 1);
      const int pos = clamp_position(a, a.positions ? a.positions[t0 + s] : 16 * blk + s);
      norm_turn<D>(a, tn, load_angles<D>(a, tn, pos), w, y[it]);
    }
  };
  // without a scale to load, rows are turned before the tile's place is known
  // (27 x 59 tokens, 32 / 8 heads, bf16: 12.1 us per call after it, 11.1 so)
  if constexpr (KV != KvType::FP8) rows();
  if ((unsigned)p >= (uint64_t)a.num_blocks) {
    if (lane_id() == 0) atomicOr(a.status, kStatusBadBlock);
    return;
  }
  const int64_t ct = (int64_t)p * a.Hkv + h;
  float* sp = KV == KvType::FP8 ? a.kv_scales + (is_v ? a.num_blocks * a.Hkv : 0) + ct : nullptr;
  const float old = KV == KvType::FP8 && o > 0 ? *sp : 0.f;
  if constexpr (KV == KvType::FP8) rows();
  float scale = 1.f;
  bool raised = false;
  if constexpr (KV == KvType::FP8) {
    float m = 0.f;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      if (!any(it)) continue;
      const int s = slot_of(it);
#pragma unroll
      for (int i = 0; i < 8; ++i) m = s >= o && s < e ? fmaxf(m, fabsf(y[it][i])) : m;
    }
    raised = raise_scale(o, old, wave_max_f(m), scale);
    if (lane_id() == 0) *sp = scale;
  }
  const Div div = make_div(scale);
  if (!is_v) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int s = slot_of(it);
      if (s < o || s >= e) continue;
      const int64_t at = ct * 16 * D + (int64_t)s * D + d0;
      if constexpr (KV == KvType::FP8) {
        float z[2][4];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i / 4][i % 4] = quotient(y[it][i], div);
        *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.k_cache) + at) = u32x2{enc4(z[0]), enc4(z[1])};
      } else {
        store8<STREAM>(a.k_cache, at, KV == KvType::BF16, y[it]);
      }
    }
    if (KV == KvType::FP8 && raised) {
      u32x4* pt = reinterpret_cast<u32x4*>(static_cast<uint8_t*>(a.k_cache) + ct * 16 * D);
      for (int i = lane_id(); i < o * D / 16; i += 64) {
        const u32x4 x = pt[i];
        u32x4 n;
#pragma unroll
        for (int w = 0; w < 4; ++w) n[w] = reencode4(x[w], old, div);
        pt[i] = n;
      }
    }
    return;
  }
  // V: through LDS into rows of dims
  constexpr int DW = KV == KvType::F32 ? 16 : KV == KvType::BF16 ? 8 : 4;  // dwords of a dim's 16 slots
  auto dim_at = [&](int d) { return d * DW + (d >> 3) * 4; };
#pragma unroll
  for (int it = 0; it < IT; it += 2) {
    if (!any(it)) continue;
    const int s = slot_of(it);  // an even one
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t* q = lds + dim_at(d0 + i);
      if constexpr (KV == KvType::F32) {
        q[s] = as_u32(y[it][i]);
        q[s + 1] = as_u32(y[it + 1][i]);
      } else if constexpr (KV == KvType::BF16) {
        q[s / 2] = pack_bf16(y[it][i], y[it + 1][i]);
      } else {
        const float z[4] = {quotient(y[it][i], div), quotient(y[it + 1][i], div), 0.f, 0.f};
        reinterpret_cast<uint16_t*>(q)[s / 2] = (uint16_t)enc4(z);
      }
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  constexpr int PIECES = D * DW / 4, PER = 64 / DW;  // 16-byte pieces of the tile; their slots
  char* vt = static_cast<char*>(a.v_cache) + ct * PIECES * 16;
#pragma unroll
  for (int i = 0; i < PIECES / 64; ++i) {
    const int pc = lane_id() + 64 * i, d = pc / (DW / 4), part = pc % (DW / 4);
    const u32x4 x = *reinterpret_cast<const u32x4*>(lds + dim_at(d) + 4 * part);
    const int first = o - part * PER, end = e - part * PER;  // live slots of the piece: first .. end - 1
    if constexpr (KV == KvType::FP8) {
      u32x4* q = reinterpret_cast<u32x4*>(vt + 16 * pc);
      if (o == 0 && e == 16) {
        put16<STREAM>(q, x);
      } else if (e - o == 1 && !(raised && o > 0)) {
        uint32_t word = x[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) word = o / 4 == w ? x[w] : word;
        vt[16 * pc + o] = (char)(word >> (8 * (o % 4)));
      } else {
        u32x4 was = *q;
        if (raised) {
          u32x4 n;
#pragma unroll
          for (int w = 0; w < 4; ++w) n[w] = reencode4(was[w], old, div);
          was = merge16(was, n, 0, o);
        }
        *q = merge16(was, x, o, e);
      }
    } else {
      if (first <= 0 && end >= PER) {
        put16<STREAM>(vt + 16 * pc, x);
      } else {
#pragma unroll
        for (int s = 0; s < PER; ++s) {
          if (s < first || s >= end) continue;
          if constexpr (KV == KvType::F32) reinterpret_cast<uint32_t*>(vt + 16 * pc)[s] = x[s];
          else reinterpret_cast<uint16_t*>(vt + 16 * pc)[s] = (uint16_t)(x[s / 2] >> (16 * (s & 1)));
        }
      }
    }
  }
}

// One new token per sequence (a decode step), or few of each or in all into a
// cache that has no scales (by_token): a wave's lane groups each take one
// KV head's K or V row of a token, so that a step's waves are all on the chip at
// once; V's elements go straight to their columns. Against a wave per (head, K or V) by
// kv_tile: 14.4 us for 512 sequences, 64 / 8 heads, fp8; see rope_token_kernel.
template <typename T, KvType KV, int D>
__device__ __forceinline__ void kv_token(const RopeArgs& a, uint32_t item) {
  constexpr int LPR = Row<D>::LPR, RPI = Row<D>::RPI;
  const bool is_v = item & 1;
  const int per = (a.Hkv + RPI - 1) / RPI, pair = (int)(item >> 1), t = pair / per, hc = pair - t * per;
  const int n = KV == KvType::FP8 ? 1 : a.n, b = KV == KvType::FP8 ? t : t / n;
  const int j = lane_id() % LPR, d0 = 8 * j, h = hc * RPI + lane_id() / LPR;
  const bool live = h < a.Hkv;
  const int hh = live ? h : a.Hkv - 1;
  const Raw<T> raw = load8<false, T>(is_v ? a.v : a.k, t * (is_v ? a.v_stride : a.k_stride) + (int64_t)hh * D + d0);
  const int full = a.seq_lens[b], len = full < 0 ? 0 : full > a.len_cap ? a.len_cap : full;
  if (len != full && hc == 0 && !is_v && lane_id() == 0) atomicOr(a.status, kStatusLenClamped);
  const int pos = len - n + (t - b * n);
  if (pos < 0) return;
  const int p = a.block_table[(int64_t)b * a.max_blocks + pos / 16], o = pos % 16;
  float y[8], w[8] = {};
  Angles g;
  const Turn tn = make_turn<D>(a);
  if (!is_v) {
    if (a.wq) load_weight<D>(a.wk, a.w_bf16, w);
    g = load_angles<D>(a, tn, clamp_position(a, a.positions ? a.positions[t] : pos));
  }
  if ((unsigned)p >= (uint64_t)a.num_blocks) {
    if (lane_id() == 0) atomicOr(a.status, kStatusBadBlock);
    return;
  }
  const int64_t ct = (int64_t)p * a.Hkv + hh;
  float* sp = KV == KvType::FP8 ? a.kv_scales + (is_v ? a.num_blocks * a.Hkv : 0) + ct : nullptr;
  const float old = KV == KvType::FP8 && o > 0 ? *sp : 0.f;
  unpack(raw, y);
  if (!is_v) norm_turn<D>(a, tn, g, w, y);
  if constexpr (KV != KvType::FP8) {
    if (!live) return;
    const int64_t tile = ct * 16 * D;
    if (!is_v) {
      store8<false>(a.k_cache, tile + (int64_t)o * D + d0, KV == KvType::BF16, y);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t at = tile + (d0 + i) * 16 + o;
        if constexpr (KV == KvType::F32) static_cast<float*>(a.v_cache)[at] = y[i];
        else static_cast<uint16_t*>(a.v_cache)[at] = to_bf16(y[i]);
      }
    }
  } else {
    // V's new codes go into every 16-byte piece of their tiles, so these are read
    // and written whole, by the whole wave, 64 pieces at a time (stores of single bytes took
    // 11.6 us per call where this takes 11.0); K's earlier tokens only under a raised scale
    constexpr int N = D / 64;
    uint8_t* first = static_cast<uint8_t*>(is_v ? a.v_cache : a.k_cache) + ((int64_t)p * a.Hkv + hc * RPI) * 16 * D;
    const int pieces = is_v ? D : o * (D / 16);
    u32x4 x[RPI][N];
    auto load = [&](uint64_t rows) {
#pragma unroll
      for (int r = 0; r < RPI; ++r)
#pragma unroll
        for (int n = 0; n < N; ++n)
          if ((rows >> (r * LPR) & 1) && lane_id() + 64 * n < pieces)
            x[r][n] = *reinterpret_cast<const u32x4*>(first + r * 16 * D + 16 * (lane_id() + 64 * n));
    };
    if (is_v) load(__ballot(live));
    float m = 0.f, scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(y[i]));
    const uint64_t raised = __ballot(raise_scale(o, old, group_max<LPR>(m), scale) && o > 0 && live);
    const Div div = make_div(scale);
    float z[2][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i / 4][i % 4] = quotient(y[i], div);
    const u32x2 codes = {enc4(z[0]), enc4(z[1])};
    if (live && j == 0) *sp = scale;
    if (!is_v) {
      if (live) *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.k_cache) + (ct * 16 + o) * D + d0) = codes;
      load(raised);
    }
    const uint64_t rows = is_v ? __ballot(live) : raised;
#pragma unroll
    for (int r = 0; r < RPI; ++r) {
      if (!(rows >> (r * LPR) & 1)) continue;
      u32x4 q[N];
#pragma unroll
      for (int n = 0; n < N; ++n) q[n] = x[r][n];
      if (raised >> (r * LPR) & 1) {
        const float was = __shfl(old, r * LPR, 64);
        const Div dr = make_div(__shfl(scale, r * LPR, 64));
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
          for (int k = 0; k < 4; ++k) q[n][k] = reencode4(x[r][n][k], was, dr);
          if (is_v) q[n] = merge16(x[r][n], q[n], 0, o);
        }
      }
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int pc = lane_id() + 64 * n;
        if (is_v) {  // dim pc, whose new code lane pc / 8 of the row holds
          const uint32_t c0 = __shfl(codes[0], r * LPR + pc / 8, 64), c1 = __shfl(codes[1], r * LPR + pc / 8, 64);
          const uint32_t code = ((pc & 4 ? c1 : c0) >> (8 * (pc & 3)) & 0xFFu) * 0x01010101u;
          q[n] = merge16(q[n], u32x4{code, code, code, code}, o, o + 1);
        }
        if (pc < pieces) *reinterpret_cast<u32x4*>(first + r * 16 * D + 16 * pc) = q[n];
      }
    }
  }
}

// One wave: every sequence's offsets.
__device__ __forceinline__ void check_offsets(const RopeArgs& a) {
  bool ok = true;
  for (int b = lane_id(); b < a.B; b += 64) ok &= sequence(a, b).ok;
  if (!ok) atomicOr(a.status, kStatusBadOffsets);
}

template <typename T, KvType KV, int D>
__global__ __launch_bounds__(64 * kWaves) void rope_token_kernel(RopeArgs a) {
  const uint32_t per = ((uint32_t)a.Hkv + Row<D>::RPI - 1) / Row<D>::RPI, kv_waves = 2u * (uint32_t)a.T * per;
  const uint32_t kv_wgs = (kv_waves + kWaves - 1) / kWaves;
  if (blockIdx.x < kv_wgs) {
    const uint32_t w = blockIdx.x * kWaves + wave_id();
    if (w < kv_waves) kv_token<T, KV, D>(a, w);
    return;
  }
  const uint32_t w = (blockIdx.x - kv_wgs) * kWaves + wave_id();
  if (w >= (uint32_t)a.T * (uint32_t)a.chunks) return;
  const int t = (int)(w / (uint32_t)a.chunks), c = (int)(w - (uint32_t)t * a.chunks);
  token_rows<T, D, kFewRows, false, false>(a, t, c * a.rows, min(c * a.rows + a.rows, a.Hq), [&]() {
    if (a.positions) return clamp_position(a, a.positions[t]);
    const int n = KV == KvType::FP8 ? 1 : a.n, b = KV == KvType::FP8 ? t : t / n;
    return clamp_position(a, max(max(min(a.seq_lens[b], a.len_cap), 0) - n + (t - b * n), 0));
  });
}

// All tokens of 64 sequences (193,538, 32 / 4 heads, bf16): 572 us, 5.6 TB/s read and
// written (a 1 GiB device copy: 5.0); 512-token chunks, 28 / 4 heads, 108 us, 5.6 TB/s. Short
// chunks are bound by a wave's chain of loads, length to block to scale, angles and
// tile: 4 tokens of 399 sequences, 32 / 8 heads, fp8: 21 us, 1.7 TB/s. An fp8 V tile
// read beside its scale rather than before it is written: no gain (22.4 and 23.3 us).
// Workgroups of KV waves first (their chains are the longer ones), the offsets'
// check after the last, then of q waves.
template <typename T, KvType KV, int D, int NI>
__global__ __launch_bounds__(64 * kWaves) void rope_append_kernel(RopeArgs a) {
  __shared__ __attribute__((aligned(16))) uint32_t lds[kWaves][tile_dwords<KV, D>()];
  const uint32_t kv_waves = 2u * (uint32_t)a.tiles * (uint32_t)a.Hkv, kv_wgs = kv_waves / kWaves + 1;
  if (blockIdx.x < kv_wgs) {
    const uint32_t w = blockIdx.x * kWaves + wave_id();
    if (w < kv_waves) kv_tile<T, KV, D, (NI > kFewRows)>(a, w, lds[wave_id()]);
    else if (w == kv_waves && a.q_offsets) check_offsets(a);
    return;
  }
  const uint32_t w = (blockIdx.x - kv_wgs) * kWaves + wave_id();
  if (w >= (uint32_t)a.T * (uint32_t)a.chunks) return;
  const int t = (int)(w / (uint32_t)a.chunks), c = (int)(w - (uint32_t)t * a.chunks);
  const int row0 = c * a.rows, end = min(row0 + a.rows, a.Hq);
  token_rows<T, D, NI, false, (NI > kFewRows)>(a, t, row0, end, [&]() {
    int b = a.n ? t / a.n : 0;
    if (a.q_offsets) b = __builtin_amdgcn_readfirstlane(wave_search(a.B, t, [&](int i) { return a.q_offsets[i]; }));
    const Seq s = sequence(a, b);
    if (!s.ok || t < s.first || t >= s.first + s.count) return -1;  // a row of no sequence
    return clamp_position(a, a.positions ? a.positions[t] : max(s.pos0 + t - s.first, 0));
  });
}

// ------------------------------------------------------------- training

// 16,384 tokens, 64 / 4 heads, bf16: 102 us, 5.65 TB/s read and written.
template <typename T, int D, int NI>
__global__ __launch_bounds__(64 * kWaves) void rope_kernel(RopeArgs a) {
  const uint32_t w = blockIdx.x * kWaves + wave_id();
  if (w >= (uint32_t)a.T * (uint32_t)a.chunks) return;
  const int t = (int)(w / (uint32_t)a.chunks), c = (int)(w - (uint32_t)t * a.chunks);
  const int row0 = c * a.rows, end = min(row0 + a.rows, a.Hq + a.Hkv);
  token_rows<T, D, NI, true, (NI > kFewRows)>(a, t, row0, end, [&]() { return clamp_position(a, a.positions[t]); });
}

// Rows of parts that rope_weight_grad_kernel sums side by side.
constexpr int kSumRows = 64;

// Gradient. Every wave takes (token, chunk of rows) pairs in turn and keeps its
// rows' part of the weights' gradients; a workgroup's go to dw_part, which with
// counts the last workgroup sums.
// 16,384 tokens, 32 / 4 heads, bf16: 93 us with the sum of 1,024 parts (4 us), 5.0 TB/s
// read and written; 1 token 6.7 us, where a second launch made it 8.0.
template <typename T, int D, int NI, bool STREAM>
__global__ __launch_bounds__(64 * kWaves) void rope_backward_kernel(RopeArgs a) {
  constexpr int RPI = Row<D>::RPI, LPR = Row<D>::LPR;
  __shared__ float sums[kWaves][2][D];
  const int r = lane_id() / LPR, d0 = 8 * (lane_id() % LPR);
  const Turn tn = make_turn<D>(a);
  const bool norm = a.wq != nullptr;
  const int rows_all = a.Hq + a.Hkv;
  float wq[8] = {}, wk[8] = {}, sq[8] = {}, sk[8] = {};
  if (norm) {
    load_weight<D>(a.wq, a.w_bf16, wq);
    load_weight<D>(a.wk, a.w_bf16, wk);
  }
  const uint32_t units = (uint32_t)a.T * (uint32_t)a.chunks;
  for (uint32_t u = blockIdx.x * kWaves + wave_id(); u < units; u += (uint32_t)a.wgs * kWaves) {
    const int t = (int)(u / (uint32_t)a.chunks), c = (int)(u - (uint32_t)t * a.chunks);
    const int row0 = c * a.rows, end = min(row0 + a.rows, rows_all);
    Raw<T> rx[NI], rg[NI];
#pragma unroll
    for (int it = 0; it < NI; ++it) {
      if (row0 + it * RPI >= end) break;
      const int h = min(row0 + it * RPI + r, end - 1);
      const bool k = h >= a.Hq;
      const int64_t head = (int64_t)(k ? h - a.Hq : h) * D + d0;
      rg[it] = load8<false, T>(k ? a.gk : a.gq, t * (k ? a.gk_stride : a.gq_stride) + head);
      if (norm) rx[it] = load8<false, T>(k ? a.k : a.q, t * (k ? a.k_stride : a.q_stride) + head);
    }
    const Angles g = load_angles<D>(a, tn, clamp_position(a, a.positions[t]));
#pragma unroll
    for (int it = 0; it < NI; ++it) {
      if (row0 + it * RPI >= end) break;
      const int h = row0 + it * RPI + r;
      const bool k = h >= a.Hq, live = h < end;
      float y[8];
      unpack(rg[it], y);
      turn<D>(tn, g, -1.f, y);
      if (norm) {
        float x[8];
        unpack(rx[it], x);
        const float rms = inv_rms<D>(x, a.eps);
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] *= rms;
          const float d = live ? y[i] * x[i] : 0.f;
          sq[i] += k ? 0.f : d;
          sk[i] += k ? d : 0.f;
          y[i] *= k ? wk[i] : wq[i];
          dot = fmaf(y[i], x[i], dot);
        }
        dot = group_sum<LPR>(dot) * (1.f / D);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = rms * (y[i] - x[i] * dot);
      }
      if (live) {
        const int64_t head = (int64_t)(k ? h - a.Hq : h) * D + d0;
        store8<STREAM>(k ? a.dk : a.dq, t * (k ? a.dk_stride : a.dq_stride) + head, a.out_bf16, y);
      }
    }
  }
  if (!norm) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int o = LPR; o < 64; o *= 2) {
      sq[i] += __shfl_xor(sq[i], o, 64);
      sk[i] += __shfl_xor(sk[i], o, 64);
    }
    if (r == 0) {
      sums[wave_id()][0][d0 + i] = sq[i];
      sums[wave_id()][1][d0 + i] = sk[i];
    }
  }
  __syncthreads();
  for (int i = (int)threadIdx.x; i < 2 * D; i += 64 * kWaves) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += sums[w][i / D][i % D];
    store_part(a.dw_part + (int64_t)blockIdx.x * 2 * D + i, x);
  }
  if (STREAM || !a.counts) return;  // calls that count are small
  parts_written();
  __syncthreads();
  uint64_t before = 0;
  if (threadIdx.x == 0) before = arrive(a.counts, a.epoch);
  if (!last_of(before, a.epoch, a.wgs)) return;
  // the parts' tree of rope_weight_grad_kernel, whose sums hold one part each here
  static_assert(kCountedWgs <= kSumRows && kSumRows == 64, "one part a sum");
  for (int i = (int)threadIdx.x; i < 2 * D; i += 64 * kWaves) {
    float v[8][8];
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        v[r][n] = load_part(a.dw_part + (int64_t)min(r + 8 * n, a.wgs - 1) * 2 * D + i);
        if (r + 8 * n >= a.wgs) v[r][n] = 0.f;
      }
    double x[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const float(&s)[8] = v[r];
      x[r] = (((double)s[0] + (double)s[4]) + ((double)s[2] + (double)s[6])) +
             (((double)s[1] + (double)s[5]) + ((double)s[3] + (double)s[7]));
    }
    const double y = ((x[0] + x[4]) + (x[2] + x[6])) + ((x[1] + x[5]) + (x[3] + x[7]));
    (i < D ? a.dwq : a.dwk)[i % D] = (float)y;
  }
}

// Sums the workgroups' parts in a fixed order: a workgroup per 16 dims of q's or
// k's weights, a row of parts for each 16 of its threads, four loads of a thread
// in flight.
__global__ __launch_bounds__(16 * kSumRows) void rope_weight_grad_kernel(RopeArgs a) {
  __shared__ double sums[kSumRows][16];
  const int i = (int)threadIdx.x % 16, r = (int)threadIdx.x / 16, at = (int)blockIdx.x * 16 + i;
  const float* part = a.dw_part + at;
  const int64_t row = 2 * a.D;
  double x = 0.;
  int g = r;
  for (; g + 3 * kSumRows < a.wgs; g += 4 * kSumRows) {
    float v[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) v[n] = part[(g + n * kSumRows) * row];
    x += ((double)v[0] + (double)v[1]) + ((double)v[2] + (double)v[3]);
  }
  for (; g < a.wgs; g += kSumRows) x += (double)part[g * row];
  sums[r][i] = x;
  __syncthreads();
  for (int n = kSumRows / 2; n > 0; n /= 2) {
    if (r < n) sums[r][i] += sums[r + n][i];
    __syncthreads();
  }
  if (r == 0) (at < a.D ? a.dwq : a.dwk)[at % a.D] = (float)sums[0][i];
}

// ------------------------------------------------------------- launches

template <typename K>
hipError_t launch(K kernel, int64_t wgs, const RopeArgs& a, hipStream_t s) {
  if (wgs <= 0) return hipSuccess;
  RopeArgs args = a;
  void* params[] = {&args};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)wgs), dim3(64 * kWaves), params, 0, s);
}

// Cuts a token's `heads` rows into equal chunks of whole wave iterations, at most ni each.
void cut(RopeArgs& a, int heads, int ni) {
  const int rpi = 64 / (a.D / 8), its = (heads + rpi - 1) / rpi;
  a.chunks = (its + ni - 1) / ni;
  a.rows = (its + a.chunks - 1) / a.chunks * rpi;
}

// Whether rope_token_kernel takes the call: rows of V written an element at a time,
// but no chain from tile to tile's tokens. us per call, rope_append_kernel /
// rope_token_kernel, 32 / 8 heads unless said: 512 x 2 tokens, 64 / 4 heads, bf16 19.0 / 12.1; 399 x 3
// bf16 18.5 / 16.1, f32 28.8 / 29.9; 399 x 4 20.9 / 21.3; 200 x 8 16.6 / 20.3; 100 x 16 12.9 /
// 18.8; 4 x 16 5.4 / 3.9; 4 x 32 5.5 / 4.3; 1 x 256, 32 / 4 heads, 5.6 / 4.6; 20 x 8 5.2 / 5.1.
template <KvType KV>
bool by_token(const RopeArgs& a) {
  return a.n == 1 || (KV != KvType::FP8 && a.n > 0 && (a.n <= 3 || (int64_t)a.T * a.Hkv <= 1024));
}

// Few rows a wave where that gives the compute units more waves than few. Calls of
// more rows also load and store past the caches (the gradient stores). us through them /
// past them, alone and between the copy that makes the inputs and what reads the results
// (append: prefill attention; others: a copy); 32 / 8 heads of 128 dims, bf16:
//   tokens            2,048                4,096                8,192            16,384          32,768
//   append     12.6 / 11.6, 71.5 / 70.3 19.0 / 21.7, 112 / 113 34.8 / 39.1, 214 / 212 84 / 75, 447 / 428 162 / 147, 1,079 / 1,055
//   forward    10.1 / 8.3, 25.8 / 25.5  19.0 / 14.8, 44 / 45   33.1 / 31.1, 93 / 92   69 / 61, 204 / 177 130 / 117, 382 / 361
//   gradient   19.7 / 19.0, 27.4 / 29.2 29.9 / 28.8, 44 / 47   50.9 / 49.0, 96 / 92   108 / 102, 183 / 187 208 / 201, 358 / 365
// The append's exceptions, around 30 MB of rotated queries, are larger for other types (f32, 2,048 tokens: 19.1 / 23.9;
// 16 / 4 heads of 64 dims, 16,384 tokens: 20.9 / 24.7, with the attention 152 / 153).
bool few(const RopeArgs& a, int heads) { return (int64_t)a.T * heads < 65536; }

template <typename T, KvType KV, int D>
hipError_t append_for(RopeArgs a, hipStream_t s) {
  if (by_token<KV>(a)) {
    cut(a, a.Hq, kFewRows);
    constexpr int rpi = Row<D>::RPI;
    const int64_t kv = (2 * (int64_t)a.T * ((a.Hkv + rpi - 1) / rpi) + kWaves - 1) / kWaves;
    return launch(&rope_token_kernel<T, KV, D>, kv + ((int64_t)a.T * a.chunks + kWaves - 1) / kWaves, a, s);
  }
  const bool f = few(a, a.Hq);
  cut(a, a.Hq, f ? kFewRows : kManyRows);
  const int64_t kv = 2 * (int64_t)a.tiles * a.Hkv / kWaves + 1;
  const int64_t q = ((int64_t)a.T * a.chunks + kWaves - 1) / kWaves;
  return f ? launch(&rope_append_kernel<T, KV, D, kFewRows>, kv + q, a, s)
           : launch(&rope_append_kernel<T, KV, D, kManyRows>, kv + q, a, s);
}

template <typename T, KvType KV>
hipError_t append_d(const RopeArgs& a, hipStream_t s) {
  return a.D == 64 ? append_for<T, KV, 64>(a, s) : append_for<T, KV, 128>(a, s);
}

template <typename T>
hipError_t append_kv(const RopeArgs& a, KvType kv, hipStream_t s) {
  return kv == KvType::F32 ? append_d<T, KvType::F32>(a, s)
         : kv == KvType::BF16 ? append_d<T, KvType::BF16>(a, s) : append_d<T, KvType::FP8>(a, s);
}

template <typename T, int D>
hipError_t rope_for(RopeArgs a, hipStream_t s) {
  const bool f = few(a, a.Hq + a.Hkv);
  cut(a, a.Hq + a.Hkv, f ? kFewRows : kManyRows);
  const int64_t wgs = ((int64_t)a.T * a.chunks + kWaves - 1) / kWaves;
  return f ? launch(&rope_kernel<T, D, kFewRows>, wgs, a, s) : launch(&rope_kernel<T, D, kManyRows>, wgs, a, s);
}

template <typename T, int D>
hipError_t backward_for(RopeArgs a, hipStream_t s) {
  cut(a, a.Hq + a.Hkv, kFewRows);
  const int64_t wgs = ((int64_t)a.T * a.chunks + kWaves - 1) / kWaves;
  if (wgs < a.wgs) a.wgs = (int32_t)wgs;
  const bool f = few(a, a.Hq + a.Hkv);
  if (!f || a.wgs == 0 || a.wgs > kCountedWgs) a.counts = nullptr;
  hipError_t e = f ? launch(&rope_backward_kernel<T, D, kFewRows, false>, a.wgs, a, s)
                   : launch(&rope_backward_kernel<T, D, kFewRows, true>, a.wgs, a, s);
  if (e != hipSuccess || !a.wq || a.counts) return e;
  RopeArgs args = a;
  void* params[] = {&args};
  return hipLaunchKernel(reinterpret_cast<const void*>(&rope_weight_grad_kernel), dim3(2 * a.D / 16),
                         dim3(16 * kSumRows), params, 0, s);
}

}  // namespace

hipError_t launch_rope_append(const RopeArgs& a, KvType kv, hipStream_t s) {
  return a.in_bf16 ? append_kv<uint16_t>(a, kv, s) : append_kv<float>(a, kv, s);
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t s) {
  if (a.in_bf16) return a.D == 64 ? rope_for<uint16_t, 64>(a, s) : rope_for<uint16_t, 128>(a, s);
  return a.D == 64 ? rope_for<float, 64>(a, s) : rope_for<float, 128>(a, s);
}

hipError_t launch_rope_backward(const RopeArgs& a, hipStream_t s) {
  if (a.in_bf16) return a.D == 64 ? backward_for<uint16_t, 64>(a, s) : backward_for<uint16_t, 128>(a, s);
  return a.D == 64 ? backward_for<float, 64>(a, s) : backward_for<float, 128>(a, s);
}

}  // namespace pda
