// Host side of include/comba_block.h: argument validation, workspace layout and
// kernel launches on the caller's stream.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "comba_block.h"
#include "comba_block_launch.h"

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxRow = (int64_t)1 << 22;  // 32-bit byte offsets inside 64 rows

size_t round_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
bool dtype_ok(comba_dtype d) { return d == COMBA_F32 || d == COMBA_BF16; }
size_t elem(comba_dtype d) { return d == COMBA_BF16 ? 2 : 4; }
comba_status done(hipError_t e) { return e == hipSuccess ? COMBA_OK : COMBA_ERR_HIP; }

// The elements between the `rows` rows of a named input: given, or contiguous.
bool row_stride(int64_t given, int64_t width, int64_t rows, bool tiles, long* row) {
  *row = given == 0 ? width : given;
  return *row >= width && *row <= (tiles ? kMaxRow : ((int64_t)1 << 60) / std::max<int64_t>(rows, 1));
}

// ---- linear attention with a decay per head -------------------------------------
// Rows, sequences and offsets as in comba.h; the longest sequence's tokens (packed
// without host offsets: all).
comba_status check_rows(const comba_decay_shape* s, comba::DecayArgs* a, int64_t* longest) {
  if (s->B < 0 || s->T < 0 || s->num_seqs < 0) return COMBA_ERR_SHAPE;
  int64_t ttot = s->T;
  if (s->cu_seqlens) {
    if (s->B != 1) return COMBA_ERR_SHAPE;
    *longest = s->T;
    if (const int32_t* cu = s->cu_seqlens_host) {
      *longest = 0;
      if (cu[0] != 0 || cu[s->num_seqs] != s->T) return COMBA_ERR_SHAPE;
      for (int i = 0; i < s->num_seqs; ++i) {
        if (cu[i + 1] < cu[i]) return COMBA_ERR_SHAPE;
        *longest = std::max<int64_t>(*longest, cu[i + 1] - cu[i]);
      }
    }
  } else {
    if (s->cu_seqlens_host || s->num_seqs != s->B) return COMBA_ERR_SHAPE;
    ttot *= s->B;
    a->Tseq = s->T;
    *longest = s->T;
  }
  if (ttot > INT32_MAX / 2 || s->num_seqs > (1 << 24)) return COMBA_ERR_SHAPE;
  if (ttot > 0 && s->num_seqs == 0) return COMBA_ERR_SHAPE;  // tokens must belong to a sequence
  a->cu_seqlens = s->cu_seqlens;
  a->S = s->num_seqs;
  a->Ttot = (int)ttot;
  return COMBA_OK;
}

// Sequences that run as segments of `seglen` tokens side by side.  A scan's workgroup takes
// about 1 us a chunk; the first pass, which finds the segments' states, adds its own walk
// and a launch.  So a sequence is cut where its own walk is longer than two shares of a CU
// and some, into segments of which every CU gets two.  Whole / cut, us of a forward, 16
// heads of 128: one row of 4,096 tokens 74 / 57, of 16,384 296 / 184; two rows of 4,096
// 88 / 88, four 156 / 198; ten packed sequences of 1 to 15,777 tokens, 36,383 in all,
// 436 / 422 (whole here: a lower limit won 2 to 3% on such batches and nothing elsewhere);
// 4 heads, one row of 65,536 846 / 193.  (Packed without host offsets: as if one sequence
// had all tokens; what is shorter than a segment stays whole.)
void cut(comba::DecayArgs* a, int64_t longest, bool* segments) {
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    cus = 256;
  const int64_t share = (int64_t)a->Ttot * a->H * comba::decay_splits(a->dv) / cus;
  const int64_t len = std::max<int64_t>((share / 2 + 63) / 64 * 64, 256);
  *segments = longest > 2 * share + 600 && longest > len;
  a->seglen = *segments ? (int)len : a->cu_seqlens ? 1 << 30 : std::max(a->Tseq, 1);
}

comba_status decay_args(const comba_decay_shape* s, comba::DecayArgs* a, bool* segments, bool tiles = true) {
  if (!s) return COMBA_ERR_NULL;
  if (!dtype_ok(s->in_dtype) || !dtype_ok(s->g_dtype)) return COMBA_ERR_DTYPE;
  if (s->g_dtype != COMBA_F32 && (s->g_dtype != s->in_dtype || s->g_per_head)) return COMBA_ERR_DTYPE;
  if (s->H < 1 || s->H > 65535 || s->Hq < 1 || s->Hk < 1 || s->Hv < 1 || s->H % s->Hq || s->H % s->Hk ||
      s->H % s->Hv || s->dk < 1 || s->dk > 256 || s->dv < 1 || s->dv > 256)
    return COMBA_ERR_SHAPE;
  *a = comba::DecayArgs{};
  int64_t longest = 0;
  const comba_status st = check_rows(s, a, &longest);
  if (st != COMBA_OK) return st;
  a->bf16 = s->in_dtype == COMBA_BF16;
  a->g_f32 = s->g_dtype == COMBA_F32;
  a->g_head = s->g_per_head != 0;
  a->H = s->H;
  a->Hq = s->Hq;
  a->Hk = s->Hk;
  a->Hv = s->Hv;
  a->dk = s->dk;
  a->dv = s->dv;
  a->scale = s->scale;
  const int64_t rows = a->Ttot;
  if (!row_stride(s->q_row, (int64_t)s->Hq * s->dk, rows, tiles, &a->q_row) ||
      !row_stride(s->k_row, (int64_t)s->Hk * s->dk, rows, tiles, &a->k_row) ||
      !row_stride(s->v_row, (int64_t)s->Hv * s->dv, rows, tiles, &a->v_row) ||
      !row_stride(s->g_row, s->H, rows, tiles, &a->g_row))
    return COMBA_ERR_SHAPE;
  if (tiles && (int64_t)s->H * std::max(s->dk, s->dv) > kMaxRow) return COMBA_ERR_SHAPE;
  if (tiles) {
    cut(a, longest, segments);
    // workgroups of a launch, which holds fewer than 2^31 threads
    const int64_t most = INT32_MAX / 512 - 64;
    if (comba::decay_slots(*a, a->seglen) > most / ((int64_t)a->H * comba::decay_splits(a->dv)) ||
        comba::decay_slots(*a, comba::DC_CH) > most / a->H)
      return COMBA_ERR_SHAPE;
  }
  return COMBA_OK;
}

struct DecayLayout {
  size_t kept, segS, segG, met, pq, pk, pv, total;
};
enum class Use { kFwd, kSave, kBwd };

size_t kept_bytes(const comba::DecayArgs& a) {
  return (size_t)comba::decay_slots(a, comba::DC_CH) * a.H * comba::state_bytes(a.bf16, a.dk, a.dv);
}
DecayLayout decay_layout(const comba::DecayArgs& a, bool segments, Use use) {
  DecayLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += round_up(bytes);
    return at;
  };
  L.kept = take(kept_bytes(a));
  const size_t slots = segments ? (size_t)comba::decay_slots(a, a.seglen) * a.H : 0;
  L.segS = take(slots * comba::decay_end_floats(a) * sizeof(float));
  L.segG = take(slots * sizeof(float));
  if (use == Use::kBwd) {
    const size_t n = (size_t)a.Ttot * a.H * sizeof(float);
    L.met = take((size_t)comba::decay_slots(a, comba::DC_CH) * a.H * comba::decay_splits(a.dv) * 8 * sizeof(float));
    L.pq = take(a.Hq < a.H ? n * a.dk : 0);
    L.pk = take(a.Hk < a.H ? n * a.dk : 0);
    L.pv = take(a.Hv < a.H ? n * a.dv : 0);
  }
  L.total = off + kAlign;
  return L;
}
size_t decay_bytes(const comba_decay_shape* shape, Use use) {
  comba::DecayArgs a;
  bool segments;
  return decay_args(shape, &a, &segments) == COMBA_OK ? decay_layout(a, segments, use).total : 0;
}
void set_segments(comba::DecayArgs* a, const DecayLayout& L, bool segments, char* base) {
  if (!segments) return;
  a->segS = reinterpret_cast<float*>(base + L.segS);
  a->segG = reinterpret_cast<float*>(base + L.segG);
}

comba_status decay_inputs(comba::DecayArgs* a, const void* q, const void* k, const void* v, const void* g,
                          const float* h0) {
  const size_t e = a->bf16 ? 2 : 4;
  if (((a->g_head || a->Ttot > 0) && !g) || (a->Ttot > 0 && (!q || !k || !v))) return COMBA_ERR_NULL;
  if (!aligned(q, e) || !aligned(k, e) || !aligned(v, e) || !aligned(g, a->g_f32 ? 4 : 2) || !aligned(h0, 4))
    return COMBA_ERR_ALIGN;
  a->q = q;
  a->k = k;
  a->v = v;
  a->g = g;
  a->h0 = h0;
  return COMBA_OK;
}

comba_status decay_fwd(Use use, const comba_decay_shape* shape, const void* q, const void* k, const void* v,
                       const void* g, const float* h0, void* o, float* ht, void* ws, size_t ws_bytes,
                       void* stream) {
  comba::DecayArgs a;
  bool segments;
  comba_status st = decay_args(shape, &a, &segments);
  if (st != COMBA_OK) return st;
  st = decay_inputs(&a, q, k, v, g, h0);
  if (st != COMBA_OK) return st;
  if ((a.Ttot > 0 && !o) || !ws) return COMBA_ERR_NULL;
  if (!aligned(o, a.bf16 ? 2 : 4) || !aligned(ht, 4) || !aligned(ws, kAlign)) return COMBA_ERR_ALIGN;
  const DecayLayout L = decay_layout(a, segments, use);
  if (ws_bytes < L.total) return COMBA_ERR_WORKSPACE;
  char* base = static_cast<char*>(ws);
  a.o = o;
  a.ht = ht;
  a.kept = base + L.kept;
  set_segments(&a, L, segments, base);
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_decay_fwd(a));
}

// ---- norms after and before a block ------------------------------------------------
comba_status block_norm_args(const comba_block_norm_shape* s, comba::BlockNormArgs* a) {
  if (!s) return COMBA_ERR_NULL;
  if (!dtype_ok(s->dtype) || !dtype_ok(s->x_dtype)) return COMBA_ERR_DTYPE;
  if (s->x_dtype != s->dtype && s->x_dtype != COMBA_F32) return COMBA_ERR_DTYPE;
  if (s->activation != COMBA_ACT_NONE && s->activation != COMBA_ACT_SILU && s->activation != COMBA_ACT_SIGMOID)
    return COMBA_ERR_SHAPE;
  if (s->rows < 0 || s->rows > INT32_MAX || s->C <= 0 || s->C > kMaxRow || !(s->eps >= 0.f)) return COMBA_ERR_SHAPE;
  *a = comba::BlockNormArgs{};
  a->bf16 = s->dtype == COMBA_BF16;
  a->x_bf16 = s->x_dtype == COMBA_BF16;
  a->act = s->activation;
  a->rows = s->rows;
  a->C = s->C;
  a->eps = s->eps;
  return row_stride(s->y_row, s->C, s->rows, false, &a->y_row) && row_stride(s->z_row, s->C, s->rows, false, &a->z_row) &&
                 row_stride(s->x_row, s->C, s->rows, false, &a->x_row)
             ? COMBA_OK
             : COMBA_ERR_SHAPE;
}

comba_status block_norm_inputs(comba::BlockNormArgs* a, const comba_block_norm_shape* s, const void* y, const void* x,
                               const void* z, const float* w1, const float* sc, const float* w2) {
  if (a->rows > 0 && !y) return COMBA_ERR_NULL;
  if (!aligned(y, elem(s->dtype)) || !aligned(z, elem(s->dtype)) || !aligned(x, elem(s->x_dtype)) || !aligned(w1, 4) ||
      !aligned(sc, 4) || !aligned(w2, 4))
    return COMBA_ERR_ALIGN;
  a->y = y;
  a->x = x;
  a->z = z;
  a->w1 = w1;
  a->sc = sc;
  a->w2 = w2;
  return COMBA_OK;
}

size_t block_norm_ws_bytes(const comba::BlockNormArgs& a) {
  return round_up((size_t)comba::block_norm_bwd_blocks(a) * 3 * a.C * sizeof(float)) + kAlign;
}

}  // namespace

extern "C" {

size_t comba_decay_fwd_workspace_bytes(const comba_decay_shape* shape) { return decay_bytes(shape, Use::kFwd); }
size_t comba_decay_save_bytes(const comba_decay_shape* shape) { return decay_bytes(shape, Use::kSave); }
size_t comba_decay_bwd_workspace_bytes(const comba_decay_shape* shape) { return decay_bytes(shape, Use::kBwd); }

comba_status comba_decay_fwd(const comba_decay_shape* shape, const void* q, const void* k, const void* v,
                             const void* g, const float* h0, void* o, float* ht, void* ws, size_t ws_bytes,
                             void* stream) {
  return decay_fwd(Use::kFwd, shape, q, k, v, g, h0, o, ht, ws, ws_bytes, stream);
}

comba_status comba_decay_fwd_save(const comba_decay_shape* shape, const void* q, const void* k, const void* v,
                                  const void* g, const float* h0, void* o, float* ht, void* ws, size_t ws_bytes,
                                  void* stream) {
  return decay_fwd(Use::kSave, shape, q, k, v, g, h0, o, ht, ws, ws_bytes, stream);
}

comba_status comba_decay_bwd(const comba_decay_shape* shape, const void* q, const void* k, const void* v,
                             const void* g, const float* h0, const void* dO, const float* dht, void* dq, void* dk,
                             void* dv, void* dg, float* dh0, const void* saved, size_t saved_bytes, void* ws,
                             size_t ws_bytes, void* stream) {
  comba::DecayArgs a;
  bool segments;
  comba_status st = decay_args(shape, &a, &segments);
  if (st != COMBA_OK) return st;
  st = decay_inputs(&a, q, k, v, g, h0);
  if (st != COMBA_OK) return st;
  if (a.g_head && dg) return COMBA_ERR_SHAPE;
  if (!saved || !ws || (a.Ttot > 0 && (!dO || !dq || !dk || !dv))) return COMBA_ERR_NULL;
  const size_t e = a.bf16 ? 2 : 4;
  if (!aligned(dO, e) || !aligned(dht, 4) || !aligned(dq, e) || !aligned(dk, e) || !aligned(dv, e) ||
      !aligned(dg, a.g_f32 ? 4 : 2) || !aligned(dh0, 4) || !aligned(saved, kAlign) || !aligned(ws, kAlign))
    return COMBA_ERR_ALIGN;
  const DecayLayout L = decay_layout(a, segments, Use::kBwd);
  if (saved_bytes < kept_bytes(a) || ws_bytes < L.total) return COMBA_ERR_WORKSPACE;
  char* base = static_cast<char*>(ws);
  a.kept = const_cast<void*>(saved);
  a.dkept = base + L.kept;
  set_segments(&a, L, segments, base);
  a.met = reinterpret_cast<float*>(base + L.met);
  a.pq = a.Hq < a.H ? reinterpret_cast<float*>(base + L.pq) : nullptr;
  a.pk = a.Hk < a.H ? reinterpret_cast<float*>(base + L.pk) : nullptr;
  a.pv = a.Hv < a.H ? reinterpret_cast<float*>(base + L.pv) : nullptr;
  a.dO = dO;
  a.dht = dht;
  a.dq = dq;
  a.dk_ = dk;
  a.dv_ = dv;
  a.dg = dg;
  a.dh0 = dh0;
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_decay_bwd(a));
}

comba_status comba_decay_step(const comba_decay_shape* shape, const void* q, const void* k, const void* v,
                              const void* g, float* state, const int32_t* slots, int32_t num_slots, void* o,
                              void* stream) {
  comba::DecayArgs a;
  bool segments;
  comba_status st = decay_args(shape, &a, &segments, false);
  if (st != COMBA_OK) return st;
  if (a.cu_seqlens || shape->T != 1 || num_slots < 0) return COMBA_ERR_SHAPE;
  if (a.S > (int)(UINT32_MAX / 256)) return COMBA_ERR_SHAPE;  // threads of a launch, 256 a row
  st = decay_inputs(&a, q, k, v, g, nullptr);
  if (st != COMBA_OK) return st;
  if (a.S > 0 && (!state || !o)) return COMBA_ERR_NULL;
  if (!aligned(o, a.bf16 ? 2 : 4) || !aligned(state, 4) || !aligned(slots, 4)) return COMBA_ERR_ALIGN;
  a.state = state;
  a.slots = slots;
  a.num_slots = num_slots;
  a.o = o;
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_decay_step(a));
}

comba_status comba_block_norm_fwd(const comba_block_norm_shape* shape, const void* y, const void* x, const void* z,
                                  const float* post_weight, const float* scale, const float* weight, void* r, void* n,
                                  void* stream) {
  comba::BlockNormArgs a;
  comba_status st = block_norm_args(shape, &a);
  if (st != COMBA_OK) return st;
  st = block_norm_inputs(&a, shape, y, x, z, post_weight, scale, weight);
  if (st != COMBA_OK) return st;
  if (a.rows > 0 && (!r || (weight && !n))) return COMBA_ERR_NULL;
  if (!aligned(r, elem(shape->x_dtype)) || !aligned(n, elem(shape->dtype))) return COMBA_ERR_ALIGN;
  a.r = r;
  a.n = n;
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_block_norm_fwd(a));
}

size_t comba_block_norm_workspace_bytes(const comba_block_norm_shape* shape) {
  comba::BlockNormArgs a;
  return block_norm_args(shape, &a) == COMBA_OK ? block_norm_ws_bytes(a) : 0;
}

comba_status comba_block_norm_bwd(const comba_block_norm_shape* shape, const void* y, const void* x, const void* z,
                                  const float* post_weight, const float* scale, const float* weight, const void* dr,
                                  const void* dn, void* dy, void* dx, void* dz, float* dpost_weight, float* dscale,
                                  float* dweight, void* ws, size_t ws_bytes, void* stream) {
  comba::BlockNormArgs a;
  comba_status st = block_norm_args(shape, &a);
  if (st != COMBA_OK) return st;
  st = block_norm_inputs(&a, shape, y, x, z, post_weight, scale, weight);
  if (st != COMBA_OK) return st;
  if (!ws || (a.rows > 0 && (!dy || (z && !dz)))) return COMBA_ERR_NULL;
  const size_t e = elem(shape->dtype), ex = elem(shape->x_dtype);
  if (!aligned(dr, ex) || !aligned(dn, e) || !aligned(dy, e) || !aligned(dx, ex) || !aligned(dz, e) ||
      !aligned(dpost_weight, 4) || !aligned(dscale, 4) || !aligned(dweight, 4) || !aligned(ws, kAlign))
    return COMBA_ERR_ALIGN;
  if (ws_bytes < block_norm_ws_bytes(a)) return COMBA_ERR_WORKSPACE;
  a.dr = dr;
  a.dn = weight ? dn : nullptr;
  a.dy = dy;
  a.dx = x ? dx : nullptr;
  a.dz = dz;
  a.dw1 = post_weight ? dpost_weight : nullptr;
  a.dsc = scale ? dscale : nullptr;
  a.dw2 = weight ? dweight : nullptr;
  a.part = static_cast<float*>(ws);
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_block_norm_bwd(a));
}

}  // extern "C"
