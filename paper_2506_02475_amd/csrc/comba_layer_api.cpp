// Host side of include/comba_layer.h: argument validation, workspace layout and
// kernel launches on the caller's stream.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "comba_layer.h"
#include "comba_layer_launch.h"

namespace {

constexpr size_t kAlign = 256;

size_t round_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

bool dtype_ok(comba_dtype d) { return d == COMBA_F32 || d == COMBA_BF16; }
size_t elem(comba_dtype d) { return d == COMBA_BF16 ? 2 : 4; }
comba_status done(hipError_t e) { return e == hipSuccess ? COMBA_OK : COMBA_ERR_HIP; }

// Rows, sequences and offsets, as in comba.h.
struct Rows {
  int S, Tseq, Ttot;
  long longest;  // tokens of the longest sequence (packed: 0 without the host offsets)
};

template <typename Shape>
comba_status check_rows(const Shape* s, Rows* r) {
  if (s->B < 0 || s->T < 0 || s->num_seqs < 0) return COMBA_ERR_SHAPE;
  int64_t ttot;
  if (s->cu_seqlens) {
    if (s->B != 1) return COMBA_ERR_SHAPE;
    ttot = s->T;
    r->Tseq = 0;
    r->longest = 0;
    if (const int32_t* cu = s->cu_seqlens_host) {
      if (cu[0] != 0 || cu[s->num_seqs] != s->T) return COMBA_ERR_SHAPE;
      for (int i = 0; i < s->num_seqs; ++i) {
        if (cu[i + 1] < cu[i]) return COMBA_ERR_SHAPE;
        if (cu[i + 1] - cu[i] > r->longest) r->longest = cu[i + 1] - cu[i];
      }
    }
  } else {
    if (s->cu_seqlens_host || s->num_seqs != s->B) return COMBA_ERR_SHAPE;
    ttot = (int64_t)s->B * s->T;
    r->Tseq = s->T;
    r->longest = s->T;
  }
  if (ttot > INT32_MAX / 2 || s->num_seqs > (1 << 24)) return COMBA_ERR_SHAPE;
  if (ttot > 0 && s->num_seqs == 0) return COMBA_ERR_SHAPE;  // tokens must belong to a sequence
  r->S = s->num_seqs;
  r->Ttot = (int)ttot;
  return COMBA_OK;
}

// Rows of up to 4M values: the byte offsets inside a tile of 96 rows stay below 2^31.
constexpr int64_t kMaxRow = (int64_t)1 << 22;

// The elements between rows of a named input: given, or contiguous.
bool row_stride(int64_t given, int64_t width, long* row) {
  *row = given == 0 ? width : given;
  return *row >= width && *row <= kMaxRow;
}

// ---- convolution -------------------------------------------------------------
comba_status conv_args(const comba_conv_shape* s, comba::ConvArgs* a) {
  if (!s) return COMBA_ERR_NULL;
  if (!dtype_ok(s->in_dtype)) return COMBA_ERR_DTYPE;
  if (s->activation != COMBA_ACT_NONE && s->activation != COMBA_ACT_SILU) return COMBA_ERR_SHAPE;
  if (s->K < 2 || s->K > 4 || s->D <= 0 || s->D > kMaxRow) return COMBA_ERR_SHAPE;
  Rows r{};
  const comba_status st = check_rows(s, &r);
  if (st != COMBA_OK) return st;
  *a = comba::ConvArgs{};
  a->bf16 = s->in_dtype == COMBA_BF16;
  a->silu = s->activation == COMBA_ACT_SILU;
  a->D = s->D;
  a->K = s->K;
  a->N = r.S;
  a->Tseq = r.Tseq;
  a->Ttot = r.Ttot;
  a->cu_seqlens = s->cu_seqlens;
  return row_stride(s->x_row, s->D, &a->x_row) ? COMBA_OK : COMBA_ERR_SHAPE;
}

size_t conv_ws_bytes(const comba::ConvArgs& a) {
  return round_up((size_t)comba::conv_bwd_runs(a) * (a.K + 1) * a.D * sizeof(float)) + kAlign;
}

// ---- selective scan -----------------------------------------------------------
struct SelectLayout {
  size_t ck, bcp, dap, segF, segdt, total;
};

// Cuts rows into segments when their workgroups, one per CU, leave CUs idle or
// wait for a long row: the main kernel then runs over segments side by side,
// after a first pass over all but one segment of each row that is cut (`pre` of
// the main kernel's time per token).  Packed rows of up to a CU's share of all
// tokens stay whole.  Takes the number with the least time, counted in tokens
// walked one after the other (`launch`: the first pass's launch and the
// segments' starts).  Measured, whole rows / segments, us: 16 states, one row of
// 8,192 tokens, 2,048 channels: forward 387 / 167, backward 1,022 / 361; 1,000
// tokens: forward 54 / 31; 4 rows of 4,096, which fill the CUs: 219 whole, 297 to
// 321 cut.
void select_segments(comba::SelectArgs* a, bool bwd) {
  a->segs = 1;
  a->seglen = a->segmin = 1 << 30;
  const int64_t tile = comba::select_tile(a->N);
  if (a->longest < 2 * tile || a->S == 0) return;  // short, or not known
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    return;
  const double pre = bwd ? 0.25 : 0.6, launch = bwd ? 64 : 128;
  const double blocks = (double)a->G * a->nblk, share = (double)a->Ttot * blocks / cus;
  auto rounds = [&](double rows) { return (double)(((int64_t)(rows * blocks) + cus - 1) / cus); };
  const double longest = (double)a->longest;
  if (a->cu_host && longest <= share) return;
  double best = a->cu_host ? longest : rounds(a->S) * longest;
  for (int p = 2; p <= 32; p *= 2) {
    const int64_t len = (a->longest + p * tile - 1) / (p * tile) * tile, n = (a->longest + len - 1) / len;
    if (n < 2) break;
    double t = launch;
    if (!a->cu_host) {
      t += (rounds((double)a->S * n) + pre * rounds((double)a->S * (n - 1))) * (double)len;
    } else {
      int64_t first = 0;  // tokens of the first pass
      for (int i = 0; i < a->S; ++i) {
        const int64_t tokens = a->cu_host[i + 1] - a->cu_host[i];
        if ((double)tokens > share) first += (tokens - 1) / len * len;
      }
      const double f = (double)first * blocks / cus;
      t += ((double)len > share ? (double)len : share) + pre * ((double)len > f ? (double)len : f);
    }
    if (t < best && (int64_t)a->S * n * a->G * a->nblk <= INT32_MAX) {
      best = t;
      a->segs = (int)n;
      a->seglen = (int)len;
      a->segmin = a->cu_host ? (int)share : 0;
    }
  }
}

// Workspace of a forward, or (save) of a saving forward and its backward, whose
// segments are chosen apart.
SelectLayout select_layout(const comba::SelectArgs& a0, bool save) {
  comba::SelectArgs a = a0;
  SelectLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += round_up(bytes);
    return at;
  };
  select_segments(&a, false);
  size_t segs = a.segs;
  if (save) {
    select_segments(&a, true);
    // states: a sequence's start at tok0 / select_ck + its number, which leaves
    // room for a partial interval per sequence
    L.ck = take(((size_t)a.Ttot / comba::select_ck(a.N) + a.S + 1) * a.D * a.N * sizeof(float));
    L.bcp = take((size_t)a.G * a.nblk * a.Ttot * 2 * a.N * sizeof(float));
    L.dap = take((size_t)a.S * a.segs * a.D * (a.N + 2) * sizeof(float));
    if ((size_t)a.segs > segs) segs = a.segs;
  }
  const size_t rows = segs > 1 ? (size_t)a.S * segs * a.D : 0;
  L.segF = take(rows * a.N * sizeof(float));
  L.segdt = take(rows * sizeof(float));
  L.total = off + kAlign;
  return L;
}

comba_status select_args(const comba_select_shape* s, comba::SelectArgs* a) {
  if (!s) return COMBA_ERR_NULL;
  if (!dtype_ok(s->in_dtype)) return COMBA_ERR_DTYPE;
  if (s->N != 8 && s->N != 16 && s->N != 32) return COMBA_ERR_SHAPE;
  if (s->D <= 0 || s->D > kMaxRow || s->G <= 0 || s->D % s->G) return COMBA_ERR_SHAPE;
  Rows r{};
  const comba_status st = check_rows(s, &r);
  if (st != COMBA_OK) return st;
  *a = comba::SelectArgs{};
  a->bf16 = s->in_dtype == COMBA_BF16;
  a->softplus = s->delta_softplus != 0;
  a->D = s->D;
  a->N = s->N;
  a->G = s->G;
  a->S = r.S;
  a->Tseq = r.Tseq;
  a->Ttot = r.Ttot;
  a->longest = r.longest;
  a->cu_host = s->cu_seqlens ? s->cu_seqlens_host : nullptr;
  a->cu_seqlens = s->cu_seqlens;
  const int bc = comba::select_block_channels(s->N);
  a->nblk = (s->D / s->G + bc - 1) / bc;
  if ((int64_t)a->S * a->G * a->nblk > INT32_MAX) return COMBA_ERR_SHAPE;
  const int64_t gn = (int64_t)s->G * s->N;
  if (!row_stride(s->u_row, s->D, &a->u_row) || !row_stride(s->delta_row, s->D, &a->delta_row) ||
      !row_stride(s->z_row, s->D, &a->z_row) || !row_stride(s->b_row, gn, &a->b_row) ||
      !row_stride(s->c_row, gn, &a->c_row))
    return COMBA_ERR_SHAPE;
  return COMBA_OK;
}

comba_status select_inputs(comba::SelectArgs* a, const void* u, const void* delta, const float* A,
                           const void* Bm, const void* Cm, const float* Dskip, const void* z,
                           const float* bias, const float* h0) {
  const size_t e = a->bf16 ? 2 : 4;
  if (!A || (a->Ttot > 0 && (!u || !delta || !Bm || !Cm))) return COMBA_ERR_NULL;
  if (!aligned(u, e) || !aligned(delta, e) || !aligned(Bm, e) || !aligned(Cm, e) || !aligned(z, e) ||
      !aligned(A, 4) || !aligned(Dskip, 4) || !aligned(bias, 4) || !aligned(h0, 4))
    return COMBA_ERR_ALIGN;
  a->u = u;
  a->delta = delta;
  a->A = A;
  a->Bm = Bm;
  a->Cm = Cm;
  a->Dskip = Dskip;
  a->z = z;
  a->bias = bias;
  a->h0 = h0;
  return COMBA_OK;
}

comba_status select_fwd(bool save, const comba_select_shape* shape, const void* u, const void* delta,
                        const float* A, const void* Bm, const void* Cm, const float* Dskip,
                        const void* z, const float* bias, const float* h0, void* y, float* ht,
                        void* ws, size_t ws_bytes, void* stream) {
  comba::SelectArgs a;
  comba_status st = select_args(shape, &a);
  if (st != COMBA_OK) return st;
  st = select_inputs(&a, u, delta, A, Bm, Cm, Dskip, z, bias, h0);
  if (st != COMBA_OK) return st;
  if ((a.Ttot > 0 && !y) || !ws) return COMBA_ERR_NULL;
  if (!aligned(y, a.bf16 ? 2 : 4) || !aligned(ht, 4) || !aligned(ws, kAlign)) return COMBA_ERR_ALIGN;
  const SelectLayout L = select_layout(a, save);
  if (ws_bytes < L.total) return COMBA_ERR_WORKSPACE;
  a.y = y;
  a.ht = ht;
  char* base = static_cast<char*>(ws);
  if (save) a.ck = reinterpret_cast<float*>(base + L.ck);
  select_segments(&a, false);
  a.segF = reinterpret_cast<float*>(base + L.segF);
  a.segdt = reinterpret_cast<float*>(base + L.segdt);
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_select_fwd(a));
}

// ---- group norm ---------------------------------------------------------------
comba_status group_norm_args(const comba_group_norm_shape* s, comba::GroupNormArgs* a) {
  if (!s) return COMBA_ERR_NULL;
  if (!dtype_ok(s->x_dtype) || !dtype_ok(s->out_dtype)) return COMBA_ERR_DTYPE;
  if (s->x_dtype != s->out_dtype && s->x_dtype != COMBA_F32) return COMBA_ERR_DTYPE;
  if (s->activation != COMBA_ACT_NONE && s->activation != COMBA_ACT_SILU &&
      s->activation != COMBA_ACT_SIGMOID)
    return COMBA_ERR_SHAPE;
  if (s->rows < 0 || s->rows > INT32_MAX || s->C <= 0 || s->C > kMaxRow || s->G <= 0 || s->C % s->G)
    return COMBA_ERR_SHAPE;
  if (!(s->eps >= 0.f)) return COMBA_ERR_SHAPE;
  *a = comba::GroupNormArgs{};
  a->x_bf16 = s->x_dtype == COMBA_BF16;
  a->out_bf16 = s->out_dtype == COMBA_BF16;
  a->act = s->activation;
  a->rows = s->rows;
  a->C = s->C;
  a->G = s->G;
  a->eps = s->eps;
  return row_stride(s->x_row, s->C, &a->x_row) && row_stride(s->z_row, s->C, &a->z_row) ? COMBA_OK
                                                                                       : COMBA_ERR_SHAPE;
}

comba_status group_norm_inputs(comba::GroupNormArgs* a, const comba_group_norm_shape* s, const void* x,
                               const float* w, const float* b, const void* z) {
  if (a->rows > 0 && !x) return COMBA_ERR_NULL;
  if (!aligned(x, elem(s->x_dtype)) || !aligned(z, elem(s->out_dtype)) || !aligned(w, 4) || !aligned(b, 4))
    return COMBA_ERR_ALIGN;
  a->x = x;
  a->w = w;
  a->b = b;
  a->z = z;
  return COMBA_OK;
}

size_t group_norm_ws_bytes(const comba::GroupNormArgs& a) {
  return round_up((size_t)comba::group_norm_bwd_blocks(a) * 2 * a.C * sizeof(float)) + kAlign;
}

}  // namespace

extern "C" {

comba_status comba_conv_fwd(const comba_conv_shape* shape, const void* x, const float* w,
                            const float* bias, const void* h0, void* y, void* ht, void* stream) {
  comba::ConvArgs a;
  const comba_status st = conv_args(shape, &a);
  if (st != COMBA_OK) return st;
  if (!w || (a.Ttot > 0 && (!x || !y))) return COMBA_ERR_NULL;
  const size_t e = a.bf16 ? 2 : 4;
  if (!aligned(x, e) || !aligned(y, e) || !aligned(h0, e) || !aligned(ht, e) || !aligned(w, 4) ||
      !aligned(bias, 4))
    return COMBA_ERR_ALIGN;
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.h0 = h0;
  a.y = y;
  a.ht = ht;
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_conv_fwd(a));
}

size_t comba_conv_workspace_bytes(const comba_conv_shape* shape) {
  comba::ConvArgs a;
  return conv_args(shape, &a) == COMBA_OK ? conv_ws_bytes(a) : 0;
}

comba_status comba_conv_bwd(const comba_conv_shape* shape, const void* x, const float* w,
                            const float* bias, const void* h0, const void* dy, const void* dht,
                            void* dx, float* dw, float* dbias, void* dh0, void* ws,
                            size_t ws_bytes, void* stream) {
  comba::ConvArgs a;
  const comba_status st = conv_args(shape, &a);
  if (st != COMBA_OK) return st;
  if (!w || !dw || !ws || (bias && !dbias) || (a.Ttot > 0 && (!x || !dy || !dx))) return COMBA_ERR_NULL;
  const size_t e = a.bf16 ? 2 : 4;
  if (!aligned(x, e) || !aligned(h0, e) || !aligned(dy, e) || !aligned(dht, e) || !aligned(dx, e) ||
      !aligned(dh0, e) || !aligned(w, 4) || !aligned(bias, 4) || !aligned(dw, 4) ||
      !aligned(dbias, 4) || !aligned(ws, kAlign))
    return COMBA_ERR_ALIGN;
  if (ws_bytes < conv_ws_bytes(a)) return COMBA_ERR_WORKSPACE;
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.h0 = h0;
  a.dy = dy;
  a.dht = dht;
  a.dx = dx;
  a.dw = dw;
  a.dbias = bias ? dbias : nullptr;
  a.dh0 = dh0;
  a.part = static_cast<float*>(ws);
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_conv_bwd(a));
}

comba_status comba_conv_step(const comba_conv_shape* shape, const void* x, const float* w,
                             const float* bias, void* state, const int32_t* slots,
                             int32_t num_slots, void* y, void* stream) {
  comba::ConvArgs a;
  const comba_status st = conv_args(shape, &a);
  if (st != COMBA_OK) return st;
  if (a.cu_seqlens || shape->T != 1 || num_slots < 0) return COMBA_ERR_SHAPE;
  if (a.N > 0 && (!x || !w || !state || !y)) return COMBA_ERR_NULL;
  const size_t e = a.bf16 ? 2 : 4;
  if (!aligned(x, e) || !aligned(y, e) || !aligned(state, e) || !aligned(w, 4) || !aligned(bias, 4) ||
      !aligned(slots, 4))
    return COMBA_ERR_ALIGN;
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.state = state;
  a.slots = slots;
  a.num_slots = num_slots;
  a.y = y;
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_conv_step(a));
}

size_t comba_select_fwd_workspace_bytes(const comba_select_shape* shape) {
  comba::SelectArgs a;
  return select_args(shape, &a) == COMBA_OK ? select_layout(a, false).total : 0;
}

size_t comba_select_bwd_workspace_bytes(const comba_select_shape* shape) {
  comba::SelectArgs a;
  return select_args(shape, &a) == COMBA_OK ? select_layout(a, true).total : 0;
}

comba_status comba_select_fwd(const comba_select_shape* shape, const void* u, const void* delta,
                              const float* A, const void* Bm, const void* Cm, const float* Dskip,
                              const void* z, const float* delta_bias, const float* h0, void* y,
                              float* ht, void* ws, size_t ws_bytes, void* stream) {
  return select_fwd(false, shape, u, delta, A, Bm, Cm, Dskip, z, delta_bias, h0, y, ht, ws, ws_bytes,
                    stream);
}

comba_status comba_select_fwd_save(const comba_select_shape* shape, const void* u,
                                   const void* delta, const float* A, const void* Bm,
                                   const void* Cm, const float* Dskip, const void* z,
                                   const float* delta_bias, const float* h0, void* y, float* ht,
                                   void* ws, size_t ws_bytes, void* stream) {
  return select_fwd(true, shape, u, delta, A, Bm, Cm, Dskip, z, delta_bias, h0, y, ht, ws, ws_bytes,
                    stream);
}

comba_status comba_select_bwd(const comba_select_shape* shape, const void* u, const void* delta,
                              const float* A, const void* Bm, const void* Cm, const float* Dskip,
                              const void* z, const float* delta_bias, const float* h0,
                              const void* dy, const float* dht, void* du, void* ddelta, float* dA,
                              void* dB, void* dC, float* dD, void* dz, float* ddelta_bias,
                              float* dh0, void* ws, size_t ws_bytes, void* stream) {
  comba::SelectArgs a;
  comba_status st = select_args(shape, &a);
  if (st != COMBA_OK) return st;
  st = select_inputs(&a, u, delta, A, Bm, Cm, Dskip, z, delta_bias, h0);
  if (st != COMBA_OK) return st;
  const bool tok = a.Ttot > 0;
  if (!dA || !ws || (Dskip && !dD) || (delta_bias && !ddelta_bias) ||
      (tok && (!dy || !du || !ddelta || !dB || !dC || (z && !dz))))
    return COMBA_ERR_NULL;
  const size_t e = a.bf16 ? 2 : 4;
  if (!aligned(dy, e) || !aligned(du, e) || !aligned(ddelta, e) || !aligned(dB, e) || !aligned(dC, e) ||
      !aligned(dz, e) || !aligned(dht, 4) || !aligned(dA, 4) || !aligned(dD, 4) ||
      !aligned(ddelta_bias, 4) || !aligned(dh0, 4) || !aligned(ws, kAlign))
    return COMBA_ERR_ALIGN;
  const SelectLayout L = select_layout(a, true);
  if (ws_bytes < L.total) return COMBA_ERR_WORKSPACE;
  char* base = static_cast<char*>(ws);
  a.ck = reinterpret_cast<float*>(base + L.ck);
  a.bcp = reinterpret_cast<float*>(base + L.bcp);
  a.dap = reinterpret_cast<float*>(base + L.dap);
  select_segments(&a, true);
  a.segF = reinterpret_cast<float*>(base + L.segF);
  a.segdt = reinterpret_cast<float*>(base + L.segdt);
  a.dy = dy;
  a.dht = dht;
  a.du = du;
  a.ddelta = ddelta;
  a.dz = dz;
  a.dB = dB;
  a.dC = dC;
  a.dA = dA;
  a.dD = Dskip ? dD : nullptr;
  a.dbias = delta_bias ? ddelta_bias : nullptr;
  a.dh0 = dh0;
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_select_bwd(a));
}

comba_status comba_select_step(const comba_select_shape* shape, const void* u, const void* delta,
                               const float* A, const void* Bm, const void* Cm, const float* Dskip,
                               const void* z, const float* delta_bias, float* state,
                               const int32_t* slots, int32_t num_slots, void* y, void* stream) {
  comba::SelectArgs a;
  comba_status st = select_args(shape, &a);
  if (st != COMBA_OK) return st;
  if (a.cu_seqlens || shape->T != 1 || num_slots < 0) return COMBA_ERR_SHAPE;
  st = select_inputs(&a, u, delta, A, Bm, Cm, Dskip, z, delta_bias, nullptr);
  if (st != COMBA_OK) return st;
  if (a.S > 0 && (!state || !y)) return COMBA_ERR_NULL;
  if (!aligned(y, a.bf16 ? 2 : 4) || !aligned(state, 4) || !aligned(slots, 4)) return COMBA_ERR_ALIGN;
  a.state = state;
  a.slots = slots;
  a.num_slots = num_slots;
  a.y = y;
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_select_step(a));
}

comba_status comba_group_norm_fwd(const comba_group_norm_shape* shape, const void* x,
                                  const float* weight, const float* bias, const void* z, void* y,
                                  void* stream) {
  comba::GroupNormArgs a;
  comba_status st = group_norm_args(shape, &a);
  if (st != COMBA_OK) return st;
  st = group_norm_inputs(&a, shape, x, weight, bias, z);
  if (st != COMBA_OK) return st;
  if (a.rows > 0 && !y) return COMBA_ERR_NULL;
  if (!aligned(y, elem(shape->out_dtype))) return COMBA_ERR_ALIGN;
  a.y = y;
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_group_norm_fwd(a));
}

size_t comba_group_norm_workspace_bytes(const comba_group_norm_shape* shape) {
  comba::GroupNormArgs a;
  return group_norm_args(shape, &a) == COMBA_OK ? group_norm_ws_bytes(a) : 0;
}

comba_status comba_group_norm_bwd(const comba_group_norm_shape* shape, const void* x,
                                  const float* weight, const float* bias, const void* z,
                                  const void* dy, void* dx, void* dz, float* dweight, float* dbias,
                                  void* ws, size_t ws_bytes, void* stream) {
  comba::GroupNormArgs a;
  comba_status st = group_norm_args(shape, &a);
  if (st != COMBA_OK) return st;
  st = group_norm_inputs(&a, shape, x, weight, bias, z);
  if (st != COMBA_OK) return st;
  if (!ws || (a.rows > 0 && (!dy || !dx || (z && !dz)))) return COMBA_ERR_NULL;
  if (!aligned(dy, elem(shape->out_dtype)) || !aligned(dz, elem(shape->out_dtype)) ||
      !aligned(dx, elem(shape->x_dtype)) || !aligned(dweight, 4) || !aligned(dbias, 4) ||
      !aligned(ws, kAlign))
    return COMBA_ERR_ALIGN;
  if (ws_bytes < group_norm_ws_bytes(a)) return COMBA_ERR_WORKSPACE;
  a.dy = dy;
  a.dx = dx;
  a.dz = dz;
  a.dw = dweight;
  a.db = dbias;
  a.part = static_cast<float*>(ws);
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_group_norm_bwd(a));
}

}  // extern "C"
