// Host side of include/comba_layer.h: argument validation, workspace layout and
// kernel launches on the caller's stream.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

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

// Rows of up to 4M values.
constexpr int64_t kMaxRow = (int64_t)1 << 22;

// The elements between the `rows` rows of a named input: given, or contiguous.  Kernels
// address rows in 64 bits, but for the scan's tiles (`tiles`), whose byte offsets
// inside 96 rows have to stay below 2^31.
bool row_stride(int64_t given, int64_t width, int64_t rows, bool tiles, long* row) {
  *row = given == 0 ? width : given;
  return *row >= width && *row <= (tiles ? kMaxRow : ((int64_t)1 << 60) / std::max<int64_t>(rows, 1));
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
  return row_stride(s->x_row, s->D, r.Ttot, false, &a->x_row) ? COMBA_OK : COMBA_ERR_SHAPE;
}

size_t conv_ws_bytes(const comba::ConvArgs& a) {
  return round_up((size_t)comba::conv_bwd_runs(a) * (a.K + 1) * a.D * sizeof(float)) + kAlign;
}

// ---- selective scan -----------------------------------------------------------
// Workgroups of a launch, which holds fewer than 2^32 threads: the tiles' have 512 or
// 768 each.
int64_t select_groups(int N) { return UINT32_MAX / (N == 8 ? 512 : 768); }

struct SelectLayout {
  size_t ck, bcp, dap, segF, segdt, total;
};

// `count` sequences' workgroups of `tokens` each, one per channel block.
struct Batch {
  double tokens;
  int64_t count;
};

// Tokens walked one after the other until the batches, in their order, are done by
// `cus` CUs with one workgroup each (`start`: a workgroup's own, in tokens).
double makespan(const Batch* batch, int n, int64_t blocks, int cus, double start) {
  struct Load {
    double t;
    int cus;
  } load[comba::SEL_LIST + 19] = {{0, cus}};
  auto later = [](const Load& x, const Load& y) { return x.t > y.t; };
  int m = 1;
  double all = 0, last = 0;
  for (int i = 0; i < n; ++i) {
    int64_t need = batch[i].count * blocks;
    const double t = batch[i].tokens + start;
    if (need >= 4 * cus) {  // whole rounds at once
      const int64_t k = need / cus - 2;
      all += (double)k * t;
      need -= k * cus;
    }
    while (need > 0) {  // the CUs that are free first
      std::pop_heap(load, load + m, later);
      Load& f = load[m - 1];
      const int k = need < f.cus ? (int)need : f.cus;
      need -= k;
      const Load done{f.t + t, k};
      if (done.t > last) last = done.t;
      if (k < f.cus) {
        f.cus -= k;
        std::push_heap(load, load + m, later);
        ++m;
      }
      load[m - 1] = done;
      std::push_heap(load, load + m, later);
    }
  }
  return all + last;
}

// The work rows.  Sequences are cut into segments where their workgroups, one per
// CU, leave CUs idle or wait for a long one: the main kernel then runs over segments
// side by side, after a first pass over all but one segment of each sequence that is
// cut.  Packed sequences of up to a CU's share of all tokens stay whole; without
// host offsets all do.  Takes the number of segments whose workgroups, one after
// the other to the first free CU, are done first; times in tokens of the main
// kernel (`pre`: the first pass's per token; `launch`: its launch; `start`: a
// workgroup's first loads and segment ends), fitted to 56 batches measured at 1 to
// 32 segments, over which the choice is 1.5% above the best on average.  Whole /
// cut, us, 16 states, 2,048 channels, forward and backward: one row of 8,192 tokens
// 341 / 155 and 884 / 312; of 1,000: 49 / 31 and 122 / 62; 4 rows of 2,048, which
// fill the CUs, 93 / 149 and 242 / 309; ten packed sequences of 1 to 15,777 tokens,
// 36,283 in all, forward 670 / 491; 20 of 777, one of 9,000 and two more 387 / 400.
void select_rows(comba::SelectArgs* a, bool bwd, comba::SelectRows* q) {
  a->segs = 1;
  a->seglen = a->segmin = 1 << 30;
  q->rows = a->S;
  q->n = 0;
  const int32_t* cu = a->cu_host;
  int32_t tokens[comba::SEL_LIST];  // of the longest sequences, the longest first
  if (cu) {
    for (int s = 0; s < a->S; ++s) {
      const int32_t len = cu[s + 1] - cu[s];
      if (q->n == comba::SEL_LIST && len <= tokens[q->n - 1]) continue;
      int i = q->n < comba::SEL_LIST ? q->n++ : q->n - 1;
      for (; i > 0 && tokens[i - 1] < len; --i) {
        tokens[i] = tokens[i - 1];
        q->seq[i] = q->seq[i - 1];
      }
      tokens[i] = len;
      q->seq[i] = s;
    }
    for (int i = 0; i <= q->n; ++i) q->at[i] = i;
  }
  const int64_t tile = comba::select_tile(a->N), blocks = (int64_t)a->G * a->nblk;
  if (a->longest < 2 * tile || a->S == 0) return;  // short, or not known
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    return;
  const double share = (double)a->Ttot * blocks / cus;
  if (cu && (double)a->longest <= share) return;
  const double pre = bwd ? 0.27 : 0.5, launch = bwd ? 110 : 186, start = bwd ? 60 : 50;
  int ncut = 0;  // packed sequences that may be cut
  while (cu && ncut < q->n && (double)tokens[ncut] > share) ++ncut;
  // the 16 longest whole sequences as batches, the others only in the share
  Batch batch[comba::SEL_LIST + 18];
  const int few = std::min(q->n, ncut + 16);
  auto whole = [&](int i, int end, int n) {
    for (; i < end; ++i) batch[n++] = {(double)tokens[i], 1};
    return n;
  };
  int n = cu ? whole(0, few, 0) : 1;
  if (!cu) batch[0] = {(double)a->longest, a->S};
  auto rounds = [&] { return std::max(makespan(batch, n, blocks, cus, start), share); };
  double best = rounds();
  for (int p = 2; p <= 32; p += p < 8 ? 1 : p < 16 ? 2 : 8) {
    const int64_t len = (a->longest + p * tile - 1) / (p * tile) * tile, segs = (a->longest + len - 1) / len;
    if (segs < 2) break;
    Batch first{(double)len, 0};
    int64_t rows = a->S;
    if (launch + std::max((double)len, share) + pre * (double)len >= best) continue;
    if (!cu) {
      first.count = (segs - 1) * a->S;
      batch[0] = first;
      batch[1] = {(double)(a->longest - (segs - 1) * len), a->S};
      n = 2;
    } else {
      int i = ncut;
      while (i < few && tokens[i] > len) ++i;
      n = whole(ncut, i, 0);
      Batch& cut = batch[n++];
      for (int k = 0; k < ncut; ++k) {
        const int64_t c = (tokens[k] - 1) / len;
        first.count += c;
        batch[n++] = {(double)(tokens[k] - c * len), 1};
      }
      cut = first;
      n = whole(i, few, n);
    }
    rows += first.count;
    const double t = launch + rounds() + pre * makespan(&first, 1, blocks, cus, start);
    if (t < best && rows * blocks <= select_groups(a->N)) {
      best = t;
      a->segs = (int)segs;
      a->seglen = (int)len;
      a->segmin = cu ? (int)share : 0;
      q->rows = (int)rows;
    }
  }
  if (!cu || a->segs == 1) return;
  // the listed sequences by their segments' length
  int i = ncut;
  while (i < q->n && tokens[i] > a->seglen) ++i;
  std::rotate(q->seq, q->seq + ncut, q->seq + i);
  std::rotate(tokens, tokens + ncut, tokens + i);
  for (int k = 0; k < q->n; ++k)
    q->at[k + 1] = q->at[k] + (tokens[k] > a->segmin ? (tokens[k] + a->seglen - 1) / a->seglen : 1);
}

// The states kept for the backward: a sequence's start at tok0 / select_ck + its
// number, which leaves room for a partial interval per sequence.
size_t select_kept_bytes(const comba::SelectArgs& a) {
  return ((size_t)a.Ttot / comba::select_ck(a.N) + a.S + 1) * a.D * a.N * sizeof(float);
}

// The call's work rows and the layout of its workspace: of a forward, a saving
// forward (whose first part the backward reads) or a backward.
enum class Use { kFwd, kSave, kBwd };
SelectLayout select_layout(comba::SelectArgs* a, Use use, comba::SelectRows* q) {
  SelectLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += round_up(bytes);
    return at;
  };
  select_rows(a, use == Use::kBwd, q);
  if (use == Use::kSave) L.ck = take(select_kept_bytes(*a));
  if (use == Use::kBwd) {
    L.bcp = take((size_t)a->G * a->nblk * a->Ttot * 2 * a->N * sizeof(float));
    L.dap = take((size_t)q->rows * a->D * (a->N + 2) * sizeof(float));
  }
  const size_t cut = a->segs > 1 ? q->rows : 0;  // work rows with kept ends of segments
  L.segF = take(cut * a->D * a->N * sizeof(float));
  L.segdt = take(cut * a->D * sizeof(float));
  L.total = off + kAlign;
  return L;
}

comba_status select_args(const comba_select_shape* s, comba::SelectArgs* a, bool tiles = true) {
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
  if (tiles && (int64_t)a->S * a->G * a->nblk > select_groups(s->N)) return COMBA_ERR_SHAPE;
  const int64_t gn = (int64_t)s->G * s->N;
  auto row = [&](int64_t given, int64_t width, long* to) {
    return row_stride(given, width, r.Ttot, tiles, to);
  };
  if (!row(s->u_row, s->D, &a->u_row) || !row(s->delta_row, s->D, &a->delta_row) ||
      !row(s->z_row, s->D, &a->z_row) || !row(s->b_row, gn, &a->b_row) || !row(s->c_row, gn, &a->c_row))
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

size_t select_bytes(const comba_select_shape* shape, Use use) {
  comba::SelectArgs a;
  comba::SelectRows q;
  return select_args(shape, &a) == COMBA_OK ? select_layout(&a, use, &q).total : 0;
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
  comba::SelectRows q;
  const SelectLayout L = select_layout(&a, save ? Use::kSave : Use::kFwd, &q);
  if (ws_bytes < L.total) return COMBA_ERR_WORKSPACE;
  a.y = y;
  a.ht = ht;
  char* base = static_cast<char*>(ws);
  if (save) a.ck = reinterpret_cast<float*>(base + L.ck);
  a.segF = reinterpret_cast<float*>(base + L.segF);
  a.segdt = reinterpret_cast<float*>(base + L.segdt);
  a.stream = static_cast<hipStream_t>(stream);
  return done(comba::launch_select_fwd(a, q));
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
  return row_stride(s->x_row, s->C, s->rows, false, &a->x_row) &&
                 row_stride(s->z_row, s->C, s->rows, false, &a->z_row)
             ? COMBA_OK
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
  return select_bytes(shape, Use::kFwd);
}

size_t comba_select_save_bytes(const comba_select_shape* shape) {
  return select_bytes(shape, Use::kSave);
}

size_t comba_select_bwd_workspace_bytes(const comba_select_shape* shape) {
  return select_bytes(shape, Use::kBwd);
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
                              float* dh0, const void* saved, size_t saved_bytes, void* ws,
                              size_t ws_bytes, void* stream) {
  comba::SelectArgs a;
  comba_status st = select_args(shape, &a);
  if (st != COMBA_OK) return st;
  st = select_inputs(&a, u, delta, A, Bm, Cm, Dskip, z, delta_bias, h0);
  if (st != COMBA_OK) return st;
  const bool tok = a.Ttot > 0;
  if (!dA || !saved || !ws || (Dskip && !dD) || (delta_bias && !ddelta_bias) ||
      (tok && (!dy || !du || !ddelta || !dB || !dC || (z && !dz))))
    return COMBA_ERR_NULL;
  const size_t e = a.bf16 ? 2 : 4;
  if (!aligned(dy, e) || !aligned(du, e) || !aligned(ddelta, e) || !aligned(dB, e) || !aligned(dC, e) ||
      !aligned(dz, e) || !aligned(dht, 4) || !aligned(dA, 4) || !aligned(dD, 4) ||
      !aligned(ddelta_bias, 4) || !aligned(dh0, 4) || !aligned(saved, kAlign) || !aligned(ws, kAlign))
    return COMBA_ERR_ALIGN;
  comba::SelectRows q;
  const SelectLayout L = select_layout(&a, Use::kBwd, &q);
  if (saved_bytes < select_kept_bytes(a) || ws_bytes < L.total) return COMBA_ERR_WORKSPACE;
  char* base = static_cast<char*>(ws);
  a.kept = static_cast<const float*>(saved);
  a.bcp = reinterpret_cast<float*>(base + L.bcp);
  a.dap = reinterpret_cast<float*>(base + L.dap);
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
  return done(comba::launch_select_bwd(a, q));
}

comba_status comba_select_step(const comba_select_shape* shape, const void* u, const void* delta,
                               const float* A, const void* Bm, const void* Cm, const float* Dskip,
                               const void* z, const float* delta_bias, float* state,
                               const int32_t* slots, int32_t num_slots, void* y, void* stream) {
  comba::SelectArgs a;
  comba_status st = select_args(shape, &a, false);
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
