// Attention, its gradient, single-token steps and rotary positions: checks of the arguments, evaluation of lazy
// operands, temporary memory and the choice of kernels (grumpy_hip_attention.h; kernels: attention_*.hip, rotary.hip).
#include "attention.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <new>

#include "ctx.h"

#define ATT_HIP(c, call)                                                                     \
  do {                                                                                       \
    hipError_t e_ = (call);                                                                  \
    if (e_ != hipSuccess) return fail(c, GR_ERR_HIP, std::string(#call ": ") + hipGetErrorString(e_)); \
  } while (0)

namespace gr {
namespace attn {

constexpr int64_t LIMIT = (int64_t(1) << 30) - 512;   // rows of queries of one head of k, and keys
constexpr int64_t FAR = int64_t(1) << 24;             // of queries from the keys, where distances count
constexpr int64_t THREADS = int64_t(1) << 32;         // what a launch may not reach
constexpr int64_t GROUPS = THREADS / 512 - 8;         // workgroups of the largest size (and what grid_of rounds up)

struct Call {
  gr_ctx* ctx;
  const char* name;
  std::vector<std::pair<gr_array, const char*>> inputs, results;

  gr_status error(gr_status s, const std::string& what) const { return fail(ctx, s, std::string(name) + ": " + what); }

  // An operand or result: handle, element type and shape.
  gr_status take(gr_array a, const char* what, int dtype, std::initializer_list<int64_t> shape, bool result) {
    const Node* n = lookup(ctx, a);
    if (!n) return error(GR_ERR_HANDLE, std::string(what) + ": bad handle");
    if (n->kind == Kind::SCALAR) return error(GR_ERR_UNSUPPORTED, std::string(what) + " is a bare scalar");
    if ((int)n->dtype != dtype) return error(GR_ERR_DTYPE, std::string(what) + " has another element type");
    bool same = n->ndim == (int)shape.size();
    int d = 0;
    for (int64_t s : shape) { if (same && n->shape[d] != s) same = false; ++d; }
    if (!same) return error(GR_ERR_SHAPE, std::string(what) + " has another shape");
    if (result) {
      StoredView v;
      if (!stored_view(n, &v)) return error(GR_ERR_UNSUPPORTED, std::string(what) + " is not (a view of) a materialised array");
      results.push_back({a, what});
    } else {
      inputs.push_back({a, what});
    }
    return GR_OK;
  }

  StoredView view(gr_array a) const {
    StoredView v;
    const Node* n = a ? lookup(ctx, a) : nullptr;
    if (n) (void)stored_view(n, &v);
    return v;
  }

  // Do two views of rank 3 or 4 share no element?  Certain where their extents do not meet, and where they are parts of one packed array: the
  // same steps between batches and rows, and within a row two stretches that do not meet.
  bool apart(gr_array a, gr_array b) const {
    const StoredView x = view(a), y = view(b);
    if (!(x.lo < y.hi && y.lo < x.hi)) return true;
    const Node *m = lookup(ctx, a), *n = lookup(ctx, b);
    if (m->ndim != 4 || n->ndim != 4 || m->dtype != n->dtype) return false;
    const int64_t size = (int64_t)itemsize(m->dtype);
    int64_t least = INT64_MAX;
    int64_t steps[2], counts[2];
    for (int d = 0; d < 2; ++d) {
      if (m->shape[d] != n->shape[d]) return false;
      counts[d] = m->shape[d];
      steps[d] = 0;
      if (counts[d] <= 1) continue;
      if (x.strides[d] != y.strides[d] || x.strides[d] <= 0) return false;
      steps[d] = x.strides[d];
      least = std::min(least, steps[d]);
    }
    if (counts[0] > 1 && counts[1] > 1) {
      const int in = steps[0] < steps[1] ? 0 : 1;
      if (steps[1 - in] < steps[in] * counts[in]) return false;
    }
    auto reach = [&](const Node* t, const StoredView& v, int64_t* lo, int64_t* hi) {
      *lo = *hi = (v.data - std::min(x.data, y.data)) / size;
      for (int d = 2; d < 4; ++d) (v.strides[d] < 0 ? *lo : *hi) += v.strides[d] * (t->shape[d] - 1);
    };
    int64_t alo, ahi, blo, bhi;
    reach(m, x, &alo, &ahi);
    reach(n, y, &blo, &bhi);
    if (std::max(ahi, bhi) - std::min(alo, blo) >= least) return false;
    return ahi < blo || bhi < alo;
  }

  // Evaluates the operands, then what reads the results' storage.  Before it: everything that can be refused is.
  gr_status settle(bool in_place_ok = false) {
    for (auto& r : results) {
      const Node* n = lookup(ctx, r.first);
      const StoredView v = view(r.first);
      if (n->count() == 0) continue;
      // an element of a result stands in one place: each step passes all that the smaller ones reach
      int order[MAXD], k = 0;
      for (int d = 0; d < n->ndim; ++d) if (n->shape[d] > 1) order[k++] = d;
      std::sort(order, order + k, [&](int a, int b) { return std::llabs(v.strides[a]) < std::llabs(v.strides[b]); });
      int64_t reach = 0;
      for (int j = 0; j < k; ++j) {
        if (std::llabs(v.strides[order[j]]) <= reach) return error(GR_ERR_UNSUPPORTED, std::string(r.second) + ": elements of the result overlap");
        reach += std::llabs(v.strides[order[j]]) * (n->shape[order[j]] - 1);
      }
      for (auto& o : results) if (&o < &r && lookup(ctx, o.first)->count() > 0 && !apart(o.first, r.first)) return error(GR_ERR_ALIAS, std::string(o.second) + " and " + r.second + " overlap");
      for (auto& i : inputs) {
        if (in_place_ok && same_view(i.first, r.first)) continue;
        const Node* m = lookup(ctx, i.first);
        StoredView w;
        if (stored_view(m, &w) && w.lo < v.hi && v.lo < w.hi && !apart(i.first, r.first))
          return error(GR_ERR_ALIAS, std::string(i.second) + " and " + r.second + " overlap");
      }
    }
    if (ctx->device < 0 && !ctx->opt_dry_run) return error(GR_ERR_NODEVICE, "context has no device");
    for (auto& i : inputs) {
      gr_status st = gr_materialize(ctx, i.first);
      if (st != GR_OK) return st;
    }
    for (auto& r : results) {
      gr_status st = prepare_write(ctx, r.first);
      if (st != GR_OK) return st;
    }
    return GR_OK;
  }

  bool same_view(gr_array a, gr_array b) const {
    if (a == b) return true;
    const Node *m = lookup(ctx, a), *n = lookup(ctx, b);
    StoredView x, y;
    if (!stored_view(m, &x) || !stored_view(n, &y) || x.data != y.data || m->ndim != n->ndim || m->dtype != n->dtype) return false;
    for (int d = 0; d < m->ndim; ++d) if (m->shape[d] != n->shape[d] || (m->shape[d] > 1 && x.strides[d] != y.strides[d])) return false;
    return true;
  }

  // (B, N, H, D), or (B, H, D) as one row
  gr_status tensor(gr_array a, const char* what, Tensor* t) const {
    const Node* n = lookup(ctx, a);
    const StoredView v = view(a);
    const int64_t size = (int64_t)itemsize(n->dtype), each = 16 / size;
    const int r = n->ndim;
    auto step = [&](int d) { return n->shape[d] > 1 ? v.strides[d] : 0; };
    if (n->shape[r - 1] > 1 && v.strides[r - 1] != 1) return error(GR_ERR_UNSUPPORTED, std::string(what) + ": the values of a row are not neighbours");
    t->p = v.data;
    t->sb = step(0);
    t->sn = r == 4 ? (n->shape[1] > 1 ? v.strides[1] : (n->shape[r - 1] + each - 1) / each * each) : 0;   // (a single row: any step)
    t->sh = step(r - 2);
    const int64_t D = n->shape[r - 1], rows = 128;
    t->aligned = (uintptr_t)v.data % 16 == 0 && t->sb % each == 0 && t->sn % each == 0 && t->sh % each == 0 && D % each == 0;
    t->direct = t->aligned && t->sn >= D && t->sn < (int64_t(1) << 30) && (t->sn * rows + D) * size < (int64_t(1) << 31) - 64;
    return GR_OK;
  }

  const int* whole(gr_array a, int64_t* s0, int64_t* s1) const {
    if (!a) return nullptr;
    const StoredView v = view(a);
    if (s0) *s0 = v.strides[0];
    if (s1) *s1 = v.strides[1];
    return (const int*)v.data;
  }

  // Temporary memory of the call.
  gr_status space(size_t bytes, char** to) {
    *to = nullptr;
    if (bytes == 0) return GR_OK;
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (ctx->device >= 0) ATT_HIP(ctx, hipStreamIsCapturing(ctx->stream, &cap));
    const bool capturing = cap != hipStreamCaptureStatusNone;
    if (bytes > ctx->attention_space_bytes) {
      if (capturing) return error(GR_ERR_OOM, "the stream is being captured and the call needs " + std::to_string(bytes) + " bytes of temporary memory: run it once before the capture");
      if (ctx->attention_space) {
        // (a graph may still use it)
        if (ctx->attention_captured) ctx->attention_kept.push_back({ctx->attention_space, ctx->attention_space_bytes});
        else ctx_free(ctx, ctx->attention_space, ctx->attention_space_bytes);
      }
      ctx->attention_space = nullptr;
      ctx->attention_space_bytes = 0;
      ctx->attention_captured = false;
      void* p = ctx_alloc(ctx, bytes);
      if (!p) return error(GR_ERR_OOM, "allocator returned NULL for " + std::to_string(bytes) + " bytes of temporary memory");
      ctx->attention_space = p;
      ctx->attention_space_bytes = bytes;
    }
    if (capturing) ctx->attention_captured = true;
    *to = (char*)ctx->attention_space;
    return GR_OK;
  }

  // A launch, bracketed by events where the context profiles (not into a graph).
  template <class F>
  gr_status launch(const char* kernel, F&& f) {
    if (ctx->device < 0) { ctx->stats.kernel_launches++; return GR_OK; }   // dry run
    hipEvent_t e0 = nullptr, e1 = nullptr;
    bool profile = ctx->opt_profile != 0;
    if (profile) {
      hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
      ATT_HIP(ctx, hipStreamIsCapturing(ctx->stream, &cap));
      profile = cap == hipStreamCaptureStatusNone;
    }
    if (profile) {
      for (hipEvent_t* ev : {&e0, &e1}) {
        if (!ctx->event_pool.empty()) { *ev = ctx->event_pool.back(); ctx->event_pool.pop_back(); }
        else ATT_HIP(ctx, hipEventCreate(ev));
      }
      ATT_HIP(ctx, hipEventRecord(e0, ctx->stream));
    }
    ATT_HIP(ctx, f());
    if (profile) {
      ATT_HIP(ctx, hipEventRecord(e1, ctx->stream));
      ctx->prof.push_back({kernel, e0, e1});
    }
    ctx->stats.kernel_launches++;
    return GR_OK;
  }
};

#define TRY(x) do { gr_status st_ = (x); if (st_ != GR_OK) return st_; } while (0)

static bool resolved(gr_ctx* ctx, gr_array a) {
  StoredView v;
  return stored_view(lookup(ctx, a), &v);
}

// Operands that are stored already have rows whose values are neighbours.  (Those still to be evaluated are looked at when they are: their own
// storage is dense, but a view of an expression stays a view of it.)
static gr_status rows_are_neighbours(Call& c, std::initializer_list<gr_array> arrays) {
  for (gr_array a : arrays) {
    Tensor t;
    if (resolved(c.ctx, a)) TRY(c.tensor(a, "an operand", &t));
  }
  return GR_OK;
}

static gr_status contiguous_stats(Call& c, gr_array lse) {
  const Node* n = lookup(c.ctx, lse);
  const StoredView v = c.view(lse);
  if (n->count() == 0) return GR_OK;
  int64_t s = 1;
  for (int d = n->ndim - 1; d >= 0; --d) {
    if (n->shape[d] > 1 && v.strides[d] != s) return c.error(GR_ERR_UNSUPPORTED, "lse is not C-contiguous");
    s *= n->shape[d];
  }
  return GR_OK;
}

static int padded(int64_t D) { return D <= 64 ? 64 : D <= 96 ? 96 : D <= 128 ? 128 : 256; }
static size_t rounded(size_t n) { return (n + 255) & ~(size_t)255; }

// The extents of q (B, N, H, D) or (B, H, D), and k (B, M, HK, D).
static gr_status extents(Call& c, gr_array q, gr_array k, int rank, int* type, Args* a) {
  const Node *x = lookup(c.ctx, q), *y = lookup(c.ctx, k);
  if (!x || !y) return c.error(GR_ERR_HANDLE, "q or k: bad handle");
  if (x->kind == Kind::SCALAR || y->kind == Kind::SCALAR) return c.error(GR_ERR_UNSUPPORTED, "q or k is a bare scalar");
  if (x->dtype != GR_F32 && x->dtype != GR_BF16) return c.error(GR_ERR_DTYPE, "q must be f32 or bf16");
  if (x->ndim != rank || y->ndim != 4) return c.error(GR_ERR_SHAPE, rank == 4 ? "q is (B, N, H, D) and k (B, M, HK, D)" : "q is (B, H, D) and k (B, M, HK, D)");
  const int64_t B = x->shape[0], N = rank == 4 ? x->shape[1] : 1, H = x->shape[rank - 2], D = x->shape[rank - 1], M = y->shape[1], HK = y->shape[2];
  if (D < 1 || D > 256) return c.error(GR_ERR_UNSUPPORTED, "heads have 1 to 256 values");
  if (HK < 1 || H < 1 || H % HK) return c.error(GR_ERR_SHAPE, "the heads of q are not a multiple of those of k");
  if (B > LIMIT || H > LIMIT || M > LIMIT || N > LIMIT || N * (H / HK) > LIMIT || B * HK > LIMIT) return c.error(GR_ERR_UNSUPPORTED, "more than 2^30 rows");
  *type = x->dtype == GR_BF16 ? TYPE_BF16 : TYPE_F32;
  a->B = (int)B; a->N = (int)N; a->H = (int)H; a->D = (int)D; a->M = (int)M; a->HK = (int)HK; a->G = (int)(H / HK);
  return GR_OK;
}

static gr_status take_scores(Call& c, const gr_scores* s, Args* a, bool step) {
  if (!s) return c.error(GR_ERR_ARG, "NULL scores");
  // What the kernels take of them (scale log2(e), scale 2^-32, cap log2(e), 2 log2(e) scale / cap) are normal floats: a factor that is zero or infinite makes NaN of
  // masked scores and of zeros.
  if (!(s->scale > 1e-28 && s->scale < 1e30)) return c.error(GR_ERR_ARG, "scale must be between 1e-28 and 1e30");
  if (s->cap != 0.0) {
    if (!(s->cap > 1e-30 && s->cap < 1e30)) return c.error(GR_ERR_ARG, "cap must be 0, or between 1e-30 and 1e30");
    if (!(s->scale / s->cap > 1e-37 && s->scale / s->cap < 1e38)) return c.error(GR_ERR_ARG, "scale / cap must be between 1e-37 and 1e38");
  }
  if (s->causal != 0 && s->causal != 1) return c.error(GR_ERR_ARG, "causal must be 0 or 1");
  if (s->position < -(int64_t(1) << 31) || s->position > (int64_t(1) << 31)) return c.error(GR_ERR_ARG, "position beyond 2^31");
  if (s->prefix && !s->causal) return c.error(GR_ERR_ARG, "a prefix without a causal mask");
  if (!s->q_documents != !s->k_documents) return c.error(GR_ERR_ARG, "documents of queries and of keys are given together");
  if (step && (s->causal || s->position || s->prefix || s->q_documents)) return c.error(GR_ERR_ARG, "causal, position, prefix and documents have no meaning for a single token");
  if (step && !s->lengths) return c.error(GR_ERR_ARG, "lengths are missing");
  // (behind 2^24 f32 holds neither single distances nor an lse of which a probability could be formed again)
  if (s->slopes && !step && (s->position > a->M + FAR || s->position + a->N < -FAR)) return c.error(GR_ERR_ARG, "with slopes, the queries stand within 2^24 of the keys");
  if (s->slopes) TRY(c.take(s->slopes, "slopes", GR_F32, {a->H}, false));
  if (s->prefix) TRY(c.take(s->prefix, "prefix", GR_I32, {a->B}, false));
  if (s->lengths) TRY(c.take(s->lengths, "lengths", GR_I32, {a->B}, false));
  if (s->q_documents) {
    TRY(c.take(s->q_documents, "q_documents", GR_I32, {a->B, a->N}, false));
    TRY(c.take(s->k_documents, "k_documents", GR_I32, {a->B, a->M}, false));
    if (a->B * (padded_rows(a->M) + padded_rows(a->N)) >= THREADS) return c.error(GR_ERR_UNSUPPORTED, "more than 2^32 document numbers");
  }
  return GR_OK;
}

static int fill_scores(Call& c, const gr_scores* s, int type, Args* a) {
  a->slopes = (const float*)c.whole(s->slopes, &a->slopes_s, nullptr);
  a->prefix = c.whole(s->prefix, &a->prefix_s, nullptr);
  a->lengths = c.whole(s->lengths, &a->lengths_s, nullptr);
  a->qdoc = c.whole(s->q_documents, &a->qdoc_sb, &a->qdoc_sn);
  a->kdoc = c.whole(s->k_documents, &a->kdoc_sb, &a->kdoc_sn);
  a->position = s->position;
  a->place = (int)std::max<int64_t>(-(int64_t(1) << 30), std::min<int64_t>(s->position, int64_t(1) << 30));
  a->causal = s->causal;
  const double log2e = 1.4426950408889634;
  const bool wide = type == TYPE_BF16 && s->cap > SHORT_CAP;
  a->scale = (float)s->scale;
  if (s->cap > 0.0) {
    a->c = (float)(s->cap * log2e);
    // (the short form takes what the hardware's power of two does)
    a->cin = (float)(type == TYPE_BF16 && !wide ? 2.0 * log2e * s->scale / s->cap : s->scale / s->cap);
  } else {
    a->c = (float)(s->scale * log2e);
  }
  return (s->cap > 0.0 ? MODE_CAP : 0) | (s->slopes ? MODE_BIAS : 0) | (wide ? MODE_WIDE : 0);
}

static int keys_of(bool divided, int size, int dp) { return divided ? 32 * shared_waves(size, dp) : tile_rows(size, dp); }

// Splits of a long dimension where there are fewer groups than compute units: as many workgroups as fit the 256 compute units at once, each with a
// tile at least.  More wait for a second turn (6 heads of 777 rows of float32, one workgroup per compute unit: forward and gradient 138 us with 6 splits
// of 42 groups, 152 with 8), fewer walk longer (1 head of 448 rows: 1, 2, 4, 8 splits take 151, 117, 86, 70 us).
static int splits_of(int64_t groups, int64_t tiles, int most, int per_cu) {
  if (groups >= 256 || groups < 1) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(256 * per_cu / groups, tiles), most));
}

// The same for calls of at most 32 rows per head, which read k and v at the rate of the memory: four workgroups per compute unit, which fit it
// together (32 sequences on 8 heads: 1, 2, 4, 8, 16 splits take 260, 177, 173, 179, 190 us; one sequence of 65537 keys on one head: 64, 128, 256
// take 31, 22, 20), but none for a walk of 8 tiles, which is over before the parts would be joined (4 sequences of 512 keys on 16 heads: 16.6 us, 20 with 2).
static int token_splits_of(int64_t groups, int64_t tiles) {
  if (tiles <= 8 || groups < 1) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>((1024 + groups - 1) / groups, tiles / 2), MAX_SPLITS));
}

// What ranges() prepares of the documents.
struct Documents {
  size_t kr = 0, qr = 0, kd = 0, qd = 0, bytes = 0;
  explicit Documents(const Args& a) {
    if (!a.kdoc) return;
    kr = rounded((size_t)a.B * ((a.M + 31) / 32) * 8);
    qr = rounded((size_t)a.B * ((a.N + 31) / 32) * 8);
    kd = rounded((size_t)a.B * padded_rows(a.M) * 4);
    qd = rounded((size_t)a.B * padded_rows(a.N) * 4);
    bytes = kr + qr + kd + qd;
  }
  void place(Args* a, char* at) const {
    a->kranges = (int*)at;
    a->qranges = (int*)(at + kr);
    a->kdocs = (int*)(at + kr + qr);
    a->qdocs = (int*)(at + kr + qr + kd);
  }
};

static gr_status forward(Call& c, Args& a, int type, int mode) {
  const int size = type == TYPE_BF16 ? 2 : 4, dp = padded(a.D);
  const int64_t rows = (int64_t)a.N * a.G, pairs = (int64_t)a.B * a.HK;
  if (rows == 0 || pairs == 0) return GR_OK;
  const bool divided = rows <= 32;
  const int keys = keys_of(divided, size, dp);
  a.blocks = (int)((rows + (divided ? 31 : 127)) / (divided ? 32 : 128));
  const int64_t tiles = ((int64_t)a.M + keys - 1) / keys;
  a.splits = divided ? token_splits_of(pairs * a.blocks, tiles) : splits_of(pairs * a.blocks, tiles, MAX_SPLITS, forward_per_cu(size, dp));
  const int64_t blocks = (int64_t)a.blocks * a.splits;
  if (blocks * pairs > GROUPS) return c.error(GR_ERR_UNSUPPORTED, "more than 2^23 blocks of rows");
  const size_t sums = a.splits > 1 ? rounded((size_t)a.splits * pairs * rows * dp * 4) : 0, ml = a.splits > 1 ? rounded((size_t)a.splits * pairs * rows * 8) : 0;
  Documents docs(a);
  char* ws;
  TRY(c.space(sums + ml + docs.bytes, &ws));
  a.part_o = (float*)ws;
  a.part_ml = (float*)(ws + sums);
  docs.place(&a, ws + sums + ml);
  if (a.kdoc && a.M > 0) TRY(c.launch("gr_attention_ranges", [&] { return ranges(a, c.ctx->stream); }));
  const unsigned grid = grid_of((int)pairs, blocks);
  TRY(c.launch(a.step ? "gr_attention_step" : "gr_attention", [&] {
    return type == TYPE_BF16 ? forward_bf16(a, dp, mode, divided, grid, c.ctx->stream) : forward_f32(a, dp, mode, divided, grid, c.ctx->stream);
  }));
  if (a.splits > 1) TRY(c.launch("gr_attention_combine", [&] { return combine(a, type, dp, c.ctx->stream); }));
  return GR_OK;
}

static gr_status attention(gr_ctx* ctx, const gr_scores* s, gr_array q, gr_array k, gr_array v, gr_array out, gr_array lse, gr_array rest) {
  Call c{ctx, "attention"};
  Args a;
  int type;
  TRY(extents(c, q, k, 4, &type, &a));
  const int dt = type == TYPE_BF16 ? GR_BF16 : GR_F32;
  TRY(c.take(q, "q", dt, {a.B, a.N, a.H, a.D}, false));
  TRY(c.take(k, "k", dt, {a.B, a.M, a.HK, a.D}, false));
  TRY(c.take(v, "v", dt, {a.B, a.M, a.HK, a.D}, false));
  TRY(take_scores(c, s, &a, false));
  TRY(c.take(out, "out", dt, {a.B, a.N, a.H, a.D}, true));
  if (lse) TRY(c.take(lse, "lse", GR_F32, {a.B, a.H, a.N}, true));
  if (rest) {
    if (type != TYPE_BF16) return c.error(GR_ERR_DTYPE, "rest is for bf16 results");
    TRY(c.take(rest, "rest", GR_BF16, {a.B, a.N, a.H, a.D}, true));
  }
  Tensor t;
  TRY(c.tensor(out, "out", &t));
  if (rest) TRY(c.tensor(rest, "rest", &t));
  if (lse) TRY(contiguous_stats(c, lse));
  TRY(rows_are_neighbours(c, {q, k, v}));
  TRY(c.settle());
  TRY(c.tensor(q, "q", &a.q));
  TRY(c.tensor(k, "k", &a.k));
  TRY(c.tensor(v, "v", &a.v));
  TRY(c.tensor(out, "out", &a.out));
  if (rest) TRY(c.tensor(rest, "rest", &a.rest));
  if (lse) a.lse = (float*)c.view(lse).data;
  const int mode = fill_scores(c, s, type, &a);
  return forward(c, a, type, mode);
}

static gr_status step(gr_ctx* ctx, const gr_scores* s, gr_array q, gr_array k, gr_array v, gr_array out) {
  Call c{ctx, "attention_step"};
  Args a;
  int type;
  TRY(extents(c, q, k, 3, &type, &a));
  const int dt = type == TYPE_BF16 ? GR_BF16 : GR_F32;
  TRY(c.take(q, "q", dt, {a.B, a.H, a.D}, false));
  TRY(c.take(k, "k", dt, {a.B, a.M, a.HK, a.D}, false));
  TRY(c.take(v, "v", dt, {a.B, a.M, a.HK, a.D}, false));
  TRY(take_scores(c, s, &a, true));
  TRY(c.take(out, "out", dt, {a.B, a.H, a.D}, true));
  Tensor t;
  TRY(c.tensor(out, "out", &t));
  TRY(rows_are_neighbours(c, {q, k, v}));
  TRY(c.settle());
  TRY(c.tensor(q, "q", &a.q));
  TRY(c.tensor(k, "k", &a.k));
  TRY(c.tensor(v, "v", &a.v));
  TRY(c.tensor(out, "out", &a.out));
  const int mode = fill_scores(c, s, type, &a);
  a.step = 1;
  return forward(c, a, type, mode);
}

static gr_status grad(gr_ctx* ctx, const gr_scores* s, gr_array q, gr_array k, gr_array v, gr_array out, gr_array rest, gr_array lse, gr_array dout,
                      gr_array dq, gr_array dk, gr_array dv) {
  Call c{ctx, "attention_grad"};
  Args a;
  int type;
  TRY(extents(c, q, k, 4, &type, &a));
  const int dt = type == TYPE_BF16 ? GR_BF16 : GR_F32, size = type == TYPE_BF16 ? 2 : 4, dp = padded(a.D);
  TRY(c.take(q, "q", dt, {a.B, a.N, a.H, a.D}, false));
  TRY(c.take(k, "k", dt, {a.B, a.M, a.HK, a.D}, false));
  TRY(c.take(v, "v", dt, {a.B, a.M, a.HK, a.D}, false));
  TRY(take_scores(c, s, &a, false));
  TRY(c.take(out, "out", dt, {a.B, a.N, a.H, a.D}, false));
  if (rest) {
    if (type != TYPE_BF16) return c.error(GR_ERR_DTYPE, "rest is for bf16 results");
    TRY(c.take(rest, "rest", GR_BF16, {a.B, a.N, a.H, a.D}, false));
  }
  TRY(c.take(lse, "lse", GR_F32, {a.B, a.H, a.N}, false));
  TRY(c.take(dout, "dout", dt, {a.B, a.N, a.H, a.D}, false));
  TRY(c.take(dq, "dq", dt, {a.B, a.N, a.H, a.D}, true));
  TRY(c.take(dk, "dk", dt, {a.B, a.M, a.HK, a.D}, true));
  TRY(c.take(dv, "dv", dt, {a.B, a.M, a.HK, a.D}, true));
  Tensor t;
  TRY(c.tensor(dq, "dq", &t));
  TRY(c.tensor(dk, "dk", &t));
  TRY(c.tensor(dv, "dv", &t));
  TRY(rows_are_neighbours(c, {q, k, v, out, dout}));
  if (rest) TRY(rows_are_neighbours(c, {rest}));
  if (resolved(ctx, lse)) TRY(contiguous_stats(c, lse));
  TRY(c.settle());
  TRY(contiguous_stats(c, lse));   // (a view of an expression has its steps only now)
  TRY(c.tensor(q, "q", &a.q));
  TRY(c.tensor(k, "k", &a.k));
  TRY(c.tensor(v, "v", &a.v));
  TRY(c.tensor(out, "out", &a.out));
  if (rest) TRY(c.tensor(rest, "rest", &a.rest));
  TRY(c.tensor(dout, "dout", &a.dout));
  TRY(c.tensor(dq, "dq", &a.dq));
  TRY(c.tensor(dk, "dk", &a.dk));
  TRY(c.tensor(dv, "dv", &a.dv));
  a.lse = (float*)c.view(lse).data;
  const int mode = fill_scores(c, s, type, &a);
  if (type == TYPE_F32) a.c *= 0.5f;   // (EXPONENT in attention_backward.h)

  const int64_t rows = (int64_t)a.N * a.G, pairs = (int64_t)a.B * a.HK;
  if (pairs == 0) return GR_OK;
  const int64_t qblocks = (rows + 127) / 128, kblocks = ((int64_t)a.M + 127) / 128;
  const int64_t tile = tile_rows(size, dp);
  const int qsplits = splits_of(pairs * qblocks, ((int64_t)a.M + tile - 1) / tile, 16, grad_q_per_cu(size, dp));
  // For dk and dv, where a workgroup walks the queries of G heads, from every place on to the end: more and shorter walks even out what causal
  // masks and documents leave of them (2 x 4096 rows in 6 documents, 16 heads on 4 of 128 bfloat16 values, 256 blocks: 746 us in one part, 267 in four
  // with their sum).  From 1024 blocks on there are several turns of them anyway, and the parts cost what they give.
  const int64_t units = (((int64_t)a.N + tile - 1) / tile) * a.G;
  int ksplits = splits_of(pairs * kblocks, units, 16, grad_kv_per_cu(size, dp));
  if (pairs * kblocks >= 256 && pairs * kblocks < 1024 && (a.causal || a.kdoc)) ksplits = (int)std::max<int64_t>(1, std::min<int64_t>(1024 / (pairs * kblocks), units / 16));
  if (std::max(qblocks * qsplits, kblocks * ksplits) * pairs > GROUPS || a.B * padded_rows(a.N) * a.H * 16 >= THREADS) return c.error(GR_ERR_UNSUPPORTED, "more than 2^23 blocks of rows");
  const size_t st = rounded((size_t)a.B * a.H * padded_rows(a.N) * 4);
  Documents docs(a);
  const size_t parts = std::max(ksplits > 1 ? rounded((size_t)ksplits * 2 * pairs * a.M * dp * 4) : 0, qsplits > 1 ? rounded((size_t)qsplits * pairs * rows * dp * 4) : 0);
  char* ws;
  TRY(c.space(2 * st + docs.bytes + parts, &ws));
  a.less = (float*)ws;
  a.delta = (float*)(ws + st);
  docs.place(&a, ws + 2 * st);
  a.part_o = (float*)(ws + 2 * st + docs.bytes);
  if (a.kdoc && a.M > 0 && a.N > 0) TRY(c.launch("gr_attention_ranges", [&] { return ranges(a, c.ctx->stream); }));
  if (a.N > 0) {
    TRY(c.launch("gr_attention_statistics", [&] { return statistics(a, type, c.ctx->stream); }));
    a.splits = qsplits;
    a.blocks = (int)qblocks;
    const unsigned grid = grid_of((int)pairs, qblocks * qsplits);
    TRY(c.launch("gr_attention_grad_q", [&] { return type == TYPE_BF16 ? grad_q_bf16(a, dp, mode, grid, c.ctx->stream) : grad_q_f32(a, dp, mode, grid, c.ctx->stream); }));
    if (qsplits > 1) TRY(c.launch("gr_attention_sum_parts", [&] { return sum_parts(a, type, dp, true, c.ctx->stream); }));
  }
  if (a.M > 0) {
    a.splits = ksplits;
    a.blocks = (int)kblocks;
    const unsigned grid = grid_of((int)pairs, kblocks * ksplits);
    TRY(c.launch("gr_attention_grad_kv", [&] { return type == TYPE_BF16 ? grad_kv_bf16(a, dp, mode, grid, c.ctx->stream) : grad_kv_f32(a, dp, mode, grid, c.ctx->stream); }));
    if (ksplits > 1) TRY(c.launch("gr_attention_sum_parts", [&] { return sum_parts(a, type, dp, false, c.ctx->stream); }));
  }
  return GR_OK;
}

static gr_status rotary_call(gr_ctx* ctx, gr_array x, gr_array positions, int64_t position, const double* frequencies, int pairs, int interleaved, int inverse,
                             double factor, gr_array out) {
  Call c{ctx, "rotary"};
  const Node* n = lookup(ctx, x);
  if (!n) return c.error(GR_ERR_HANDLE, "x: bad handle");
  if (n->kind == Kind::SCALAR) return c.error(GR_ERR_UNSUPPORTED, "x is a bare scalar");
  if (n->dtype != GR_F32 && n->dtype != GR_BF16) return c.error(GR_ERR_DTYPE, "x must be f32 or bf16");
  if (n->ndim != 4) return c.error(GR_ERR_SHAPE, "x is (B, N, H, D)");
  const int64_t B = n->shape[0], N = n->shape[1], H = n->shape[2], D = n->shape[3];
  const int dt = n->dtype;
  if (pairs < 0 || pairs > MAX_PAIRS || (pairs > 0 && !frequencies)) return c.error(GR_ERR_ARG, "0 to 256 pairs, with a frequency each");
  if (2 * (int64_t)pairs > D) return c.error(GR_ERR_SHAPE, "a head has fewer than 2 pairs values");
  if ((interleaved != 0 && interleaved != 1) || (inverse != 0 && inverse != 1)) return c.error(GR_ERR_ARG, "interleaved and inverse must be 0 or 1");
  if (!(std::fabs(factor) <= FLT_MAX)) return c.error(GR_ERR_ARG, "factor must be a finite float32");
  if (position < -(int64_t(1) << 40) || position > (int64_t(1) << 40)) return c.error(GR_ERR_ARG, "position beyond 2^40");
  for (int i = 0; i < pairs; ++i) if (!std::isfinite(frequencies[i])) return c.error(GR_ERR_ARG, "a frequency is not finite");
  if (B > LIMIT || N > LIMIT || D > LIMIT || B * N > LIMIT) return c.error(GR_ERR_UNSUPPORTED, "more than 2^30 tokens or values of a head");
  TRY(c.take(x, "x", dt, {B, N, H, D}, false));
  if (positions) TRY(c.take(positions, "positions", GR_I32, {B, N}, false));
  TRY(c.take(out, "out", dt, {B, N, H, D}, true));
  Rotary r;
  TRY(c.tensor(out, "out", &r.y));
  TRY(rows_are_neighbours(c, {x}));
  TRY(c.settle(true));
  TRY(c.tensor(x, "x", &r.x));
  TRY(c.tensor(out, "out", &r.y));
  r.positions = c.whole(positions, &r.positions_sb, &r.positions_sn);
  r.position = position;
  r.B = (int)B; r.N = (int)N; r.D = (int)D; r.pairs = pairs; r.interleaved = interleaved; r.inverse = inverse;
  r.factor = (float)factor;
  for (int i = 0; i < pairs; ++i) r.turns[i] = frequencies[i] * 0.15915494309189535;   // 1 / (2 pi)
  if (B * N * H * D == 0) return GR_OK;
  if (H > LIMIT) return c.error(GR_ERR_UNSUPPORTED, "more than 2^30 heads");
  r.H = (int)H;
  // Tokens of a workgroup: enough vectors for its 256 threads, and no more than 32 KiB of sines; for few tokens fewer, and runs of heads.
  const int64_t vectors = std::max<int64_t>(1, D * (int64_t)itemsize((gr_dtype)dt) / 32), tokens = B * N;
  int64_t per = std::max<int64_t>(1, std::min<int64_t>(1024 / (H * vectors) + 1, 4096 / std::max(1, pairs)));
  while (per > 1 && (tokens + per - 1) / per < 512) per /= 2;
  r.tokens = (int)per;
  int64_t heads = H;
  while (heads > 1 && (tokens + per - 1) / per * ((H + heads - 1) / heads) < 256 && heads * vectors * per > 256) heads = (heads + 1) / 2;
  while ((H + heads - 1) / heads > 65535) heads *= 2;
  r.heads = (int)heads;
  return c.launch("gr_rotary", [&] { return rotary(r, dt == GR_BF16 ? TYPE_BF16 : TYPE_F32, ctx->stream); });
}

}  // namespace attn

// No exception leaves the C ABI.
template <class F>
static gr_status guarded(gr_ctx* ctx, F&& f) {
  if (!ctx) return GR_ERR_ARG;
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail(ctx, GR_ERR_OOM, "out of host memory");
  } catch (...) {
    return fail(ctx, GR_ERR_HIP, "unexpected exception");
  }
}

}  // namespace gr

using namespace gr;

extern "C" {

gr_status gr_attention(gr_ctx* ctx, const gr_scores* scores, gr_array q, gr_array k, gr_array v, gr_array out, gr_array lse, gr_array rest) {
  return guarded(ctx, [&] { return attn::attention(ctx, scores, q, k, v, out, lse, rest); });
}

gr_status gr_attention_grad(gr_ctx* ctx, const gr_scores* scores, gr_array q, gr_array k, gr_array v, gr_array out, gr_array rest, gr_array lse,
                            gr_array dout, gr_array dq, gr_array dk, gr_array dv) {
  return guarded(ctx, [&] { return attn::grad(ctx, scores, q, k, v, out, rest, lse, dout, dq, dk, dv); });
}

gr_status gr_attention_step(gr_ctx* ctx, const gr_scores* scores, gr_array q, gr_array k, gr_array v, gr_array out) {
  return guarded(ctx, [&] { return attn::step(ctx, scores, q, k, v, out); });
}

gr_status gr_rotary(gr_ctx* ctx, gr_array x, gr_array positions, int64_t position, const double* frequencies, int pairs, int interleaved, int inverse,
                    double factor, gr_array out) {
  return guarded(ctx, [&] { return attn::rotary_call(ctx, x, positions, position, frequencies, pairs, interleaved, inverse, factor, out); });
}

}  // extern "C"
