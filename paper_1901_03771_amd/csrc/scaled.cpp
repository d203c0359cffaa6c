// Root-mean-square norms, 8-bit tensors with scales and their products: checks of the arguments, evaluation of lazy operands, temporary memory and
// the choice of kernels (grumpy_hip_scaled.h; kernels: norm.hip, quantize.hip, scaled_dot.hip).
#include "scaled.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "../../include/grumpy_hip_scaled.h"
#include "call.h"

namespace gr {
namespace scaled {

constexpr int64_t LIMIT = int64_t(1) << 30;      // extents that kernels hold in 32 bits
constexpr int64_t GROUPS = int64_t(1) << 22;     // workgroups of a launch: 512 threads of each do not reach 2^32

struct Call : gr::Call {
  static int type_of(int dtype) { return dtype == GR_F32 ? F32 : dtype == GR_BF16 ? BF16 : E4M3; }

  gr_status take_shape(gr_array a, const char* what, int dtype, const int64_t* shape, int ndim, bool result) {
    switch (ndim) {
      case 1: return take(a, what, dtype, {shape[0]}, result);
      case 2: return take(a, what, dtype, {shape[0], shape[1]}, result);
      case 3: return take(a, what, dtype, {shape[0], shape[1], shape[2]}, result);
      default: return take(a, what, dtype, {shape[0], shape[1], shape[2], shape[3]}, result);
    }
  }

  gr_status float_operand(gr_array a, const char* what, const Node** n) const {
    *n = lookup(ctx, a);
    if (!*n) return error(GR_ERR_HANDLE, std::string(what) + ": bad handle");
    if ((*n)->kind == Kind::SCALAR) return error(GR_ERR_UNSUPPORTED, std::string(what) + " is a bare scalar");
    if ((*n)->dtype != GR_F32 && (*n)->dtype != GR_BF16) return error(GR_ERR_DTYPE, std::string(what) + " must be f32 or bf16");
    return GR_OK;
  }

  // Where arrays are stored already, the values of their rows are neighbours.
  gr_status neighbours(std::initializer_list<std::pair<gr_array, const char*>> arrays) const {
    for (auto& a : arrays) TRY(neighbours(a.first, a.second));
    return GR_OK;
  }
  gr_status neighbours(gr_array a, const char* what) const {
    if (!a || !resolved(ctx, a)) return GR_OK;
    const Node* n = lookup(ctx, a);
    const StoredView v = view(a);
    if (n->count() > 0 && n->shape[n->ndim - 1] > 1 && v.strides[n->ndim - 1] != 1) return error(GR_ERR_UNSUPPORTED, std::string(what) + ": the values of a row are not neighbours");
    return GR_OK;
  }

  int64_t step(gr_array a, int d) const {
    const Node* n = lookup(ctx, a);
    return n->shape[d] > 1 ? view(a).strides[d] : 0;
  }
};

// The rows of tensors of one shape, axes that can be walked as one taken together.
struct Walk {
  Call& c;
  gr_array arrays[5];
  Rows* rows[5];
  int count = 0;
  explicit Walk(Call& call) : c(call) {}
  void add(gr_array a, Rows* r) { if (a) { arrays[count] = a; rows[count++] = r; } }
  void fill(Norm* n) {
    const Node* x = lookup(c.ctx, arrays[0]);
    int64_t extents[3] = {1, 1, 1}, steps[5][3] = {};
    StoredView views[5];
    for (int t = 0; t < count; ++t) {
      views[t] = c.view(arrays[t]);
      rows[t]->p = views[t].data;
    }
    int k = 0;
    for (int d = 0; d + 1 < x->ndim; ++d) {
      if (x->shape[d] <= 1) continue;
      bool joined = k > 0;
      for (int t = 0; t < count && joined; ++t) joined = steps[t][k - 1] == views[t].strides[d] * x->shape[d];
      if (joined) extents[k - 1] *= x->shape[d];
      else extents[k++] = x->shape[d];
      for (int t = 0; t < count; ++t) steps[t][k - 1] = views[t].strides[d];
    }
    n->n1 = k >= 2 ? (int)extents[k - 2] : 1;
    n->n2 = k >= 2 ? (int)extents[k - 1] : 1;
    for (int t = 0; t < count; ++t) {
      rows[t]->s0 = k == 1 || k == 3 ? steps[t][0] : 0;
      rows[t]->s1 = k >= 2 ? steps[t][k - 2] : 0;
      rows[t]->s2 = k >= 2 ? steps[t][k - 1] : 0;
    }
  }
};

struct RowsOf { int64_t rows = 1, D = 0; };
static gr_status rows_of(Call& c, const Node* x, const char* what, RowsOf* r) {
  if (x->ndim < 1 || x->ndim > 4) return c.error(GR_ERR_SHAPE, std::string(what) + " has 1 to 4 axes");
  r->D = x->shape[x->ndim - 1];
  if (r->D > MOST_VALUES) return c.error(GR_ERR_UNSUPPORTED, "more than 32768 values in a row");
  for (int d = 0; d + 1 < x->ndim; ++d) {
    r->rows *= x->shape[d];
    if (r->rows > LIMIT) return c.error(GR_ERR_UNSUPPORTED, "more than 2^30 rows");
  }
  return GR_OK;
}

static gr_status take_weight(Call& c, gr_array weight, int dtype, int64_t D, double eps, double offset) {
  if (!(eps >= 1e-12 && eps <= 1.0)) return c.error(GR_ERR_ARG, "eps must be between 1e-12 and 1");
  if (!(std::fabs(offset) <= FLT_MAX)) return c.error(GR_ERR_ARG, "offset must be a finite float32");
  if (!weight) return offset == 0.0 ? GR_OK : c.error(GR_ERR_ARG, "an offset without a weight");
  const Node* w = lookup(c.ctx, weight);
  if (!w) return c.error(GR_ERR_HANDLE, "weight: bad handle");
  return c.take(weight, "weight", w->kind != Kind::SCALAR && (int)w->dtype == dtype ? dtype : GR_F32, {D}, false);
}
static void fill_weight(Call& c, gr_array weight, double eps, double offset, Norm* a) {
  a->eps = (float)eps;
  a->offset = (float)offset;
  if (!weight) return;
  const StoredView v = c.view(weight);
  if (lookup(c.ctx, weight)->dtype == GR_BF16) a->weight16 = v.data;
  else a->weight = (const float*)v.data;
  a->weight_s = c.step(weight, 0);
  if (a->D == 1) a->weight_s = 1;
}

static int64_t rows_at_once(Shape s) { return s.threads < 256 ? 256 / s.threads : 1; }

static gr_status rms_norm(gr_ctx* ctx, gr_array x, gr_array residual, gr_array weight, double eps, double offset, gr_array total, gr_array out, gr_array scales) {
  Call c{ctx, "rms_norm"};
  const Node *n, *o;
  RowsOf r;
  TRY(c.float_operand(x, "x", &n));
  TRY(rows_of(c, n, "x", &r));
  const int dt = n->dtype, ndim = n->ndim;
  int64_t shape[4], blocks[4];
  std::copy(n->shape, n->shape + ndim, shape);
  std::copy(shape, shape + ndim, blocks);
  blocks[ndim - 1] = blocks_of(r.D);
  TRY(c.take_shape(x, "x", dt, shape, ndim, false));
  if (residual) TRY(c.take_shape(residual, "residual", dt, shape, ndim, false));
  TRY(take_weight(c, weight, dt, r.D, eps, offset));
  if (total && !residual) return c.error(GR_ERR_ARG, "total without a residual is x");
  if (total) TRY(c.take_shape(total, "total", dt, shape, ndim, true));
  o = lookup(ctx, out);
  if (!o) return c.error(GR_ERR_HANDLE, "out: bad handle");
  const bool eight = o->kind != Kind::SCALAR && o->dtype == GR_E4M3;
  TRY(c.take_shape(out, "out", eight ? (int)GR_E4M3 : dt, shape, ndim, true));
  if (eight != (scales != 0)) return c.error(GR_ERR_ARG, eight ? "an 8-bit result has scales" : "scales are for an 8-bit result");
  if (scales) TRY(c.take_shape(scales, "scales", GR_F32, blocks, ndim, true));
  TRY(c.neighbours({{x, "x"}, {residual, "residual"}, {total, "total"}, {out, "out"}}));
  TRY(c.settle(true));
  TRY(c.neighbours({{x, "x"}, {residual, "residual"}}));   // (views of what has just been evaluated)
  if (r.rows == 0 || r.D == 0) return GR_OK;
  Norm a;
  a.rows = r.rows;
  a.D = (int)r.D;
  Walk w(c);
  w.add(x, &a.x);
  w.add(residual, &a.residual);
  w.add(total, &a.total);
  w.add(out, &a.out);
  w.add(scales, &a.scales);
  w.fill(&a);
  if (scales) a.scales_s = c.step(scales, ndim - 1);
  fill_weight(c, weight, eps, offset, &a);
  const int type = Call::type_of(dt);
  const Shape s = norm_shape(type, a.D, false);
  const int64_t per = rows_at_once(s), groups = (a.rows + per - 1) / per;
  const unsigned grid = (unsigned)std::min<int64_t>(groups, s.threads <= 512 ? 2048 : 512);   // about what fits the compute units at once
  return c.launch("gr_rms_norm", [&] { return norm(a, type, eight, s, grid, ctx->stream); });
}

static gr_status rms_norm_grad(gr_ctx* ctx, gr_array dout, gr_array total, gr_array weight, gr_array dtotal, double eps, double offset, gr_array dx, gr_array dweight) {
  Call c{ctx, "rms_norm_grad"};
  const Node* n;
  RowsOf r;
  TRY(c.float_operand(total, "total", &n));
  TRY(rows_of(c, n, "total", &r));
  const int dt = n->dtype, ndim = n->ndim;
  int64_t shape[4];
  std::copy(n->shape, n->shape + ndim, shape);
  TRY(c.take_shape(total, "total", dt, shape, ndim, false));
  TRY(c.take_shape(dout, "dout", dt, shape, ndim, false));
  if (dtotal) TRY(c.take_shape(dtotal, "dtotal", dt, shape, ndim, false));
  TRY(take_weight(c, weight, dt, r.D, eps, offset));
  TRY(c.take_shape(dx, "dx", dt, shape, ndim, true));
  if (dweight) TRY(c.take(dweight, "dweight", GR_F32, {r.D}, true));
  TRY(c.neighbours({{total, "total"}, {dout, "dout"}, {dtotal, "dtotal"}, {dx, "dx"}}));
  TRY(c.settle(true));
  TRY(c.neighbours({{total, "total"}, {dout, "dout"}, {dtotal, "dtotal"}}));
  if (r.D == 0) return GR_OK;
  Norm a;
  a.rows = r.rows;
  a.D = (int)r.D;
  Walk w(c);
  w.add(total, &a.x);
  w.add(dout, &a.dout);
  w.add(dtotal, &a.residual);
  w.add(dx, &a.dx);
  w.fill(&a);
  fill_weight(c, weight, eps, offset, &a);
  const int type = Call::type_of(dt);
  const Shape s = norm_shape(type, a.D, true);
  const int64_t per = rows_at_once(s), groups = (a.rows + per - 1) / per;
  // (each leaves a row of sums: 8192 rows of 4096 bf16 values take 57, 61, 67 us with 512, 768, 1024 workgroups, 71 with 256)
  a.groups = (int)std::min<int64_t>(groups, s.threads == 1024 ? 256 : 512);
  if (dweight) {
    char* ws;
    TRY(c.space(rounded((size_t)a.groups * a.D * 4), &ws));
    a.parts = (float*)ws;
    a.dweight = (float*)c.view(dweight).data;
    a.dweight_s = c.step(dweight, 0);
  }
  if (a.rows > 0) TRY(c.launch("gr_rms_norm_grad", [&] { return norm_grad(a, type, s, (unsigned)a.groups, ctx->stream); }));
  if (dweight) TRY(c.launch("gr_rms_norm_sum", [&] { return norm_sum(a, ctx->stream); }));
  return GR_OK;
}

static gr_status quantize_call(gr_ctx* ctx, gr_array x, int blocks, int transposed, gr_array out, gr_array scales) {
  Call c{ctx, "quantize"};
  const Node* n;
  TRY(c.float_operand(x, "x", &n));
  if (n->ndim != 2) return c.error(GR_ERR_SHAPE, "x is (M, K)");
  if ((blocks != 0 && blocks != 1) || (transposed != 0 && transposed != 1)) return c.error(GR_ERR_ARG, "blocks and transposed must be 0 or 1");
  const int64_t M = n->shape[0], K = n->shape[1], R = transposed ? K : M, C = transposed ? M : K;
  const int dt = n->dtype;
  // (the fewest rows that a workgroup has are 8, and a tile is 128 x 128)
  if ((blocks || transposed ? blocks_of(M) : (M + 7) / 8) * blocks_of(K) > GROUPS * (blocks || transposed ? 1 : 2)) return c.error(GR_ERR_UNSUPPORTED, "more values than a launch holds");
  TRY(c.take(x, "x", dt, {M, K}, false));
  TRY(c.take(out, "out", GR_E4M3, {R, C}, true));
  TRY(c.take(scales, "scales", GR_F32, {blocks ? blocks_of(R) : R, blocks_of(C)}, true));
  TRY(c.neighbours(x, "x"));
  TRY(c.neighbours(out, "out"));
  TRY(c.settle());
  TRY(c.neighbours(x, "x"));
  if (M == 0 || K == 0) return GR_OK;
  Quantize a;
  a.x = c.view(x).data;
  a.x_s = c.step(x, 0);
  a.out = c.view(out).data;
  a.out_s = c.step(out, 0);
  a.scales = (float*)c.view(scales).data;
  a.scales_sm = c.step(scales, 0);
  a.scales_sk = c.step(scales, 1);
  a.M = M;
  a.K = K;
  return c.launch("gr_quantize", [&] { return quantize(a, Call::type_of(dt), blocks != 0, transposed != 0, ctx->stream); });
}

// The form of a product, its tiles, and how many splits of the blocks of K there are where tiles are few.
static int choose(Dot* d, int out, bool blocks) {
  const int64_t M = d->M, N = d->N, K = d->K, KB = d->KB;
  auto tiles_of = [&](int64_t tm, int64_t tn) {
    d->mt = (int)((M + tm - 1) / tm);
    d->nt = (int)((N + tn - 1) / tn);
    return (int64_t)d->mt * d->nt;
  };
  // Straight into LDS where rows are of whole vectors, do not overlap, and those of a tile lie within 2^31 bytes; else through registers (512 rows by 4096 x 4080: 18.5 us, by 4096 x 4088 and
  // 4096 x 4095 25).
  auto direct = [&](const uint8_t* p, int64_t rows, int64_t s) { return (uintptr_t)p % 16 == 0 && (rows == 1 || (s % 16 == 0 && s >= K && s <= (int64_t(1) << 22))) && K <= (int64_t(1) << 22); };
  const bool straight = K % 16 == 0 && direct(d->a, M, d->a_s) && direct(d->b, N, d->b_s);
  // Few rows: bound by the memory that b is read from, which 256 workgroups keep busy.  Rounds of 16 blocks, and a join of splits, take what was measured (us).  (4 rows by 4096 x 4096: 7.5 with one, 8.8
  // with two splits; by 4096 x 14336 18.7 and 15.0; by 1024 x 8192 10.9, 10.1, 8.4 with 1, 2, 4.  16 rows by 4096 x 4096 8.4, tiles of 64 x 128 9.6; 32 rows by 4096 x 14336: 20.8 and 15.0, by
  // 4096 x 4088, through registers, 8.5 and 13.3.)
  if (M <= (straight ? 16 : 32)) {
    const int64_t most = std::max<int64_t>(1, 256 / tiles_of(32, 32));
    double least = 0.0;
    for (int64_t s = 1; s == 1 || (s <= most && 16 * (s - 1) < KB); ++s) {   // (until a round is all)
      const double us = 1.7 * (double)((KB + 16 * s - 1) / (16 * s)) + (s > 1 ? 2.0 + 0.6 * (double)((s + 7) / 8) : 0.0);
      if (s > 1 && us >= least) continue;
      least = us;
      d->splits = (int)s;
    }
    return ((uintptr_t)d->a | (uintptr_t)d->b | (uintptr_t)(M > 1 ? d->a_s : 0) | (uintptr_t)(N > 1 ? d->b_s : 0) | (uintptr_t)(K % BLOCK ? K : 0)) % 4 == 0 ? DOT_FEW : DOT_FEW_WORDS;
  }
  // Else tiles of 128 rows of b and 64 or 128 of a, with splits of K, or of 256 x 256 (straight, bf16 results), whichever takes least by what was measured (us): a
  // start, the blocks of a workgroup alone and what its neighbours add, rounds of one or two workgroups a compute unit, and the join of splits: a launch, its parts written and read.  (512 x 4096 x 4096: 16 with 256 tiles of 64
  // rows, 26 with 128 of 128 rows, 23 with those in two splits; 1024 x 8192 x 4096: 51 and 42; 64 x 4096 x 14336: 39, 25, 17, 17 with 1, 2, 4, 8; 192 x 4096 x 14336: 41, 27, 25, 28 with 1, 2, 5,
  // 8; 8192^3: 746, 602 and 451 with the three tiles; 2304 x 8192 x 4096, 288 of the largest: 105, 97, 106; 64 x 65536 x 4096: 68, 69, 77; with
  // scales of b's rows 8192^3 674 and 625 with the larger two, 4096 x 6144 x 16384, 384 of the largest, 488 and 586; through registers, 512 x 4096 x 4095: 25 and 33, 1024 x 4096 x 4095: 44 and 33.)
  const bool proper = out == GR_F32;
  struct Form { int which; int64_t high, wide, slots; double start, alone, more; };
  const Form low = straight ? Form{DOT_LOW, 64, 128, 512, 3.0, proper ? 0.70 : blocks ? 0.34 : 0.42, proper ? 0.45 : blocks ? 0.35 : 0.37}
                            : Form{DOT_STAGED_LOW, 64, 128, 512, 3.0, proper ? 0.87 : 0.66, proper ? 0.95 : 0.66};
  const Form middle = straight ? Form{DOT_DIRECT, 128, 128, 512, 5.0, proper ? 1.13 : blocks ? 0.65 : 0.72, proper ? 0.72 : blocks ? 0.54 : 0.57}
                               : Form{DOT_STAGED, 128, 128, 256, 5.0, proper ? 1.00 : 0.70, proper ? 0.30 : 0.19};
  const Form large = {DOT_LARGE, 256, 256, 256, 6.0, blocks ? 0.60 : 1.20, blocks ? 1.15 : 1.20};
  // A launch holds GROUPS workgroups of any form; where tiles of 64 rows are more, those of 128 rows are no more than that.
  const Form* best = nullptr;
  double least = 0.0;
  for (const Form* f : {&low, &middle, &large}) {
    if (f == &middle && M <= 64) continue;
    if (f == &large && (M <= 128 || !straight || proper)) continue;
    const int64_t tiles = tiles_of(f->high, f->wide);
    for (int64_t s = 1; tiles * s <= GROUPS && (s == 1 || (f != &large && s <= 16 && s <= KB / 4)); ++s) {
      const int64_t groups = tiles * s, over = groups % f->slots;
      double beside = std::min(1.0, (double)groups / f->slots), rounds = 1.0;
      if (f->slots == 512) beside = groups > 256 ? 1.2 * beside - 0.2 : 0.0;
      if (groups > f->slots) rounds = (double)(groups / f->slots) + (over == 0 ? 0.0 : f->slots == 256 ? 1.0 : 0.5 + 0.5 * (double)over / f->slots);
      const double us = f->start + (double)((KB + s - 1) / s) * rounds * (f->alone + f->more * beside) + (s > 1 ? 5.5 + (double)(s * M * N) * 8e-7 : 0.0);
      if (best && us >= least) continue;
      least = us;
      best = f;
      d->splits = (int)s;
    }
  }
  tiles_of(best->high, best->wide);
  return best->which;
}

static gr_status dot_call(gr_ctx* ctx, gr_array a, gr_array a_scales, gr_array b, gr_array b_scales, gr_array out) {
  Call c{ctx, "dot_scaled"};
  const Node *x = lookup(ctx, a), *y = lookup(ctx, b), *s = lookup(ctx, b_scales), *o = lookup(ctx, out);
  if (!x || !y || !s || !o) return c.error(GR_ERR_HANDLE, std::string(!x ? "a" : !y ? "b" : !s ? "b_scales" : "out") + ": bad handle");
  for (const Node* n : {x, y, s, o}) if (n->kind == Kind::SCALAR) return c.error(GR_ERR_UNSUPPORTED, "an operand is a bare scalar");
  if (x->dtype != GR_E4M3 || y->dtype != GR_E4M3) return c.error(GR_ERR_DTYPE, "a and b must be e4m3");
  if (o->dtype != GR_F32 && o->dtype != GR_BF16) return c.error(GR_ERR_DTYPE, "out must be f32 or bf16");
  if (x->ndim != 2 || y->ndim != 2 || x->shape[1] != y->shape[1]) return c.error(GR_ERR_SHAPE, "a is (M, K) and b (N, K)");
  const int64_t M = x->shape[0], N = y->shape[0], K = x->shape[1], KB = blocks_of(K);
  if (M > LIMIT || N > LIMIT || K > LIMIT) return c.error(GR_ERR_UNSUPPORTED, "more than 2^30 rows or places");
  const int dt = o->dtype;
  const bool blocks = s->ndim == 2 && s->shape[0] == blocks_of(N);
  TRY(c.take(a, "a", GR_E4M3, {M, K}, false));
  TRY(c.take(a_scales, "a_scales", GR_F32, {M, KB}, false));
  TRY(c.take(b, "b", GR_E4M3, {N, K}, false));
  TRY(c.take(b_scales, "b_scales", GR_F32, {blocks ? blocks_of(N) : N, KB}, false));
  TRY(c.take(out, "out", dt, {M, N}, true));
  TRY(c.neighbours({{a, "a"}, {b, "b"}, {out, "out"}}));
  Dot d;
  if (blocks_of(M) * blocks_of(N) > GROUPS || N > GROUPS * 32) return c.error(GR_ERR_UNSUPPORTED, "more results than a launch holds");   // (32 columns a workgroup at least)
  TRY(c.settle());
  if (M == 0 || N == 0) return GR_OK;
  d.a = (const uint8_t*)c.view(a).data;
  d.a_s = c.step(a, 0);
  d.b = (const uint8_t*)c.view(b).data;
  d.b_s = c.step(b, 0);
  d.sa = (const float*)c.view(a_scales).data;
  d.sa_m = c.step(a_scales, 0);
  d.sa_k = c.step(a_scales, 1);
  d.sb = (const float*)c.view(b_scales).data;
  d.sb_n = c.step(b_scales, 0);
  d.sb_k = c.step(b_scales, 1);
  d.out = c.view(out).data;
  d.out_s = c.step(out, 0);
  d.M = (int)M;
  d.N = (int)N;
  d.K = (int)K;
  d.KB = (int)KB;
  const int form = choose(&d, dt, blocks);
  if (d.splits > 1) {
    char* ws;
    TRY(c.space(rounded((size_t)d.splits * M * N * 4), &ws));
    d.parts = (float*)ws;
  }
  const int type = Call::type_of(dt);
  TRY(c.launch("gr_dot_scaled", [&] { return dot(d, form, blocks, type, ctx->stream); }));
  if (d.splits > 1) TRY(c.launch("gr_dot_scaled_join", [&] { return dot_join(d, type, ctx->stream); }));
  return GR_OK;
}

}  // namespace scaled
}  // namespace gr

using namespace gr;

extern "C" {

gr_status gr_rms_norm(gr_ctx* ctx, gr_array x, gr_array residual, gr_array weight, double eps, double offset, gr_array total, gr_array out, gr_array scales) {
  return guarded(ctx, [&] { return scaled::rms_norm(ctx, x, residual, weight, eps, offset, total, out, scales); });
}

gr_status gr_rms_norm_grad(gr_ctx* ctx, gr_array dout, gr_array total, gr_array weight, gr_array dtotal, double eps, double offset, gr_array dx, gr_array dweight) {
  return guarded(ctx, [&] { return scaled::rms_norm_grad(ctx, dout, total, weight, dtotal, eps, offset, dx, dweight); });
}

gr_status gr_quantize(gr_ctx* ctx, gr_array x, int blocks, int transposed, gr_array out, gr_array scales) {
  return guarded(ctx, [&] { return scaled::quantize_call(ctx, x, blocks, transposed, out, scales); });
}

gr_status gr_dot_scaled(gr_ctx* ctx, gr_array a, gr_array a_scales, gr_array b, gr_array b_scales, gr_array out) {
  return guarded(ctx, [&] { return scaled::dot_call(ctx, a, a_scales, b, b_scales, out); });
}

}  // extern "C"
