// What the calls that launch kernels of their own share on the host side (attention.cpp, scaled.cpp): checks of operands and results, evaluation
// of lazy operands, temporary memory, launches.
#pragma once

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <climits>
#include <cstdlib>
#include <new>

#include "ctx.h"

#define CALL_HIP(c, call)                                                                    \
  do {                                                                                       \
    hipError_t e_ = (call);                                                                  \
    if (e_ != hipSuccess) return fail(c, GR_ERR_HIP, std::string(#call ": ") + hipGetErrorString(e_)); \
  } while (0)

#define TRY(x) do { gr_status st_ = (x); if (st_ != GR_OK) return st_; } while (0)

namespace gr {

// The operands or results of a call, by handle and name: none has more.  (Nothing is allocated for them: a call of small tensors is bound by the host.)
struct Named {
  std::pair<gr_array, const char*> list[16];
  int n = 0;
  void push_back(const std::pair<gr_array, const char*>& a) { if (n == 16) throw std::bad_alloc(); list[n++] = a; }
  const std::pair<gr_array, const char*>* begin() const { return list; }
  const std::pair<gr_array, const char*>* end() const { return list + n; }
};

struct Call {
  gr_ctx* ctx;
  const char* name;
  Named inputs, results;

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

  // Do two views share no element?  Certain where their extents do not meet, and where they are parts of one packed array: the
  // same steps between batches and rows (the first two axes, of two axes the first), and within a row two stretches that do not meet.
  bool apart(gr_array a, gr_array b) const {
    const StoredView x = view(a), y = view(b);
    if (!(x.lo < y.hi && y.lo < x.hi)) return true;
    const Node *m = lookup(ctx, a), *n = lookup(ctx, b);
    if (m->ndim != n->ndim || m->ndim < 2 || m->ndim > 4 || m->dtype != n->dtype) return false;
    const int outer = m->ndim == 2 ? 1 : 2;
    const int64_t size = (int64_t)itemsize(m->dtype);
    int64_t least = INT64_MAX;
    int64_t steps[2] = {0, 0}, counts[2] = {1, 1};
    for (int d = 0; d < outer; ++d) {
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
      for (int d = outer; d < t->ndim; ++d) (v.strides[d] < 0 ? *lo : *hi) += v.strides[d] * (t->shape[d] - 1);
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

  // Temporary memory of the call.
  gr_status space(size_t bytes, char** to) {
    *to = nullptr;
    if (bytes == 0) return GR_OK;
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (ctx->device >= 0) CALL_HIP(ctx, hipStreamIsCapturing(ctx->stream, &cap));
    const bool capturing = cap != hipStreamCaptureStatusNone;
    if (bytes > ctx->call_space_bytes) {
      if (capturing) return error(GR_ERR_OOM, "the stream is being captured and the call needs " + std::to_string(bytes) + " bytes of temporary memory: run it once before the capture");
      if (ctx->call_space) {
        // (a graph may still use it)
        if (ctx->call_captured) ctx->call_kept.push_back({ctx->call_space, ctx->call_space_bytes});
        else ctx_free(ctx, ctx->call_space, ctx->call_space_bytes);
      }
      ctx->call_space = nullptr;
      ctx->call_space_bytes = 0;
      ctx->call_captured = false;
      void* p = ctx_alloc(ctx, bytes);
      if (!p) return error(GR_ERR_OOM, "allocator returned NULL for " + std::to_string(bytes) + " bytes of temporary memory");
      ctx->call_space = p;
      ctx->call_space_bytes = bytes;
    }
    if (capturing) ctx->call_captured = true;
    *to = (char*)ctx->call_space;
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
      CALL_HIP(ctx, hipStreamIsCapturing(ctx->stream, &cap));
      profile = cap == hipStreamCaptureStatusNone;
    }
    if (profile) {
      for (hipEvent_t* ev : {&e0, &e1}) {
        if (!ctx->event_pool.empty()) { *ev = ctx->event_pool.back(); ctx->event_pool.pop_back(); }
        else CALL_HIP(ctx, hipEventCreate(ev));
      }
      CALL_HIP(ctx, hipEventRecord(e0, ctx->stream));
    }
    (void)hipGetLastError();   // (an error that an earlier call of the thread has left would be taken for the launch's)
    CALL_HIP(ctx, f());
    if (profile) {
      CALL_HIP(ctx, hipEventRecord(e1, ctx->stream));
      ctx->prof.push_back({kernel, e0, e1});
    }
    ctx->stats.kernel_launches++;
    return GR_OK;
  }
};

inline bool resolved(gr_ctx* ctx, gr_array a) {
  StoredView v;
  return stored_view(lookup(ctx, a), &v);
}

inline size_t rounded(size_t n) { return (n + 255) & ~(size_t)255; }

// The context's device is the current one while a call runs, whichever the caller's is.
struct OnDevice {
  int before = -1;
  explicit OnDevice(int device) {
    if (device < 0) return;
    if (hipGetDevice(&before) != hipSuccess || before == device || hipSetDevice(device) != hipSuccess) before = -1;
  }
  ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};

// No exception leaves the C ABI.
template <class F>
gr_status guarded(gr_ctx* ctx, F&& f) {
  if (!ctx) return GR_ERR_ARG;
  const OnDevice on(ctx->device);
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail(ctx, GR_ERR_OOM, "out of host memory");
  } catch (...) {
    return fail(ctx, GR_ERR_HIP, "unexpected exception");
  }
}

}  // namespace gr
