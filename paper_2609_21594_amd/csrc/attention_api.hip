// C ABI of the attention block: argument checks, scratch layout, launches.
// The kernels live in attention_kernels.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <exception>
#include <vector>

#include "../../include/muon_hip.h"
#include "attention_internal.h"

namespace {

using muon::Extent;
using muon::Heads;
using muon::Strided;

constexpr int64_t kMaxTokens = int64_t(1) << 30;   // token counts and tile indices are 32 bits on the device
constexpr int64_t kMaxTokenStride = int64_t(1) << 24;  // bytes: a tile's rows are addressed by 32-bit offsets
constexpr int64_t kMaxClipBlocks = 1 << 23, kMaxClipRows = kMaxClipBlocks * muon::kClipRowsFew;
constexpr int kMaxHeadDim = 128, kMaxRotaryDim = 1024;

struct Why {
  char text[256] = {0};
  muon_status_t fail(muon_status_t st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof text, fmt, ap);
    va_end(ap);
    return st;
  }
  muon_status_t invalid(const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof text, fmt, ap);
    va_end(ap);
    return MUON_ERR_INVALID_ARGUMENT;
  }
};

struct CurrentDevice {
  int prev = -1;
  bool ok = false;
  explicit CurrentDevice(int dev) {
    if (hipGetDevice(&prev) != hipSuccess) return;
    ok = prev == dev || hipSetDevice(dev) == hipSuccess;
    if (prev == dev) prev = -1;
  }
  ~CurrentDevice() { if (prev >= 0) (void)hipSetDevice(prev); }
};

// The handle's timer, but not for launches that go into a graph: events recorded
// there belong to its replays and cannot be waited for.
muon::LaunchTimer* timer_on(muon_handle_t h, hipStream_t stream) {
  muon::LaunchTimer* const t = muon::handle_timer(h);
  if (!t) return nullptr;
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(stream, &capture) == hipSuccess) return capture == hipStreamCaptureStatusNone ? t : nullptr;
  (void)hipGetLastError();
  return nullptr;
}

int64_t elem_size(int dtype) { return dtype == MUON_BF16 ? 2 : 4; }
bool known_dtype(int dtype) { return dtype == MUON_BF16 || dtype == MUON_F32; }
size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

// A heads array of the given extents; strides of dimensions of size 1 become 0.
struct View {
  Heads h{};
  Strided s{};
  Extent e{};
};
muon_status_t make_view(const muon_heads_t& x, const char* name, int64_t batch, int64_t tokens, int64_t heads, int64_t dim,
                        int64_t es, int64_t align, bool written, View& v, Why& why) {
  const int64_t counts[3] = {heads, tokens, batch};
  int64_t st[3] = {x.head_stride, x.token_stride, x.batch_stride};
  const int64_t n = batch * tokens * heads;
  if (n > 0 && !x.data) return why.invalid("%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(x.data) % uintptr_t(align)) return why.invalid("%s is not %lld-byte aligned", name, (long long)align);
  uintptr_t span = uintptr_t(dim * es);
  for (int k = 0; k < 3; ++k) {
    if (counts[k] <= 1) { st[k] = 0; continue; }
    if (st[k] < 0 || st[k] > (int64_t(1) << 40)) return why.invalid("%s: stride out of range", name);
    if (st[k] * es % align) return why.invalid("%s: strides must be multiples of %lld bytes", name, (long long)align);
    st[k] *= es;
    if (st[k] > 0 && counts[k] - 1 > (int64_t(1) << 46) / st[k]) return why.invalid("%s: extent out of range", name);
    span += uintptr_t(st[k]) * uintptr_t(counts[k] - 1);
  }
  if (st[1] > kMaxTokenStride)
    return why.fail(MUON_ERR_UNSUPPORTED, "%s: a token stride of %lld bytes (at most %lld)", name, (long long)st[1],
                    (long long)kMaxTokenStride);
  if (written && n > 0) {  // elements must be distinct
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int p, int q) { return st[p] < st[q]; });
    int64_t inner = dim * es;
    for (int k : order) {
      if (counts[k] <= 1) continue;
      if (st[k] < inner) return why.invalid("%s: its elements overlap (an output must be a plain or strided tensor)", name);
      inner += st[k] * (counts[k] - 1);
    }
  }
  v.h = Heads{static_cast<char*>(x.data), st[2], st[1], st[0]};
  const uintptr_t lo = reinterpret_cast<uintptr_t>(x.data);
  if (n == 0) return MUON_OK;
  v.s = Strided{lo, dim * es, {st[0], st[1], st[2]}, {heads, tokens, batch}, written};
  v.e = Extent{lo, lo + span};
  return MUON_OK;
}

Strided flat(const void* p, int64_t bytes, bool written) {
  return Strided{reinterpret_cast<uintptr_t>(p), bytes, {0, 0, 0}, {1, 1, 1}, written};
}
Extent extent(const void* p, int64_t bytes) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return Extent{lo, lo + uintptr_t(bytes)};
}

// What the kernels multiply logits with, for exponentials of base 2.
float scale2_of(const muon_attention_t* a) { return float(double(a->scale) * 1.4426950408889634074); }

// Sizes alone.
muon_status_t check_sizes(const muon_attention_t* a, Why& why) {
  if (!a) return why.invalid("the request is NULL");
  if (!known_dtype(a->dtype)) return why.invalid("unknown dtype");
  if (a->q_heads < 1 || a->kv_heads < 1 || a->q_heads > 65536 || a->q_heads % a->kv_heads)
    return why.invalid("q_heads (%d) must be a positive multiple of kv_heads (%d)", a->q_heads, a->kv_heads);
  if (a->head_dim < 1) return why.invalid("head_dim must be >= 1");
  const int unit = int(16 / elem_size(a->dtype));
  if (a->head_dim > kMaxHeadDim || a->head_dim % unit)
    return why.fail(MUON_ERR_UNSUPPORTED, "head_dim %d: multiples of %d up to %d", a->head_dim, unit, kMaxHeadDim);
  if (a->batch < 0 || a->q_tokens < 0 || a->k_tokens < 0 || a->batch > kMaxTokens || a->q_tokens > kMaxTokens ||
      a->k_tokens > kMaxTokens)
    return why.invalid("batch or tokens out of range");
  if (a->causal != 0 && a->causal != 1) return why.invalid("causal must be 0 or 1");
  if ((a->fill_rest != 0 && a->fill_rest != 1) || (a->fill_rest && !a->q_offsets))
    return why.invalid("fill_rest must be 0 or 1, and needs offsets");
  if (a->reserved != 0) return why.invalid("reserved must be 0");
  if (!std::isfinite(a->scale) || !(a->scale > 0.f) || !std::isfinite(scale2_of(a)))
    return why.invalid("scale must be > 0, and scale * log2(e) finite");
  if (a->window < 0 || (a->window > 0 && !a->causal)) return why.invalid("window must be >= 0, and needs causal");
  if (!a->q_offsets != !a->k_offsets) return why.invalid("q_offsets and k_offsets go together");
  if (!a->q_lengths != !a->k_lengths) return why.invalid("q_lengths and k_lengths go together");
  if (a->q_offsets && a->q_lengths) return why.invalid("offsets and lengths exclude each other");
  if (a->q_offsets ? (a->batch != 1 || a->sequences < 0 || a->sequences > kMaxTokens) : a->sequences != 0)
    return why.invalid("packed requests have batch 1 and sequences >= 0, others sequences 0");
  // a launch has fewer than 2^24 workgroups of 256: tiles of 128 rows and one
  // more a sequence, and 8 or more rows a workgroup in the passes over rows
  const double rows = double(a->batch) * a->q_heads * double(std::max(a->q_tokens, a->k_tokens));
  const double tiles = rows / 128 + double(a->batch) * a->q_heads * double(a->sequences + 1);
  if (rows > double(1 << 25) || tiles > double(1 << 23))
    return why.fail(MUON_ERR_UNSUPPORTED, "too many rows in one call (heads x tokens: at most 2^25)");
  return MUON_OK;
}

muon::Seqs seqs_of(const muon_attention_t* a) {
  muon::Seqs s{};
  s.batch = a->batch;
  s.q_tokens = int32_t(a->q_tokens);
  s.k_tokens = int32_t(a->k_tokens);
  s.n_seq = int32_t(a->sequences);
  s.q_off = a->q_offsets; s.k_off = a->k_offsets;
  s.q_len = a->q_lengths; s.k_len = a->k_lengths;
  return s;
}
int32_t window_of(const muon_attention_t* a) {  // one beyond every gap is none
  return int32_t(std::min<int64_t>(a->window, int64_t(1) << 30));
}

struct ScratchPlan {
  int splits = 1, kv_parts = 1;
  size_t part_o = 0, part_ml = 0, lse2 = 0, delta = 0, norm = 0, dk = 0, dv = 0;
  size_t sq = 0, sk = 0, sv = 0, sdo = 0, bytes = 0;
};
ScratchPlan plan_scratch(const muon_attention_t* a, bool backward) {
  ScratchPlan p;
  const muon::Seqs s = seqs_of(a);
  const int64_t rows = a->batch * a->q_heads * a->q_tokens, keys = a->batch * a->kv_heads * a->k_tokens;
  const auto take = [&](size_t& at, size_t bytes) { at = p.bytes; p.bytes += up256(bytes); };
  if (rows == 0 && (!backward || keys == 0)) return p;
  if (!backward) {
    p.splits = muon::forward_splits(s, a->q_heads, a->kv_heads, a->head_dim, a->causal != 0, window_of(a));
    if (p.splits > 1) {
      take(p.part_o, size_t(rows) * size_t(p.splits) * size_t(a->head_dim) * 4);
      take(p.part_ml, size_t(rows) * size_t(p.splits) * 8);
    }
  } else {
    take(p.lse2, size_t(rows) * 4);
    take(p.delta, size_t(rows) * 4);
    if (a->dtype == MUON_F32) take(p.norm, size_t(rows) * 4);
    p.kv_parts = muon::backward_parts(s, a->q_heads, a->kv_heads, a->causal != 0, window_of(a));
    if (p.kv_parts > 1) {
      take(p.dk, size_t(keys) * size_t(p.kv_parts) * size_t(a->head_dim) * 4);
      take(p.dv, size_t(keys) * size_t(p.kv_parts) * size_t(a->head_dim) * 4);
    }
  }
  if (a->dtype == MUON_F32) {
    take(p.sk, muon::split_bytes(keys, a->head_dim));
    take(p.sv, muon::split_bytes(keys, a->head_dim));
    if (backward) {
      take(p.sq, muon::split_bytes(rows, a->head_dim));
      take(p.sdo, muon::split_bytes(rows, a->head_dim));
    }
  }
  return p;
}

// All checks that need no device; the kernels' arguments, and the buffers'
// extents for the runtime's answer about them.
constexpr int kMaxBuffers = 20;
struct Checked {
  muon::AttnArgs args{};
  Extent extents[kMaxBuffers];
  size_t n = 0;
};
muon_status_t check_attention(const muon_attention_t* a, const muon_attention_grad_t* g, Checked& c, Why& why) {
  muon_status_t st = check_sizes(a, why);
  if (st != MUON_OK) return st;
  Strided bufs[kMaxBuffers];
  size_t nb = 0;
  const int64_t es = elem_size(a->dtype);
  muon::AttnArgs& k = c.args;
  k.seqs = seqs_of(a);
  const auto add = [&](const Strided& s, const Extent& e) {
    if (e.hi <= e.lo) return;
    bufs[nb++] = s;
    c.extents[c.n++] = e;
  };
  const auto heads = [&](const muon_heads_t& x, const char* name, int64_t tokens, int64_t n, bool written, Heads& to) {
    View v;
    const muon_status_t r = make_view(x, name, a->batch, tokens, n, a->head_dim, es, 16, written, v, why);
    if (r != MUON_OK) return r;
    to = v.h;
    add(v.s, v.e);
    return MUON_OK;
  };
  if ((st = heads(a->q, "q", a->q_tokens, a->q_heads, false, k.q)) != MUON_OK) return st;
  if ((st = heads(a->k, "k", a->k_tokens, a->kv_heads, false, k.k)) != MUON_OK) return st;
  if ((st = heads(a->v, "v", a->k_tokens, a->kv_heads, false, k.v)) != MUON_OK) return st;
  if ((st = heads(a->out, "out", a->q_tokens, a->q_heads, !g, k.out)) != MUON_OK) return st;
  if (a->residual.data) {
    if (a->dtype != MUON_BF16) return why.invalid("residual: fp32 outputs have none");
    if ((st = heads(a->residual, "residual", a->q_tokens, a->q_heads, !g, k.res)) != MUON_OK) return st;
  }
  const int64_t rows = a->batch * a->q_heads * a->q_tokens;
  if (rows > 0 && !a->lse) return why.invalid("lse is NULL");
  if (reinterpret_cast<uintptr_t>(a->lse) % 4) return why.invalid("lse is not 4-byte aligned");
  if (rows > 0) add(flat(a->lse, rows * 4, !g), extent(a->lse, rows * 4));
  k.lse = a->lse;
  if (!g && a->max_logits) {
    if (reinterpret_cast<uintptr_t>(a->max_logits) % 4) return why.invalid("max_logits is not 4-byte aligned");
    add(flat(a->max_logits, a->q_heads * 4, true), extent(a->max_logits, a->q_heads * 4));
    k.max_logits = a->max_logits;
  }
  if (g) {
    if ((st = heads(g->dout, "dout", a->q_tokens, a->q_heads, false, k.dout)) != MUON_OK) return st;
    if ((st = heads(g->dq, "dq", a->q_tokens, a->q_heads, true, k.dq)) != MUON_OK) return st;
    if ((st = heads(g->dk, "dk", a->k_tokens, a->kv_heads, true, k.dk)) != MUON_OK) return st;
    if ((st = heads(g->dv, "dv", a->k_tokens, a->kv_heads, true, k.dv)) != MUON_OK) return st;
  }
  const int32_t* lists[4] = {a->q_offsets, a->k_offsets, a->q_lengths, a->k_lengths};
  for (int i = 0; i < 4; ++i) {
    if (!lists[i]) continue;
    if (reinterpret_cast<uintptr_t>(lists[i]) % 4) return why.invalid("offsets and lengths must be 4-byte aligned");
    const int64_t bytes = (i < 2 ? a->sequences + 1 : a->batch) * 4;
    if (bytes > 0) add(flat(lists[i], bytes, false), extent(lists[i], bytes));
  }
  const ScratchPlan p = plan_scratch(a, g != nullptr);
  if (p.bytes > 0) {
    if (!a->scratch || a->scratch_bytes < p.bytes)
      return why.invalid("scratch has %zu bytes, the call needs %zu", a->scratch ? a->scratch_bytes : size_t(0), p.bytes);
    if (reinterpret_cast<uintptr_t>(a->scratch) % 256) return why.invalid("scratch is not 256-byte aligned");
    add(flat(a->scratch, int64_t(p.bytes), true), extent(a->scratch, int64_t(p.bytes)));
  }
  if (!muon::buffers_disjoint(bufs, nb)) return why.invalid("an output or the scratch memory overlaps another buffer");
  k.q_heads = a->q_heads;
  k.kv_heads = a->kv_heads;
  k.group = a->q_heads / a->kv_heads;
  k.dim = a->head_dim;
  k.causal = a->causal;
  k.window = window_of(a);
  k.fill = a->fill_rest;
  k.scale = a->scale;
  k.scale2 = scale2_of(a);
  k.splits = p.splits;
  k.kv_parts = p.kv_parts;
  char* const s = static_cast<char*>(a->scratch);
  const auto part = [&](size_t at) { return reinterpret_cast<float*>(s + at); };
  if (p.splits > 1) {
    k.part_o = part(p.part_o);
    k.part_ml = reinterpret_cast<float2*>(s + p.part_ml);
  }
  if (g) {
    k.lse2 = part(p.lse2);
    k.delta = part(p.delta);
    if (a->dtype == MUON_F32) k.norm = part(p.norm);
    if (p.kv_parts > 1) { k.part_dk = part(p.dk); k.part_dv = part(p.dv); }
  }
  if (a->dtype == MUON_F32) {
    k.split_k = s + p.sk; k.split_v = s + p.sv;
    k.split_q = s + p.sq; k.split_do = s + p.sdo;
  }
  return MUON_OK;
}

void tell(const Why& why, char* msg, size_t len) {
  if (msg && len) snprintf(msg, len, "%s", why.text);
}

muon_status_t attend(muon_handle_t h, const muon_attention_t* a, const muon_attention_grad_t* g, void* stream) {
  muon::handle_clear_error(h);
  Why why;
  Checked c;
  const muon_status_t st = check_attention(a, g, c, why);
  if (st != MUON_OK) { muon::handle_error(h, "%s", why.text); return st; }
  if (!muon::extents_on_device(h, c.extents, c.n)) return MUON_ERR_INVALID_ARGUMENT;
  CurrentDevice dev(muon::handle_device(h));
  if (!dev.ok) { muon::handle_error(h, "cannot select device %d", muon::handle_device(h)); return MUON_ERR_DEVICE; }
  const int dt = a->dtype == MUON_BF16 ? muon::DT_BF16 : muon::DT_F32;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = g ? muon::run_attention_backward(c.args, dt, s, timer_on(h, s))
                         : muon::run_attention_forward(c.args, dt, s, timer_on(h, s));
  if (e == hipSuccess) return MUON_OK;
  muon::handle_error(h, "kernel launch: %s", hipGetErrorString(e));
  return MUON_ERR_DEVICE;
}

// No C++ exception crosses the interface: the only ones possible here are the
// standard library's on exhausted host memory.
template <typename F>
muon_status_t guarded(muon_handle_t h, F&& f) {
  try {
    return f();
  } catch (const std::exception&) {
    if (h) muon::handle_error(h, "out of host memory");
    return MUON_ERR_OUT_OF_MEMORY;
  }
}

constexpr size_t kRotaryBuffers = 2 * muon::kRotaryMax + 2;
muon_status_t check_rotary(const muon_rotary_t* r, const muon_rotary_tensor_t* t, muon::RotaryArgs& k, Extent* ext,
                           size_t& ne, Why& why) {
  Strided bufs[kRotaryBuffers];
  size_t nb = 0;
  if (!r || !t) return why.invalid("the request is NULL");
  if (!known_dtype(r->dtype)) return why.invalid("unknown dtype");
  if (r->n_tensors < 1 || r->n_tensors > muon::kRotaryMax) return why.invalid("1 to %d tensors a call", muon::kRotaryMax);
  if (r->head_dim < 1) return why.invalid("head_dim must be >= 1");
  if (r->head_dim > kMaxRotaryDim) return why.fail(MUON_ERR_UNSUPPORTED, "head_dim %d: at most %d", r->head_dim, kMaxRotaryDim);
  if (r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > r->head_dim)
    return why.invalid("rotary_dim must be even, 2 to head_dim");
  if (r->layout != 0 && r->layout != 1) return why.invalid("layout must be 0 (halves) or 1 (neighbours)");
  if (r->inverse != 0 && r->inverse != 1) return why.invalid("inverse must be 0 or 1");
  if (!std::isfinite(r->scale)) return why.invalid("scale must be finite");
  if (r->batch < 0 || r->tokens < 0 || r->batch > kMaxTokens || r->tokens > kMaxTokens)
    return why.invalid("batch or tokens out of range");
  if (double(r->batch) * double(r->tokens) >= double(1 << 24))  // a token a workgroup at the least
    return why.fail(MUON_ERR_UNSUPPORTED, "too many tokens in one call (at most 2^24)");
  const int64_t es = elem_size(r->dtype), all = r->batch * r->tokens;
  if (all == 0) return MUON_OK;
  if (!r->freqs) return why.invalid("freqs is NULL");
  if (reinterpret_cast<uintptr_t>(r->freqs) % 8) return why.invalid("freqs is not 8-byte aligned");
  bufs[nb++] = flat(r->freqs, r->rotary_dim * 4, false);
  ext[ne++] = extent(r->freqs, r->rotary_dim * 4);
  if (r->positions) {
    const int64_t ps = r->positions_int64 ? 8 : 4;
    if (reinterpret_cast<uintptr_t>(r->positions) % uintptr_t(ps)) return why.invalid("positions are not aligned to their size");
    const int64_t bs = r->batch > 1 ? r->position_batch_stride : 0, ts = r->tokens > 1 ? r->position_token_stride : 0;
    if (bs < 0 || ts < 0 || bs > (int64_t(1) << 40) || ts > (int64_t(1) << 24)) return why.invalid("positions: stride out of range");
    if (bs > 0 && r->batch > (int64_t(1) << 46) / bs) return why.invalid("positions: extent out of range");
    const int64_t span = ((r->batch - 1) * bs + (r->tokens - 1) * ts + 1) * ps;
    bufs[nb++] = flat(r->positions, span, false);
    ext[ne++] = extent(r->positions, span);
    k.pos_batch = bs;
    k.pos_token = ts;
  }
  const int half = r->rotary_dim / 2, unit = int(16 / es);
  for (int i = 0; i < r->n_tensors; ++i) {
    View x, y;
    if (t[i].heads < 0 || t[i].heads > 65536) return why.invalid("tensor %d: heads out of range", i);
    if (t[i].heads == 0) continue;
    const bool same = t[i].x.data == t[i].y.data;
    if (same && (t[i].x.batch_stride != t[i].y.batch_stride || t[i].x.token_stride != t[i].y.token_stride ||
                 t[i].x.head_stride != t[i].y.head_stride))
      return why.invalid("tensor %d: in place, x and y must have the same strides", i);
    muon_status_t st = make_view(t[i].x, "x", r->batch, r->tokens, t[i].heads, r->head_dim, es, es, same, x, why);
    if (st != MUON_OK) return st;
    if ((st = make_view(t[i].y, "y", r->batch, r->tokens, t[i].heads, r->head_dim, es, es, true, y, why)) != MUON_OK) return st;
    const auto by16 = [](const Heads& v) {
      return reinterpret_cast<uintptr_t>(v.p) % 16 == 0 && v.batch % 16 == 0 && v.token % 16 == 0 && v.head % 16 == 0;
    };
    k.t[i].x = x.h;
    k.t[i].y = y.h;
    k.t[i].heads = int32_t(t[i].heads);
    k.t[i].vec = by16(x.h) && by16(y.h) && r->head_dim % unit == 0 &&
                 (r->layout == 1 ? r->rotary_dim : half) % unit == 0;
    if (!same) { bufs[nb++] = x.s; ext[ne++] = x.e; }
    bufs[nb++] = y.s;
    ext[ne++] = y.e;
  }
  if (!muon::buffers_disjoint(bufs, nb)) return why.invalid("an output overlaps another buffer");
  k.n = r->n_tensors;
  k.batch = r->batch;
  k.tokens = r->tokens;
  k.positions = r->positions;
  k.positions64 = r->positions_int64 != 0;
  k.first = r->first_position;
  k.freqs = r->freqs;
  k.dim = r->head_dim;
  k.rot = r->rotary_dim;
  k.interleaved = r->layout;
  k.scale = r->scale;
  k.sign = r->inverse ? -1.f : 1.f;
  return MUON_OK;
}

muon_status_t rotary(muon_handle_t h, const muon_rotary_t* r, const muon_rotary_tensor_t* t, void* stream) {
  muon::handle_clear_error(h);
  Why why;
  muon::RotaryArgs k{};
  Extent ext[kRotaryBuffers];
  size_t ne = 0;
  const muon_status_t st = check_rotary(r, t, k, ext, ne, why);
  if (st != MUON_OK) { muon::handle_error(h, "%s", why.text); return st; }
  if (r->batch * r->tokens == 0) return MUON_OK;
  if (!muon::extents_on_device(h, ext, ne)) return MUON_ERR_INVALID_ARGUMENT;
  CurrentDevice dev(muon::handle_device(h));
  if (!dev.ok) { muon::handle_error(h, "cannot select device %d", muon::handle_device(h)); return MUON_ERR_DEVICE; }
  const hipError_t e = muon::run_rotary(k, r->dtype == MUON_BF16 ? muon::DT_BF16 : muon::DT_F32,
                                        static_cast<hipStream_t>(stream), timer_on(h, static_cast<hipStream_t>(stream)));
  if (e == hipSuccess) return MUON_OK;
  muon::handle_error(h, "kernel launch: %s", hipGetErrorString(e));
  return MUON_ERR_DEVICE;
}

muon_status_t check_clip(const muon_qk_clip_t* entries, int64_t n, std::vector<Extent>& ext, Why& why) {
  std::vector<Strided> bufs;
  if (n < 0) return why.invalid("n must be >= 0");
  if (n > 0 && !entries) return why.invalid("entries is NULL");
  for (int64_t i = 0; i < n; ++i) {
    const muon_qk_clip_t& e = entries[i];
    const long long at = (long long)i;
    if (!known_dtype(e.dtype)) return why.invalid("entry %lld: unknown dtype", at);
    if (e.reserved != 0) return why.invalid("entry %lld: reserved must be 0", at);
    if (e.q_heads < 1 || e.kv_heads < 1 || e.q_heads > 65536 || e.q_heads % e.kv_heads)
      return why.invalid("entry %lld: q_heads must be a positive multiple of kv_heads", at);
    if (e.head_dim < 1 || e.head_dim > 8192 || e.cols < 1 || e.cols > (int64_t(1) << 28))
      return why.invalid("entry %lld: head_dim or cols out of range", at);
    if ((int64_t(e.q_heads) + e.kv_heads) * e.head_dim > kMaxClipRows)
      return why.fail(MUON_ERR_UNSUPPORTED, "entry %lld: too many rows", at);
    if (!std::isfinite(e.threshold) || !(e.threshold > 0.f))
      return why.invalid("entry %lld: threshold must be finite and > 0", at);
    const int64_t es = elem_size(e.dtype), ql = e.q_ld ? e.q_ld : e.cols, kl = e.k_ld ? e.k_ld : e.cols;
    if (ql < e.cols || kl < e.cols || ql > (int64_t(1) << 32) || kl > (int64_t(1) << 32))
      return why.invalid("entry %lld: a row stride must be 0 or at least cols", at);
    if (!e.wq || !e.wk || !e.max_logits) return why.invalid("entry %lld: NULL pointer", at);
    const uintptr_t q = reinterpret_cast<uintptr_t>(e.wq), kp = reinterpret_cast<uintptr_t>(e.wk),
                    m = reinterpret_cast<uintptr_t>(e.max_logits);
    if (q % uintptr_t(es) || kp % uintptr_t(es) || m % 4)
      return why.invalid("entry %lld: pointer not aligned to its element size", at);
    const int64_t rq = int64_t(e.q_heads) * e.head_dim, rk = int64_t(e.kv_heads) * e.head_dim;
    bufs.push_back(Strided{q, e.cols * es, {ql * es, 0, 0}, {rq, 1, 1}, true});
    bufs.push_back(Strided{kp, e.cols * es, {kl * es, 0, 0}, {rk, 1, 1}, true});
    bufs.push_back(flat(e.max_logits, e.q_heads * 4, false));
    ext.push_back(extent(e.wq, ((rq - 1) * ql + e.cols) * es));
    ext.push_back(extent(e.wk, ((rk - 1) * kl + e.cols) * es));
    ext.push_back(extent(e.max_logits, e.q_heads * 4));
  }
  if (!muon::buffers_disjoint(bufs.data(), bufs.size())) return why.invalid("weights overlap another buffer");
  return MUON_OK;
}

muon_status_t qk_clip(muon_handle_t h, const muon_qk_clip_t* entries, int64_t n, int reset, void* stream) {
  muon::handle_clear_error(h);
  Why why;
  std::vector<Extent> ext;
  const muon_status_t st = reset != 0 && reset != 1 ? why.invalid("reset must be 0 or 1") : check_clip(entries, n, ext, why);
  if (st != MUON_OK) { muon::handle_error(h, "%s", why.text); return st; }
  if (n == 0) return MUON_OK;
  if (!muon::extents_on_device(h, ext.data(), ext.size())) return MUON_ERR_INVALID_ARGUMENT;
  CurrentDevice dev(muon::handle_device(h));
  if (!dev.ok) { muon::handle_error(h, "cannot select device %d", muon::handle_device(h)); return MUON_ERR_DEVICE; }
  const hipStream_t s = static_cast<hipStream_t>(stream);
  muon::LaunchTimer* const timer = timer_on(h, s);
  int64_t all = 0;
  for (int64_t i = 0; i < n; ++i) all += (int64_t(entries[i].q_heads) + entries[i].kv_heads) * entries[i].head_dim;
  const int32_t per = all / muon::kClipRows >= 1024 ? muon::kClipRows : muon::kClipRowsFew;
  // every clip is enqueued before any reset: entries may share logits
  for (int pass = 0; pass < (reset ? 2 : 1); ++pass)
    for (int dt : {MUON_BF16, MUON_F32})
      for (int64_t i = 0; i < n;) {
        muon::ClipArgs k{};
        k.rows = per;
        for (; i < n && k.n < muon::kClipMax; ++i) {
          const muon_qk_clip_t& e = entries[i];
          if (e.dtype != dt) continue;
          const int64_t es = elem_size(dt), ql = e.q_ld ? e.q_ld : e.cols, kl = e.k_ld ? e.k_ld : e.cols;
          muon::ClipEntry& c = k.e[k.n];
          c.wq = static_cast<char*>(e.wq);
          c.wk = static_cast<char*>(e.wk);
          c.ldq = ql * es;
          c.ldk = kl * es;
          c.logits = e.max_logits;
          c.q_heads = e.q_heads;
          c.kv_heads = e.kv_heads;
          c.dim = e.head_dim;
          c.cols = int32_t(e.cols);
          c.threshold = e.threshold;
          c.vec = reinterpret_cast<uintptr_t>(e.wq) % 16 == 0 && reinterpret_cast<uintptr_t>(e.wk) % 16 == 0 &&
                  c.ldq % 16 == 0 && c.ldk % 16 == 0;
          const int64_t rows = (int64_t(e.q_heads) + e.kv_heads) * e.head_dim;
          const int64_t blocks = (rows + per - 1) / per;
          if (k.first[k.n] + blocks > 2 * kMaxClipBlocks - 1) break;  // the next launch takes it
          k.first[k.n + 1] = int32_t(k.first[k.n] + blocks);
          ++k.n;
        }
        const hipError_t e = pass ? muon::run_reset_logits(k, s)
                                  : muon::run_qk_clip(k, dt == MUON_BF16 ? muon::DT_BF16 : muon::DT_F32, s, timer);
        if (e != hipSuccess) {
          muon::handle_error(h, "kernel launch: %s", hipGetErrorString(e));
          return MUON_ERR_DEVICE;
        }
      }
  return MUON_OK;
}

}  // namespace

extern "C" {

muon_status_t muon_attention_scratch(const muon_attention_t* a, int backward, size_t* bytes) {
  if (!bytes) return MUON_ERR_INVALID_ARGUMENT;
  *bytes = 0;
  Why why;
  const muon_status_t st = check_sizes(a, why);
  if (st != MUON_OK) return st;
  *bytes = plan_scratch(a, backward != 0).bytes;
  return MUON_OK;
}

muon_status_t muon_validate_attention(const muon_attention_t* a, const muon_attention_grad_t* g, char* msg, size_t msg_len) {
  if (msg && msg_len) msg[0] = '\0';
  return guarded(nullptr, [&] {
    Why why;
    Checked c;
    const muon_status_t st = check_attention(a, g, c, why);
    tell(why, msg, msg_len);
    return st;
  });
}

muon_status_t muon_validate_rotary(const muon_rotary_t* r, const muon_rotary_tensor_t* tensors, char* msg, size_t msg_len) {
  if (msg && msg_len) msg[0] = '\0';
  return guarded(nullptr, [&] {
    Why why;
    muon::RotaryArgs k{};
    Extent ext[kRotaryBuffers];
    size_t ne = 0;
    const muon_status_t st = check_rotary(r, tensors, k, ext, ne, why);
    tell(why, msg, msg_len);
    return st;
  });
}

muon_status_t muon_validate_qk_clip(const muon_qk_clip_t* entries, int64_t n, char* msg, size_t msg_len) {
  if (msg && msg_len) msg[0] = '\0';
  return guarded(nullptr, [&] {
    Why why;
    std::vector<Extent> ext;
    const muon_status_t st = check_clip(entries, n, ext, why);
    tell(why, msg, msg_len);
    return st;
  });
}

muon_status_t muon_attention_forward(muon_handle_t h, const muon_attention_t* a, void* stream) {
  if (!h) return MUON_ERR_INVALID_ARGUMENT;
  return guarded(h, [&] { return attend(h, a, nullptr, stream); });
}

muon_status_t muon_attention_backward(muon_handle_t h, const muon_attention_t* a, const muon_attention_grad_t* g,
                                      void* stream) {
  if (!h) return MUON_ERR_INVALID_ARGUMENT;
  return guarded(h, [&] {
    if (!g) {
      muon::handle_clear_error(h);
      muon::handle_error(h, "the gradients are NULL");
      return MUON_ERR_INVALID_ARGUMENT;
    }
    return attend(h, a, g, stream);
  });
}

muon_status_t muon_rotary(muon_handle_t h, const muon_rotary_t* r, const muon_rotary_tensor_t* tensors, void* stream) {
  if (!h) return MUON_ERR_INVALID_ARGUMENT;
  return guarded(h, [&] { return rotary(h, r, tensors, stream); });
}

muon_status_t muon_qk_clip(muon_handle_t h, const muon_qk_clip_t* entries, int64_t n, int reset, void* stream) {
  if (!h) return MUON_ERR_INVALID_ARGUMENT;
  return guarded(h, [&] { return qk_clip(h, entries, n, reset, stream); });
}

}  // extern "C"
