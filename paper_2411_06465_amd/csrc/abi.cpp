// C ABI of the layer-shard library: argument validation, the exact memory
// estimate, the arena / activation-stash allocator, kernel timing, and the
// orchestration of the forward, backward and LM-head kernel sequences.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <map>
#include <mutex>
#include <set>
#include <string>
#include <vector>

#include "../../include/l4d.h"
#include "kernels.h"

using namespace l4d;

// ============================================================== errors

static thread_local std::string g_err;

static int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_err = buf;
  return code;
}

extern "C" const char* l4d_last_error(void) { return g_err.c_str(); }

#define HIP_TRY(expr)                                                                   \
  do {                                                                                  \
    hipError_t e_ = (expr);                                                             \
    if (e_ != hipSuccess) return fail(L4D_EDEVICE, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

// ============================================================== kernel timing

namespace {
struct Pending {
  const char* name;
  hipEvent_t a, b;
};
std::mutex g_prof_mu;
bool g_prof_on = false;
std::string g_prof_only;            // non-empty: time only the launches with this label
std::vector<Pending> g_pending;
std::vector<hipEvent_t> g_event_pool;
std::map<std::string, std::pair<int64_t, double>> g_totals;
std::vector<const char*> g_order;  // labels of the timed launches since the last reset, in launch order

hipEvent_t take_event() {
  if (!g_event_pool.empty()) {
    hipEvent_t e = g_event_pool.back();
    g_event_pool.pop_back();
    return e;
  }
  hipEvent_t e = nullptr;
  if (hipEventCreate(&e) != hipSuccess) return nullptr;
  return e;
}

int drain_pending() {
  for (auto& p : g_pending) {
    float ms = 0.f;
    hipError_t e = hipEventSynchronize(p.b);
    if (e == hipSuccess) e = hipEventElapsedTime(&ms, p.a, p.b);
    if (e != hipSuccess) return fail(L4D_EDEVICE, "profile events: %s", hipGetErrorString(e));
    auto& t = g_totals[p.name];
    g_order.push_back(p.name);
    t.first += 1;
    t.second += ms;
    g_event_pool.push_back(p.a);
    g_event_pool.push_back(p.b);
  }
  g_pending.clear();
  return L4D_OK;
}

// Launch `fn` (returning hipError_t) bracketed by events when timing is on.
template <class F>
int launch(const char* name, hipStream_t s, F&& fn) {
  hipEvent_t a = nullptr, b = nullptr;
  if (g_prof_on && (g_prof_only.empty() || g_prof_only == name)) {
    std::lock_guard<std::mutex> lk(g_prof_mu);
    a = take_event();
    b = take_event();
    if (a) (void)hipEventRecord(a, s);
  }
  hipError_t e = fn();
  if (e != hipSuccess) return fail(L4D_EDEVICE, "launch of %s failed: %s", name, hipGetErrorString(e));
  if (a && b) {
    (void)hipEventRecord(b, s);
    std::lock_guard<std::mutex> lk(g_prof_mu);
    g_pending.push_back({name, a, b});
  }
  return L4D_OK;
}
}  // namespace

extern "C" int l4d_profile_enable(int on) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  g_prof_on = on != 0;
  return L4D_OK;
}

extern "C" int l4d_profile_only(const char* name) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  g_prof_only = name ? name : "";
  return L4D_OK;
}

extern "C" int l4d_profile_reset(void) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  int rc = drain_pending();
  g_totals.clear();
  g_order.clear();
  return rc;
}

extern "C" int l4d_profile_read(const char* name, int64_t* launches, double* total_ms) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  int rc = drain_pending();
  if (rc) return rc;
  int64_t n = 0;
  double ms = 0;
  for (auto& kv : g_totals)
    if (!name || kv.first == name) {
      n += kv.second.first;
      ms += kv.second.second;
    }
  if (launches) *launches = n;
  if (total_ms) *total_ms = ms;
  return L4D_OK;
}

extern "C" int l4d_profile_dump(char* buf, uint64_t buf_len, uint64_t* needed) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  int rc = drain_pending();
  if (rc) return rc;
  std::string out;
  char line[256];
  for (auto& kv : g_totals) {
    snprintf(line, sizeof line, "%s %lld %.6f\n", kv.first.c_str(), (long long)kv.second.first, kv.second.second);
    out += line;
  }
  if (needed) *needed = out.size() + 1;
  if (buf && buf_len) {
    size_t n = std::min<size_t>(out.size(), buf_len - 1);
    memcpy(buf, out.data(), n);
    buf[n] = 0;
  }
  return L4D_OK;
}

extern "C" int l4d_profile_order(char* buf, uint64_t buf_len, uint64_t* needed) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  int rc = drain_pending();
  if (rc) return rc;
  std::string out;
  for (const char* n : g_order) {
    out += n;
    out += '\n';
  }
  if (needed) *needed = out.size() + 1;
  if (buf && buf_len) {
    size_t n = std::min<size_t>(out.size(), buf_len - 1);
    memcpy(buf, out.data(), n);
    buf[n] = 0;
  }
  return L4D_OK;
}

// ============================================================== memory estimate

namespace {
typedef __int128 i128;

struct Rat {  // num / den, den > 0
  i128 num, den;
};

uint64_t ceil_u64(Rat r, bool& inexact) {
  i128 q = r.num / r.den, rem = r.num % r.den;
  if (rem != 0) {
    inexact = true;
    q += 1;
  }
  return (uint64_t)q;
}

int check_model(const l4d_model* m, const l4d_parallel* p) {
  if (!m || !p) return fail(L4D_EINVAL, "model and parallel layout are required");
  if (m->hidden <= 0 || m->n_heads <= 0 || m->n_kv_heads <= 0 || m->ffn <= 0 || m->n_layers <= 0 ||
      m->vocab <= 0)
    return fail(L4D_EINVAL, "model sizes must be positive");
  if (p->seq <= 0 || p->micro_batch <= 0 || p->tp <= 0 || p->cp <= 0 || p->pp <= 0 || p->dp <= 0)
    return fail(L4D_EINVAL, "sequence, micro-batch and parallel sizes must be positive");
  if (m->hidden % m->n_heads) return fail(L4D_EINVAL, "hidden %% n_heads != 0");
  if (m->n_heads % m->n_kv_heads) return fail(L4D_EINVAL, "n_heads %% n_kv_heads != 0");
  if (m->n_heads % p->tp || m->n_kv_heads % p->tp) return fail(L4D_EINVAL, "heads not divisible by tp");
  if (m->ffn % p->tp) return fail(L4D_EINVAL, "ffn %% tp != 0");
  if (m->vocab % p->tp) return fail(L4D_EINVAL, "vocab %% tp != 0");
  if (p->seq % p->cp) return fail(L4D_EINVAL, "seq %% cp != 0");
  if (m->n_layers % p->pp) return fail(L4D_EINVAL, "n_layers %% pp != 0");
  if (p->tp_rank < 0 || p->tp_rank >= p->tp || p->cp_rank < 0 || p->cp_rank >= p->cp)
    return fail(L4D_EINVAL, "rank out of range");
  return L4D_OK;
}
}  // namespace

extern "C" int mem_estimate(const l4d_model* m, const l4d_parallel* p, l4d_mem* out) {
  int rc = check_model(m, p);
  if (rc) return rc;
  if (!out) return fail(L4D_EINVAL, "out is NULL");
  const i128 h = m->hidden, a = m->n_heads, k = m->n_kv_heads, f = m->ffn, L = m->n_layers, v = m->vocab;
  const i128 s = p->seq, b = p->micro_batch, t = p->tp, c = p->cp, pp = p->pp, d = p->dp;
  // ell * (a t) = 2h^2(a+k) + 3 h f a + 2 h a t   (Eqs. 1, 2 divided by t, plus the two norms)
  const i128 E = 2 * h * h * (a + k) + 3 * h * f * a + 2 * h * a * t;
  Rat psi;
  if (p->pp == 1) psi = {2 * h * v * a + h * a * t + L * E, a * t};   // embedding + head + final norm
  else psi = {h * v * a * pp + L * E, a * t * pp};                   // first stage (Eq. 7)
  bool inexact = false;
  out->params_per_gpu = ceil_u64(psi, inexact);
  out->weight_bytes = ceil_u64({2 * psi.num, psi.den}, inexact);
  out->grad_bytes = ceil_u64({4 * psi.num, psi.den}, inexact);
  out->optim_bytes = ceil_u64({12 * psi.num, psi.den * d * c}, inexact);
  // per layer: s b (12 a h + 4 k h + 8 f a) / (t c a)     (Eq. 12 / (tc))
  const i128 lay = 12 * a * h + 4 * k * h + 8 * f * a;
  out->act_bytes_per_layer = ceil_u64({s * b * lay, t * c * a}, inexact);
  // Eq. 17: s b [L lay + 8 p a h + [p=1] 4 a (h + v)] / (t c a)
  i128 act = L * lay + 8 * pp * a * h;
  if (p->pp == 1) act += 4 * a * (h + v);
  out->act_bytes = ceil_u64({s * b * act, t * c * a}, inexact);
  out->total_bytes = out->weight_bytes + out->grad_bytes + out->optim_bytes + out->act_bytes;
  out->inexact = inexact ? 1u : 0u;
  return L4D_OK;
}

extern "C" int mem_fit(const l4d_mem* est, uint64_t device_bytes, int* fit) {
  if (!est || !fit || device_bytes == 0) return fail(L4D_EINVAL, "est, fit and device_bytes are required");
  // total <= 0.8 M  <=>  5 total <= 4 M, in 128-bit integers
  const unsigned __int128 t5 = (unsigned __int128)est->total_bytes * 5, m4 = (unsigned __int128)device_bytes * 4;
  *fit = t5 <= m4 ? L4D_FITS : (est->total_bytes <= device_bytes ? L4D_NEAR_LIMIT : L4D_OOM);
  return L4D_OK;
}

// ============================================================== arena

struct l4d_arena {
  uintptr_t base;
  uint64_t cap;
  std::map<uint64_t, uint64_t> free_;  // offset -> size
  uint64_t in_use = 0, peak = 0;
  std::set<const l4d_stash*> live;
};

namespace {
constexpr uint64_t kAlign = 256;
uint64_t align_up(uint64_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

bool arena_alloc(l4d_arena* A, uint64_t size, uint64_t* off) {
  size = align_up(std::max<uint64_t>(size, 1));
  for (auto it = A->free_.begin(); it != A->free_.end(); ++it) {
    if (it->second >= size) {
      *off = it->first;
      uint64_t rest = it->second - size, roff = it->first + size;
      A->free_.erase(it);
      if (rest) A->free_[roff] = rest;
      A->in_use += size;
      A->peak = std::max(A->peak, A->in_use);
      return true;
    }
  }
  return false;
}

void arena_free(l4d_arena* A, uint64_t off, uint64_t size) {
  size = align_up(std::max<uint64_t>(size, 1));
  A->in_use -= size;
  auto it = A->free_.emplace(off, size).first;
  auto nx = std::next(it);
  if (nx != A->free_.end() && it->first + it->second == nx->first) {
    it->second += nx->second;
    A->free_.erase(nx);
  }
  if (it != A->free_.begin()) {
    auto pv = std::prev(it);
    if (pv->first + pv->second == it->first) {
      pv->second += it->second;
      A->free_.erase(it);
    }
  }
}

// A transient workspace: a list of sub-buffers carved from one arena block.
struct Workspace {
  l4d_arena* A = nullptr;
  uint64_t off = 0, size = 0;
  bool held = false;
  ~Workspace() {
    if (held) arena_free(A, off, size);
  }
};

struct Carver {  // bump-allocates aligned pieces of a byte range
  uint64_t used = 0;
  uint64_t take(uint64_t bytes) {
    uint64_t o = used;
    used += align_up(bytes);
    return o;
  }
};
}  // namespace

extern "C" int l4d_arena_create(void* dev_base, uint64_t capacity, l4d_arena** out) {
  if (!out) return fail(L4D_EINVAL, "out is NULL");
  if (!dev_base && capacity) return fail(L4D_EINVAL, "dev_base is NULL");
  if (reinterpret_cast<uintptr_t>(dev_base) % kAlign) return fail(L4D_EINVAL, "dev_base must be 256-byte aligned");
  auto* A = new l4d_arena();
  A->base = reinterpret_cast<uintptr_t>(dev_base);
  A->cap = capacity / kAlign * kAlign;
  if (A->cap) A->free_[0] = A->cap;
  *out = A;
  return L4D_OK;
}

extern "C" int l4d_arena_destroy(l4d_arena* A) {
  if (!A) return L4D_OK;
  if (!A->live.empty()) return fail(L4D_EINVAL, "arena still holds %zu live stash(es)", A->live.size());
  delete A;
  return L4D_OK;
}

extern "C" int l4d_arena_stats(const l4d_arena* A, uint64_t* in_use, uint64_t* peak, uint64_t* capacity) {
  if (!A) return fail(L4D_EINVAL, "arena is NULL");
  if (in_use) *in_use = A->in_use;
  if (peak) *peak = A->peak;
  if (capacity) *capacity = A->cap;
  return L4D_OK;
}

// ============================================================== shard geometry

namespace {
struct Shard {
  int64_t h, a, k, f, s, b, t, c, tr, cr;
  int64_t d, a_t, k_t, f_t, s_c, s_sp;
  float eps, base;
  ChunkMap qmap;
  int n_remote_runs;
  int64_t rem_chunk_start[4], rem_chunk_count[4];  // runs of consecutive remote chunks (chunk ids)
  int64_t chunk_len;
};

int make_shard(const l4d_model* m, const l4d_parallel* p, Shard* S) {
  int rc = check_model(m, p);
  if (rc) return rc;
  Shard& x = *S;
  x.h = m->hidden; x.a = m->n_heads; x.k = m->n_kv_heads; x.f = m->ffn;
  x.s = p->seq; x.b = p->micro_batch; x.t = p->tp; x.c = p->cp; x.tr = p->tp_rank; x.cr = p->cp_rank;
  x.eps = m->rms_eps; x.base = m->rope_base;
  x.d = x.h / x.a; x.a_t = x.a / x.t; x.k_t = x.k / x.t; x.f_t = x.f / x.t;
  x.s_c = x.s / x.c;
  if (x.s_c % x.t) return fail(L4D_EINVAL, "local sequence %lld not divisible by tp", (long long)x.s_c);
  x.s_sp = x.s_c / x.t;
  if (x.d != 64 && x.d != 128) return fail(L4D_EINVAL, "head dim %lld unsupported (64 or 128)", (long long)x.d);
  if (x.h % 8 || x.f_t % 8) return fail(L4D_EINVAL, "hidden and ffn/tp must be multiples of 8");
  if (x.h > 8192) return fail(L4D_EINVAL, "hidden > 8192 unsupported");
  if (x.c > 1 && x.s % (2 * x.c)) return fail(L4D_EINVAL, "seq %% (2 cp) != 0");
  if (x.b * x.s_c > (int64_t)1 << 30 || x.h * x.s > (int64_t)1 << 40)
    return fail(L4D_EINVAL, "problem too large");
  // CP layout: 2c chunks, rank r owns r and 2c-1-r (Sec. 2.1 / 3.2.3 load-balanced reading)
  if (x.c == 1) {
    x.chunk_len = x.s;
    x.qmap = ChunkMap{1, (int32_t)x.s, {0, 0}};
    x.n_remote_runs = 0;
  } else {
    x.chunk_len = x.s / (2 * x.c);
    x.qmap = ChunkMap{2, (int32_t)x.chunk_len, {(int32_t)x.cr, (int32_t)(2 * x.c - 1 - x.cr)}};
    x.n_remote_runs = 0;
    int64_t i = 0;
    while (i < 2 * x.c) {
      if (i == x.cr || i == 2 * x.c - 1 - x.cr) { ++i; continue; }
      int64_t j = i;
      while (j + 1 < 2 * x.c && j + 1 != x.cr && j + 1 != 2 * x.c - 1 - x.cr) ++j;
      x.rem_chunk_start[x.n_remote_runs] = i;
      x.rem_chunk_count[x.n_remote_runs] = j - i + 1;
      ++x.n_remote_runs;
      i = j + 1;
    }
  }
  return L4D_OK;
}

int64_t qkv_cols(const Shard& x) { return (x.a_t + 2 * x.k_t) * x.d; }
}  // namespace

// ============================================================== stash

enum StashKind { kLayerStash = 0, kHeadStash = 1, kEmbStash = 2 };

struct l4d_stash {
  l4d_arena* arena;
  uint64_t block_off, block_size;
  uint64_t off[L4D_STASH_COUNT], bytes[L4D_STASH_COUNT];
  uint64_t formula, aux, padding;
  Shard shape;
  int kind = kLayerStash;
  int count = L4D_STASH_COUNT;
  bool packed = false;       // a layer call over packed documents
};

namespace {
void stash_sizes(const Shard& x, uint64_t* bytes) {
  const uint64_t sp = x.b * x.s_sp * x.h * 2, tok = x.b * x.s_c;
  bytes[L4D_STASH_X] = bytes[L4D_STASH_XN1] = bytes[L4D_STASH_H1] = bytes[L4D_STASH_XN2] = sp;
  bytes[L4D_STASH_Q] = bytes[L4D_STASH_CTX] = tok * x.a_t * x.d * 2;
  bytes[L4D_STASH_K] = bytes[L4D_STASH_V] = tok * x.k_t * x.d * 2;
  bytes[L4D_STASH_GATE] = bytes[L4D_STASH_UP] = bytes[L4D_STASH_ACT] = bytes[L4D_STASH_PROD] = tok * x.f_t * 2;
  bytes[L4D_STASH_LSE] = x.b * x.a_t * x.s_c * 4;
}

// One arena block holding `count` tensors of the given sizes, 256-byte aligned;
// the tensor `aux_slot` (or none, -1) is reported as aux, the rest as formula.
int stash_reserve_sized(l4d_arena* A, const Shard& x, int kind, int count, const uint64_t* bytes, int aux_slot,
                        l4d_stash** out) {
  auto* st = new l4d_stash();
  st->arena = A;
  st->shape = x;
  st->kind = kind;
  st->count = count;
  uint64_t total = 0, raw = 0;
  for (int i = 0; i < count; ++i) {
    st->bytes[i] = bytes[i];
    st->off[i] = total;
    total += align_up(st->bytes[i]);
    if (i != aux_slot) raw += st->bytes[i];
  }
  st->formula = raw;
  st->aux = aux_slot >= 0 ? st->bytes[aux_slot] : 0;
  st->padding = total - raw - st->aux;
  if (!arena_alloc(A, total, &st->block_off)) {
    delete st;
    return fail(L4D_ENOMEM, "stash needs %llu bytes; arena has %llu of %llu in use", (unsigned long long)total,
                (unsigned long long)A->in_use, (unsigned long long)A->cap);
  }
  st->block_size = total;
  A->live.insert(st);
  *out = st;
  return L4D_OK;
}

int stash_reserve(l4d_arena* A, const Shard& x, l4d_stash** out) {
  uint64_t bytes[L4D_STASH_COUNT];
  stash_sizes(x, bytes);
  return stash_reserve_sized(A, x, kLayerStash, L4D_STASH_COUNT, bytes, L4D_STASH_LSE, out);
}

template <class T = uint16_t>
T* sptr(const l4d_stash* st, int which) {
  return reinterpret_cast<T*>(st->arena->base + st->block_off + st->off[which]);
}
}  // namespace

extern "C" int l4d_stash_reserve(l4d_arena* A, const l4d_model* m, const l4d_parallel* p, l4d_stash** out) {
  if (!A || !out) return fail(L4D_EINVAL, "arena and out are required");
  Shard x;
  int rc = make_shard(m, p, &x);
  if (rc) return rc;
  return stash_reserve(A, x, out);
}

extern "C" int l4d_stash_bytes(const l4d_stash* st, uint64_t* formula, uint64_t* aux, uint64_t* padding) {
  if (!st) return fail(L4D_EINVAL, "stash is NULL");
  if (formula) *formula = st->formula;
  if (aux) *aux = st->aux;
  if (padding) *padding = st->padding;
  return L4D_OK;
}

extern "C" int l4d_stash_tensor(const l4d_stash* st, int which, void** ptr, uint64_t* bytes) {
  if (!st) return fail(L4D_EINVAL, "stash is NULL");
  if (which < 0 || which >= st->count) return fail(L4D_EINVAL, "no stash tensor %d", which);
  if (ptr) *ptr = sptr<void>(st, which);
  if (bytes) *bytes = st->bytes[which];
  return L4D_OK;
}

extern "C" int l4d_stash_release(l4d_arena* A, l4d_stash* st) {
  if (!A || !st) return fail(L4D_EINVAL, "arena and stash are required");
  if (st->arena != A || !A->live.count(st)) return fail(L4D_EINVAL, "stash does not belong to this arena");
  arena_free(A, st->block_off, st->block_size);
  A->live.erase(st);
  delete st;
  return L4D_OK;
}

// ============================================================== workspace plans

namespace {
struct FwdWs {
  uint64_t rope, o_send, ffn_send, total;
};
struct BwdWs {
  uint64_t rope, dgu, dxn2, dh1, dh1_f32, dctx, delta, dqkv, dxn1, partial, dxn2_send, dxn1_send, dkv, ffn_part, proj_part,
      total;
};

// fp32 partials of a GEMM cut into `splits` parts.
uint64_t partial_bytes(int64_t M, int64_t N, int splits, bool acc_f32) {
  return splits <= 1 ? 0 : (uint64_t)(acc_f32 ? splits - 1 : splits) * M * N * 4;
}

uint64_t split_ws_bytes(int64_t M, int64_t N, int64_t K, bool acc_f32 = true) {
  const EpiKind kind = acc_f32 ? EpiKind::AccF32 : EpiKind::StoreBF16;
  return partial_bytes(M, N, gemm_plan(M, N, K, kind, gemm_max_splits(M, N, K, acc_f32), true).splits, acc_f32);
}

FwdWs plan_fwd(const Shard& x, const l4d_peer_outputs* sends) {
  Carver cv;
  FwdWs w;
  const uint64_t peer_rows = x.b * (x.t - 1) * x.s_sp * x.h * 2;
  w.rope = cv.take(x.s_c * (x.d / 2) * 8);
  w.o_send = (x.t > 1 && !(sends && sends->o_partial)) ? cv.take(peer_rows) : 0;
  w.ffn_send = (x.t > 1 && !(sends && sends->ffn_partial)) ? cv.take(peer_rows) : 0;
  w.total = cv.used;
  return w;
}

BwdWs plan_bwd(const Shard& x, const l4d_peer_outputs* sends) {
  Carver cv;
  BwdWs w;
  const uint64_t tok = x.b * x.s_c, sp = x.b * x.s_sp * x.h * 2;
  const uint64_t peer_rows = x.b * (x.t - 1) * x.s_sp * x.h * 2;
  w.rope = cv.take(x.s_c * (x.d / 2) * 8);
  w.dgu = cv.take(tok * 2 * x.f_t * 2);
  w.dxn2 = cv.take(2 * sp);       // fp32: only the norm backward reads it
  w.dh1 = cv.take(sp);            // bf16: operand of the output-projection products
  w.dh1_f32 = cv.take(2 * sp);    // fp32: the residual the norm-1 backward adds
  w.dctx = cv.take(tok * x.a_t * x.d * 2);
  w.delta = cv.take(x.b * x.a_t * x.s_c * 4);
  w.dqkv = cv.take(tok * qkv_cols(x) * 2);
  w.dxn1 = cv.take(2 * sp);       // fp32
  w.partial = cv.take((uint64_t)rmsnorm_bwd_partials(x.b * x.s_sp) * x.h * 4);
  const uint64_t partial_end = cv.used;
  w.dxn2_send = (x.t > 1 && !(sends && sends->dxn2_partial)) ? cv.take(peer_rows) : 0;
  w.dxn1_send = (x.t > 1 && !(sends && sends->dxn1_partial)) ? cv.take(peer_rows) : 0;
  // fp32 dK/dV partials when the query heads of a kv-head are split (at most a/k slices)
  const int64_t group = x.a / x.k;
  w.dkv = group > 1 ? cv.take(2 * (uint64_t)group * x.b * x.s * x.k_t * x.d * 4) : 0;
  // fp32 partials of the GEMMs that split their K range lie where nothing lives at
  // that time: those of the FFN's weight gradients from dh1 to the norm partials, which
  // are written after them, those of the two projections in dgu and dxn2, which are
  // read before them.  Only what does not fit there takes room of its own.
  const int64_t tk = (int64_t)tok;
  const uint64_t ffn = std::max(split_ws_bytes(x.h, x.f_t, tk), split_ws_bytes(2 * x.f_t, x.h, tk));
  const uint64_t proj = std::max({split_ws_bytes(x.h, x.a_t * x.d, tk), split_ws_bytes(qkv_cols(x), x.h, tk),
                                  split_ws_bytes(tk, x.a_t * x.d, x.h, false)});   // and the O dX GEMM
  const bool ffn_in = ffn <= partial_end - w.dh1, proj_in = proj <= w.dh1 - w.dgu;
  const uint64_t own = std::max(ffn_in ? 0 : ffn, proj_in ? 0 : proj);
  const uint64_t own_off = own ? cv.take(own) : 0;
  w.ffn_part = ffn_in ? w.dh1 : own_off;
  w.proj_part = proj_in ? w.dgu : own_off;
  w.total = cv.used;
  return w;
}

int take_ws(l4d_arena* A, uint64_t bytes, Workspace& ws) {
  ws.A = A;
  ws.size = bytes;
  if (!arena_alloc(A, bytes, &ws.off))
    return fail(L4D_ENOMEM, "workspace needs %llu bytes; arena has %llu of %llu in use", (unsigned long long)bytes,
                (unsigned long long)A->in_use, (unsigned long long)A->cap);
  ws.held = true;
  return L4D_OK;
}
}  // namespace

extern "C" int l4d_layer_workspace_bytes(const l4d_model* m, const l4d_parallel* p, uint64_t* fwd, uint64_t* bwd) {
  Shard x;
  int rc = make_shard(m, p, &x);
  if (rc) return rc;
  if (fwd) *fwd = align_up(plan_fwd(x, nullptr).total);
  if (bwd) *bwd = align_up(plan_bwd(x, nullptr).total);
  return L4D_OK;
}

namespace {
constexpr uint64_t kScratchBytes = 64ull << 20;   // lm_head_xent_noalloc's static workspace

// Workspace of lm_head_xent: the bf16 logits, and where few token rows give few
// tiles the fp32 partials of d_hidden, whose K range (the vocabulary shard) is cut
// into `splits` parts (`full` bytes; the logits alone run it unsplit).  The split
// depends on the sizes alone -- where the logits fit the static workspace, on
// what is left of it -- so that both entry points sum in the same order.
struct LmWs {
  uint64_t logits, full;
  int splits;
};
LmWs plan_lm(int64_t n, int64_t h, int64_t v_t) {
  constexpr uint64_t kMaxSplits = 8;
  LmWs w;
  const uint64_t part = std::max<uint64_t>((uint64_t)n * h * 4, 1);
  w.logits = align_up((uint64_t)n * v_t * 2);
  const uint64_t cap = w.logits <= kScratchBytes ? std::min(kMaxSplits, (kScratchBytes - w.logits) / part) : kMaxSplits;
  w.splits = n > 0 ? gemm_plan(n, h, v_t, EpiKind::StoreBF16, (int)std::max<uint64_t>(cap, 1)).splits : 1;
  w.full = align_up(w.logits + partial_bytes(n, h, w.splits, false));
  return w;
}
}  // namespace

extern "C" int l4d_lm_head_workspace_bytes(int64_t n, int64_t h, int64_t v_t, uint64_t* bytes) {
  if (n < 0 || h <= 0 || v_t <= 0) return fail(L4D_EINVAL, "bad LM-head sizes");
  // a long ragged shard is still quoted with n x h floats, as when d_hidden was summed there
  const LmWs w = plan_lm(n, h, v_t);
  const uint64_t quoted = w.logits + (v_t % 128 != 0 && v_t >= 1024 ? align_up((uint64_t)n * h * 4) : 0);
  if (bytes) *bytes = std::max(w.full, quoted);
  return L4D_OK;
}

// ============================================================== layer helpers

namespace {
inline RowSrc gathered(const void* own, const void* peer, const Shard& x) {
  if (x.t == 1) return RowSrc::plain(own, x.h);
  return RowSrc{static_cast<const uint16_t*>(own), static_cast<const uint16_t*>(peer), x.h, (int32_t)x.s_c,
                (int32_t)x.s_sp, (int32_t)x.tr, (int32_t)x.t};
}

inline Operand op(RowSrc src, int64_t rows) { return Operand{src, (int32_t)rows, 0, 0}; }

inline EpiParams epi_residual(const Shard& x, uint16_t* own_out, const void* resid, const void* receipt,
                              void* send, float* own_out_f32 = nullptr) {
  EpiParams e{};
  e.kind = EpiKind::ResidualSP;
  e.ldc = x.h;
  e.own_out = own_out;
  e.own_out_f32 = own_out_f32;
  e.resid = static_cast<const uint16_t*>(resid);
  e.receipt = static_cast<const uint16_t*>(receipt);
  e.send = static_cast<uint16_t*>(send);
  e.s_c = (int32_t)x.s_c;
  e.s_sp = (int32_t)x.s_sp;
  e.r = (int32_t)x.tr;
  e.t = (int32_t)x.t;
  return e;
}

inline EpiParams epi_acc(float* c, int64_t ldc) {
  EpiParams e{};
  e.kind = EpiKind::AccF32;
  e.c = c;
  e.ldc = ldc;
  return e;
}

inline EpiParams epi_store(void* c, int64_t ldc) {
  EpiParams e{};
  e.kind = EpiKind::StoreBF16;
  e.c = c;
  e.ldc = ldc;
  return e;
}

// split_ws: room for the fp32 partials of a K range cut into at most max_splits
// parts (AccF32 and StoreBF16 only; 0 = a product of the layer backward, by its
// rules; NULL = never split).
int run_gemm(const char* name, hipStream_t s, int64_t M, int64_t N, int64_t K, Operand A, Layout la, Operand B,
             Layout lb, EpiParams e, float* split_ws = nullptr, int max_splits = 0) {
  GemmParams p{};
  p.M = (int32_t)M;
  p.N = (int32_t)N;
  p.K = (int32_t)K;
  p.A = A;
  p.B = B;
  p.epi = e;
  const bool acc = e.kind == EpiKind::AccF32;
  const bool layer = split_ws && max_splits == 0;
  if (!split_ws || !(acc || e.kind == EpiKind::StoreBF16)) max_splits = 1;
  else if (layer) max_splits = gemm_max_splits(M, N, K, acc);
  const GemmPlan plan = gemm_plan(M, N, K, e.kind, max_splits, layer);
  p.tile = plan.tile;
  p.stream_c = plan.stream_c;
  p.k_splits = plan.splits;
  p.partial = split_ws;
  int rc = launch(name, s, [&] { return gemm(p, la, lb, s); });
  if (rc || p.k_splits <= 1) return rc;
  return launch("gemm_splitk_reduce", s, [&] {
    return acc ? gemm_split_reduce(static_cast<float*>(e.c), e.ldc, split_ws, M, N, p.k_splits, s)
               : gemm_split_store(static_cast<uint16_t*>(e.c), e.ldc, split_ws, M, N, p.k_splits, s);
  });
}

// Key runs of the attention: local chunks (stash K/V) then remote runs.
void key_segments(const Shard& x, AttnParams& ap, const uint16_t* K, const uint16_t* V, const uint16_t* rK,
                  const uint16_t* rV, uint16_t* dqkv, uint16_t* d_rk, uint16_t* d_rv, const uint16_t* cp_dk,
                  const uint16_t* cp_dv) {
  const int64_t kvw = x.k_t * x.d, qc = qkv_cols(x);
  ap.n_seg = 0;
  const int n_local = x.c == 1 ? 1 : 2;
  const int64_t run = x.c == 1 ? x.s : x.chunk_len;
  for (int i = 0; i < n_local; ++i) {
    KvSeg& g = ap.seg[ap.n_seg++];
    g = KvSeg{};
    const int64_t row0 = i * run;
    g.k = K + row0 * kvw;
    g.v = V + row0 * kvw;
    g.ld = kvw;
    g.bstride = x.s_c * kvw;
    if (dqkv) {
      g.dk = dqkv + row0 * qc + x.a_t * x.d;
      g.dv = dqkv + row0 * qc + (x.a_t + x.k_t) * x.d;
      g.d_ld = qc;
      g.d_bstride = x.s_c * qc;
    }
    if (cp_dk) {
      g.rk = cp_dk + row0 * kvw;
      g.rv = cp_dv + row0 * kvw;
    }
    g.n = (int32_t)run;
    g.pos0 = (int32_t)(x.qmap.chunk_id[i] * x.qmap.chunk_len);
    g.rope = 1;
    g.rope_row0 = (int32_t)row0;
  }
  int64_t rrow = 0;
  const int64_t rem_tokens = x.s - x.s_c;
  for (int r = 0; r < x.n_remote_runs; ++r) {
    KvSeg& g = ap.seg[ap.n_seg++];
    g = KvSeg{};
    const int64_t n = x.rem_chunk_count[r] * x.chunk_len;
    g.k = rK + rrow * kvw;
    g.v = rV + rrow * kvw;
    g.ld = kvw;
    g.bstride = rem_tokens * kvw;
    if (d_rk) {
      g.dk = d_rk + rrow * kvw;
      g.dv = d_rv + rrow * kvw;
      g.d_ld = kvw;
      g.d_bstride = rem_tokens * kvw;
    }
    g.n = (int32_t)n;
    g.pos0 = (int32_t)(x.rem_chunk_start[r] * x.chunk_len);
    g.rope = 0;
    rrow += n;
  }
}

AttnParams attn_params(const Shard& x) {
  AttnParams ap{};
  ap.n_split = 1;
  ap.b = (int32_t)x.b;
  ap.a_t = (int32_t)x.a_t;
  ap.k_t = (int32_t)x.k_t;
  ap.d_h = (int32_t)x.d;
  ap.n_q = (int32_t)x.s_c;
  ap.q_ld = x.a_t * x.d;
  ap.q_bstride = x.s_c * x.a_t * x.d;
  ap.qmap = x.qmap;
  ap.scale = 1.0f / std::sqrt((float)x.d);
  return ap;
}

int check_peers(const Shard& x, const l4d_peer_inputs* pi, bool bwd) {
  if (x.c > 1 && (!pi || !pi->remote_k || !pi->remote_v))
    return fail(L4D_EINVAL, "cp > 1 needs remote_k and remote_v");
  if (x.t > 1) {
    if (!pi || !pi->sp_peer_xn1 || !pi->sp_peer_xn2)
      return fail(L4D_EINVAL, "tp > 1 needs sp_peer_xn1 and sp_peer_xn2");
    if (bwd && (!pi->sp_peer_dy || !pi->sp_peer_dh1))
      return fail(L4D_EINVAL, "tp > 1 backward needs sp_peer_dy and sp_peer_dh1");
  }
  if (x.c > 1 && pi && ((pi->cp_peer_dk == nullptr) != (pi->cp_peer_dv == nullptr)))
    return fail(L4D_EINVAL, "cp_peer_dk and cp_peer_dv go together");
  return L4D_OK;
}
}  // namespace

// ============================================================== packed documents: checks and plans

namespace {
int check_packing(const l4d_packing* pk) {
  if (!pk) return fail(L4D_EINVAL, "packing is required");
  if (pk->tokens < 0 || pk->tokens > (int64_t)1 << 30 || pk->n_seqs < 0 || pk->n_seqs > (int64_t)1 << 30)
    return fail(L4D_EINVAL, "packing: tokens and n_seqs must lie in 0 .. 2^30");
  if (pk->n_seqs > 0 && !pk->starts) return fail(L4D_EINVAL, "packing: starts is required");
  if (reinterpret_cast<uintptr_t>(pk->starts) % 8) return fail(L4D_EINVAL, "packing: starts must be 8-byte aligned");
  return L4D_OK;
}
Packing device_packing(const l4d_packing* pk) {
  return Packing{pk->starts, (int32_t)pk->n_seqs, (int32_t)pk->tokens};
}

// ------------------------------------------------------------ rotary positions

constexpr int64_t kMaxRopeRows = (int64_t)1 << 25;   // a wave per row: 2^31 threads of a launch's 2^32

// f_j / 2 pi of every pair, in double.
int rope_turns(const l4d_rope* r, double* turns) {
  constexpr double kTwoPi = 6.283185307179586476925286766559;
  if (r->head_dim < 2 || r->head_dim > 2 * kMaxRopePairs) return fail(L4D_EINVAL, "rope: head_dim must lie in 2 .. 512");
  if (r->rot_dim < 2 || r->rot_dim > r->head_dim || r->rot_dim % 2)
    return fail(L4D_EINVAL, "rope: rot_dim must be even and lie in 2 .. head_dim");
  if (r->layout != L4D_ROPE_HALF && r->layout != L4D_ROPE_INTERLEAVED) return fail(L4D_EINVAL, "rope: unknown layout");
  if (r->scaling < L4D_ROPE_PLAIN || r->scaling > L4D_ROPE_RAMP) return fail(L4D_EINVAL, "rope: unknown scaling");
  if (!(r->base > 1.0) || !std::isfinite(r->base)) return fail(L4D_EINVAL, "rope: base must be finite and above 1");
  if (!(r->amplitude > 0.0) || !std::isfinite((float)r->amplitude))
    return fail(L4D_EINVAL, "rope: the amplitude must be finite and positive");
  const bool scaled = r->scaling != L4D_ROPE_PLAIN, bands = r->scaling == L4D_ROPE_BANDS || r->scaling == L4D_ROPE_RAMP;
  if (scaled && (!(r->factor > 0.0) || !std::isfinite(r->factor)))
    return fail(L4D_EINVAL, "rope: factor must be finite and positive");
  if (bands && (!(r->original > 0.0) || !std::isfinite(r->original) || !(r->low > 0.0) || !(r->high > r->low) ||
                !std::isfinite(r->high)))
    return fail(L4D_EINVAL, "rope: need original > 0 and 0 < low < high");
  const double rot = (double)r->rot_dim, log_base = std::log(r->base);
  double j0 = 0.0, j1 = 0.0;
  if (r->scaling == L4D_ROPE_RAMP) {
    // the pair that makes `t` turns over the original context: base^(-2j/rot) original = 2 pi t
    const auto pair_of = [&](double t) { return rot * std::log(r->original / (kTwoPi * t)) / (2.0 * log_base); };
    j0 = std::max(std::floor(pair_of(r->high)), 0.0);
    j1 = std::min(std::ceil(pair_of(r->low)), rot - 1.0);
  }
  for (int64_t j = 0; j < r->rot_dim / 2; ++j) {
    const double f = std::exp(-2.0 * (double)j / rot * log_base);
    double keep = 1.0;                       // g_j
    if (r->scaling == L4D_ROPE_LINEAR) keep = 0.0;
    else if (r->scaling == L4D_ROPE_BANDS) keep = (r->original * f / kTwoPi - r->low) / (r->high - r->low);
    else if (r->scaling == L4D_ROPE_RAMP) keep = 1.0 - std::min(std::max(((double)j - j0) / (j1 > j0 ? j1 - j0 : 0.001), 0.0), 1.0);
    keep = std::min(std::max(keep, 0.0), 1.0);
    turns[j] = (scaled ? f * ((1.0 - keep) / r->factor + keep) : f) / kTwoPi;
  }
  return L4D_OK;
}

// The rows that a tensor of a call occupies, in bytes: n rows of `width` bytes, `ld` apart.
struct RowRange {
  uintptr_t p;
  uint64_t width, ld, n;
  uint64_t span() const { return n ? (n - 1) * ld + width : 0; }
};
// Whether two tensors of n rows share a byte.  With equal strides rows may interleave
// (columns of one fused array); with different ones ranges that meet count as shared.
bool rows_meet(const RowRange& a, const RowRange& b) {
  if (a.p >= b.p + b.span() || b.p >= a.p + a.span()) return false;
  if (a.ld != b.ld) return true;
  const uint64_t off = b.p >= a.p ? (b.p - a.p) % a.ld : (a.ld - (a.p - b.p) % a.ld) % a.ld;   // b's column in a's rows
  return off < a.width || off + b.width > a.ld;
}
// The same, exact for different strides too.
bool rows_share(const RowRange& a, const RowRange& b) {
  if (a.ld == b.ld || !rows_meet(a, b)) return rows_meet(a, b);
  const RowRange &few = a.n <= b.n ? a : b, &many = a.n <= b.n ? b : a;
  for (uint64_t i = 0; i < few.n; ++i) {
    const uintptr_t lo = few.p + i * few.ld;
    const uint64_t j = lo < many.p + many.width ? 0 : (lo - many.p - many.width) / many.ld + 1;     // first row that ends behind lo
    if (j < many.n && many.p + j * many.ld < lo + few.width) return true;
  }
  return false;
}

// f_j / 2 pi and the axis of every pair.
int rope_axes(const l4d_rope* r, const l4d_rope_axes* x, RopeRotate* a) {
  int rc = rope_turns(r, a->turns);
  if (rc || !x) return rc;
  const int64_t n = x->n_axes, pairs = r->rot_dim / 2;
  if (n < 1 || n > 4) return fail(L4D_EINVAL, "rope axes: n_axes must lie in 1 .. 4");
  if (x->order != L4D_AXES_SECTIONS && x->order != L4D_AXES_CYCLED) return fail(L4D_EINVAL, "rope axes: unknown order");
  if (x->frequencies != L4D_AXES_SHARED && x->frequencies != L4D_AXES_OWN)
    return fail(L4D_EINVAL, "rope axes: unknown frequencies");
  int64_t sum = 0;
  for (int64_t i = 0; i < n; ++i) {
    if (x->pairs[i] < 1 || x->pairs[i] > pairs) return fail(L4D_EINVAL, "rope axes: an axis without pairs, or with more than rot_dim/2");
    sum += x->pairs[i];
  }
  if (sum != pairs) return fail(L4D_EINVAL, "rope axes: the pairs must add up to rot_dim/2");
  for (int64_t i = 1; x->order == L4D_AXES_CYCLED && i < n; ++i)
    if (i + n * (x->pairs[i] - 1) >= pairs) return fail(L4D_EINVAL, "rope axes: too many pairs of an axis to be dealt in turn");
  double own[4][kMaxRopePairs];
  for (int64_t i = 0; x->frequencies == L4D_AXES_OWN && i < n; ++i) {
    l4d_rope one = *r;
    one.rot_dim = 2 * x->pairs[i];
    if ((rc = rope_turns(&one, own[i]))) return rc;
  }
  int64_t used[4] = {};
  for (int64_t j = 0, section = 0; j < pairs; ++j) {
    int64_t at = j % n;
    if (x->order == L4D_AXES_CYCLED) at = j < n * x->pairs[at] ? at : 0;
    else at = section += used[section] == x->pairs[section];
    a->axis[j] = (uint8_t)at;
    if (x->frequencies == L4D_AXES_OWN) a->turns[j] = own[at][used[at]];
    ++used[at];
  }
  a->n_axes = (int32_t)n;
  return L4D_OK;
}

// The checks and parameters that calls over heads share, tensors apart.
int rope_setup(const l4d_rope* r, const l4d_rope_axes* axes, int dtype, int64_t tokens, const l4d_packing* pk,
               const int64_t* positions, RopeRotate* a) {
  if (!r) return fail(L4D_EINVAL, "rope is required");
  if (dtype != L4D_BF16 && dtype != L4D_F32) return fail(L4D_EINVAL, "rope: unknown dtype");
  if (tokens < 0 || tokens > kMaxRopeRows) return fail(L4D_EINVAL, "rope: tokens must lie in 0 .. 2^25");
  int rc;
  if (pk && (rc = check_packing(pk))) return rc;
  if (pk && pk->tokens != tokens) return fail(L4D_EINVAL, "rope: the packing is of another number of tokens");
  if (reinterpret_cast<uintptr_t>(positions) % 8) return fail(L4D_EINVAL, "rope: positions must be 8-byte aligned");
  if (axes && !positions && tokens > 0) return fail(L4D_EINVAL, "rope axes: positions are required");
  if ((rc = rope_axes(r, axes, a))) return rc;
  a->pk = pk ? device_packing(pk) : Packing{nullptr, -1, (int32_t)tokens};
  a->positions = positions;
  a->tokens = (int32_t)tokens;
  a->d_h = (int32_t)r->head_dim;
  a->rot = (int32_t)r->rot_dim;
  a->f32 = dtype == L4D_F32;
  a->interleaved = r->layout == L4D_ROPE_INTERLEAVED;
  a->amplitude = (float)r->amplitude;
  return L4D_OK;
}

// Whether a call over heads writes what its waves look up: the positions, or the documents' starts.
bool on_lookups(const RowRange& out, const l4d_rope_axes* axes, int64_t tokens, const l4d_packing* pk, const int64_t* positions) {
  const uint64_t n = 8ull * tokens * (axes ? axes->n_axes : 1), s = pk ? 8ull * (pk->n_seqs + 1) : 0;
  return (positions && rows_share(out, RowRange{reinterpret_cast<uintptr_t>(positions), n, n, 1})) ||
         (pk && pk->starts && rows_share(out, RowRange{reinterpret_cast<uintptr_t>(pk->starts), s, s, 1}));
}

int rope_call(const char* name, const l4d_rope* r, const l4d_rope_axes* axes, int dtype, int64_t tokens,
              const l4d_packing* pk, const int64_t* positions, const l4d_rope_heads* q, const l4d_rope_heads* k, int inverse,
              void* stream_ptr) {
  if (!r || !q) return fail(L4D_EINVAL, "rope and q are required");
  RopeRotate a{};
  int rc = rope_setup(r, axes, dtype, tokens, pk, positions, &a);
  if (rc) return rc;
  if (tokens == 0) return L4D_OK;                    // an empty array may have no address
  const int64_t size = dtype == L4D_F32 ? 4 : 2;
  const l4d_rope_heads* in[2] = {q, k};
  RowRange from[2], to[2];
  for (const l4d_rope_heads* t : in) {
    if (!t) continue;
    if (!t->x || !t->y) return fail(L4D_EINVAL, "rope: a tensor is NULL");
    if (t->heads < 1 || t->heads > 8192) return fail(L4D_EINVAL, "rope: heads must lie in 1 .. 8192");
    const int64_t cols = t->heads * r->head_dim;
    if (t->x_ld < cols || t->y_ld < cols || t->x_ld > (int64_t)1 << 31 || t->y_ld > (int64_t)1 << 31)
      return fail(L4D_EINVAL, "rope: a row stride is shorter than the heads, or above 2^31");
    const uintptr_t x = reinterpret_cast<uintptr_t>(t->x), y = reinterpret_cast<uintptr_t>(t->y);
    if (x % size || y % size) return fail(L4D_EINVAL, "rope: a tensor is misaligned");
    const RowRange rx{x, (uint64_t)(cols * size), (uint64_t)(t->x_ld * size), (uint64_t)tokens};
    const RowRange ry{y, (uint64_t)(cols * size), (uint64_t)(t->y_ld * size), (uint64_t)tokens};
    if (!(x == y && t->x_ld == t->y_ld) && x < y + ry.span() && y < x + rx.span())
      return fail(L4D_EINVAL, "rope: input and output overlap");
    if (a.n_tensors && a.t[0].y == t->y) return fail(L4D_EINVAL, "rope: q and k have the same output");
    // one launch turns both: what it writes of one tensor must be nothing it reads or writes of the other
    if (a.n_tensors && (rows_meet(ry, from[0]) || rows_meet(to[0], rx) || rows_meet(to[0], ry)))
      return fail(L4D_EINVAL, "rope: an output of q or k overlaps the other tensor");
    if (on_lookups(ry, axes, tokens, pk, positions)) return fail(L4D_EINVAL, "rope: an output overlaps positions or starts");
    from[a.n_tensors] = rx, to[a.n_tensors] = ry;
    a.t[a.n_tensors++] = RopeHeads{t->x, t->y, t->x_ld, t->y_ld, (int32_t)t->heads};
  }
  if (pk && pk->n_seqs == 0) return L4D_OK;
  a.inverse = inverse;
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  return launch(name, s, [&] { return rope_rotate(a, s); });
}

// ------------------------------------------------------------ norm and rotation of heads

// One tensor of a call: its arrays, the last one the output; g and d_g of head_dim elements.
struct NormTensor {
  const void *x, *dy;
  void* out;
  const void* gain;
  float* d_gain;
  int64_t heads, x_ld, dy_ld, out_ld;
};
int norm_call(const char* name, const l4d_rope* r, const l4d_rope_axes* axes, int dtype, int64_t tokens, const l4d_packing* pk,
              const int64_t* positions, float eps, const NormTensor* in, int n, bool backward, l4d_arena* A, void* stream_ptr) {
  QkNorm p{};
  int rc = rope_setup(r, axes, dtype, tokens, pk, positions, &p.r);
  if (rc) return rc;
  if (r->head_dim % 2) return fail(L4D_EINVAL, "qk_norm: head_dim must be even");
  if (!(eps >= 1e-30f) || !std::isfinite(eps)) return fail(L4D_EINVAL, "qk_norm: eps must be finite and at least 1e-30");
  if (tokens == 0) return L4D_OK;                    // an empty array may have no address
  const uint64_t size = dtype == L4D_F32 ? 4 : 2, d = (uint64_t)r->head_dim, rows = (uint64_t)tokens;
  struct Array { RowRange at; int tensor; };
  Array ins[6], outs[4];
  int n_in = 0, n_out = 0;
  for (int i = 0; i < n; ++i) {
    const NormTensor& t = in[i];
    if (!t.x || !t.out || !t.gain || (backward && (!t.dy || !t.d_gain))) return fail(L4D_EINVAL, "qk_norm: an array is NULL");
    if (t.heads < 1 || t.heads > 8192) return fail(L4D_EINVAL, "qk_norm: heads must lie in 1 .. 8192");
    const int64_t cols = t.heads * r->head_dim, most = (int64_t)1 << 31;
    if (t.x_ld < cols || t.out_ld < cols || t.x_ld > most || t.out_ld > most || (backward && (t.dy_ld < cols || t.dy_ld > most)))
      return fail(L4D_EINVAL, "qk_norm: a row stride is shorter than the heads, or above 2^31");
    const auto off = [&](const void* x, uint64_t by) { return reinterpret_cast<uintptr_t>(x) % by != 0; };
    if (off(t.x, size) || off(t.out, size) || off(t.gain, size) || (backward && (off(t.dy, size) || off(t.d_gain, 4))))
      return fail(L4D_EINVAL, "qk_norm: an array is misaligned");
    const auto range = [&](const void* x, int64_t ld) {
      return RowRange{reinterpret_cast<uintptr_t>(x), cols * size, ld * size, rows};
    };
    ins[n_in++] = {range(t.x, t.x_ld), i};
    ins[n_in++] = {RowRange{reinterpret_cast<uintptr_t>(t.gain), d * size, d * size, 1}, -1};
    if (backward) {
      ins[n_in++] = {range(t.dy, t.dy_ld), i};
      outs[n_out++] = {RowRange{reinterpret_cast<uintptr_t>(t.d_gain), d * 4, d * 4, 1}, -1};
    }
    outs[n_out++] = {range(t.out, t.out_ld), i};
    p.r.t[i] = RopeHeads{t.x, t.out, t.x_ld, t.out_ld, (int32_t)t.heads};
    p.gain[i] = t.gain;
    p.dy[i] = t.dy;
    p.dy_ld[i] = t.dy_ld;
    p.d_gain[i] = t.d_gain;
  }
  // An output may lie exactly on an input of its own tensor; nothing else it writes may be read or written twice.
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j) {
      const RowRange &a = outs[i].at, &b = ins[j].at;
      if (outs[i].tensor >= 0 && outs[i].tensor == ins[j].tensor && a.p == b.p && a.ld == b.ld) continue;
      if (rows_meet(a, b)) return fail(L4D_EINVAL, "qk_norm: an output overlaps an input");
    }
    for (int j = 0; j < i; ++j)
      if (rows_meet(outs[i].at, outs[j].at)) return fail(L4D_EINVAL, "qk_norm: two outputs overlap");
    if (on_lookups(outs[i].at, axes, tokens, pk, positions)) return fail(L4D_EINVAL, "qk_norm: an output overlaps positions or starts");
  }
  if (backward && !A) return fail(L4D_EINVAL, "arena is required");
  if (pk && pk->n_seqs == 0) return L4D_OK;
  p.r.n_tensors = n;
  p.eps = eps;
  p.backward = backward;
  Workspace ws;
  if (backward) {
    if ((rc = take_ws(A, align_up((uint64_t)qk_norm_parts(tokens) * 2 * d * 4), ws))) return rc;
    p.partial = reinterpret_cast<float*>(A->base + ws.off);
  }
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  return launch(name, s, [&] { return qk_norm_rope(p, s); });
}

// ------------------------------------------------------------ dropout and residual

int dropout_call(const char* name, int dtype, int64_t rows, int64_t cols, const void* x, int64_t x_ld, const void* res,
                 int64_t r_ld, void* y, int64_t y_ld, double p, const int64_t* rng, int64_t first_row, void* stream_ptr) {
  if (dtype != L4D_BF16 && dtype != L4D_F32) return fail(L4D_EINVAL, "dropout: unknown dtype");
  if (rows < 0 || rows > (int64_t)1 << 31 || cols < 0 || cols > (int64_t)1 << 24 || rows * cols > (int64_t)1 << 34)
    return fail(L4D_EINVAL, "dropout: rows must lie in 0 .. 2^31, cols in 0 .. 2^24, their product in 0 .. 2^34");
  if (first_row < 0 || first_row > (int64_t)1 << 38) return fail(L4D_EINVAL, "dropout: first_row must lie in 0 .. 2^38");
  if (!(p >= 0.0) || std::nearbyint(p * 4294967296.0) > 4294967295.0)
    return fail(L4D_EINVAL, "dropout: p must lie in [0, 1)");
  if (rows == 0 || cols == 0) return L4D_OK;         // an empty array may have no address
  if (!x || !y || !rng) return fail(L4D_EINVAL, "dropout: an array is NULL");
  if (reinterpret_cast<uintptr_t>(rng) % 8) return fail(L4D_EINVAL, "dropout: rng must be 8-byte aligned");
  const uint64_t size = dtype == L4D_F32 ? 4 : 2;
  const void* arrays[3] = {x, y, res};
  const int64_t lds[3] = {x_ld, y_ld, r_ld};
  RowRange at[3];
  for (int i = 0; i < (res ? 3 : 2); ++i) {
    if (reinterpret_cast<uintptr_t>(arrays[i]) % size) return fail(L4D_EINVAL, "dropout: an array is misaligned");
    if (lds[i] < cols || lds[i] > (int64_t)1 << 31)
      return fail(L4D_EINVAL, "dropout: a row stride is shorter than the columns, or above 2^31");
    at[i] = RowRange{reinterpret_cast<uintptr_t>(arrays[i]), cols * size, lds[i] * size, (uint64_t)rows};
  }
  const RowRange words{reinterpret_cast<uintptr_t>(rng), 16, 16, 1};
  if (rows_meet(at[1], words)) return fail(L4D_EINVAL, "dropout: the output overlaps rng");
  for (int i = 0; i < (res ? 3 : 2); i += 2)
    if (!(at[1].p == at[i].p && at[1].ld == at[i].ld) && rows_meet(at[1], at[i]))
      return fail(L4D_EINVAL, "dropout: input and output overlap");
  DropoutAdd a{};
  a.x = x, a.residual = res, a.y = y;
  a.rows = rows, a.cols = cols, a.x_ld = x_ld, a.r_ld = r_ld, a.y_ld = y_ld;
  a.rng = rng;
  a.first = (uint64_t)first_row * (uint64_t)cols;
  a.threshold = (uint32_t)std::nearbyint(p * 4294967296.0);
  a.scale = (float)(1.0 / (1.0 - p));
  a.f32 = dtype == L4D_F32;
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  return launch(name, s, [&] { return dropout_add(a, s); });
}
}  // namespace

namespace {
constexpr int kMaxSinks = 4096;
struct AttnRows {        // one tensor of a call
  const char* name;
  const void* p;
  int64_t ld, heads;
};
int attn_shape(const l4d_attn* at, PackedAttn* p) {
  if (!at) return fail(L4D_EINVAL, "attn is required");
  if (at->head_dim != 64 && at->head_dim != 128)
    return fail(L4D_EINVAL, "head dim %lld unsupported (64 or 128)", (long long)at->head_dim);
  if (at->n_heads < 1 || at->n_heads > (int64_t)1 << 16 || at->n_kv_heads < 1 || at->n_heads % at->n_kv_heads)
    return fail(L4D_EINVAL, "n_heads must lie in 1 .. 2^16 and be a multiple of n_kv_heads");
  if (!(at->scale >= 0.f) || !std::isfinite(at->scale)) return fail(L4D_EINVAL, "the scale must be finite and >= 0");
  p->heads = (int32_t)at->n_heads;
  p->kv_heads = (int32_t)at->n_kv_heads;
  p->d_h = (int32_t)at->head_dim;
  p->scale = at->scale > 0.f ? at->scale : 1.0f / std::sqrt((float)at->head_dim);
  return L4D_OK;
}
int attn_rows(const AttnRows* t, int n, int64_t d) {
  for (int i = 0; i < n; ++i) {
    if (!t[i].p) return fail(L4D_EINVAL, "%s is required", t[i].name);
    if (reinterpret_cast<uintptr_t>(t[i].p) % 16) return fail(L4D_EINVAL, "%s must be 16-byte aligned", t[i].name);
    if (t[i].ld < t[i].heads * d || t[i].ld % 8 || t[i].ld > (int64_t)1 << 22)
      return fail(L4D_EINVAL, "the row stride of %s must cover its heads, be a multiple of 8 and at most 2^22", t[i].name);
  }
  return L4D_OK;
}
// No output may start where another tensor does.
int attn_distinct(const AttnRows* t, int n, int first_out) {
  for (int i = first_out; i < n; ++i)
    for (int j = 0; j < i; ++j)
      if (t[i].p == t[j].p) return fail(L4D_EINVAL, "%s and %s are the same array", t[i].name, t[j].name);
  return L4D_OK;
}
// Nothing a call writes (its tensors from first_out on; lse in the forward) may be read or written twice by it.
int attn_apart(const AttnRows* t, int n, int first_out, const l4d_attn* at, const float* lse, const l4d_packing* pk) {
  RowRange r[10];
  const char* name[10];
  const uint64_t rows = (uint64_t)pk->tokens, sums = 4ull * at->n_heads * rows, starts = 8ull * (pk->n_seqs + 1);
  int m = 0;
  for (int i = 0; i < n; ++i, ++m) {
    r[m] = RowRange{reinterpret_cast<uintptr_t>(t[i].p), 2ull * t[i].heads * at->head_dim, 2ull * t[i].ld, rows};
    name[m] = t[i].name;
  }
  r[m] = RowRange{reinterpret_cast<uintptr_t>(lse), sums, sums, 1};
  name[m++] = "lse";
  if (pk->starts) {
    r[m] = RowRange{reinterpret_cast<uintptr_t>(pk->starts), starts, starts, 1};
    name[m++] = "starts";
  }
  uintptr_t end[10];
  for (int i = 0; i < m; ++i) end[i] = r[i].p + r[i].span();
  const int last_out = n == 4 ? n : n - 1;
  for (int j = first_out; j <= last_out; ++j)
    for (int i = 0; i < m; ++i)
      if (i != j && r[i].p < end[j] && r[j].p < end[i] && rows_share(r[i], r[j]))
        return fail(L4D_EINVAL, "%s and %s overlap", name[i], name[j]);
  return L4D_OK;
}
// dQ first: it also writes delta, which dK/dV reads.
int packed_attn_backward(const PackedAttn& p, hipStream_t s) {
  int rc;
  if ((rc = launch("attn_packed_dq", s, [&] { return attn_packed_bwd(p, 2, s); }))) return rc;
  if ((rc = launch("attn_packed_dkdv", s, [&] { return attn_packed_bwd(p, 1, s); }))) return rc;
  if (p.n_split > 1) return launch("attn_packed_reduce", s, [&] { return attn_packed_bwd(p, 3, s); });
  return L4D_OK;
}
int window_attn_backward(const WindowAttn& p, hipStream_t s) {
  int rc;
  if ((rc = launch("attn_window_dq", s, [&] { return attn_window_bwd(p, 2, s); }))) return rc;
  if ((rc = launch("attn_window_dkdv", s, [&] { return attn_window_bwd(p, 1, s); }))) return rc;
  if (p.n_split > 1 && (rc = launch("attn_window_reduce", s, [&] { return attn_window_bwd(p, 3, s); }))) return rc;
  if (p.far_parts) return launch("attn_window_sinks", s, [&] { return attn_window_bwd(p, 4, s); });
  return L4D_OK;
}
// A window that no row of `tokens` rows reaches past hides nothing: the call is the one without.
int attn_window(const l4d_window* w, int64_t tokens, WindowAttn* p) {
  if (!w) return fail(L4D_EINVAL, "window is required");
  if (w->window < 1) return fail(L4D_EINVAL, "the window must be at least 1");
  if (w->sinks < 0 || w->sinks > kMaxSinks) return fail(L4D_EINVAL, "sinks must lie in 0 .. %d", kMaxSinks);
  p->pk.tokens = (int32_t)tokens;
  if (w->window >= tokens) return L4D_OK;
  p->window = (int32_t)w->window;
  p->sinks = (int32_t)w->sinks;
  attn_window_chunks(p);
  return L4D_OK;
}
struct PackedWs {
  uint64_t delta, lse2, items, partial, sinks, total;
};
PackedWs plan_packed(const WindowAttn& p, int64_t tokens) {
  Carver cv;
  PackedWs w{};
  w.delta = cv.take((uint64_t)p.heads * tokens * 4);
  w.lse2 = cv.take((uint64_t)p.heads * tokens * 4);
  w.items = cv.take(p.window ? (uint64_t)attn_window_items(p) * 16 : (uint64_t)attn_packed_items(tokens) * 8);
  const int splits = attn_packed_most_splits(tokens, p.heads, p.kv_heads);
  w.partial = splits > 1 ? cv.take(2ull * splits * tokens * p.kv_heads * p.d_h * 4) : 0;
  w.sinks = cv.take(2ull * p.far_parts * splits * p.kv_heads * p.sinks * p.d_h * 4);
  w.total = cv.used;
  return w;
}
}  // namespace

namespace {
// A layer call over packed documents: what replaces the sequence of equal rows.
struct LayerPacking {
  const l4d_packing* pk;
  RopeRotate rope;             // head size, angles and amplitude; no tensors
};
int layer_packing(const Shard& x, const l4d_packing* pk, const l4d_rope* rope, LayerPacking* lp) {
  int rc = check_packing(pk);
  if (rc) return rc;
  if (x.c != 1 || x.b != 1) return fail(L4D_EINVAL, "packed documents need cp == 1 and micro_batch == 1");
  if (pk->tokens != x.s) return fail(L4D_EINVAL, "the packing has %lld tokens, the layer %lld", (long long)pk->tokens, (long long)x.s);
  if (pk->n_seqs == 0) return fail(L4D_EINVAL, "packing: a layer call needs at least one document");
  l4d_rope plain{};
  plain.head_dim = plain.rot_dim = x.d;
  plain.base = x.base;
  plain.amplitude = 1.0;
  if (!rope) rope = &plain;
  if (rope->head_dim != x.d || rope->rot_dim != x.d || rope->layout != L4D_ROPE_HALF)
    return fail(L4D_EINVAL, "the layer turns whole heads of %lld in the half layout", (long long)x.d);
  lp->pk = pk;
  lp->rope = RopeRotate{};
  if ((rc = rope_turns(rope, lp->rope.turns))) return rc;
  lp->rope.pk = device_packing(pk);
  lp->rope.tokens = (int32_t)pk->tokens;
  lp->rope.d_h = lp->rope.rot = (int32_t)x.d;
  lp->rope.amplitude = (float)rope->amplitude;
  PackedAttn p{};
  p.pk = device_packing(pk);
  p.heads = (int32_t)x.a_t;
  p.kv_heads = (int32_t)x.k_t;
  p.d_h = (int32_t)x.d;
  if (!attn_packed_fits(p) || pk->tokens > kMaxRopeRows) return fail(L4D_EINVAL, "problem too large");
  return L4D_OK;
}
// The layer's attention over its documents: Q, K, V, ctx and LSE of the stash.
PackedAttn packed_layer_attn(const Shard& x, const LayerPacking& lp, const l4d_stash* st) {
  PackedAttn p{};
  p.pk = device_packing(lp.pk);
  p.heads = (int32_t)x.a_t;
  p.kv_heads = (int32_t)x.k_t;
  p.d_h = (int32_t)x.d;
  p.scale = 1.0f / std::sqrt((float)x.d);
  attn_packed_plan(&p);
  p.q = sptr(st, L4D_STASH_Q);
  p.k = sptr(st, L4D_STASH_K);
  p.v = sptr(st, L4D_STASH_V);
  p.o = sptr(st, L4D_STASH_CTX);
  p.q_ld = p.o_ld = x.a_t * x.d;
  p.k_ld = p.v_ld = x.k_t * x.d;
  p.lse = sptr<float>(st, L4D_STASH_LSE);
  return p;
}
}  // namespace

// ============================================================== layer forward

// packing == nullptr: sequences of equal length, with the model's own RoPE.
static int layer_forward(const l4d_model* m, const l4d_parallel* p, const l4d_packing* packing, const l4d_rope* scaled,
                         const l4d_layer_weights* w, const void* x_in, const l4d_peer_inputs* peers,
                         const l4d_peer_outputs* sends, void* y, l4d_arena* A, l4d_stash** stash_out, void* stream_ptr) {
  Shard x;
  int rc = make_shard(m, p, &x);
  if (rc) return rc;
  LayerPacking lp{};
  if (packing && (rc = layer_packing(x, packing, scaled, &lp))) return rc;
  if (!w || !w->norm1 || !w->qkv || !w->o || !w->norm2 || !w->gate_up || !w->down)
    return fail(L4D_EINVAL, "all six weights are required");
  if (!x_in || !y || !A || !stash_out) return fail(L4D_EINVAL, "x, y, arena and stash_out are required");
  if ((rc = check_peers(x, peers, false))) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);

  const FwdWs plan = plan_fwd(x, sends);
  l4d_stash* st = nullptr;
  if ((rc = stash_reserve(A, x, &st))) return rc;
  Workspace ws;
  if ((rc = take_ws(A, plan.total, ws))) {
    l4d_stash_release(A, st);
    return rc;
  }
  uint8_t* wsb = reinterpret_cast<uint8_t*>(A->base + ws.off);
  float2* rope = reinterpret_cast<float2*>(wsb + plan.rope);
  const l4d_peer_inputs none{};
  const l4d_peer_inputs& pi = peers ? *peers : none;
  void* o_send = (sends && sends->o_partial) ? sends->o_partial : (void*)(wsb + plan.o_send);
  void* ffn_send = (sends && sends->ffn_partial) ? sends->ffn_partial : (void*)(wsb + plan.ffn_send);
  const int64_t tok = x.b * x.s_c, nq = x.a_t * x.d, nk = x.k_t * x.d;

  auto body = [&]() -> int {
    int r;
    const RopeTable table{rope, x.qmap, (int32_t)x.s_c, (int32_t)x.d, std::log((double)x.base)};
    // norm-1, stashing its input x as it goes, and the RoPE table
    if ((r = launch("rmsnorm1_fwd", s, [&] {
           return rmsnorm_fwd(static_cast<const uint16_t*>(x_in), static_cast<const uint16_t*>(w->norm1),
                              sptr(st, L4D_STASH_XN1), x.b * x.s_sp, (int32_t)x.h, x.eps, s, sptr(st, L4D_STASH_X),
                              lp.pk ? nullptr : &table);
         })))
      return r;
    if (lp.pk && (r = launch("rope_table_packed", s, [&] { return rope_table(lp.rope, rope, s); }))) return r;
    // [Q|K|V] = xn1_full W_qkv^T, RoPE on Q, K
    EpiParams eq{};
    eq.kind = EpiKind::QkvRope;
    eq.q = sptr(st, L4D_STASH_Q);
    eq.k = sptr(st, L4D_STASH_K);
    eq.v = sptr(st, L4D_STASH_V);
    eq.nq = (int32_t)nq;
    eq.nk = (int32_t)nk;
    eq.rope = rope;
    eq.d_h = (int32_t)x.d;
    eq.s_c = (int32_t)x.s_c;
    if ((r = run_gemm("gemm_qkv", s, tok, qkv_cols(x), x.h, op(gathered(sptr(st, L4D_STASH_XN1), pi.sp_peer_xn1, x), tok),
                      Layout::KC, op(RowSrc::plain(w->qkv, x.h), qkv_cols(x)), Layout::KC, eq)))
      return r;
    // attention
    if (lp.pk) {
      const PackedAttn pa = packed_layer_attn(x, lp, st);
      if ((r = launch("clear_outside", s, [&] { return clear_outside(pa.pk, pa.o, pa.o_ld, nq, s); }))) return r;
      if ((r = launch("attn_packed_fwd", s, [&] { return attn_packed_fwd(pa, s); }))) return r;
    } else {
      AttnParams ap = attn_params(x);
      ap.q = sptr(st, L4D_STASH_Q);
      ap.o = sptr(st, L4D_STASH_CTX);
      ap.lse = sptr<float>(st, L4D_STASH_LSE);
      key_segments(x, ap, sptr(st, L4D_STASH_K), sptr(st, L4D_STASH_V), static_cast<const uint16_t*>(pi.remote_k),
                   static_cast<const uint16_t*>(pi.remote_v), nullptr, nullptr, nullptr, nullptr, nullptr);
      if ((r = launch("attn_fwd", s, [&] { return attn_fwd(ap, s); }))) return r;
    }
    // h1 = x + ctx W_o^T (own rows; peers' rows are sent)
    if ((r = run_gemm("gemm_o", s, tok, x.h, nq, op(RowSrc::plain(sptr(st, L4D_STASH_CTX), nq), tok), Layout::KC,
                      op(RowSrc::plain(w->o, nq), x.h), Layout::KC,
                      epi_residual(x, sptr(st, L4D_STASH_H1), x_in, pi.sp_peer_o, o_send))))
      return r;
    if ((r = launch("rmsnorm2_fwd", s, [&] {
           return rmsnorm_fwd(sptr(st, L4D_STASH_H1), static_cast<const uint16_t*>(w->norm2), sptr(st, L4D_STASH_XN2),
                              x.b * x.s_sp, (int32_t)x.h, x.eps, s);
         })))
      return r;
    // [G|U] = xn2_full W_gu^T with the SwiGLU epilogue
    EpiParams eg{};
    eg.kind = EpiKind::SwiGLUFwd;
    eg.g_out = sptr(st, L4D_STASH_GATE);
    eg.u_out = sptr(st, L4D_STASH_UP);
    eg.act_out = sptr(st, L4D_STASH_ACT);
    eg.prod_out = sptr(st, L4D_STASH_PROD);
    eg.f = (int32_t)x.f_t;
    Operand bgu{RowSrc::plain(w->gate_up, x.h), (int32_t)(2 * x.f_t), (int32_t)x.f_t, x.f_t};
    if ((r = run_gemm("gemm_gate_up", s, tok, 2 * x.f_t, x.h, op(gathered(sptr(st, L4D_STASH_XN2), pi.sp_peer_xn2, x), tok),
                      Layout::KC, bgu, Layout::KC, eg)))
      return r;
    // y = h1 + prod W_down^T
    if ((r = run_gemm("gemm_down", s, tok, x.h, x.f_t, op(RowSrc::plain(sptr(st, L4D_STASH_PROD), x.f_t), tok),
                      Layout::KC, op(RowSrc::plain(w->down, x.f_t), x.h), Layout::KC,
                      epi_residual(x, static_cast<uint16_t*>(y), sptr(st, L4D_STASH_H1), pi.sp_peer_ffn, ffn_send))))
      return r;
    return L4D_OK;
  };
  rc = body();
  if (rc) {
    l4d_stash_release(A, st);
    return rc;
  }
  st->packed = lp.pk != nullptr;
  *stash_out = st;
  return L4D_OK;
}

extern "C" int llama_layer_fwd(const l4d_model* m, const l4d_parallel* p, const l4d_layer_weights* w,
                               const void* x_in, const l4d_peer_inputs* peers, const l4d_peer_outputs* sends,
                               void* y, l4d_arena* A, l4d_stash** stash_out, void* stream_ptr) {
  return layer_forward(m, p, nullptr, nullptr, w, x_in, peers, sends, y, A, stash_out, stream_ptr);
}

extern "C" int llama_layer_packed_fwd(const l4d_model* m, const l4d_parallel* p, const l4d_packing* packing,
                                      const l4d_rope* rope, const l4d_layer_weights* w, const void* x_in,
                                      const l4d_peer_inputs* peers, const l4d_peer_outputs* sends, void* y,
                                      l4d_arena* A, l4d_stash** stash_out, void* stream_ptr) {
  if (!packing) return fail(L4D_EINVAL, "packing is required");
  return layer_forward(m, p, packing, rope, w, x_in, peers, sends, y, A, stash_out, stream_ptr);
}

// ============================================================== layer backward

static int layer_backward(const l4d_model* m, const l4d_parallel* p, const l4d_packing* packing, const l4d_rope* scaled,
                          const l4d_layer_weights* w, const l4d_peer_inputs* peers, const l4d_peer_outputs* sends,
                          l4d_stash* st, const void* dy, void* dx, const l4d_layer_grads* dw, void* d_remote_k,
                          void* d_remote_v, l4d_arena* A, void* stream_ptr) {
  Shard x;
  int rc = make_shard(m, p, &x);
  if (rc) return rc;
  LayerPacking lp{};
  if (packing && (rc = layer_packing(x, packing, scaled, &lp))) return rc;
  if (!w || !w->norm1 || !w->qkv || !w->o || !w->norm2 || !w->gate_up || !w->down)
    return fail(L4D_EINVAL, "all six weights are required");
  if (!dw || !dw->norm1 || !dw->qkv || !dw->o || !dw->norm2 || !dw->gate_up || !dw->down)
    return fail(L4D_EINVAL, "all six gradient accumulators are required");
  if (!st || !A || !dy || !dx) return fail(L4D_EINVAL, "stash, arena, dy and dx are required");
  if (st->arena != A || !A->live.count(st)) return fail(L4D_EINVAL, "stash does not belong to this arena");
  if (st->kind != kLayerStash) return fail(L4D_EINVAL, "not a layer stash");
  const Shard& sx = st->shape;
  if (sx.h != x.h || sx.a != x.a || sx.k != x.k || sx.f != x.f || sx.s != x.s || sx.b != x.b || sx.t != x.t ||
      sx.c != x.c || sx.tr != x.tr || sx.cr != x.cr)
    return fail(L4D_EINVAL, "stash was made for another shape");
  if (st->packed != (packing != nullptr)) return fail(L4D_EINVAL, "the stash is of %s layer call", st->packed ? "a packed" : "an unpacked");
  if (x.c > 1 && (!d_remote_k || !d_remote_v)) return fail(L4D_EINVAL, "cp > 1 needs d_remote_k and d_remote_v");
  if ((rc = check_peers(x, peers, true))) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);

  const BwdWs plan = plan_bwd(x, sends);
  Workspace ws;
  if ((rc = take_ws(A, plan.total, ws))) return rc;
  uint8_t* wsb = reinterpret_cast<uint8_t*>(A->base + ws.off);
  auto W = [&](uint64_t off) { return reinterpret_cast<uint16_t*>(wsb + off); };
  float2* rope = reinterpret_cast<float2*>(wsb + plan.rope);
  uint16_t *dgu = W(plan.dgu), *dh1 = W(plan.dh1), *dctx = W(plan.dctx), *dqkv = W(plan.dqkv);
  auto F = [&](uint64_t off) { return reinterpret_cast<float*>(wsb + off); };
  float *dxn2 = F(plan.dxn2), *dxn1 = F(plan.dxn1), *dh1_f32 = F(plan.dh1_f32);
  float* delta = reinterpret_cast<float*>(wsb + plan.delta);
  float* partial = reinterpret_cast<float*>(wsb + plan.partial);
  float *ffn_part = F(plan.ffn_part), *proj_part = F(plan.proj_part);
  const l4d_peer_inputs none{};
  const l4d_peer_inputs& pi = peers ? *peers : none;
  void* dxn2_send = (sends && sends->dxn2_partial) ? sends->dxn2_partial : (void*)W(plan.dxn2_send);
  void* dxn1_send = (sends && sends->dxn1_partial) ? sends->dxn1_partial : (void*)W(plan.dxn1_send);
  const int64_t tok = x.b * x.s_c, nq = x.a_t * x.d, qc = qkv_cols(x), rows_sp = x.b * x.s_sp;
  const int32_t npart = rmsnorm_bwd_partials(rows_sp);

  auto body = [&]() -> int {
    int r;
    const RopeTable table{rope, x.qmap, (int32_t)x.s_c, (int32_t)x.d, std::log((double)x.base)};
    const RowSrc dy_full = gathered(dy, pi.sp_peer_dy, x);
    // d(prod) = dy_full W_down, consumed by the SwiGLU backward in the epilogue
    EpiParams es{};
    es.kind = EpiKind::SwiGLUBwd;
    es.g_in = sptr(st, L4D_STASH_GATE);
    es.u_in = sptr(st, L4D_STASH_UP);
    es.act_in = sptr(st, L4D_STASH_ACT);
    es.dgu = dgu;
    es.f = (int32_t)x.f_t;
    if ((r = run_gemm("gemm_down_dx", s, tok, x.f_t, x.h, op(dy_full, tok), Layout::KC,
                      op(RowSrc::plain(w->down, x.f_t), x.f_t), Layout::MN, es)))
      return r;
    // dW_down += dy_full^T prod
    if ((r = run_gemm("gemm_down_dw", s, x.h, x.f_t, tok, op(dy_full, x.h), Layout::MN,
                      op(RowSrc::plain(sptr(st, L4D_STASH_PROD), x.f_t), x.f_t), Layout::MN, epi_acc(dw->down, x.f_t), ffn_part)))
      return r;
    // d(xn2) = dGU W_gu (own rows + receipt; peers' rows sent)
    if ((r = run_gemm("gemm_gate_up_dx", s, tok, x.h, 2 * x.f_t, op(RowSrc::plain(dgu, 2 * x.f_t), tok), Layout::KC,
                      op(RowSrc::plain(w->gate_up, x.h), x.h), Layout::MN,
                      epi_residual(x, nullptr, nullptr, pi.sp_peer_dxn2, dxn2_send, dxn2))))
      return r;
    const RowSrc xn2_full = gathered(sptr(st, L4D_STASH_XN2), pi.sp_peer_xn2, x);
    if ((r = run_gemm("gemm_gate_up_dw", s, 2 * x.f_t, x.h, tok, op(RowSrc::plain(dgu, 2 * x.f_t), 2 * x.f_t),
                      Layout::MN, op(xn2_full, x.h), Layout::MN, epi_acc(dw->gate_up, x.h), ffn_part)))
      return r;
    // norm-2 backward + residual: dh1 in bf16 (product operand) and fp32 (residual of dx)
    if ((r = launch("rmsnorm2_bwd", s, [&] {
           const NormBwdIo io{nullptr, dxn2, static_cast<const uint16_t*>(dy), nullptr, dh1, dh1_f32};
           return rmsnorm_bwd(sptr(st, L4D_STASH_H1), static_cast<const uint16_t*>(w->norm2), io, partial, npart,
                              rows_sp, (int32_t)x.h, x.eps, s);
         })))
      return r;
    // the gain gradient's sum, and the RoPE table for the attention backward
    if ((r = launch("reduce_gain", s, [&] { return reduce_rows_add(partial, npart, (int32_t)x.h, dw->norm2, s, lp.pk ? nullptr : &table); })))
      return r;
    // attention output projection
    const RowSrc dh1_full = gathered(dh1, pi.sp_peer_dh1, x);
    if ((r = run_gemm("gemm_o_dx", s, tok, nq, x.h, op(dh1_full, tok), Layout::KC, op(RowSrc::plain(w->o, nq), nq),
                      Layout::MN, epi_store(dctx, nq), proj_part)))
      return r;
    if ((r = run_gemm("gemm_o_dw", s, x.h, nq, tok, op(dh1_full, x.h), Layout::MN,
                      op(RowSrc::plain(sptr(st, L4D_STASH_CTX), nq), nq), Layout::MN, epi_acc(dw->o, nq), proj_part)))
      return r;
    // attention backward -> dQKV (inverse RoPE applied), remote dK/dV
    if (lp.pk) {
      PackedAttn pa = packed_layer_attn(x, lp, st);
      pa.dout = dctx;
      pa.do_ld = nq;
      pa.delta = delta;
      // dxn1 is written after the attention: its 4 d bytes per row and head hold lse2 and, behind it, the list
      pa.lse2 = dxn1;
      pa.items = reinterpret_cast<int32_t*>(dxn1 + (x.a_t * x.s + 3) / 4 * 4);
      pa.rope = rope;                 // dQ and dK are turned back before their one rounding, as in the unpacked layer
      pa.dq = dqkv;
      pa.dk = dqkv + nq;
      pa.dv = dqkv + nq + x.k_t * x.d;
      pa.dq_ld = pa.dk_ld = pa.dv_ld = qc;
      pa.dkv_partial = reinterpret_cast<float*>(wsb + plan.dkv);
      if ((r = launch("clear_outside", s, [&] { return clear_outside(pa.pk, dqkv, qc, qc, s); }))) return r;
      if ((r = launch("rope_table_packed", s, [&] { return rope_table(lp.rope, rope, s); }))) return r;
      if ((r = packed_attn_backward(pa, s))) return r;
    } else {
      AttnParams ap = attn_params(x);
      ap.q = sptr(st, L4D_STASH_Q);
      ap.o = sptr(st, L4D_STASH_CTX);
      ap.lse = sptr<float>(st, L4D_STASH_LSE);
      ap.dout = dctx;
      ap.delta = delta;
      ap.dq = dqkv;
      ap.dq_ld = qc;
      ap.rope = rope;
      key_segments(x, ap, sptr(st, L4D_STASH_K), sptr(st, L4D_STASH_V), static_cast<const uint16_t*>(pi.remote_k),
                   static_cast<const uint16_t*>(pi.remote_v), dqkv, static_cast<uint16_t*>(d_remote_k),
                   static_cast<uint16_t*>(d_remote_v), static_cast<const uint16_t*>(pi.cp_peer_dk),
                   static_cast<const uint16_t*>(pi.cp_peer_dv));
      ap.total_keys = 0;
      for (int i = 0; i < ap.n_seg; ++i) {
        ap.seg_key0[i] = ap.total_keys;
        ap.total_keys += ap.seg[i].n;
      }
      ap.n_split = attn_bwd_splits(ap);
      if (ap.n_split > 1) {
        ap.dkv_partial = reinterpret_cast<float*>(wsb + plan.dkv);
        ap.partial_half = (int64_t)ap.n_split * x.b * ap.total_keys * x.k_t * x.d;
      }
      // dQ first: it also writes delta = rowsum(dO * O), which dK/dV reads
      if ((r = launch("attn_bwd_dq", s, [&] { return attn_bwd(ap, 2, s); }))) return r;
      if ((r = launch("attn_bwd_dkdv", s, [&] { return attn_bwd(ap, 1, s); }))) return r;
      if (ap.n_split > 1 && (r = launch("attn_dkv_reduce", s, [&] { return attn_bwd(ap, 3, s); }))) return r;
    }
    // QKV projection
    if ((r = run_gemm("gemm_qkv_dx", s, tok, x.h, qc, op(RowSrc::plain(dqkv, qc), tok), Layout::KC,
                      op(RowSrc::plain(w->qkv, x.h), x.h), Layout::MN,
                      epi_residual(x, nullptr, nullptr, pi.sp_peer_dxn1, dxn1_send, dxn1))))
      return r;
    const RowSrc xn1_full = gathered(sptr(st, L4D_STASH_XN1), pi.sp_peer_xn1, x);
    if ((r = run_gemm("gemm_qkv_dw", s, qc, x.h, tok, op(RowSrc::plain(dqkv, qc), qc), Layout::MN, op(xn1_full, x.h),
                      Layout::MN, epi_acc(dw->qkv, x.h), proj_part)))
      return r;
    // norm-1 backward + residual
    if ((r = launch("rmsnorm1_bwd", s, [&] {
           const NormBwdIo io{nullptr, dxn1, nullptr, dh1_f32, static_cast<uint16_t*>(dx), nullptr};
           return rmsnorm_bwd(sptr(st, L4D_STASH_X), static_cast<const uint16_t*>(w->norm1), io, partial, npart,
                              rows_sp, (int32_t)x.h, x.eps, s);
         })))
      return r;
    if ((r = launch("reduce_gain", s, [&] { return reduce_rows_add(partial, npart, (int32_t)x.h, dw->norm1, s); })))
      return r;
    return L4D_OK;
  };
  rc = body();
  if (rc) return rc;
  return l4d_stash_release(A, st);
}

extern "C" int llama_layer_bwd(const l4d_model* m, const l4d_parallel* p, const l4d_layer_weights* w,
                               const l4d_peer_inputs* peers, const l4d_peer_outputs* sends, l4d_stash* st,
                               const void* dy, void* dx, const l4d_layer_grads* dw, void* d_remote_k,
                               void* d_remote_v, l4d_arena* A, void* stream_ptr) {
  return layer_backward(m, p, nullptr, nullptr, w, peers, sends, st, dy, dx, dw, d_remote_k, d_remote_v, A, stream_ptr);
}

extern "C" int llama_layer_packed_bwd(const l4d_model* m, const l4d_parallel* p, const l4d_packing* packing,
                                      const l4d_rope* rope, const l4d_layer_weights* w, const l4d_peer_inputs* peers,
                                      const l4d_peer_outputs* sends, l4d_stash* st, const void* dy, void* dx,
                                      const l4d_layer_grads* dw, l4d_arena* A, void* stream_ptr) {
  if (!packing) return fail(L4D_EINVAL, "packing is required");
  return layer_backward(m, p, packing, rope, w, peers, sends, st, dy, dx, dw, nullptr, nullptr, A, stream_ptr);
}

// ============================================================== LM head

namespace {
int lm_xent_check(int64_t n, int64_t h, int64_t v_t, int64_t v0, const void* hidden, const void* w_lm,
                  const int64_t* targets, const float* peer_lse, const float* peer_z, const float* loss,
                  const void* d_hidden, const float* d_w) {
  if (n < 0 || h <= 0 || v_t <= 0 || v0 < 0) return fail(L4D_EINVAL, "bad LM-head sizes");
  if (h % 8 || v_t % 8) return fail(L4D_EINVAL, "hidden and vocab shard must be multiples of 8");
  if (n * v_t > ((int64_t)1 << 40) || n > INT32_MAX || v_t > INT32_MAX) return fail(L4D_EINVAL, "problem too large");
  if (!hidden || !w_lm || !targets || !loss || !d_hidden || !d_w)
    return fail(L4D_EINVAL, "hidden, w_lm, targets, loss, d_hidden and d_w_lm are required");
  if ((peer_lse == nullptr) != (peer_z == nullptr))
    return fail(L4D_EINVAL, "peer_lse and peer_target_logit go together");
  return L4D_OK;
}

// The LM-head kernel sequence over `bytes` >= plan_lm(n, h, v_t).logits bytes of
// device workspace at ws (256-byte aligned; nothing in it needs to start at
// zero: every byte is written before it is read).
int lm_xent_run(int64_t n, int64_t h, int64_t v_t, int64_t v0, const void* hidden, const void* w_lm,
                const int64_t* targets, const float* peer_lse, const float* peer_z, float grad_scale, float* loss,
                void* d_hidden, float* d_w, uint8_t* ws, uint64_t bytes, hipStream_t s) {
  const LmWs plan = plan_lm(n, h, v_t);
  uint16_t* logits = reinterpret_cast<uint16_t*>(ws);
  float* partial = plan.splits > 1 && bytes >= plan.full ? reinterpret_cast<float*>(ws + plan.logits) : nullptr;
  int rc;
  if ((rc = run_gemm("gemm_lm_logits", s, n, v_t, h, op(RowSrc::plain(hidden, h), n), Layout::KC,
                     op(RowSrc::plain(w_lm, h), v_t), Layout::KC, epi_store(logits, v_t))))
    return rc;
  if ((rc = launch("xent_rows", s, [&] {
         return xent_rows(logits, n, (int32_t)v_t, v0, targets, peer_lse, peer_z, grad_scale, loss, logits, s);
       })))
    return rc;
  if ((rc = run_gemm("gemm_lm_dx", s, n, h, v_t, op(RowSrc::plain(logits, v_t), n), Layout::KC,
                     op(RowSrc::plain(w_lm, h), h), Layout::MN, epi_store(d_hidden, h), partial, plan.splits)))
    return rc;
  return run_gemm("gemm_lm_dw", s, v_t, h, n, op(RowSrc::plain(logits, v_t), v_t), Layout::MN,
                  op(RowSrc::plain(hidden, h), h), Layout::MN, epi_acc(d_w, h));
}

// Workspace of lm_head_xent_noalloc: one array per device, held by the loaded
// code object until the process ends.  Host code must use the address that
// hipGetSymbolAddress returns for the current device, never the array's name.
static __device__ __align__(256) uint8_t scratch[kScratchBytes];
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

// The current device's scratch address, resolved once per device.
int scratch_on_current_device(uint8_t** out) {
  int dev = -1;
  HIP_TRY(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return fail(L4D_EDEVICE, "device %d out of range", dev);
  std::lock_guard<std::mutex> lk(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    const hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess || !p)
      return fail(L4D_EDEVICE, "hipGetSymbolAddress(scratch) on device %d: %s", dev, hipGetErrorString(e));
    g_scratch_ptr[dev] = p;
  }
  *out = static_cast<uint8_t*>(g_scratch_ptr[dev]);
  return L4D_OK;
}
}  // namespace

extern "C" int lm_head_xent(int64_t n, int64_t h, int64_t v_t, int64_t v0, const void* hidden, const void* w_lm,
                            const int64_t* targets, const float* peer_lse, const float* peer_z, float grad_scale,
                            float* loss, void* d_hidden, float* d_w, l4d_arena* A, void* stream_ptr) {
  int rc = lm_xent_check(n, h, v_t, v0, hidden, w_lm, targets, peer_lse, peer_z, loss, d_hidden, d_w);
  if (rc) return rc;
  if (!A) return fail(L4D_EINVAL, "arena is required");
  if (n == 0) return L4D_OK;
  // an arena without room for the partials of d_hidden still runs the call, unsplit
  const LmWs plan = plan_lm(n, h, v_t);
  Workspace ws;
  ws.A = A;
  ws.size = plan.full;
  ws.held = arena_alloc(A, ws.size, &ws.off);
  if (!ws.held && (rc = take_ws(A, plan.logits, ws))) return rc;
  return lm_xent_run(n, h, v_t, v0, hidden, w_lm, targets, peer_lse, peer_z, grad_scale, loss, d_hidden, d_w,
                     reinterpret_cast<uint8_t*>(A->base + ws.off), ws.size, static_cast<hipStream_t>(stream_ptr));
}

extern "C" int lm_head_xent_noalloc(int64_t n, int64_t h, int64_t v_t, int64_t v0, const void* hidden,
                                    const void* w_lm, const int64_t* targets, const float* peer_lse,
                                    const float* peer_z, float grad_scale, float* loss, void* d_hidden, float* d_w,
                                    void* stream_ptr) {
  int rc = lm_xent_check(n, h, v_t, v0, hidden, w_lm, targets, peer_lse, peer_z, loss, d_hidden, d_w);
  if (rc) return rc;
  const uint64_t need = plan_lm(n, h, v_t).logits;
  if (need > kScratchBytes)
    return fail(L4D_EINVAL, "LM head needs %llu bytes of workspace; the static scratch holds %llu",
                (unsigned long long)need, (unsigned long long)kScratchBytes);
  if (n == 0) return L4D_OK;
  uint8_t* ws = nullptr;
  if ((rc = scratch_on_current_device(&ws))) return rc;
  return lm_xent_run(n, h, v_t, v0, hidden, w_lm, targets, peer_lse, peer_z, grad_scale, loss, d_hidden, d_w, ws,
                     kScratchBytes, static_cast<hipStream_t>(stream_ptr));
}

// ============================================================== the ends of the model

namespace {
bool same_shard(const Shard& a, const Shard& b) {
  return a.h == b.h && a.a == b.a && a.k == b.k && a.f == b.f && a.s == b.s && a.b == b.b && a.t == b.t &&
         a.c == b.c && a.tr == b.tr && a.cr == b.cr;
}

int check_ends_stash(l4d_arena* A, const l4d_stash* st, int kind, const Shard& x) {
  if (!st || !A) return fail(L4D_EINVAL, "stash and arena are required");
  if (st->arena != A || !A->live.count(st)) return fail(L4D_EINVAL, "stash does not belong to this arena");
  if (st->kind != kind) return fail(L4D_EINVAL, kind == kHeadStash ? "not an LM-head stash" : "not an embedding stash");
  if (!same_shard(st->shape, x)) return fail(L4D_EINVAL, "stash was made for another shape");
  return L4D_OK;
}

// Vocabulary shard of this TP rank; v % t and (v/t) % 8 are required.
int vocab_shard(const l4d_model* m, const Shard& x, int64_t* v_t, int64_t* v0) {
  if (m->vocab % x.t) return fail(L4D_EINVAL, "vocab %% tp != 0");
  *v_t = m->vocab / x.t;
  if (*v_t % 8) return fail(L4D_EINVAL, "vocab / tp must be a multiple of 8");
  if ((int64_t)x.b * x.s_c * *v_t > ((int64_t)1 << 40)) return fail(L4D_EINVAL, "problem too large");
  *v0 = x.tr * *v_t;
  return L4D_OK;
}
}  // namespace

extern "C" int embedding_fwd(const l4d_model* m, const l4d_parallel* p, const int64_t* ids, const void* w_emb,
                             const void* receipt, void* send, void* x_out, l4d_arena* A, l4d_stash** stash_out,
                             void* stream_ptr) {
  Shard x;
  int rc = make_shard(m, p, &x);
  if (rc) return rc;
  int64_t v_t, v0;
  if ((rc = vocab_shard(m, x, &v_t, &v0))) return rc;
  if (!ids || !w_emb || !x_out || !A || !stash_out) return fail(L4D_EINVAL, "ids, w_emb, x_out, arena and stash_out are required");
  if ((x.t > 1) != (send != nullptr)) return fail(L4D_EINVAL, "send is required iff tp > 1");
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  const uint64_t bytes[1] = {(uint64_t)x.b * x.s_c * 8};
  l4d_stash* st = nullptr;
  if ((rc = stash_reserve_sized(A, x, kEmbStash, L4D_EMB_COUNT, bytes, -1, &st))) return rc;
  auto body = [&]() -> int {
    return launch("embed_fwd", s, [&] {
      return embed_fwd(ids, static_cast<const uint16_t*>(w_emb), v0, (int32_t)v_t, (int32_t)x.h, x.b * x.s_c,
                       (int32_t)x.s_c, (int32_t)x.s_sp, (int32_t)x.tr, (int32_t)x.t,
                       static_cast<const uint16_t*>(receipt), static_cast<uint16_t*>(x_out),
                       static_cast<uint16_t*>(send), sptr<int64_t>(st, L4D_EMB_IDS), s);
    });
  };
  if ((rc = body())) {
    l4d_stash_release(A, st);
    return rc;
  }
  *stash_out = st;
  return L4D_OK;
}

extern "C" int embedding_bwd(const l4d_model* m, const l4d_parallel* p, l4d_stash* st, const void* dx,
                             const void* peer_dx, float* d_w_emb, l4d_arena* A, void* stream_ptr) {
  Shard x;
  int rc = make_shard(m, p, &x);
  if (rc) return rc;
  int64_t v_t, v0;
  if ((rc = vocab_shard(m, x, &v_t, &v0))) return rc;
  if ((rc = check_ends_stash(A, st, kEmbStash, x))) return rc;
  if (!dx || !d_w_emb) return fail(L4D_EINVAL, "dx and d_w_emb are required");
  if ((x.t > 1) != (peer_dx != nullptr)) return fail(L4D_EINVAL, "peer_dx is required iff tp > 1");
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  // the sorted tokens; an arena without room for them still runs the call, unsorted
  Workspace ws;
  ws.A = A;
  ws.size = align_up(embed_bwd_ws_bytes(x.b * x.s_c, (int32_t)x.h, (int32_t)x.t));
  ws.held = ws.size && arena_alloc(A, ws.size, &ws.off);
  uint64_t* keys = ws.held ? reinterpret_cast<uint64_t*>(A->base + ws.off) : nullptr;
  if ((rc = launch("embed_bwd", s, [&] {
         return embed_bwd(sptr<const int64_t>(st, L4D_EMB_IDS), keys, gathered(dx, peer_dx, x), v0, (int32_t)v_t,
                          (int32_t)x.h, x.b * x.s_c, d_w_emb, s);
       })))
    return rc;
  return l4d_stash_release(A, st);
}

extern "C" int lm_head_fwd(const l4d_model* m, const l4d_parallel* p, const void* x_in, const void* w_norm,
                           const void* w_lm, const int64_t* targets, const void* peer_xn, const float* peer_lse,
                           const float* peer_z, float* loss, l4d_arena* A, l4d_stash** stash_out, void* stream_ptr) {
  Shard x;
  int rc = make_shard(m, p, &x);
  if (rc) return rc;
  int64_t v_t, v0;
  if ((rc = vocab_shard(m, x, &v_t, &v0))) return rc;
  if (!x_in || !w_norm || !w_lm || !targets || !loss || !A || !stash_out)
    return fail(L4D_EINVAL, "x, w_norm, w_lm, targets, loss, arena and stash_out are required");
  if (x.t > 1 && (!peer_xn || !peer_lse || !peer_z))
    return fail(L4D_EINVAL, "tp > 1 needs peer_xn, peer_lse and peer_target_logit");
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  const int64_t tok = x.b * x.s_c;
  const uint64_t sp = (uint64_t)x.b * x.s_sp * x.h * 2;
  const uint64_t bytes[L4D_HEAD_COUNT] = {sp, sp, (uint64_t)tok * v_t * 4};
  l4d_stash* st = nullptr;
  if ((rc = stash_reserve_sized(A, x, kHeadStash, L4D_HEAD_COUNT, bytes, -1, &st))) return rc;
  auto body = [&]() -> int {
    int r;
    if ((r = launch("rmsnorm_fwd", s, [&] {
           return rmsnorm_fwd(static_cast<const uint16_t*>(x_in), static_cast<const uint16_t*>(w_norm),
                              sptr(st, L4D_HEAD_XN), x.b * x.s_sp, (int32_t)x.h, x.eps, s, sptr(st, L4D_HEAD_X));
         })))
      return r;
    EpiParams e{};
    e.kind = EpiKind::StoreF32;
    e.c = sptr<float>(st, L4D_HEAD_PROBS);
    e.ldc = v_t;
    if ((r = run_gemm("gemm_head_logits", s, tok, v_t, x.h, op(gathered(sptr(st, L4D_HEAD_XN), peer_xn, x), tok),
                      Layout::KC, op(RowSrc::plain(w_lm, x.h), v_t), Layout::KC, e)))
      return r;
    return launch("xent_probs", s, [&] {
      return xent_probs(sptr<float>(st, L4D_HEAD_PROBS), tok, (int32_t)v_t, v0, targets, peer_lse, peer_z, loss, s);
    });
  };
  if ((rc = body())) {
    l4d_stash_release(A, st);
    return rc;
  }
  *stash_out = st;
  return L4D_OK;
}

extern "C" int lm_head_bwd(const l4d_model* m, const l4d_parallel* p, const void* w_norm, const void* w_lm,
                           const int64_t* targets, const void* peer_xn, const void* peer_dxn, void* dxn_send,
                           float grad_scale, l4d_stash* st, void* dx, float* d_w_norm, float* d_w_lm, l4d_arena* A,
                           void* stream_ptr) {
  Shard x;
  int rc = make_shard(m, p, &x);
  if (rc) return rc;
  int64_t v_t, v0;
  if ((rc = vocab_shard(m, x, &v_t, &v0))) return rc;
  if ((rc = check_ends_stash(A, st, kHeadStash, x))) return rc;
  if (!w_norm || !w_lm || !targets || !dx || !d_w_norm || !d_w_lm)
    return fail(L4D_EINVAL, "w_norm, w_lm, targets, dx, d_w_norm and d_w_lm are required");
  if (x.t > 1 && !peer_xn) return fail(L4D_EINVAL, "tp > 1 needs peer_xn");
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  const int64_t tok = x.b * x.s_c, rows_sp = x.b * x.s_sp;
  const int32_t npart = rmsnorm_bwd_partials(rows_sp);
  Carver cv;
  const uint64_t o_dl = cv.take((uint64_t)tok * v_t * 2), o_dxn = cv.take((uint64_t)rows_sp * x.h * 2);
  const uint64_t o_part = cv.take((uint64_t)npart * x.h * 4);
  const uint64_t o_send = (x.t > 1 && !dxn_send) ? cv.take((uint64_t)x.b * (x.t - 1) * x.s_sp * x.h * 2) : 0;
  Workspace ws;
  if ((rc = take_ws(A, cv.used, ws))) return rc;
  uint8_t* wsb = reinterpret_cast<uint8_t*>(A->base + ws.off);
  uint16_t* dl = reinterpret_cast<uint16_t*>(wsb + o_dl);
  uint16_t* dxn = reinterpret_cast<uint16_t*>(wsb + o_dxn);
  float* partial = reinterpret_cast<float*>(wsb + o_part);
  void* send = x.t > 1 ? (dxn_send ? dxn_send : (void*)(wsb + o_send)) : nullptr;
  if ((rc = launch("xent_grad", s, [&] {
         return xent_grad(sptr<const float>(st, L4D_HEAD_PROBS), tok, (int32_t)v_t, v0, targets, grad_scale, dl, s);
       })))
    return rc;
  // d(xn) over the gathered rows: own rows + the peers' partials, the peers' rows sent
  if ((rc = run_gemm("gemm_head_dx", s, tok, x.h, v_t, op(RowSrc::plain(dl, v_t), tok), Layout::KC,
                     op(RowSrc::plain(w_lm, x.h), x.h), Layout::MN, epi_residual(x, dxn, nullptr, peer_dxn, send))))
    return rc;
  if ((rc = launch("rmsnorm_bwd", s, [&] {
         const NormBwdIo io{dxn, nullptr, nullptr, nullptr, static_cast<uint16_t*>(dx), nullptr};
         return rmsnorm_bwd(sptr(st, L4D_HEAD_X), static_cast<const uint16_t*>(w_norm), io, partial, npart,
                            rows_sp, (int32_t)x.h, x.eps, s);
       })))
    return rc;
  if ((rc = launch("reduce_gain", s, [&] { return reduce_rows_add(partial, npart, (int32_t)x.h, d_w_norm, s); })))
    return rc;
  if ((rc = run_gemm("gemm_head_dw", s, v_t, x.h, tok, op(RowSrc::plain(dl, v_t), v_t), Layout::MN,
                     op(gathered(sptr(st, L4D_HEAD_XN), peer_xn, x), x.h), Layout::MN, epi_acc(d_w_lm, x.h))))
    return rc;
  return l4d_stash_release(A, st);
}

// ============================================================== packed documents

extern "C" int rope_fwd(const l4d_rope* r, int dtype, int64_t tokens, const l4d_packing* pk, const int64_t* positions,
                        const l4d_rope_heads* q, const l4d_rope_heads* k, void* stream_ptr) {
  return rope_call("rope_fwd", r, nullptr, dtype, tokens, pk, positions, q, k, 0, stream_ptr);
}

extern "C" int rope_bwd(const l4d_rope* r, int dtype, int64_t tokens, const l4d_packing* pk, const int64_t* positions,
                        const l4d_rope_heads* q, const l4d_rope_heads* k, void* stream_ptr) {
  return rope_call("rope_bwd", r, nullptr, dtype, tokens, pk, positions, q, k, 1, stream_ptr);
}

extern "C" int rope_axes_fwd(const l4d_rope* r, const l4d_rope_axes* axes, int dtype, int64_t tokens, const l4d_packing* pk,
                             const int64_t* positions, const l4d_rope_heads* q, const l4d_rope_heads* k, void* stream_ptr) {
  if (!axes) return fail(L4D_EINVAL, "axes is required");
  return rope_call("rope_axes_fwd", r, axes, dtype, tokens, pk, positions, q, k, 0, stream_ptr);
}
extern "C" int rope_axes_bwd(const l4d_rope* r, const l4d_rope_axes* axes, int dtype, int64_t tokens, const l4d_packing* pk,
                             const int64_t* positions, const l4d_rope_heads* q, const l4d_rope_heads* k, void* stream_ptr) {
  if (!axes) return fail(L4D_EINVAL, "axes is required");
  return rope_call("rope_axes_bwd", r, axes, dtype, tokens, pk, positions, q, k, 1, stream_ptr);
}

// ------------------------------------------------------------ norm and rotation of heads

extern "C" int qk_norm_rope_fwd(const l4d_rope* r, const l4d_rope_axes* axes, int dtype, int64_t tokens,
                                const l4d_packing* pk, const int64_t* positions, float eps, const l4d_norm_heads* q,
                                const l4d_norm_heads* k, void* stream_ptr) {
  if (!q) return fail(L4D_EINVAL, "q is required");
  NormTensor t[2];
  int n = 0;
  for (const l4d_norm_heads* h : {q, k})
    if (h) t[n++] = NormTensor{h->x, nullptr, h->y, h->gain, nullptr, h->heads, h->x_ld, 0, h->y_ld};
  return norm_call("qk_norm_rope_fwd", r, axes, dtype, tokens, pk, positions, eps, t, n, false, nullptr, stream_ptr);
}
extern "C" int l4d_qk_norm_workspace_bytes(int64_t tokens, int64_t head_dim, uint64_t* bytes) {
  if (tokens < 0 || tokens > kMaxRopeRows) return fail(L4D_EINVAL, "rope: tokens must lie in 0 .. 2^25");
  if (head_dim < 2 || head_dim > 2 * kMaxRopePairs) return fail(L4D_EINVAL, "rope: head_dim must lie in 2 .. 512");
  if (bytes) *bytes = align_up((uint64_t)qk_norm_parts(tokens) * 2 * head_dim * 4);
  return L4D_OK;
}
extern "C" int qk_norm_rope_bwd(const l4d_rope* r, const l4d_rope_axes* axes, int dtype, int64_t tokens,
                                const l4d_packing* pk, const int64_t* positions, float eps, const l4d_norm_heads_grad* q,
                                const l4d_norm_heads_grad* k, l4d_arena* A, void* stream_ptr) {
  if (!q) return fail(L4D_EINVAL, "q is required");
  NormTensor t[2];
  int n = 0;
  for (const l4d_norm_heads_grad* h : {q, k})
    if (h) t[n++] = NormTensor{h->x, h->dy, h->dx, h->gain, h->d_gain, h->heads, h->x_ld, h->dy_ld, h->dx_ld};
  return norm_call("qk_norm_rope_bwd", r, axes, dtype, tokens, pk, positions, eps, t, n, true, A, stream_ptr);
}

// ------------------------------------------------------------ dropout and residual

extern "C" int dropout_add_fwd(int dtype, int64_t rows, int64_t cols, const void* x, int64_t x_ld, const void* residual,
                               int64_t residual_ld, void* y, int64_t y_ld, double p, const int64_t* rng, int64_t first_row,
                               void* stream_ptr) {
  return dropout_call("dropout_add_fwd", dtype, rows, cols, x, x_ld, residual, residual_ld, y, y_ld, p, rng, first_row,
                      stream_ptr);
}
extern "C" int dropout_add_bwd(int dtype, int64_t rows, int64_t cols, const void* dy, int64_t dy_ld, void* dx, int64_t dx_ld,
                               double p, const int64_t* rng, int64_t first_row, void* stream_ptr) {
  return dropout_call("dropout_add_bwd", dtype, rows, cols, dy, dy_ld, nullptr, 0, dx, dx_ld, p, rng, first_row, stream_ptr);
}

// ------------------------------------------------------------ packed attention

extern "C" int l4d_attn_packed_workspace_bytes(const l4d_attn* at, int64_t tokens, uint64_t* bytes) {
  if (tokens < 0 || tokens > (int64_t)1 << 30) return fail(L4D_EINVAL, "tokens must lie in 0 .. 2^30");
  WindowAttn p{};
  int rc = attn_shape(at, &p);
  if (rc) return rc;
  if (bytes) *bytes = align_up(plan_packed(p, tokens).total);
  return L4D_OK;
}
extern "C" int l4d_attn_window_workspace_bytes(const l4d_window* w, const l4d_attn* at, int64_t tokens, uint64_t* bytes) {
  if (tokens < 0 || tokens > (int64_t)1 << 30) return fail(L4D_EINVAL, "tokens must lie in 0 .. 2^30");
  WindowAttn p{};
  int rc;
  if ((rc = attn_shape(at, &p)) || (rc = attn_window(w, tokens, &p))) return rc;
  if (bytes) *bytes = align_up(plan_packed(p, tokens).total);
  return L4D_OK;
}

// With windowed: attention within w.
static int attn_forward(bool windowed, const l4d_window* w, const l4d_attn* at, const l4d_packing* pk, const void* q,
                        int64_t q_ld, const void* k, int64_t k_ld, const void* v, int64_t v_ld, void* o, int64_t o_ld,
                        float* lse, void* stream_ptr) {
  int rc = check_packing(pk);
  if (rc) return rc;
  WindowAttn p{};
  if ((rc = attn_shape(at, &p))) return rc;
  if (windowed && (rc = attn_window(w, pk->tokens, &p))) return rc;
  if (pk->tokens == 0) return L4D_OK;                // an empty array may have no address
  const AttnRows t[4] = {{"q", q, q_ld, at->n_heads}, {"k", k, k_ld, at->n_kv_heads}, {"v", v, v_ld, at->n_kv_heads},
                         {"o", o, o_ld, at->n_heads}};
  if ((rc = attn_rows(t, 4, at->head_dim)) || (rc = attn_distinct(t, 4, 3))) return rc;
  if (!lse || reinterpret_cast<uintptr_t>(lse) % 4) return fail(L4D_EINVAL, "lse is required, 4-byte aligned");
  p.pk = device_packing(pk);
  if (p.window ? !attn_window_fits(p) : !attn_packed_fits(p)) return fail(L4D_EINVAL, "problem too large");
  if ((rc = attn_apart(t, 4, 3, at, lse, pk))) return rc;
  if (pk->n_seqs == 0) return L4D_OK;
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.o = static_cast<uint16_t*>(o);
  p.q_ld = q_ld, p.k_ld = k_ld, p.v_ld = v_ld, p.o_ld = o_ld;
  p.lse = lse;
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  if (p.window) return launch("attn_window_fwd", s, [&] { return attn_window_fwd(p, s); });
  return launch("attn_packed_fwd", s, [&] { return attn_packed_fwd(p, s); });
}

extern "C" int attn_packed_fwd(const l4d_attn* at, const l4d_packing* pk, const void* q, int64_t q_ld, const void* k,
                               int64_t k_ld, const void* v, int64_t v_ld, void* o, int64_t o_ld, float* lse,
                               void* stream_ptr) {
  return attn_forward(false, nullptr, at, pk, q, q_ld, k, k_ld, v, v_ld, o, o_ld, lse, stream_ptr);
}
extern "C" int attn_window_fwd(const l4d_window* w, const l4d_attn* at, const l4d_packing* pk, const void* q, int64_t q_ld,
                               const void* k, int64_t k_ld, const void* v, int64_t v_ld, void* o, int64_t o_ld, float* lse,
                               void* stream_ptr) {
  return attn_forward(true, w, at, pk, q, q_ld, k, k_ld, v, v_ld, o, o_ld, lse, stream_ptr);
}

static int attn_backward(bool windowed, const l4d_window* w, const l4d_attn* at, const l4d_packing* pk, const void* q,
                         int64_t q_ld, const void* k, int64_t k_ld, const void* v, int64_t v_ld, const void* o, int64_t o_ld,
                         const float* lse, const void* d_o, int64_t do_ld, void* dq, int64_t dq_ld, void* dk, int64_t dk_ld,
                         void* dv, int64_t dv_ld, l4d_arena* A, void* stream_ptr) {
  int rc = check_packing(pk);
  if (rc) return rc;
  WindowAttn p{};
  if ((rc = attn_shape(at, &p))) return rc;
  if (windowed && (rc = attn_window(w, pk->tokens, &p))) return rc;
  if (pk->tokens == 0) return L4D_OK;                // an empty array may have no address
  const int64_t a = at->n_heads, g = at->n_kv_heads;
  const AttnRows t[8] = {{"q", q, q_ld, a}, {"k", k, k_ld, g}, {"v", v, v_ld, g}, {"o", o, o_ld, a},
                         {"d_o", d_o, do_ld, a}, {"dq", dq, dq_ld, a}, {"dk", dk, dk_ld, g}, {"dv", dv, dv_ld, g}};
  if ((rc = attn_rows(t, 8, at->head_dim)) || (rc = attn_distinct(t, 8, 5))) return rc;
  if (!lse || reinterpret_cast<uintptr_t>(lse) % 4) return fail(L4D_EINVAL, "lse is required, 4-byte aligned");
  if (!A) return fail(L4D_EINVAL, "arena is required");
  p.pk = device_packing(pk);
  if (p.window ? !attn_window_fits(p) : !attn_packed_fits(p)) return fail(L4D_EINVAL, "problem too large");
  if ((rc = attn_apart(t, 8, 5, at, lse, pk))) return rc;
  if (pk->n_seqs == 0) return L4D_OK;
  const PackedWs plan = plan_packed(p, pk->tokens);
  Workspace ws;
  if ((rc = take_ws(A, plan.total, ws))) return rc;
  uint8_t* wsb = reinterpret_cast<uint8_t*>(A->base + ws.off);
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.o = static_cast<uint16_t*>(const_cast<void*>(o));
  p.lse = const_cast<float*>(lse);
  p.dout = static_cast<const uint16_t*>(d_o);
  p.dq = static_cast<uint16_t*>(dq);
  p.dk = static_cast<uint16_t*>(dk);
  p.dv = static_cast<uint16_t*>(dv);
  p.q_ld = q_ld, p.k_ld = k_ld, p.v_ld = v_ld, p.o_ld = o_ld, p.do_ld = do_ld;
  p.dq_ld = dq_ld, p.dk_ld = dk_ld, p.dv_ld = dv_ld;
  p.delta = reinterpret_cast<float*>(wsb + plan.delta);
  p.lse2 = reinterpret_cast<float*>(wsb + plan.lse2);
  p.items = reinterpret_cast<int32_t*>(wsb + plan.items);
  p.dkv_partial = reinterpret_cast<float*>(wsb + plan.partial);
  p.sink_partial = reinterpret_cast<float*>(wsb + plan.sinks);
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  if (p.window) {
    attn_window_plan(&p);
    return window_attn_backward(p, s);
  }
  attn_packed_plan(&p);
  return packed_attn_backward(p, s);
}

extern "C" int attn_packed_bwd(const l4d_attn* at, const l4d_packing* pk, const void* q, int64_t q_ld, const void* k,
                               int64_t k_ld, const void* v, int64_t v_ld, const void* o, int64_t o_ld, const float* lse,
                               const void* d_o, int64_t do_ld, void* dq, int64_t dq_ld, void* dk, int64_t dk_ld, void* dv,
                               int64_t dv_ld, l4d_arena* A, void* stream_ptr) {
  return attn_backward(false, nullptr, at, pk, q, q_ld, k, k_ld, v, v_ld, o, o_ld, lse, d_o, do_ld, dq, dq_ld, dk, dk_ld, dv,
                       dv_ld, A, stream_ptr);
}
extern "C" int attn_window_bwd(const l4d_window* w, const l4d_attn* at, const l4d_packing* pk, const void* q, int64_t q_ld,
                               const void* k, int64_t k_ld, const void* v, int64_t v_ld, const void* o, int64_t o_ld,
                               const float* lse, const void* d_o, int64_t do_ld, void* dq, int64_t dq_ld, void* dk,
                               int64_t dk_ld, void* dv, int64_t dv_ld, l4d_arena* A, void* stream_ptr) {
  return attn_backward(true, w, at, pk, q, q_ld, k, k_ld, v, v_ld, o, o_ld, lse, d_o, do_ld, dq, dq_ld, dk, dk_ld, dv, dv_ld,
                       A, stream_ptr);
}

// ============================================================== loss without stored logits

namespace {
// Columns of a piece of the vocabulary: forward (its statistics: 8 bytes for 64
// columns) and backward (its gradient: 4 bytes a column).  More tokens take fewer
// columns, down to 8192: narrower pieces leave d_w's product too few tiles and add
// fp32 d_hidden once more each (forward and backward with pieces of 4096, 8192, 32768
// columns: 8192 tokens, hidden 4096, 32064 columns 9.09, 8.92, 9.00 ms; 32768 tokens,
// hidden 2048, 32000 columns 21.8, 19.2, 19.1; 2048 tokens, 128256 columns 11.0, 10.2, 9.5).
int64_t loss_piece_cols(int64_t n, int64_t v_t, int64_t least, int64_t elements) {
  const int64_t cols = std::max(least, elements / std::max<int64_t>(n, 1) / 256 * 256);
  return std::min(cols, (v_t + 7) / 8 * 8);
}
struct LossWs {
  int64_t fwd_piece, bwd_piece;                      // columns
  uint64_t stats, zt, run, fwd;                      // forward: offsets and total
  uint64_t g, dh, gt, rep, part, bwd;                // backward: g [parts][n][bwd_piece], rep = hidden once per part
  int parts, dx_splits;                              // bf16 parts of G; parts of the K range of G W
};
// Bf16 parts of G in the product with hidden: two leave 2.4e-6 (rms) of an element and,
// with the targets' elements completed, 1e-7 to 1e-6 of d_w.  A shard that holds
// no token's target has only the small elements; with few tokens that happens, and
// there the product is bound by d_w's own traffic: the third part costs nothing.
constexpr int64_t kThreeParts = 256;
constexpr int kDxSplits = 8;
LossWs plan_loss(int64_t n, int64_t h, int64_t v_t) {
  LossWs w{};
  w.fwd_piece = loss_piece_cols(n, v_t, 65536, (int64_t)1 << 31);
  w.bwd_piece = loss_piece_cols(n, v_t, 8192, (int64_t)1 << 26);
  w.parts = n <= kThreeParts ? 3 : 2;
  const GemmPlan dx = gemm_plan(n, h, std::min(w.bwd_piece, v_t), EpiKind::AccF32, kDxSplits);
  w.dx_splits = dx.splits;
  Carver f, b;
  w.stats = f.take((uint64_t)n * ((w.fwd_piece + 255) / 256 * 4) * 8);
  w.zt = f.take((uint64_t)n * 4);
  w.run = f.take((uint64_t)n * 8);
  w.fwd = f.used;
  w.g = b.take((uint64_t)n * w.bwd_piece * 2 * w.parts);
  w.dh = b.take((uint64_t)n * h * 4);
  w.gt = b.take((uint64_t)n * 4);
  w.rep = b.take((uint64_t)n * h * 2 * w.parts);
  w.part = b.take((uint64_t)n * h * 4 * (w.dx_splits - 1));
  w.bwd = b.used;
  return w;
}
// rows: arrays of bf16 rows; words: the others, which need no more than their element's alignment (4 or 8 bytes)
int loss_check(int64_t n, int64_t h, int64_t v_t, int64_t v0, std::initializer_list<const void*> rows,
               std::initializer_list<const void*> words, const int64_t* targets) {
  if (n < 0 || h <= 0 || v_t <= 0 || v0 < 0 || v0 > INT64_MAX - v_t) return fail(L4D_EINVAL, "bad LM-head sizes");
  if (h % 8 || h > 8192) return fail(L4D_EINVAL, "hidden must be a multiple of 8 and at most 8192");
  if (n > (int64_t)1 << 20 || v_t > (int64_t)1 << 24) return fail(L4D_EINVAL, "problem too large");   // grid sizes
  for (const void* p : rows)
    if (!p || reinterpret_cast<uintptr_t>(p) % 16)
      return fail(L4D_EINVAL, "hidden, w_lm and d_hidden are required, 16-byte aligned");
  for (const void* p : words)
    if (!p || reinterpret_cast<uintptr_t>(p) % 4) return fail(L4D_EINVAL, "loss, lse and d_w_lm are required, 4-byte aligned");
  if (words.size() && (!targets || reinterpret_cast<uintptr_t>(targets) % 8))
    return fail(L4D_EINVAL, "targets is required, 8-byte aligned");
  return L4D_OK;
}
// The product of the logits of `cols` columns from row w of the head, with epilogue e.
int loss_logits(int64_t n, int64_t h, const void* hidden, const uint16_t* w, int64_t cols, const EpiParams& e, hipStream_t s) {
  return run_gemm(e.kind == EpiKind::LossStats ? "gemm_loss_stats" : "gemm_loss_grad", s, n, cols, h,
                  op(RowSrc::plain(hidden, h), n), Layout::KC, op(RowSrc::plain(w, h), cols), Layout::KC, e);
}
}  // namespace

extern "C" int l4d_lm_loss_workspace_bytes(int64_t n, int64_t h, int64_t v_t, uint64_t* fwd, uint64_t* bwd) {
  int rc = loss_check(n, h, v_t, 0, {}, {}, nullptr);
  if (rc) return rc;
  const LossWs w = plan_loss(n, h, v_t);
  if (fwd) *fwd = align_up(w.fwd);
  if (bwd) *bwd = align_up(w.bwd);
  return L4D_OK;
}

extern "C" int lm_loss_fwd(int64_t n, int64_t h, int64_t v_t, int64_t v0, const void* hidden, const void* w_lm,
                           const int64_t* targets, const float* peer_lse, const float* peer_z, float* loss, float* lse,
                           float* target_logit, l4d_arena* A, void* stream_ptr) {
  int rc = loss_check(n, h, v_t, v0, {hidden, w_lm}, {loss, lse}, targets);
  if (rc) return rc;
  if ((peer_lse == nullptr) != (peer_z == nullptr)) return fail(L4D_EINVAL, "peer_lse and peer_target_logit go together");
  if (!A) return fail(L4D_EINVAL, "arena is required");
  if (n == 0) return L4D_OK;
  const LossWs plan = plan_loss(n, h, v_t);
  Workspace ws;
  if ((rc = take_ws(A, plan.fwd, ws))) return rc;
  uint8_t* wsb = reinterpret_cast<uint8_t*>(A->base + ws.off);
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  LossJoin j{};
  j.stats = reinterpret_cast<float2*>(wsb + plan.stats);
  j.run = reinterpret_cast<float2*>(wsb + plan.run);
  j.zt = reinterpret_cast<float*>(wsb + plan.zt);
  j.n = n, j.v0 = v0, j.v_t = v_t;
  j.targets = targets;
  j.peer_lse = peer_lse, j.peer_z = peer_z;
  j.loss = loss, j.lse = lse, j.target_logit = target_logit;
  EpiParams e{};
  e.kind = EpiKind::LossStats;
  e.targets = targets;
  e.stats = reinterpret_cast<float2*>(wsb + plan.stats);
  e.zt = reinterpret_cast<float*>(wsb + plan.zt);
  for (int64_t c0 = 0; c0 < v_t; c0 += plan.fwd_piece) {
    const int64_t cols = std::min(plan.fwd_piece, v_t - c0);
    e.v0 = v0 + c0;
    if ((rc = loss_logits(n, h, hidden, static_cast<const uint16_t*>(w_lm) + c0 * h, cols, e, s))) return rc;
    j.n_blocks = (int32_t)loss_stat_blocks(cols, gemm_plan(n, cols, h, e.kind, 1).tile);
    j.first = c0 == 0;
    j.last = c0 + cols == v_t;
    if ((rc = launch("loss_join", s, [&] { return loss_join(j, s); }))) return rc;
  }
  return L4D_OK;
}

extern "C" int lm_loss_bwd(int64_t n, int64_t h, int64_t v_t, int64_t v0, const void* hidden, const void* w_lm,
                           const int64_t* targets, const float* lse, const float* d_loss, float grad_scale,
                           void* d_hidden, float* d_w, l4d_arena* A, void* stream_ptr) {
  int rc = loss_check(n, h, v_t, v0, {hidden, w_lm, d_hidden}, {lse, d_w}, targets);
  if (rc) return rc;
  if (!std::isfinite(grad_scale)) return fail(L4D_EINVAL, "grad_scale must be finite");
  if (d_hidden == hidden || d_hidden == w_lm) return fail(L4D_EINVAL, "d_hidden is an input's array");
  if (!A) return fail(L4D_EINVAL, "arena is required");
  if (n == 0) return L4D_OK;
  const LossWs plan = plan_loss(n, h, v_t);
  Workspace ws;
  if ((rc = take_ws(A, plan.bwd, ws))) return rc;
  uint8_t* wsb = reinterpret_cast<uint8_t*>(A->base + ws.off);
  const int64_t ld = plan.bwd_piece;
  float *dh = reinterpret_cast<float*>(wsb + plan.dh), *gt = reinterpret_cast<float*>(wsb + plan.gt);
  uint16_t* g = reinterpret_cast<uint16_t*>(wsb + plan.g);
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  EpiParams e{};
  e.kind = EpiKind::LossGrad;
  e.targets = targets;
  e.lse = lse;
  e.d_loss = d_loss;
  e.grad_scale = grad_scale;
  e.zt = gt;
  e.g = g;
  e.g_parts = plan.parts;
  e.ldc = ld;
  EpiParams store{};           // dh of the first piece: an fp32 store, unless its K range is cut
  store.kind = EpiKind::ResidualSP;
  store.ldc = h;
  store.own_out_f32 = dh;
  store.t = 1;
  uint16_t* rep = reinterpret_cast<uint16_t*>(wsb + plan.rep);
  float* part = reinterpret_cast<float*>(wsb + plan.part);
  const bool split = plan.dx_splits > 1;
  if (split && (rc = launch("loss_zero_dh", s, [&] { return zero_f32(dh, n * h, s); }))) return rc;
  // G^T hidden runs over parts x n rows: one part of G after another, hidden again for each
  if ((rc = launch("loss_repeat", s, [&] {
         return repeat_bf16(static_cast<const uint16_t*>(hidden), rep, n * h, plan.parts, s);
       })))
    return rc;
  for (int64_t c0 = 0; c0 < v_t; c0 += ld) {
    const int64_t cols = std::min(ld, v_t - c0);
    const uint16_t* w = static_cast<const uint16_t*>(w_lm) + c0 * h;
    e.v0 = v0 + c0;
    if ((rc = loss_logits(n, h, hidden, w, cols, e, s))) return rc;
    if ((rc = run_gemm("gemm_loss_dx", s, n, h, cols, op(RowSrc::plain(g, ld), n), Layout::KC, op(RowSrc::plain(w, h), h),
                       Layout::MN, c0 == 0 && !split ? store : epi_acc(dh, h), split ? part : nullptr,
                       split ? plan.dx_splits : 0)))
      return rc;
    if ((rc = run_gemm("gemm_loss_dw", s, cols, h, plan.parts * n, op(RowSrc::plain(g, ld), (cols + 7) / 8 * 8), Layout::MN,
                       op(RowSrc::plain(rep, h), h), Layout::MN, epi_acc(d_w + c0 * h, h))))
      return rc;
  }
  const LossTargets t{n, v0, v_t, (int32_t)h, targets, gt, plan.parts, dh, static_cast<const uint16_t*>(hidden),
                      static_cast<const uint16_t*>(w_lm), static_cast<uint16_t*>(d_hidden), d_w};
  return launch("loss_finish_grad", s, [&] { return loss_finish_grad(t, s); });
}

// ============================================================== optimizer

extern "C" int l4d_adam_step(const l4d_adam* hp, int64_t n, float* grad, float* master, float* m, float* v,
                             void* weight, void* stream_ptr) {
  if (!hp) return fail(L4D_EINVAL, "hyperparameters are required");
  if (n < 0) return fail(L4D_EINVAL, "n must be >= 0");
  if (hp->step < 1) return fail(L4D_EINVAL, "step counts from 1");
  if (!(hp->beta1 >= 0.f && hp->beta1 < 1.f) || !(hp->beta2 >= 0.f && hp->beta2 < 1.f))
    return fail(L4D_EINVAL, "beta1 and beta2 must lie in [0, 1)");
  if (!(hp->eps >= 0.f) || !std::isfinite(hp->eps)) return fail(L4D_EINVAL, "eps must be finite and >= 0");
  if (!std::isfinite(hp->lr) || !std::isfinite(hp->weight_decay) || !std::isfinite(hp->grad_scale))
    return fail(L4D_EINVAL, "lr, weight_decay and grad_scale must be finite");
  if (!grad || !master || !m || !v || !weight) return fail(L4D_EINVAL, "grad, master, m, v and weight are required");
  const void* f32s[4] = {grad, master, m, v};
  for (const void* p : f32s)
    if (reinterpret_cast<uintptr_t>(p) % 16) return fail(L4D_EINVAL, "fp32 arrays must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(weight) % 8) return fail(L4D_EINVAL, "the weight must be 8-byte aligned");
  if (n == 0) return L4D_OK;
  if (n > (int64_t(1) << 33)) return fail(L4D_EINVAL, "shard too large (more than 2^33 parameters)");
  const uintptr_t lo[5] = {(uintptr_t)grad, (uintptr_t)master, (uintptr_t)m, (uintptr_t)v, (uintptr_t)weight};
  const uint64_t len[5] = {4ull * n, 4ull * n, 4ull * n, 4ull * n, 2ull * n};
  for (int i = 0; i < 5; ++i)
    for (int j = i + 1; j < 5; ++j)
      if (lo[i] < lo[j] + len[j] && lo[j] < lo[i] + len[i]) return fail(L4D_EINVAL, "the arrays overlap");
  const double b1 = hp->beta1, b2 = hp->beta2, t = static_cast<double>(hp->step);
  AdamConsts c;
  c.beta1 = hp->beta1;
  c.beta2 = hp->beta2;
  c.one_m_beta1 = static_cast<float>(1.0 - b1);
  c.one_m_beta2 = static_cast<float>(1.0 - b2);
  c.lr = hp->lr;
  c.decay = static_cast<float>(static_cast<double>(hp->lr) * hp->weight_decay);
  c.r1 = static_cast<float>(1.0 / -std::expm1(t * std::log(b1)));
  c.rs2 = static_cast<float>(1.0 / std::sqrt(-std::expm1(t * std::log(b2))));
  c.eps = hp->eps;
  c.scale = hp->grad_scale;
  c.scale_dev = hp->grad_scale_dev;
  hipStream_t s = static_cast<hipStream_t>(stream_ptr);
  return launch("adam_step", s, [&] {
    return adam_step(c, n, grad, master, m, v, static_cast<uint16_t*>(weight), hp->zero_grad, s);
  });
}
