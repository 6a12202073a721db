// C ABI of the training step (declared in include/mi355am.h): argument
// validation, workspace planning, the launch sequence of the forward and
// backward passes, and per-class kernel timing with HIP events.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <string>
#include <vector>

#include "../../include/mi355am.h"
#include "am_internal.h"

namespace {

thread_local std::string g_err;

am_status fail(am_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_err = buf;
  return st;
}

am_status hip_check(hipError_t e, const char* what) {
  if (e == hipSuccess) return AM_OK;
  return fail(AM_EHIP, "%s: %s", what, hipGetErrorString(e));
}

#define AM_TRY(expr)                        \
  do {                                      \
    am_status st_ = (expr);                 \
    if (st_ != AM_OK) return st_;           \
  } while (0)

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// ---------------------------------------------------------------- timing --

struct ProfRec {
  int cls;
  hipEvent_t a, b;
  double flops, bytes;
};

struct Prof {
  bool on = false;
  uint32_t mask = 0;
  int32_t every = 1;                    // record every n-th launch of a class
  int64_t seen[AM_K_NCLASSES] = {};     // launches of the class since begin
  std::vector<hipEvent_t> pool;
  size_t next = 0;
  std::vector<ProfRec> recs;
  int64_t launches[AM_K_NCLASSES] = {};
  double ms[AM_K_NCLASSES] = {}, flops[AM_K_NCLASSES] = {}, bytes[AM_K_NCLASSES] = {};
} g_prof;

hipEvent_t prof_event() {
  if (g_prof.next == g_prof.pool.size()) {
    // timing only: no system-scope fence (cache write-back) at each record,
    // which would otherwise add a gap of several microseconds per bracket
    hipEvent_t e;
    if (hipEventCreateWithFlags(&e, hipEventDisableSystemFence) != hipSuccess) return nullptr;
    g_prof.pool.push_back(e);
  }
  return g_prof.pool[g_prof.next++];
}

// Brackets the kernels launched during its lifetime with events when the
// class is being recorded (every n-th launch of the class when sampling).
class Timed {
 public:
  Timed(int cls, hipStream_t s, double flops, double bytes) : s_(s) {
    if (!g_prof.on || !(g_prof.mask & (1u << cls))) return;
    rec_.cls = cls;
    counted_ = true;
    if (g_prof.seen[cls]++ % g_prof.every != 0) return;
    rec_.flops = flops;
    rec_.bytes = bytes;
    rec_.a = prof_event();
    rec_.b = prof_event();
    if (rec_.a && rec_.b && hipEventRecord(rec_.a, s_) == hipSuccess) active_ = true;
  }
  ~Timed() {
    if (active_ && hipEventRecord(rec_.b, s_) == hipSuccess) g_prof.recs.push_back(rec_);
  }
  void cancel() {  // nothing was launched
    if (counted_) --g_prof.seen[rec_.cls];
    counted_ = active_ = false;
  }

 private:
  hipStream_t s_;
  ProfRec rec_{};
  bool counted_ = false;
  bool active_ = false;
};

// ------------------------------------------------------------- the model --

int vec_of(int dtype) { return dtype == AM_BF16 ? 8 : 4; }
int esz_of(int dtype) { return dtype == AM_BF16 ? 2 : 4; }

am_status check_model(const am_model* m) {
  if (!m) return fail(AM_EINVAL, "model is NULL");
  if (m->dtype != AM_F32 && m->dtype != AM_BF16) return fail(AM_EINVAL, "dtype %d unknown", m->dtype);
  if (m->layers < 1 || m->input_dim < 1 || m->hidden < 1 || m->classes < 1)
    return fail(AM_EINVAL, "model sizes must be positive");
  if (m->hidden % 16) return fail(AM_EUNSUPPORTED, "hidden %d is not a multiple of 16", m->hidden);
  const int v = vec_of(m->dtype);
  if (m->input_dim % v || m->classes % v)
    return fail(AM_EUNSUPPORTED, "input_dim and classes must be multiples of %d for this dtype", v);
  if ((int64_t)m->hidden * 4 * (int64_t)(m->hidden > m->input_dim ? m->hidden : m->input_dim) >= (1ll << 31))
    return fail(AM_EUNSUPPORTED, "layer too large");
  return AM_OK;
}

struct Offsets {
  std::vector<int64_t> wx, wh, b;
  int64_t wo, bo, n;
};

Offsets param_layout(const am_model* m) {
  Offsets o;
  const int64_t G = 4ll * m->hidden;
  int64_t pos = 0;
  for (int l = 0; l < m->layers; ++l) {
    const int64_t D = l == 0 ? m->input_dim : m->hidden;
    o.wx.push_back(pos); pos += G * D;
    o.wh.push_back(pos); pos += G * m->hidden;
    o.b.push_back(pos); pos += G;
  }
  o.wo = pos; pos += (int64_t)m->classes * m->hidden;
  o.bo = pos; pos += m->classes;
  o.n = pos;
  return o;
}

// Schedule of a batch: active counts per step and packed row offsets.
struct Schedule {
  int T = 0, B = 0;
  std::vector<int64_t> counts, offs;
  std::vector<int32_t> lens;
  int64_t N = 0;
};

am_status make_schedule(int32_t T, int32_t B, const int32_t* lengths, Schedule& s) {
  if (T < 0 || B < 1) return fail(AM_EINVAL, "need T >= 0 and B >= 1 (T=%d, B=%d)", T, B);
  s.T = T; s.B = B;
  s.lens.assign(B, T);
  if (lengths) {
    if (B > 1024) return fail(AM_EUNSUPPORTED, "variable-length batches allow B <= 1024");
    for (int b = 0; b < B; ++b) {
      if (lengths[b] < 0 || lengths[b] > T)
        return fail(AM_EINVAL, "lengths[%d] = %d outside [0, %d]", b, lengths[b], T);
      if (b > 0 && lengths[b] > lengths[b - 1])
        return fail(AM_EINVAL, "lengths must be non-increasing (lengths[%d] > lengths[%d])", b, b - 1);
      s.lens[b] = lengths[b];
    }
  }
  s.counts.assign(T, 0);
  s.offs.assign(T + 1, 0);
  int64_t nb = B;
  for (int t = 0; t < T; ++t) {
    while (nb > 0 && s.lens[nb - 1] <= t) --nb;
    s.counts[t] = nb;
    s.offs[t + 1] = s.offs[t] + nb;
  }
  s.N = s.offs[T];
  if (s.N >= (1ll << 31)) return fail(AM_EUNSUPPORTED, "too many frames");
  return AM_OK;
}

// The persistent layer kernels are used when they fit; AM_STEP_KERNELS=1 in
// the environment forces one launch per time step instead.
bool persistent_enabled() {
  const char* v = getenv("AM_STEP_KERNELS");
  if (v && v[0] && v[0] != '0') return false;
  const char* r = getenv("AM_RECURRENCE");
  return !(r && strcmp(r, "step") == 0);
}

// The bf16 per-step forward runs each step as one launch with the cell in
// the product's epilogue; AM_STEP_FUSION=0 in the environment keeps the
// product and the cell as two launches (tests compare the two bit for bit).
bool step_cell_fusion() {
  const char* v = getenv("AM_STEP_FUSION");
  return !(v && v[0] == '0' && v[1] == 0);
}

// AM_RECURRENCE=xcd|device|step picks one recurrence path (for tests);
// unset, the XCD-local kernels are tried first, then the device-scope ones.
bool xcd_enabled() {
  const char* r = getenv("AM_RECURRENCE");
  return persistent_enabled() && !(r && strcmp(r, "device") == 0);
}
bool device_persistent_enabled() {
  const char* r = getenv("AM_RECURRENCE");
  return persistent_enabled() && !(r && strcmp(r, "xcd") == 0);
}

// Scratch of the persistent kernels: the sync area at offset 0 of the
// workspace, one SYNC_BYTES slot per recurrence launch of a pass (each
// launch's step flags and XCC ids; several per layer where the sequences go
// in rounds), so that one clear at the
// start of a pass serves all its launches instead of one small clear kernel
// before each.  The last word of slot 0 is the barrier time-out flag of
// every launch, zeroed once per forward pass and only ever set afterwards,
// so a time-out anywhere in a forward + backward pair stays visible to
// am_workspace_check.
constexpr int64_t SYNC_BYTES = 8192;
// k-splits of the per-step backward product dA_{t+1} W_h (five fill 240 of
// the 256 CUs with the 48 tiles of B = 512, H = 1536)
constexpr int STEP_SPLITS = 5;
constexpr int64_t SYNC_STICKY_WORD = SYNC_BYTES / 4 - 1;
static_assert(am::XCD_SYNC_WORDS * 4 == SYNC_BYTES, "a round's slot follows the one before");
// Slots of one recurrence: one for each round of sequences it may be run in
// (a round holds at least 128).
int sync_rounds(int64_t B) {
  const int64_t r = (B + 127) / 128;
  return (int)(r < 1 ? 1 : r > am::XCD_MAX_ROUNDS ? am::XCD_MAX_ROUNDS : r);
}
// First slot of recurrence k of a pass over B sequences.
void* sync_slot(void* area, int k, int64_t B) {
  return static_cast<char*>(area) + (int64_t)k * sync_rounds(B) * SYNC_BYTES;
}
int* sync_err(void* area) { return static_cast<int*>(area) + SYNC_STICKY_WORD; }
am::XcdSync xcd_sync(void* slot, int* err) {
  unsigned* u = static_cast<unsigned*>(slot);
  am::XcdSync y;
  y.flags = u;  // flag line of block k < 16: u[32 k .. 32 k + 31], a word per member
  y.xcc = reinterpret_cast<int*>(u + 512);  // XCC line of block k: u[512 + 32 k ..], the same
  y.err = err;
  y.units = 0;
  y.fenced = 0;
  return y;
}
static_assert(1024 + 512 <= SYNC_STICKY_WORD,
              "a slot holds the flag and XCC lines, and the second flag lines of a launch of all layers, "
              "below the time-out word");

bool is_varlen(const Schedule& sc) {
  for (int b = 0; b < sc.B; ++b)
    if (sc.lens[b] != sc.T) return true;
  return false;
}

// Whether the XCD-local kernels take this layer's recurrence: bf16, the
// shape instantiated, and (variable lengths) T within the schedule's 16-bit
// lengths.
bool xcd_shape(bool bf, int64_t H, int T, int B, bool varlen) {
  return bf && xcd_enabled() && am::lstm_xcd_covers((int)H, B, T) &&
         (!varlen || T <= 65535);
}
bool xcd_path(bool bf, int64_t H, const Schedule& sc) {
  return xcd_shape(bf, H, sc.T, sc.B, is_varlen(sc));
}

// Narrow layers run one workgroup per 16 sequences, unless the environment
// asks for the XCD-local or the device-scope kernels (tests).  At 128 cells a
// step's products in one compute unit outlast the exchange between several (3
// x 128, 5 chunks of 78 frames, step: 862 us against 798), so the XCD-local
// kernels go first there.
bool solo_shape(bool bf, int64_t H, int T, int B, bool varlen) {
  auto set = [](const char* name) {
    const char* v = getenv(name);
    return v && v[0] && !(v[0] == '0' && v[1] == 0);
  };
  return persistent_enabled() && !set("AM_RECURRENCE") && !set("AM_XCD_FENCED") &&
         !set("AM_XCD_BLOCKS") && am::lstm_solo_covers((int)H, bf) && (!varlen || T <= 65535) &&
         !(H == 128 && xcd_shape(bf, H, T, B, varlen));
}
// Whether the forward pass runs every layer in one launch: where the XCD-local
// kernels would run them one after another (and no environment variable asks
// for one path) and the layers' blocks of sequences have room side by side.
bool pipe_shape(bool bf, int64_t H, int64_t L, int T, int B, bool varlen) {
  const char* r = getenv("AM_RECURRENCE");
  const char* o = getenv("AM_XCD_BLOCKS");
  return !(r && r[0]) && !(o && o[0] == '1') && xcd_shape(bf, H, T, B, varlen) &&
         !solo_shape(bf, H, T, B, varlen) && am::lstm_pipe_covers((int)H, B, (int)L);
}

// AM_DEBUG=1 in the environment: entry points that consume indices held in
// device buffers synchronise and check them.
bool debug_checks() {
  const char* v = getenv("AM_DEBUG");
  return v && v[0] == '1' && v[1] == 0;
}

am::PersistSchedule persist_schedule(const Schedule& sc) {
  am::PersistSchedule ps;
  ps.T = sc.T;
  ps.B = sc.B;
  ps.N = (int)sc.N;
  ps.first = 0;
  ps.varlen = 0;
  for (int b = 0; b < sc.B; ++b)
    if (sc.lens[b] != sc.T) ps.varlen = 1;
  memset(ps.lens, 0, sizeof ps.lens);
  if (ps.varlen)
    for (int b = 0; b < sc.B; ++b) ps.lens[b] = (uint16_t)sc.lens[b];
  return ps;
}

// Workspace carve-up (256-byte aligned regions).
struct WsLayout {
  std::vector<int64_t> h, hs, c, g;  // per layer
  int64_t p_da, dh, wht, dc, c0, h0, pre, splitk, splitk_floats, sync, total;
  static constexpr int MAX_SPLITS = 8;
};

int64_t align256(int64_t x) { return (x + 255) & ~int64_t(255); }

WsLayout ws_layout(const am_model* m, int64_t B, int64_t N) {
  WsLayout w;
  const int64_t e = esz_of(m->dtype), H = m->hidden, G = 4 * H, L = m->layers;
  int64_t pos = 0;
  auto take = [&](int64_t bytes) { int64_t at = pos; pos += align256(bytes); return at; };
  // step-barrier scratch of the persistent kernels (a slot per layer and
  // direction of the pass) and the time-out flag
  w.sync = take(2 * L * sync_rounds(B) * SYNC_BYTES);
  for (int l = 0; l < L; ++l) {
    w.h.push_back(take(N * H * e));
    w.hs.push_back(take(N * H * e));
    w.c.push_back(take(N * H * 4));
    w.g.push_back(take(N * G * e));
  }
  w.p_da = take(N * G * e);
  w.dh = take(N * H * e);
  w.wht = take(L * G * H * e);  // W_h^T of every layer (transposed in one launch)
  w.dc = take(B * H * 4);
  w.c0 = take(L * B * H * 4);
  w.h0 = take(L * B * H * e);
  // one step's recurrent product (per-step path): [B][4H] fp32 forward, up to
  // STEP_SPLITS k-split partials [B][H] fp32 backward
  w.pre = take(B * H * 4 * (STEP_SPLITS > 4 ? STEP_SPLITS : 4));
  // split-K partials of the weight-gradient products (plus partial row sums)
  const int64_t D0 = m->input_dim;
  const int64_t wide = (D0 > H ? D0 : H) + H;
  int64_t mn = G * wide + G;
  if ((int64_t)m->classes * H + m->classes > mn) mn = (int64_t)m->classes * H + m->classes;
  w.splitk_floats = WsLayout::MAX_SPLITS * mn;
  w.splitk = take(w.splitk_floats * 4);
  w.total = pos;
  return w;
}

template <typename P> P* at(void* base, int64_t off) {
  return reinterpret_cast<P*>(static_cast<char*>(base) + off);
}

double gemm_bytes(int64_t M, int64_t N, int64_t K, int64_t e, int64_t out) {
  return (double)(M * K + N * K) * e + (double)(M * N) * out;
}

am_status run_gemm(int cls, const am::GemmArgs& g, hipStream_t s) {
  const int64_t e = g.bf16 ? 2 : 4;
  Timed tm(cls, s, 2.0 * g.M * g.N * (double)g.K, gemm_bytes(g.M, g.N, g.K, e, g.c_f32 ? 4 : e));
  return hip_check(am::gemm(g, s), "gemm");
}

am::GemmArgs mk_gemm(const void* A, int64_t lda, bool ak, const void* B, int64_t ldb, bool bk,
                     void* C, int64_t ldc, bool cf32, const void* bias, int M, int N, int K,
                     bool bf16) {
  am::GemmArgs g;
  g.A = A; g.lda = lda; g.a_kmajor = ak;
  g.B = B; g.ldb = ldb; g.b_kmajor = bk;
  g.C = C; g.ldc = ldc; g.c_f32 = cf32;
  g.bias = bias; g.M = M; g.N = N; g.K = K; g.bf16 = bf16;
  return g;
}

// One layer's recurrence, forward in time, over the packed rows of a
// schedule: narrow layers by a workgroup per 16 sequences, else the XCD-local
// persistent kernel where it covers the shape, else the device-scope persistent
// kernel, else one launch per time step.
struct FwdLayer {
  const void* P;      // [N][4H] input projections + bias
  const void* Wh;     // [4H][H]
  const void* h0;     // [B][H] activation type, or null (zero)
  const float* c0;    // [B][H]
  void* H; void* Hs; float* C; void* G;  // outputs [N][H], [N][H], [N][H], [N][4H]
  void* sync;         // this launch's slot of the workspace's sync area (cleared)
  int* err;           // the time-out flag
  float* pre;         // [B][4H] fp32 scratch of the per-step path
};

am_status forward_recurrence(const FwdLayer& f, const Schedule& sc, bool bf, int64_t H,
                             hipStream_t s) {
  const int64_t e = bf ? 2 : 4, G = 4 * H;
  const int T = sc.T, B = sc.B;
  if (sc.N > 0 && persistent_enabled()) {
    am::PersistFwd pa;
    pa.P = f.P;
    pa.Wh = f.Wh;
    pa.h0 = f.h0;
    pa.c0 = f.c0;
    pa.H = f.H;
    pa.Hs = f.Hs;
    pa.C = f.C;
    pa.G = f.G;
    pa.counters = static_cast<unsigned*>(f.sync);
    pa.err = f.err;
    pa.ring = bf ? f.pre : nullptr;  // (RING_SLOTS rows of H bf16 in 4H fp32)
    pa.hidden = (int)H;
    const am::PersistSchedule ps = persist_schedule(sc);
    const double flops = 2.0 * sc.N * G * H;
    const double bytes = (double)sc.N * (G * e * 2 + H * (2 * e + 4)) + (double)G * H * e;
    bool used = false;
    if (solo_shape(bf, H, T, B, ps.varlen != 0)) {
      Timed tm(AM_K_LSTM_FWD, s, flops, bytes);
      return hip_check(am::lstm_fwd_solo_launch(pa, ps, bf, s), "lstm forward layer (solo)");
    }
    if (xcd_path(bf, H, sc)) {
      Timed tm(AM_K_LSTM_FWD, s, flops, bytes);
      AM_TRY(hip_check(am::lstm_fwd_xcd_launch(pa, ps, xcd_sync(f.sync, f.err), s, &used),
                       "lstm forward layer (xcd)"));
      if (!used) tm.cancel();
    }
    if (!used && device_persistent_enabled() && am::lstm_persistent_fits(true, (int)H, B, bf, T)) {
      Timed tm(AM_K_LSTM_FWD, s, flops, bytes);
      AM_TRY(hip_check(am::lstm_fwd_persistent(pa, ps, bf, s, &used), "lstm forward layer"));
      if (!used) tm.cancel();
    }
    if (used) return AM_OK;
  }
  const char* Hl = static_cast<const char*>(f.H);
  const float* Cl = f.C;
  const bool fuse_cell = step_cell_fusion();
  for (int t = 0; t < T; ++t) {
    const int64_t nb = sc.counts[t];
    if (nb == 0) break;
    const int64_t o = sc.offs[t];
    am::LstmFwdStep a;
    a.P = static_cast<const char*>(f.P) + o * G * e;
    a.Wh = f.Wh;
    if (t == 0) {
      a.hprev = f.h0;
      a.cprev = f.c0;
    } else {
      a.hprev = Hl + sc.offs[t - 1] * H * e;
      a.cprev = Cl + sc.offs[t - 1] * H;
    }
    a.H = static_cast<char*>(f.H) + o * H * e;
    a.Hs = static_cast<char*>(f.Hs) + o * H * e;
    a.C = f.C + o * H;
    a.G = static_cast<char*>(f.G) + o * G * e;
    a.nb = (int)nb;
    a.hidden = (int)H;
    a.bf16 = bf;
    if (bf) {
      // the step's recurrent product as a batched product (few rows: square
      // tiles that fill the CUs) with the cell in its epilogue; else the
      // product into fp32 scratch, then the cell
      float* pre = nullptr;
      if (a.hprev && fuse_cell) {
        bool done = false;
        Timed tm(AM_K_LSTM_FWD, s, 2.0 * nb * G * H,
                 gemm_bytes(nb, G, H, e, 0) + (double)nb * (G * e + H * (2 * e + 8) + G * e));
        AM_TRY(hip_check(am::gemm_bf16_lstm_fwd_step(a, s, &done), "lstm forward step (fused)"));
        if (done) continue;
        tm.cancel();
      }
      if (a.hprev) {
        AM_TRY(run_gemm(AM_K_LSTM_FWD,
                        mk_gemm(a.hprev, H, true, f.Wh, H, true, f.pre, G, true, nullptr, (int)nb,
                                (int)G, (int)H, true), s));
        pre = f.pre;
      }
      Timed tm(AM_K_LSTM_FWD, s, 0.0, (double)nb * (G * (4.0 + e) + H * (2 * e + 8) + G * e));
      AM_TRY(hip_check(am::lstm_cell_fwd(pre, a, s), "lstm forward cell"));
      continue;
    }
    const double bytes = (double)(nb * H + G * H + nb * G) * e + nb * H * 4.0 +
                         (double)nb * (H * (2 * e + 4) + G * e);
    Timed tm(AM_K_LSTM_FWD, s, 2.0 * nb * G * H, bytes);
    AM_TRY(hip_check(am::lstm_fwd_step(a, s), "lstm forward step"));
  }
  return AM_OK;
}

// Weight gradient  [C | C2] = A^T [B | B2]  (K = frames), fp32, with the
// row sums of A (the bias gradient) and split-K scratch from the workspace.
am::GemmArgs mk_wgrad(const void* A, int64_t lda, const void* B, int64_t ldb, int nB,
                      const void* B2, int64_t ldb2, int nB2, float* C, int64_t ldc, float* C2,
                      int64_t ldc2, float* rowsum, int M, int K, bool bf16, float* ws,
                      int64_t ws_floats) {
  am::GemmArgs g;
  g.A = A; g.lda = lda; g.a_kmajor = false;
  g.B = B; g.ldb = ldb; g.b_kmajor = false;
  g.C = C; g.ldc = ldc; g.c_f32 = true;
  if (B2) {
    g.B2 = B2; g.ldb2 = ldb2; g.n_split = nB;
    g.C2 = C2; g.ldc2 = ldc2;
  }
  g.rowsum = rowsum;
  g.M = M; g.N = nB + (B2 ? nB2 : 0); g.K = K; g.bf16 = bf16;
  g.ws = ws; g.ws_floats = ws_floats;
  return g;
}

// Teacher: per layer, forward Wx [4H][D_l], Wh [4H][H], b [4H], then the
// backward direction's; D_0 = input_dim, D_l = 2H; then Wo [C][2H], bo [C].
struct TeacherOffsets {
  std::vector<int64_t> wx, wh, b;  // [layer * 2 + direction]
  int64_t wo, bo, n;
};

TeacherOffsets teacher_layout(const am_model* m) {
  TeacherOffsets o;
  const int64_t H = m->hidden, G = 4 * H;
  int64_t pos = 0;
  for (int l = 0; l < m->layers; ++l) {
    const int64_t D = l == 0 ? m->input_dim : 2 * H;
    for (int d = 0; d < 2; ++d) {
      o.wx.push_back(pos); pos += G * D;
      o.wh.push_back(pos); pos += G * H;
      o.b.push_back(pos); pos += G;
    }
  }
  o.wo = pos; pos += (int64_t)m->classes * 2 * H;
  o.bo = pos; pos += m->classes;
  o.n = pos;
  return o;
}

struct TeacherWs {
  int64_t sync, offs, lens, cat0, cat1, rev, p, hdir, hs, c, g, c0, pre, total;
};

TeacherWs teacher_ws_layout(const am_model* m, int64_t T, int64_t B, int64_t N) {
  TeacherWs w;
  const int64_t e = esz_of(m->dtype), H = m->hidden, G = 4 * H;
  const int64_t Dmax = m->input_dim > 2 * H ? m->input_dim : 2 * H;
  int64_t pos = 0;
  auto take = [&](int64_t bytes) { int64_t at = pos; pos += align256(bytes); return at; };
  w.sync = take(2 * m->layers * sync_rounds(B) * SYNC_BYTES);  // a slot per layer and direction
  w.offs = take((T + 1) * 8);
  w.lens = take(B * 4);
  w.cat0 = take(N * 2 * H * e);
  w.cat1 = take(N * 2 * H * e);
  w.rev = take(N * Dmax * e);
  w.p = take(N * G * e);
  w.hdir = take(N * H * e);
  w.hs = take(N * H * e);
  w.c = take(N * H * 4);
  w.g = take(N * G * e);
  w.c0 = take(B * H * 4);
  w.pre = take(B * G * 4);
  w.total = pos;
  return w;
}

// ------------------------------------------------- threshold encode --

am_status check_encode_args(int64_t n, const float* grad, const float* residual, float tau,
                            const uint32_t* words, int64_t capacity, const int64_t* count) {
  if (n < 0 || n >= (1ll << 31)) return fail(AM_EINVAL, "n = %lld outside [0, 2^31)", (long long)n);
  if (!(tau > 0.f)) return fail(AM_EINVAL, "tau must be > 0");
  if (!count) return fail(AM_EINVAL, "count is NULL");
  if (n > 0 && (!grad || !residual || !words)) return fail(AM_EINVAL, "NULL pointer");
  if (capacity < n) return fail(AM_ECAPACITY, "capacity %lld < n %lld", (long long)capacity, (long long)n);
  return AM_OK;
}

// The encode launches on a scratch area of gtc_encode_scratch_bytes(n)
// (the codes, then the tile counts); every byte the kernels read there is
// written by the same call first, so the area needs no clearing.
am_status encode_with_scratch(int64_t n, const float* grad, float* residual, float tau,
                              uint32_t* words, int64_t* count, void* scratch, hipStream_t s) {
  Timed tm(AM_K_ENCODE, s, 0.0, 12.0 * n);
  uint32_t* codes = at<uint32_t>(scratch, 0);
  int32_t* tile = at<int32_t>(scratch, am::gtc_codes_bytes(n));
  return hip_check(am::gtc_encode(n, grad, residual, tau, words, count, codes, tile, s), "encode");
}

// Scratch of grad_threshold_encode_noalloc: a device array owned by the
// library for the life of the process (each GPU holds its own copy).  In
// host code its name only stands in for the symbol; the device address of
// a GPU's copy comes from hipGetSymbolAddress with that GPU current, once,
// and is kept per device.
constexpr int64_t NOALLOC_SCRATCH_BYTES = am::gtc_encode_scratch_bytes(AM_ENCODE_NOALLOC_MAX_N);
static __device__ __align__(256) unsigned char encode_scratch[NOALLOC_SCRATCH_BYTES];

constexpr int MAX_DEVICES = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[MAX_DEVICES] = {};

am_status encode_scratch_of(hipStream_t s, void** out) {
  int cur = 0, dev = 0;
  AM_TRY(hip_check(hipGetDevice(&cur), "hipGetDevice"));
  dev = cur;
  if (s) AM_TRY(hip_check(hipStreamGetDevice(s, &dev), "hipStreamGetDevice"));
  if (dev < 0 || dev >= MAX_DEVICES) return fail(AM_EUNSUPPORTED, "device %d >= %d", dev, MAX_DEVICES);
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    if (dev != cur) AM_TRY(hip_check(hipSetDevice(dev), "hipSetDevice"));
    void* p = nullptr;
    const hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(encode_scratch));
    if (dev != cur) AM_TRY(hip_check(hipSetDevice(cur), "hipSetDevice"));
    AM_TRY(hip_check(e, "hipGetSymbolAddress(encode scratch)"));
    if (!p || !aligned(p, 256)) return fail(AM_EHIP, "encode scratch has no 256-byte aligned address");
    g_scratch_ptr[dev] = p;
  }
  *out = g_scratch_ptr[dev];
  return AM_OK;
}

// ------------------------------------------- gated linear recurrences --

// Rows of H elements that an operator reads or writes.
// (`frame`: rows that a kernel reaches by 32-bit offsets from the first.)
am_status check_rows(int64_t N, int32_t H, int32_t dtype, const void* p, int64_t ld, const char* name,
                     int64_t frame = 0) {
  if (N > 0 && !p) return fail(AM_EINVAL, "NULL %s", name);
  if (!aligned(p, (uintptr_t)esz_of(dtype))) return fail(AM_EINVAL, "%s is not aligned to its elements", name);
  if (ld < H) return fail(AM_EINVAL, "row stride %lld of %s is less than %d", (long long)ld, name, H);
  if (frame > 0 && ld > ((1ll << 30) - 8) / frame)
    return fail(AM_EUNSUPPORTED, "frames of %s beyond 2^30 - 8 elements", name);
  return AM_OK;
}

// The time-out flag is the last word of a first slot, where am_workspace_check
// looks; the words of linked tiles follow it, so that one clear serves both.
struct GatedLayout {
  int64_t sync, offs, lens, tails, saved, parts, tickets, stretches, states, total;
};
GatedLayout gated_layout(int64_t T, int64_t B, int64_t H, bool varlen, bool train) {
  GatedLayout l{};
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += align256(bytes);
    return here;
  };
  const am::GatedLinks k = am::gated_links(T, B, H);
  if (varlen || train || k.words > 0) l.sync = take(SYNC_BYTES);
  if (k.words > 0) {
    l.tickets = take(k.words * 4);
    l.stretches = take(k.stretches * 8);
    l.states = take(k.states * 8);
  }
  if (varlen) {
    l.offs = take((T + 1) * 4);
    l.lens = take(B * 4);
    l.tails = take(B * 4);
  }
  if (train) {
    l.saved = take((T + am::GR_TILE - 1) / am::GR_TILE * B * H * 4);
    l.parts = take((k.words > 0 ? k.stretches : B * H) * 4);
  }
  l.total = at;
  return l;
}

// The arguments that forward and backward share; fills in a's schedule.
am_status check_gated(int32_t T, int32_t B, int32_t H, int32_t dtype, const int32_t* lengths,
                      const float* lam, float c, bool train, void* ws, int64_t ws_bytes,
                      am::GatedRecurrence& a, GatedLayout& l) {
  if (T < 0 || B < 1 || H < 1) return fail(AM_EINVAL, "need T >= 0, B >= 1 and H >= 1 (T=%d, B=%d, H=%d)", T, B, H);
  if (dtype != AM_F32 && dtype != AM_BF16) return fail(AM_EINVAL, "dtype %d unknown", dtype);
  if (!lam || !aligned(lam, 4)) return fail(AM_EINVAL, "NULL or unaligned lam");
  if (!(c > 0.f && c <= 3.4e38f)) return fail(AM_EINVAL, "c must be positive and finite");
  a.N = (int64_t)T * B;
  a.T = T;
  if (lengths) {
    if (B > 1024) return fail(AM_EUNSUPPORTED, "variable-length batches allow B <= 1024");
    a.N = 0;
    for (int b = 0; b < B; ++b) {
      if (lengths[b] < 0 || lengths[b] > T)
        return fail(AM_EINVAL, "lengths[%d] = %d outside [0, %d]", b, lengths[b], T);
      if (b > 0 && lengths[b] > lengths[b - 1])
        return fail(AM_EINVAL, "lengths must be non-increasing (lengths[%d] > lengths[%d])", b, b - 1);
      a.N += lengths[b];
    }
    a.T = lengths[0];
  }
  // (the kernels count frames in 32 bits, up to the end of a tile or a workgroup of
  // 256 past the last)
  if (a.N >= (1ll << 31) - 256) return fail(AM_EUNSUPPORTED, "too many frames");
  l = gated_layout(T, B, H, lengths != nullptr, train);
  if (l.total > 0 && (!ws || !aligned(ws, 256) || ws_bytes < l.total))
    return fail(AM_EWORKSPACE, "needs %lld workspace bytes, 256-byte aligned", (long long)l.total);
  a.B = B;
  a.H = H;
  a.lam = lam;
  a.c = c;
  if (l.total > 0) a.err = sync_err(at<void>(ws, l.sync));
  a.tickets = at<uint32_t>(ws, l.tickets);
  a.stretches = at<uint64_t>(ws, l.stretches);
  a.states = at<uint64_t>(ws, l.states);
  if (lengths) {
    a.offs = at<int32_t>(ws, l.offs);
    a.lens = at<int32_t>(ws, l.lens);
    a.tails = at<int32_t>(ws, l.tails);
  }
  return AM_OK;
}

struct DeltaLayout { int64_t offs, lens, tails, saved, dsaved, u, dr, parts, seg_n, seg_m, seg_mt, seg_d, total; };
DeltaLayout delta_layout(int64_t T, int64_t B, int64_t H, int32_t dk, int32_t dv, bool varlen, bool train) {
  DeltaLayout l{};
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += align256(bytes);
    return here;
  };
  if (varlen) {
    l.offs = take((T + 1) * 4);
    l.lens = take(B * 4);
    l.tails = take(B * 4);
  }
  if (train) {  // (the first chunk starts from s0, the last one's gradient from dsT)
    const int64_t chunks = T > 0 ? (T - 1) / am::GD_CHUNK + 1 : 0;
    const int64_t columns = B * H * am::gd_padded(dv);
    l.saved = take(chunks ? (chunks - 1) * columns * am::gd_padded(dk) * 4 : 0);
    l.dsaved = take(chunks * columns * am::gd_padded(dk) * 4);
    l.u = take(chunks * columns * am::GD_CHUNK * am::GD_TERMS * 2);
    l.dr = take(chunks * columns * am::GD_CHUNK * am::GD_TERMS * 2);
    l.parts = take(chunks * B * H * 4);
  }
  const int64_t segs = T > 0 ? am::delta_segments(T, B * H, dv, train).count : 1;
  if (segs > 1) {
    const int64_t key = am::gd_padded(dk), state = segs * B * H * key * 4;
    l.seg_n = take(state * am::gd_padded(dv));
    l.seg_m = take(state * key);
    l.seg_mt = take(state * key);
    if (train) l.seg_d = take(state * am::gd_padded(dv));
  }
  l.total = at;
  return l;
}

// Heads that a launch has workgroups for (2^32 threads, 512 a workgroup), of a training
// pass those of every chunk.
bool delta_heads(int64_t T, int64_t B, int64_t heads, bool train) {
  const int64_t most = 1 << 23;
  return B < most && heads < most && B * heads * (train ? T / am::GD_CHUNK + 1 : 1) < most;
}

bool delta_sizes(int32_t T, int32_t B, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv) {
  return T >= 0 && B >= 1 && heads >= 1 && key_heads >= 1 && heads % key_heads == 0 && dk >= 1 && dv >= 1;
}

// The arguments that forward and backward share; fills in a.
am_status check_delta(int32_t T, int32_t B, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv,
                      int32_t dtype, const int32_t* lengths, const void* q, int64_t ldq, const void* k,
                      int64_t ldk, const void* v, int64_t ldv, const void* r, int64_t ldr, const void* b,
                      int64_t ldb, const float* lam, float c, float eps, const float* s0, bool train, void* ws,
                      int64_t ws_bytes, am::GatedDelta& a, DeltaLayout& l) {
  if (!delta_sizes(T, B, heads, key_heads, dk, dv))
    return fail(AM_EINVAL, "need T >= 0, B, dk, dv >= 1 and key_heads a divisor of heads (T=%d, B=%d, dk=%d, dv=%d, heads=%d, key_heads=%d)",
                T, B, dk, dv, heads, key_heads);
  if (dk > am::GD_MAX_DIM || dv > am::GD_MAX_DIM)
    return fail(AM_EUNSUPPORTED, "heads of at most %d x %d", am::GD_MAX_DIM, am::GD_MAX_DIM);
  if (dtype != AM_F32 && dtype != AM_BF16) return fail(AM_EINVAL, "dtype %d unknown", dtype);
  if (!lam || !aligned(lam, 4)) return fail(AM_EINVAL, "NULL or unaligned lam");
  if (!(c > 0.f && c <= 3.4e38f)) return fail(AM_EINVAL, "c must be positive and finite");
  if (!(eps > 0.f && eps <= 3.4e38f)) return fail(AM_EINVAL, "eps must be positive and finite");
  if (!aligned(s0, 4)) return fail(AM_EINVAL, "states must be 4-byte aligned");
  a.N = (int64_t)T * B;
  a.T = T;
  if (lengths) {
    if (B > 1024) return fail(AM_EUNSUPPORTED, "variable-length batches allow B <= 1024");
    a.N = 0;
    for (int n = 0; n < B; ++n) {
      if (lengths[n] < 0 || lengths[n] > T)
        return fail(AM_EINVAL, "lengths[%d] = %d outside [0, %d]", n, lengths[n], T);
      if (n > 0 && lengths[n] > lengths[n - 1])
        return fail(AM_EINVAL, "lengths must be non-increasing (lengths[%d] > lengths[%d])", n, n - 1);
      a.N += lengths[n];
    }
    a.T = lengths[0];
  }
  if (a.N >= (1ll << 31) - 256 || T > (1 << 30)) return fail(AM_EUNSUPPORTED, "too many frames");
  if (!delta_heads(T, B, heads, train)) return fail(AM_EUNSUPPORTED, "too many heads");
  AM_TRY(check_rows(a.N, key_heads * dk, dtype, q, ldq, "q"));
  AM_TRY(check_rows(a.N, key_heads * dk, dtype, k, ldk, "k"));
  AM_TRY(check_rows(a.N, heads * dv, dtype, v, ldv, "v"));
  AM_TRY(check_rows(a.N, heads, dtype, r, ldr, "r"));
  AM_TRY(check_rows(a.N, heads, dtype, b, ldb, "b"));
  l = delta_layout(T, B, heads, dk, dv, lengths != nullptr, train);
  if (l.total > 0 && (!ws || !aligned(ws, 256) || ws_bytes < l.total))
    return fail(AM_EWORKSPACE, "needs %lld workspace bytes, 256-byte aligned", (long long)l.total);
  a.q = q; a.k = k; a.v = v; a.r = r; a.b = b;
  a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldr = ldr; a.ldb = ldb;
  a.B = B; a.H = heads; a.G = key_heads;
  a.dk = dk; a.dv = dv;
  a.lam = lam;
  a.c = c;
  a.eps = eps;
  a.s0 = s0;
  if (lengths) {
    a.offs = at<int32_t>(ws, l.offs);
    a.lens = at<int32_t>(ws, l.lens);
  }
  // (from T, as the workspace is laid out)
  const am::DeltaSegments cut = am::delta_segments(T, (int64_t)B * heads, dv, train);
  a.segs = T > 0 ? cut.count : 1;
  a.per = T > 0 ? cut.per : 1;
  a.seg_n = at<float>(ws, l.seg_n);
  a.seg_m = at<float>(ws, l.seg_m);
  a.seg_mt = at<float>(ws, l.seg_mt);
  a.seg_d = at<float>(ws, l.seg_d);
  return AM_OK;
}

am_status check_norm(int64_t N, int32_t H, int32_t dtype, int32_t res_dtype, const void* o, int64_t ldo,
                     const void* gate, int64_t ldg, const float* w_post, const float* scale, const void* res,
                     const float* w_next, float eps, am::GatedNorm& a) {
  if (N < 0 || H < 1) return fail(AM_EINVAL, "need N >= 0 and H >= 1 (N=%lld, H=%d)", (long long)N, H);
  if (H > am::GATED_NORM_MAX_H) return fail(AM_EUNSUPPORTED, "rows of at most %d elements", am::GATED_NORM_MAX_H);
  if ((dtype != AM_F32 && dtype != AM_BF16) || (res_dtype != AM_F32 && res_dtype != AM_BF16))
    return fail(AM_EINVAL, "dtype %d or res_dtype %d unknown", dtype, res_dtype);
  if (!(eps > 0.f && eps <= 3.4e38f)) return fail(AM_EINVAL, "eps must be positive and finite");
  // (an empty matrix may have no address)
  if (N > 0 && !o && (gate || w_post || scale)) return fail(AM_EINVAL, "gate, w_post or scale without o");
  if (N > 0 && !o && !w_next) return fail(AM_EINVAL, "neither o nor w_next: nothing to do");
  AM_TRY(check_rows(N, H, res_dtype, res, H, "res"));
  if (o) AM_TRY(check_rows(N, H, dtype, o, ldo, "o"));
  if (gate) AM_TRY(check_rows(N, H, dtype, gate, ldg, "gate"));
  if (!aligned(w_post, 4) || !aligned(scale, 4) || !aligned(w_next, 4))
    return fail(AM_EINVAL, "w_post, scale and w_next must be 4-byte aligned");
  a.N = N;
  a.H = H;
  a.eps = eps;
  a.o = N > 0 ? o : nullptr;
  a.ldo = ldo;
  a.gate = gate;
  a.ldg = ldg;
  a.res = res;
  a.w_post = w_post;
  a.scale = scale;
  a.w_next = w_next;
  return AM_OK;
}

// Codes and scales of a matrix in 8 bits.
am_status check_q8(int64_t rows, int64_t cols, const void* codes, int64_t ldc, const void* scales, int64_t lds,
                   const char* name) {
  if (rows > 0 && cols > 0 && (!codes || !scales)) return fail(AM_EINVAL, "NULL codes or scales of %s", name);
  if (!aligned(codes, 16) || ldc % 16 != 0)
    return fail(AM_EINVAL, "rows of codes of %s must start on 16 bytes (row stride %lld)", name, (long long)ldc);
  if (ldc < (cols + 15) / 16 * 16)
    return fail(AM_EINVAL, "codes of %s need rows of %lld bytes, got %lld", name, (long long)((cols + 15) / 16 * 16),
                (long long)ldc);
  if (!aligned(scales, 4) || lds % 4 != 0)
    return fail(AM_EINVAL, "rows of scales of %s must start on 4 bytes (row stride %lld)", name, (long long)lds);
  if (lds < (cols + 511) / 512 * 4)
    return fail(AM_EINVAL, "scales of %s need rows of %lld bytes, got %lld", name, (long long)((cols + 511) / 512 * 4),
                (long long)lds);
  const int64_t most = int64_t(1) << 62;
  if (rows > 0 && (ldc > most / rows || lds > most / rows)) return fail(AM_EINVAL, "%s is too large", name);
  return AM_OK;
}

double norm_bytes(const am::GatedNorm& a, int dtype, int res_dtype, bool backward) {
  const double e = esz_of(dtype), f = esz_of(res_dtype);
  const double act = (a.o ? 1 : 0) + (a.gate ? 1 : 0);
  if (!backward) return (double)a.N * a.H * (e * (act + (a.w_next ? 1 : 0)) + f * (a.o ? 2 : 1));
  return (double)a.N * a.H * (e * (2 * act + (a.w_next ? 1 : 0)) + f * (a.dres_out ? 3 : 2));
}

}  // namespace

// ================================================================= C ABI ==

extern "C" {

const char* am_status_string(int32_t st) {
  switch (st) {
    case AM_OK: return "ok";
    case AM_EINVAL: return "invalid argument";
    case AM_ECAPACITY: return "output capacity too small";
    case AM_EUNSUPPORTED: return "unsupported configuration";
    case AM_EHIP: return "HIP error";
    case AM_EWORKSPACE: return "workspace missing or too small";
    case AM_ETIMEOUT: return "step barrier timed out";
    default: return "unknown status";
  }
}

const char* am_last_error(void) { return g_err.c_str(); }

int64_t am_param_count(const am_model* m) {
  if (check_model(m) != AM_OK) return -1;
  return param_layout(m).n;
}

am_status am_param_offsets(const am_model* m, int64_t* offsets) {
  AM_TRY(check_model(m));
  if (!offsets) return fail(AM_EINVAL, "offsets is NULL");
  Offsets o = param_layout(m);
  for (int l = 0; l < m->layers; ++l) {
    offsets[3 * l] = o.wx[l];
    offsets[3 * l + 1] = o.wh[l];
    offsets[3 * l + 2] = o.b[l];
  }
  offsets[3 * m->layers] = o.wo;
  offsets[3 * m->layers + 1] = o.bo;
  return AM_OK;
}

int32_t am_recurrence_path(const am_model* m, int32_t T, int32_t B, int32_t varlen,
                           int32_t forward) {
  if (check_model(m) != AM_OK || T < 0 || B < 1) return -1;
  const bool bf = m->dtype == AM_BF16, fw = forward != 0;
  if (!persistent_enabled()) return AM_PATH_STEP;
  if (solo_shape(bf, m->hidden, T, B, varlen != 0)) return AM_PATH_SOLO;
  if (fw && pipe_shape(bf, m->hidden, m->layers, T, B, varlen != 0)) return AM_PATH_PIPE;
  if (xcd_shape(bf, m->hidden, T, B, varlen != 0)) return AM_PATH_XCD;
  if (device_persistent_enabled() && am::lstm_persistent_fits(fw, m->hidden, B, bf, T))
    return AM_PATH_DEVICE;
  return AM_PATH_STEP;
}

int64_t am_workspace_bytes(const am_model* m, int32_t T, int32_t B, int64_t N) {
  if (check_model(m) != AM_OK || T < 0 || B < 1 || N < 0 || N > (int64_t)T * B) return -1;
  return ws_layout(m, B, N).total;
}

int64_t am_ce_workspace_bytes(int64_t N) {
  if (N < 0) return -1;
  return align256(am::soft_ce_partials(N) * 4) + 256;
}

int64_t am_encode_workspace_bytes(int64_t n) {
  if (n < 0) return -1;
  return am::gtc_encode_scratch_bytes(n);
}

am_status am_cast_f32_to_bf16(int64_t n, const float* src, void* dst, void* stream) {
  if (n < 0) return fail(AM_EINVAL, "n < 0");
  if (n > 0 && (!src || !dst)) return fail(AM_EINVAL, "NULL pointer");
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_MISC, s, 0.0, 6.0 * n);
  return hip_check(am::cast_f32_bf16(n, src, static_cast<uint16_t*>(dst), s), "cast");
}

am_status sgd_apply(int64_t n, float* master, void* weights_bf16, const float* update, float lr,
                    void* stream) {
  if (n < 0) return fail(AM_EINVAL, "n < 0");
  if (n > 0 && (!master || !update)) return fail(AM_EINVAL, "NULL pointer");
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_SGD, s, 2.0 * n, (weights_bf16 ? 14.0 : 12.0) * n);
  return hip_check(am::sgd_apply_f32(n, master, static_cast<uint16_t*>(weights_bf16), update, lr, s),
                   "sgd_apply");
}

am_status grad_threshold_encode(int64_t n, const float* grad, float* residual, float tau,
                                uint32_t* words, int64_t capacity, int64_t* count, void* ws,
                                int64_t ws_bytes, void* stream) {
  AM_TRY(check_encode_args(n, grad, residual, tau, words, capacity, count));
  const int64_t need = am_encode_workspace_bytes(n);
  if (!ws || ws_bytes < need || !aligned(ws, 256))
    return fail(AM_EWORKSPACE, "encode needs %lld workspace bytes (256-aligned)", (long long)need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return encode_with_scratch(n, grad, residual, tau, words, count, ws, s);
}

am_status grad_threshold_encode_noalloc(int64_t n, const float* grad, float* residual, float tau,
                                        uint32_t* words, int64_t capacity, int64_t* count,
                                        void* stream) {
  AM_TRY(check_encode_args(n, grad, residual, tau, words, capacity, count));
  if (n > AM_ENCODE_NOALLOC_MAX_N)
    return fail(AM_EUNSUPPORTED, "grad_threshold_encode_noalloc handles n <= %lld (n = %lld); "
                "use grad_threshold_encode with a workspace", (long long)AM_ENCODE_NOALLOC_MAX_N,
                (long long)n);
  hipStream_t s = static_cast<hipStream_t>(stream);
  void* scratch = nullptr;
  AM_TRY(encode_scratch_of(s, &scratch));
  return encode_with_scratch(n, grad, residual, tau, words, count, scratch, s);
}

am_status grad_threshold_decode(const uint32_t* words, const int64_t* count, int64_t capacity,
                                float tau, int64_t n, float* dense, int32_t accumulate,
                                void* stream) {
  if (n < 0 || n >= (1ll << 31)) return fail(AM_EINVAL, "n outside [0, 2^31)");
  if (capacity < 0) return fail(AM_EINVAL, "capacity < 0");
  if (!count || (n > 0 && !dense) || (capacity > 0 && !words)) return fail(AM_EINVAL, "NULL pointer");
  if (accumulate != 0 && accumulate != 1) return fail(AM_EINVAL, "accumulate must be 0 or 1");
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_DECODE, s, 0.0, (accumulate ? 8.0 : 4.0) * n);
  return hip_check(am::gtc_decode(words, count, capacity, tau, n, dense, accumulate != 0, s), "decode");
}

am_status grad_threshold_decode_sgd(const uint32_t* words, const int64_t* count, int64_t capacity,
                                    float tau, int64_t n, float lr, float* master,
                                    void* weights_bf16, void* stream) {
  if (n < 0 || n >= (1ll << 31)) return fail(AM_EINVAL, "n outside [0, 2^31)");
  if (capacity < 0) return fail(AM_EINVAL, "capacity < 0");
  if (!count || (n > 0 && !master) || (capacity > 0 && !words)) return fail(AM_EINVAL, "NULL pointer");
  hipStream_t s = static_cast<hipStream_t>(stream);
  // bytes: with lr +0.0 or positive and finite only the named elements are
  // touched, 14 (or 12) bytes per word, which the host cannot count without
  // reading the count: none are recorded here; otherwise the master read and
  // written and the bf16 copy written (the words not counted)
  const uint32_t lb = __builtin_bit_cast(uint32_t, lr);
  const bool named_only = lb == 0u || (lr > 0.f && lr <= 3.402823466e38f);
  Timed tm(AM_K_SGD, s, named_only ? 0.0 : 2.0 * n, named_only ? 0.0 : (weights_bf16 ? 10.0 : 8.0) * n);
  return hip_check(am::gtc_decode_sgd(words, count, capacity, tau, n, lr, master,
                                      static_cast<uint16_t*>(weights_bf16), s),
                   "decode + sgd");
}

int64_t am_decode_multi_workspace_bytes(int32_t streams, int64_t n) {
  if (streams < 0 || n < 0) return -1;
  return align256((int64_t)streams * (am::gtc_tiles(n) + 1) * 4);
}

am_status grad_threshold_decode_multi(int32_t streams, const uint32_t* words, int64_t capacity,
                                      const int64_t* counts, float tau, int64_t n, float* dense,
                                      int32_t accumulate, void* ws, int64_t ws_bytes,
                                      void* stream) {
  if (n < 0 || n >= (1ll << 31)) return fail(AM_EINVAL, "n outside [0, 2^31)");
  if (streams < 0 || streams > 32767) return fail(AM_EINVAL, "streams outside [0, 32767]");
  if (capacity < 0) return fail(AM_EINVAL, "capacity < 0");
  if ((n > 0 && !dense) || (streams > 0 && (!counts || (capacity > 0 && !words))))
    return fail(AM_EINVAL, "NULL pointer");
  if (accumulate != 0 && accumulate != 1) return fail(AM_EINVAL, "accumulate must be 0 or 1");
  const int64_t need = am_decode_multi_workspace_bytes(streams, n);
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 256)))
    return fail(AM_EWORKSPACE, "multi-stream decode needs %lld workspace bytes (256-aligned)",
                (long long)need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_DECODE, s, 0.0, (accumulate ? 8.0 : 4.0) * n);
  return hip_check(am::gtc_decode_multi(streams, words, capacity, counts, tau, n, dense,
                                        accumulate != 0, static_cast<int32_t*>(ws), s),
                   "multi-stream decode");
}

am_status bmuf_block_update(int64_t n, int32_t count, int32_t workers, const float* models,
                            int64_t model_stride, float* global_model, float* delta, float eta,
                            float eta_next, float zeta, float* local_master, void* local_bf16,
                            void* stream) {
  if (n < 0) return fail(AM_EINVAL, "n < 0");
  if (count < 1 || workers < 1) return fail(AM_EINVAL, "count and workers must be >= 1");
  if (count > 1 && model_stride < n) return fail(AM_EINVAL, "model_stride < n");
  if (n > 0 && (!models || !global_model || !delta)) return fail(AM_EINVAL, "NULL pointer");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const double bytes = (4.0 * count + 16.0 + (local_master ? 4.0 : 0.0) + (local_bf16 ? 2.0 : 0.0)) * n;
  Timed tm(AM_K_BMUF, s, 0.0, bytes);
  return hip_check(am::bmuf_update(n, count, workers, models, model_stride, global_model, delta,
                                   eta, eta_next, zeta, local_master,
                                   static_cast<uint16_t*>(local_bf16), s),
                   "bmuf_block_update");
}

int32_t am_lfr_frames(int32_t raw_frames, int32_t stack, int32_t skip, int32_t offset) {
  if (raw_frames < 0 || stack < 1 || skip < 1 || offset < 0 || offset >= skip) return -1;
  const int32_t r = raw_frames - offset - stack;
  return r < 0 ? 0 : r / skip + 1;
}

am_status lfr_features(int32_t B, const int32_t* raw_lengths, const float* raw, int32_t raw_dim,
                       int32_t stack, int32_t skip, int32_t offset, const float* mean,
                       const float* std, void* x, int32_t x_dtype, void* stream) {
  if (B < 0 || B > 1024) return fail(AM_EUNSUPPORTED, "B must be in [0, 1024]");
  if (raw_dim < 1 || stack < 1 || skip < 1 || offset < 0 || offset >= skip)
    return fail(AM_EINVAL, "need raw_dim, stack, skip >= 1 and 0 <= offset < skip");
  if ((int64_t)stack * raw_dim > 4096) return fail(AM_EUNSUPPORTED, "stack * raw_dim > 4096");
  if (x_dtype != AM_F32 && x_dtype != AM_BF16) return fail(AM_EINVAL, "unknown x dtype");
  if (B > 0 && !raw_lengths) return fail(AM_EINVAL, "raw_lengths is NULL");
  am::LfrArgs a;
  memset(&a, 0, sizeof a);
  a.B = B; a.raw_dim = raw_dim; a.stack = stack; a.skip = skip; a.offset = offset;
  int64_t frames = 0, raws = 0;
  int32_t prev = 0, longest = 0;
  for (int b = 0; b < B; ++b) {
    if (raw_lengths[b] < 0 || raw_lengths[b] > 65535)
      return fail(AM_EUNSUPPORTED, "raw_lengths[%d] = %d outside [0, 65535]", b, raw_lengths[b]);
    const int32_t T = am_lfr_frames(raw_lengths[b], stack, skip, offset);
    if (b > 0 && T > prev)
      return fail(AM_EINVAL, "stacked lengths must be non-increasing (utterance %d)", b);
    if (b == 0) longest = T;
    prev = T;
    frames += T;
    raws += raw_lengths[b];
    a.U[b] = (uint16_t)raw_lengths[b];
  }
  if (raws > 0 && !raw) return fail(AM_EINVAL, "raw is NULL");
  if (frames > 0 && (!x || !mean || !std)) return fail(AM_EINVAL, "NULL x, mean or std");
  a.raw = raw; a.mean = mean; a.std = std; a.x = x;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const double bytes = (double)frames * stack * raw_dim * (4 + (x_dtype == AM_BF16 ? 2 : 4));
  Timed tm(AM_K_MISC, s, 0.0, bytes);
  return hip_check(am::lfr_features(a, longest, frames, x_dtype == AM_BF16, s), "lfr_features");
}

am_status delay_targets(int32_t T, int32_t B, const int32_t* lengths, int32_t K, int32_t delay,
                        const int32_t* idx, const float* prob, int32_t* idx_out, float* prob_out,
                        uint8_t* mask_out, void* stream) {
  if (T > 65535) return fail(AM_EUNSUPPORTED, "T > 65535");
  if (K < 0 || delay < 0) return fail(AM_EINVAL, "need K >= 0 and delay >= 0");
  Schedule sc;
  AM_TRY(make_schedule(T, B, lengths, sc));
  if (sc.N > 0 && (!mask_out || (K > 0 && (!idx || !prob || !idx_out || !prob_out))))
    return fail(AM_EINVAL, "NULL pointer");
  am::DelayArgs a;
  memset(&a, 0, sizeof a);
  if (B > 1024) return fail(AM_EUNSUPPORTED, "B > 1024");
  a.T = T; a.B = B; a.K = K; a.delay = delay;
  for (int b = 0; b < B; ++b) a.len[b] = (uint16_t)sc.lens[b];
  a.idx = idx; a.prob = prob; a.idx_out = idx_out; a.prob_out = prob_out; a.mask_out = mask_out;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_MISC, s, 0.0, (double)sc.N * (16.0 * K + 1));
  return hip_check(am::delay_targets(a, s), "delay_targets");
}

int64_t am_teacher_param_count(const am_model* m) {
  if (check_model(m) != AM_OK) return -1;
  return teacher_layout(m).n;
}

am_status am_teacher_param_offsets(const am_model* m, int64_t* offsets) {
  AM_TRY(check_model(m));
  if (!offsets) return fail(AM_EINVAL, "offsets is NULL");
  const TeacherOffsets o = teacher_layout(m);
  for (int k = 0; k < 2 * m->layers; ++k) {
    offsets[3 * k] = o.wx[k];
    offsets[3 * k + 1] = o.wh[k];
    offsets[3 * k + 2] = o.b[k];
  }
  offsets[6 * m->layers] = o.wo;
  offsets[6 * m->layers + 1] = o.bo;
  return AM_OK;
}

int64_t am_teacher_workspace_bytes(const am_model* m, int32_t T, int32_t B, int64_t N) {
  if (check_model(m) != AM_OK || T < 0 || B < 1 || N < 0 || N > (int64_t)T * B) return -1;
  return teacher_ws_layout(m, T, B, N).total;
}

am_status blstm_teacher_forward(const am_model* m, const void* params, const void* x,
                                const int32_t* lengths, int32_t T, int32_t B, float* logits,
                                void* ws, int64_t ws_bytes, void* stream) {
  AM_TRY(check_model(m));
  if (B > 1024 || T > 65535) return fail(AM_EUNSUPPORTED, "the teacher allows B <= 1024, T <= 65535");
  Schedule sc;
  AM_TRY(make_schedule(T, B, lengths, sc));
  if (!params || !ws) return fail(AM_EINVAL, "NULL params or workspace");
  if (sc.N > 0 && (!x || !logits)) return fail(AM_EINVAL, "NULL x or logits");
  if (!aligned(params, 16) || !aligned(x, 16) || !aligned(logits, 16) || !aligned(ws, 256))
    return fail(AM_EINVAL, "params, x, logits must be 16-byte and ws 256-byte aligned");
  const TeacherWs w = teacher_ws_layout(m, T, B, sc.N);
  if (ws_bytes < w.total)
    return fail(AM_EWORKSPACE, "teacher forward needs %lld workspace bytes", (long long)w.total);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf = m->dtype == AM_BF16;
  const int64_t e = esz_of(m->dtype), H = m->hidden, G = 4 * H, L = m->layers;
  const TeacherOffsets po = teacher_layout(m);
  const char* P8 = static_cast<const char*>(params);
  const int N = (int)sc.N;

  // schedule tables for the time reversal (built on the device from the
  // lengths passed by value); a zero initial cell state
  {
    am::SchedTables st;
    memset(&st, 0, sizeof st);
    st.T = T; st.B = B;
    for (int b = 0; b < B; ++b) st.len[b] = (uint16_t)sc.lens[b];
    st.offs = at<int64_t>(ws, w.offs);
    st.lens = at<int32_t>(ws, w.lens);
    AM_TRY(hip_check(am::schedule_tables(st, s), "schedule tables"));
  }
  AM_TRY(hip_check(am::fill_zero2(at<float>(ws, w.c0), B * H, at<float>(ws, w.sync),
                                  2 * L * sync_rounds(B) * SYNC_BYTES / 4, s), "c0 and sync clear"));
  auto gather = [&](const void* src, int64_t src_ld, void* dst, int64_t dst_ld, int64_t col,
                    int width, bool reverse) {
    am::GatherRows g;
    g.src = src; g.src_ld = src_ld; g.dst = dst; g.dst_ld = dst_ld; g.dst_col = col;
    g.width = width; g.N = sc.N; g.T = T;
    g.offs = at<int64_t>(ws, w.offs); g.lens = at<int32_t>(ws, w.lens);
    g.reverse = reverse ? 1 : 0;
    Timed tm(AM_K_MISC, s, 0.0, 2.0 * sc.N * width * e);
    return hip_check(am::gather_rows(g, bf, s), "gather rows");
  };

  for (int l = 0; l < L; ++l) {
    const int64_t D = l == 0 ? m->input_dim : 2 * H;
    const void* X = l == 0 ? x : at<void>(ws, (l - 1) % 2 ? w.cat1 : w.cat0);
    void* out = at<void>(ws, l % 2 ? w.cat1 : w.cat0);
    for (int d = 0; d < 2; ++d) {
      const int k = 2 * l + d;
      const void* in = X;
      if (d == 1) {  // the backward direction reads the sequences reversed
        AM_TRY(gather(X, D, at<void>(ws, w.rev), D, 0, (int)D, true));
        in = at<void>(ws, w.rev);
      }
      AM_TRY(run_gemm(AM_K_GEMM_FWD,
                      mk_gemm(in, D, true, P8 + po.wx[k] * e, D, true, at<void>(ws, w.p), G, false,
                              P8 + po.b[k] * e, N, (int)G, (int)D, bf), s));
      FwdLayer f;
      f.P = at<void>(ws, w.p);
      f.Wh = P8 + po.wh[k] * e;
      f.h0 = nullptr;
      f.c0 = at<float>(ws, w.c0);
      f.H = at<void>(ws, w.hdir);
      f.Hs = at<void>(ws, w.hs);
      f.C = at<float>(ws, w.c);
      f.G = at<void>(ws, w.g);
      f.sync = sync_slot(at<void>(ws, w.sync), k, B);
      f.err = sync_err(at<void>(ws, w.sync));
      f.pre = at<float>(ws, w.pre);
      AM_TRY(forward_recurrence(f, sc, bf, H, s));
      AM_TRY(gather(at<void>(ws, w.hdir), H, out, 2 * H, d * H, (int)H, d == 1));
    }
  }
  return run_gemm(AM_K_GEMM_FWD,
                  mk_gemm(at<void>(ws, (L - 1) % 2 ? w.cat1 : w.cat0), 2 * H, true, P8 + po.wo * e,
                          2 * H, true, logits, m->classes, true, P8 + po.bo * e, N, m->classes,
                          (int)(2 * H), bf), s);
}

am_status kbest_logits(int64_t N, int32_t C, int32_t K, const float* logits, int32_t* idx,
                       float* val, void* stream) {
  if (N < 0 || C < 1 || K < 0 || K > C) return fail(AM_EINVAL, "need N >= 0, C >= 1, 0 <= K <= C");
  if (K > 64) return fail(AM_EUNSUPPORTED, "K > 64");
  if (C > 8192) return fail(AM_EUNSUPPORTED, "C > 8192");
  if (N > 0 && K > 0 && (!logits || !idx || !val)) return fail(AM_EINVAL, "NULL pointer");
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_MISC, s, 0.0, (double)N * (4.0 * C + 8.0 * K));
  return hip_check(am::topk_rows(N, C, K, logits, idx, val, s), "kbest_logits");
}

am_status kbest_posteriors(int64_t N, int32_t K, const float* val, float* prob, void* stream) {
  if (N < 0 || K < 0) return fail(AM_EINVAL, "need N >= 0 and K >= 0");
  if (N > 0 && K > 0 && (!val || !prob)) return fail(AM_EINVAL, "NULL pointer");
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_MISC, s, 0.0, (double)N * 8.0 * K);
  return hip_check(am::kbest_posteriors(N, K, val, prob, s), "kbest_posteriors");
}

am_status sparse_soft_ce(int64_t N, int32_t C, int32_t K, const float* logits, const int32_t* idx,
                         const float* prob, const uint8_t* mask, int32_t reduction, float* loss,
                         void* dlogits, int32_t dlogits_dtype, void* ws, int64_t ws_bytes,
                         void* stream) {
  if (N < 0 || C < 1 || K < 0) return fail(AM_EINVAL, "need N >= 0, C >= 1, K >= 0");
  if (C % 4) return fail(AM_EUNSUPPORTED, "C must be a multiple of 4");
  if (C > 8192) return fail(AM_EUNSUPPORTED, "C > 8192 classes");
  if (reduction != AM_MEAN_VALID && reduction != AM_SUM) return fail(AM_EINVAL, "unknown reduction");
  if (dlogits_dtype != AM_F32 && dlogits_dtype != AM_BF16) return fail(AM_EINVAL, "unknown dlogits dtype");
  if (!loss) return fail(AM_EINVAL, "loss is NULL");
  if (N > 0 && (!logits || !dlogits || (K > 0 && (!idx || !prob))))
    return fail(AM_EINVAL, "NULL pointer");
  if (!aligned(logits, 16) || !aligned(dlogits, dlogits_dtype == AM_BF16 ? 8 : 16))
    return fail(AM_EINVAL, "logits / dlogits must be 16-byte aligned");
  const int64_t need = am_ce_workspace_bytes(N);
  if (!ws || ws_bytes < need || !aligned(ws, 256))
    return fail(AM_EWORKSPACE, "soft_ce needs %lld workspace bytes (256-aligned)", (long long)need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (debug_checks() && N > 0 && K > 0) {
    // every target index in [-1, C): copied to the host after the work
    // queued before this call, then checked
    std::vector<int32_t> h((size_t)(N * K));
    AM_TRY(hip_check(hipMemcpyAsync(h.data(), idx, h.size() * 4, hipMemcpyDeviceToHost, s),
                     "AM_DEBUG index copy"));
    AM_TRY(hip_check(hipStreamSynchronize(s), "AM_DEBUG stream sync"));
    for (size_t i = 0; i < h.size(); ++i)
      if (h[i] < -1 || h[i] >= C)
        return fail(AM_EINVAL, "target index %d of row %lld, slot %lld outside [-1, %d)", h[i],
                    (long long)(i / K), (long long)(i % K), C);
  }
  am::SoftCeArgs a;
  a.N = N; a.C = C; a.K = K; a.z = logits; a.idx = idx; a.prob = prob; a.mask = mask;
  a.reduction = reduction; a.loss = loss; a.dz = dlogits; a.dz_bf16 = dlogits_dtype == AM_BF16;
  a.n_partials = am::soft_ce_partials(N);
  a.ws_partials = at<float>(ws, 0);
  a.ws_scale = at<float>(ws, align256(a.n_partials * 4));
  const double bytes = (double)N * C * (4 + (a.dz_bf16 ? 2 : 4)) + (double)N * K * 8;
  Timed tm(AM_K_CE, s, 0.0, bytes);
  return hip_check(am::soft_ce(a, s), "sparse_soft_ce");
}

am_status lstm_am_forward(const am_model* m, const void* params, const void* x,
                          const int32_t* lengths, const float* h0, const float* c0, int32_t T,
                          int32_t B, float* logits, float* hT, float* cT, void* ws,
                          int64_t ws_bytes, void* stream) {
  AM_TRY(check_model(m));
  Schedule sc;
  AM_TRY(make_schedule(T, B, lengths, sc));
  if (!params || !ws) return fail(AM_EINVAL, "NULL params or workspace");
  if (sc.N > 0 && (!x || !logits)) return fail(AM_EINVAL, "NULL x or logits");
  if (!aligned(params, 16) || !aligned(x, 16) || !aligned(logits, 16) || !aligned(ws, 256))
    return fail(AM_EINVAL, "params, x, logits must be 16-byte and ws 256-byte aligned");
  const WsLayout w = ws_layout(m, B, sc.N);
  if (ws_bytes < w.total)
    return fail(AM_EWORKSPACE, "forward needs %lld workspace bytes", (long long)w.total);

  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf = m->dtype == AM_BF16;
  const int64_t e = esz_of(m->dtype), H = m->hidden, G = 4 * H, L = m->layers;
  const Offsets po = param_layout(m);
  const char* P8 = static_cast<const char*>(params);

  // initial cell state (copied, or zero) and initial hidden state (converted)
  {
    Timed tm(AM_K_MISC, s, 0.0, 8.0 * L * B * H);
    float* c0w = at<float>(ws, w.c0);
    // a new forward + backward pair: every slot of the sync area and the
    // barrier time-out flag with it
    AM_TRY(hip_check(am::init_state(at<float>(ws, w.sync), 2 * L * sync_rounds(B) * SYNC_BYTES / 4, c0, c0w,
                                    h0, at<void>(ws, w.h0), L * B * H, bf, s), "initial state"));
  }

  // few sequences: every layer in one launch behind the first projection
  const bool pipe = sc.N > 0 && pipe_shape(bf, H, L, T, B, is_varlen(sc));
  bool piped = false;
  for (int l = 0; l < L && !piped; ++l) {
    const int64_t D = l == 0 ? m->input_dim : H;
    const void* X = l == 0 ? x : at<void>(ws, w.h[l - 1]);
    void* P = at<void>(ws, w.p_da);
    AM_TRY(run_gemm(AM_K_GEMM_FWD,
                    mk_gemm(X, D, true, P8 + po.wx[l] * e, D, true, P, G, false, P8 + po.b[l] * e,
                            (int)sc.N, (int)G, (int)D, bf), s));
    if (pipe && l == 0) {
      am::PipeFwd pf{};
      for (int k = 0; k < L; ++k) {
        am::PipeLayer& q = pf.l[k];
        q.Wh = P8 + po.wh[k] * e;
        q.WxN = k + 1 < L ? P8 + po.wx[k + 1] * e : nullptr;
        q.bN = k + 1 < L ? P8 + po.b[k + 1] * e : nullptr;
        q.h0 = h0 ? at<char>(ws, w.h0) + (int64_t)k * B * H * e : nullptr;
        q.c0 = at<float>(ws, w.c0) + (int64_t)k * B * H;
        q.H = at<void>(ws, w.h[k]);
        q.Hs = at<void>(ws, w.hs[k]);
        q.C = at<float>(ws, w.c[k]);
        q.G = at<void>(ws, w.g[k]);
      }
      pf.P = P;
      pf.layers = (int)L;
      pf.hidden = (int)H;
      void* area = at<void>(ws, w.sync);
      const double nl = (double)sc.N * L;
      Timed tm(AM_K_LSTM_FWD, s, 2.0 * nl * G * H + 2.0 * (nl - sc.N) * G * H,
               nl * (G * e * 2 + H * (2 * e + 4)) + 2.0 * L * G * H * e);
      AM_TRY(hip_check(am::lstm_fwd_pipe_launch(pf, persist_schedule(sc),
                                                xcd_sync(sync_slot(area, 0, B), sync_err(area)), s, &piped),
                       "lstm forward, all layers"));
      if (piped) break;
      tm.cancel();
    }
    FwdLayer f;
    f.P = at<void>(ws, w.p_da);
    f.Wh = P8 + po.wh[l] * e;
    f.h0 = h0 ? at<char>(ws, w.h0) + (int64_t)l * B * H * e : nullptr;
    f.c0 = at<float>(ws, w.c0) + (int64_t)l * B * H;
    f.H = at<void>(ws, w.h[l]);
    f.Hs = at<void>(ws, w.hs[l]);
    f.C = at<float>(ws, w.c[l]);
    f.G = at<void>(ws, w.g[l]);
    f.sync = sync_slot(at<void>(ws, w.sync), l, B);
    f.err = sync_err(at<void>(ws, w.sync));
    f.pre = at<float>(ws, w.pre);
    AM_TRY(forward_recurrence(f, sc, bf, H, s));
  }
  AM_TRY(run_gemm(AM_K_GEMM_FWD,
                  mk_gemm(at<void>(ws, w.h[L - 1]), H, true, P8 + po.wo * e, H, true, logits,
                          m->classes, true, P8 + po.bo * e, (int)sc.N, m->classes, (int)H, bf), s));

  if (hT || cT) {
    for (int b0 = 0; b0 < B; b0 += 256) {
      am::GatherState g;
      g.Hrows = at<void>(ws, w.h[0]);
      g.h_bf16 = bf;
      g.Crows = at<float>(ws, w.c[0]);
      g.layer_bytes = L > 1 ? w.h[1] - w.h[0] : 0;  // (every layer's regions are laid out alike)
      g.h0 = h0;
      g.c0 = c0;
      g.hT = hT;
      g.cT = cT;
      g.layers = (int)L;
      g.B = B;
      g.hidden = (int)H;
      const int nb = B - b0 < 256 ? B - b0 : 256;
      for (int i = 0; i < nb; ++i) {
        const int len = sc.lens[b0 + i];
        g.rows[i] = len > 0 ? (int)(sc.offs[len - 1] + b0 + i) : -1;
      }
      Timed tm(AM_K_MISC, s, 0.0, 16.0 * L * nb * H);
      AM_TRY(hip_check(am::gather_state(g, b0, nb, s), "final state"));
    }
  }
  return AM_OK;
}

am_status lstm_am_backward(const am_model* m, const void* params, const void* x,
                           const int32_t* lengths, int32_t T, int32_t B, const void* dlogits,
                           void* ws, int64_t ws_bytes, float* grads, void* stream) {
  AM_TRY(check_model(m));
  Schedule sc;
  AM_TRY(make_schedule(T, B, lengths, sc));
  if (!params || !ws || !grads) return fail(AM_EINVAL, "NULL params, workspace or grads");
  if (sc.N > 0 && (!x || !dlogits)) return fail(AM_EINVAL, "NULL x or dlogits");
  if (!aligned(params, 16) || !aligned(x, 16) || !aligned(dlogits, 16) || !aligned(grads, 16) ||
      !aligned(ws, 256))
    return fail(AM_EINVAL, "params, x, dlogits, grads must be 16-byte and ws 256-byte aligned");
  const WsLayout w = ws_layout(m, B, sc.N);
  if (ws_bytes < w.total)
    return fail(AM_EWORKSPACE, "backward needs %lld workspace bytes", (long long)w.total);

  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf = m->dtype == AM_BF16;
  const int64_t e = esz_of(m->dtype), H = m->hidden, G = 4 * H, L = m->layers, Cc = m->classes;
  const int N = (int)sc.N;
  const Offsets po = param_layout(m);
  const char* P8 = static_cast<const char*>(params);
  float* skws = at<float>(ws, w.splitk);
  // the backward launches' slots of the sync area (not slot 0's time-out flag)
  AM_TRY(hip_check(am::fill_zero(static_cast<float*>(sync_slot(at<void>(ws, w.sync), (int)L, B)),
                                 L * sync_rounds(B) * SYNC_BYTES / 4, s), "sync clear"));

  // output layer: dWo = dZ^T H_top and dbo = column sums of dZ (one pass),
  // then dH_top = dZ Wo
  AM_TRY(run_gemm(AM_K_GEMM_BWD_WGT,
                  mk_wgrad(dlogits, Cc, at<void>(ws, w.h[L - 1]), H, (int)H, nullptr, 0, 0,
                           grads + po.wo, H, nullptr, 0, grads + po.bo, (int)Cc, N, bf, skws,
                           w.splitk_floats), s));
  void* DH = at<void>(ws, w.dh);
  AM_TRY(run_gemm(AM_K_GEMM_BWD_DATA,
                  mk_gemm(dlogits, Cc, true, P8 + po.wo * e, H, false, DH, H, false, nullptr, N,
                          (int)H, (int)Cc, bf), s));

  char* dA = at<char>(ws, w.p_da);
  auto wht = [&](int l) { return static_cast<void*>(at<char>(ws, w.wht) + (int64_t)l * G * H * e); };
  float* dc = at<float>(ws, w.dc);
  // the XCD-local recurrences read W_h^T: every layer's, transposed up front
  // in one launch (falls back to one transpose per layer below)
  int fused_steps = 0;  // steps that the one-launch step would take
  for (int t = 0; t < T; ++t)
    fused_steps += am::lstm_bwd_step_fused_covers((int)H, (int)sc.counts[t]);
  bool wht_ready = false;
  if (sc.N > 0 && xcd_path(bf, H, sc) && !solo_shape(bf, H, T, B, is_varlen(sc))) {
    Timed tm(AM_K_MISC, s, 0.0, 2.0 * L * G * H * e);
    wht_ready = true;
    for (int l0 = 0; l0 < L && wht_ready; l0 += am::TransposeBatch::MAX) {
      am::TransposeBatch tb{};
      const int n = (int)(L - l0 < am::TransposeBatch::MAX ? L - l0 : am::TransposeBatch::MAX);
      for (int i = 0; i < n; ++i) {
        tb.src[i] = P8 + po.wh[l0 + i] * e;
        tb.dst[i] = wht(l0 + i);
      }
      const hipError_t err = am::transpose_bf16_batch(tb, n, (int)G, (int)H, s);
      if (err == hipErrorInvalidValue) wht_ready = false;  // (alignment) per layer instead
      else AM_TRY(hip_check(err, "Wh transposes"));
    }
    if (!wht_ready) tm.cancel();
  }
  for (int l = L - 1; l >= 0; --l) {
    void* WhT = wht(l);
    const int64_t D = l == 0 ? m->input_dim : H;
    const char* Gl = at<char>(ws, w.g[l]);
    const float* Cl = at<float>(ws, w.c[l]);
    bool used = false;
    if (sc.N > 0 && persistent_enabled()) {
      am::PersistBwd pa;
      pa.Wh = P8 + po.wh[l] * e;
      pa.WhT = WhT;
      pa.dHa = DH;
      pa.G = Gl;
      pa.C = Cl;
      pa.c0 = at<float>(ws, w.c0) + (int64_t)l * B * H;
      pa.dA = dA;
      void* slot = sync_slot(at<void>(ws, w.sync), (int)L + l, B);
      pa.counters = static_cast<unsigned*>(slot);
      pa.err = sync_err(at<void>(ws, w.sync));
      pa.hidden = (int)H;
      const am::PersistSchedule ps = persist_schedule(sc);
      const double flops = 2.0 * (sc.N - sc.counts[0]) * G * H;
      const double bytes = (double)sc.N * (G * e * 2 + H * (e + 8)) + (double)G * H * e;
      if (solo_shape(bf, H, T, B, ps.varlen != 0)) {
        Timed tm(AM_K_LSTM_BWD, s, flops, bytes);
        used = true;
        AM_TRY(hip_check(am::lstm_bwd_solo_launch(pa, ps, bf, s), "lstm backward layer (solo)"));
      } else if (xcd_path(bf, H, sc)) {
        if (!wht_ready) {
          Timed tm(AM_K_MISC, s, 0.0, 2.0 * G * H * e);
          AM_TRY(hip_check(am::transpose(P8 + po.wh[l] * e, WhT, (int)G, (int)H, bf, s), "Wh transpose"));
        }
        Timed tm(AM_K_LSTM_BWD, s, flops, bytes);
        AM_TRY(hip_check(am::lstm_bwd_xcd_launch(pa, ps, xcd_sync(slot, pa.err), s, &used),
                         "lstm backward layer (xcd)"));
        if (!used) tm.cancel();
      }
      if (!used && device_persistent_enabled() && am::lstm_persistent_fits(false, (int)H, B, bf, T)) {
        Timed tm(AM_K_LSTM_BWD, s, flops, bytes);
        AM_TRY(hip_check(am::lstm_bwd_persistent(pa, ps, bf, s, &used), "lstm backward layer"));
        if (!used) tm.cancel();
      }
    }
    // (per step in bf16: the fused step reads W_h^T, the split product W_h)
    const bool fused = !used && bf && am::lstm_bwd_fused_pays((int)H, fused_steps);
    if (!used && (!bf || fused)) {
      Timed tm(AM_K_MISC, s, 0.0, 2.0 * G * H * e);
      AM_TRY(hip_check(am::transpose(P8 + po.wh[l] * e, WhT, (int)G, (int)H, bf, s), "Wh transpose"));
    }
    for (int t = T - 1; t >= 0 && !used; --t) {
      const int64_t nb = sc.counts[t];
      if (nb == 0) continue;
      const int64_t nbn = t + 1 < T ? sc.counts[t + 1] : 0;
      const int64_t o = sc.offs[t];
      am::LstmBwdStep a;
      a.dAnext = nbn > 0 ? dA + sc.offs[t + 1] * G * e : nullptr;
      a.nbn = (int)nbn;
      a.WhT = WhT;
      a.dHa = static_cast<char*>(DH) + o * H * e;
      a.G = Gl + o * G * e;
      a.C = Cl + o * H;
      a.Cprev = t == 0 ? at<float>(ws, w.c0) + (int64_t)l * B * H : Cl + sc.offs[t - 1] * H;
      a.dc = dc;
      a.dA = dA + o * G * e;
      a.nb = (int)nb;
      a.hidden = (int)H;
      a.bf16 = bf;
      if (fused && am::lstm_bwd_step_fused_covers((int)H, (int)nb)) {
        Timed tm(AM_K_LSTM_BWD, s, 2.0 * nbn * G * H,
                 (double)(nbn * G + G * H) * e + (double)nb * (H * (e + 16.0) + G * 2 * e));
        AM_TRY(hip_check(am::lstm_bwd_step_fused_launch(a, s), "lstm backward step (fused)"));
        continue;
      }
      if (bf) {
        // dA_{t+1} Wh as a batched product (few rows: square tiles), then
        // the cell backward
        // (k split up to STEP_SPLITS ways: the partials fill the fp32 scratch)
        float* dhrec = at<float>(ws, w.pre);
        int splits = 0;
        if (nbn > 0) {
          const am::GemmArgs g = mk_gemm(a.dAnext, G, true, P8 + po.wh[l] * e, H, false, dhrec, H,
                                         true, nullptr, (int)nbn, (int)H, (int)G, true);
          Timed tm(AM_K_LSTM_BWD, s, 2.0 * nbn * H * G, gemm_bytes(nbn, H, G, e, 4));
          AM_TRY(hip_check(am::gemm_bf16_splitk_rows(g, STEP_SPLITS, dhrec, &splits, s), "recurrent product"));
        }
        Timed tm(AM_K_LSTM_BWD, s, 0.0, (double)nb * (H * (4.0 * (splits > 0 ? splits : 1) + e + 16) + G * 2 * e));
        AM_TRY(hip_check(am::lstm_cell_bwd(nbn > 0 ? dhrec : nullptr, splits, a, s), "lstm backward cell"));
        continue;
      }
      const double bytes = (double)(nbn * G + G * H + nb * H + nb * G) * e +
                           nb * H * 12.0 + (double)nb * G * e;
      Timed tm(AM_K_LSTM_BWD, s, 2.0 * nbn * G * H, bytes);
      AM_TRY(hip_check(am::lstm_bwd_step(a, s), "lstm backward step"));
    }
    const void* X = l == 0 ? x : at<void>(ws, w.h[l - 1]);
    // [dWx | dWh] = dA^T [X | Hs] and db = column sums of dA, one pass
    AM_TRY(run_gemm(AM_K_GEMM_BWD_WGT,
                    mk_wgrad(dA, G, X, D, (int)D, at<void>(ws, w.hs[l]), H, (int)H,
                             grads + po.wx[l], D, grads + po.wh[l], H, grads + po.b[l], (int)G, N,
                             bf, skws, w.splitk_floats), s));
    if (l > 0)
      AM_TRY(run_gemm(AM_K_GEMM_BWD_DATA,
                      mk_gemm(dA, G, true, P8 + po.wx[l] * e, D, false, DH, H, false, nullptr, N,
                              (int)H, (int)G, bf), s));
  }
  // a step barrier of this forward + backward pair that timed out leaves the
  // gradient invalid: it is replaced by zeros on the device, so that a caller
  // that encodes and applies it before am_workspace_check adds nothing to
  // its residual or weights
  Timed tm(AM_K_MISC, s, 0.0, 4.0);
  return hip_check(am::zero_if_set(sync_err(at<void>(ws, w.sync)), grads, po.n, s), "time-out guard");
}

// ------------------------------------------- gated linear recurrences --

int64_t am_gated_recurrence_workspace_bytes(int32_t T, int32_t B, int32_t H, int32_t varlen, int32_t train) {
  if (T < 0 || B < 1 || H < 1) return -1;
  return gated_layout(T, B, H, varlen != 0, train != 0).total;
}

am_status gated_recurrence_forward(int32_t T, int32_t B, int32_t H, int32_t dtype, const int32_t* lengths,
                                   const void* x, const void* r, const void* i, int64_t ld, const float* lam,
                                   float c, const float* h0, void* h, float* hT, int32_t train, void* ws,
                                   int64_t ws_bytes, void* stream) {
  am::GatedRecurrence a{};
  GatedLayout l;
  AM_TRY(check_gated(T, B, H, dtype, lengths, lam, c, train != 0, ws, ws_bytes, a, l));
  AM_TRY(check_rows(a.N, H, dtype, x, ld, "x", B));
  AM_TRY(check_rows(a.N, H, dtype, r, ld, "r", B));
  AM_TRY(check_rows(a.N, H, dtype, i, ld, "i", B));
  AM_TRY(check_rows(a.N, H, dtype, h, H, "h", B));
  if (!aligned(h0, 4) || !aligned(hT, 4)) return fail(AM_EINVAL, "h0 and hT must be 4-byte aligned");
  a.x = x; a.r = r; a.i = i;
  a.ld = ld;
  a.h0 = h0;
  a.h = h;
  a.hT = hT;
  if (train) a.saved = at<float>(ws, l.saved);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_GATED, s, 20.0 * a.N * H, 4.0 * esz_of(dtype) * a.N * H + 8.0 * B * H);
  return hip_check(am::gated_forward(a, lengths, dtype == AM_BF16, s), "gated recurrence");
}

am_status gated_recurrence_backward(int32_t T, int32_t B, int32_t H, int32_t dtype, const int32_t* lengths,
                                    const void* x, const void* r, const void* i, int64_t ld, const float* lam,
                                    float c, const void* dh, int64_t lddh, const float* dhT, void* dx, void* dr,
                                    void* di, int64_t ldd, float* dlam, float* dh0, void* ws,
                                    int64_t ws_bytes, void* stream) {
  am::GatedRecurrence a{};
  GatedLayout l;
  AM_TRY(check_gated(T, B, H, dtype, lengths, lam, c, true, ws, ws_bytes, a, l));
  AM_TRY(check_rows(a.N, H, dtype, x, ld, "x", B));
  AM_TRY(check_rows(a.N, H, dtype, r, ld, "r", B));
  AM_TRY(check_rows(a.N, H, dtype, i, ld, "i", B));
  AM_TRY(check_rows(a.N, H, dtype, dh, lddh, "dh", B));
  AM_TRY(check_rows(a.N, H, dtype, dx, ldd, "dx", B));
  AM_TRY(check_rows(a.N, H, dtype, dr, ldd, "dr", B));
  AM_TRY(check_rows(a.N, H, dtype, di, ldd, "di", B));
  if (!dlam) return fail(AM_EINVAL, "NULL dlam");
  if (!aligned(dhT, 4) || !aligned(dh0, 4) || !aligned(dlam, 4))
    return fail(AM_EINVAL, "dhT, dh0 and dlam must be 4-byte aligned");
  a.x = x; a.r = r; a.i = i; a.dh = dh;
  a.dx = dx; a.dr = dr; a.di = di;
  a.ld = ld;
  a.lddh = lddh;
  a.ldd = ldd;
  a.dhT = dhT;
  a.dh0 = dh0;
  a.dlam = dlam;
  a.saved = at<float>(ws, l.saved);
  a.parts = at<float>(ws, l.parts);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_GATED, s, 40.0 * a.N * H, 7.0 * esz_of(dtype) * a.N * H + 8.0 * B * H);
  return hip_check(am::gated_backward(a, dtype == AM_BF16, s), "gated recurrence backward");
}

int64_t am_gated_delta_workspace_bytes(int32_t T, int32_t B, int32_t heads, int32_t key_heads, int32_t dk,
                                       int32_t dv, int32_t dtype, int32_t varlen, int32_t train) {
  if (!delta_sizes(T, B, heads, key_heads, dk, dv) || dk > am::GD_MAX_DIM || dv > am::GD_MAX_DIM) return -1;
  if ((dtype != AM_F32 && dtype != AM_BF16) || T > (1 << 30) || (int64_t)T * B >= (1ll << 32) || (varlen && B > 1024)) return -1;
  if (!delta_heads(T, B, heads, train != 0) || (!varlen && (int64_t)T * B >= (1ll << 31) - 256)) return -1;
  return delta_layout(T, B, heads, dk, dv, varlen != 0, train != 0).total;
}

am_status gated_delta_forward(int32_t T, int32_t B, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv,
                              int32_t dtype, const int32_t* lengths, const void* q, int64_t ldq, const void* k,
                              int64_t ldk, const void* v, int64_t ldv, const void* r, int64_t ldr,
                              const void* b, int64_t ldb, const float* lam, float c, float eps,
                              const float* s0, void* o, int64_t ldo, float* sT, int32_t train, void* ws,
                              int64_t ws_bytes, void* stream) {
  am::GatedDelta a{};
  DeltaLayout l;
  AM_TRY(check_delta(T, B, heads, key_heads, dk, dv, dtype, lengths, q, ldq, k, ldk, v, ldv, r, ldr, b, ldb,
                     lam, c, eps, s0, train != 0, ws, ws_bytes, a, l));
  AM_TRY(check_rows(a.N, heads * dv, dtype, o, ldo, "o"));
  if (!aligned(sT, 4)) return fail(AM_EINVAL, "states must be 4-byte aligned");
  a.o = o;
  a.ldo = ldo;
  a.sT = sT;
  a.train = train != 0;
  if (train) a.saved = at<float>(ws, l.saved);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_GATED, s, 6.0 * a.N * heads * dk * dv,
           (double)esz_of(dtype) * a.N * (2.0 * key_heads * dk + 2.0 * heads * dv + 2.0 * heads) + 8.0 * B * heads * dk * dv);
  if (lengths) {
    am::GatedSchedule g{};
    g.offs = at<int32_t>(ws, l.offs);
    g.lens = at<int32_t>(ws, l.lens);
    g.tails = at<int32_t>(ws, l.tails);
    g.T = a.T;
    g.B = B;
    AM_TRY(hip_check(am::gated_schedule(g, lengths, s), "gated delta schedule"));
  }
  return hip_check(am::gated_delta_forward(a, dtype == AM_BF16, s), "gated delta rule");
}

am_status gated_delta_backward(int32_t T, int32_t B, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv,
                               int32_t dtype, const int32_t* lengths, const void* q, int64_t ldq, const void* k,
                               int64_t ldk, const void* v, int64_t ldv, const void* r, int64_t ldr,
                               const void* b, int64_t ldb, const float* lam, float c, float eps,
                               const float* s0, const void* d_o, int64_t lddo, const float* dsT, void* dq,
                               int64_t lddq, void* dk_, int64_t lddk, void* dv_, int64_t lddv, void* dr,
                               int64_t lddr, void* db, int64_t lddb, float* dlam, float* ds0, void* ws,
                               int64_t ws_bytes, void* stream) {
  am::GatedDelta a{};
  DeltaLayout l;
  AM_TRY(check_delta(T, B, heads, key_heads, dk, dv, dtype, lengths, q, ldq, k, ldk, v, ldv, r, ldr, b, ldb,
                     lam, c, eps, s0, true, ws, ws_bytes, a, l));
  AM_TRY(check_rows(a.N, heads * dv, dtype, d_o, lddo, "d_o"));
  AM_TRY(check_rows(a.N, key_heads * dk, dtype, dq, lddq, "dq"));
  AM_TRY(check_rows(a.N, key_heads * dk, dtype, dk_, lddk, "dk"));
  AM_TRY(check_rows(a.N, heads * dv, dtype, dv_, lddv, "dv"));
  AM_TRY(check_rows(a.N, heads, dtype, dr, lddr, "dr"));
  AM_TRY(check_rows(a.N, heads, dtype, db, lddb, "db"));
  if (!dlam || !aligned(dlam, 4)) return fail(AM_EINVAL, "NULL or unaligned dlam");
  if (!aligned(dsT, 4) || !aligned(ds0, 4)) return fail(AM_EINVAL, "states must be 4-byte aligned");
  a.train = true;
  a.d_o = d_o; a.lddo = lddo;
  a.dq = dq; a.dk_ = dk_; a.dv_ = dv_; a.dr = dr; a.db = db;
  a.lddq = lddq; a.lddk = lddk; a.lddv = lddv; a.lddr = lddr; a.lddb = lddb;
  a.dsT = dsT;
  a.ds0 = ds0;
  a.dlam = dlam;
  a.saved = at<float>(ws, l.saved);
  a.dsaved = at<float>(ws, l.dsaved);
  a.u = at<uint16_t>(ws, l.u);
  a.dr_rows = at<uint16_t>(ws, l.dr);
  a.parts = at<float>(ws, l.parts);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_GATED, s, 12.0 * a.N * heads * dk * dv,
           (double)esz_of(dtype) * a.N * (4.0 * key_heads * dk + 3.0 * heads * dv + 4.0 * heads) + 8.0 * B * heads * dk * dv);
  return hip_check(am::gated_delta_backward(a, dtype == AM_BF16, s), "gated delta rule backward");
}

am_status gated_norm_forward(int64_t N, int32_t H, int32_t dtype, int32_t res_dtype, const void* o,
                             int64_t ldo, const void* gate, int64_t ldg, const float* w_post,
                             const float* scale, const void* res, const float* w_next, float eps,
                             void* res_out, void* y, float* rstd, void* stream) {
  am::GatedNorm a{};
  AM_TRY(check_norm(N, H, dtype, res_dtype, o, ldo, gate, ldg, w_post, scale, res, w_next, eps, a));
  if (o) AM_TRY(check_rows(N, H, res_dtype, res_out, H, "res_out"));
  else if (N > 0 && res_out) return fail(AM_EINVAL, "res_out without o");
  if (w_next) AM_TRY(check_rows(N, H, dtype, y, H, "y"));
  else if (y) return fail(AM_EINVAL, "y without w_next");
  if (!aligned(rstd, 4)) return fail(AM_EINVAL, "rstd must be 4-byte aligned");
  a.res_out = res_out;
  a.y = y;
  a.rstd = rstd;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_NORM, s, 16.0 * N * H, norm_bytes(a, dtype, res_dtype, false));
  return hip_check(am::gated_norm_forward(a, dtype == AM_BF16, res_dtype == AM_BF16, s), "gated norm");
}

int64_t am_gated_norm_workspace_bytes(int64_t N, int32_t H) {
  if (N < 0 || H < 1 || H > am::GATED_NORM_MAX_H) return -1;
  return align256((int64_t)am::GATED_NORM_BLOCKS * 2 * H * 4);
}

am_status gated_norm_backward(int64_t N, int32_t H, int32_t dtype, int32_t res_dtype, const void* o,
                              int64_t ldo, const void* gate, int64_t ldg, const float* w_post,
                              const float* scale, const void* res, const float* w_next, float eps,
                              const float* rstd, const void* dy, const void* dres_out, void* d_o,
                              int64_t lddo, void* dgate, int64_t lddg, void* dres, float* dw_post,
                              float* dscale, float* dw_next, void* ws, int64_t ws_bytes, void* stream) {
  am::GatedNorm a{};
  AM_TRY(check_norm(N, H, dtype, res_dtype, o, ldo, gate, ldg, w_post, scale, res, w_next, eps, a));
  if (N > 0 && (!rstd || !aligned(rstd, 4))) return fail(AM_EINVAL, "NULL or unaligned rstd");
  if (w_next) AM_TRY(check_rows(N, H, dtype, dy, H, "dy"));
  else if (dy) return fail(AM_EINVAL, "dy without w_next");
  if (dres_out) AM_TRY(check_rows(N, H, res_dtype, dres_out, H, "dres_out"));
  AM_TRY(check_rows(N, H, res_dtype, dres, H, "dres"));
  if (o) AM_TRY(check_rows(N, H, dtype, d_o, lddo, "d_o"));
  else if (N > 0 && d_o) return fail(AM_EINVAL, "d_o without o");
  if (gate) AM_TRY(check_rows(N, H, dtype, dgate, lddg, "dgate"));
  else if (N > 0 && dgate) return fail(AM_EINVAL, "dgate without gate");
  if ((dw_post && !w_post) || (dscale && !scale) || (dw_next && !w_next))
    return fail(AM_EINVAL, "gradient of a factor that is NULL");
  if ((w_post && !dw_post) || (scale && !dscale) || (w_next && !dw_next))
    return fail(AM_EINVAL, "NULL gradient of w_post, scale or w_next");
  if (!aligned(dw_post, 4) || !aligned(dscale, 4) || !aligned(dw_next, 4))
    return fail(AM_EINVAL, "gradients of the factors must be 4-byte aligned");
  if (!ws || !aligned(ws, 256)) return fail(AM_EWORKSPACE, "NULL or unaligned workspace");
  if (ws_bytes < am_gated_norm_workspace_bytes(N, H))
    return fail(AM_EWORKSPACE, "backward needs %lld workspace bytes",
                (long long)am_gated_norm_workspace_bytes(N, H));
  a.rstd = const_cast<float*>(rstd);
  a.dy = dy;
  a.dres_out = dres_out;
  a.d_o = d_o;
  a.lddo = lddo;
  a.dgate = dgate;
  a.lddg = lddg;
  a.dres = dres;
  a.dw_post = dw_post;
  a.dscale = dscale;
  a.dw_next = dw_next;
  a.parts = static_cast<float*>(ws);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_NORM, s, 44.0 * N * H, norm_bytes(a, dtype, res_dtype, true));
  return hip_check(am::gated_norm_backward(a, dtype == AM_BF16, res_dtype == AM_BF16, s), "gated norm backward");
}

am_status gated_norm_forward_q8(int64_t N, int32_t H, int32_t dtype, int32_t res_dtype, const void* o,
                                int64_t ldo, const void* gate, int64_t ldg, const float* w_post,
                                const float* scale, const void* res, const float* w_next, float eps,
                                void* res_out, void* y, float* rstd, void* codes, int64_t ldc, void* scales,
                                int64_t lds, void* stream) {
  am::GatedNorm a{};
  AM_TRY(check_norm(N, H, dtype, res_dtype, o, ldo, gate, ldg, w_post, scale, res, w_next, eps, a));
  if (!w_next) return fail(AM_EINVAL, "NULL w_next");
  if (o) AM_TRY(check_rows(N, H, res_dtype, res_out, H, "res_out"));
  else if (N > 0 && res_out) return fail(AM_EINVAL, "res_out without o");
  if (y) AM_TRY(check_rows(N, H, dtype, y, H, "y"));
  if (!aligned(rstd, 4)) return fail(AM_EINVAL, "rstd must be 4-byte aligned");
  AM_TRY(check_q8(N, H, codes, ldc, scales, lds, "y"));
  if (N == 0) return AM_OK;
  a.res_out = res_out;
  a.y = y;
  a.rstd = rstd;
  a.codes = static_cast<uint8_t*>(codes);
  a.scales = static_cast<uint8_t*>(scales);
  a.ldc = ldc;
  a.lds = lds;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_NORM, s, 18.0 * N * H,
           norm_bytes(a, dtype, res_dtype, false) + (double)N * H * (1.0 - (y ? 0 : esz_of(dtype))));
  return hip_check(am::gated_norm_forward(a, dtype == AM_BF16, res_dtype == AM_BF16, s), "gated norm");
}

am_status q8_quantise(int64_t rows, int64_t cols, int32_t dtype, const void* x, int64_t ld, int32_t tiles,
                      void* codes, int64_t ldc, void* scales, int64_t lds, void* codes_t, int64_t ldct,
                      void* scales_t, int64_t ldst, void* stream) {
  if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31))
    return fail(AM_EINVAL, "need 0 <= rows, cols < 2^31 (rows=%lld, cols=%lld)", (long long)rows, (long long)cols);
  if (dtype != AM_F32 && dtype != AM_BF16) return fail(AM_EINVAL, "dtype %d unknown", dtype);
  if (tiles != 0 && tiles != 1) return fail(AM_EINVAL, "tiles must be 0 or 1");
  if (!codes != !scales || !codes_t != !scales_t) return fail(AM_EINVAL, "codes without scales, or scales without codes");
  if (rows == 0 || cols == 0) return AM_OK;
  if (!codes && !codes_t) return fail(AM_EINVAL, "neither codes nor codes_t: nothing to do");
  AM_TRY(check_rows(cols > 0 ? rows : 0, (int32_t)cols, dtype, x, ld, "x"));
  if (codes) AM_TRY(check_q8(rows, cols, codes, ldc, scales, lds, "x"));
  if (codes_t) AM_TRY(check_q8(cols, rows, codes_t, ldct, scales_t, ldst, "x transposed"));
  if ((rows + 127) / 128 * ((cols + 127) / 128) >= (1ll << 31)) return fail(AM_EUNSUPPORTED, "matrix too large");
  am::Q8Quantise a{};
  a.rows = rows;
  a.cols = cols;
  a.ld = ld;
  a.x = x;
  a.tiles = tiles != 0;
  a.wide = aligned(x, 16) && ld * esz_of(dtype) % 16 == 0 && cols % 8 == 0;
  a.codes = static_cast<uint8_t*>(codes);
  a.scales = static_cast<uint8_t*>(scales);
  a.ldc = ldc;
  a.lds = lds;
  a.codes_t = static_cast<uint8_t*>(codes_t);
  a.scales_t = static_cast<uint8_t*>(scales_t);
  a.ldct = ldct;
  a.ldst = ldst;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_Q8, s, 4.0 * rows * cols,
           (double)rows * cols * (esz_of(dtype) + (codes ? 1 : 0) + (codes_t ? 1 : 0)));
  return hip_check(am::q8_quantise(a, dtype == AM_BF16, s), "q8 quantise");
}

int64_t am_q8_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  const int64_t most = 1ll << 31;
  if (M < 0 || N < 0 || K < 0 || M >= most || N >= most || K >= most) return -1;
  return M == 0 || N == 0 ? 0 : align256(am::q8_plan(M, N, K).bytes);
}

am_status q8_matmul(int64_t M, int64_t N, int64_t K, const void* a, int64_t lda, const void* a_scales,
                    int64_t ldas, const void* b, int64_t ldb, const void* b_scales, int64_t ldbs,
                    int32_t b_tiles, const float* bias, void* out, int64_t ldo, int32_t accumulate,
                    void* ws, int64_t ws_bytes, void* stream) {
  const int64_t need = am_q8_matmul_workspace_bytes(M, N, K);
  if (need < 0)
    return fail(AM_EINVAL, "need 0 <= M, N, K < 2^31 (M=%lld, N=%lld, K=%lld)", (long long)M, (long long)N, (long long)K);
  if ((b_tiles != 0 && b_tiles != 1) || (accumulate != 0 && accumulate != 1))
    return fail(AM_EINVAL, "b_tiles and accumulate must be 0 or 1");
  if (M == 0 || N == 0) return AM_OK;
  if (K > 0) {  // (without elements of the sum there is nothing to read)
    AM_TRY(check_q8(M, K, a, lda, a_scales, ldas, "a"));
    AM_TRY(check_q8(N, K, b, ldb, b_scales, ldbs, "b"));
  }
  AM_TRY(check_rows(M, (int32_t)N, AM_BF16, out, ldo, "out"));
  if (!aligned(bias, 4)) return fail(AM_EINVAL, "bias must be 4-byte aligned");
  if (lda >= (1 << 24) || ldb >= (1 << 24)) return fail(AM_EUNSUPPORTED, "rows of 2^24 codes or more");
  if ((M + 63) / 64 * ((N + 63) / 64) >= (1ll << 24)) return fail(AM_EUNSUPPORTED, "product too large");
  if (need > 0 && (!ws || !aligned(ws, 256) || ws_bytes < need))
    return fail(AM_EWORKSPACE, "needs %lld workspace bytes, 256-byte aligned", (long long)need);
  am::Q8Matmul m{};
  m.M = M; m.N = N; m.K = K;
  m.a = static_cast<const uint8_t*>(a);
  m.a_scale = static_cast<const uint8_t*>(a_scales);
  m.b = static_cast<const uint8_t*>(b);
  m.b_scale = static_cast<const uint8_t*>(b_scales);
  m.lda = lda; m.ldas = ldas; m.ldb = ldb; m.ldbs = ldbs; m.ldo = ldo;
  m.b_tiles = b_tiles != 0;
  m.accumulate = accumulate != 0;
  m.wide = aligned(out, 16) && ldo % 8 == 0;
  m.bias = bias;
  m.out = static_cast<uint16_t*>(out);
  m.parts = static_cast<float*>(ws);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Timed tm(AM_K_Q8, s, 2.0 * M * N * K, (double)(M + N) * K + 2.0 * M * N * (accumulate ? 2 : 1));
  return hip_check(am::q8_matmul(m, s), "q8 product");
}

am_status adamw_apply(int32_t count, const am_adamw_tensor* tensors, int32_t grad_dtype, int32_t state_bits,
                      double lr, double beta1, double beta2, double eps, int64_t step,
                      const float* grad_scale, uint32_t seed, void* stream) {
  if (count < 0 || (count > 0 && !tensors)) return fail(AM_EINVAL, "bad tensor list");
  if (grad_dtype != AM_F32 && grad_dtype != AM_BF16) return fail(AM_EINVAL, "grad_dtype %d unknown", grad_dtype);
  if (state_bits != 32 && state_bits != 8) return fail(AM_EINVAL, "state_bits must be 32 or 8");
  if (!(lr >= 0.0 && lr <= 3.4e38) || !(eps >= 0.0 && eps <= 3.4e38))
    return fail(AM_EINVAL, "lr and eps must be finite and not negative");
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
    return fail(AM_EINVAL, "beta1 and beta2 must be in [0, 1)");
  if (step < 1) return fail(AM_EINVAL, "step counts from 1");
  if (!aligned(grad_scale, 4)) return fail(AM_EINVAL, "grad_scale must be 4-byte aligned");
  const bool codes = state_bits == 8;
  int64_t all = 0;
  for (int k = 0; k < count; ++k) {
    const am_adamw_tensor& t = tensors[k];
    if (t.n < 0 || t.n >= (1ll << 40)) return fail(AM_EINVAL, "tensor %d: %lld elements", k, (long long)t.n);
    if (!(t.weight_decay >= 0.0 && t.weight_decay <= 3.4e38))
      return fail(AM_EINVAL, "tensor %d: weight_decay must be finite and not negative", k);
    if (t.n == 0) continue;
    if (!t.master || !t.grad || !t.m || !t.v || (codes && (!t.m_scale || !t.v_scale)))
      return fail(AM_EINVAL, "tensor %d: NULL master, grad, moment or scale", k);
    const uintptr_t ga = grad_dtype == AM_BF16 ? 2 : 4, ma = codes ? 1 : 4;
    if (!aligned(t.master, 4) || !aligned(t.weights_bf16, 2) || !aligned(t.grad, ga) || !aligned(t.m, ma) ||
        !aligned(t.v, ma) || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))
      return fail(AM_EINVAL, "tensor %d: pointer not aligned to its elements", k);
    all += t.n;
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t bytes = (10 + (grad_dtype == AM_BF16 ? 2 : 4) + (codes ? 4 : 16)) * all;
  Timed tm(AM_K_ADAMW, s, 14.0 * all, (double)bytes);
  am::AdamwBatch a{};
  a.b1 = (float)beta1;
  a.c1 = (float)(1.0 - beta1);
  a.b2 = (float)beta2;
  a.c2 = (float)(1.0 - beta2);
  a.eps = (float)eps;
  a.root = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
  a.step = (float)(lr / (1.0 - pow(beta1, (double)step)));
  a.grad_scale = grad_scale;
  uint64_t groups = 0;
  for (int k = 0; k < count; ++k) {
    const am_adamw_tensor& t = tensors[k];
    if (t.n > 0) {
      const uint64_t need = (uint64_t)((t.n + am::ADAMW_CHUNK - 1) / am::ADAMW_CHUNK);
      if (a.count == am::AdamwBatch::MAX || (a.count > 0 && groups + need >= (1ull << 31))) {
        AM_TRY(hip_check(am::adamw_launch(a, grad_dtype == AM_BF16, codes, bytes, s), "adamw"));
        a.count = 0;
        groups = 0;
      }
      am::AdamwOne& o = a.t[a.count];
      o.w = t.master;
      o.w16 = static_cast<uint16_t*>(t.weights_bf16);
      o.g = t.grad;
      o.m = t.m;
      o.v = t.v;
      o.m_scale = t.m_scale;
      o.v_scale = t.v_scale;
      o.n = t.n;
      o.keep = (float)(1.0 - lr * t.weight_decay);
      o.key = seed + (uint32_t)k * 0x9E3779B9u;
      a.first[a.count] = (uint32_t)groups;
      groups += need;
      a.first[++a.count] = (uint32_t)groups;
    }
  }
  if (a.count > 0) return hip_check(am::adamw_launch(a, grad_dtype == AM_BF16, codes, bytes, s), "adamw");
  return AM_OK;
}

// ---------------------------------------------------------------- timing --

am_status am_workspace_check(const void* ws, int64_t ws_bytes, void* stream) {
  if (!ws || !aligned(ws, 256)) return fail(AM_EINVAL, "NULL or unaligned workspace");
  if (ws_bytes < SYNC_BYTES) return fail(AM_EWORKSPACE, "workspace smaller than its sync region");
  hipStream_t s = static_cast<hipStream_t>(stream);
  int flag = 0;
  AM_TRY(hip_check(hipMemcpyAsync(&flag, static_cast<const char*>(ws) + SYNC_STICKY_WORD * 4,
                                  sizeof flag, hipMemcpyDeviceToHost, s), "flag read"));
  AM_TRY(hip_check(hipStreamSynchronize(s), "stream sync"));
  if (flag) return fail(AM_ETIMEOUT, "a step barrier of a persistent recurrence kernel timed out");
  return AM_OK;
}

am_status am_profile_begin(uint32_t class_mask) {
  g_prof.on = true;
  g_prof.mask = class_mask;
  g_prof.next = 0;
  g_prof.recs.clear();
  for (int k = 0; k < AM_K_NCLASSES; ++k) {
    g_prof.seen[k] = 0;
    g_prof.launches[k] = 0;
    g_prof.ms[k] = g_prof.flops[k] = g_prof.bytes[k] = 0.0;
  }
  return AM_OK;
}

am_status am_profile_sample_every(int32_t n) {
  if (n < 1) return fail(AM_EINVAL, "sampling interval must be at least 1");
  g_prof.every = n;
  return AM_OK;
}

am_status am_profile_end(void) {
  g_prof.on = false;
  for (const ProfRec& r : g_prof.recs) {
    AM_TRY(hip_check(hipEventSynchronize(r.b), "event sync"));
    float ms = 0.f;
    AM_TRY(hip_check(hipEventElapsedTime(&ms, r.a, r.b), "event elapsed"));
    g_prof.launches[r.cls] += 1;
    g_prof.ms[r.cls] += ms;
    g_prof.flops[r.cls] += r.flops;
    g_prof.bytes[r.cls] += r.bytes;
  }
  g_prof.recs.clear();
  return AM_OK;
}

am_status am_profile_get(int32_t cls, int64_t* launches, double* ms, double* flops, double* bytes) {
  if (cls < 0 || cls >= AM_K_NCLASSES) return fail(AM_EINVAL, "unknown kernel class");
  if (launches) *launches = g_prof.launches[cls];
  if (ms) *ms = g_prof.ms[cls];
  if (flops) *flops = g_prof.flops[cls];
  if (bytes) *bytes = g_prof.bytes[cls];
  return AM_OK;
}

}  // extern "C"
