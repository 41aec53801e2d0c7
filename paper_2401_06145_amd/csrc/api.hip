// Host side of the C-ABI (include/spconv.h): argument checks, workspace plans,
// the Map-step orchestration (Section 5.1) and the GMaS plan (Section 5.2).
#include <algorithm>
#include <chrono>
#include <cstdio>
#include <cmath>
#include <cstring>
#include <mutex>
#include <new>
#include <string>
#include <unordered_map>
#include <vector>

#include "attention.h"
#include "pages.h"
#include "rotate.h"
#include "common.h"
#include "spconv.h"

using namespace spc;

struct spconv_map {
  int mode = 0, K = 0, K3 = 0, stride = 1, tstride = 1;
  int64_t n_in = 0, n_out = 0;
  const int32_t* out_coords = nullptr;
  const int32_t* pin = nullptr;   // concatenated pair lists, offset-major
  const int32_t* pout = nullptr;
  std::vector<int64_t> counts;    // |M_k|
  std::vector<int64_t> ptr;       // prefix of counts, K3 + 1 entries
  // metadata tables, offset-major over sorted positions (entry k * stride + p:
  // buffer row of point p's pair at offset k, or -1), and the caller row of each
  // sorted position (NULL: identity); NULL tables for a map without pairs
  const int32_t* imt = nullptr;
  const int32_t* omt = nullptr;
  int64_t imt_stride = 0, omt_stride = 0;
  const uint32_t* in_perm = nullptr;
  const uint32_t* out_perm = nullptr;
  bool transposed = false;
  // A symmetric submanifold map leaves its source-side table (imt) to be filled
  // from the pair lists by the first forward call that gathers through it; the
  // fused gather reads the pair lists and never needs it.
  mutable bool imt_pending = false;
  const uint32_t* seg_dev = nullptr;  // device pair starts, K3 + 1 entries
  uint32_t* inv_scratch = nullptr;    // n_in words of the build's scratch
};

namespace {

thread_local std::string g_err;

int fail(int code, const std::string& msg) {
  g_err = msg;
  return code;
}

int hip_fail(hipError_t e, const char* where) {
  return fail(SPCONV_EHIP, std::string(where) + ": " + hipGetErrorString(e));
}

#define SPC_TRY(expr, where)              \
  do {                                    \
    hipError_t _e = (expr);               \
    if (_e != hipSuccess) return hip_fail(_e, where); \
  } while (0)

size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// Bump allocator over a workspace; with base == nullptr it only measures.
struct Bump {
  char* base;
  size_t off = 0;
  explicit Bump(void* b) : base(static_cast<char*>(b)) {}
  template <typename T>
  T* take(int64_t n) {
    off = align_up(off, 256);
    T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
    off += (size_t)(n > 0 ? n : 0) * sizeof(T);
    return p;
  }
  void* take_bytes(size_t n) {
    off = align_up(off, 256);
    void* p = base ? base + off : nullptr;
    off += n;
    return p;
  }
};

// ---------------------------------------------------------------------------
// Phase timing (measurement API): HIP events around each phase on the stream.
// ---------------------------------------------------------------------------
const char* prof_name(int id) {
  static const char* kNames[PROF_IDS] = {
      "bounds", "sort", "outcoords", "backward", "balance", "forward", "readback", "metadata", "gather", "gemm",
      "scatter", "hash", "", "", "", "",
      "k_minmax", "k_radix_hist", "k_radix_scatter", "k_scan", "k_copy", "k_down_keys", "k_unique", "k_backward",
      "k_forward_count", "k_forward_write", "k_fill", "k_radix_local", "k_gather", "k_gemm", "k_scatter", "k_pack",
      "k_hash_insert", "k_hash_probe", "k_scatter_centre", "k_conv_small", "k_rms_norm", "k_scaled_linear", "k_attention",
      "k_attention_join", "k_rotate", "k_cache_write", "k_cache_read"};
  return (id >= 0 && id < PROF_IDS) ? kNames[id] : "";
}
struct PhaseRec {
  int phase;
  hipEvent_t a, b;
};
std::mutex g_prof_mu;
uint64_t g_prof_mask = 0;
std::vector<PhaseRec> g_recs;
std::vector<hipEvent_t> g_pool;

hipEvent_t ev_get() {
  hipEvent_t e = nullptr;
  if (!g_pool.empty()) {
    e = g_pool.back();
    g_pool.pop_back();
  } else if (hipEventCreateWithFlags(&e, hipEventDisableSystemFence) != hipSuccess) {
    // timing events only: no system-scope release needed around the timed kernels
    e = nullptr;
  }
  return e;
}

struct OpenRec {
  int id;
  hipStream_t s;
  hipEvent_t a;
};

}  // namespace

namespace spc {
ProfScope::ProfScope(int id, hipStream_t s) {
  if (!((g_prof_mask >> id) & 1ull)) return;
  std::lock_guard<std::mutex> lk(g_prof_mu);
  hipEvent_t a = ev_get();
  if (!a) return;
  (void)hipEventRecord(a, s);
  rec = new (std::nothrow) OpenRec{id, s, a};
}
ProfScope::~ProfScope() {
  if (!rec) return;
  OpenRec* r = static_cast<OpenRec*>(rec);
  std::lock_guard<std::mutex> lk(g_prof_mu);
  hipEvent_t b = ev_get();
  if (b) {
    (void)hipEventRecord(b, r->s);
    g_recs.push_back({r->id, r->a, b});
  }
  delete r;
}
}  // namespace spc

namespace {
using PhaseScope = spc::ProfScope;

// Mapped, coherent host buffer into which a map build's write pass publishes the
// control block's head (one per thread: a build returns only once it has read
// it).  Allocated on a thread's first build and kept; the device address of
// mapped memory is the same on every device.
struct PubBuffer {
  uint32_t* host = nullptr;
  uint32_t* dev = nullptr;
  uint32_t seq = 0;
};
thread_local PubBuffer g_pub;

PubBuffer* pub_buffer() {
  if (!g_pub.host) {
    void* p = nullptr;
    if (hipHostMalloc(&p, kPubBytes, hipHostMallocMapped | hipHostMallocPortable | hipHostMallocCoherent) != hipSuccess)
      return nullptr;
    void* d = nullptr;
    if (hipHostGetDevicePointer(&d, p, 0) != hipSuccess) {
      (void)hipHostFree(p);
      return nullptr;
    }
    std::memset(p, 0, kPubBytes);
    g_pub.host = static_cast<uint32_t*>(p);
    g_pub.dev = static_cast<uint32_t*>(d);
  }
  return &g_pub;
}

// Waits until the write pass has published sequence number `seq`: spins on the
// flag for up to 2 ms (the head is published at the start of the pass), then
// blocks on the stream, after which the flag must be set.
hipError_t pub_wait(const PubBuffer* pb, uint32_t seq, hipStream_t s, bool* ok) {
  const uint32_t* flag = pb->host + kPubFlagOffset / 4;
  const auto t0 = std::chrono::steady_clock::now();
  for (uint32_t spin = 0;; ++spin) {
    if (__atomic_load_n(flag, __ATOMIC_ACQUIRE) == seq) {
      *ok = true;
      return hipSuccess;
    }
    if ((spin & 1023u) == 1023u && std::chrono::steady_clock::now() - t0 > std::chrono::milliseconds(2)) break;
    __builtin_ia32_pause();
  }
  const hipError_t e = hipStreamSynchronize(s);
  *ok = __atomic_load_n(flag, __ATOMIC_ACQUIRE) == seq;
  return e;
}

// ---------------------------------------------------------------------------
// Map workspace plan
// ---------------------------------------------------------------------------
struct MapBufs {
  uint64_t* skeys;
  uint32_t* sidx;
  uint64_t* qkeys;
  uint32_t* qrow;
  int32_t* qcoords;
  int32_t* pin;
  int32_t* pout;
  uint32_t* counts;
  ControlBlock* cb;
  uint64_t* kalt;
  uint32_t* valt;
  uint64_t* dkeys;
  uint32_t* dvals;
  uint32_t* flags;
  uint32_t* pos;
  void* sort_tmp;
  uint32_t* bounds;  // per work item (offset, block): end of its query block
  int32_t* res;   // T_q, kept as the map's query-side metadata table
  int32_t* ts;    // T_s, the source-side table
  // Row strides of the two tables: the point counts rounded up to 32 entries, so
  // that every row starts on a 128-byte line.  The scatter (and the gather) read
  // 32 consecutive positions of a row per workgroup; with unpadded rows those
  // straddled two lines, each shared with a neighbouring workgroup that usually
  // runs on another die and fetched it again.
  int64_t res_stride;
  int64_t ts_stride;
  uint32_t* item_cnt;
  uint32_t* item_off;
  uint64_t* hkeys;  // hash-table search only
  uint32_t* hvals;
  int log2cap;
  int32_t* mm_partial;
  void* scan_tmp;
  int64_t max_items;  // work items: K3 * nb_items
  int64_t nb;         // source blocks of B keys
  int64_t nb_items;   // blocks per offset of the work items: nb, or for the hash-table
                      // search blocks of Cq queries
};

struct Tunables {
  int B = 1024;
  int Cq = 1024;
  int wg = 256;
  int count_group = 0;  // offsets per count-pass workgroup (0: size rule)
  bool presorted = false;
  bool hash = false;  // hash-table search instead of the sorted-array search
};

// Search hyperparameters (Section 5.1.4) left at 0 follow the source-set size:
// B = 1024, Cq = 1024 and 256-thread workgroups below 2^18 points, B = 4096,
// Cq = 2048 and 512 threads from there on (measured on gfx950: the 300k-point indoor
// room's search 90.7 -> 75.2 us, 4M-16M uniform and LiDAR clouds 2-13% faster;
// below 2^18 points the smaller blocks win: LiDAR 120k 31.1 vs 34.6 us, the 200k
// downsampling map 23.1 vs 27.7 us).  The rule applies only when none of the three
// is given.
void apply_size_rule(const spconv_options* opt, int64_t n_src, Tunables* t) {
  if (opt && (opt->B || opt->Cq || opt->wg)) return;
  if (n_src >= ((int64_t)1 << 18)) {
    t->B = 4096;
    t->Cq = 2048;
    t->wg = 512;
  }
}

int read_tunables(const spconv_options* opt, Tunables* t) {
  if (!opt) return SPCONV_OK;
  if (opt->B) {
    if (opt->B < 64 || opt->B > 4096 || (opt->B & (opt->B - 1)))
      return fail(SPCONV_EINVAL, "B must be a power of two in [64, 4096]");
    t->B = opt->B;
  }
  if (opt->Cq) {
    const int r = opt->Cq / 256;
    if (opt->Cq % 256 != 0 || !(r == 1 || r == 2 || r == 4 || r == 8))
      return fail(SPCONV_EINVAL, "Cq must be 256, 512, 1024 or 2048");
    t->Cq = opt->Cq;
  }
  if (opt->wg) {
    if (opt->wg != 128 && opt->wg != 256 && opt->wg != 512) return fail(SPCONV_EINVAL, "wg must be 128, 256 or 512");
    t->wg = opt->wg;
  }
  {
    const int r = t->Cq / t->wg;
    if (t->Cq % t->wg != 0 || !(r == 1 || r == 2 || r == 4 || r == 8))
      return fail(SPCONV_EINVAL, "Cq / wg must be 1, 2, 4 or 8");
  }
  if (opt->count_group < 0 || opt->count_group > 64) return fail(SPCONV_EINVAL, "count_group must be in [0, 64]");
  t->count_group = opt->count_group;
  t->presorted = opt->presorted != 0;
  if (opt->search < 0 || opt->search > 1) return fail(SPCONV_EINVAL, "search must be 0 or 1");
  t->hash = opt->search == 1;
  return SPCONV_OK;
}

size_t plan_map(void* base, int64_t n_src, int64_t nq_max, int K3, const Tunables& tu, int mode, MapBufs* b) {
  Bump m(base);
  const int64_t nmax = std::max(n_src, nq_max);
  b->nb = (n_src + tu.B - 1) / tu.B;
  b->nb_items = tu.hash ? (nq_max + tu.Cq - 1) / tu.Cq : b->nb;
  b->max_items = (int64_t)K3 * b->nb_items;
  b->skeys = m.take<uint64_t>(n_src);
  b->sidx = m.take<uint32_t>(n_src);
  b->qkeys = (mode == SPCONV_SUBM) ? nullptr : m.take<uint64_t>(nq_max);
  b->qrow = (mode == SPCONV_SUBM) ? nullptr : m.take<uint32_t>(nq_max);
  b->qcoords = (mode == SPCONV_DOWN) ? m.take<int32_t>(4 * nq_max) : nullptr;
  b->pin = m.take<int32_t>((int64_t)K3 * nq_max);
  b->pout = m.take<int32_t>((int64_t)K3 * nq_max);
  b->counts = m.take<uint32_t>(K3);
  b->cb = m.take<ControlBlock>(1);
  // build-time scratch
  b->kalt = m.take<uint64_t>(nmax);
  b->valt = m.take<uint32_t>(nmax);
  b->dkeys = (mode == SPCONV_DOWN) ? m.take<uint64_t>(n_src) : nullptr;
  b->dvals = (mode == SPCONV_DOWN) ? m.take<uint32_t>(n_src) : nullptr;
  b->flags = (mode == SPCONV_DOWN) ? m.take<uint32_t>(n_src) : nullptr;
  b->pos = (mode == SPCONV_DOWN) ? m.take<uint32_t>(n_src) : nullptr;
  b->sort_tmp = m.take_bytes(radix_temp_bytes(nmax));
  b->bounds = m.take<uint32_t>(b->max_items);
  b->res_stride = (int64_t)align_up((size_t)nq_max, 32);
  b->ts_stride = (int64_t)align_up((size_t)n_src, 32);
  b->res = m.take<int32_t>((int64_t)K3 * b->res_stride);
  b->ts = m.take<int32_t>((int64_t)K3 * b->ts_stride);
  b->item_cnt = m.take<uint32_t>(b->max_items);
  b->item_off = m.take<uint32_t>(b->max_items);
  b->mm_partial = static_cast<int32_t*>(m.take_bytes(minmax_temp_bytes()));
  b->scan_tmp = m.take_bytes(scan_temp_bytes(std::max(n_src, b->max_items)));
  b->log2cap = 0;
  b->hkeys = nullptr;
  b->hvals = nullptr;
  if (tu.hash) {
    // 2^log2cap >= 2 n slots: load at most 1/2
    int lg = 2;
    while (((int64_t)1 << lg) < 2 * std::max<int64_t>(n_src, 1)) ++lg;
    b->log2cap = lg;
    b->hkeys = m.take<uint64_t>((int64_t)1 << lg);
    b->hvals = m.take<uint32_t>((int64_t)1 << lg);
  }
  return align_up(m.off, 256);
}

int check_map_args(int64_t n_in, int64_t n_out, int K, int stride, int t, int mode) {
  if (K < 1 || K > 5) return fail(SPCONV_EUNSUPPORTED, "K must be in [1, 5]");
  if (t < 1) return fail(SPCONV_EINVAL, "tensor_stride must be >= 1");
  if (mode != SPCONV_SUBM && mode != SPCONV_DOWN && mode != SPCONV_UP) return fail(SPCONV_EINVAL, "bad mode");
  if (mode == SPCONV_SUBM && stride != 1) return fail(SPCONV_EINVAL, "SPCONV_SUBM requires stride 1");
  if (stride < 1) return fail(SPCONV_EINVAL, "stride must be >= 1");
  if (n_in < 0 || n_out < 0) return fail(SPCONV_EINVAL, "negative size");
  if (n_in >= (int64_t)1 << 31 || n_out >= (int64_t)1 << 31) return fail(SPCONV_EUNSUPPORTED, "more than 2^31 rows");
  // pair indices (and GEMM buffer rows) are int32: K^3 * max(n_in, n_out) bounds their count
  if ((int64_t)K * K * K * std::max(n_in, n_out) >= (int64_t)1 << 31)
    return fail(SPCONV_EUNSUPPORTED, "K^3 * rows must stay below 2^31");
  return SPCONV_OK;
}

// ---------------------------------------------------------------------------
// GMaS plan: GEMM grouping (Section 5.2.2) and tiles (Algorithm 1)
// ---------------------------------------------------------------------------
struct GmasPlan {
  int dtype = 0, elem = 4, pelem = 4, part_dtype = 0;
  int t_gather = 0, t_scatter = 0;
  int grouping = SPCONV_GROUP_RAGGED;
  int gather = 2;  // 1: Algorithm 1 into a buffer; 2: fused into the GEMM's operand loads
  int gemm_tile_rows = 0;  // 0: the occupancy rule
  // odd-K submanifold maps: the centre offset's product is computed inside the
  // scatter (k_scatter_centre) and the GEMMs skip that offset; -1: not fused
  int centre_k = -1;
  int64_t rows_pairs = 0;                 // all pairs of the map (partial buffer rows)
  int64_t rows_real = 0, rows_padded = 0;  // the GEMMs' rows, without and with padding
  int n_launches = 0;
  std::vector<std::vector<GemmSeg>> launches;  // one entry per GEMM launch (group)
};

int elem_bytes(int dtype) { return dtype == SPCONV_F32 ? 4 : 2; }

// Groups consecutive entries of `order` (offset ids) minimising
// sum_g (launch_cost + members_g * max_count_g); returns group boundaries.
std::vector<int> dp_groups(const std::vector<int>& order, const std::vector<int64_t>& cnt, int64_t launch_cost) {
  const int n = (int)order.size();
  std::vector<int64_t> best(n + 1, INT64_MAX);
  std::vector<int> from(n + 1, 0);
  best[0] = 0;
  for (int j = 1; j <= n; ++j) {
    int64_t mx = 0;
    for (int i = j - 1; i >= 0; --i) {
      mx = std::max(mx, cnt[order[i]]);
      const int64_t c = best[i] + launch_cost + (int64_t)(j - i) * mx;
      if (c < best[j]) {
        best[j] = c;
        from[j] = i;
      }
    }
  }
  std::vector<int> cuts;
  for (int j = n; j > 0; j = from[j]) cuts.push_back(j);
  cuts.push_back(0);
  std::reverse(cuts.begin(), cuts.end());
  return cuts;
}

// Large regions that the forward writes once and a later kernel reads once (the
// GEMM partial rows, the layer's output rows) go out with non-temporal stores.
// Otherwise their dirty lines stay in the caches, and the next kernels' traffic has to
// write them back.
constexpr int64_t kStreamPartialBytes = (int64_t)128 << 20;
// float32 partials, whose products give the caches more time per byte, stream from 256 MiB:
// layers of 128 to 256 MiB, streamed, took up to 1.19 times k_gemm's time (112k voxels,
// K = 2, 4 -> 192 111.7 us), stored plainly at most 1.05 (99.0), over 141 shapes 0.98 times the
// streamed form's; of 256 to 384 MiB streamed ones 0.98 times the plain ones' over 67.
constexpr int64_t kStreamPartialBytesF32 = (int64_t)256 << 20;
constexpr int64_t kStreamOutputBytes = (int64_t)64 << 20;

int make_plan(const spconv_map* m, int c_in, int c_out, int dtype, const spconv_options* opt, GmasPlan* p) {
  if (!m) return fail(SPCONV_EINVAL, "map is NULL");
  if (dtype != SPCONV_F32 && dtype != SPCONV_F16 && dtype != SPCONV_BF16) return fail(SPCONV_EUNSUPPORTED, "dtype");
  p->dtype = dtype;
  p->elem = elem_bytes(dtype);
  if (c_in < 1 || c_out < 1 || c_in > 1024 || c_out > 1024) return fail(SPCONV_EUNSUPPORTED, "channels must be in [1, 1024]");
  if ((c_in * p->elem) % 16 != 0) return fail(SPCONV_EUNSUPPORTED, "c_in rows must be whole 16-byte vectors");
  if (c_out % 16 != 0) return fail(SPCONV_EUNSUPPORTED, "c_out must be a multiple of 16");
  // GEMM partials: 1 = float32, 2 = the layer dtype; default the layer dtype (the
  // scatter sums them in float32 either way)
  const int pd = opt ? opt->partial_dtype : 0;
  if (pd < 0 || pd > 2) return fail(SPCONV_EINVAL, "partial_dtype must be 0, 1 or 2");
  p->part_dtype = (pd == 1) ? SPCONV_F32 : dtype;
  p->pelem = elem_bytes(p->part_dtype);
  // tiles: default one 16-byte vector per thread for gather and for the partial reads of scatter
  p->t_gather = (opt && opt->t_gather) ? opt->t_gather : 16 / p->elem;
  // scatter: one 16-byte partial vector per thread (the row-group scatter, which reads
  // each output's table entries once)
  p->t_scatter = (opt && opt->t_scatter) ? opt->t_scatter : 16 / p->pelem;
  if (p->t_gather <= 0 || c_in % p->t_gather != 0 || (p->t_gather * p->elem) % 16 != 0 ||
      (p->t_gather * p->elem / 16) > 16 || ((p->t_gather * p->elem / 16) & (p->t_gather * p->elem / 16 - 1)))
    return fail(SPCONV_EINVAL, "t_gather must divide c_in and span 1, 2, 4, 8 or 16 16-byte vectors");
  const int ts = p->t_scatter;
  if (!(ts == 4 || ts == 8 || ts == 16 || ts == 32 || ts == 64) || c_out % ts != 0 || (ts * p->pelem) % 16 != 0)
    return fail(SPCONV_EINVAL, "t_scatter must be 4..64 (power of two), divide c_out and span whole 16-byte partial vectors");
  p->grouping = (opt && opt->grouping) ? opt->grouping - 1 : SPCONV_GROUP_RAGGED;
  if (p->grouping < 0 || p->grouping > 2) return fail(SPCONV_EINVAL, "grouping");
  p->gather = (opt && opt->gather) ? opt->gather : SPCONV_GATHER_FUSED;
  p->gemm_tile_rows = opt ? opt->gemm_tile_rows : 0;
  if (p->gemm_tile_rows < 0 || p->gemm_tile_rows > (1 << 20)) return fail(SPCONV_EINVAL, "gemm_tile_rows must be in [0, 2^20]");
  if (p->gather != SPCONV_GATHER_BUFFER && p->gather != SPCONV_GATHER_FUSED)
    return fail(SPCONV_EINVAL, "gather must be 0, SPCONV_GATHER_BUFFER or SPCONV_GATHER_FUSED");

  const int K3 = m->K3;
  p->rows_pairs = m->ptr[K3];
  p->rows_padded = 0;
  p->launches.clear();
  const int centre = opt ? opt->centre : 0;
  if (centre < 0 || centre > 2) return fail(SPCONV_EINVAL, "centre must be 0, 1 or 2");
  p->centre_k = -1;
  if (centre != 1) {
    const int kc = (K3 - 1) / 2;
    const bool applies = m->mode == SPCONV_SUBM && m->K % 2 == 1 && m->omt && m->n_out > 0 &&
                         m->counts[kc] == m->n_out && p->gather == SPCONV_GATHER_FUSED &&
                         c_in <= 256 && c_out <= 256 && centre_fusable(c_in, c_out, dtype, p->part_dtype);
    if (applies) p->centre_k = kc;
    else if (centre == 2)
      return fail(SPCONV_EUNSUPPORTED, "centre = 2: the centre offset cannot be fused into the scatter here (needs "
                                       "an odd-K submanifold map, the fused gather, a 16-bit layer, c_in % 8 == 0 "
                                       "and c_out % 32 == 0, both at most 256)");
  }
  auto in_gemm = [&](int k) { return m->counts[k] > 0 && k != p->centre_k; };
  p->rows_real = p->rows_pairs - (p->centre_k >= 0 ? m->counts[p->centre_k] : 0);
  // Buffer rows follow the concatenated pair lists (row of pair e of offset k =
  // ptr[k] + e); grouping decides launches and padded heights only.
  if (p->grouping == SPCONV_GROUP_RAGGED) {
    std::vector<int> order;
    for (int k = 0; k < K3; ++k)
      if (in_gemm(k)) order.push_back(k);
    std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return m->counts[a] > m->counts[b]; });
    std::vector<GemmSeg> segs;
    for (int k : order) segs.push_back(GemmSeg{k, m->ptr[k], m->counts[k], m->counts[k]});
    p->rows_padded = p->rows_real;
    if (!segs.empty()) p->launches.push_back(segs);
  } else {
    std::vector<int> order(K3);
    for (int k = 0; k < K3; ++k) order[k] = k;
    if (p->grouping == SPCONV_GROUP_SORTED)  // non-decreasing pair count
      std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return m->counts[a] < m->counts[b]; });
    std::vector<int> nz;
    for (int k : order)
      if (in_gemm(k)) nz.push_back(k);
    const int64_t L = (opt && opt->launch_cost_rows > 0) ? opt->launch_cost_rows : 32768;
    const std::vector<int> cuts = dp_groups(nz, m->counts, L);
    for (size_t g = 0; g + 1 < cuts.size(); ++g) {
      int64_t h = 0;
      for (int i = cuts[g]; i < cuts[g + 1]; ++i) h = std::max(h, m->counts[nz[i]]);
      std::vector<GemmSeg> segs;
      for (int i = cuts[g]; i < cuts[g + 1]; ++i) {
        const int k = nz[i];
        segs.push_back(GemmSeg{k, m->ptr[k], m->counts[k], h});
        p->rows_padded += h;
      }
      p->launches.push_back(segs);
    }
  }
  p->n_launches = (int)p->launches.size();
  return SPCONV_OK;
}

struct FwdBufs {
  void* wt;  // transposed weights for the full-width GEMM, or NULL
  void* buf_in;
  void* buf_out;
};

size_t plan_forward_ws(void* base, const spconv_map* m, int c_in, int c_out, const GmasPlan& p, FwdBufs* b) {
  Bump a(base);
  b->wt = (gemm_wide(c_in, c_out, p.dtype, p.part_dtype) && gemm_wide_transposed(c_in, c_out, p.dtype))
              ? a.take_bytes((size_t)m->K3 * c_in * c_out * p.elem)
              : nullptr;
  // the fused gather reads the input rows directly: no gathered buffer
  b->buf_in = (p.gather == SPCONV_GATHER_BUFFER) ? a.take_bytes((size_t)p.rows_pairs * c_in * p.elem) : nullptr;
  // one spare row past the partials: the full-width GEMM's stores of rows without data
  // (rows are pair indices: with the centre fused its rows stay unused)
  b->buf_out = a.take_bytes((size_t)(p.rows_pairs + 1) * c_out * p.pelem);
  return align_up(a.off, 256);
}

// Whether a call runs as the one-kernel form (conv_small.hip).  Grouping and GEMM tile
// rows only shape launches of the separate steps, and do not rule it out.
bool one_kernel(const spconv_map* m, const void* x, const void* w, const void* y, int c_in, int c_out,
                const GmasPlan& p, const spconv_options* opt) {
  // options that name a form of the separate steps keep them
  if (opt && (opt->centre || opt->gather || opt->partial_dtype || opt->t_gather || opt->t_scatter)) return false;
  if (p.rows_pairs == 0 || !m->omt || !conv_small_applies(m->n_in, m->n_out, p.rows_pairs, m->K3, c_in, c_out, p.dtype))
    return false;
  // outputs are written while other workgroups still read inputs and weights
  auto apart = [](const void* a, int64_t na, const void* b, int64_t nb) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return pa + (uintptr_t)na <= pb || pb + (uintptr_t)nb <= pa;
  };
  const int64_t yb = m->n_out * c_out * p.elem;
  return apart(x, m->n_in * c_in * p.elem, y, yb) && apart(w, (int64_t)m->K3 * c_in * c_out * p.elem, y, yb);
}

}  // namespace

// ===========================================================================
// C-ABI
// ===========================================================================
extern "C" {

const char* spconv_last_error(void) { return g_err.c_str(); }

size_t spconv_map_workspace_bytes(int64_t n_in, int64_t n_out, int K, int mode, const spconv_options* opt) {
  if (check_map_args(n_in, n_out, K, mode == SPCONV_SUBM ? 1 : 2, 1, mode) != SPCONV_OK) return 0;
  Tunables tu;
  if (read_tunables(opt, &tu) != SPCONV_OK) return 0;
  const int64_t n_src = (mode == SPCONV_UP) ? n_out : n_in;
  apply_size_rule(opt, n_src, &tu);
  const int64_t nq_max = n_in;
  MapBufs b;
  return plan_map(nullptr, n_src, nq_max, K * K * K, tu, mode, &b);
}

}  // extern "C"

namespace {

// Sort passes to plan for a build before its key layout is known (the layout is
// computed on the device, so the host never waits for the bounds): the count the
// same inputs needed last time, else the last count needed on this thread (start:
// 4 passes, a 32-bit key).  A build whose key turns out wider is redone with the
// passes it needs.  Inputs are told apart by address, sizes and layer arguments
// only, so a new cloud at a reused address inherits a plan; a wrong plan costs at
// most that redo (or, planned too long, digit passes that copy).
// Sort plan of a map build, kept per input from the previous build of it: the
// digit passes of the digit-by-digit sort, and whether the small sorts may go by
// bucket (no bucket of the previous build was too large for one workgroup).
struct SortPlan {
  int passes = 4;
  bool by_bucket = true;
};
struct PassHint {
  std::unordered_map<std::string, SortPlan> by_input;
  int last = 4;
};
thread_local PassHint g_pass_hint;

std::string pass_key(const int32_t* a, int64_t na, const int32_t* b, int64_t nb, int K, int stride, int t, int mode) {
  char buf[160];
  snprintf(buf, sizeof(buf), "%p/%lld/%p/%lld/%d/%d/%d/%d", (const void*)a, (long long)na, (const void*)b,
           (long long)nb, K, stride, t, mode);
  return buf;
}

int build_map_impl(const int32_t* d_in_coords, int64_t n_in, const int32_t* d_out_coords, int64_t n_out, int K,
                   int stride, int tensor_stride, int mode, const spconv_options* opt, void* d_workspace,
                   size_t ws_bytes, void* stream, spconv_map** out_map, int passes, bool by_bucket,
                   int* passes_needed, bool* bucket_failed) {
  *passes_needed = 0;
  *bucket_failed = false;
  if (!out_map) return fail(SPCONV_EINVAL, "out_map is NULL");
  *out_map = nullptr;
  int st = check_map_args(n_in, mode == SPCONV_UP ? n_out : 0, K, stride, tensor_stride, mode);
  if (st != SPCONV_OK) return st;
  if (n_in > 0 && !d_in_coords) return fail(SPCONV_EINVAL, "d_in_coords is NULL");
  if (mode == SPCONV_UP && n_out > 0 && !d_out_coords) return fail(SPCONV_EINVAL, "d_out_coords is NULL");
  if (mode != SPCONV_UP) n_out = 0;
  Tunables tu;
  if ((st = read_tunables(opt, &tu)) != SPCONV_OK) return st;
  if (tu.hash && mode != SPCONV_SUBM) return fail(SPCONV_EUNSUPPORTED, "the hash-table search covers SPCONV_SUBM only");
  const int K3 = K * K * K;
  const int64_t n_src = (mode == SPCONV_UP) ? n_out : n_in;
  apply_size_rule(opt, n_src, &tu);
  const int64_t nq_max = n_in;
  MapBufs b;
  const size_t need = plan_map(nullptr, n_src, nq_max, K3, tu, mode, &b);
  if (!d_workspace || ws_bytes < need) return fail(SPCONV_ENOSPC, "map workspace too small");
  if (reinterpret_cast<uintptr_t>(d_workspace) % 256 != 0) return fail(SPCONV_EINVAL, "workspace must be 256-byte aligned");
  plan_map(d_workspace, n_src, nq_max, K3, tu, mode, &b);
  hipStream_t s = static_cast<hipStream_t>(stream);

  spconv_map* m = new (std::nothrow) spconv_map();
  if (!m) return fail(SPCONV_EINVAL, "out of host memory");
  m->mode = mode;
  m->K = K;
  m->K3 = K3;
  m->stride = stride;
  m->tstride = tensor_stride;
  m->n_in = n_in;
  m->n_out = (mode == SPCONV_SUBM) ? n_in : (mode == SPCONV_UP ? n_out : 0);
  m->out_coords = (mode == SPCONV_SUBM) ? d_in_coords : (mode == SPCONV_UP ? d_out_coords : b.qcoords);
  m->pin = b.pin;
  m->pout = b.pout;
  m->counts.assign(K3, 0);
  m->ptr.assign(K3 + 1, 0);
  auto done_empty = [&]() {
    *out_map = m;
    return SPCONV_OK;
  };
  if (n_in == 0 || n_src == 0) return done_empty();

  const int32_t* src_coords = (mode == SPCONV_UP) ? d_out_coords : d_in_coords;
  auto bail = [&](int code) {
    delete m;
    return code;
  };
  // key layout on the device (no host wait): bounds partials, then the layout,
  // computed by the source sort's first kernel when that is a tile histogram of the
  // coordinates, else by one workgroup of its own
  const KeyLayout* L = &b.cb->layout;
  LayoutArgs la{};
  const bool sort_first = !tu.hash && !tu.presorted;
  {
    PhaseScope ph(PH_BOUNDS, s);
    int np = 0;
    hipError_t e = launch_minmax(d_in_coords, n_in, d_out_coords, mode == SPCONV_UP ? n_out : 0, b.mm_partial,
                                 b.cb, &np, s);
    // builds that do not sort the keys digit by digit take any key width (up to 62
    // bits): no sort, or every sort by bucket
    const bool all_bucket = by_bucket && radix_bucket_applies(n_src) && (mode != SPCONV_UP || radix_bucket_applies(n_in));
    const int plan = (tu.hash || (tu.presorted && mode != SPCONV_DOWN) || all_bucket) ? 8 : passes;
    la = LayoutArgs{b.mm_partial, np, K, stride, tensor_stride, K3, plan, b.cb};
    if (e == hipSuccess && !sort_first) e = launch_layout(la, s);
    if (e != hipSuccess) return bail(hip_fail(e, "coordinate bounds"));
  }
  if (tu.hash) {
    PhaseScope ph(PH_HASH, s);
    hipError_t e = launch_hash_build(d_in_coords, n_in, L, b.hkeys, b.hvals, b.log2cap, b.skeys, b.sidx, &b.cb->err, s);
    if (e != hipSuccess) return bail(hip_fail(e, "hash build"));
  } else {
    PhaseScope ph(PH_SORT, s);
    // sorted inputs (a previous layer's outputs) only need their keys packed (Section 5.1.1)
    hipError_t e = tu.presorted ? launch_pack(src_coords, n_src, L, b.skeys, b.sidx, s)
                                : radix_sort_kv(src_coords, L, b.skeys, b.sidx, b.kalt, b.valt, n_src, passes, by_bucket,
                                                b.sort_tmp, &b.cb->err, &la, s);
    if (e == hipSuccess && mode == SPCONV_UP)
      e = tu.presorted ? launch_pack(d_in_coords, n_in, L, b.qkeys, b.qrow, s)
                       : radix_sort_kv(d_in_coords, L, b.qkeys, b.qrow, b.kalt, b.valt, n_in, passes, by_bucket,
                                       b.sort_tmp, &b.cb->err, nullptr, s);
    if (e != hipSuccess) return bail(hip_fail(e, "sort"));
  }
  if (mode == SPCONV_DOWN) {
    PhaseScope ph(PH_OUTCOORDS, s);
    const int64_t cell = (int64_t)tensor_stride * stride;
    hipError_t e = launch_down_keys(b.skeys, n_src, L, cell, b.dkeys, b.dvals, s);
    if (e == hipSuccess)
      e = radix_sort_kv(nullptr, L, b.dkeys, b.dvals, b.kalt, b.valt, n_src, passes, by_bucket, b.sort_tmp,
                        &b.cb->err, nullptr, s);
    if (e == hipSuccess)
      e = unique_keys(b.dkeys, n_src, L, b.flags, b.pos, b.scan_tmp, b.qkeys, b.qrow, b.qcoords, b.cb, s);
    if (e != hipSuccess) return bail(hip_fail(e, "output coordinates"));
  }

  SearchArgs a;
  std::memset(&a, 0, sizeof(a));
  a.skeys = b.skeys;
  a.sidx = b.sidx;
  a.n_src = n_src;
  a.qkeys = (mode == SPCONV_SUBM) ? b.skeys : b.qkeys;
  a.qrow = (mode == SPCONV_SUBM) ? b.sidx : b.qrow;
  a.n_q = nq_max;
  a.n_q_dev = (mode == SPCONV_DOWN) ? &b.cb->n_q : nullptr;
  a.K3 = K3;
  a.dk = b.cb->dk;
  a.B = tu.B;
  a.Cq = tu.Cq;
  a.wg = tu.wg;
  a.count_group = tu.count_group;
  // A table T_q far larger than the caches streams to memory: the write pass reads
  // it back from there either way, and left dirty in the caches it slowed the
  // write pass (LiDAR Map 2.75 -> 2.68 ms at 15.9M voxels, 0.790 -> 0.768 ms at
  // 4.07M; at 1.08M voxels, 117 MB of table, streaming lost 6 us).
  a.stream_tq = (int64_t)K3 * b.res_stride * (int64_t)sizeof(int32_t) >= ((int64_t)256 << 20) ? 1 : 0;
  a.swap_roles = (mode == SPCONV_UP) ? 1 : 0;
  a.check_q = (mode == SPCONV_UP) ? 1 : 0;
  a.res = b.res;
  a.res_stride = b.res_stride;
  a.ts = b.ts;
  a.ts_stride = b.ts_stride;
  a.sym = (mode == SPCONV_SUBM && K % 2 == 1) ? 1 : 0;
  a.write_ts = a.sym ? 0 : 1;
  a.pair_cap = (int64_t)K3 * nq_max;
  PubBuffer* pb = pub_buffer();
  if (!pb) return bail(fail(SPCONV_EHIP, "mapped host buffer allocation failed"));
  if (++pb->seq == 0) pb->seq = 1;
  a.pub = pb->dev;
  a.pub_seq = pb->seq;
  // work items (k, b): the sorted search's source blocks, or the hash-table
  // search's blocks of Cq queries; the passes split a query block into chunks of
  // at most Cq themselves, so the balancing step needs no scan of its own
  const int64_t nb = b.nb_items;
  {
    PhaseScope ph(PH_BACKWARD, s);
    hipError_t e = tu.hash ? launch_hash_items(K3, nq_max, tu.Cq, nb, b.bounds, s)
                           : launch_backward(a, nb, b.bounds, b.cb, s);
    if (e != hipSuccess) return bail(hip_fail(e, "backward search"));
  }
  if (!a.sym) {
    // sources without a partner at some offset: no query visits their entry
    PhaseScope ph(PH_METADATA, s);
    hipError_t e = launch_fill_u32(reinterpret_cast<uint32_t*>(b.ts), 0xFFFFFFFFu, (int64_t)K3 * b.ts_stride, s);
    if (e != hipSuccess) return bail(hip_fail(e, "metadata fill"));
  }
  {
    PhaseScope ph(PH_FORWARD, s);
    hipError_t e = tu.hash ? launch_hash_count(a, b.hkeys, b.hvals, b.log2cap, nb, b.item_cnt, s)
                           : launch_forward(a, false, b.bounds, nb, b.item_cnt, nullptr, b.pin, b.pout, b.cb, s);
    if (e == hipSuccess) e = scan_exclusive_u32(b.item_cnt, b.item_off, b.max_items, &b.cb->n_pairs, b.scan_tmp, s);
    if (e == hipSuccess)
      e = launch_forward(a, true, b.bounds, nb, b.item_cnt, b.item_off, b.pin, b.pout, b.cb, s);
    if (e != hipSuccess) return bail(hip_fail(e, "forward search"));
  }
  {
    // the head as the write pass published it (the pass may still be running)
    PhaseScope ph(PH_READBACK, s);
    bool ok = false;
    hipError_t e = pub_wait(pb, a.pub_seq, s, &ok);
    if (e != hipSuccess) return bail(hip_fail(e, "count read-back"));
    if (!ok) return bail(fail(SPCONV_EHIP, "the write pass did not publish its counts"));
    ControlBlock head;
    std::memcpy(&head, pb->host, kControlHeadBytes);
    const ControlBlock* hc = &head;
    if (hc->err & kErrRange)
      return bail(fail(SPCONV_ERANGE, "coordinate extent (plus kernel reach) needs more than 62 key bits"));
    if (hc->err & kErrBucket) {
      // a bucket too large for one workgroup: the caller redoes the build digit by digit
      *passes_needed = (hc->layout.total_bits + 7) / 8;
      *bucket_failed = true;
      return bail(SPCONV_OK);
    }
    if (hc->err & kErrWide) {
      // the key is wider than the sort planned for: the caller redoes the build
      *passes_needed = (hc->layout.total_bits + 7) / 8;
      return bail(SPCONV_OK);
    }
    *passes_needed = (hc->layout.total_bits + 7) / 8;
    if (hc->err & kErrDup) return bail(fail(SPCONV_EDUP, "duplicate coordinates"));
    if (hc->err & kErrOverflow) return bail(fail(SPCONV_EHIP, "overflow of the work items or of the hash table"));
    if (hc->err & kErrSpin) return bail(fail(SPCONV_EHIP, "a look-back exceeded its wait bound"));
    if (hc->err & kErrUnsorted)
      return bail(fail(SPCONV_EINVAL, "rows declared presorted are not in ascending (b, x, y, z) order"));
    if (mode == SPCONV_DOWN) m->n_out = hc->n_q;
    for (int k = 0; k < K3; ++k) {
      m->counts[k] = (int64_t)hc->seg_pair_start[k + 1] - hc->seg_pair_start[k];
      m->ptr[k + 1] = hc->seg_pair_start[k + 1];
    }
    if (m->ptr[K3] != hc->n_pairs) return bail(fail(SPCONV_EHIP, "pair count mismatch"));
  }
  // T_q is indexed by sorted query position, T_s by sorted source position.
  // Inputs are the sources except for a direct UP map, whose inputs are the
  // queries; presorted rows are their own sorted positions.
  // (hash-table maps index the inputs in caller order: no permutation)
  const uint32_t* src_perm = (tu.presorted || tu.hash) ? nullptr : b.sidx;
  const uint32_t* q_perm = (mode == SPCONV_SUBM) ? src_perm
                           : (mode == SPCONV_DOWN ? nullptr : (tu.presorted ? nullptr : b.qrow));
  if (mode == SPCONV_UP) {
    m->imt = b.res;
    m->imt_stride = b.res_stride;
    m->in_perm = q_perm;
    m->omt = b.ts;
    m->omt_stride = b.ts_stride;
    m->out_perm = src_perm;
  } else {
    m->imt = b.ts;
    m->imt_stride = b.ts_stride;
    m->in_perm = src_perm;
    m->omt = b.res;
    m->omt_stride = b.res_stride;
    m->out_perm = q_perm;
  }
  if (!a.write_ts) {
    m->imt_pending = true;
    m->seg_dev = b.cb->seg_pair_start;
    m->inv_scratch = b.valt;
  }
  *out_map = m;
  return SPCONV_OK;
}

}  // namespace

extern "C" {

int spconv_build_map(const int32_t* d_in_coords, int64_t n_in, const int32_t* d_out_coords, int64_t n_out, int K,
                     int stride, int tensor_stride, int mode, const spconv_options* opt, void* d_workspace,
                     size_t ws_bytes, void* stream, spconv_map** out_map) {
  PassHint& hint = g_pass_hint;
  const std::string key = pass_key(d_in_coords, n_in, d_out_coords, n_out, K, stride, tensor_stride, mode);
  const auto it = hint.by_input.find(key);
  SortPlan plan;
  if (it != hint.by_input.end())
    plan = it->second;
  else
    plan.passes = hint.last;
  int needed = 0, st = SPCONV_OK;
  // at most one redo for a too large bucket and one for a key wider than planned
  for (int attempt = 0; attempt < 3; ++attempt) {
    bool bucket_failed = false;
    st = build_map_impl(d_in_coords, n_in, d_out_coords, n_out, K, stride, tensor_stride, mode, opt, d_workspace,
                        ws_bytes, stream, out_map, plan.passes, plan.by_bucket, &needed, &bucket_failed);
    if (st != SPCONV_OK || *out_map) break;
    if (bucket_failed && plan.by_bucket) {
      plan.by_bucket = false;
      if (needed > plan.passes) plan.passes = needed;
    } else if (needed > plan.passes) {
      plan.passes = needed;
    } else {
      return fail(SPCONV_EHIP, "key layout changed between two builds");
    }
  }
  if (st == SPCONV_OK && !*out_map) return fail(SPCONV_EHIP, "map build did not settle on a sort plan");
  if (needed > 0) {
    if (hint.by_input.size() >= 256) hint.by_input.clear();
    plan.passes = needed;
    hint.by_input[key] = plan;
    hint.last = needed;
  }
  return st;
}

int spconv_map_transpose(const spconv_map* down, spconv_map** out_map) {
  if (!down || !out_map) return fail(SPCONV_EINVAL, "NULL argument");
  *out_map = nullptr;
  if (down->mode != SPCONV_DOWN) return fail(SPCONV_EINVAL, "only SPCONV_DOWN maps can be transposed");
  spconv_map* m = new (std::nothrow) spconv_map(*down);
  if (!m) return fail(SPCONV_EINVAL, "out of host memory");
  m->mode = SPCONV_UP;
  m->transposed = true;
  m->n_in = down->n_out;
  m->n_out = down->n_in;
  m->pin = down->pout;
  m->pout = down->pin;
  std::swap(m->imt, m->omt);
  std::swap(m->imt_stride, m->omt_stride);
  std::swap(m->in_perm, m->out_perm);
  m->out_coords = nullptr;  // the fine coordinates are the DOWN map's inputs (caller-owned)
  *out_map = m;
  return SPCONV_OK;
}

int64_t spconv_map_n_in(const spconv_map* m) { return m ? m->n_in : -1; }
int64_t spconv_map_n_out(const spconv_map* m) { return m ? m->n_out : -1; }
int spconv_map_kvol(const spconv_map* m) { return m ? m->K3 : -1; }
const int32_t* spconv_map_out_coords(const spconv_map* m) { return m ? m->out_coords : nullptr; }

int spconv_map_counts(const spconv_map* m, int64_t* h_counts) {
  if (!m || !h_counts) return fail(SPCONV_EINVAL, "NULL argument");
  for (int k = 0; k < m->K3; ++k) h_counts[k] = m->counts[k];
  return SPCONV_OK;
}

int spconv_map_pairs(const spconv_map* m, int k, const int32_t** d_in_idx, const int32_t** d_out_idx, int64_t* count) {
  if (!m || !d_in_idx || !d_out_idx || !count) return fail(SPCONV_EINVAL, "NULL argument");
  if (k < 0 || k >= m->K3) return fail(SPCONV_EINVAL, "offset index out of range");
  *d_in_idx = m->pin + m->ptr[k];
  *d_out_idx = m->pout + m->ptr[k];
  *count = m->counts[k];
  return SPCONV_OK;
}

int spconv_map_copy_pairs(const spconv_map* m, int32_t* d_in_idx, int32_t* d_out_idx, void* stream) {
  if (!m) return fail(SPCONV_EINVAL, "map is NULL");
  const int64_t n = m->ptr[m->K3];
  if (n == 0) return SPCONV_OK;
  if (!d_in_idx || !d_out_idx) return fail(SPCONV_EINVAL, "NULL destination");
  hipStream_t s = static_cast<hipStream_t>(stream);
  SPC_TRY(hipMemcpyAsync(d_in_idx, m->pin, (size_t)n * 4, hipMemcpyDeviceToDevice, s), "copy pairs");
  SPC_TRY(hipMemcpyAsync(d_out_idx, m->pout, (size_t)n * 4, hipMemcpyDeviceToDevice, s), "copy pairs");
  return SPCONV_OK;
}

int spconv_map_copy_out_coords(const spconv_map* m, int32_t* d_coords, void* stream) {
  if (!m) return fail(SPCONV_EINVAL, "map is NULL");
  if (m->n_out == 0) return SPCONV_OK;
  if (!d_coords) return fail(SPCONV_EINVAL, "NULL destination");
  if (!m->out_coords) return fail(SPCONV_EINVAL, "this map does not hold its output coordinates");
  SPC_TRY(hipMemcpyAsync(d_coords, m->out_coords, (size_t)m->n_out * 16, hipMemcpyDeviceToDevice,
                         static_cast<hipStream_t>(stream)),
          "copy coordinates");
  return SPCONV_OK;
}

void spconv_free_map(spconv_map* m) { delete m; }

size_t spconv_forward_workspace_bytes(const spconv_map* m, int c_in, int c_out, int dtype, const spconv_options* opt) {
  GmasPlan p;
  if (make_plan(m, c_in, c_out, dtype, opt, &p) != SPCONV_OK) return 0;
  FwdBufs b;
  return plan_forward_ws(nullptr, m, c_in, c_out, p, &b);
}

int spconv_forward_plan(const spconv_map* m, int c_in, int c_out, int dtype, const spconv_options* opt,
                        spconv_plan_info* info) {
  if (!info) return fail(SPCONV_EINVAL, "info is NULL");
  GmasPlan p;
  const int st = make_plan(m, c_in, c_out, dtype, opt, &p);
  if (st != SPCONV_OK) return st;
  info->rows_real = p.rows_real;
  info->rows_padded = p.rows_padded;
  info->n_gemm_launches = p.n_launches;
  info->t_gather = p.t_gather;
  info->t_scatter = p.t_scatter;
  info->grouping = p.grouping;
  info->gather = p.gather;
  info->centre = p.centre_k >= 0 ? 1 : 0;
  return SPCONV_OK;
}

int spconv_forward(const spconv_map* m, const void* d_x, const void* d_w, void* d_y, int c_in, int c_out, int dtype,
                   const spconv_options* opt, void* d_workspace, size_t ws_bytes, void* stream) {
  return spconv_forward_ex(m, d_x, d_w, d_y, c_in, c_out, dtype, nullptr, 0, opt, d_workspace, ws_bytes, stream);
}

int spconv_concat_rows(const void* d_a, int c_a, const void* d_b, int c_b, void* d_out, int64_t n, int dtype,
                       void* stream) {
  if (dtype != SPCONV_F32 && dtype != SPCONV_F16 && dtype != SPCONV_BF16) return fail(SPCONV_EUNSUPPORTED, "dtype");
  const int e = elem_bytes(dtype);
  if (n < 0 || c_a < 0 || c_b < 0 || (c_a * e) % 16 != 0 || (c_b * e) % 16 != 0)
    return fail(SPCONV_EUNSUPPORTED, "concat needs 16-byte channel blocks");
  if (n == 0 || c_a + c_b == 0) return SPCONV_OK;
  if (!d_out || (c_a && !d_a) || (c_b && !d_b)) return fail(SPCONV_EINVAL, "NULL pointer");
  SPC_TRY(launch_concat(d_a, c_a, d_b, c_b, d_out, n, e, static_cast<hipStream_t>(stream)), "concat");
  return SPCONV_OK;
}

}  // extern "C"

namespace {

int forward_impl(const spconv_map* m, const void* d_x, const void* d_w, void* d_y, int c_in, int c_out, int dtype,
                 const void* d_residual, int relu, const spconv_options* opt, void* d_workspace, size_t ws_bytes,
                 void* stream) {
  GmasPlan p;
  int st = make_plan(m, c_in, c_out, dtype, opt, &p);
  if (st != SPCONV_OK) return st;
  if (m->n_out > 0 && !d_y) return fail(SPCONV_EINVAL, "d_y is NULL");
  if (p.rows_pairs > 0 && (!d_x || !d_w)) return fail(SPCONV_EINVAL, "d_x / d_w is NULL");
  auto misaligned = [](const void* q) { return (reinterpret_cast<uintptr_t>(q) & 15) != 0; };
  if (misaligned(d_x) || misaligned(d_w) || misaligned(d_y) || misaligned(d_residual))
    return fail(SPCONV_EINVAL, "d_x, d_w, d_y and d_residual must be 16-byte aligned");
  FwdBufs b;
  const size_t need = plan_forward_ws(nullptr, m, c_in, c_out, p, &b);
  if (need > 0 && (!d_workspace || ws_bytes < need)) return fail(SPCONV_ENOSPC, "forward workspace too small");
  if (reinterpret_cast<uintptr_t>(d_workspace) % 256 != 0) return fail(SPCONV_EINVAL, "workspace must be 256-byte aligned");
  plan_forward_ws(d_workspace, m, c_in, c_out, p, &b);
  if (m->n_out == 0) return SPCONV_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (one_kernel(m, d_x, d_w, d_y, c_in, c_out, p, opt)) {
    PhaseScope ph(PH_GEMM, s);
    SPC_TRY(launch_conv_small(d_x, m->n_in, d_w, m->pin, m->omt, m->omt_stride, m->out_perm, p.rows_pairs, m->K3,
                              d_y, d_residual, relu, m->n_out, c_in, c_out, dtype, s),
            "one-kernel convolution");
    return SPCONV_OK;
  }
  // a map without tables has no pairs: the scatter then writes zeros (plus the epilogue)
  const int K3 = m->omt ? m->K3 : 0;
  if (p.rows_pairs > 0) {
    const bool fused = p.gather == SPCONV_GATHER_FUSED;
    if (!fused && m->imt_pending) {
      PhaseScope ph(PH_METADATA, s);
      int32_t* ts = const_cast<int32_t*>(m->imt);
      SPC_TRY(launch_fill_u32(reinterpret_cast<uint32_t*>(ts), 0xFFFFFFFFu, (int64_t)m->K3 * m->imt_stride, s),
              "source-side table fill");
      SPC_TRY(launch_ts_from_pairs(m->pin, m->seg_dev, m->K3, m->ptr[m->K3], m->in_perm, m->n_in, m->inv_scratch, ts,
                                   m->imt_stride, s),
              "source-side table from the pairs");
      m->imt_pending = false;
    }
    if (!fused) {
      PhaseScope ph(PH_GATHER, s);
      SPC_TRY(launch_gather(d_x, m->n_in, c_in, p.elem, m->imt, m->imt_stride, m->in_perm, K3, b.buf_in, p.t_gather,
                            s),
              "gather");
    }
    {
      PhaseScope ph(PH_GEMM, s);
      if (b.wt) SPC_TRY(launch_transpose_w(d_w, b.wt, m->K3, c_in, c_out, s), "weight transpose");
      // fused: the A rows are the input rows of the pairs (pair r reads x[pin[r]])
      const void* a_src = fused ? d_x : b.buf_in;
      const int32_t* a_rows = fused ? m->pin : nullptr;
      const bool stream = (int64_t)p.rows_pairs * c_out * p.pelem >=
                          (dtype == SPCONV_F32 ? kStreamPartialBytesF32 : kStreamPartialBytes);
      for (const auto& segs : p.launches)
        SPC_TRY(launch_gemm(segs.data(), (int)segs.size(), a_src, a_rows, d_w, b.wt, b.buf_out,
                            static_cast<char*>(b.buf_out) + (size_t)p.rows_pairs * c_out * p.pelem, c_in, c_out,
                            dtype, p.part_dtype, p.gemm_tile_rows, stream, s),
                "grouped GEMM");
    }
  }
  {
    PhaseScope ph(PH_SCATTER, s);
    const bool stream = m->n_out * c_out * p.elem >= kStreamOutputBytes;
    if (p.centre_k >= 0)
      SPC_TRY(launch_scatter_centre(d_x, m->out_perm, d_w, b.wt, p.centre_k, b.buf_out, m->omt, m->omt_stride, K3,
                                    d_y, d_residual, relu, m->n_out, c_in, c_out, dtype, p.part_dtype, stream, s),
              "scatter with the centre offset");
    else
      SPC_TRY(launch_scatter(b.buf_out, p.part_dtype, m->n_out, c_out, m->omt, m->omt_stride, m->out_perm, K3, d_y,
                             dtype, p.t_scatter, d_residual, relu, stream, s),
              "scatter");
  }
  return SPCONV_OK;
}

// Scratch of the allocation-free forward: device memory the library holds itself,
// one copy per GPU for the whole process.  In host code `scratch` names a host-side
// stand-in, so host code only ever uses the device address that hipGetSymbolAddress
// returns for the current device, kept per device below.
static __device__ __align__(256) unsigned char scratch[SPCONV_NOALLOC_SCRATCH_BYTES];

std::mutex g_scratch_mu;
std::vector<void*> g_scratch_addr;  // by device ordinal; NULL until looked up

// The current device's address of `scratch`, looked up on the first call on that
// device (with it current) and kept.
int scratch_address(void** out) {
  int dev = 0;
  SPC_TRY(hipGetDevice(&dev), "hipGetDevice");
  std::lock_guard<std::mutex> lk(g_scratch_mu);
  if (dev < 0) return fail(SPCONV_EHIP, "negative device ordinal");
  if ((size_t)dev >= g_scratch_addr.size()) g_scratch_addr.resize((size_t)dev + 1, nullptr);
  if (!g_scratch_addr[dev]) {
    void* p = nullptr;
    SPC_TRY(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)), "scratch address");
    if (!p) return fail(SPCONV_EHIP, "scratch address is NULL");
    g_scratch_addr[dev] = p;
  }
  *out = g_scratch_addr[dev];
  return SPCONV_OK;
}

}  // namespace

extern "C" {

int spconv_forward_ex(const spconv_map* m, const void* d_x, const void* d_w, void* d_y, int c_in, int c_out,
                      int dtype, const void* d_residual, int relu, const spconv_options* opt, void* d_workspace,
                      size_t ws_bytes, void* stream) {
  return forward_impl(m, d_x, d_w, d_y, c_in, c_out, dtype, d_residual, relu, opt, d_workspace, ws_bytes, stream);
}

int spconv_forward_noalloc(const spconv_map* m, const void* d_x, const void* d_w, void* d_y, int c_in, int c_out,
                           int dtype, const void* d_residual, int relu, const spconv_options* opt, void* stream) {
  GmasPlan p;
  int st = make_plan(m, c_in, c_out, dtype, opt, &p);
  if (st != SPCONV_OK) return st;
  FwdBufs b;
  const size_t need = plan_forward_ws(nullptr, m, c_in, c_out, p, &b);
  if (need > (size_t)SPCONV_NOALLOC_SCRATCH_BYTES)
    return fail(SPCONV_ENOSPC, "layer needs " + std::to_string(need) + " bytes of forward workspace; the "
                "allocation-free forward holds " + std::to_string((size_t)SPCONV_NOALLOC_SCRATCH_BYTES));
  void* ws = nullptr;
  if ((st = scratch_address(&ws)) != SPCONV_OK) return st;
  return forward_impl(m, d_x, d_w, d_y, c_in, c_out, dtype, d_residual, relu, opt, ws,
                      (size_t)SPCONV_NOALLOC_SCRATCH_BYTES, stream);
}

}  // extern "C"

// ---------------------------------------------------------------------------
// Transformer operators
// ---------------------------------------------------------------------------
namespace {

bool known_dtype(int dtype) { return dtype == SPCONV_F32 || dtype == SPCONV_F16 || dtype == SPCONV_BF16; }
// A launcher's error as a status; hipErrorInvalidConfiguration is its refusal of the size.
int launched(hipError_t e, const char* where) {
  if (e == hipErrorInvalidConfiguration) return fail(SPCONV_EUNSUPPORTED, std::string(where) + ": more work than one launch takes");
  return e == hipSuccess ? SPCONV_OK : hip_fail(e, where);
}
bool misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

int check_attention(const spconv_attention_args* a) {
  if (!a) return fail(SPCONV_EINVAL, "args is NULL");
  if (!known_dtype(a->dtype)) return fail(SPCONV_EUNSUPPORTED, "dtype");
  if (a->n_q < 0 || a->n_k < 0 || a->n_docs < 0 || a->max_q < 0 || a->max_k < 0)
    return fail(SPCONV_EINVAL, "negative size");
  if (a->n_q > 0x7fffffff || a->n_k > 0x7fffffff) return fail(SPCONV_EUNSUPPORTED, "more than 2^31 - 1 rows");
  if (a->heads <= 0 || a->kv_heads <= 0 || a->heads % a->kv_heads != 0)
    return fail(SPCONV_EINVAL, "heads must be a multiple of kv_heads");
  if (a->max_k > 1 << 30) return fail(SPCONV_EUNSUPPORTED, "more than 2^30 keys in a document");
  if (a->heads > 65535) return fail(SPCONV_EUNSUPPORTED, "more than 65535 heads");
  if (a->head_dim < 8 || a->head_dim > 256 || a->head_dim % 8 != 0)
    return fail(SPCONV_EUNSUPPORTED, "head_dim must be a multiple of 8 up to 256");
  if (!(a->scale > 0.0f) || !std::isfinite(a->scale)) return fail(SPCONV_EINVAL, "scale must be positive and finite");
  if (!(a->cap >= 0.0f) || !std::isfinite(a->cap)) return fail(SPCONV_EINVAL, "cap must be finite and not negative");
  if ((a->d_q_pos == nullptr) != (a->d_k_pos == nullptr) || (a->d_q_pos && !a->d_slopes))
    return fail(SPCONV_EINVAL, "voxels are given for queries and keys, with slopes, or not at all");
  return SPCONV_OK;
}

// cap tanh(u), u = scale s / cap, as s times a polynomial of u^2.  Up to a cap of 64 the polynomials
// are the fits with the least largest error (of tanh: 1.3e-7 for |u| <= 1/2, and for |u| <= 0.11 by
// two terms; for float32 rows 3.1e-9), which is 8e-6 of a score at most.  That error grows with
// the cap: above 64 they are the series of tanh, taken where the first term left out is below
// float32's resolution of the score (by two terms also where it is below 8e-6).
void set_cap(AttnArgs* k, float cap, float scale, bool fine) {
  static const double kFit[2][5] = {{0.9999976762, -0.333206552, 0.131451455, -0.04337247954, 0.0},
                                    {0.9999999316, -0.3333277618, 0.1332057066, -0.05276212995, 0.01673756559}};
  static const double kSeries[5] = {1.0, -1.0 / 3, 2.0 / 15, -17.0 / 315, 62.0 / 2835};
  const bool fit = cap <= 64.0f;
  // a cap near float32's least number: its scores are all but 0
  const double by = std::min((double)scale / cap, 1e30), unit = scale * 1.4426950408889634;
  k->cap = cap;
  k->cap_log2 = (float)(cap * 1.4426950408889634);
  k->cap_by = (float)by;
  k->tanh_by = (float)(2 * 1.4426950408889634 * by);
  for (int i = 0; i < 5; ++i) k->poly[i] = (float)((fit ? kFit[fine][i] : kSeries[i]) * unit);
  k->poly_most = (float)std::min((fit ? 0.5 : fine ? 0.3 : 0.2) / by, 3e38);
  // two terms take u^2's factor into their coefficient, which must stay far from float32's ends
  const double low = fit ? 0.11 : std::max(0.026, std::pow(6e-5 / cap, 0.2));
  k->low_most = by >= 1e-12 && by <= 1e12 ? (float)(low / by) : -1.0f;
  k->low_top = (float)(0.99999 * cap * 1.4426950408889634 * std::tanh(low));  // a rounding below
  k->low[0] = (float)((fit ? 0.99999394 : 1.0) * unit);
  k->low[1] = (float)((fit ? -0.33132737 : -1.0 / 3) * unit * by * by);
}

AttnPlan plan_of(const spconv_attention_args* a, bool paged = false) {
  return attention_plan(a->n_q, a->n_docs, a->max_q, a->max_k, a->heads, a->kv_heads, a->head_dim, a->dtype,
                        a->causal != 0, paged);
}

size_t attention_bytes(const spconv_attention_args* a, const AttnPlan& p, void* base, f32x2** ml, float** o) {
  if (p.splits <= 1) return 0;
  Bump b(base);
  const int64_t rows = (int64_t)p.splits * a->n_q * a->heads;
  f32x2* m = b.take<f32x2>(rows);
  float* f = b.take<float>(rows * a->head_dim);
  if (ml) *ml = m;
  if (o) *o = f;
  return b.off;
}

// What both attention calls give their kernels, keys and the split of the launch apart.
AttnArgs attention_common(const spconv_attention_args* a, const AttnPlan& p) {
  constexpr float kLog2e = 1.4426950408889634f;
  AttnArgs k = {};
  k.q = a->d_q, k.out = a->d_out;
  k.q_row = a->q_row, k.q_head = a->q_head, k.out_row = a->out_row, k.out_head = a->out_head;
  k.q_start = a->d_q_start, k.k_len = a->d_k_len, k.prefix = a->d_prefix, k.slopes = a->d_slopes;
  k.n_q = a->n_q, k.n_docs = a->n_docs, k.max_q = a->max_q, k.max_k = a->max_k;
  k.heads = a->heads, k.kv_heads = a->kv_heads, k.d = a->head_dim, k.causal = a->causal;
  if (a->cap > 0.0f) set_cap(&k, a->cap, a->scale, a->dtype == SPCONV_F32);
  k.slope_by = a->cap > 0.0f ? kLog2e : 1.0f / a->scale;
  k.exp_by = a->cap > 0.0f ? 1.0f : a->scale * kLog2e;
  // below every finite score that matters, and finite in both units
  k.floor = -3e38f / std::max(1.0f, k.exp_by);
  k.slots = (int)p.slots, k.doc_slots = p.doc_slots, k.splits = p.splits, k.chunk = p.chunk;
  return k;
}

constexpr int kMostPage = 1 << 16;

// A cache of pages for rows of `dtype`; `n` rows of the call (no pointers are needed for none).
int check_pages(const spconv_pages* p, int dtype, int64_t n) {
  if (!p) return fail(SPCONV_EINVAL, "pages is NULL");
  if (!known_dtype(dtype)) return fail(SPCONV_EUNSUPPORTED, "dtype");
  if (n < 0 || p->n_pages < 0 || p->n_docs < 0 || p->table_row < 0) return fail(SPCONV_EINVAL, "negative size");
  if (n > 0x7fffffff) return fail(SPCONV_EUNSUPPORTED, "more than 2^31 - 1 rows");
  if (p->n_pages > 0x7fffffff) return fail(SPCONV_EUNSUPPORTED, "more than 2^31 - 1 pages");
  if (p->kv_heads <= 0) return fail(SPCONV_EINVAL, "no key heads");
  if (p->kv_heads > 65535) return fail(SPCONV_EUNSUPPORTED, "more than 65535 heads");
  if ((p->d_k_scale == nullptr) != (p->d_v_scale == nullptr))
    return fail(SPCONV_EINVAL, "scales are given for keys and values, or for neither");
  if (p->head_dim < 8 || p->head_dim > 256 || p->head_dim % (p->d_k_scale ? 16 : 8) != 0)
    return fail(SPCONV_EUNSUPPORTED, "head_dim must be a multiple of 8 (8-bit pages: of 16) up to 256");
  if (p->page < 1 || p->page > kMostPage || (p->page & (p->page - 1)) != 0)
    return fail(SPCONV_EUNSUPPORTED, "rows of a page must be a power of two up to 65536");
  if ((int64_t)p->kv_heads * p->page * p->head_dim > 1 << 29)  // (offsets inside a page have 32 bits, in bytes)
    return fail(SPCONV_EUNSUPPORTED, "more than 2^29 elements in a page of keys");
  if ((int64_t)p->table_row * p->page > 1 << 30) return fail(SPCONV_EUNSUPPORTED, "more than 2^30 keys in a document");
  if (n == 0 || p->n_docs == 0) return SPCONV_OK;
  if ((p->n_pages > 0 && (!p->d_k || !p->d_v)) || (p->table_row > 0 && !p->d_table)) return fail(SPCONV_EINVAL, "NULL pointer");
  if (misaligned16(p->d_k) || misaligned16(p->d_v)) return fail(SPCONV_EINVAL, "pages must be 16-byte aligned");
  for (const void* q : {(const void*)p->d_k_scale, (const void*)p->d_v_scale, (const void*)p->d_table})
    if (reinterpret_cast<uintptr_t>(q) % 4 != 0) return fail(SPCONV_EINVAL, "pointer not aligned to its elements");
  return SPCONV_OK;
}

PageArgs page_args(const spconv_pages* p) {
  return PageArgs{p->d_k, p->d_v, p->d_k_scale, p->d_v_scale, p->d_table, p->n_docs, p->table_row, (int)p->n_pages,
                  __builtin_ctz((unsigned)p->page), p->kv_heads, p->head_dim};
}

// Rows outside of the pages, keys and values.
int check_rows(const void* k, int64_t k_row, int64_t k_head, const void* v, int64_t v_row, int64_t v_head, int dtype) {
  if (!k || !v) return fail(SPCONV_EINVAL, "NULL pointer");
  if (misaligned16(k) || misaligned16(v)) return fail(SPCONV_EINVAL, "rows must be 16-byte aligned");
  for (int64_t stride : {k_row, k_head, v_row, v_head})
    if (stride < 0 || stride * (int64_t)elem_bytes(dtype) % 16 != 0)
      return fail(SPCONV_EUNSUPPORTED, "strides must be multiples of 16 bytes");
  return SPCONV_OK;
}

int check_cached_attention(const spconv_pages* p, const spconv_attention_args* a) {
  int st = check_attention(a);
  if (st != SPCONV_OK) return st;
  if ((st = check_pages(p, a->dtype, 0)) != SPCONV_OK) return st;
  if (p->kv_heads != a->kv_heads || p->head_dim != a->head_dim || p->n_docs != a->n_docs)
    return fail(SPCONV_EINVAL, "pages and queries differ in key heads, head_dim or documents");
  if (a->d_q_pos) return fail(SPCONV_EUNSUPPORTED, "pages hold no voxels");
  if (a->n_q * (a->heads / a->kv_heads) > 0x7fffffff)
    return fail(SPCONV_EUNSUPPORTED, "more than 2^31 - 1 queries of the heads of a key head");
  return SPCONV_OK;
}

}  // namespace

extern "C" {

int spconv_rms_norm(const void* d_x, int64_t ld_x, const void* d_residual, int64_t ld_residual, const void* d_gamma,
                    void* d_sum, int64_t ld_sum, void* d_y, int64_t ld_y, float* d_scale, int64_t ld_scale, int64_t n,
                    int c, int dtype, int bits8, float eps, void* stream) {
  if (!known_dtype(dtype)) return fail(SPCONV_EUNSUPPORTED, "dtype");
  if (n < 0 || c <= 0) return fail(SPCONV_EINVAL, "negative number of rows, or no columns");
  if (n > 0x7fffffff) return fail(SPCONV_EUNSUPPORTED, "more than 2^31 - 1 rows");
  if (bits8 && c % 16 != 0) return fail(SPCONV_EUNSUPPORTED, "8-bit rows need 16-byte rows: c % 16 == 0");
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(SPCONV_EINVAL, "eps must be finite and not negative");
  if (ld_x < c || ld_y < c || (d_residual && ld_residual < c) || (d_sum && ld_sum < c) ||
      (bits8 && ld_scale < (c + kScaleBlock - 1) / kScaleBlock))
    return fail(SPCONV_EINVAL, "row stride shorter than a row");
  if (d_sum && !d_residual) return fail(SPCONV_EINVAL, "d_sum without d_residual");
  if (n == 0) return SPCONV_OK;
  if (!d_x || !d_gamma || !d_y || (bits8 && !d_scale)) return fail(SPCONV_EINVAL, "NULL pointer");
  const uintptr_t e = elem_bytes(dtype);
  for (const void* p : {d_x, d_residual, d_gamma, (const void*)d_sum, bits8 ? nullptr : (const void*)d_y})
    if (reinterpret_cast<uintptr_t>(p) % e != 0) return fail(SPCONV_EINVAL, "pointer not aligned to its elements");
  if (bits8 && reinterpret_cast<uintptr_t>(d_scale) % 4 != 0) return fail(SPCONV_EINVAL, "d_scale must be 4-byte aligned");
  SPC_TRY(launch_rms_norm(d_x, ld_x, d_residual, ld_residual, d_gamma, d_sum, ld_sum, d_y, ld_y, d_scale, ld_scale, n, c,
                          dtype, bits8 != 0, eps, static_cast<hipStream_t>(stream)),
          "norm");
  return SPCONV_OK;
}

int spconv_scaled_linear(const void* d_x, int64_t ld_x, const float* d_x_scale, int64_t ld_x_scale, const void* d_w,
                         int64_t ld_w, const float* d_w_scale, int64_t ld_w_scale, void* d_y, int64_t ld_y, int64_t m,
                         int n, int k, int dtype, int relu, int exact, void* stream) {
  if (!known_dtype(dtype)) return fail(SPCONV_EUNSUPPORTED, "dtype");
  if (m < 0 || n < 0 || k < 0) return fail(SPCONV_EINVAL, "negative size");
  if (k % 16 != 0 || (k > 0 && (ld_x % 16 != 0 || ld_w % 16 != 0)))
    return fail(SPCONV_EUNSUPPORTED, "8-bit rows need 16-byte rows: k, ld_x and ld_w multiples of 16");
  const int kb = (k + kScaleBlock - 1) / kScaleBlock;
  if (ld_x < k || ld_w < k || ld_y < n || ld_x_scale < kb || ld_w_scale < kb)
    return fail(SPCONV_EINVAL, "row stride shorter than a row");
  if (m > 0x7fffffff) return fail(SPCONV_EUNSUPPORTED, "more than 2^31 - 1 rows");
  if (ld_x > kMostLinearStride || ld_w > kMostLinearStride || ld_x_scale > kMostLinearStride / 4)
    return fail(SPCONV_EUNSUPPORTED, "rows of d_x, d_w and d_x_scale at most 8 MiB apart");
  if (m == 0 || n == 0) return SPCONV_OK;
  if (!d_y || (k > 0 && (!d_x || !d_x_scale || !d_w || !d_w_scale))) return fail(SPCONV_EINVAL, "NULL pointer");
  if (misaligned16(d_x) || misaligned16(d_w)) return fail(SPCONV_EINVAL, "d_x and d_w must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(d_y) % elem_bytes(dtype) != 0 || reinterpret_cast<uintptr_t>(d_x_scale) % 4 != 0 ||
      reinterpret_cast<uintptr_t>(d_w_scale) % 4 != 0)
    return fail(SPCONV_EINVAL, "pointer not aligned to its elements");
  return launched(launch_scaled_linear(d_x, ld_x, d_x_scale, ld_x_scale, d_w, ld_w, d_w_scale, ld_w_scale, d_y, ld_y, m, n,
                                       k, dtype, relu, exact != 0, static_cast<hipStream_t>(stream)),
                  "scaled product");
}

size_t spconv_attention_workspace_bytes(const spconv_attention_args* a) {
  if (check_attention(a) != SPCONV_OK) return 0;
  return attention_bytes(a, plan_of(a), nullptr, nullptr, nullptr);
}

int spconv_attention(const spconv_attention_args* a, void* d_workspace, size_t ws_bytes, void* stream) {
  const int st = check_attention(a);
  if (st != SPCONV_OK) return st;
  if (a->n_q == 0 || a->n_docs == 0) return SPCONV_OK;
  if (a->max_q == 0) return fail(SPCONV_EINVAL, "max_q is 0 but there are queries");
  if (!a->d_q || !a->d_out || !a->d_q_start || !a->d_k_start || (a->n_k > 0 && a->max_k > 0 && (!a->d_k || !a->d_v)))
    return fail(SPCONV_EINVAL, "NULL pointer");
  if (misaligned16(a->d_q) || misaligned16(a->d_k) || misaligned16(a->d_v) || misaligned16(a->d_out))
    return fail(SPCONV_EINVAL, "d_q, d_k, d_v and d_out must be 16-byte aligned");
  const int64_t e = elem_bytes(a->dtype);
  for (int64_t stride : {a->q_row, a->q_head, a->k_row, a->k_head, a->v_row, a->v_head, a->out_row, a->out_head})
    if (stride < 0 || stride * e % 16 != 0) return fail(SPCONV_EUNSUPPORTED, "strides must be multiples of 16 bytes");
  if (a->k_row * e > kMostRowBytes || a->v_row * e > kMostRowBytes)
    return fail(SPCONV_EUNSUPPORTED, "rows of d_k and d_v at most 32 MiB apart");
  if ((a->heads > 1 && a->out_head < a->head_dim) || (a->n_q > 1 && a->out_row < a->head_dim))
    return fail(SPCONV_EINVAL, "rows or heads of d_out overlap");
  const AttnPlan p = plan_of(a);
  AttnArgs k = attention_common(a, p);
  const size_t need = attention_bytes(a, p, d_workspace, &k.part_ml, &k.part_o);
  if (need > 0 && (!d_workspace || ws_bytes < need)) return fail(SPCONV_ENOSPC, "attention workspace too small");
  if (reinterpret_cast<uintptr_t>(d_workspace) % 256 != 0) return fail(SPCONV_EINVAL, "workspace must be 256-byte aligned");
  k.k = a->d_k, k.v = a->d_v;
  k.k_row = a->k_row, k.k_head = a->k_head, k.v_row = a->v_row, k.v_head = a->v_head;
  k.k_start = a->d_k_start, k.q_pos = a->d_q_pos, k.k_pos = a->d_k_pos, k.n_k = a->n_k;
  return launched(launch_attention(k, p, a->dtype, static_cast<hipStream_t>(stream)), "attention");
}

size_t spconv_cached_attention_workspace_bytes(const spconv_pages* pages, const spconv_attention_args* a) {
  if (check_cached_attention(pages, a) != SPCONV_OK) return 0;
  return attention_bytes(a, plan_of(a, true), nullptr, nullptr, nullptr);
}

int spconv_cached_attention(const spconv_pages* pages, const spconv_attention_args* a, void* d_workspace, size_t ws_bytes,
                            void* stream) {
  int st = check_cached_attention(pages, a);
  if (st != SPCONV_OK) return st;
  if (a->n_q == 0 || a->n_docs == 0) return SPCONV_OK;
  if ((st = check_pages(pages, a->dtype, a->n_q)) != SPCONV_OK) return st;
  if (a->max_q == 0) return fail(SPCONV_EINVAL, "max_q is 0 but there are queries");
  if (!a->d_q || !a->d_out || !a->d_q_start || !a->d_k_len) return fail(SPCONV_EINVAL, "NULL pointer");
  if (misaligned16(a->d_q) || misaligned16(a->d_out)) return fail(SPCONV_EINVAL, "d_q and d_out must be 16-byte aligned");
  const int64_t e = elem_bytes(a->dtype);
  for (int64_t stride : {a->q_row, a->q_head, a->out_row, a->out_head})
    if (stride < 0 || stride * e % 16 != 0) return fail(SPCONV_EUNSUPPORTED, "strides must be multiples of 16 bytes");
  if ((a->heads > 1 && a->out_head < a->head_dim) || (a->n_q > 1 && a->out_row < a->head_dim))
    return fail(SPCONV_EINVAL, "rows or heads of d_out overlap");
  const AttnPlan p = plan_of(a, true);
  AttnArgs k = attention_common(a, p);
  const size_t need = attention_bytes(a, p, d_workspace, &k.part_ml, &k.part_o);
  if (need > 0 && (!d_workspace || ws_bytes < need)) return fail(SPCONV_ENOSPC, "attention workspace too small");
  if (reinterpret_cast<uintptr_t>(d_workspace) % 256 != 0) return fail(SPCONV_EINVAL, "workspace must be 256-byte aligned");
  const PageArgs pg = page_args(pages);
  k.k = pg.k, k.v = pg.v, k.k_scale = pg.k_scale, k.v_scale = pg.v_scale;
  k.paged = 1, k.table = pg.table, k.table_row = pg.table_row, k.n_pages = pg.n_pages, k.shift = pg.shift;
  k.n_k = (int64_t)pg.table_row << pg.shift;
  return launched(launch_attention(k, p, a->dtype, static_cast<hipStream_t>(stream)), "attention over pages");
}

int spconv_cache_write(const spconv_pages* pages, const void* d_k, int64_t k_row, int64_t k_head, const void* d_v,
                       int64_t v_row, int64_t v_head, const int32_t* d_q_start, const int32_t* d_k_len, int64_t n,
                       int dtype, void* stream) {
  int st = check_pages(pages, dtype, n);
  if (st != SPCONV_OK || n == 0 || pages->n_docs == 0) return st;
  if ((st = check_rows(d_k, k_row, k_head, d_v, v_row, v_head, dtype)) != SPCONV_OK) return st;
  if (!d_q_start || !d_k_len) return fail(SPCONV_EINVAL, "NULL pointer");
  return launched(launch_cache(page_args(pages), HeadRows{const_cast<void*>(d_k), k_row, k_head},
                               HeadRows{const_cast<void*>(d_v), v_row, v_head}, d_q_start, d_k_len, n, dtype,
                               static_cast<hipStream_t>(stream)),
                  "cache write");
}

int spconv_cache_read(const spconv_pages* pages, void* d_k, int64_t k_row, int64_t k_head, void* d_v, int64_t v_row,
                      int64_t v_head, const int32_t* d_start, int64_t n, int dtype, void* stream) {
  int st = check_pages(pages, dtype, n);
  if (st != SPCONV_OK || n == 0 || pages->n_docs == 0) return st;
  if ((st = check_rows(d_k, k_row, k_head, d_v, v_row, v_head, dtype)) != SPCONV_OK) return st;
  for (int64_t row : {k_row, v_row})
    if (n > 1 && row < pages->head_dim) return fail(SPCONV_EINVAL, "rows of the output overlap");
  for (int64_t head : {k_head, v_head})
    if (pages->kv_heads > 1 && head < pages->head_dim) return fail(SPCONV_EINVAL, "heads of the output overlap");
  if (!d_start) return fail(SPCONV_EINVAL, "NULL pointer");
  return launched(launch_cache(page_args(pages), HeadRows{d_k, k_row, k_head}, HeadRows{d_v, v_row, v_head}, d_start, nullptr,
                               n, dtype, static_cast<hipStream_t>(stream)),
                  "cache read");
}

int spconv_rotate_heads(const spconv_rotation* r, void* stream) {
  if (!r) return fail(SPCONV_EINVAL, "args is NULL");
  if (!known_dtype(r->dtype)) return fail(SPCONV_EUNSUPPORTED, "dtype");
  if (r->n < 0 || r->heads <= 0 || r->kv_heads < 0) return fail(SPCONV_EINVAL, "negative size, or no heads");
  if (r->n > 0x7fffffff) return fail(SPCONV_EUNSUPPORTED, "more than 2^31 - 1 rows");
  if (r->heads > 65535 || r->kv_heads > 65535) return fail(SPCONV_EUNSUPPORTED, "more than 65535 heads");
  if (r->head_dim < 1 || r->head_dim > kMostRotated) return fail(SPCONV_EUNSUPPORTED, "head_dim must be 1 to 256");
  if (r->rotated < 0 || r->rotated > r->head_dim || r->rotated % 2 != 0)
    return fail(SPCONV_EINVAL, "rotated columns must be an even number, at most head_dim");
  if (!(r->eps >= 0.0f) || !std::isfinite(r->eps)) return fail(SPCONV_EINVAL, "eps must be finite and not negative");
  if (!std::isfinite(r->gain)) return fail(SPCONV_EINVAL, "gain must be finite");
  if (r->n == 0) return SPCONV_OK;
  RotateArgs k = {{r->d_q, r->d_k}, {r->d_q_out, r->d_k_out}, {r->q_row, r->k_row}, {r->q_head, r->k_head},
                  {r->q_out_row, r->k_out_row}, {r->q_out_head, r->k_out_head}, {r->d_q_gamma, r->d_k_gamma}, r->d_pos,
                  r->d_freq, r->n, {r->heads, r->kv_heads}, r->head_dim, r->rotated, r->voxels != 0, r->eps, r->gain, 1, 1};
  const uintptr_t e = elem_bytes(r->dtype);
  for (int i = 0; i < 2; ++i) {
    if (k.heads[i] == 0) {
      k.x[i] = nullptr, k.y[i] = nullptr, k.gamma[i] = nullptr;
      k.x_row[i] = k.x_head[i] = k.y_row[i] = k.y_head[i] = 0;
      continue;
    }
    if (!k.x[i] || !k.y[i]) return fail(SPCONV_EINVAL, "NULL pointer");
    if (k.x_row[i] < 0 || k.x_head[i] < 0) return fail(SPCONV_EINVAL, "negative stride");
    if ((r->n > 1 && k.y_row[i] < r->head_dim) || (k.heads[i] > 1 && k.y_head[i] < r->head_dim) || k.y_row[i] < 0 || k.y_head[i] < 0)
      return fail(SPCONV_EINVAL, "rows or heads of the output overlap");
    for (const void* p : {k.x[i], (const void*)k.y[i], k.gamma[i]})
      if (reinterpret_cast<uintptr_t>(p) % e != 0) return fail(SPCONV_EINVAL, "pointer not aligned to its elements");
  }
  if (r->rotated > 0 && (!r->d_pos || !r->d_freq)) return fail(SPCONV_EINVAL, "NULL pointer");
  if (reinterpret_cast<uintptr_t>(r->d_pos) % 4 != 0 || reinterpret_cast<uintptr_t>(r->d_freq) % 8 != 0)
    return fail(SPCONV_EINVAL, "pointer not aligned to its elements");
  return launched(launch_rotate(k, r->dtype, r->interleaved != 0, static_cast<hipStream_t>(stream)), "rotation");
}

// --------------------------------------------------------------- measurement
int spconv_profile_enable(uint64_t mask) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  g_prof_mask = mask;
  return SPCONV_OK;
}

int spconv_profile_phase_count(void) { return PROF_IDS; }
const char* spconv_profile_phase_name(int i) { return prof_name(i); }

int spconv_profile_read(double* ms, int64_t* launches, int n, int reset) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  if (!ms || !launches || n < PROF_IDS) return fail(SPCONV_EINVAL, "need spconv_profile_phase_count() entries");
  for (int i = 0; i < PROF_IDS; ++i) {
    ms[i] = 0.0;
    launches[i] = 0;
  }
  for (auto& r : g_recs) {
    float t = 0.f;
    if (hipEventSynchronize(r.b) != hipSuccess) return fail(SPCONV_EHIP, "event sync");
    if (hipEventElapsedTime(&t, r.a, r.b) != hipSuccess) return fail(SPCONV_EHIP, "event elapsed");
    ms[r.phase] += t;
    launches[r.phase] += 1;
  }
  if (reset) {
    for (auto& r : g_recs) {
      g_pool.push_back(r.a);
      g_pool.push_back(r.b);
    }
    g_recs.clear();
  }
  return SPCONV_OK;
}

}  // extern "C"
