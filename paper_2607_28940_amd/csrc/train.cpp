// C ABI of the training operators: checks, work planning and launches of
// tx_rel_attn_*, tx_event_attn_* and tx_preference_*. Host code only.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#pragma GCC visibility push(default)
#include "transx.h"
#pragma GCC visibility pop

#include "api_internal.h"
#include "meta_put.h"
#include "preference.h"
#include "train_attn.h"

using namespace tx;

namespace {

constexpr int64_t kMaxRows = 0x7fffffff - 4096;
constexpr int64_t kMaxGrid = 0xffffffffll / 256;  // blocks of 256 threads in a launch
// How a launch is cut into blocks (256 CUs). Narrow blocks below kWideGrid wide
// ones: 1000 causal tokens of 8 heads (64 wide blocks) forward 48 -> 17 us, dq 50
// -> 26, dk and dv 52 -> 25; 4096 (256) 100 -> 86, 127 -> 112, 149 -> 137; 17 k
// queries of 2.3 k keys (1136) 98 -> 149.
// Where that leaves fewer blocks than the card holds, the other side of a block
// is divided into parts, towards kFullGrid blocks of an equal share, but none
// below kMinSteps 64-row tiles (kMinStepsF32 in fp32, whose tiles take longer) a
// wave, and not at all if that would not halve the block: what the parts write
// and the join reads costs more than it saves (4096 tokens 86 -> 131 us towards
// 1024 blocks, 1000 tokens 17 -> 31 us at 2 tiles a part).
constexpr int64_t kWideGrid = 512, kFullGrid = 512;
// Shared key heads: with a full card packed blocks throughout (few rows of 32
// users, 16 heads on 4: 94 -> 83 us forward, 111 -> 97 dq). With less, packed ones
// read the keys a quarter as often but run a chain of tiles four times as long: of
// 4 heads at d_head 64 and less from 4096 keys on (3 users of 8192, 45 rows each:
// 53 -> 43 us; of 1024: 14 -> 24); two heads (8192: 48 us both) and d_head 128, half
// as many blocks a CU (49 -> 59), do not gain.
constexpr int kPackKeys = 4096;
constexpr int64_t kSortGrid = 4096;
constexpr int kMaxParts = 64, kMinSteps = 4, kMinStepsF32 = 2;

// Metadata goes up as kernel arguments, 3 KB a launch: no staging buffer whose
// reuse would have to wait, and a captured graph keeps its own copy.
hipError_t put_all(char* dst, const std::vector<char>& src, hipStream_t s) {
  for (size_t o = 0; o < src.size(); o += sizeof(MetaArg)) {
    const hipError_t e = put_meta(dst + o, src.data() + o, std::min(sizeof(MetaArg), src.size() - o), s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

int check_offsets(const int64_t* off, int64_t n, const char* what) {
  if (!off) return fail(TX_E_INVALID, "%s offsets are null", what);
  if (off[0] < 0) return fail(TX_E_INVALID, "%s offsets start at %lld", what, (long long)off[0]);
  for (int64_t i = 0; i < n; ++i)
    if (off[i + 1] < off[i]) return fail(TX_E_INVALID, "%s offsets decrease at %lld", what, (long long)i);
  if (off[n] > kMaxRows) return fail(TX_E_UNSUPPORTED, "%s offsets reach %lld rows", what, (long long)off[n]);
  return TX_OK;
}

int check_stream(hipStream_t st) {
  if (!st) return TX_OK;
  int dev = -1;
  hipDevice_t sdev = -1;
  TX_HIP(hipGetDevice(&dev));
  TX_HIP(hipStreamGetDevice(st, &sdev));
  if (sdev != dev) return fail(TX_E_INVALID, "stream belongs to device %d, the current device is %d", sdev, dev);
  return TX_OK;
}

int check_ws(const void* ws, size_t have, size_t need) {
  if (need == 0) return TX_OK;
  if (!ws) return fail(TX_E_INVALID, "workspace is null");
  if ((uintptr_t)ws & 255) return fail(TX_E_INVALID, "workspace not 256-byte aligned");
  if (have < need) return fail(TX_E_NOMEM, "workspace %zu bytes < %zu", have, need);
  return TX_OK;
}

// ------------------------------------------------------------------ attention

int check_attn_config(const tx_attn_config* c, bool rel) {
  if (!c) return fail(TX_E_INVALID, "config is null");
  if (c->dtype != TX_F32 && c->dtype != TX_BF16) return fail(TX_E_INVALID, "dtype %d unknown", c->dtype);
  if (c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads)
    return fail(TX_E_INVALID, "n_heads %d must be a positive multiple of n_kv_heads %d", c->n_heads, c->n_kv_heads);
  if (c->n_heads > 65536) return fail(TX_E_UNSUPPORTED, "n_heads %d above 65536", c->n_heads);
  if (c->d_head != 32 && c->d_head != 64 && c->d_head != 128)
    return fail(TX_E_UNSUPPORTED, "d_head %d not in {32, 64, 128}", c->d_head);
  if (c->rel_pos_buckets < 0 || (!rel && c->rel_pos_buckets))
    return fail(TX_E_INVALID, "rel_pos_buckets %d", c->rel_pos_buckets);
  if (c->rel_pos_buckets > kTrainMaxRel)
    return fail(TX_E_UNSUPPORTED, "rel_pos_buckets %d above %d", c->rel_pos_buckets, kTrainMaxRel);
  if (!(c->scale >= 0.f) || !std::isfinite(c->scale))
    return fail(TX_E_INVALID, "scale must be finite and not negative");
  return TX_OK;
}

// rows: one past the last row in use; out: written, so rows and heads lie apart
int check_rows(const tx_rows* t, const char* what, int es, int64_t heads, int dh, int64_t rows, bool out,
               HeadRows* dst) {
  if (!t) return fail(TX_E_INVALID, "%s is null", what);
  if (rows > 0 && !t->data) return fail(TX_E_INVALID, "%s data is null", what);
  if (((uintptr_t)t->data & 15) || (t->row_stride * es) % 16 || (t->head_stride * es) % 16)
    return fail(TX_E_INVALID, "%s: data and strides must be multiples of 16 bytes", what);
  if (t->row_stride < 0 || t->head_stride < 0) return fail(TX_E_INVALID, "%s: negative stride", what);
  if (t->row_stride > (16 << 20) / es)
    return fail(TX_E_UNSUPPORTED, "%s: row stride %lld above 16 MiB", what, (long long)t->row_stride);
  if (t->head_stride > ((int64_t)1 << 55) / heads) return fail(TX_E_UNSUPPORTED, "%s: head stride", what);
  if (out && rows > 0) {
    const bool heads_in_row = (heads == 1 || t->head_stride >= dh) &&
                              (rows == 1 || t->row_stride >= (heads - 1) * t->head_stride + dh);
    const bool rows_in_head = (rows == 1 || t->row_stride >= dh) &&
                              (heads == 1 || t->head_stride >= (rows - 1) * t->row_stride + dh);
    if (!heads_in_row && !rows_in_head) return fail(TX_E_INVALID, "%s: its rows or heads overlap", what);
  }
  *dst = HeadRows{(char*)t->data, t->row_stride * es, t->head_stride * es};
  return TX_OK;
}

// Where a tensor is written, nothing else begins (what else overlaps is the caller's to avoid).
int check_apart(const TrainArgs& a, int64_t rows_q, int64_t rows_k, bool backward) {
  const struct {
    const HeadRows* t;
    const char* name;
    int64_t rows;
    bool out;
  } all[] = {{&a.q, "q", rows_q, false},         {&a.k, "k", rows_k, false},       {&a.v, "v", rows_k, false},
             {&a.o, "out", rows_q, !backward},   {&a.dO, "d_out", rows_q, false},  {&a.dq, "d_q", rows_q, true},
             {&a.dk, "d_k", rows_k, true},       {&a.dv, "d_v", rows_k, true}};
  const int n = backward ? 8 : 4;
  for (int i = 0; i < n; ++i)
    for (int j = 0; all[i].out && j < n; ++j)
      if (i != j && all[i].rows && all[j].rows && all[i].t->p == all[j].t->p)
        return fail(TX_E_INVALID, "%s is written and begins where %s does", all[i].name, all[j].name);
  return TX_OK;
}

// Groups of a call with their units of work, and the layout of its workspace.
struct AttnPlan {
  std::vector<TrainGroup> groups;
  std::vector<int32_t> ev_row, ev_prefix;  // event form
  int q_rows = kWideRows, k_rows = kWideRows, pack = 0;
  bool q_narrow = false, k_narrow = false;
  int64_t units_q = 0, units_k = 0, tiles = 0, slots_q = 0, slots_k = 0;
  double pairs = 0;                        // visible (query, key) pairs
  int64_t rows_q = 0, rows_k = 0;          // rows of the call
  int64_t end_q = 0, end_k = 0;            // one past the last row
  int64_t q_base = 0;
  std::vector<char> meta;
  size_t o_row = 0, o_prefix = 0, o_q = 0, o_k = 0;  // in meta; o_q, o_k 0: none
  size_t bytes = 0;
  struct {
    size_t row_lim, tile_lim, stat, partial, drel, drel2;
  } at;
};

// Parts of a block that goes through `steps` tiles, `target` to a part.
int parts_of(int64_t steps, int64_t target) {
  if (steps < 2 * target) return 1;
  return (int)std::min<int64_t>(kMaxParts, (steps + target - 1) / target);
}

// (block: a power of two)
int64_t blocks_of(int64_t rows, int block = kWideRows) { return (rows + block - 1) >> __builtin_ctz(block); }
int64_t tiles_of(int64_t rows) { return blocks_of(rows, kTrainQTile); }

// Indexes of `work`, most first (in 1024 steps of the largest; equals in order).
std::vector<uint32_t> most_first(const std::vector<int64_t>& work) {
  constexpr int kSteps = 1024;
  const size_t n = work.size();
  std::vector<uint32_t> order(n);
  int64_t top = 1;
  for (const int64_t w : work) top = std::max(top, w);
  const double scale = (kSteps - 1) / (double)top;
  uint32_t at[kSteps + 1] = {};
  std::vector<uint16_t> step(n);
  for (size_t i = 0; i < n; ++i) ++at[(step[i] = (uint16_t)(kSteps - 1 - (int)(work[i] * scale))) + 1];
  for (int t = 0; t < kSteps; ++t) at[t + 1] += at[t];
  for (size_t i = 0; i < n; ++i) order[at[step[i]]++] = (uint32_t)i;
  return order;
}

// Units of one side by the tiles they go through, longest first, so that the
// blocks that end a launch are short ones (12 users of 1.5 to 4.1 k keys, 17 k
// queries: dk and dv 188 -> 157 us, forward 97 -> 91). Only for calls of a few
// rounds of blocks (kSortGrid): longer ones even out by themselves, and there a
// group's blocks together find its rows in the L2 caches.
bool sorted_units(const AttnPlan& p, bool keys, int64_t heads) {
  return (keys ? p.units_k : p.units_q) * heads <= kSortGrid && p.groups.size() <= 0xffff;
}
std::vector<uint32_t> order_units(const AttnPlan& p, bool keys, bool rel) {
  const int rows = keys ? p.k_rows : p.q_rows;
  std::vector<int64_t> work, at;
  std::vector<uint32_t> ref;
  for (size_t i = 0; i < p.groups.size(); ++i) {
    const TrainGroup& g = p.groups[i];
    const int64_t blocks = blocks_of(keys ? g.nk : g.nq, rows), parts = keys ? g.parts_k : g.parts_q;
    at.assign(blocks + 1, 0);
    if (rel) {
      for (int64_t b = 0; b < blocks; ++b) at[b] = keys ? g.nq - b * rows : std::min<int64_t>(g.nq, (b + 1) * rows);
    } else {
      for (int e = g.e0; e < g.e1; ++e) {
        const int64_t r0 = p.ev_row[e] - g.q0, r1 = (e + 1 < g.e1 ? p.ev_row[e + 1] : g.q0 + g.nq) - g.q0;
        if (r1 <= r0 || p.ev_prefix[e] == 0) continue;
        if (keys) {
          at[0] += r1 - r0;
          at[(p.ev_prefix[e] - 1) / rows + 1] -= r1 - r0;
        } else {
          for (int64_t b = r0 / rows; b <= (r1 - 1) / rows; ++b) at[b] = std::max<int64_t>(at[b], p.ev_prefix[e]);
        }
      }
      if (keys)
        for (int64_t b = 1; b < blocks; ++b) at[b] += at[b - 1];
    }
    for (int64_t b = 0; b < blocks; ++b)
      for (int64_t part = 0; part < parts; ++part) {  // (queries: the last block is the first unit)
        work.push_back(at[b] / parts);
        ref.push_back((uint32_t)(i | ((keys ? b : blocks - 1 - b) * parts + part) << 16));
      }
  }
  std::vector<uint32_t> order = most_first(work);
  for (uint32_t& x : order) x = ref[x];
  return order;
}

// run: with the contents of the metadata, not its size alone
void finish_plan(const tx_attn_config& c, bool backward, bool rel, bool run, AttnPlan& p) {
  const int H = c.n_heads, G = c.n_kv_heads, dh = c.d_head;
  // keys that the group's rows reach (tile steps of a query block)
  auto reach = [&](const TrainGroup& g) -> int64_t {
    if (rel) return g.nk;
    int32_t m = 0;
    for (int e = g.e0; e < g.e1; ++e) m = std::max(m, p.ev_prefix[e]);
    return m;
  };
  std::vector<int64_t> keys(p.groups.size());
  for (size_t i = 0; i < p.groups.size(); ++i) keys[i] = reach(p.groups[i]);
  if (run && p.groups.size() > 1) {
    // most work first: blocks are dealt to the card in order
    std::vector<int64_t> work(p.groups.size());
    for (size_t i = 0; i < work.size(); ++i) work[i] = keys[i] * p.groups[i].nq;
    std::vector<TrainGroup> sorted;
    std::vector<int64_t> sorted_keys;
    for (const uint32_t i : most_first(work)) sorted.push_back(p.groups[i]), sorted_keys.push_back(keys[i]);
    p.groups.swap(sorted);
    keys.swap(sorted_keys);
  }
  // wide blocks where they would fill the card, narrow ones otherwise
  int64_t wide_q = 0, wide_k = 0;
  double pairs_of_rows = 0;
  for (size_t i = 0; i < p.groups.size(); ++i) {
    const TrainGroup& g = p.groups[i];
    wide_q += blocks_of(g.nq) * H, wide_k += blocks_of(g.nk) * G;
    pairs_of_rows += (double)g.nq * keys[i];
  }
  const int per = H / G;
  p.pack = rel ? 0 : per % 4 == 0 ? 2 : per % 2 == 0 ? 1 : 0;
  if (wide_q < kWideGrid && !(p.pack == 2 && dh <= 64 && pairs_of_rows >= kPackKeys * (double)p.rows_q)) p.pack = 0;
  p.q_narrow = !p.pack && wide_q < kWideGrid;
  p.k_narrow = wide_k < kWideGrid;
  // a narrow block's tiles (128 KB at d_head 128) leave room for the bias sums of
  // some 1300 buckets
  if (backward && rel && train_dq_lds(c.dtype == TX_BF16, dh, c.rel_pos_buckets, p.q_narrow) > kTrainMaxLds)
    p.q_narrow = false;
  p.q_rows = p.q_narrow ? kNarrowRows : kWideRows >> p.pack;
  p.k_rows = p.k_narrow ? kNarrowRows : kWideRows;
  int64_t steps_q = 0, steps_k = 0;
  for (size_t i = 0; i < p.groups.size(); ++i) {
    const TrainGroup& g = p.groups[i];
    const double share = rel ? 0.5 : 1.0;  // a causal block covers half of the group's tiles on average
    steps_q += (int64_t)std::ceil(blocks_of(g.nq, p.q_rows) * tiles_of(keys[i]) * share) * (H >> p.pack);
    steps_k += (int64_t)std::ceil(blocks_of(g.nk, p.k_rows) * tiles_of(g.nq) * per * share) * G;
  }
  const int min_steps = c.dtype == TX_F32 ? kMinStepsF32 : kMinSteps;
  auto target = [&](int64_t total, bool narrow) {
    return std::max<int64_t>(narrow ? 4 * min_steps : min_steps, (total + kFullGrid - 1) / kFullGrid);
  };
  const int64_t target_q = target(steps_q, p.q_narrow), target_k = target(steps_k, p.k_narrow);
  for (size_t i = 0; i < p.groups.size(); ++i) {
    TrainGroup& g = p.groups[i];
    const int64_t bq = blocks_of(g.nq, p.q_rows), bk = blocks_of(g.nk, p.k_rows);
    g.parts_q = g.nq ? parts_of(tiles_of(keys[i]), target_q) : 1;
    g.unit_q = (int32_t)p.units_q;
    g.slot_q = (int32_t)p.slots_q;
    g.qt0 = (int32_t)p.tiles;
    p.units_q += bq * g.parts_q;
    if (g.parts_q > 1) p.slots_q += bq * g.parts_q * H;
    p.tiles += tiles_of(g.nq);
    g.parts_k = g.nk ? parts_of(tiles_of(g.nq) * per, target_k) : 1;
    g.unit_k = (int32_t)p.units_k;
    g.slot_k = (int32_t)p.slots_k;
    p.units_k += bk * g.parts_k;
    if (g.parts_k > 1) p.slots_k += bk * g.parts_k * G;
  }
  size_t meta = 0;
  auto put = [&](const void* src, size_t n) {
    const size_t o = align_up(meta, 64);
    meta = o + n;
    if (run) {
      p.meta.resize(meta);
      if (n) memcpy(p.meta.data() + o, src, n);
    }
    return o;
  };
  if (run) p.meta.reserve(p.groups.size() * sizeof(TrainGroup) + (p.ev_row.size() + p.ev_prefix.size()) * 4 + 65536);
  put(p.groups.data(), p.groups.size() * sizeof(TrainGroup));
  p.o_row = put(p.ev_row.data(), p.ev_row.size() * 4);
  p.o_prefix = put(p.ev_prefix.data(), p.ev_prefix.size() * 4);
  auto put_order = [&](bool of_keys, int64_t heads) -> size_t {
    if (!sorted_units(p, of_keys, heads)) return 0;
    if (!run) return put(nullptr, (of_keys ? p.units_k : p.units_q) * 4);
    const std::vector<uint32_t> order = order_units(p, of_keys, rel);
    return put(order.data(), order.size() * 4);
  };
  p.o_q = put_order(false, H >> p.pack);
  if (backward) p.o_k = put_order(true, G);
  Carver cv(nullptr);
  auto take = [&](size_t n) {
    cv.take<char*>(n);
    return cv.off - n;
  };
  take(meta);
  p.at.row_lim = take(rel ? 0 : (p.rows_q + 1) * 4);
  p.at.tile_lim = take(rel ? 0 : p.tiles * sizeof(TileLim));
  p.at.stat = take(backward ? (size_t)H * p.rows_q * 8 : 0);
  // dq and then dk, dv use the slots in turn
  const size_t sq = p.slots_q * (backward ? train_dq_slot(p.q_rows, dh) : train_fwd_slot(p.q_rows, dh));
  const size_t sk = backward ? p.slots_k * train_dkv_slot(p.k_rows, dh) : 0;
  p.at.partial = take(std::max(sq, sk) * 4);
  const size_t HR = rel && backward ? (size_t)H * c.rel_pos_buckets : 0;
  p.at.drel = take(HR * p.units_q * 4);
  p.at.drel2 = take(HR * ((p.units_q + 31) / 32) * 4);
  p.bytes = align_up(cv.off + 256);
}

int plan_rel(const tx_attn_config* c, bool backward, bool run, int32_t n, const int64_t* off, AttnPlan& p) {
  TX_CHECK(check_attn_config(c, true));
  if (n < 0) return fail(TX_E_INVALID, "n_seq %d", n);
  TX_CHECK(check_offsets(off, n, "sequence"));
  p.q_base = off[0];
  p.rows_q = p.rows_k = off[n] - off[0];
  p.end_q = p.end_k = off[n];
  p.groups.reserve(n);
  for (int32_t i = 0; i < n; ++i) {
    const int64_t L = off[i + 1] - off[i];
    if (!L) continue;
    TrainGroup g{};
    g.q0 = g.k0 = (int32_t)off[i];
    g.nq = g.nk = (int32_t)L;
    p.groups.push_back(g);
    p.pairs += 0.5 * L * (L + 1);
  }
  finish_plan(*c, backward, true, run, p);
  return TX_OK;
}

int plan_event(const tx_attn_config* c, bool backward, bool run, int32_t n, const int64_t* ko, const int64_t* eo,
               const int64_t* qo, const int64_t* prefix, AttnPlan& p) {
  TX_CHECK(check_attn_config(c, false));
  if (n < 0) return fail(TX_E_INVALID, "n_users %d", n);
  TX_CHECK(check_offsets(ko, n, "key"));
  TX_CHECK(check_offsets(eo, n, "event"));
  if (eo[0] != 0) return fail(TX_E_INVALID, "event offsets start at %lld, not 0", (long long)eo[0]);
  const int64_t ne = eo[n];
  TX_CHECK(check_offsets(qo, ne, "query"));
  if (ne && !prefix) return fail(TX_E_INVALID, "prefix lengths are null");
  p.q_base = qo[0];
  p.rows_q = qo[ne] - qo[0];
  p.rows_k = ko[n] - ko[0];
  p.end_q = qo[ne];
  p.end_k = ko[n];
  p.groups.reserve(n);
  p.ev_row.resize(ne);
  p.ev_prefix.resize(ne);
  for (int32_t u = 0; u < n; ++u) {
    TrainGroup g{};
    g.q0 = (int32_t)qo[eo[u]];
    g.nq = (int32_t)(qo[eo[u + 1]] - qo[eo[u]]);
    g.k0 = (int32_t)ko[u];
    g.nk = (int32_t)(ko[u + 1] - ko[u]);
    g.e0 = (int32_t)eo[u];
    g.e1 = (int32_t)eo[u + 1];
    for (int64_t e = eo[u]; e < eo[u + 1]; ++e) {
      if (prefix[e] < 0 || prefix[e] > g.nk)
        return fail(TX_E_INVALID, "event %lld: prefix %lld outside 0 .. %d", (long long)e, (long long)prefix[e], g.nk);
      p.ev_row[e] = (int32_t)qo[e];
      p.ev_prefix[e] = (int32_t)prefix[e];
      p.pairs += (double)(qo[e + 1] - qo[e]) * prefix[e];
    }
    if (g.nq || (backward && g.nk)) p.groups.push_back(g);
  }
  finish_plan(*c, backward, false, run, p);
  return TX_OK;
}

struct AttnTensors {
  const tx_rows *q, *k, *v, *out, *d_out, *d_q, *d_k, *d_v;
  const void* rel;
  void* d_rel;
  float* lse;
  int64_t lse_stride;
};

int run_attn(const tx_attn_config& c, bool backward, bool rel, const AttnPlan& p, const AttnTensors& x, void* ws,
             size_t ws_bytes, hipStream_t st) {
  const int es = c.dtype == TX_BF16 ? 2 : 4, H = c.n_heads, G = c.n_kv_heads, dh = c.d_head, R = c.rel_pos_buckets;
  const bool bf = c.dtype == TX_BF16;
  TrainArgs a{};
  TX_CHECK(check_rows(x.q, "q", es, H, dh, p.rows_q, false, &a.q));
  TX_CHECK(check_rows(x.k, "k", es, G, dh, p.rows_k, false, &a.k));
  TX_CHECK(check_rows(x.v, "v", es, G, dh, p.rows_k, false, &a.v));
  TX_CHECK(check_rows(x.out, "out", es, H, dh, p.rows_q, !backward, &a.o));
  if (backward) {
    TX_CHECK(check_rows(x.d_out, "d_out", es, H, dh, p.rows_q, false, &a.dO));
    TX_CHECK(check_rows(x.d_q, "d_q", es, H, dh, p.rows_q, true, &a.dq));
    TX_CHECK(check_rows(x.d_k, "d_k", es, G, dh, p.rows_k, true, &a.dk));
    TX_CHECK(check_rows(x.d_v, "d_v", es, G, dh, p.rows_k, true, &a.dv));
  }
  if (rel && R > 0) {
    if (!x.rel || ((uintptr_t)x.rel % es)) return fail(TX_E_INVALID, "rel is null or misaligned");
    if (backward && (!x.d_rel || ((uintptr_t)x.d_rel % es))) return fail(TX_E_INVALID, "d_rel is null or misaligned");
  }
  if (p.rows_q > 0 && (!x.lse || ((uintptr_t)x.lse & 3))) return fail(TX_E_INVALID, "lse is null or misaligned");
  if (x.lse_stride < p.end_q)
    return fail(TX_E_INVALID, "lse stride %lld below %lld rows", (long long)x.lse_stride, (long long)p.end_q);
  if (std::max(p.units_q * H, p.units_k * G) > kMaxGrid)
    return fail(TX_E_UNSUPPORTED, "%lld blocks in one launch", (long long)std::max(p.units_q * H, p.units_k * G));
  if ((int64_t)H * R > 65535 * 256) return fail(TX_E_UNSUPPORTED, "%d heads of %d buckets", H, R);
  const bool drel = rel && backward && R > 0;
  if (p.rows_q == 0 && (!backward || p.rows_k == 0) && !drel) return TX_OK;
  TX_CHECK(check_ws(ws, ws_bytes, p.bytes));
  TX_CHECK(check_apart(a, p.rows_q, p.rows_k, backward));
  TX_CHECK(check_stream(st));

  char* const w = (char*)ws;
  const bool limits = !rel && p.tiles > 0, in_one = limits && p.meta.size() <= sizeof(MetaArg);
  int32_t* const row_lim = (int32_t*)(w + p.at.row_lim);
  TileLim* const tile_lim = (TileLim*)(w + p.at.tile_lim);
  if (in_one)
    TX_HIP(launch_train_put_limits(w, p.meta.data(), p.meta.size(), (int32_t)p.groups.size(), (int32_t)p.tiles, p.o_row,
                                   p.o_prefix, row_lim, (int32_t)p.q_base, tile_lim, st));
  else
    TX_HIP(put_all(w, p.meta, st));
  a.groups = (const TrainGroup*)w;
  a.n_groups = (int32_t)p.groups.size();
  a.H = H, a.G = G;
  a.lse = x.lse;
  a.lse_ld = x.lse_stride;
  a.stat_ld = p.rows_q;
  a.row_stat = (float*)(w + p.at.stat);
  a.rel = x.rel;
  a.R = R;
  a.row_lim = row_lim;
  a.tile_lim = tile_lim;
  a.q_base = (int32_t)p.q_base;
  a.scale = c.scale > 0.f ? c.scale : (float)(1.0 / std::sqrt((double)dh));
  a.scale_log2 = (float)(a.scale * 1.4426950408889634);
  a.partial = (float*)(w + p.at.partial);
  a.q_rows = p.q_rows, a.k_rows = p.k_rows;
  a.q_narrow = p.q_narrow, a.k_narrow = p.k_narrow;
  a.pack = p.pack;
  a.n_units = (int32_t)p.units_q, a.k_units = (int32_t)p.units_k;
  a.q_chunk = place_chunk(p.units_q, H >> p.pack);
  a.k_chunk = place_chunk(p.units_k, G);
  a.q_order = p.o_q ? (const uint32_t*)(w + p.o_q) : nullptr;
  a.k_order = p.o_k ? (const uint32_t*)(w + p.o_k) : nullptr;
  a.drel_part = (float*)(w + p.at.drel);
  if (limits && !in_one)
    TX_HIP(launch_train_limits(a.groups, a.n_groups, (int32_t)p.tiles, (const int32_t*)(w + p.o_row),
                               (const int32_t*)(w + p.o_prefix), row_lim, a.q_base, tile_lim, st));
  // algorithmic work: 2 d_h flops per pair and product, each tensor once
  const double prod = 2.0 * dh * H * p.pairs, qb = (double)es * dh * H * p.rows_q, kb = (double)es * dh * G * p.rows_k;
  const double stat = 4.0 * H * p.rows_q;
  if (!backward) {
    TX_LAUNCH(K_TRAIN_FWD, 2 * prod, 2 * qb + 2 * kb + stat, launch_train_fwd(bf, dh, rel, a, st));
    if (p.slots_q) TX_LAUNCH(K_TRAIN_FWD, 0, 0, launch_train_fwd_join(bf, dh, a, st));
    return TX_OK;
  }
  if (p.units_q) TX_LAUNCH(K_TRAIN_DQ, 3 * prod, 4 * qb + 2 * kb + 2 * stat, launch_train_dq(bf, dh, rel, a, st));
  if (p.slots_q) TX_LAUNCH(K_TRAIN_DQ, 0, 0, launch_train_dq_join(bf, dh, a, st));
  if (drel) TX_LAUNCH(K_TRAIN_DQ, 0, 0, launch_train_drel(bf, a, (float*)(w + p.at.drel2), x.d_rel, st));
  if (p.units_k)
    TX_LAUNCH(K_TRAIN_DKV, 4 * prod, 2 * qb + 4 * kb + 2 * stat,
              launch_train_dkv(bf, dh, rel, a, st));
  if (p.slots_k) TX_LAUNCH(K_TRAIN_DKV, 0, 0, launch_train_dkv_join(bf, dh, a, st));
  return TX_OK;
}

// ------------------------------------------------------------------ preference loss

int check_pref(const tx_preference_config* c, int32_t n, const int64_t* off) {
  if (!c) return fail(TX_E_INVALID, "config is null");
  if (c->dtype != TX_F32 && c->dtype != TX_BF16) return fail(TX_E_INVALID, "dtype %d unknown", c->dtype);
  if (c->n_actions < 1) return fail(TX_E_INVALID, "n_actions %d", c->n_actions);
  if (!std::isfinite(c->beta)) return fail(TX_E_INVALID, "beta is not finite");
  if (!(c->smoothing >= 0.f && c->smoothing <= 1.f)) return fail(TX_E_INVALID, "smoothing outside 0 .. 1");
  if (n < 0) return fail(TX_E_INVALID, "n_pairs %d", n);
  if (n > (1 << 24)) return fail(TX_E_UNSUPPORTED, "n_pairs %d above %d", n, 1 << 24);
  return check_offsets(off, 2 * (int64_t)n, "answer");
}

struct PrefPlan {
  size_t at_row = 0, bytes = 0;
  int64_t row0 = 0, rows = 0;
};

void plan_pref(int32_t n, const int64_t* off, PrefPlan& p) {
  p.row0 = off[0];
  p.rows = off[2 * (int64_t)n] - off[0];
  p.at_row = align_up((2 * (size_t)n + 1) * 4);
  p.bytes = align_up(p.at_row + p.rows * 8 + 256);  // forward: doubles, backward: floats
}

// The answers' row offsets (from the first) on the device: lengths of 16 bits as
// kernel arguments, summed up there, twice as many a launch as offsets would be;
// offsets where an answer is longer.
hipError_t put_answer_offsets(int32_t* dst, const int64_t* off, int64_t n, hipStream_t s) {
  for (int64_t i = 0; i <= n;) {
    PrefOffsets a;
    a.base = (int32_t)(off[i] - off[0]);
    int32_t m = 0;  // offsets i .. i + m: one more than lengths
    while (m < PrefOffsets::kLengths && i + m < n && off[i + m + 1] - off[i + m] <= 0xffff) {
      a.len[m] = (uint16_t)(off[i + m + 1] - off[i + m]);
      ++m;
    }
    a.n = m;
    const hipError_t e = launch_pref_offsets(dst + i, a, s);
    if (e != hipSuccess) return e;
    i += m + 1;
  }
  return hipSuccess;
}

int check_pref_tensors(const tx_preference_config* c, const PrefPlan& p, const void* logits, int64_t ld,
                       const int32_t* actions, const void* const* f32, const char* const* names, int n_f32) {
  const size_t es = c->dtype == TX_BF16 ? 2 : 4;
  if (ld < c->n_actions) return fail(TX_E_INVALID, "row stride %lld below n_actions %d", (long long)ld, c->n_actions);
  if (p.rows > 0 && ld > ((int64_t)1 << 60) / (p.row0 + p.rows))
    return fail(TX_E_INVALID, "row stride %lld", (long long)ld);
  if (p.rows && (!logits || (uintptr_t)logits % es)) return fail(TX_E_INVALID, "logits are null or misaligned");
  if (p.rows && (!actions || ((uintptr_t)actions & 3))) return fail(TX_E_INVALID, "actions are null or misaligned");
  for (int i = 0; i < n_f32; ++i)
    if (!f32[i] || ((uintptr_t)f32[i] & 3)) return fail(TX_E_INVALID, "%s is null or misaligned", names[i]);
  return TX_OK;
}

// No C++ exception leaves a C entry.
template <class F>
int guarded(F f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail(TX_E_NOMEM, "out of host memory");
  } catch (...) {
    return fail(TX_E_INVALID, "internal error");
  }
}

}  // namespace

extern "C" {

size_t tx_rel_attn_workspace_bytes(const tx_attn_config* cfg, int32_t backward, int32_t n, const int64_t* off) {
  AttnPlan p;
  return guarded([&] { return plan_rel(cfg, backward != 0, false, n, off, p); }) == TX_OK ? p.bytes : 0;
}

int tx_rel_attn_forward(const tx_attn_config* cfg, int32_t n, const int64_t* off, const tx_rows* q, const tx_rows* k,
                        const tx_rows* v, const void* rel, const tx_rows* out, float* lse, int64_t lse_stride, void* ws,
                        size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    AttnPlan p;
    TX_CHECK(plan_rel(cfg, false, true, n, off, p));
    const AttnTensors x{q, k, v, out, nullptr, nullptr, nullptr, nullptr, rel, nullptr, lse, lse_stride};
    return run_attn(*cfg, false, true, p, x, ws, ws_bytes, stream);
  });
}

int tx_rel_attn_backward(const tx_attn_config* cfg, int32_t n, const int64_t* off, const tx_rows* q, const tx_rows* k,
                         const tx_rows* v, const void* rel, const tx_rows* out, const float* lse, int64_t lse_stride,
                         const tx_rows* d_out, const tx_rows* d_q, const tx_rows* d_k, const tx_rows* d_v, void* d_rel,
                         void* ws, size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    AttnPlan p;
    TX_CHECK(plan_rel(cfg, true, true, n, off, p));
    const AttnTensors x{q, k, v, out, d_out, d_q, d_k, d_v, rel, d_rel, const_cast<float*>(lse), lse_stride};
    return run_attn(*cfg, true, true, p, x, ws, ws_bytes, stream);
  });
}

size_t tx_event_attn_workspace_bytes(const tx_attn_config* cfg, int32_t backward, int32_t n, const int64_t* ko,
                                     const int64_t* eo, const int64_t* qo, const int64_t* prefix) {
  AttnPlan p;
  return guarded([&] { return plan_event(cfg, backward != 0, false, n, ko, eo, qo, prefix, p); }) == TX_OK ? p.bytes : 0;
}

int tx_event_attn_forward(const tx_attn_config* cfg, int32_t n, const int64_t* ko, const int64_t* eo, const int64_t* qo,
                          const int64_t* prefix, const tx_rows* q, const tx_rows* k, const tx_rows* v,
                          const tx_rows* out, float* lse, int64_t lse_stride, void* ws, size_t ws_bytes,
                          hipStream_t stream) {
  return guarded([&] {
    AttnPlan p;
    TX_CHECK(plan_event(cfg, false, true, n, ko, eo, qo, prefix, p));
    const AttnTensors x{q, k, v, out, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, lse, lse_stride};
    return run_attn(*cfg, false, false, p, x, ws, ws_bytes, stream);
  });
}

int tx_event_attn_backward(const tx_attn_config* cfg, int32_t n, const int64_t* ko, const int64_t* eo,
                           const int64_t* qo, const int64_t* prefix, const tx_rows* q, const tx_rows* k, const tx_rows* v,
                           const tx_rows* out, const float* lse, int64_t lse_stride, const tx_rows* d_out,
                           const tx_rows* d_q, const tx_rows* d_k, const tx_rows* d_v, void* ws, size_t ws_bytes,
                           hipStream_t stream) {
  return guarded([&] {
    AttnPlan p;
    TX_CHECK(plan_event(cfg, true, true, n, ko, eo, qo, prefix, p));
    const AttnTensors x{q, k, v, out, d_out, d_q, d_k, d_v, nullptr, nullptr, const_cast<float*>(lse), lse_stride};
    return run_attn(*cfg, true, false, p, x, ws, ws_bytes, stream);
  });
}

size_t tx_preference_workspace_bytes(const tx_preference_config* cfg, int32_t n, const int64_t* off) {
  PrefPlan p;
  return guarded([&] {
           TX_CHECK(check_pref(cfg, n, off));
           plan_pref(n, off, p);
           return (int)TX_OK;
         }) == TX_OK ? p.bytes : 0;
}

int tx_preference_forward(const tx_preference_config* cfg, int32_t n, const int64_t* off, const void* logits,
                          int64_t row_stride, const int32_t* actions, const float* ref_logp, float* loss, float* logp,
                          float* row_lse, void* ws, size_t ws_bytes, hipStream_t st) {
  return guarded([&]() -> int {
    TX_CHECK(check_pref(cfg, n, off));
    if (n == 0) return TX_OK;
    PrefPlan p;
    plan_pref(n, off, p);
    const void* f32[] = {loss, logp, p.rows ? row_lse : loss};
    const char* names[] = {"loss", "logp", "row_lse"};
    TX_CHECK(check_pref_tensors(cfg, p, logits, row_stride, actions, f32, names, 3));
    if ((uintptr_t)ref_logp & 3) return fail(TX_E_INVALID, "ref_logp is misaligned");
    TX_CHECK(check_ws(ws, ws_bytes, p.bytes));
    TX_CHECK(check_stream(st));
    TX_HIP(put_answer_offsets((int32_t*)ws, off, 2 * (int64_t)n, st));
    double* const picked = (double*)((char*)ws + p.at_row);
    const bool bf = cfg->dtype == TX_BF16;
    const double nk = (double)p.rows * cfg->n_actions;
    if (p.rows)
      TX_LAUNCH(K_TRAIN_PREF, 3 * nk, nk * (bf ? 2 : 4) + 16.0 * p.rows,
                launch_pref_rows(bf, logits, row_stride, cfg->n_actions, actions, p.row0, p.rows, row_lse, picked, st));
    TX_LAUNCH(K_TRAIN_PREF, 0, 8.0 * p.rows,
              launch_pref_pairs(picked, (const int32_t*)ws, n, ref_logp, cfg->beta, cfg->smoothing, logp, loss, st));
    return TX_OK;
  });
}

int tx_preference_backward(const tx_preference_config* cfg, int32_t n, const int64_t* off, const void* logits,
                           int64_t row_stride, const int32_t* actions, const float* ref_logp, const float* logp,
                           const float* row_lse, const float* d_loss, void* d_logits, int64_t d_row_stride, void* ws,
                           size_t ws_bytes, hipStream_t st) {
  return guarded([&]() -> int {
    TX_CHECK(check_pref(cfg, n, off));
    if (n == 0) return TX_OK;
    PrefPlan p;
    plan_pref(n, off, p);
    if (p.rows == 0) return TX_OK;
    const void* f32[] = {logp, row_lse, d_loss};
    const char* names[] = {"logp", "row_lse", "d_loss"};
    TX_CHECK(check_pref_tensors(cfg, p, logits, row_stride, actions, f32, names, 3));
    if ((uintptr_t)ref_logp & 3) return fail(TX_E_INVALID, "ref_logp is misaligned");
    const bool bf = cfg->dtype == TX_BF16;
    if (!d_logits || (uintptr_t)d_logits % (bf ? 2 : 4)) return fail(TX_E_INVALID, "d_logits is null or misaligned");
    if (d_row_stride < cfg->n_actions || d_row_stride > ((int64_t)1 << 60) / (p.row0 + p.rows))
      return fail(TX_E_INVALID, "d_logits row stride %lld", (long long)d_row_stride);
    TX_CHECK(check_ws(ws, ws_bytes, p.bytes));
    if (d_logits == logits) return fail(TX_E_INVALID, "d_logits is written and begins where logits do");
    TX_CHECK(check_stream(st));
    TX_HIP(put_answer_offsets((int32_t*)ws, off, 2 * (int64_t)n, st));
    float* const coef = (float*)((char*)ws + p.at_row);
    const double nk = (double)p.rows * cfg->n_actions;
    TX_LAUNCH(K_TRAIN_PREF, 0, 4.0 * p.rows,
              launch_pref_coef((const int32_t*)ws, n, ref_logp, logp, d_loss, cfg->beta, cfg->smoothing, coef, st));
    TX_LAUNCH(K_TRAIN_PREF, 3 * nk, 2 * nk * (bf ? 2 : 4) + 12.0 * p.rows,
              launch_pref_grad(bf, logits, row_stride, cfg->n_actions, actions, p.row0, p.rows, row_lse, coef, d_logits,
                               d_row_stride, st));
    return TX_OK;
  });
}

}  // extern "C"
