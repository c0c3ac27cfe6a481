// The plan of the attention under a rule, run on the CPU: whatever a call's arrays hold, every piece it hands out lies inside the
// call's rows, pages and records, no tile of a piece has keys of both sides of a gap, and the keys that a row sees are covered once.
//
// A case on stdin: prefix(0/1) hq hkv dh dtype cache_dtype max_seqs max_pages nseqs rows ngroups max_len window firsts(0/1) opens(0/1),
// then seqs[nseqs], cu (nseqs + 1 or ngroups + 1 entries), prefix_lens[ngroups], lens[max_seqs], first[rows], open_lens[nseqs]. One line
// out for each: ok and the numbers of pieces, records and keys of pieces, or what is wrong.
#include <cstdio>
#include <cstdlib>

#include "hip/hip_runtime.h"
#define __builtin_amdgcn_rcpf HostName<float>()
#include "spd_ruleattn.hip"

namespace spd {
void set_call_error(const std::string&) {}
spd_status check_cache(const char*, const spd_cache*, bool) { return SPD_OK; }
spd_status check_workspace(const char*, const void*, size_t, size_t) { return SPD_OK; }
spd_status check_rows(const char*, const void*, int64_t, int, int, int) { return SPD_OK; }
spd_status check_launch(const char*) { return SPD_OK; }

namespace {
struct Case {
  bool prefix;
  int hq, dtype, max_len, window;
  spd_cache c{};
  std::vector<int> seqs, cu, plens, lens, first, open;
  SeqArgs a{};
};

std::string fault(const char* what, long long i, long long v) {
  return std::string(what) + " (" + std::to_string(i) + ": " + std::to_string(v) + ")";
}

std::string look(Case& k, long long& pieces, long long& used, long long& keys) {
  const int rows = k.a.rows, G = k.a.G, hkv = k.c.n_kv_heads;
  const Request q = request(k.c, k.hq, k.a.nseqs, rows, k.a.ngroups, k.max_len, k.prefix, true);
  if (q.direct) return "no plan";
  k.a.rpt = q.rpt;
  std::vector<char> ws(q.at_ml + 256, (char)0x7e);
  RuledPlanArgs p{};
  static_cast<PlanArgs&>(p) = plan_args(k.a, k.dtype, q, ws.data());
  p.rule.window = k.window;
  p.rule.first = k.first.empty() ? nullptr : k.first.data();
  p.rule.open = k.open.empty() ? nullptr : k.open.data();
  HostGroup group;
  const bool small = p.jobs <= kSmallPlanWG;
  const bool ends = group.run(small ? kSmallPlanWG : kPlanWG, [&] {
    if (k.prefix)
      small ? k_plan_attention<true, kSmallPlanWG, RULE_KEYS>(p) : k_plan_attention<true, kPlanWG, RULE_KEYS>(p);
    else
      small ? k_plan_attention<false, kSmallPlanWG, RULE_KEYS>(p) : k_plan_attention<false, kPlanWG, RULE_KEYS>(p);
  });
  if (!ends) return "threads wait for others that never come";
  for (size_t i = q.at_ml; i < ws.size(); i++)
    if (ws[i] != 0x7e) return fault("written behind the lists", (long long)i, ws[i]);
  const int n = p.count[0], units = q.merge ? p.count[1] : 0;
  const RuledItem* items = (const RuledItem*)p.items;
  const RuledMerge* merges = (const RuledMerge*)p.merges;
  pieces = n;
  if (n < 0 || (size_t)n > q.items) return fault("more pieces than places", (long long)q.items, n);
  if (units < 0 || (size_t)units > q.units) return fault("more units than places", (long long)q.units, units);
  std::vector<int> writer(q.records, -1);
  std::vector<std::vector<int>> held((size_t)rows * G);  // the pieces of a row's query, of one KV head
  for (int i = 0; i < n; i++) {
    const RuledItem& it = items[i];
    if (it.nrows < 1 || it.row0 < 0 || it.nrows > rows || it.row0 > rows - it.nrows) return fault("a piece's rows", i, it.row0);
    if (it.table < 0 || it.table >= k.c.max_seqs) return fault("a piece's sequence", i, it.table);
    const Span s = span_of<RULE_KEYS>(it);
    if (it.k0 < 0 || it.k1 < it.k0 || s.a < 0 || s.b < s.a || s.b > 16 * k.c.max_pages) return fault("a piece's keys", i, s.b);
    if (it.gap < 0 || it.gap % 16 || (it.gap && (it.gap_at - (it.k0 & ~15)) % (it.mode & ITEM_FEW ? 32 : 64))) return fault("a tile with keys of both sides", i, it.gap_at);
    const int len = std::min(std::max(k.lens[it.table], 0), 16 * k.c.max_pages);
    if (s.b > len) return fault("keys behind the sequence's", i, s.b);
    keys += it.k1 - it.k0;
    const int nq = it.nrows * G;
    if (nq > 128 || ((it.mode & ITEM_FEW) && nq > 16) || ((it.mode & ITEM_PAIR) && nq > 32)) return fault("a piece's queries", i, nq);
    if (it.rec < -1 || (it.rec >= 0 && (size_t)it.rec + (size_t)hkv * nq > q.records)) return fault("a piece's records", i, it.rec);
    for (int j = 0; j < nq; j++) {
      if (it.rec < 0) held[(size_t)it.row0 * G + j].push_back(i);
      for (int g = 0; g < hkv && it.rec >= 0; g++) {
        int& w = writer[(size_t)it.rec + (size_t)g * nq + j];
        if (w >= 0) return fault("a record written twice", i, w);
        w = i;
        used++;
      }
    }
  }
  std::vector<int> merged((size_t)rows * G, 0);
  for (int u = 0; u < units; u++) {
    const Unit un = p.units[u];
    if (un.merge < 0 || (size_t)un.merge >= q.merges) return fault("a unit's merge", u, un.merge);
    const RuledMerge& m = merges[un.merge];
    if (m.row0 < 0 || m.nrows < 1 || m.row0 > rows - m.nrows || un.query < 0) return fault("a merge's rows", u, m.row0);
    for (int j = un.query; j < std::min(un.query + q.qpu, m.nrows * G); j++) {
      merged[(size_t)m.row0 * G + j]++;
      for (int g = 0; g < hkv; g++)
        for (int x = 0; x < 2; x++)
          for (int piece = 0; piece < m.pieces[x]; piece++) {
            const size_t at = (size_t)m.rec[x] + (size_t)(piece * hkv + g) * m.queries[x] + m.first[x] + j;
            if (m.rec[x] < 0 || at >= q.records || writer[at] < 0) return fault("a record read that no piece wrote", u, (long long)at);
            const RuledItem& it = items[writer[at]];
            const int nq = it.nrows * G;
            if ((int)((at - it.rec) % nq) + it.row0 * G != m.row0 * G + j || (int)((at - it.rec) / nq) != g) return fault("another query's record", u, (long long)at);
            if (g == 0) held[(size_t)m.row0 * G + j].push_back(writer[at]);
          }
    }
  }
  for (int r = 0; r < rows; r++) {
    int seq = -1, len = 0, pos = -1, open = 0;
    if (k.prefix) {
      seq = k.seqs[r];
      if (seq < 0 || seq >= k.c.max_seqs) seq = -1;
      if (seq >= 0) len = std::min(std::max(k.lens[seq], 0), 16 * k.c.max_pages);
      pos = len - 1;
      if (!k.open.empty()) open = k.open[r];
    } else {
      for (int i = 0; i < k.a.nseqs; i++)
        if (k.cu[i] >= 0 && k.cu[i] <= r && r < k.cu[i + 1] && k.seqs[i] >= 0 && k.seqs[i] < k.c.max_seqs) {
          seq = k.seqs[i];
          len = std::min(std::max(k.lens[seq], 0), 16 * k.c.max_pages);
          pos = len - (k.cu[i + 1] - r);
          if (!k.open.empty()) open = k.open[i];
        }
    }
    bool ascends = true;
    for (size_t i = 0; i + 1 < k.cu.size(); i++) ascends = ascends && k.cu[i] <= k.cu[i + 1];
    if (!k.prefix && !ascends) continue;  // whose rows these are is not said: in bounds is all
    open = std::min(std::max(open, 0), len);
    for (int j = 0; j < G; j++) {
      const std::vector<int>& v = held[(size_t)r * G + j];
      const int ends = merged[(size_t)r * G + j];
      int writes = ends;
      for (int i : v) writes += items[i].rec < 0;
      if (writes != (seq >= 0)) return fault("outputs of a row", r, writes);
      std::vector<char> times(len, 0);
      for (int i : v)
        for (int c = items[i].k0; c < items[i].k1; c++) {
          const int x = key_of<RULE_KEYS>(items[i], c);
          if (x < len) times[x]++;  // of a shared piece, beyond a shorter row
        }
      for (int x = 0; x < len; x++) {
        long long lo = k.first.empty() ? 0 : k.first[r];
        if (k.window > 0) lo = std::max(lo, (long long)pos - k.window + 1);
        const bool sees = pos >= 0 && (x < open || (x >= lo && x <= pos));
        if (sees && times[x] != 1) return fault("a key left out or taken twice", r, x);
        if (times[x] > 1) return fault("a key in two pieces", r, x);
      }
    }
  }
  return "";
}
}  // namespace
}  // namespace spd

int main() {
  using namespace spd;
  int v[15];
  auto read = [](std::vector<int>& a, int n) {
    a.resize(n);
    for (int& x : a)
      if (scanf("%d", &x) != 1) exit(2);
  };
  for (;;) {
    for (int& x : v)
      if (scanf("%d", &x) != 1) return &x == v ? 0 : 2;
    Case k;
    k.prefix = v[0] != 0;
    k.hq = v[1];
    k.c.n_layers = 1;
    k.c.num_pages = 1;
    k.c.n_kv_heads = v[2];
    k.c.head_dim = v[3];
    k.dtype = v[4];
    k.c.dtype = v[5];
    k.c.max_seqs = v[6];
    k.c.max_pages = v[7];
    k.max_len = v[11];
    k.window = v[12];
    read(k.seqs, v[8]);
    read(k.cu, (k.prefix ? v[10] : v[8]) + 1);
    read(k.plens, v[10]);
    read(k.lens, v[6]);
    if (v[13]) read(k.first, v[9]);
    if (v[14]) read(k.open, v[8]);
    k.c.lens = k.lens.data();
    k.a = args_of(&k.c, 0, nullptr, 0, nullptr, 0, k.hq, k.seqs.data(), v[8]);
    k.a.cu = k.prefix && v[10] == 0 ? nullptr : k.cu.data();
    k.a.prefix = k.plens.data();
    k.a.rows = v[9];
    k.a.ngroups = v[10];
    long long pieces = 0, used = 0, keys = 0;
    const std::string s = look(k, pieces, used, keys);
    if (s.empty())
      printf("ok %lld %lld %lld\n", pieces, used, keys);
    else
      printf("%s\n", s.c_str());
    fflush(stdout);
  }
}
