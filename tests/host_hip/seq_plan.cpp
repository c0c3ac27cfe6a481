// The plan of the attention over a cache of several sequences, run on the CPU: whatever a call's arrays hold, every piece it hands
// out lies inside the call's rows, pages and records, and every row's keys are covered once.
//
// A case on stdin: prefix(0/1) hq hkv dh dtype cache_dtype max_seqs max_pages nseqs rows ngroups max_len, then seqs[nseqs], cu (nseqs + 1
// or ngroups + 1 entries), prefix_lens[ngroups], lens[max_seqs]. One line out for each: ok and the numbers of pieces and records, or
// what is wrong.
#include <cstdio>
#include <cstdlib>

#include "spd_seqattn.hip"

namespace spd {
void set_call_error(const std::string&) {}
spd_status check_cache(const char*, const spd_cache*, bool) { return SPD_OK; }
spd_status check_workspace(const char*, const void*, size_t, size_t) { return SPD_OK; }
spd_status check_rows(const char*, const void*, int64_t, int, int, int) { return SPD_OK; }
spd_status check_launch(const char*) { return SPD_OK; }

namespace {
struct Case {
  bool prefix;
  int hq, dtype, max_len;
  spd_cache c{};
  std::vector<int> seqs, cu, plens, lens;
  SeqArgs a{};
};

std::string fault(const char* what, long long i, long long v) {
  return std::string(what) + " (" + std::to_string(i) + ": " + std::to_string(v) + ")";
}

// "" or what is wrong; pieces, records used
std::string look(Case& k, long long& pieces, long long& used) {
  const int rows = k.a.rows, G = k.a.G, hkv = k.c.n_kv_heads;
  const Request q = request(k.c, k.hq, k.a.nseqs, rows, k.a.ngroups, k.max_len, k.prefix);
  if (q.direct) return "no plan";
  k.a.rpt = q.rpt;
  std::vector<char> ws(q.at_ml + 256, (char)0x7e);  // words that no plan means
  const PlanArgs p = plan_args(k.a, k.dtype, q, ws.data());
  HostGroup group;
  const bool small = p.jobs <= kSmallPlanWG;
  const bool ends = group.run(small ? kSmallPlanWG : kPlanWG, [&] {
    if (k.prefix)
      small ? k_plan_attention<true, kSmallPlanWG>(p) : k_plan_attention<true, kPlanWG>(p);
    else
      small ? k_plan_attention<false, kSmallPlanWG>(p) : k_plan_attention<false, kPlanWG>(p);
  });
  if (!ends) return "threads wait for others that never come";
  for (size_t i = q.at_ml; i < ws.size(); i++)
    if (ws[i] != 0x7e) return fault("written behind the lists", (long long)i, ws[i]);
  const int n = p.count[0], units = q.merge ? p.count[1] : 0;
  pieces = n;
  if (n < 0 || (size_t)n > q.items) return fault("more pieces than places", (long long)q.items, n);
  if (units < 0 || (size_t)units > q.units) return fault("more units than places", (long long)q.units, units);
  std::vector<int> writer(q.records, -1);
  struct Run {
    int a, b;
  };
  std::vector<std::vector<Run>> seen((size_t)rows * G);  // the keys of a row's query, for the heads of one KV head
  auto limit = [&](int r, const Item& it) {
    if (!(it.mode & ITEM_FLAT)) return it.lim0 + r - it.row0;
    const int s = k.seqs[r];
    return s >= 0 && s < k.c.max_seqs ? std::min(std::max(k.lens[s], 0), 16 * k.c.max_pages) : 0;
  };
  for (int i = 0; i < n; i++) {
    const Item& it = p.items[i];
    if (it.nrows < 1 || it.row0 < 0 || it.nrows > rows || it.row0 > rows - it.nrows) return fault("a piece's rows", i, it.row0);
    if (it.table < 0 || it.table >= k.c.max_seqs) return fault("a piece's sequence", i, it.table);
    if (it.k0 < 0 || it.k1 < it.k0 || it.k1 > 16 * k.c.max_pages) return fault("a piece's keys", i, it.k1);
    const int nq = it.nrows * G;
    if (nq > 128 || ((it.mode & ITEM_FEW) && nq > 16) || ((it.mode & ITEM_PAIR) && nq > 32)) return fault("a piece's queries", i, nq);
    if (it.rec < -1 || (it.rec >= 0 && (size_t)it.rec + (size_t)hkv * nq > q.records)) return fault("a piece's records", i, it.rec);
    for (int j = 0; j < nq; j++) {
      if (it.rec < 0) {
        seen[(size_t)it.row0 * G + j].push_back({it.k0, std::min(limit(it.row0 + j / G, it), it.k1)});
        if (it.k0 != 0) return fault("an output of a part of the keys", i, it.k0);
      }
      for (int g = 0; g < hkv && it.rec >= 0; g++) {
        int& w = writer[(size_t)it.rec + (size_t)g * nq + j];
        if (w >= 0) return fault("a record written twice", i, w);
        w = i;
        used++;
      }
    }
  }
  for (int u = 0; u < units; u++) {
    const Unit un = p.units[u];
    if (un.merge < 0 || (size_t)un.merge >= q.merges) return fault("a unit's merge", u, un.merge);
    const Merge& m = p.merges[un.merge];
    if (m.row0 < 0 || m.nrows < 1 || m.row0 > rows - m.nrows || un.query < 0) return fault("a merge's rows", u, m.row0);
    for (int j = un.query; j < std::min(un.query + q.qpu, m.nrows * G); j++)
      for (int g = 0; g < hkv; g++)
        for (int x = 0; x < 2; x++)
          for (int piece = 0; piece < m.pieces[x]; piece++) {
            const long long at = (long long)m.rec[x] + (long long)(piece * hkv + g) * m.queries[x] + m.first[x] + j;
            if (at < 0 || at >= (long long)q.records || writer[at] < 0) return fault("a merge reads what no piece writes", u, at);
            const Item& it = p.items[writer[at]];
            if ((at - it.rec) / (it.nrows * G) != g || it.row0 * G + (at - it.rec) % (it.nrows * G) != (long long)m.row0 * G + j)
              return fault("a merge reads another query's record", u, at);
            if (g == 0) seen[(size_t)m.row0 * G + j].push_back({it.k0, std::min(limit(it.row0 + (int)((at - it.rec) % (it.nrows * G)) / G, it), it.k1)});
          }
  }
  for (int r = 0; r < rows; r++) {
    int lim = 0;
    bool any = false;
    if (k.prefix) {
      const int s = k.seqs[r];
      any = s >= 0 && s < k.c.max_seqs;
      if (any) lim = std::min(std::max(k.lens[s], 0), 16 * k.c.max_pages);
    } else {
      for (int i = 0; i < k.a.nseqs; i++)
        if (k.cu[i] >= 0 && k.cu[i] <= r && r < k.cu[i + 1] && k.seqs[i] >= 0 && k.seqs[i] < k.c.max_seqs) {
          any = true;
          lim = std::min(std::max(k.lens[k.seqs[i]], 0), 16 * k.c.max_pages) - (k.cu[i + 1] - r) + 1;
        }
    }
    bool ascends = true;
    for (size_t i = 0; i + 1 < k.cu.size(); i++) ascends = ascends && k.cu[i] <= k.cu[i + 1];
    if (!k.prefix && !ascends) continue;  // whose rows these are is not said: in bounds is all
    for (int j = 0; j < G; j++) {
      std::vector<Run>& v = seen[(size_t)r * G + j];
      if (any == v.empty()) return fault(any ? "a row that no piece has" : "a row of no sequence", r, (long long)v.size());
      std::sort(v.begin(), v.end(), [](Run x, Run y) { return x.a != y.a ? x.a < y.a : x.b < y.b; });
      int at = 0;
      for (const Run& x : v) {
        if (x.b <= x.a) continue;  // none of its keys
        if (x.a != at) return fault("a key left out or taken twice", r, x.a);
        at = x.b;
      }
      if (at != std::max(lim, 0)) return fault("a row's last key", r, at);
    }
  }
  return "";
}
}  // namespace
}  // namespace spd

int main() {
  using namespace spd;
  int v[12];
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
    read(k.seqs, v[8]);
    read(k.cu, (k.prefix ? v[10] : v[8]) + 1);
    read(k.plens, v[10]);
    read(k.lens, v[6]);
    k.c.lens = k.lens.data();
    k.a = args_of(&k.c, 0, nullptr, 0, nullptr, 0, k.hq, k.seqs.data(), v[8]);
    k.a.cu = k.prefix && v[10] == 0 ? nullptr : k.cu.data();
    k.a.prefix = k.plens.data();
    k.a.rows = v[9];
    k.a.ngroups = v[10];
    long long pieces = 0, used = 0;
    const std::string s = look(k, pieces, used);
    if (s.empty())
      printf("ok %lld %lld\n", pieces, used);
    else
      printf("%s\n", s.c_str());
    fflush(stdout);
  }
}
