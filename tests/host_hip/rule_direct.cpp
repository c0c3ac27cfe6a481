// The pieces of a call under a rule that goes without a plan, worked out on the CPU as its workgroups do: whatever the call's arrays hold,
// each lies inside the call's rows and pages, no tile of it has keys of both sides of a gap, every row of a sequence is in one of
// them, and the keys that a row sees are in it once.
//
// A case on stdin is rule_plan.cpp's. One line out for each: ok and the numbers of pieces and keys, "plan" where the call has one, or what
// is wrong.
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
std::string fault(const char* what, long long i, long long v) {
  return std::string(what) + " (" + std::to_string(i) + ": " + std::to_string(v) + ")";
}

struct Case {
  bool prefix;
  int hq, dtype, max_len, window;
  spd_cache c{};
  std::vector<int> seqs, cu, plens, lens, first, open;
};

std::string look(Case& k, int rows, long long& pieces, long long& keys) {
  const int nseqs = (int)k.seqs.size(), ngroups = (int)k.plens.size(), hkv = k.c.n_kv_heads, G = k.hq / hkv, most = 16 * k.c.max_pages;
  const Request plain = request(k.c, k.hq, nseqs, rows, ngroups, k.max_len, k.prefix, true);  // of the workspace's call
  const Request q = request(k.c, k.hq, nseqs, rows, ngroups, k.max_len, k.prefix, true, k.window, !k.open.empty());
  if (plain.bytes < q.bytes) return fault("a workspace smaller than its call's", (long long)plain.bytes, (long long)q.bytes);
  if (!q.direct) return "plan";
  if (q.bytes != 0) return fault("a workspace that no launch reads", 0, (long long)q.bytes);
  RuledSeqArgs a{};
  static_cast<SeqArgs&>(a) = args_of(&k.c, 0, nullptr, 0, nullptr, 0, k.hq, k.seqs.data(), nseqs);
  a.rows = rows;
  a.rpt = q.rpt;
  a.cu = k.prefix ? nullptr : k.cu.data();
  a.rule.window = k.window;
  a.rule.first = k.first.empty() ? nullptr : k.first.data();
  a.rule.open = k.open.empty() ? nullptr : k.open.data();
  bool ascends = true;
  for (size_t i = 0; i + 1 < k.cu.size() && !k.prefix; i++) ascends = ascends && k.cu[i] <= k.cu[i + 1];
  std::vector<int> held(rows, 0);
  HostGroup wave;
  RuledItem lanes[64];
  bool is[64];
  for (int y = 0; y < q.jobs; y++) {
    if (!wave.run(64, [&] { is[threadIdx.x] = direct_item<RULE_KEYS>(a, y, lanes[threadIdx.x]); })) return "lanes wait for others that never come";
    const RuledItem it = lanes[0];
    for (int l = 1; l < 64; l++)
      if (is[l] != is[0] || (is[0] && (lanes[l].row0 != it.row0 || lanes[l].k0 != it.k0 || lanes[l].k1 != it.k1))) return fault("lanes that differ", y, l);
    if (!is[0]) continue;
    pieces++;
    if (it.nrows < 1 || it.row0 < 0 || it.row0 > rows - it.nrows || it.nrows * G > 16) return fault("a piece's rows", y, it.row0);
    if (it.table < 0 || it.table >= k.c.max_seqs) return fault("a piece's sequence", y, it.table);
    if (it.rec != -1 || !(it.mode & ITEM_FEW)) return fault("a piece's kind", y, it.mode);
    const int len = std::min(std::max(k.lens[it.table], 0), most);
    const Span s = span_of<RULE_KEYS>(it);
    if (it.k0 < 0 || it.k1 < it.k0 || s.a < 0 || s.b < s.a || s.b > len) return fault("a piece's keys", y, s.b);
    if (it.gap < 0 || it.gap % 16 || (it.gap && (it.gap_at - (it.k0 & ~15)) % kFewKeys)) return fault("a tile with keys of both sides", y, it.gap_at);
    keys += it.k1 - it.k0;
    for (int r = it.row0; r < it.row0 + it.nrows; r++) {
      held[r]++;
      const int pos = (it.mode & ITEM_FLAT ? len : it.lim0 + r - it.row0) - 1;
      const int i = k.prefix ? r : Batch::last(nseqs, r, [&](int x) { return k.cu[x]; });
      if (ascends && !k.prefix && pos != std::max<long long>((long long)len - (k.cu[i + 1] - r), -(1 << 30))) return fault("a row's key", r, pos);
      if (!ascends) continue;
      const int open = k.open.empty() ? 0 : std::min(std::max(k.open[i], 0), len);
      std::vector<char> times(len, 0);
      for (int c = it.k0; c < it.k1; c++) times[key_of<RULE_KEYS>(it, c)]++;
      for (int x = 0; x < len; x++) {
        long long lo = k.first.empty() ? 0 : k.first[r];
        if (k.window > 0) lo = std::max(lo, (long long)pos - k.window + 1);
        const bool sees = pos >= 0 && (x < open || (x >= lo && x <= pos));
        if (times[x] > 1 || (sees && times[x] != 1)) return fault("a key left out or taken twice", r, x);
      }
    }
  }
  for (int r = 0; r < rows && ascends; r++) {
    int want = 0;
    for (int i = 0; i < nseqs; i++) {
      const bool mine = k.prefix ? i == r : k.cu[i] <= r && r < k.cu[i + 1];
      want += mine && k.seqs[i] >= 0 && k.seqs[i] < k.c.max_seqs;
    }
    if (held[r] != want) return fault("outputs of a row", r, held[r]);
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
    long long pieces = 0, keys = 0;
    const std::string s = look(k, v[9], pieces, keys);
    if (s.empty())
      printf("ok %lld %lld\n", pieces, keys);
    else
      printf("%s\n", s.c_str());
    fflush(stdout);
  }
}
