// Walks every workgroup of attention over shared prefixes through its shares, as the kernel does, and checks that each share of the
// prefixes and of the sequences is taken exactly once, that no workgroup is without work, and that none takes two shares where as many
// workgroups as there are shares run at a time.  Reads calls from stdin, one a line:
//   n_layers h_kv rows n_prefix  P_1 members_1 .. P_n members_n  L_1 .. L_n_seq
// Prints one line per call: "ok <prefix shares> <own shares> <workgroups> <query-row tiles>" (of a layer) or "bad <what>".
#include <cstdio>
#include <string>
#include <vector>

#include "jq_shares.h"

using namespace jq;

struct Tab { std::vector<int32_t> cu_seq{0}; };
struct Call {  // what plan_shared reads of a plan
    int32_t n_layers, n_seq, h_kv, rows;
    Tab tab;
};

static std::string walk(const Call& p, const Call& pp, const std::vector<int32_t>& members, const SharedPlan& sp) {
    std::vector<std::vector<int>> prefix_seen((size_t)pp.n_seq), own_seen((size_t)p.n_seq);
    int64_t shares = 0;
    auto groups_of = [&](int i) { return ((members[i + 1] - members[i]) * p.rows + sp.prefix_tiles * kTileRows - 1) / (sp.prefix_tiles * kTileRows); };
    auto splits_of = [&](int i) { return (sp.cu_part[i + 1] - sp.cu_part[i]) / ((members[i + 1] - members[i]) * p.rows); };
    for (int i = 0; i < pp.n_seq; ++i) prefix_seen[i].assign((size_t)splits_of(i) * p.h_kv * groups_of(i), 0);
    for (int s = 0; s < p.n_seq; ++s) own_seen[s].assign((size_t)(sp.own_split[s + 1] - sp.own_split[s]) * p.h_kv * sp.own_groups, 0);
    for (auto& v : prefix_seen) shares += (int64_t)v.size();
    for (auto& v : own_seen) shares += (int64_t)v.size();
    if (sp.first_groups != groups_of(0) || sp.first_splits != splits_of(0)) return "the first prefix";
    const bool at_a_time = p.n_layers * shares <= kSharedChip;
    int s = 0;
    for (int bx = 0; bx < sp.grid; ++bx) {
        int n = 0;
        if (bx < sp.prefix_blocks) {
            while (s + 1 < pp.n_seq && sp.cu_split[s + 1] <= bx) ++s;
            const int groups = groups_of(s), units = splits_of(s) * p.h_kv;
            const UnitAt at = unit_at(bx - sp.cu_split[s], units, groups);
            if (at.unit < 0 || at.unit >= units || at.group < 0 || at.group >= groups) return "share outside its prefix";
            if (prefix_seen[s][(size_t)at.unit * groups + at.group]++) return "share of a prefix taken twice";
            ++n;
        }
        for (int u = first_own(bx, sp.prefix_blocks, sp.grid); u < sp.own_blocks; u += sp.grid) {
            if (u < 0) return "share in front of the sequences";
            const int units = sp.own_split[p.n_seq] * p.h_kv;
            const UnitAt at = unit_at(u, units, sp.own_groups);
            if (at.unit < 0 || at.unit >= units || at.group < 0 || at.group >= sp.own_groups) return "share outside the sequences";
            int q = 0;
            while (sp.own_split[q + 1] <= at.unit / p.h_kv) ++q;
            const int in = (at.unit / p.h_kv - sp.own_split[q]) * p.h_kv + at.unit % p.h_kv;
            if (own_seen[q][(size_t)in * sp.own_groups + at.group]++) return "share of a sequence taken twice";
            ++n;
        }
        if (n == 0) return "workgroup without work";
        if (n > 1 && at_a_time) return "two shares behind one another that were planned side by side";
    }
    for (auto& v : prefix_seen)
        for (int n : v)
            if (n != 1) return "share of a prefix left out";
    for (auto& v : own_seen)
        for (int n : v)
            if (n != 1) return "share of a sequence left out";
    return "";
}

int main() {
    Call p{}, pp{};
    while (std::scanf("%d %d %d %d", &p.n_layers, &p.h_kv, &p.rows, &pp.n_seq) == 4) {
        std::vector<int32_t> members{0};
        p.tab = pp.tab = Tab{};
        for (int i = 0; i < pp.n_seq; ++i) {
            int P, m;
            if (std::scanf("%d %d", &P, &m) != 2) return 1;
            pp.tab.cu_seq.push_back(pp.tab.cu_seq.back() + P);
            members.push_back(members.back() + m);
        }
        p.n_seq = members.back();
        for (int s = 0; s < p.n_seq; ++s) {
            int L;
            if (std::scanf("%d", &L) != 1) return 1;
            p.tab.cu_seq.push_back(p.tab.cu_seq.back() + L);
        }
        SharedPlan sp{};
        plan_shared(p, pp, members.data(), &sp);
        const std::string bad = !sp.fits ? "does not fit" : walk(p, pp, members, sp);
        if (bad.empty()) std::printf("ok %d %d %d %d\n", sp.prefix_blocks, sp.own_blocks, sp.grid, sp.prefix_tiles);
        else std::printf("bad %s\n", bad.c_str());
    }
    return 0;
}
