"""What the kernels of attention over the 8-bit cache keep in the workspace, without a GPU.  The counters by which the last workgroup of
a group of rows is found (small calls): each group of a call has one of its own, and calls that a program lets overlap leave
nothing behind for later ones.  The table of runs by which partial results are merged: all that a call's own table names lies in the
workspace, and so does what is read by the table of another call."""
import os
import subprocess

import pytest

import paper_2508_19740_amd as sp
from test_cache_host import CSRC, HEAD, ROOT

COUNTERS = HEAD + r"""
#include <map>
#include <random>
#include <set>
#include <vector>
typedef std::vector<std::pair<uint32_t, uint32_t>> Call;      // a counter and a number of arrivals for each group of rows
static bool fail(const char* what) { printf("%s\n", what); return false; }

// The groups of a call over the whole cache, with lengths of its own or without.
static bool dense(const Plan& p, long n, int nq, const std::vector<int32_t>* lens, Call* call)
{
    cache::DensePlan d;
    if (cache::plan_dense(p, 256, n, nq, lens ? lens->data() : nullptr, &d) != SPOTLIGHT_OK || !d.joins) return true;
    const cache::DenseShares& s = d.shares;
    std::vector<long> runs(p.B, s.nsplit);
    if (lens) {
        auto units = [&](int b) { return static_cast<long>((std::min<long>(std::max((*lens)[b], 0), n) + 127) / 128); };
        long total = 0, chunk = s.units;
        for (int b = 0; b < p.B; ++b) total += units(b);
        if (s.most_runs) {
            const long spare = s.most_runs - p.B, safe = (total + spare - 1) / spare;
            chunk = std::max((total + s.most_runs - 1) / s.most_runs, 1L);
            for (int tries = 0; chunk < safe; ++tries) {
                long made = 0;
                for (int b = 0; b < p.B; ++b) made += std::max((units(b) + chunk - 1) / chunk, 1L);
                if (made <= s.most_runs) break;
                chunk = tries < 3 ? std::max(chunk + 1, chunk * made / s.most_runs) : safe;
            }
            chunk = std::min(std::max(chunk, 1L), static_cast<long>(s.units));
        }
        for (int b = 0; b < p.B; ++b) runs[b] = std::max((units(b) + chunk - 1) / chunk, 1L);
    }
    std::set<uint32_t> used;
    uint32_t first = 0;
    for (int b = 0; b < p.B; first += runs[b++]) {
        const uint32_t nsplit = runs[b];
        if (nsplit == 1) continue;
        if (nsplit > kJoinSplits) return fail("more parts than a counter is for");
        for (float inv : {1.0f / nsplit, nextafterf(1.0f / nsplit, 0.0f), nextafterf(1.0f / nsplit, 1.0f)})      // as the kernel divides
            if (static_cast<uint32_t>((first + 0.5f) * inv) != first / nsplit) return fail("quotient");
        for (int kv = 0; kv < p.Hkv; ++kv)
            for (uint32_t tile = 0; tile < s.tiles; ++tile) {
                const uint32_t at = (first / nsplit * p.Hkv + kv) * s.tiles + tile, c = cache::arrival_counter(at, nsplit);
                if (at >= kJoinGroups / nsplit || c >= kArrivedCounters || !used.insert(c).second) return fail("counter");
                call->push_back({c, nsplit});
            }
    }
    return true;
}

// The groups of a call over gathered rows.
static bool gathered(int heads, int nsplit, Call* call)
{
    if (!cache::joins_in_place(static_cast<int64_t>(heads) * nsplit, 1, nsplit)) return true;
    std::set<uint32_t> used;
    for (int h = 0; h < heads; ++h) {
        const uint32_t c = cache::arrival_counter(h, nsplit);
        if (c >= kArrivedCounters || !used.insert(c).second) return fail("counter");
        call->push_back({c, static_cast<uint32_t>(nsplit)});
    }
    return true;
}

int main(int argc, char** argv)
{
    const bool cleared = argc > 1;              // the mistake: the last workgroup clears the counter, and all sizes share it
    std::mt19937 rng(7);
    // no two (group, size) share a counter
    std::set<uint32_t> all;
    for (uint32_t nsplit = 2; nsplit <= kJoinSplits; ++nsplit)
        for (uint32_t at = 0; at < kJoinGroups / nsplit; ++at) {
            const uint32_t c = cache::arrival_counter(at, nsplit);
            if (c >= kArrivedCounters || !all.insert(c).second) return 1;
        }
    std::vector<Call> calls;
    for (int B : {1, 2, 3, 16, 60})
        for (int Hkv : {1, 2, 4, 8})
            for (int G : {1, 4})
                for (long n : {300L, 1000L, 4096L, 8192L}) {
                    const spotlight_config cfg = config(B, Hkv * G, Hkv, n, 1);
                    Plan p;
                    if (make_plan(&cfg, &p) != SPOTLIGHT_OK) return 2;
                    for (int nq : {1, 3, 9, 40})
                        for (int kind = 0; kind < 6; ++kind) {
                            std::vector<int32_t> lens(B);
                            for (int b = 0; b < B; ++b)
                                lens[b] = kind == 1 ? n : kind == 2 ? (b == B / 2 ? n : 1) : kind == 3 ? static_cast<int32_t>(n * (b + 1) / B) : static_cast<int32_t>(rng() % (n + 1));
                            Call c;
                            if (!dense(p, n, nq, kind ? &lens : nullptr, &c)) return 1;
                            if (!c.empty()) calls.push_back(c);
                        }
                }
    for (int heads : {1, 2, 3, 7, 32, 100})
        for (int nsplit = 2; nsplit < 70; ++nsplit) {
            Call c;
            if (!gathered(heads, nsplit, &c)) return 1;
            if (!c.empty()) calls.push_back(c);
        }
    if (calls.size() < 300) return 3;
    // calls one by one and overlapping, in any order of arrivals
    std::vector<uint32_t> counter(kArrivedCounters, 0);
    auto arrive = [&](uint32_t c, uint32_t nsplit) {
        uint32_t& v = counter[cleared ? c % kJoinGroups : c];
        const uint32_t before = v;
        v = cleared ? (before == nsplit - 1 ? 0 : before + 1) : before >= nsplit - 1 ? 0 : before + 1;      // an increment that wraps
        return before == nsplit - 1;
    };
    for (int round = 0; round < 3000; ++round) {
        std::vector<std::pair<uint32_t, uint32_t>> arrivals;
        const int together = round % 3 + 1;
        std::map<uint32_t, std::pair<uint32_t, uint32_t>> last;      // of a lone call: how many were told to be last, and arrivals left
        for (int i = 0; i < together; ++i)
            for (const auto& g : calls[rng() % calls.size()]) {
                for (uint32_t k = 0; k < g.second; ++k) arrivals.push_back(g);
                last[g.first] = {0, g.second};
            }
        std::shuffle(arrivals.begin(), arrivals.end(), rng);
        for (const auto& a : arrivals) {
            const bool is_last = arrive(a.first, a.second);
            if (together > 1) continue;
            auto& l = last[a.first];
            l.second -= 1;
            l.first += is_last;
            if (is_last != (l.second == 0)) { printf("round %d: told %d with %u to come\n", round, is_last, l.second); return 4; }
        }
        for (uint32_t v : counter)
            if (!cleared && v != 0) { printf("round %d leaves a count\n", round); return 5; }
    }
    return 0;
}
"""


TABLES = HEAD + r"""
#include <random>
#include <vector>
int main()
{
    std::mt19937 rng(3);
    long merged = 0, refused = 0;
    for (int B : {1, 3, 16, 100})
        for (int Hkv : {1, 4, 8})
            for (int G : {1, 4, 7})
                for (long n : {300L, 5000L, 131072L, 1L << 25}) {
                    const spotlight_config cfg = config(B, Hkv * G, Hkv, n, 1);
                    Plan p;
                    if (make_plan(&cfg, &p) != SPOTLIGHT_OK) return 2;
                    std::vector<cache::DensePlan> plans;
                    for (int nq : {1, 2, 17, 128, 300, 4096})
                        for (int ragged : {0, 1}) {
                            cache::DensePlan d;
                            int32_t one;
                            if (nq <= n && cache::plan_dense(p, 256, n, nq, ragged ? &one : nullptr, &d) == SPOTLIGHT_OK && d.splits) plans.push_back(d);
                        }
                    // sequences of lengths of their own: a run each and at least one to spare, by which the kernel divides
                    for (const auto& d : plans)
                        if (d.shares.most_runs && (d.shares.most_runs <= static_cast<uint32_t>(B) || d.shares.by_spare.d != d.shares.most_runs - B)) return 6;
                    for (const auto& mine : plans)
                        for (const auto& table : plans) {
                            cache::MergeRows r = {};
                            r.by_heads = cache::fast_div(Hkv);
                            r.tiles = mine.shares.tiles;
                            r.tile_rows = mine.shares.tile_rows;
                            r.room = p.dense_rows;
                            const uint32_t most = table.shares.most_runs ? table.shares.most_runs : table.shares.nsplit * B;
                            for (int k = 0; k < 20; ++k) {
                                const uint32_t number = k == 0 ? std::min(most, table.shares.nsplit) : 1 + rng() % std::min(most, table.shares.nsplit);
                                const uint2 run = {k == 1 ? 0 : k == 0 ? most - number : static_cast<uint32_t>(rng() % (most - number + 1)), number};
                                const cache::RowParts x = cache::parts_of(r, run, Hkv - 1, r.tiles - 1, r.tile_rows - 1);
                                const long last = x.at + (x.nsplit - 1) * x.step;
                                if (&mine == &table && x.nsplit != static_cast<int>(number)) return 3;      // its own: all of it
                                if (x.nsplit != 0 && (x.at < 0 || last >= p.dense_rows)) return 4;
                                (x.nsplit ? merged : refused) += 1;
                            }
                        }
                }
    return merged > 1000 && refused > 1000 ? 0 : 5;
}
"""


def _build(folder, source):
    src = folder / "host.cpp"
    exe = str(src)[:-4]
    src.write_text(source)
    lib = sp.lib._name
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-w", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
                    "-I", CSRC, str(src), "-o", exe, lib, f"-Wl,-rpath,{os.path.dirname(lib)}", "-L/opt/rocm/lib",
                    "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"], check=True)
    return exe


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return _build(tmp_path_factory.mktemp("counters"), COUNTERS)


def test_counters_recover(program):
    run = subprocess.run([program], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout


def test_the_model_sees_counters_that_do_not(program):
    """With one counter for groups of any size, cleared by the last, overlapping calls leave a later call without its last."""
    run = subprocess.run([program, "cleared"], capture_output=True, text=True)
    assert run.returncode == 4, run.stdout


def test_the_merge_stays_in_the_workspace(tmp_path):
    run = subprocess.run([_build(tmp_path, TABLES)], capture_output=True, text=True)
    assert run.returncode == 0, run.returncode
