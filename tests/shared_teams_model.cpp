// The two softmax teams and the two warps that issue products in the attention that reads shared tokens once (csrc/mate_decode_shared.cu), as roles that take their
// steps in a random order.  A barrier is waited for by the parity of a phase, as on the GPU; a product is done some time after it has been issued, those of one warp
// in their order.  What is looked for: waits that pass for another phase than the one that they are for, memory that somebody else still uses, runs
// that stand still.
#include <cstdint>
#include <deque>
#include <functional>
#include <random>
#include <vector>

namespace {
struct Barrier {
    int count, arrived = 0, done = 0;  // phases
    void arrive() {
        if (++arrived == count) arrived = 0, ++done;
    }
    bool passes(int phase) const { return (done & 1) != (phase & 1); }
};
struct Step {
    std::function<bool()> ready;  // null: at once
    std::function<void()> take;
};
}  // namespace

// variant: 0 as built; 1: a team does not wait until the other one has read O and the sums; 2: S goes by the place of the tile before the last without its P V;
// 3: both teams wait for the last P V of a part, of which one knows nothing about the phase in front.
// out: wrong waits, memory in use, runs that stood still
extern "C" void run_teams(int variant, int runs, int most, unsigned seed, int32_t *out) {
    std::mt19937 rng(seed);
    out[0] = out[1] = out[2] = 0;
    for (int run = 0; run < runs; ++run) {
        Barrier s_full[2] = {{1}, {1}}, p_full[2] = {{1}, {1}}, pv_done[2] = {{1}, {1}}, based[2] = {{1}, {1}}, pair{2};
        std::vector<int> parts(1 + rng() % 6);  // tiles of each
        for (int &n : parts) n = rng() % (most + 1);
        // what is where
        int s_of[2] = {-1, -1}, p_of[2] = {-1, -1}, pv_issued = -1, pv_over = -1, base_of[2] = {-1, -1};  // numbers of tiles
        int part_of_o = -1, reading_o = 0, stats_part[2] = {-1, -1};
        auto wait = [&](Barrier &b, int phase) {
            return Step{[&b, phase] { return b.passes(phase); }, [&b, phase, out] { out[0] += b.done <= phase; }};
        };
        auto act = [&](std::function<void()> f) { return Step{nullptr, f}; };
        auto check = [&](bool fine) { out[1] += !fine; };
        std::deque<Step> role[4];
        std::deque<std::function<void()>> flying[2];  // products of each issuing warp
        int pairs = 0, first = 0;
        for (size_t part = 0; part < parts.size(); first += parts[part], ++part) {
            const int last = first + parts[part] - 1, pa = (int)part;
            for (int c = first; c <= last; ++c) {
                const int team = c & 1, half = c >> 1;
                auto &t = role[team];
                t.push_back(wait(s_full[team], half));
                if (c == first)
                    t.push_back(act([&, pa, c] {
                        check(pv_issued == pv_over && reading_o == 0 && part_of_o == pa - 1);  // O is made 0
                        part_of_o = pa;
                    }));
                t.push_back(act([&, team, c] {
                    check(s_of[team] == c);
                    p_of[team] = c;
                }));
                if (c > first) {
                    t.push_back(wait(based[team ^ 1], (c - 1) >> 1));
                    t.push_back(act([&, team, c] { check(base_of[team ^ 1] == c - 1); }));
                }
                t.push_back(act([&, team, c] {
                    check(base_of[team] < c);
                    base_of[team] = c;
                    based[team].arrive();
                }));
                if (c > first && rng() % 3 == 0) {  // O is scaled, or added to
                    t.push_back(wait(pv_done[(c - 1) & 1], (c - 1) >> 1));
                    t.push_back(act([&, c] { check(pv_over == c - 1 && pv_issued == c - 1 && reading_o == 0); }));
                }
                t.push_back(act([&, team] { p_full[team].arrive(); }));
                // products
                if (c >= 2 && variant != 2) role[2].push_back(wait(pv_done[team], half - 1));
                role[2].push_back(act([&, team, c] {
                    flying[0].push_back([&, team, c] {
                        check(c < 2 || pv_over >= c - 2);
                        s_of[team] = c;
                        s_full[team].arrive();
                    });
                }));
                role[3].push_back(wait(p_full[team], half));
                role[3].push_back(act([&, team, c] {
                    check(p_of[team] == c && reading_o == 0);
                    pv_issued = c;
                    flying[1].push_back([&, team, c] {
                        check(p_of[team] == c && s_of[team] == c);
                        pv_over = c;
                        pv_done[team].arrive();
                    });
                }));
            }
            for (int team = 0; team < 2; ++team) {  // the end of a part
                auto &t = role[team];
                if (last >= first && ((last & 1) == team || variant == 3)) t.push_back(wait(pv_done[last & 1], last >> 1));
                t.push_back(act([&, team, pa] {
                    check(stats_part[team] == pa - 1);
                    stats_part[team] = pa;
                    pair.arrive();
                }));
                t.push_back(wait(pair, pairs));
                t.push_back(act([&, last, pa] {
                    check(stats_part[0] == pa && stats_part[1] == pa && pv_over == pv_issued && (last < 0 || pv_over >= last));
                    ++reading_o;
                }));
                t.push_back(act([&, pa, team] {
                    check(stats_part[0] == pa && stats_part[1] == pa);
                    --reading_o;
                    if (part_of_o < pa) part_of_o = pa;  // (a part without tiles)
                    pair.arrive();
                }));
                if (variant != 1) t.push_back(wait(pair, pairs + 1));
            }
            pairs += 2;
        }
        for (;;) {
            std::vector<int> can;
            bool left = false;
            for (int i = 0; i < 4; ++i)
                if (!role[i].empty()) {
                    left = true;
                    if (!role[i].front().ready || role[i].front().ready()) can.push_back(i);
                }
            for (int i = 0; i < 2; ++i)
                if (!flying[i].empty()) left = true, can.push_back(4 + i);
            if (can.empty()) {
                out[2] += left;
                break;
            }
            const int i = can[rng() % can.size()];
            if (i < 4) {
                const Step step = role[i].front();
                role[i].pop_front();
                step.take();
            } else {
                const auto f = flying[i - 4].front();
                flying[i - 4].pop_front();
                f();
            }
        }
    }
}
