// The bounded waits of a warp (csrc/wait_together.h) with its lanes as threads, which vote at barriers.  What a lane sees -- the phase over, the flag up --
// changes at a random moment of its own, as it may between two lanes of a warp that go apart.
#include <barrier>
#include <cstdint>
#include <random>
#include <thread>
#include <vector>

#include "wait_together.h"

namespace {
constexpr int kLanes = 32;
struct Warp {
    std::barrier<> sync{kLanes};
    bool x[kLanes];
    bool up = false;
};
struct Lane {
    Warp &w;
    int lane, over_from, up_from;  // tries from which on it sees the phase over, and the flag up
    mutable int tries = 0;
    bool there() const { return tries++ >= over_from; }
    bool given_up() const { return tries > up_from; }
    void give_up() const { if (lane == 0) w.up = true; }
    template <typename F>
    bool vote(bool y, F f) const {
        w.x[lane] = y;
        w.sync.arrive_and_wait();
        bool r = w.x[0];
        for (int i = 1; i < kLanes; ++i) r = f(r, w.x[i]);
        w.sync.arrive_and_wait();
        return r;
    }
    bool all(bool y) const { return vote(y, [](bool a, bool b) { return a && b; }); }
    bool any(bool y) const { return vote(y, [](bool a, bool b) { return a || b; }); }
};
// Every lane for itself.
bool wait_apart(const Lane &l, uint32_t tries) {
    for (uint32_t i = 0; i < tries; ++i) {
        if (l.there()) return true;
        if (l.given_up()) return false;
    }
    l.give_up();
    return false;
}
}  // namespace

// out: runs whose lanes went apart; answers that were wrong (a wait that ended well without the phase being over for all, or badly without
// a flag or the tries having run out)
extern "C" void run_waits(int together, int runs, int tries, unsigned seed, int32_t *out) {
    std::mt19937 rng(seed);
    out[0] = out[1] = 0;
    for (int run = 0; run < runs; ++run) {
        Warp w;
        const int most = 2 * tries, over = rng() % most, up = rng() % most;
        std::vector<Lane> lanes;
        for (int i = 0; i < kLanes; ++i) lanes.push_back({w, i, over + (int)(rng() % 2), up + (int)(rng() % 2)});
        bool r[kLanes];
        std::vector<std::thread> threads;
        for (int i = 0; i < kLanes; ++i)
            threads.emplace_back([&, i] { r[i] = together ? mate::wait_together(lanes[i], (uint32_t)tries) : wait_apart(lanes[i], (uint32_t)tries); });
        for (auto &t : threads) t.join();
        int last_over = 0, first_up = most + 1;
        bool same = true;
        for (int i = 0; i < kLanes; ++i) {
            same &= r[i] == r[0];
            last_over = std::max(last_over, lanes[i].over_from), first_up = std::min(first_up, lanes[i].up_from);
        }
        out[0] += !same;
        // (try number last_over is the first that all lanes pass; the flag is looked at behind try number first_up)
        const bool well = last_over < tries && last_over <= first_up;
        if (together) out[1] += r[0] != well || (w.up != (!r[0] && first_up >= tries));
    }
}
