// Plays the end of a call of the layer for a few tokens (csrc/ciera_tokens_end.hpp) through in many orders in which its blocks can get
// there, drawn from a fixed seed.  Each block has one tile of one group, and works on one stage of the next
// block's: two warps that take stages in turn and wait for that group, one that tells of the block's own tile by two additions, which
// nothing but a fence orders, and the rest, which tells that the block is done and ends the call.
//   tokens_end BLOCKS RULE ORDERS   RULE 0: the header's; 1, 2: what it must not be (the model has to see it)
//   tokens_end give_up
//   tokens_end wait MOST THERE GIVEN_UP
// prints how many orders there were, in how many a warp waited for a value that had been set back, and in how many a counter was not
// zero behind the call.
#include <stdio.h>
#include <stdlib.h>
#include <ucontext.h>

#include <functional>
#include <memory>
#include <vector>

#include "ciera_tokens_end.hpp"

static int blocks;
static std::vector<int> counters;                     // done, tickets, whole, each block's group
static std::vector<std::vector<std::pair<int, int>>> on_their_way;  // additions of each block that have not arrived yet
enum { kDone, kTickets, kWhole, kGroups };

// ---- threads of which one runs at a time; which one goes on is a choice, and all choices are gone through
struct Fiber {
    ucontext_t at;
    std::vector<char> stack = std::vector<char>(1 << 15);
    std::function<void()> body;
    std::function<bool()> ready;
    bool over = false;
};
static std::vector<std::unique_ptr<Fiber>> fibers;
static Fiber* running;
static ucontext_t scheduler;
static void pause_until(std::function<bool()> ready) {
    running->ready = ready;
    swapcontext(&running->at, &scheduler);
}
static void step() { pause_until([] { return true; }); }
static void start(int which) {
    fibers[which]->body();
    fibers[which]->over = true;
    swapcontext(&fibers[which]->at, &scheduler);
}
static void spawn(std::function<void()> body) {
    fibers.push_back(std::make_unique<Fiber>());
    Fiber& f = *fibers.back();
    f.body = body;
    f.ready = [] { return true; };
    getcontext(&f.at);
    f.at.uc_stack.ss_sp = f.stack.data();
    f.at.uc_stack.ss_size = f.stack.size();
    f.at.uc_link = &scheduler;
    makecontext(&f.at, (void (*)())start, 1, (int)fibers.size() - 1);
}

static void add(int block, int counter) { on_their_way[block].push_back({counter, 1}); }  // a relaxed addition
static void arrive(int block, size_t i) {
    const auto a = on_their_way[block][i];
    on_their_way[block].erase(on_their_way[block].begin() + (long)i);
    counters[a.first] += a.second;
}
static void fence(int block) {
    while (!on_their_way[block].empty()) arrive(block, 0);
}

struct Block {
    int rank;
    int* ended;  // warps of the block that have
    void join() { pause_until([this] { return *ended == 3; }); }
    bool all_done() {
        pause_until([] { return counters[kDone] >= blocks; });
        return true;
    }
    void ticket() {
        fence(rank);
        step();
        if (++counters[kTickets] == blocks) {
            step();
            for (int i = 0; i < kGroups; ++i) counters[i] = 0;
        }
    }
    void clear() { counters[kGroups + (rank + 2) % blocks] = 0; }  // (told of by one block, read by another)
    void sum() { step(); }
    void spoil() {}
};

// the bounded wait: prints whether it came true, after how many looks, and how often it gave up
static int waits(unsigned most, unsigned there, unsigned given_up) {
    unsigned looks = 0, told = 0;
    const bool ok = ciera::poll(most, [&] { return ++looks == there; }, [&] { return looks == given_up; }, [&] { ++told; });
    printf("%d %u %u\n", ok, looks, told);
    return 0;
}

// a block that gives up: prints what it is asked for
struct GivesUp {
    void join() { printf("join "); }
    bool all_done() { return false; }
    void spoil() { printf("spoil\n"); }
    void ticket() { printf("ticket "); }
    void clear() { printf("clear "); }
    void sum() { printf("sum "); }
};

int main(int argc, char** argv) {
    if (argc == 2) {
        GivesUp b;
        return ciera::end_call(b) ? 1 : 0;
    }
    if (argc == 5) return waits((unsigned)atoi(argv[2]), (unsigned)atoi(argv[3]), (unsigned)atoi(argv[4]));
    if (argc != 4) return 2;
    blocks = atoi(argv[1]);
    const int rule = atoi(argv[2]);
    const long most = atol(argv[3]);
    unsigned long long seed = 1;
    long orders = 0, stuck = 0, left = 0;
    while (orders < most) {
        counters.assign(kGroups + blocks, 0);
        on_their_way.assign(blocks, {});
        fibers.clear();
        std::vector<int> ended(blocks, 0), copied(blocks, 0);
        for (int r = 0; r < blocks; ++r) {
            spawn([r, rule, &ended] {
                int tiles = 0;
                ciera::tell([&] { return tiles++ == 0; }, [&] { add(r, kGroups + r); }, [&] { if (rule != 2) fence(r); }, [&] { add(r, kWhole); });
                ++ended[r];
            });
            for (unsigned warp = 0; warp < 2; ++warp)
                spawn([r, rule, warp, &ended, &copied] {
                    const bool part = ciera::takes_part(0, 1, warp, 2);
                    if (part || rule == 1) {
                        const int group = kGroups + (r + 1) % blocks;
                        step();
                        if (counters[kWhole] < blocks) pause_until([group] { return counters[group] >= 1; });
                    }
                    if (part) copied[r] = true;
                    ++ended[r];
                });
            spawn([r, &ended, &copied] {
                pause_until([r, &copied] { return (bool)copied[r]; });
                ++counters[kDone];
                Block b{r, &ended[r]};
                ciera::end_call(b);
            });
        }
        for (;;) {
            std::vector<std::function<void()>> can;
            for (auto& f : fibers)
                if (!f->over && f->ready()) {
                    Fiber* g = f.get();
                    can.push_back([g] {
                        running = g;
                        swapcontext(&scheduler, &g->at);
                    });
                }
            for (int b = 0; b < blocks; ++b)
                for (size_t i = 0; i < on_their_way[b].size(); ++i) can.push_back([b, i] { arrive(b, i); });
            if (can.empty()) break;
            seed = seed * 6364136223846793005ull + 1442695040888963407ull;
            can[(seed >> 33) % can.size()]();
        }
        ++orders;
        for (auto& f : fibers)
            if (!f->over) {
                ++stuck;
                break;
            }
        bool zero = true, all = true;
        for (auto& f : fibers) all &= f->over;
        for (int c : counters) zero &= c == 0;
        left += all && !zero;
    }
    printf("%ld %ld %ld\n", orders, stuck, left);
    return 0;
}
