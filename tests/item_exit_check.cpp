// goes_on (attn_position.cuh): warps that meet in named barriers while they work on an item leave together, also where a wait that was given up
// elsewhere raises the flag between their looks at it.  Two threads stand for two warps; the first one's look is followed by the flag, then
// comes the second one's.
#include "device_on_cpu.h"

#include <atomic>

static std::barrier<> g_meet(2);
static std::atomic<int> g_said[2];

static bool group_any(int who, bool x)
{
    g_said[who] = x;
    g_meet.arrive_and_wait();
    const bool r = g_said[0] || g_said[1];
    g_meet.arrive_and_wait();
    return r;
}

// What the two warps decide; together: they share one look.
static void decide(bool together, bool had, int32_t n, bool raise, bool (&went)[2])
{
    volatile uint32_t flag = 0;
    std::atomic<bool> first_looked{false};
    std::thread first([&] {
        went[0] = gt::position::goes_on(had, n, &flag, [&](bool x) {
            if (raise) flag = 1;
            first_looked = true;
            return together ? group_any(0, x) : x;
        });
    });
    std::thread second([&] {
        while (!first_looked) std::this_thread::yield();
        went[1] = gt::position::goes_on(true, n, &flag, [&](bool x) { return together ? group_any(1, x) : x; });
    });
    first.join();
    second.join();
}

int main()
{
    int failed = 0;
    auto expect = [&](const char* what, const bool (&went)[2], bool a, bool b) {
        if (went[0] == a && went[1] == b) return;
        printf("%s: the first warp %s, the second %s\n", what, went[0] ? "goes on" : "leaves", went[1] ? "goes on" : "leaves");
        ++failed;
    };
    bool went[2];
    decide(true, true, 100, false, went);
    expect("nothing given up", went, true, true);
    decide(true, true, 0, false, went);
    expect("no more items", went, false, false);
    decide(true, true, 100, true, went);
    expect("the flag between two looks", went, false, false);
    decide(true, false, 100, false, went);
    expect("a wait of the first one's own", went, false, false);
    decide(false, true, 100, true, went);
    expect("each on its own (the planted mistake)", went, true, false);
    return failed;
}
