// The work lists of packed batches (write_work_list, write_list), run on the CPU with a warp of 32 threads: every entry is written, by all that
// write it alike, none beyond the end, every block of every graph is there, and what is left says "unused", with and without rows behind the last graph.
#include "device_on_cpu.h"

struct Batch {
    std::vector<int32_t> cu;
    int32_t n_total;
    bool by_work;
};
static int g_failed = 0;

template <int kRows>
void check(const Batch& b, std::vector<int4>& list, std::vector<int>& writers)
{
    const int32_t graphs = (int32_t)b.cu.size() - 1, entries = b.n_total / kRows + graphs, guard = 64;
    const int4 untouched = make_int4(-77, -77, -77, -77);
    auto same = [](const int4& x, const int4& y) { return x.x == y.x && x.y == y.y && x.z == y.z && x.w == y.w; };
    const int lane = (int)threadIdx.x;
    std::vector<int4> whole;
    if (lane == 0) {
        writers.assign(entries + guard, 0);
        whole.assign(entries + guard, untouched);
    }
    for (int32_t g = 0; g < graphs; ++g) {
        if (lane == 0) list.assign(entries + guard, untouched);
        g_step.arrive_and_wait();
        gt::position::write_list<kRows>(list.data(), entries, b.cu.data(), graphs, g, b.by_work);
        g_step.arrive_and_wait();
        if (lane == 0)
            for (int32_t i = 0; i < entries + guard; ++i)
                if (!same(list[i], untouched)) {
                    writers[i] = writers[i] == 0 || same(whole[i], list[i]) ? 1 : 2;
                    whole[i] = list[i];
                }
    }
    if (lane == 0) {
        std::vector<int32_t> blocks(graphs);
        int bad = 0, last_work = 1 << 30;
        for (int32_t g = 0; g < graphs; ++g) blocks[g] = (b.cu[g + 1] - b.cu[g] + kRows - 1) / kRows;
        std::vector<std::vector<int>> seen(graphs);
        for (int32_t g = 0; g < graphs; ++g) seen[g].assign(blocks[g], 0);
        for (int32_t i = 0; i < entries + guard; ++i) {
            bad += writers[i] != (i < entries ? 1 : 0);
            const int4 e = whole[i];
            if (i >= entries || e.x == -1 || writers[i] == 0) continue;
            if (e.x < 0 || e.x >= graphs || e.y < 0 || e.y >= blocks[e.x] || e.z != b.cu[e.x] || e.w != b.cu[e.x + 1] - b.cu[e.x]) { ++bad; continue; }
            ++seen[e.x][e.y];
            if (b.by_work) {
                bad += blocks[e.x] - e.y > last_work;
                last_work = blocks[e.x] - e.y;
            }
        }
        for (auto& of : seen)
            for (int n : of) bad += n != 1;
        if (bad != 0) {
            printf("%d graphs, %d rows, %d behind the last one, blocks of %d%s: %d entries wrong\n", graphs, b.n_total, b.n_total - b.cu[graphs], kRows,
                   b.by_work ? ", by work" : "", bad);
            ++g_failed;
        }
    }
    g_step.arrive_and_wait();
}

int main()
{
    std::mt19937 rng(5);
    std::vector<Batch> batches;
    auto add = [&](int32_t graphs, int32_t low, int32_t high, int32_t behind) {
        Batch b{{0}, 0, false};
        for (int32_t g = 0; g < graphs; ++g) b.cu.push_back(b.cu.back() + low + (int32_t)(rng() % (unsigned)(high - low + 1)));
        b.n_total = std::max(1, b.cu.back() + behind);
        batches.push_back(b);
        if (graphs <= gt::kListSorted) {
            b.by_work = true;
            batches.push_back(b);
        }
    };
    for (int32_t behind : {0, 1, 300, 5000})
        for (int32_t graphs : {2, 31, 64, 65, 70}) {
            add(graphs, 0, 700, behind);
            add(graphs, 100, 373, behind);
            add(graphs, 0, 3, behind);
        }
    for (int32_t graphs : {2, 66}) add(graphs, 0, 0, 900);
    std::vector<int4> list;
    std::vector<int> writers;
    std::vector<std::thread> lanes;
    for (unsigned lane = 0; lane < 32; ++lane)
        lanes.emplace_back([&, lane] {
            threadIdx.x = lane;
            for (const Batch& b : batches) {
                check<128>(b, list, writers);
                check<256>(b, list, writers);
            }
        });
    for (auto& t : lanes) t.join();
    printf("%d of %d batches\n", (int)batches.size() * 2 - g_failed, (int)batches.size() * 2);
    return g_failed != 0;
}
