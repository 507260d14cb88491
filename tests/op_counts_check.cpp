// The record of waits that ran out (paper_2607_18957_gb300/csrc/cfa_ops.h): threads that ask at any time
// are each told of everything that has been counted, and of nothing twice.
#include <atomic>
#include <cstdio>
#include <thread>
#include <vector>

#include "cfa_ops.h"

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

int main()
{
    cfa_op_counts a = {0, 0}, b = {0, 0};
    CHECK(cfa_op_news(&a, {0, 0}) == 0);
    CHECK(cfa_op_news(&a, {3, 0}) == 1); // one asks
    CHECK(cfa_op_news(&a, {3, 0}) == 0);
    CHECK(cfa_op_news(&b, {3, 0}) == 1); // and the other is told all the same
    CHECK(cfa_op_news(&a, {4, 1}) == 2);
    CHECK(cfa_op_news(&a, {5, 1}) == 1); // what comes between two calls of a thread is news
    CHECK(cfa_op_news(&b, {5, 1}) == 2);
    CHECK(cfa_op_news(&a, {1, 0}) == 1); // a device that started again
    CHECK(cfa_op_news(&a, {1, 0}) == 0);
    CHECK(cfa_op_news(&b, {0, 0}) == 0);
    a = {0xFFFFFFFFu, 0};
    CHECK(cfa_op_news(&a, {2, 0}) == 1); // past 32 bits

    std::atomic<uint32_t> count{0};
    std::atomic<bool> over{false};
    std::vector<uint32_t> told(4, 0);
    std::vector<std::thread> threads;
    for (int i = 0; i < 4; ++i)
        threads.emplace_back([&, i] {
            cfa_op_counts seen = {0, 0};
            for (bool last = false; !last;) {
                last = over.load();
                const uint32_t was = seen.ran_out;
                const cfa_op_counts now = {count.load(), 0};
                if (cfa_op_news(&seen, now) == 1) told[i] += now.ran_out - was;
            }
        });
    for (int i = 0; i < 100000; ++i) count.fetch_add(1);
    over.store(true);
    for (auto &t : threads) t.join();
    for (uint32_t n : told) CHECK(n == 100000);
    return 0;
}
