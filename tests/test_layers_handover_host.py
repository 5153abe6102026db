"""The flag that hands the sums of a cut tile over, in every order in which its two sides may come, call after call with the same mark (as a
captured call is replayed): it is down at the end, and no call takes the sums of the one before for its own."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2409_02097_b200", "csrc")

PROGRAM = r'''
#include <condition_variable>
#include <cstdio>
#include <mutex>
#include <string>
#include <thread>
#include "handover.h"

// The two sides take turns at the flag as `order` says; one that is done is passed over.
struct Turns {
    std::mutex m;
    std::condition_variable c;
    std::string order;
    size_t at = 0;
    bool done[2] = {false, false};
    unsigned long long flag = 0;
    bool mine(int side)
    {
        while (at < order.size() && done[order[at] - '0']) ++at;
        return at >= order.size() ? side == 0 || done[0] : order[at] - '0' == side;
    }
    template <typename F>
    unsigned long long step(int side, F f)
    {
        std::unique_lock<std::mutex> l(m);
        c.wait(l, [&] { return mine(side); });
        const unsigned long long was = flag;
        f(flag);
        if (at < order.size()) ++at;
        c.notify_all();
        return was;
    }
    void end(int side)
    {
        std::unique_lock<std::mutex> l(m);
        done[side] = true;
        c.notify_all();
    }
};

int main()
{
    const unsigned long long mark = 0x9E3779B97F4A7C15ull;
    int fetched = 0, left = 0;
    for (int bits = 0; bits < 64; ++bits)
        for (unsigned long long before : {0ull, 1ull, 77ull, ~0ull}) {
            unsigned long long flag = before;
            for (int call = 0; call < 3; ++call) {
                Turns t;
                for (int i = 0; i < 6; ++i) t.order += ((bits >> i) & 1) != 0 ? '1' : '0';
                t.flag = flag;
                bool there = false, got = false, stale = false;
                std::thread helper([&] {
                    lf::handover_raise([&](unsigned long long v) { return t.step(0, [&](unsigned long long& f) { f = v; there = true; }); }, mark);
                    t.end(0);
                });
                std::thread fetcher([&] {
                    got = t.step(1, [](unsigned long long&) {}) == mark;  // its last look
                    if (got) {
                        stale = !there;
                        t.step(1, [](unsigned long long& f) { f = 0; });
                    } else {
                        lf::handover_leave([&](unsigned long long v) { return t.step(1, [&](unsigned long long& f) { f = v; }); }, mark);
                    }
                    t.end(1);
                });
                helper.join();
                fetcher.join();
                flag = t.flag;
                ++(got ? fetched : left);
                if (stale || flag != 0) {
                    std::printf("order %s, call %d: flag %llx, stale %d\n", t.order.c_str(), call, flag, stale);
                    return 1;
                }
            }
        }
    std::printf("OK %d %d\n", fetched, left);
    return fetched > 0 && left > 0 ? 0 : 2;
}
'''


def test_no_flag_is_left_up(tmp_path):
    source, program = tmp_path / "handover.cpp", tmp_path / "handover"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-pthread", "-I", CSRC, "-o", str(program), str(source)], check=True)
    out = subprocess.run([str(program)], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.startswith("OK"), out.stdout
