"""The way of two warps that meet at named barriers, compiled for the host: whichever waits of theirs run out, neither is left standing at a barrier, and they
end together."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_03383_b200", "csrc")

SOURCE = """
#include <algorithm>
#include <atomic>
#include <chrono>
#include <condition_variable>
#include <mutex>
#include <thread>
#include "in_step.cuh"

// Two threads meet; one that stands for too long reports it.
struct Meeting {
    std::mutex lock;
    std::condition_variable change;
    int here = 0, turn = 0, met = 0;
    bool all = true, answer = true, stuck = false;
    int limit_ms = 0;
    bool meet(bool x) {
        std::unique_lock<std::mutex> l(lock);
        if (stuck) return false;
        all = all && x;
        if (++here == 2) {
            answer = all;
            all = true;
            here = 0;
            ++turn;
            ++met;
            change.notify_all();
            return answer;
        }
        const int t = turn;
        if (!change.wait_for(l, std::chrono::milliseconds(limit_ms), [&] { return turn != t || stuck; })) {
            stuck = true;
            change.notify_all();
        }
        return !stuck && answer;
    }
};

struct Warp {
    Meeting *m;
    int fails, id;
    std::atomic<bool> *flag;
    int waits = 0, pieces = 0;
    bool wait() {
        if (waits++ != fails) return true;
        *flag = true;
        return false;
    }
};

static float shared_value[2];

// Pieces of `tiles` tiles each, as the softmax warps of the attention over pages go through them.  Of codes (carried): the end of a piece is behind the next one's
// queries, and an exchange meets twice.  Of bf16: it meets once, and once more in front of a tile's second terms, where there are such.
static void walk(Warp &w, int n_pieces, int tiles, bool carried, bool two, bool sees_flag) {
    using namespace mtv;
    const float none = -1e30f;
    float m = none;
    int left_at = 0;
    auto exchange = [&](float x) {
        shared_value[w.id] = x;
        w.m->meet(true);
        const float other = shared_value[w.id ^ 1];
        if (carried) w.m->meet(true);
        return other;
    };
    // what the two halves of a row have in a tile: nothing in some, more and more in others
    auto own = [&](int n, int t) { return (n + t + w.id) % 3 == 0 ? none : (float)(t * (n % 2 ? 5 : 1) + w.id); };
    auto other_half = [&](int n, int t) { return (n + t + (w.id ^ 1)) % 3 == 0 ? none : (float)(t * (n % 2 ? 5 : 1) + (w.id ^ 1)); };
    auto asked = [&](bool ask) { return !w.m->meet(!ask); };
    pieces_in_step([&](int) { return !(sees_flag && *w.flag) && w.wait(); }, [&](bool x) { return w.m->meet(x); }, [&](int n) {
        const bool more = n < n_pieces;
        if (carried) {
            if (more) {
                if (!w.wait()) { left_at = -1; return Way::LEFT; }
                exchange(0.f);
            }
            if (n && !w.wait()) { left_at = 0; return more ? Way::LEFT : Way::END; }
        }
        if (!more) return Way::END;
        ++w.pieces;
        m = none;
        for (int t = 0; t < tiles; ++t) {
            if (!w.wait()) { left_at = t; return Way::LEFT; }
            bool move = t == 0;
            for (;;) {
                if (move) {
                    const float x = own(n, t);
                    exchange(x);
                    m = std::max(m, std::max(own(n, t), other_half(n, t)));
                    break;
                }
                if (!asked(m == none || own(n, t) > m + 3.f)) break;
                move = true;
            }
            if (t == tiles - 1) exchange(1.f);
            if (two && (move || t == tiles - 1)) w.m->meet(true);
        }
        if (!carried && !w.wait()) { left_at = tiles; return Way::LEFT; }
        return Way::ON;
    }, [&] {
        if (left_at < 0) {
            exchange(0.f);
            left_at = 0;
        }
        follow_tiles(left_at, 0, tiles, [&] { return asked(false); }, [&](bool last) {
            exchange(none);
            if (two && !last) w.m->meet(true);
        }, [&] {
            exchange(1.f);
            if (two) w.m->meet(true);
        });
    });
}

// The same with a warp that leaves where its wait ran out.
static void walk_alone(Warp &w, int n_pieces, int tiles) {
    for (int n = 0; n < n_pieces && !w.m->stuck; ++n)
        for (int t = 0; t < tiles && !w.m->stuck; ++t) {
            if (!w.wait()) return;
            w.m->meet(true);
        }
}

extern "C" int run(int fails0, int fails1, int sees, int n_pieces, int tiles, int kind, int alone, int limit_ms, int *out) {
    Meeting m;
    std::atomic<bool> flag(false);
    m.limit_ms = limit_ms;
    // (one flag of both, or each sees its own alone: a flag may be set behind the other's look)
    std::atomic<bool> flags[2] = {{false}, {false}};
    Warp w[2] = {{&m, fails0, 0, sees >> 2 ? &flag : &flags[0]}, {&m, fails1, 1, sees >> 2 ? &flag : &flags[1]}};
    std::thread t0([&] { alone ? walk_alone(w[0], n_pieces, tiles) : walk(w[0], n_pieces, tiles, kind == 1, kind == 2, sees & 1); });
    std::thread t1([&] { alone ? walk_alone(w[1], n_pieces, tiles) : walk(w[1], n_pieces, tiles, kind == 1, kind == 2, sees >> 1 & 1); });
    t0.join();
    t1.join();
    for (int i = 0; i < 2; ++i) {
        out[i * 2] = w[i].pieces;
        out[i * 2 + 1] = w[i].waits;
    }
    return m.stuck ? -1 : m.here ? -2 : m.met;
}
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    d = tmp_path_factory.mktemp("step")
    src, lib = d / "step.cpp", d / "step.so"
    src.write_text(SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-pthread", "-I", CSRC, "-o", str(lib), str(src)])
    L = C.CDLL(str(lib))

    def call(fails0, fails1, sees=3, pieces=3, tiles=3, kind=1, alone=0, limit_ms=20000):
        out = (C.c_int * 4)()
        return L.run(fails0, fails1, sees, pieces, tiles, kind, alone, limit_ms, out), list(out)
    return call


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("sees", [0, 3, 5, 7])
@pytest.mark.parametrize("tiles", [1, 4])
def test_waits_that_run_out(run, tiles, sees, kind):
    met, (pieces, waits, *other) = run(-1, -1, sees, tiles=tiles, kind=kind)
    assert met > 0 and pieces == 3 and other == [pieces, waits]
    for fails0 in range(-1, waits):
        for fails1 in range(-1, waits):
            met, (pieces0, waits0, pieces1, waits1) = run(fails0, fails1, sees, tiles=tiles, kind=kind)
            assert met >= 1, (fails0, fails1)                              # (-1: one stands at a barrier; -2: one stood there at the end)
            assert abs(pieces0 - pieces1) <= 1 and waits0 <= waits and waits1 <= waits
            assert fails0 < 0 or waits0 <= fails0 + 1, (fails0, fails1)    # nothing is waited for behind a wait that ran out


def test_a_warp_that_leaves_alone_is_noticed(run):
    assert run(-1, -1, alone=1)[0] == 9
    assert run(4, -1, alone=1, limit_ms=200)[0] == -1


@pytest.mark.parametrize("name", ["attention_paged.cu", "attention_paged_fp8.cu"])
def test_the_kernels_go_this_way(name):
    """No way out of the softmax warps' part but the common one, in front of which they meet."""
    text = open(os.path.join(CSRC, name)).read()
    part = text[text.index("// ------------------------------------------------------------ softmax:"):]
    part = part[:part.index("bar.sync 1")] if "bar.sync 1" in part else part[:part.index("pa_cta_sync()")]
    assert "pieces_in_step(" in part and "follow_tiles(" in part
    for at in part.split("if (!wait(")[1:]:
        assert "Way::LEFT" in at[:300]
    assert "break; }" not in part and "ok = false" not in part
