// The ring of csrc/piece_ring.cuh played as the 4-bit head's warps play it, with copies that land late, and given up at every
// point: every copy asked for is waited for once, in order, with the parity its slot's barrier then has; no slot is asked for
// while a copy is on its way to it; nothing is asked for after the ring has been given up.
#include <cstdio>
#include <vector>

#include "piece_ring.cuh"

using polyspec::PieceRing;

static int failed = 0;
static void check(bool ok, const char* what, int size, int copies, int stop)
{
    if (!ok) { std::printf("size %d, %d copies, given up at %d: %s\n", size, copies, stop, what); ++failed; }
}

// Given up when `stop` copies have been used (never, if there are no more than that).
static void play(int size, int copies, int stop)
{
    PieceRing ring(size, copies);
    std::vector<int> uses(size, 0);             // copies asked for into each slot so far
    std::vector<bool> flying(size, false);
    int asked = 0, waited = 0;
    auto ask = [&]() {
        if (!ring.may_ask()) return;
        check(!flying[ring.ask_at], "asked into a slot in flight", size, copies, stop);
        flying[ring.ask_at] = true;
        ++uses[ring.ask_at];
        ++asked;
        ring.asked();
    };
    auto wait = [&](int slot, uint32_t parity) {
        check(slot == waited % size, "order", size, copies, stop);
        check(flying[slot], "waited for a slot with no copy on its way", size, copies, stop);
        check(parity == static_cast<uint32_t>(uses[slot] - 1) % 2, "parity", size, copies, stop);
        flying[slot] = false;
        ++waited;
    };
    for (int i = 0; i < size; ++i) ask();
    bool lost = false;
    for (int i = 0; i < copies && !lost; ++i) {
        if (i == stop) {
            ring.give_up(wait);
            lost = true;
            break;
        }
        wait(ring.at, ring.phase);
        ask();
        ring.next();
    }
    const int before = asked;
    ask();
    check(asked == before, "asked at the end", size, copies, stop);
    check(waited == asked, "copies left on their way", size, copies, stop);
    check(lost ? asked == (stop + size < copies ? stop + size : copies) : asked == copies, "copies asked for", size, copies, stop);
    for (int i = 0; i < size; ++i) check(!flying[i], "a slot in flight at the end", size, copies, stop);
}

int main()
{
    for (int size = 1; size <= 6; ++size)
        for (int copies = 0; copies <= 20; ++copies)
            for (int stop = 0; stop <= copies; ++stop) play(size, copies, stop);
    std::printf("%d failed checks\n", failed);
    return failed != 0;
}
