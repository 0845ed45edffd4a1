// The turns of a ring of shared-memory slots that one warp fills with asynchronous copies and empties in the same order: which
// slot the next copy goes to, which one is waited for next and with what parity, and how many copies are on their way.  The user
// asks `size` times at the start, and then once for each copy used, before next(): so a slot asked into is always free.  No CUDA
// in it but the qualifiers, so that it can be played on the host.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define POLYSPEC_HD __host__ __device__ __forceinline__
#else
#define POLYSPEC_HD inline
#endif

namespace polyspec {

struct PieceRing {
    int size;               // slots
    int to_ask;             // copies still to be asked for
    int flying = 0;         // asked for and not done with
    int ask_at = 0, at = 0;
    uint32_t phase = 0;     // parity of the slot waited for next

    POLYSPEC_HD PieceRing(int size_, int copies) : size(size_), to_ask(copies) {}

    // There is another copy, to go into slot ask_at.
    POLYSPEC_HD bool may_ask() const { return to_ask > 0; }
    POLYSPEC_HD void asked()
    {
        --to_ask;
        ++flying;
        if (++ask_at == size) ask_at = 0;
    }
    // Done with the copy in slot `at`.
    POLYSPEC_HD void next()
    {
        --flying;
        if (++at == size) { at = 0; phase ^= 1u; }
    }
    // A wait has run out: nothing more is asked for; the copies on their way, in slots at, at + 1, ..., are waited for with
    // `wait(slot, parity)`, which returns after a bounded time, before their memory may be used otherwise or given up.
    template <class Wait>
    POLYSPEC_HD void give_up(Wait wait)
    {
        to_ask = 0;
        while (flying > 0) {
            wait(at, phase);
            next();
        }
    }
};

}  // namespace polyspec
