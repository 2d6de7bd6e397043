// Copies of a ring of stages. Plain arithmetic, for host and device.
#pragma once
#include "pieces.h"

namespace cs {

// wait(stage, parity) for each copy that may still be under way once `issued` of them have been issued, one after the other around
// the ring: the last one of every stage. Parity is that of the phase which the copy completes at its stage's barrier; a copy that was never
// issued must not be asked for, since the phase before it would answer.
template <class Wait>
CS_BOTH void copies_under_way(int issued, int stages, Wait wait)
{
    for (int i = issued > stages ? issued - stages : 0; i < issued; ++i) wait(i % stages, (i / stages) & 1);
}

}  // namespace cs
