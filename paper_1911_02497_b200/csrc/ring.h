// What is still under way at the end of a ring of stages. Plain arithmetic, for host and device.
#pragma once
#include "pieces.h"

namespace cs {

// wait(stage, parity) for each copy that may still be under way once `issued` of them have been issued, one after the other around
// the ring: the last one of every stage. Parity is that of the phase which the copy completes at its stage's barrier, or the commit of the
// products that read it at theirs; a copy that was never issued must not be asked for, since the phase before it would answer.
template <class Wait>
CS_BOTH void copies_under_way(int issued, int stages, Wait wait)
{
    for (int i = issued > stages ? issued - stages : 0; i < issued; ++i) wait(i % stages, (i / stages) & 1);
}

// Batches of items are filled by two sides in turn, and each is committed once its last item is in use; a last batch with fewer items is not.
// Whether the last batch that `side` filled is committed (a commit that nobody has waited for yet).
CS_BOTH bool last_batch_commits(long long items, int batch, int side)
{
    const long long batches = (items + batch - 1) / batch, last = batches - 1 - (batches - 1 + side) % 2;
    return batches > side && (last + 1) * batch <= items;
}

}  // namespace cs
