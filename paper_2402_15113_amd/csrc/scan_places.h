// The order in which a scan's workgroups take their tasks.  Host and device code.
#pragma once

#include <stdint.h>

namespace tgm {

// A runner waits for places of its own channel block, which may not have started.  At
// most kMaxRunners workgroups of a call do so at any time, so that the call goes on as
// long as one more fits the chip: with 512 at a time (two a CU), 63 such calls at once
// all end, whatever their widths.
//  - Narrow calls, of V runners for each channel block and no more than kMaxRunners in all:
//    every block has a counter, by which its workgroups (those of blockIdx.x % blocks)
//    take the runners' tasks and the places in order as they start.
//  - Wide ones: each wavefront of a runner (W of them) has a chain of its own, V chains a
//    block, and there is one counter.  The blocks come in slices of kMaxRunners runners; a
//    slice's runners, then its places, all blocks' place 0, all blocks' place 1, ...  What
//    has started is a run of tasks from the first on, and once a slice's last task is
//    taken nothing in it waits for a workgroup that has not started.
constexpr int32_t kMaxRunners = 8;

struct ScanTasks {
    int32_t blocks, groups;   // channel blocks, places of each
    int32_t V, W;

    constexpr bool narrow() const { return blocks * V <= kMaxRunners; }
    // blocks of a whole slice, runners for n blocks, tasks of a slice of n blocks
    constexpr int32_t deep() const { return kMaxRunners * W / V; }
    constexpr int32_t runners(int32_t n) const { return (n * V + W - 1) / W; }
    constexpr uint32_t tasks(int32_t n) const
    {
        return (uint32_t)runners(n) + (uint32_t)n * (uint32_t)groups;
    }
    constexpr int64_t all() const
    {
        if (narrow())
            return ((int64_t)groups + V) * blocks;
        const int32_t whole = blocks / deep(), rest = blocks - whole * deep();
        return (int64_t)whole * tasks(deep()) + tasks(rest);
    }
};

struct ScanTask {
    int32_t block;   // place >= 0: the channel block; else the slice's first one
    int32_t place;   // < 0: runner -1 - place of the slice
};

// The ticket-th task of a wide call's counter.
constexpr ScanTask wide_task(const ScanTasks &c, uint32_t ticket)
{
    const uint32_t slice = ticket / c.tasks(c.deep()), t = ticket - slice * c.tasks(c.deep());
    const int32_t first = (int32_t)slice * c.deep();
    const int32_t n = c.blocks - first < c.deep() ? c.blocks - first : c.deep();
    const uint32_t runners = (uint32_t)c.runners(n);
    if (t < runners)
        return ScanTask{first, -1 - (int32_t)t};
    const uint32_t place = (t - runners) / (uint32_t)n;
    return ScanTask{first + (int32_t)(t - runners - place * (uint32_t)n), (int32_t)place};
}

}  // namespace tgm
