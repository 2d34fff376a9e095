// How many blocks of a kernel that holds rows of logits in shared memory an SM takes, and into how many stages each cuts its ring.
#pragma once

namespace ftp {

constexpr int kRingBytes = 200 * 1024;           // of the rings of all blocks of an SM
constexpr int kLossBlocksPerSm = 8;              // blocks of a loss, whatever its kernel: its workspace has room for a sum of each

struct RowRing { int blocks, stages; };

// `resident`: blocks that the kernel's registers and threads allow an SM.  Rings of two stages at least, and of up to four where as many
// blocks as that (a loss: as its workspace has room for) still fit.
inline RowRing row_ring(int resident, int stage_bytes, bool loss)
{
    RowRing r{loss && resident > kLossBlocksPerSm ? kLossBlocksPerSm : resident, 0};
    while (r.blocks > 1 && 2 * r.blocks * stage_bytes > kRingBytes) --r.blocks;
    r.stages = kRingBytes / (r.blocks * stage_bytes);
    if (r.stages > 4) r.stages = 4;
    return r;
}

}  // namespace ftp
