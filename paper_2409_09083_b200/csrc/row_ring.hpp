// How many blocks of a kernel that holds rows of logits in shared memory an SM takes, and into how many stages each cuts its ring.
#pragma once

namespace ftp {

constexpr int kRingBytes = 200 * 1024;           // of the rings of all blocks of an SM
constexpr int kLossBlocksPerSm = 8;              // blocks of a loss, whatever its kernel: its workspace has room for a sum of each

struct RowRing { int blocks, stages; };

// `resident`: blocks that the kernel's registers and threads allow an SM.  Rings of two stages at least, and of up to four where as many
// blocks as that (a loss: as its workspace has room for) still fit.  The kernel's own 5.7 KB and the 1 KB that a block costs are not counted:
// where as many blocks as the registers allow fit by less than that, one of them starts only when another ends (loss of 8000 fp32 rows: 36
// us with 1656 and 1836 classes, 44 to 51 from 1664 to 1828).
inline RowRing row_ring(int resident, int stage_bytes, bool loss)
{
    RowRing r{loss && resident > kLossBlocksPerSm ? kLossBlocksPerSm : resident, 0};
    while (r.blocks > 1 && 2 * r.blocks * stage_bytes > kRingBytes) --r.blocks;
    r.stages = kRingBytes / (r.blocks * stage_bytes);
    if (r.stages > 4) r.stages = 4;
    return r;
}

}  // namespace ftp
