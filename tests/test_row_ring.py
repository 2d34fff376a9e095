"""The rule that shapes the rings of rows (csrc/row_ring.hpp), compiled for the CPU and looked over for every number of blocks an SM that a
kernel's registers may come to, not for today's alone."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2409_09083_b200", "csrc")

PROGRAM = """
#include <cstdio>
#include "row_ring.hpp"
int main()
{
    for (int loss = 0; loss < 2; ++loss)
        for (int resident = 1; resident <= 32; ++resident)
            for (int stage = 16; stage <= 64 * 1024; stage += 16) {
                const ftp::RowRing r = ftp::row_ring(resident, stage, loss);
                if (r.blocks < 1 || r.blocks > resident || r.stages < 2 || r.stages > 4 || r.blocks * r.stages * stage > ftp::kRingBytes ||
                    (loss && r.blocks > ftp::kLossBlocksPerSm)) {
                    std::printf("loss %d, %d resident blocks, stages of %d bytes: %d blocks of %d stages\\n", loss, resident, stage, r.blocks, r.stages);
                    return 1;
                }
            }
    return 0;
}
"""


def test_rings_fit_and_a_loss_has_no_more_blocks_than_its_workspace_has_sums(tmp_path):
    source, binary = tmp_path / "ring.cpp", tmp_path / "ring"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, str(source), "-o", str(binary)], check=True)
    done = subprocess.run([str(binary)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout


def test_every_grid_of_a_loss_keeps_to_the_workspace():
    """The three launches that ftp_loss_logprob chooses from: two cap their blocks where they are counted, one takes the rule above."""
    with open(os.path.join(CSRC, "logprob.cu")) as f:
        text = f.read()
    assert "kMostBlocks = kLossBlocksPerSm * kSms" in text
    for name in ("run_warp_rows", "run_map", "run_block_rows"):
        at = text.index(f"int {name}(")
        body = text[at:text.index("\n}\n", at)]
        assert "fit < kLossBlocksPerSm ? fit : kLossBlocksPerSm" in body or "row_ring(" in body and "MODE == kLoss)" in body, name
