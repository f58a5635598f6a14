"""The build ends where a kernel's registers are not what its source shares out."""
import pytest

from paper_2609_09800_b200 import build

LOG = """ptxas info    : Compiling entry function '_Z14k_prefix_tilesA' for 'sm_100a'
ptxas info    : Function properties for _Z14k_prefix_tilesA
    0 bytes stack frame, 0 bytes spill stores, 0 bytes spill loads
ptxas info    : Used %d registers, used 16 barriers
ptxas info    : Compiling entry function '_Z5otherv' for 'sm_100a'
ptxas info    : Used 33 registers
ptxas info    : Compiling entry function '_Z14k_prefix_tilesB' for 'sm_100a'
ptxas info    : Used %d registers, used 16 barriers
"""


def test_the_number_that_the_source_counts_on():
    build.check_registers({"k_prefix_tiles": 80}, LOG % (80, 80))
    build.check_registers({"k_prefix_tiles": 80, "other": 33}, LOG % (80, 80))
    for log in (LOG % (80, 72), LOG % (72, 72), "", LOG.replace("k_prefix_tiles", "k_renamed") % (80, 80)):
        with pytest.raises(RuntimeError, match="k_prefix_tiles"):
            build.check_registers({"k_prefix_tiles": 80}, log)


def test_its_shares_add_up_to_it():
    """What the warps of a block ask for is what the block was launched with."""
    import os
    import re
    for src, kernels in build.REGISTERS.items():
        with open(os.path.join(build.CSRC, src)) as f:
            text = f.read()
        shares = [int(n) for n in re.findall(r"setmaxnreg\.\w+\.sync\.aligned\.u32 (\d+);", text)]
        assert shares == [56, 40, 96]                        # warps 16 to 19, 20 to 23, 0 to 15
        assert 4 * 56 + 4 * 40 + 16 * 96 == 24 * kernels["k_prefix_tiles"]
