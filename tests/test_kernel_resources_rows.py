"""The kernels of row blocks and 8-bit checkpoints keep nothing in scratch memory, and leave the wavefronts they count on room in the registers
(the compiler's own resource report, no GPU needed)."""
import re
from concurrent.futures import ThreadPoolExecutor

from paper_2508_16769_amd import build


def test_row_kernels_use_no_scratch_memory():
    with ThreadPoolExecutor(max_workers=3) as pool:
        act8, block, dense = pool.map(build.kernel_resources, ("act8.hip", "block.hip", "dense.hip"))
    rows = {k: v for k, v in {**act8, **block}.items() if re.search(r"(block_fwd|block_bwd|act8_pack|act8_unpack|block_sums)_kernel", k)}
    grads = {k: v for k, v in {**act8, **dense}.items() if re.search(r"(act8_wgrad|act8_wgrad_sum|saved8_bwd)_kernel", k)}
    assert len(rows) >= 200 and len(grads) == 16, (len(rows), len(grads))
    for name, r in {**rows, **grads}.items():
        assert r["ScratchSize"] == 0 and r["VGPRs Spill"] == 0, (name, r)
    for name, r in rows.items():            # two workgroups of four wavefronts per compute unit, three where rows have any width
        assert r["Occupancy"] >= (3 if "RowTileILi1E" in name else 2), (name, r)
    for name, r in grads.items():           # a workgroup of eight wavefronts per compute unit
        assert r["Occupancy"] >= 2, (name, r)
