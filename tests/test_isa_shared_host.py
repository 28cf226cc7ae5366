"""The tile loops of the shared attention's query blocks, as compiled: instances of the prefill attention's loop, on other pages and with probabilities in two parts."""
import re

import pytest

from test_isa_host import MFMA, compile_to_isa, replay_lds_counter


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    lines = compile_to_isa(tmp_path_factory.mktemp("isa_shared"), "kernels_attn_shared.hip")
    starts = [i for i, l in enumerate(lines) if re.match(r"^_ZN3dyn\S*:", l)]
    return {lines[i]: lines[i:j] for i, j in zip(starts, starts[1:] + [len(lines)])}


def test_query_blocks_touch_no_operand_before_its_wait(kernels):
    found = {name: body for name, body in kernels.items() if "attn_shared_kernelILb" in name}
    assert len(found) == 2
    for name, body in found.items():
        reads = [j for j, x in enumerate(body) if x.strip().startswith("ds_read") and "ASMSTART" in body[j - 1]]
        assert len(reads) == 4 * 4 + 8 * 4                               # one copy of the loop for both lists: four K pages of four operands, eight V groups of four
        head = max(j for j, x in enumerate(body) if "Loop Header" in x and j < reads[0])
        last_mfma = max(j for j, x in enumerate(body) if MFMA in x)
        violations, n = replay_lds_counter(body[head:last_mfma + 1])
        assert n == 48 and not violations, (name, violations[:5])


def test_everything_stays_in_registers(kernels):
    """A spill in the loop would be scratch loads and stores between reads and waits placed by hand."""
    sizes = {name: int(re.search(r"ScratchSize: (\d+)", "\n".join(body)).group(1)) for name, body in kernels.items() if "; ScratchSize" in "\n".join(body)}
    assert len(sizes) >= 14 and not any(sizes.values()), sizes
