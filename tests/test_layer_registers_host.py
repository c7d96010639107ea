"""No kernel of the layer operators keeps registers in scratch memory, read from the compiler's report (no GPU needed)."""
import shutil

import pytest

from tests.test_attention_registers_host import test_no_spilled_registers as no_spilled_registers


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("source,kernels", [("dn_short_conv.hip", 18), ("dn_layer_norm.hip", 72)])
def test_no_spilled_registers(source, kernels, tmp_path):
    no_spilled_registers(source, kernels, tmp_path)
