"""The transforms of the serving operators use DPP multiply-adds in inline assembly: the wait states
that the compiler does not insert there, checked on the assembly that it makes of those kernels."""
import shutil
import subprocess

import pytest

from paper_2607_07964_amd import build as B
from test_dpp_wait_states import dpp_hazards


@pytest.mark.skipif(shutil.which(B.HIPCC) is None, reason="no hipcc here")
@pytest.mark.parametrize("source,least", [("kvcache.hip", 300), ("online_sides.hip", 3000)])
def test_serving_dpp_wait_states(source, least, tmp_path):
    out = tmp_path / "kernels.s"
    subprocess.run([B.HIPCC, *B.FLAGS, "-x", "hip", "--offload-device-only", "-S",
                    f"{B.CSRC}/{source}", "-o", str(out)], check=True, capture_output=True)
    found, bad = dpp_hazards(out.read_text())
    assert found > least and bad == []
