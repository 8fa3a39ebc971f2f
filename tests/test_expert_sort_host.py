"""How the experts' sort is cut into blocks: bytes of its workspace tell (CPU only)."""
import os

import pytest


@pytest.fixture(scope="module")
def binding():
    from paper_2502_16982_amd import binding as b
    if not os.path.exists(b.library_path()):
        from paper_2502_16982_amd import build
        build.build_library()
    return b


@pytest.mark.parametrize("pairs,blocks", [(1, 0), (256, 0), (1024, 0), (1025, 3), (2048, 4), (131072, 256), (131073, 171), (1 << 30, 256)])
def test_blocks(binding, pairs, blocks):
    """One block needs no workspace; several leave a count per expert each."""
    assert binding.muon_expert_sort_bytes(pairs, 1, 66) == blocks * 66 * 4
