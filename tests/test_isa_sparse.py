"""Static checks on the generated gfx950 code of decoding with shared prefixes and over
chosen pages (CPU only): nothing in scratch memory, LDS within a CU, and tile loops that
read operands ahead of the matrix products and wait for no copy and no scalar load
between them, as those of the paged decoding."""
from __future__ import annotations

import subprocess
from pathlib import Path

import pytest
from test_isa import CSRC, HIPCC, LDS_PER_CU, _blocks, _find, _metadata


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    if not Path(HIPCC).exists():
        pytest.skip("hipcc not available")
    from paper_2512_22234_amd.build import compile_flags
    texts = {}
    for src in ("shared.hip", "sparse.hip"):
        out = tmp_path_factory.mktemp("isa") / (src + ".s")
        flags = [f for f in compile_flags(src) if f != "-fPIC"]
        r = subprocess.run([HIPCC, *flags, f"-I{CSRC}", "--cuda-device-only", "-S", "-o", str(out), str(CSRC / src)],
                           capture_output=True, text=True, timeout=600)
        assert r.returncode == 0, r.stderr[-2000:]
        texts[src] = out.read_text()
    return texts


def test_nothing_in_scratch_memory(assembly):
    for text in assembly.values():
        for name, f in _metadata(text).items():
            assert f.get("private_segment_fixed_size", 0) == 0, name
            assert f["group_segment_fixed_size"] <= LDS_PER_CU, name
    _find(_metadata(assembly["shared.hip"]), "shared_merge_kernel")
    for part in ("summarize_kernel", "score_kernel", "select_kernel"):
        _find(_metadata(assembly["sparse.hip"]), part)


@pytest.mark.parametrize("src", ["shared.hip", "sparse.hip"])
def test_tile_loops(assembly, src):
    """Blocks of eight products and more of every paged kernel."""
    names = _find(_metadata(assembly[src]), "paged_kernel")
    for name in names:
        seen = 0
        for block in _blocks(assembly[src], name):
            if sum("v_mfma" in x for x in block) < 8:
                continue
            seen += 1
            products = [i for i, x in enumerate(block) if "v_mfma" in x]
            inner = block[products[0]:products[-1]]
            assert not any("vmcnt" in x or x.startswith("s_load") for x in inner), (name, block[0])
            drained = sum("v_mfma" in y and "lgkmcnt(0)" in x for x, y in zip(block, block[1:]))
            assert drained <= 2, (name, drained)
        assert seen >= 2, name


@pytest.mark.parametrize("D,products,copies", [(64, 8, 4), (128, 16, 8)])
def test_prefix_tile_loops(assembly, D, products, copies):
    """The prefixes' kernel: the scores' products with the copies of a tile among them, then the output's, without a wait
    for copies, a scalar load or a repeated wait for all reads in between."""
    blocks = [b for b in _blocks(assembly["shared.hip"], f"prefix_kernelILi{D}E") if sum("v_mfma" in x for x in b) >= 8]
    assert [sum("v_mfma" in x for x in b) for b in blocks] == [products, 2 * products]
    for block, n in zip(blocks, (copies, 0)):
        at = [i for i, x in enumerate(block) if "v_mfma" in x]
        inner = block[at[0]:at[-1]]
        assert not any("vmcnt" in x or x.startswith("s_load") for x in inner), (D, block[0])
        assert sum("v_mfma" in y and "lgkmcnt(0)" in x for x, y in zip(block, block[1:])) <= 2, (D, block[0])
        assert sum("buffer_load" in x for x in block) == n == sum("buffer_load" in x and "lds" in x for x in block), (D, block[0])
