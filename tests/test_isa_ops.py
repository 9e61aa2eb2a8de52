"""Static checks on the generated gfx950 code of the paged decoding, the head
norms and the page plan (CPU only: hipcc cross-compiles): nothing in scratch
memory, LDS within a CU, and in the paged kernel's tile loops operands read
ahead of the matrix products, which wait for no copy and no scalar load (a
scalar load in flight turns every wait for an LDS read into one for all)."""
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
    for src in ("paged.hip", "rope.hip", "plan.hip"):
        out = tmp_path_factory.mktemp("isa") / (src + ".s")
        flags = [f for f in compile_flags(src) if f != "-fPIC"]
        r = subprocess.run([HIPCC, *flags, f"-I{CSRC}", "--cuda-device-only", "-S", "-o", str(out), str(CSRC / src)],
                           capture_output=True, text=True, timeout=600)
        assert r.returncode == 0, r.stderr[-2000:]
        texts[src] = out.read_text()
    return texts


def test_nothing_in_scratch_memory(assembly):
    kernels = {k: v for text in assembly.values() for k, v in _metadata(text).items()}
    for part in ("paged_kernel", "dec_combine_kernel", "rope_fwd_kernel", "rope_bwd_kernel", "plan_kernel"):
        for name, f in _find(kernels, part).items():
            assert f.get("private_segment_fixed_size", 0) == 0, name


def test_lds_fits_one_cu(assembly):
    for name, f in _find(_metadata(assembly["paged.hip"]), "paged_kernel").items():
        assert 0 < f["group_segment_fixed_size"] <= LDS_PER_CU, (name, f)


@pytest.mark.parametrize("part,loops", [("paged_kernelILi128ELi1", 4), ("paged_kernelILi128ELi2", 4), ("paged_kernelILi128ELi4", 4),
                                        ("paged_kernelILi64ELi2", 4), ("paged_kernelILi64ELi4", 4)])
def test_paged_tile_loops(assembly, part, loops):
    """Blocks of eight products and more: scores and output, with and without the streaming hint."""
    seen = 0
    for block in _blocks(assembly["paged.hip"], part):
        if sum("v_mfma" in x for x in block) < 8:
            continue
        seen += 1
        products = [i for i, x in enumerate(block) if "v_mfma" in x]
        inner = block[products[0]:products[-1]]
        assert not any("vmcnt" in x or x.startswith("s_load") for x in inner), block[0]
        drained = sum("v_mfma" in y and "lgkmcnt(0)" in x for x, y in zip(block, block[1:]))
        assert drained <= 2, (part, drained)
    assert seen == loops
