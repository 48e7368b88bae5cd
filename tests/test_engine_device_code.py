"""The gfx950 code the compiler makes of the kernels around the step (no GPU):
properties that no output shows."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_20186_amd import build as B

pytestmark = pytest.mark.skipif(shutil.which(B.HIPCC) is None, reason="no hipcc")

SOURCES = ("switchsd_logits.hip", "switchsd_pages.hip")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Assembly and descriptor of every kernel, by (mangled) name."""
    found = {}
    for src in SOURCES:
        out = str(tmp_path_factory.mktemp("asm") / "kernels.s")
        subprocess.run([B.HIPCC] + B.COMMON + B.DEVICE +
                       ["-x", "hip", "--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o",
                        out], check=True, capture_output=True, text=True, timeout=600)
        text = open(out).read()
        bodies = dict(re.findall(r"^(\w+):\s*; @\1\n(.*?)^\.Lfunc_end", text, re.M | re.S))
        meta = re.findall(r"^\s*\.amdhsa_kernel (\w+)\n(.*?)\.end_amdhsa_kernel", text,
                          re.M | re.S)
        found.update({n: (bodies[n], d) for n, d in meta})
    return found


def test_no_scratch_and_registers(kernels):
    """No scratch memory; the verification of logits keeps four waves to a SIMD
    (128 registers), of floats under a mask three."""
    assert len([n for n in kernels if "k_verify" in n]) == 24
    assert len([n for n in kernels if "k_process" in n]) == 30
    for n, (_, meta) in kernels.items():
        assert int(re.search(r"private_segment_fixed_size (\d+)", meta).group(1)) == 0, n
        if "k_verify" in n and not n.split("Evv")[0].endswith("Lb1EEEvNS_12LogitsParamsE"):
            regs = int(re.search(r"amdhsa_next_free_vgpr (\d+)", meta).group(1))
            assert regs <= 168, (n, regs)


def test_rows_are_read_as_vectors(kernels):
    """Rows at any element's address are read with 16-byte loads, and no packed
    float instruction is used."""
    for n, (body, _) in kernels.items():
        if "k_verify" in n or "k_process" in n:
            tiny = n.endswith("Lb1EEEvNS_12LogitsParamsE")
            wide = [l for l in body.splitlines()
                    if "global_load_dwordx4" in l and l.rstrip().endswith("nt")]
            assert bool(wide) != tiny, n
        assert "v_pk_add_f32" not in body and "v_pk_mul_f32" not in body, n
        assert "v_pk_fma_f32" not in body, n


def test_buffer_stores_are_bounded_by_the_row(kernels):
    """Stores that a lane leaves out go behind the buffer's record count, which
    bounds the lane's offset but not the scalar offset: that one is 0."""
    for n, (body, _) in kernels.items():
        stores = re.findall(r"buffer_store_\w+ \S+ \S+ s\[\d+:\d+\], (\S+) offen(.*)", body)
        assert len(stores) == body.count("buffer_store_"), n
        assert all(o == "0" and "offset:" not in rest for o, rest in stores), n
        assert "buffer_load_" not in body, n


def test_registers_of_the_verification(kernels):
    """Four waves to a SIMD (128 registers); floats under a mask, whole rows per
    wave, three (168).  Vocabularies of less than a vector are not held to it."""
    seen = set()
    for n, (_, meta) in kernels.items():
        m = re.search(r"k_verifyILi(\d)ELi(\d)ELi(\d)ELb(\d)ELb(\d)EE", n)
        if not m:
            assert "k_verify" not in n, n
            continue
        src, split, unroll, mask, tiny = (int(v) for v in m.groups())
        seen.add((src, split, unroll, mask, tiny))
        if not tiny:
            regs = int(re.search(r"amdhsa_next_free_vgpr (\d+)", meta).group(1))
            assert regs <= (168 if src == 2 and split == 1 and mask else 128), (n, regs)
    # each type: quarter rows of one and two vectors, whole rows, the tiny one,
    # each with and without masks
    assert seen == {(s, w, u, k, t) for s in range(3) for k in range(2)
                    for w, u, t in ((4, 1, 0), (4, 2, 0), (1, 2, 0), (4, 1, 1))}
