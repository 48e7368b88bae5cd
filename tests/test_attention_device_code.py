"""The gfx950 code the compiler makes of the attention and the log probabilities
(no GPU): properties that no output shows."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_20186_amd import build as B

pytestmark = pytest.mark.skipif(shutil.which(B.HIPCC) is None, reason="no hipcc")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Assembly and descriptor of every kernel, by (mangled) name."""
    found = {}
    for src in ("switchsd_attention.hip", "switchsd_logprobs.hip"):
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


def number(meta, key):
    return int(re.search(key + r"\s+(\d+)", meta).group(1))


def test_kernels_and_no_packed_float(kernels):
    """Both types, with 16- and 8-bit caches, of three widths; no packed float
    instruction is used."""
    count = {k: len([n for n in kernels if k in n])
             for k in ("k_attend_few", "k_attend_many", "k_merge", "k_store", "k_logprobI",
                       "k_logprob_grad")}
    assert count == {"k_attend_few": 12, "k_attend_many": 12, "k_merge": 24, "k_store": 4,
                     "k_logprobI": 3, "k_logprob_grad": 3}
    for n, (body, _) in kernels.items():
        assert not re.search(r"v_pk_(add|mul|fma)_f32", body), n


def test_two_work_groups_on_a_compute_unit(kernels):
    """Registers (512 for a SIMD's waves) and LDS (160 KB) leave room for two
    work-groups of the narrower heads, for one of 256-wide ones."""
    for n, (_, meta) in kernels.items():
        regs, lds = number(meta, "amdhsa_next_free_vgpr"), number(meta, "group_segment_fixed_size")
        if "k_attend" in n:
            two = "ELi256E" not in n
            assert regs <= (256 if two else 512), (n, regs)
            assert lds <= 163840 // (2 if two else 1), (n, lds)
        if "k_logprobI" in n:
            assert regs <= 128, (n, regs)


def test_no_scratch_where_rows_stream(kernels):
    """No scratch memory but in the attention of 256-wide heads."""
    for n, (_, meta) in kernels.items():
        if "k_attend" in n and "ELi256E" in n:
            continue
        assert number(meta, "private_segment_fixed_size") == 0, n


def test_products_are_fed_ahead(kernels):
    """No product in the shared-tile kernel waits for a read that was issued right
    before it: where one does follow a read, the wait leaves that read in flight."""
    for n, (body, _) in kernels.items():
        if "k_attend_many" not in n:
            continue
        ops = [x.split(";")[0].strip() for x in body.splitlines()
               if x.startswith("\t") and not x.strip().startswith((";", "."))]
        products = [i for i, op in enumerate(ops) if "mfma" in op]
        assert len(products) >= 16, n
        tight = [i for i in products
                 if "lgkmcnt(0)" in ops[i - 1] and ops[i - 2].startswith("ds_read")]
        assert not tight, (n, len(tight), len(products))
