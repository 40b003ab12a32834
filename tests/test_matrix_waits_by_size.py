"""The check of tests/test_matrix_waits.py with the wait of each product's own size: one of 32 x 32 x 16 keeps the matrix unit for twice as many passes as one of 16 x 16 x 32, and its result is
there four slots later.  CPU only."""
import os
import re
import subprocess

import pytest

import test_matrix_waits as waits
from paper_2502_13652_amd import binding

SLOTS = {"16x16x32": 8, "32x32x16": 12}                      # what the compiler itself waits between a product and its reader in one block


def early_reads(assembly, monkeypatch):
    monkeypatch.setattr(waits, "SLOTS", max(SLOTS.values()))
    total, found = waits.early_reads(assembly)
    size = lambda product: re.match(r"v_mfma_f32_(\d+x\d+x\d+)_", product).group(1)
    assert set(re.findall(r"v_mfma_f32_(\d+x\d+x\d+)", assembly)) <= set(SLOTS) and len(re.findall(r"\tv_mfma_", assembly)) == total      # (a product of another kind has no wait here)
    return total, [f for f in found if f[2] < SLOTS[size(f[0])]]


@pytest.mark.parametrize("size,registers,slots", [("16x16x32", 3, 8), ("32x32x16", 15, 12)])
def test_the_check_counts_by_the_products_size(size, registers, slots, monkeypatch):
    text = """
_Zk:
	v_mfma_f32_%s_bf16 a[0:%d], v[44:47], v[48:51], a[0:%d]
	s_nop %d
	s_cbranch_scc1 .L2
.L1:
	v_accvgpr_read_b32 v20, a%d
	s_endpgm
.L2:
	s_branch .L1
.Lfunc_end0:
"""
    for nop in (slots - 2, slots - 3, 0):
        total, found = early_reads(text % (size, registers, registers, nop, registers), monkeypatch)
        assert total == 1 and {reader for _, reader, _ in found} == ({"v_accvgpr_read_b32 v20, a%d" % registers} if nop + 2 < slots else set())
        assert not found or min(s for _, _, s in found) == nop + 2


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """The library's device code as assembly, and what the compiler printed."""
    out = str(tmp_path_factory.mktemp("waits") / "device.s")
    flags = [f for f in binding.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    package = os.path.dirname(binding.__file__)
    r = subprocess.run(["hipcc"] + flags + ["-S", "--offload-device-only", "-I", os.path.join(os.path.dirname(package), "include"), os.path.join(package, "csrc", "c2t_lib.hip"), "-o", out],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    with open(out) as f:
        return f.read(), r.stdout


def test_no_matrix_result_is_read_early(compiled, monkeypatch):
    total, found = early_reads(compiled[0], monkeypatch)
    assert total > 500 and not found, found[:8]


def test_loads_into_lds_find_their_place_in_m0(compiled):
    """Each load into LDS has its address set for it in its own block, by the compiler, which knows of it: no warning of a register that is not the code's to change."""
    assert "inline-asm" not in compiled[1], compiled[1][:1000]
    loads = 0
    for block in re.split(r"\n\.L\w+:", compiled[0]):
        code = [line.strip() for line in block.split("\n")]
        m0 = False
        for line in code:
            m0 = m0 or re.match(r"s_\w+ m0,", line) is not None
            if line.startswith("global_load_lds"):
                loads += 1
                assert m0, line
                m0 = False
    assert loads > 100
