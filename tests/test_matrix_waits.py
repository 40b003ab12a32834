"""A matrix instruction's result may be read by other instructions only some issue slots later, and nothing but the compiler's count of them keeps an earlier read from
getting what was there before.  It has been seen to count wrongly where product and read lie in different blocks, so the library's own device code, compiled to assembly, is
checked: from each matrix instruction along every path that control may take.  CPU only."""
import os
import re
import subprocess
import tempfile

from paper_2502_13652_amd import binding

SLOTS = 8                                                    # what the compiler itself waits between a 16 x 16 x 32 product and its reader in one block


def _registers(text):
    out = set()
    for kind, lo, hi, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        out.update((kind, i) for i in (range(int(lo), int(hi) + 1) if lo else [int(one)]))
    return out


def early_reads(assembly):
    """(matrix instructions, [(instruction, its reader, slots between them)]) of a compiler's assembly listing."""
    total, found = 0, []
    for body in re.findall(r"\n_Z\w+:[^\n]*\n(.*?)\.Lfunc_end", assembly, re.S):
        if "v_mfma" not in body:
            continue
        code, labels = [], {}
        for line in body.split("\n"):
            line = line.split(";")[0].strip()
            if line.endswith(":"):
                labels[line[:-1]] = len(code)
            elif line and not line.startswith("."):
                code.append(line)

        def after(i):
            op = code[i].split()[0]
            if op == "s_branch":
                return [labels[code[i].split()[1]]]
            return [] if op == "s_endpgm" else [i + 1] + ([labels[code[i].split()[1]]] if op.startswith("s_cbranch") else [])
        for i, line in enumerate(code):
            if not line.startswith("v_mfma"):
                continue
            total += 1
            result = _registers(line.split(None, 1)[1].split(",")[0])
            best, todo = {}, [(j, 0) for j in after(i)]
            while todo:
                j, slots = todo.pop()
                if j >= len(code) or slots >= SLOTS or best.get(j, SLOTS) <= slots:
                    continue
                best[j] = slots
                op, _, rest = code[j].partition(" ")
                if op == "s_nop":
                    todo += [(x, slots + int(rest) + 1) for x in after(j)]
                    continue
                # a matrix instruction that adds to the same registers may follow at once; its other operands may not be they
                touched = _registers(",".join(rest.split(", ")[1:3]) if op.startswith("v_mfma") else rest)
                if not op.startswith("s_") and touched & result:
                    found.append((line, code[j], slots))
                    continue
                todo += [(x, slots + 1) for x in after(j)]
    return total, found


def test_the_check_finds_an_early_read_behind_a_branch():
    text = """
_Zk:
	v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], 0
	s_cbranch_scc1 .L2
	s_nop 7
.L1:
	v_add_f32_e32 v20, v1, v21
	s_endpgm
.L2:
	v_mov_b32_e32 v30, v31
	s_branch .L1
.Lfunc_end0:
"""
    total, found = early_reads(text)
    assert total == 1 and [(r, s) for _, r, s in found] == [("v_add_f32_e32 v20, v1, v21", 3)]
    assert early_reads(text.replace("v_mov_b32_e32 v30, v31", "s_nop 6"))[1] == []


def test_no_matrix_result_is_read_early():
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "device.s")
        flags = [f for f in binding.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
        source = os.path.join(os.path.dirname(binding.__file__), "csrc", "c2t_lib.hip")
        r = subprocess.run(["hipcc"] + flags + ["-S", "--offload-device-only", "-I", os.path.join(os.path.dirname(os.path.dirname(binding.__file__)), "include"), source, "-o", out],
                           stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout
        with open(out) as f:
            total, found = early_reads(f.read())
    assert total > 500 and not found, found[:5]
