"""Compiled code of the products by kind of row and of orthogonalise: the rules of the gated block's kernels (tests/test_layer_codeobj.py)."""
import re
import subprocess

from tests.test_layer_codeobj import OBJDUMP, kernels, objects  # noqa: F401

MINE = ("k_grouped_", "k_orth_")


def test_products(objects):  # noqa: F811
    """No kernel keeps values in private memory, and one that keeps them in accumulation registers has no lane-conditional code before its sums are
    complete."""
    seen = relocating = 0
    for path in objects:
        found = {k: v for k, v in kernels(path).items() if any(m in k for m in MINE)}
        if not found:
            continue
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], capture_output=True, text=True, check=True).stdout
        for block in re.split(r"\n(?=[0-9a-f]+ <)", text):
            m = re.match(r"[0-9a-f]+ <([^>]+)>:", block)
            if not m or m.group(1) not in found:
                continue
            seen += 1
            name, (agprs, private) = m.group(1), found[m.group(1)]
            ins = [line.strip() for line in block.splitlines()[1:] if line.strip()]
            assert private == 0, name
            assert not any(i.startswith(("v_pk_add_f32", "v_pk_mul_f32", "v_pk_fma_f32")) for i in ins), name
            if agprs == 0:
                continue
            relocating += 1
            products = [j for j, i in enumerate(ins) if "mfma" in i]
            writes = [i for i in ins[:products[-1]] if "saveexec" in i or re.match(r"(s_\w+|v_cmpx\w*) exec\b", i)]
            assert not writes, (name, writes[:3])
    assert seen > 60 and relocating > 0
