"""Where a kernel lets the next one of its stream launch, read from the sources:
after its loads and stores, or, in the kernels named here, between its main loop
and the stores of what that loop left in registers or TMEM."""

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2404_08573_gb300", "csrc")
# kernel: what is still to come after its signal
NAMED = {
    "ff_gemm_tc_body.inc": "the epilogue: the main loop's products are done",
    "k_fp8_pair": "the stores of the pair's last tile",
    "k_fp8_split": "the exchange of partial sums and the stores; TMEM is handed back",
    "k_fp4_pair": "the stores of the pair's last tile",
    "k_fp4_split": "the exchange of partial sums and the stores; TMEM is handed back",
    "k_rms_grad": "the stores of one block's sums, which the next kernel folds",
}


def signals():
    """(file, enclosing kernel, the rest of its body) of every signal."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        name = os.path.basename(path)
        text = re.sub(r"//[^\n]*", "", open(path).read())
        if name == "ff_ptx.cuh":
            continue
        for m in re.finditer(r"griddep_launch_dependents\(\)\s*;", text):
            if name.endswith(".inc"):
                yield name, name, text[m.end():]
                continue
            start = text.rindex("__global__", 0, m.start())
            kernel = re.search(r"\b(k_\w+)\s*\(", text[start:]).group(1)
            depth, end = 0, text.index("{", start + text[start:].index(kernel))
            while True:
                depth += {"{": 1, "}": -1}.get(text[end], 0)
                if depth == 0:
                    break
                end += 1
            assert end > m.start(), f"{name}: a signal outside a kernel"
            yield name, kernel, text[m.end():end]


def test_signals_come_after_a_kernels_work():
    seen = set()
    for name, kernel, rest in signals():
        seen.add(kernel)
        if kernel not in NAMED:
            assert not re.sub(r"[{}\s]|return;", "", rest), f"{name}: {kernel} signals before {rest.strip()[:60]!r}"
    assert seen >= set(NAMED), "a kernel named here does not signal any more"
