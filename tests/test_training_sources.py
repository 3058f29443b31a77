"""What the training operators' CUDA sources have to promise the compiler, and may not."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_36074_b200", "csrc")
FILES = [os.path.basename(p) for p in sorted(glob.glob(os.path.join(CSRC, "kernels_*.cu"))) if "train_rows.cuh" in open(p).read()]


def functions(text):
    """{name: (is a kernel, parameters, body)}"""
    text = re.sub(r"//[^\n]*", "", text)
    found = {}
    for m in re.finditer(r"(__global__|__device__)[^;{}()]*(?:__launch_bounds__\([^()]*\)\s*)?\b(\w+)\s*\(([^()]*)\)\s*\{", text):
        depth, i = 1, m.end()
        while depth:
            depth += (text[i] == "{") - (text[i] == "}")
            i += 1
        found[m.group(2)] = (m.group(1) == "__global__", m.group(3), text[m.end():i])
    return found


def test_the_files_are_found():
    assert FILES == ["kernels_clip.cu", "kernels_norm.cu", "kernels_xent.cu"]
    early = [n for f in FILES for n, (kernel, _, body) in functions(open(os.path.join(CSRC, f)).read()).items() if kernel and "grid_ready()" in body]
    assert {"k_clip_norm", "k_clip_scale", "k_norm_dw_join", "k_xent_any", "k_xent_rows"} <= set(early)


@pytest.mark.parametrize("name", FILES)
def test_kernels_that_begin_early_promise_nothing_about_what_the_kernel_before_writes(name):
    """const T* __restrict__ says that nobody writes the data while the kernel runs, which lets the compiler read it before the
    kernel has waited; a kernel that begins while its forerunner still writes may not say so, nor its helpers."""
    found = functions(open(os.path.join(CSRC, name)).read())
    early = {n for n, (_, _, body) in found.items() if "grid_ready()" in body}
    reached = set(early)
    for n in early:
        reached |= {m for m in found if re.search(rf"\b{m}\b\s*[<(]", found[n][2])}
    written = {p for n, (kernel, params, _) in found.items() if kernel and n not in early
               for p in re.findall(r"(?<!const )\b\w+\*\s*(?:__restrict__\s+)?(\w+)", re.sub(r"const \w+\*\s*(?:__restrict__\s+)?\w+", "", params))}
    wrong = [(n, p) for n in sorted(reached) for p in re.findall(r"const \w+\*\s*__restrict__\s+(\w+)", found[n][1]) if p in written]
    assert not wrong
