"""Turns the training operators' CUDA sources into C++ that runs on the host (emulation.h): inline PTX becomes calls, shared
memory a block's arena, launches loops over clusters.  The kernels' own code stays as it is."""
from __future__ import annotations

import os
import re

FILES = ("device_utils.cuh", "train_common.cuh", "train_rows.cuh", "kernels_norm.cu", "kernels_xent.cu")
CTYPES = {"f32": "float", "f16": "__half", "bf16": "__nv_bfloat16"}


def _closing(s, i, opening="(", closing=")"):
    """Index of the bracket that closes the one at i (strings are passed over)."""
    depth, quoted = 0, False
    while True:
        c = s[i]
        if quoted:
            if c == "\\":
                i += 1
            elif c == '"':
                quoted = False
        elif c == '"':
            quoted = True
        elif c == opening:
            depth += 1
        elif c == closing:
            depth -= 1
            if depth == 0:
                return i
        i += 1


def _split(s, sep):
    """s at every sep outside brackets and strings."""
    out, depth, cur, quoted, i = [], 0, "", False, 0
    while i < len(s):
        c = s[i]
        if quoted:
            cur += c
            if c == "\\":
                i += 1
                cur += s[i]
            elif c == '"':
                quoted = False
        elif c == sep and depth == 0:
            out.append(cur)
            cur = ""
        else:
            quoted = c == '"'
            depth += (c in "([{") - (c in ")]}")
            cur += c
        i += 1
    return out + [cur]


def _ptx(s):
    """asm volatile("name ..." : outputs : inputs) -> emu::op_name(outputs, inputs)"""
    while True:
        m = re.search(r"\basm\s*(volatile)?\s*\(", s)
        if not m:
            return s
        end = _closing(s, m.end() - 1)
        body = s[m.end():end]
        strings = re.match(r'\s*((?:"(?:\\.|[^"\\])*"\s*)+)', body)
        text = "".join(re.findall(r'"((?:\\.|[^"\\])*)"', strings.group(1)))
        rest = body[strings.end():].replace("::", ": :")
        lists = [p.strip() for p in _split(rest, ":")][1:] if rest.strip() else []
        operands = [re.match(r'"[^"]*"\s*\((.*)\)$', o.strip(), re.S).group(1) for p in lists[:2] for o in _split(p, ",") if o.strip()]
        name = next((n for n, mark in (("try_wait", "mbarrier.try_wait"), ("cluster_barrier", "barrier.cluster.arrive"),
                                       ("cluster_rank", "cluster_ctarank")) if mark in text), None)
        name = name or re.sub(r"\W", "_", text.split()[0].rstrip(";"))
        s = s[:m.start()] + f"emu::op_{name}({', '.join(operands)})" + s[end + 1:]


class _Shared:
    """__shared__ declarations -> references into the block's arena"""

    def __init__(self):
        self.count = 0

    def one(self, m):
        self.count += 1
        declared = m.group(1)
        if "<" in declared:                                          # (a > outside brackets closes no template here)
            at = declared.rindex(">") + 1
            kind, names = declared[:at], declared[at:]
        else:
            kind, names = declared.split(None, 1)
        ids = [re.match(r"\s*(\w+)", n).group(1) for n in _split(names, ",")]
        k = self.count
        return (f"struct emuS{k} {{ {kind} {names}; }}; auto& emus{k} = *(emuS{k}*)emu::shared({k}, sizeof(emuS{k})); "
                + " ".join(f"auto& {i} = emus{k}.{i};" for i in ids))

    def __call__(self, s):
        s = re.sub(r"extern __shared__ __align__\(128\) unsigned char (\w+)\[\];",
                   r"unsigned char* \1 = (unsigned char*)emu::shared(0, emu::dynamic_bytes());", s)
        return re.sub(r"__shared__ ([^;]+);", self.one, s)


def _launches(s):
    """kernel<<<grid, threads, ...>>>(arguments) -> emu::launch_plain(kernel, grid, threads, arguments)"""
    while "<<<" in s:
        i = s.index("<<<")
        j = s.index(">>>", i)
        end = _closing(s, j + 3)
        b = i
        if s[b - 1] == ">":
            depth = 0
            while True:
                b -= 1
                depth += (s[b] == ">") - (s[b] == "<")
                if depth == 0:
                    break
        while re.match(r"\w", s[b - 1]):
            b -= 1
        grid, threads = _split(s[i + 3:j], ",")[:2]
        s = s[:b] + f"emu::launch_plain({s[b:i]}, dim3({grid}), {threads}, {s[j + 4:end]})" + s[end + 1:]
    return s


def _cut(s, begin, end, instead):
    a = s.index(begin)
    return s[:a] + instead + s[s.index(end, a):]


def translate(csrc, header, out, only, polls=None):
    """Writes the translated sources of one element type to the folder `out`; polls: the limit of a wait for a row and of the one after it."""
    shared = _Shared()
    for name in FILES:
        with open(os.path.join(csrc, name)) as f:
            s = f.read()
        s = s.replace('#include "../../include/gem_nlr.h"', f'#include "{header}"')
        if name == "train_rows.cuh":
            s = _cut(s, "// Groups of C blocks of kernel K", "// Clusters (or blocks) to launch for n rows",
                     "template <auto K, int C> int resident_clusters(int) { return emu::resident; }\n")
            s = _cut(s, "// Launch of `blocks` blocks", "}  // namespace gemnlr", "using emu::launch_rows;\nusing emu::launch_early;\n")
            if polls:
                s, n = re.subn(r"kPolls = [^,]+, kLandPolls = [^,]+,", f"kPolls = {polls[0]}, kLandPolls = {polls[1]},", s)
                assert n == 1
        if name == "train_common.cuh":
            s = _cut(s, "template <typename F> inline int by_type", "constexpr int kTrainSMs",
                     f"template <typename F> inline int by_type(int32_t, F f) {{ return f({CTYPES[only]}{{}}); }}\n")
        if name.endswith(".cu"):
            s = s.replace("by_type(wtype,", "emu::by_weight_type(wtype,")
        if name != "device_utils.cuh":
            s = _launches(shared(_ptx(s)))
        with open(os.path.join(out, name), "w") as f:
            f.write(s)
    with open(os.path.join(out, "all.cpp"), "w") as f:
        f.write('#include <cuda_runtime.h>\n#include <cuda_bf16.h>\n#include <cuda_fp16.h>\n#include "emulation.h"\n'
                "namespace emu { template <typename F> int by_weight_type(int w, F f) { if (w == 0) return f(float{}); "
                f"return f({CTYPES[only]}{{}}); }} }}\n" + '#include FILE_UNDER_TEST\n#include "entries.h"\n')
