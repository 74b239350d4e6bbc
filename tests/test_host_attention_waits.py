"""Copies from memory into LDS that attention's kernels start, on the path of every branch (compiled for the device here, no GPU needed): none is on its way when a
workgroup ends, whose LDS may be another one's from then on."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1810_08723_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARGS = "const AttentionArgs, uint32_t"
KERNELS = {
    "rows": ("attention_forward.hpp", [f"attention_rows_kernel<{t}, {d}, true, {w}, {k}>({ARGS})" for t, d, w, k in (("f16", 128, 8, 64), ("bf16", 64, 4, 64), ("float", 128, 4, 32))]),
    "queries": ("attention_backward.hpp", [f"attention_queries_kernel<{t}, {d}, true, 4, {k}>({ARGS}, f32x2 *, f32x2 *)" for t, d, k in (("f16", 128, 64), ("bf16", 64, 64), ("float", 64, 32))]),
    "keys": ("attention_backward.hpp", [f"attention_keys_kernel<{t}, {d}, true, {w}>({ARGS}, const f32x2 *, const f32x2 *)" for t, d, w in (("f16", 128, 8), ("bf16", 80, 8), ("float", 128, 4))]),
}


def on_their_way(lines):
    """Lines of an end of the program that some path reaches with a copy into LDS that it has not waited for, and copies in all.  Of a path are known the last pair of scalar
    registers that it set to 0 or -1 as a whole, which is how the compiler says where a branch came from, and what a branch on it does"""
    labels = {line[:-1]: i for i, line in enumerate(lines) if line.endswith(":")}
    todo, seen, ends = [(0, False, None, None)], set(), set()
    while todo:
        at, out, pair, vcc = todo.pop()
        while (at, out, pair, vcc) not in seen and at < len(lines):
            seen.add((at, out, pair, vcc))
            words = lines[at].replace(",", " ").split()
            name = words[0]
            assert not name.startswith(("s_setpc", "s_swappc", "s_call")), lines[at]
            if re.match(r"(global|buffer)_load_\w*lds", name) or (name.startswith("buffer_load") and "lds" in words):
                out = True
            elif name == "s_waitcnt" and "vmcnt(0)" in words:
                out = False
            elif name in ("s_cbranch_vccz", "s_cbranch_vccnz") and vcc is not None:
                if vcc == (name == "s_cbranch_vccnz"):
                    at = labels[words[1]]
                    continue
            elif name.startswith("s_cbranch"):
                todo.append((labels[words[1]], out, pair, vcc))
            elif name == "s_branch":
                at = labels[words[1]]
                continue
            elif name == "s_endpgm":
                ends |= {at} if out else set()
                break
            elif name in ("s_and_b64", "s_andn2_b64") and words[1:3] == ["vcc", "exec"] and pair and pair[0] == words[3]:
                vcc = pair[1] == (name == "s_and_b64")          # (some lane is there)
                at += 1
                continue
            if "vcc" in words[1:2] or name.startswith("v_cmp") or len(words) > 2 and words[2] == "vcc":
                vcc = None
            if name == "s_mov_b64" and words[2] in ("0", "-1"):
                pair = (words[1], words[2] == "-1")
            elif pair and words[1:] and touches(words, pair[0]):
                pair = None
            at += 1
    return sorted(ends), sum(re.match(r"global_load_lds", line) is not None for line in lines)


def touches(words, pair):
    """Whether a scalar register of the pair may be written: where it is among the first two operands"""
    own = {int(n) for n in re.findall(r"\d+", pair)}
    for w in words[1:3]:
        m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)", w)
        if m and own & (set(range(int(m[1]), int(m[2]) + 1)) if m[1] else {int(m[3])}):
            return True
    return False


def test_the_search_itself():
    load, wait, end = "global_load_lds_dwordx4 v[0:1], off", "s_waitcnt vmcnt(0) lgkmcnt(0)", "s_endpgm"
    assert on_their_way([load, wait, end]) == ([], 1)
    assert on_their_way([load, "s_waitcnt lgkmcnt(0)", end]) == ([2], 1)
    assert on_their_way([load, "s_cbranch_scc1 .L1", wait, ".L1:", end]) == ([4], 1)
    assert on_their_way(["s_cbranch_scc1 .L1", load, wait, ".L1:", end]) == ([], 1)
    assert on_their_way([".L0:", wait, load, "s_cbranch_scc1 .L0", end]) == ([4], 1)
    assert on_their_way(["s_branch .L1", ".L0:", end, ".L1:", load, "s_branch .L0"]) == ([2], 1)
    known = ["s_mov_b64 s[4:5], -1", "s_and_b64 vcc, exec, s[4:5]", "s_cbranch_vccz .L1", wait, ".L1:", end]
    assert on_their_way([load] + known) == ([], 1)
    assert on_their_way([load, known[0], "s_load_dwordx2 s[4:5], s[0:1], 0x0"] + known[1:]) == ([7], 1)
    assert on_their_way([load] + known[:2] + ["v_cmp_eq_u32_e32 vcc, 0, v0"] + known[2:]) == ([7], 1)
    assert on_their_way([load, "s_mov_b64 s[4:5], 0"] + known[1:]) == ([6], 1)


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
@pytest.mark.parametrize("which", list(KERNELS))
def test_copies_have_arrived_before_the_end(which, tmp_path):
    from paper_1810_08723_amd.build import COMMON
    header, kernels = KERNELS[which]
    made = " ".join(f"template __global__ void {k};" for k in kernels)
    source, listing = tmp_path / "kernels.hip", tmp_path / "kernels.s"
    source.write_text(f'#include "{os.path.join(CSRC, header)}"\nnamespace ocn {{ namespace {{ {made} }} }}\n')
    r = subprocess.run([HIPCC, *COMMON, "--cuda-device-only", "-S", "-x", "hip", str(source), "-o", str(listing)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    found, lines = {}, None
    for line in listing.read_text().splitlines():
        line = line.split(";")[0].strip()
        kernel = re.match(r"(_Z\w*attention_\w+_kernel\w*):$", line)
        if kernel:
            lines = found[kernel.group(1)] = []
        elif line.startswith(".Lfunc_end") or line.startswith(".section"):
            lines = None
        elif lines is not None and line and (line.endswith(":") or not line.startswith(".")):
            lines.append(line)
    found = {name: lines for name, lines in found.items() if f"attention_{which}" in name}
    assert len(found) == len(kernels)
    for lines in found.values():       # (a copy may follow a scalar instruction's result after one wait, a vector instruction's only after five)
        assert all(line.startswith("s_") for line in lines if re.match(r"\w+ m0\b", line))
    found = {name: on_their_way(lines) for name, lines in found.items()}
    for name, (ends, copies) in found.items():
        assert copies > 0 and not ends, (name, copies, ends)


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
@pytest.mark.parametrize("copy", ["load_to_lds", "load_word_to_lds"])
def test_copies_say_that_they_set_their_place(copy, tmp_path):
    """The compiler, which keeps the register of a copy's place in LDS from one of its own copies to the next, sets it again behind one of these"""
    from paper_1810_08723_amd.build import COMMON
    source, listing = tmp_path / "kernel.hip", tmp_path / "kernel.s"
    source.write_text(f'''#include "{os.path.join(CSRC, "attention_tiles.hpp")}"
namespace ocn {{
typedef __attribute__((address_space(1))) const uint32_t *Global;
typedef __attribute__((address_space(3))) uint32_t *Lds;
extern "C" __global__ void three_copies(const uint32_t *from, uint32_t *to, uint32_t at) {{
  __shared__ __align__(16) uint32_t held[1024];
  __builtin_amdgcn_global_load_lds((Global)from, (Lds)held, 4, 0, 0);
  {copy}(lds_address((const char *)held) + at, (const char *)from);
  __builtin_amdgcn_global_load_lds((Global)(from + 64), (Lds)held, 4, 0, 0);
  arrived();
  to[threadIdx.x] = held[threadIdx.x];
}}
}}
''')
    r = subprocess.run([HIPCC, *COMMON, "--cuda-device-only", "-S", "-x", "hip", str(source), "-o", str(listing)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    body = listing.read_text().split("three_copies:")[1].split(".Lfunc_end")[0]
    order = [m[1] for m in re.finditer(r"^\s*(s_mov_b32 m0|global_load_lds)", body, flags=re.M)]
    assert order == ["s_mov_b32 m0", "global_load_lds"] * 3
