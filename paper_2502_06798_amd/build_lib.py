"""Build libapc.so (gfx950) in-tree with hipcc.

Each source compiles to an object in parallel, then one link step.  Always
compiles when called; the binding only loads what is built.
"""
from __future__ import annotations

import concurrent.futures
import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libapc.so")
BUILD = os.path.join(HERE, "_build")
SOURCES = ["apc.cpp", "rowfactor.hip", "match.hip", "tile.hip", "tile_f32.hip", "tile_f16.hip", "tile_bf16.hip", "tile_e4m3.hip", "qs.hip", "qs_f16.hip", "qs_bf16.hip", "qs_e4m3.hip", "qs8_f16.hip", "qs8_bf16.hip", "qs8_e4m3.hip", "assign.hip", "gather.hip", "resident.hip", "shards.hip", "quantize.hip", "f32small.hip", "norm.hip", "kv.hip", "attend.hip", "rotate.hip", "prompt.hip", "prompt_f16.hip", "prompt_bf16.hip", "prompt_e4m3.hip"]

# Kernels in these sources load into LDS with asm and wait for those loads by
# counting vector-memory operations themselves; a register spill would add
# scratch loads to the count, so their code must not use scratch memory.
COUNTED = ["qs_f16.hip", "qs_bf16.hip", "qs_e4m3.hip", "qs8_f16.hip", "qs8_bf16.hip", "qs8_e4m3.hip"]
# The tiled kernel counts too, but waits until at most so many operations are
# outstanding as it knows to be newer than what it needs: operations that the
# compiler adds only make a wait longer.  Its tiles of 256 queries spill a few
# registers (bytes per lane, the other tiles none); more would cost time.  The
# attention kernels use none, the norm's those of float32 rows beyond 16,384.
SCRATCH = {"tile_f32.hip": 0, "tile_f16.hip": 24, "tile_bf16.hip": 24, "tile_e4m3.hip": 12, "attend.hip": 0, "norm.hip": 240,
           "prompt_f16.hip": 0, "prompt_bf16.hip": 0, "prompt_e4m3.hip": 0}

# Kernels in these sources keep values of every lane in registers across
# branches that only some lanes take.  Where registers are short the compiler
# may move such a value to another place inside the branch, and the other lanes'
# is lost; so no kernel may write an accumulation register or scratch memory there.
ALL_LANES = ["attend.hip", "prompt_f16.hip", "prompt_bf16.hip", "prompt_e4m3.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         # no packed fp32 instructions: hipcc would otherwise form them from plain float code
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # MFMA results in VGPRs: no copies of the accumulators between register files
         "-mllvm", "-amdgpu-mfma-vgpr-form"]
# Per-source additions.  The query-stationary kernels keep their per-lane lists
# as separate registers: promoted to one vector, a list is copied whole on
# every pass of the insertion loop.
SOURCE_FLAGS = {src: ["-mllvm", "-disable-promote-alloca-to-vector"]
                for src in ("qs_f16.hip", "qs_bf16.hip", "qs_e4m3.hip", "qs8_f16.hip", "qs8_bf16.hip", "qs8_e4m3.hip")}


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, *SOURCE_FLAGS.get(src, []), "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    return obj


def masked_moves(asm: str) -> list:
    """The instructions of a kernel's assembly that write an accumulation register or scratch memory where the
    execution mask may be narrowed: followed along the branches with the masks saved and not yet restored (where two
    ways meet, the longer list)."""
    blocks, order, name, n = {"": []}, [""], "", 0
    for line in asm.split("\n"):
        label = re.match(r"(\.LBB\w+):", line)
        line = line.split(";")[0].strip()
        if label or re.match(r"s_c?branch|s_endpgm", blocks[name][-1] if blocks[name] else ""):
            n += 1
            name = label.group(1) if label else f"after {n}"
            blocks[name] = []
            order.append(name)
        if line and not label and not line.startswith("."):
            blocks[name].append(line)
    saved_at, todo, found = {"": ()}, [""], set()
    while todo:
        name = todo.pop()
        saved, copy, ways, on = list(saved_at[name]), "?", [], True
        for line in blocks[name]:
            if m := re.match(r"s_(\w+)_saveexec_b64 (\S+),", line):
                if m.group(1) != "or":                          # (or: the other side of the same branch)
                    saved.append(m.group(2))
            elif m := re.match(r"s_mov_b64 (\S+), exec$", line):
                copy = m.group(1)
            elif line.startswith("s_mov_b64 exec,"):
                saved.append(copy)
            elif m := re.match(r"s_or_b64 exec, exec, (\S+)", line):
                saved = saved[:saved.index(m.group(1))] if m.group(1) in saved else saved[:-1]
            elif m := re.match(r"s_(c?)branch\S* (\.LBB\w+)", line):
                ways.append((m.group(2), tuple(saved)))
                on = bool(m.group(1))
            elif line.startswith("s_endpgm"):
                on = False
            elif saved and re.match(r"v_accvgpr_(write|mov)|scratch_", line):
                found.add(line)
        after = order.index(name) + 1
        if on and after < len(order):
            ways.append((order[after], tuple(saved)))
        for way, masks in ways:
            # (a loop that saves a mask each time round ends with 64)
            if way in blocks and (way not in saved_at or len(saved_at[way]) < len(masks) <= 64):
                saved_at[way] = masks
                todo.append(way)
    return sorted(found)


def _check_kernels(src: str) -> None:
    asm = os.path.join(BUILD, os.path.splitext(src)[0] + ".s")
    cmd = [HIPCC, *FLAGS, *SOURCE_FLAGS.get(src, []), "--cuda-device-only", "-S", "-x", "hip",
           os.path.join(CSRC, src), "-o", asm]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc -S failed for {src}:\n{r.stderr}")
    text, most = open(asm).read(), SCRATCH.get(src, 0)
    bad = [(m.group(1), int(m.group(2))) for m in re.finditer(
        r"\.amdhsa_kernel (\S+)(?:.|\n)*?\.amdhsa_private_segment_fixed_size (\d+)", text) if int(m.group(2)) > most]
    if bad:
        raise RuntimeError(f"{src}: kernels using more than {most} bytes of scratch memory per lane"
                           f"{'' if src in SCRATCH else ' (their LDS-load waits would be wrong)'}: {bad}")
    if src in ALL_LANES:
        kernels = re.findall(r"\n(_Z\S+):[^\n]*\n((?:.|\n)*?)\n\.Lfunc_end", text)
        bad = [(name, moves[:4]) for name, body in kernels if (moves := masked_moves(body))]
        if bad or not kernels:
            raise RuntimeError(f"{src}: moves to accumulation registers or scratch memory that only some lanes do: {bad}")


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=8) as ex:
        checks = [ex.submit(_check_kernels, src) for src in [*COUNTED, *SCRATCH]]
        objs = list(ex.map(_compile, SOURCES))
        for c in checks:
            c.result()
    tmp = OUT + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, OUT)
    if verbose:
        print(f"built {OUT}")
    return OUT


# Host code of the library (argument checks, tables, the host planner) under
# AddressSanitizer and UndefinedBehaviorSanitizer: apc.cpp compiled with the
# sanitizers on its host side only, linked with the other objects of the
# normal build (their device code is unchanged).
SAN_HOST = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
            "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer",
            "-Xarch_host", "-g"]


def build_sanitized(out_dir: str) -> str:
    """libapc.so in out_dir with apc.cpp's host code instrumented; needs a
    normal build's objects (build() first)."""
    os.makedirs(out_dir, exist_ok=True)
    obj = os.path.join(out_dir, "apc_san.o")
    cmd = [HIPCC, *FLAGS, *SAN_HOST, "-x", "hip", "-c", os.path.join(CSRC, "apc.cpp"), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for the sanitized apc.cpp:\n{r.stderr}")
    objs = [obj] + [os.path.join(BUILD, os.path.splitext(src)[0] + ".o") for src in SOURCES if src != "apc.cpp"]
    out = os.path.join(out_dir, "libapc.so")
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-shared-libasan", *SAN_HOST, "-o", out, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    if r.returncode != 0:
        raise RuntimeError(f"sanitized link failed:\n{r.stderr}")
    return out


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
