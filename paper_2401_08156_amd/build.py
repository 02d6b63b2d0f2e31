"""Compile the HIP library for gfx950 in-tree (hipcc cross-compiles without a GPU)."""
import os
import subprocess
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libvmsreplay.so")
EXT = os.path.join(_HERE, "_vms_torch.so")       # the operators' autograd nodes (host code), linked against LIB
EXT_SOURCE = "vms_torch_ops.cpp"
SOURCES = ["vms_replay.hip", "vms_demo.hip", "vms_live.hip", "vms_peaks.hip"]
OPS_SOURCES = ["vms_dropout.hip", "vms_norm.hip", "vms_lowrank.hip"]
HEADERS = ["ops_common.hpp", "../../include/vms_ops.h", "wave_hw.hpp", "wave_ops.hpp", "replay_plan.hpp", "replay_kernels.hpp", "replay_fine.hpp", "selftest.hpp", "../../include/vms_replay.h", "../../include/vms_live.h"]

# The replay loops branch on wave-uniform conditions only (whatever would switch lanes off is written
# with selects or kept in non-inlined functions).  With the option below LLVM leaves such regions as
# they are instead of rebuilding them around exec-mask style flow blocks: fewer branches per event.
HIPCC_FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-shared", "-fPIC", "-Wall",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-mllvm", "-structurizecfg-skip-uniform-regions=1",
               "-mllvm", "-align-all-nofallthru-blocks=6",      # branch targets on 64-byte lines: measured 2 % faster
               # one wavefront per SIMD and trace: schedule for latency (instruction-level parallelism inside the
               # wave), not for occupancy; measured 3 % (stitching) and 8 % (splitting kernel) faster
               "-mllvm", "-amdgpu-sched-strategy=max-ilp", "-mllvm", "-enable-post-misched=0",
               # no lifetime markers for locals: with them every `continue` out of a scope that holds a local
               # whose address was taken goes through a shared clean-up block and a switch on where to go next,
               # which LLVM does not thread away in these kernels (one flag test and two branches per event)
               "-Xclang", "-disable-lifetime-markers",
               "-Wno-inline-asm"]       # write_lane() names m0, which the compiler reserves but does not use here

# The operators' kernels are loops over wide tensors: the compiler's own scheduling, for many wavefronts a SIMD.
OPS_FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-shared", "-fPIC", "-Wall",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _torch():
    """PyTorch, or None where it is not installed: the library does not need it, the autograd nodes do."""
    try:
        import torch
    except ImportError:
        return None
    return torch


def _stale():
    built = [LIB] if _torch() is None else [LIB, EXT]
    if not all(os.path.exists(f) for f in built):
        return True
    t = min(os.path.getmtime(f) for f in built)
    deps = [os.path.join(CSRC, s) for s in SOURCES + OPS_SOURCES + [EXT_SOURCE] + HEADERS]
    return any(os.path.exists(d) and os.path.getmtime(d) > t for d in deps)


def build(force=False, save_temps_dir=None):
    """Build libvmsreplay.so and, where PyTorch is installed, _vms_torch.so next to this file; returns the library's path."""
    if not force and not _stale():
        return LIB
    jobs = [(s, flags) for group, flags in ((SOURCES, HIPCC_FLAGS), (OPS_SOURCES, OPS_FLAGS)) for s in group]
    if save_temps_dir:
        os.makedirs(save_temps_dir, exist_ok=True)
    with tempfile.TemporaryDirectory() as objects:
        def compile_one(job):
            source, flags = job
            obj = os.path.join(objects, source + ".o")
            cmd = ["hipcc"] + [f for f in flags if f != "-shared"] + ["-c", os.path.join(CSRC, source), "-o", obj]
            return obj, _run(cmd + ["--save-temps"] * bool(save_temps_dir), save_temps_dir or CSRC)
        ext, out = os.path.join(objects, EXT_SOURCE + ".o"), []
        with ThreadPoolExecutor(4) as pool:
            node = _torch() and pool.submit(_run, _ext_command() + ["-c", os.path.join(CSRC, EXT_SOURCE), "-o", ext], CSRC)
            done = list(pool.map(compile_one, jobs))
            out += [text for _, text in done]
            out.append(_run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + [obj for obj, _ in done], CSRC))
            if node:
                out.append(node.result())
                out.append(_run(["g++", "-shared", "-o", EXT, ext, "-L" + _torch_dir("lib"), "-L" + _HERE, "-l:" + os.path.basename(LIB),
                                 "-Wl,-rpath,$ORIGIN"] + ["-l" + l for l in ("c10", "c10_hip", "torch", "torch_cpu", "torch_python")], CSRC))
            else:
                out.append("no PyTorch: " + os.path.basename(EXT) + " (the operators for its tensors) is not built")
    out = "\n".join(text for text in out if text.strip())
    if out:
        print(out)
    return LIB


def _torch_dir(*parts):
    import torch
    return os.path.join(os.path.dirname(torch.__file__), *parts)


def _ext_command():
    """g++ with PyTorch's headers; HIP's own ask for the platform's name when another compiler reads them."""
    import torch
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1", "-DTORCH_API_INCLUDE_EXTENSION_H",
            "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
            "-isystem", _torch_dir("include"), "-isystem", _torch_dir("include", "torch", "csrc", "api", "include"),
            "-isystem", sysconfig.get_paths()["include"], "-isystem", "/opt/rocm/include"]


def _run(cmd, cwd):
    """The command's own words; raises where it fails."""
    r = subprocess.run(cmd, cwd=cwd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(cmd[0] + " failed:\n" + out)
    return out
