"""Builds the sources of rotary positions and of the cache's budget for the host, as host_wave.py does those of the cache itself, with host_layers/hip/hip_runtime.h in the place of HIP's own header."""
import ctypes
import os
import re
import shutil
import subprocess

import torch

import host_wave
from host_wave import CLANG, CSRC, REPORTS, ROOT, Memory

SOURCES = ["apmm_api_budget.hip", "apmm_rotary.hip", "apmm_budget_weights.hip", "apmm_budget_evict.hip"]
HEADERS = ["apmm_api.h", "apmm_budget.h", "apmm_rotary.h"]


def on_host(text):
    text = re.sub(r'asm\("v_max3_f32 %0, %1, %2, %3" : "=v"\((\w+)\) : "v"\((\w+)\), "v"\((\w+)\), "v"\((\w+)\)\);', r"\1 = fmaxf(fmaxf(\2, \3), \4);", text)
    text = re.sub(r'asm\("v_and_or_b32 %0, %1, %2, %3" : "=v"\((\w+)\) : "v"\((\w+)\), "s"\((\w+)\), "v"\((\w+)\)\);', r"\1 = (\2 & \3) | \4;", text)
    text = re.sub(r'(if \(R > 1\) )?asm volatile\("" ::? [^;]*\);', "", text)
    text = re.sub(r'(if \(R > 1\) )?asm volatile\("" ::: "memory"\);', "", text)
    text = re.sub(r"(\w+(?:<[\w, ]+>)?)<<<(\w+), (dim3\([^()]*\)|\w+), 0, stream>>>\(((?:[^()]|\([^()]*\))*)\)", r"host_layers::launch(\2, \3, [&] { \1(\4); })", text)
    return host_wave.on_host(text)


def build(folder):
    here = os.path.join(str(folder), "package", "csrc")
    shutil.copytree(os.path.join(ROOT, "include"), os.path.join(str(folder), "include"), dirs_exist_ok=True)
    os.makedirs(here, exist_ok=True)
    for name in os.listdir(CSRC):
        if name in SOURCES + HEADERS or (name.startswith("apmm_kv") and name.endswith(".h")):
            with open(os.path.join(CSRC, name)) as f, open(os.path.join(here, name), "w") as g:
                g.write(on_host(f.read()))
    with open(os.path.join(here, "reports.cpp"), "w") as f:
        f.write(REPORTS)
    flags = [CLANG, "-O2", "-std=c++17", "-mf16c", "-mfma", "-ffp-contract=off", "-fPIC", "-w", "-I", os.path.join(ROOT, "tests", "host_layers"), "-I", here]
    running = [(name, subprocess.Popen(flags + ["-x", "c++", "-c", os.path.join(here, name), "-o", os.path.join(here, name + ".o")], stderr=subprocess.PIPE, text=True))
               for name in SOURCES + ["reports.cpp"]]
    for name, p in running:
        err = p.communicate()[1]
        assert p.returncode == 0, name + ": " + err[-3000:]
    to = os.path.join(str(folder), "liblayers_host.so")
    subprocess.run(flags + ["-shared"] + [os.path.join(here, name + ".o") for name, _ in running] + ["-o", to], check=True, capture_output=True, text=True)
    return to


class Host(host_wave.Host):
    """The calls on tensors of the host, each in a child process."""

    def __init__(self, path):
        from paper_2409_17870_amd import binding
        self.binding, lib = binding, ctypes.CDLL(path)
        vp, i64, ci, cf = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
        cache, batch, rotation, rows = ctypes.POINTER(binding.ApmmKvCache), ctypes.POINTER(binding.ApmmKvBatch), ctypes.POINTER(binding.ApmmRotation), [vp, i64, i64]
        lib.apmm_rotary.argtypes = [i64, ci, ci, ci] + rows + [vp, rotation, ci] + rows + [vp]
        lib.apmm_kv_write_rotary.argtypes = [cache, batch, ci, vp, rotation] + rows * 4 + [vp]
        lib.apmm_kv_weights.argtypes = [cache, batch, ci] + rows + [vp, i64, i64, i64, cf, cf, i64, i64, vp, ctypes.c_size_t, vp]
        lib.apmm_kv_weights_workspace_bytes.argtypes, lib.apmm_kv_weights_workspace_bytes.restype = [cache, batch, ci], ctypes.c_size_t
        lib.apmm_kv_evict.argtypes = [cache, ci, vp, vp, i64, i64, vp, i64, i64, i64, i64, i64, i64, vp, i64, i64, vp, vp, vp, vp, ctypes.c_size_t, vp]
        lib.apmm_kv_evict_workspace_bytes.argtypes, lib.apmm_kv_evict_workspace_bytes.restype = [cache, ci, i64], ctypes.c_size_t
        self.lib = lib

    def rotation(self, frequencies, interleaved, magnitude):
        return self.binding.ApmmRotation(frequencies.data_ptr(), frequencies.shape[0], interleaved, magnitude)

    def rotary(self, x, positions, frequencies, interleaved=0, magnitude=1.0, inverse=0):
        out = Memory().empty(x.shape, x.dtype).fill_(float("nan"))
        self.call(self.lib.apmm_rotary, *x.shape, int(x.dtype == torch.bfloat16), x.data_ptr(), x.stride(0), x.stride(1), positions.data_ptr(),
                  self.rotation(frequencies, interleaved, magnitude), inverse, out.data_ptr(), out.stride(0), out.stride(1), None)
        return out.clone()

    def write_rotary(self, q, k, v, codes, scales, table, lengths, frequencies, starts=None, positions=None, interleaved=0, magnitude=1.0):
        out = Memory().empty(q.shape, q.dtype).fill_(float("nan"))
        rows = [x for t in (q, out, k, v) for x in (t.data_ptr(), t.stride(0), t.stride(1))]
        self.call(self.lib.apmm_kv_write_rotary, *self.structs(codes, scales, table, lengths, starts, k.shape[0]), q.shape[1], None if positions is None else positions.data_ptr(),
                  self.rotation(frequencies, interleaved, magnitude), *rows, None)
        return out.clone()

    def weights(self, q, codes, scales, table, lengths, w, starts=None, window=0, sinks=0, decay=1.0):
        cache, batch = self.structs(codes, scales, table, lengths, starts, q.shape[0])
        need = self.lib.apmm_kv_weights_workspace_bytes(cache, batch, q.shape[1])
        work = Memory().empty((need,), torch.uint8).fill_(0xff)
        self.call(self.lib.apmm_kv_weights, cache, batch, q.shape[1], q.data_ptr(), q.stride(0), q.stride(1), w.data_ptr(), w.stride(0), w.stride(1), w.shape[2], decay, q.shape[2] ** -0.5,
                  window, sinks, work.data_ptr(), need, None)
        return w

    def evict(self, codes, scales, table, lengths, w, budget, to, sinks=0, recent=0):
        cache, _ = self.structs(codes, scales, table, lengths, None, lengths.shape[0])
        m, shape = Memory(), (lengths.shape[0], scales.shape[1], budget)
        need = self.lib.apmm_kv_evict_workspace_bytes(cache, shape[0], table.shape[1])
        work = m.empty((need,), torch.uint8).fill_(0xff)
        kept, weights, n = m.empty(shape, torch.int32), m.empty(shape, torch.float32), m.empty(shape[:1], torch.int32)
        self.call(self.lib.apmm_kv_evict, cache, shape[0], lengths.data_ptr(), table.data_ptr(), table.stride(0), table.shape[1], w.data_ptr(), w.stride(0), w.stride(1), w.shape[2], budget, sinks,
                  recent, to.data_ptr(), to.stride(0), to.shape[1], n.data_ptr(), kept.data_ptr(), weights.data_ptr(), work.data_ptr(), need, None)
        return kept.clone(), weights.clone(), n.clone()
