"""Builds the sources of rotary positions, of the cache's budget and of the products with four-bit weights for the host, as host_wave.py does those of the cache itself, with
host_layers/hip/hip_runtime.h in the place of HIP's own header."""
import ctypes
import os
import re
import shutil
import subprocess

import torch

import host_wave
from host_wave import CLANG, CSRC, REPORTS, ROOT, Memory

SOURCES = ["apmm_api_budget.hip", "apmm_rotary.hip", "apmm_budget_weights.hip", "apmm_budget_evict.hip"]
PRODUCTS = ["apmm_api_w4.hip", "apmm_w4.hip", "apmm_w4_tiles.hip"]
HEADERS = ["apmm_api.h", "apmm_budget.h", "apmm_rotary.h", "apmm_w4.h"]


def replaced(text, *pairs):
    for was, by in pairs:
        assert text.count(was) == 1, was
        text = text.replace(was, by)
    return text


def loads_that_arrive_late(text):
    """apmm_w4_tiles.hip: its loads to LDS by hand, which arrive where the wave waits for so many that no more than those it names are on their way; every load counts, whoever waits for it."""
    return replaced(
        text,
        ('asm volatile("s_mov_b32 m0, %0\\n\\ts_nop 0\\n\\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(base) : "memory", "m0");', "host_layers::load_to_lds(lds, voff, base);"),
        ('asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\\n\\ts_barrier" ::"n"(N) : "memory");', "host_layers::arrive(N); __syncthreads();"),
        ("(uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4 *)&rows[0][0]", "host_layers::lds_begins(rows, sizeof(rows))"),
        ("auto load_weights = [&](int b, Weights &to) {", "auto load_weights = [&](int b, Weights &to) { host_layers::issued(2 + kGroups);"),
        ("for (int i = threadIdx.x; i < kTokens * 16; i += 64 * kWaves * H) {", "host_layers::arrive(0); for (int i = threadIdx.x; i < kTokens * 16; i += 64 * kWaves * H) {"))


def on_host(text):
    text = re.sub(r'asm\("v_max3_f32 %0, %1, %2, %3" : "=v"\((\w+)\) : "v"\((\w+)\), "v"\((\w+)\), "v"\((\w+)\)\);', r"\1 = fmaxf(fmaxf(\2, \3), \4);", text)
    text = re.sub(r'asm\("v_and_or_b32 %0, %1, %2, %3" : "=v"\((\w+)\) : "v"\((\w+)\), "s"\((\w+)\), "v"\((\w+)\)\);', r"\1 = (\2 & \3) | \4;", text)
    text = re.sub(r'(if \(R > 1\) )?asm volatile\("" ::? [^;]*\);', ";", text)
    text = re.sub(r'(if \(R > 1\) )?asm volatile\("" ::: "memory"\);', ";", text)
    text = re.sub(r"(\w+(?:<[\w, ]+>)?)<<<(.+?), (dim3\([^()]*\)|\w+), 0, stream>>>\(((?:[^()]|\([^()]*\))*)\)", r"host_layers::launch(\2, \3, [&] { \1(\4); })", text)
    return host_wave.on_host(text)


def build(folder, sources=SOURCES):
    here = os.path.join(str(folder), "package", "csrc")
    shutil.copytree(os.path.join(ROOT, "include"), os.path.join(str(folder), "include"), dirs_exist_ok=True)
    os.makedirs(here, exist_ok=True)
    for name in os.listdir(CSRC):
        if name in sources + HEADERS or (name.startswith("apmm_kv") and name.endswith(".h")):
            with open(os.path.join(CSRC, name)) as f, open(os.path.join(here, name), "w") as g:
                text = f.read()
                g.write(on_host(loads_that_arrive_late(text) if name == "apmm_w4_tiles.hip" else text))
    with open(os.path.join(here, "reports.cpp"), "w") as f:
        f.write(REPORTS)
    flags = [CLANG, "-O0" if sources is PRODUCTS else "-O2", "-std=c++17", "-mf16c", "-mfma", "-ffp-contract=off", "-fPIC", "-w", "-I", os.path.join(ROOT, "tests", "host_layers"), "-I", here]
    running = [(name, subprocess.Popen(flags + ["-x", "c++", "-c", os.path.join(here, name), "-o", os.path.join(here, name + ".o")], stderr=subprocess.PIPE, text=True))
               for name in sources + ["reports.cpp"]]
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


class Products(host_wave.Host):
    """The calls of the products with four-bit weights (of a library of PRODUCTS)."""

    def __init__(self, path):
        lib = ctypes.CDLL(path)
        vp, i64, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
        lib.apmm_w4_packed_bytes.argtypes, lib.apmm_w4_packed_bytes.restype = [i64, i64, ci], ctypes.c_size_t
        lib.apmm_w4_workspace_bytes.argtypes, lib.apmm_w4_workspace_bytes.restype = [i64, i64, i64, ci], ctypes.c_size_t
        lib.apmm_w4_pack.argtypes = [vp, vp, i64, i64, ci, ci, vp, vp]
        lib.apmm_w4_gemm.argtypes = [i64, i64, i64, ci, ci, vp, i64, vp, vp, i64, vp, ctypes.c_size_t, vp]
        self.lib = lib

    def pack(self, codes, scales, group):
        N, K = codes.shape
        packed = Memory().empty((self.lib.apmm_w4_packed_bytes(N, K, group),), torch.uint8).fill_(0xff)
        self.call(self.lib.apmm_w4_pack, codes.data_ptr(), scales.data_ptr(), N, K, group, int(scales.dtype == torch.bfloat16), packed.data_ptr(), None)
        return packed

    def gemm(self, x, packed, N, group, y):
        (M, K), m = x.shape, Memory()
        need = self.lib.apmm_w4_workspace_bytes(M, N, K, group)
        work = m.empty((need,), torch.uint8).fill_(0xff)
        self.call(self.lib.apmm_w4_gemm, M, N, K, group, int(x.dtype == torch.bfloat16), x.data_ptr(), x.stride(0), packed.data_ptr(), y.data_ptr(), y.stride(0), work.data_ptr(), need, None)
        return y
