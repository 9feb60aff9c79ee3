"""Builds the key/value cache's sources for the host with host_wave/hip/hip_runtime.h in the place of HIP's own header, so that their device code runs on the CPU."""
import ctypes
import mmap
import os
import re
import shutil
import subprocess

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2409_17870_amd", "csrc")
CLANG = os.environ.get("HOST_CLANG", "/opt/rocm/llvm/bin/clang++")
SOURCES = ["apmm_api_kv.hip", "apmm_kv_store.hip", "apmm_kv_attention.hip", "apmm_kv_attention_rows.hip", "apmm_kv_attention_tiles.hip"]

REPORTS = r"""
#include "apmm_api.h"
namespace apmm {
apmm_status fail(apmm_status st, const char *) { return st; }
apmm_status fail_hip(hipError_t, const char *) { return APMM_ERR_HIP; }
}
"""


def on_host(text):
    """Launches become calls, the assembly of one instruction its meaning, that which only names a register nothing."""
    text = re.sub(r"(\w+<[\w, ]+>)<<<(.+?), (dim3\([^;>]*?\)|\w+), 0, stream>>>\((.*?)\);", r"host_wave::launch(\2, \3, [&] { \1(\4); });", text)
    text = re.sub(r'asm\("v_cvt_flr_i32_f32 %0, %1" : "=v"\((\w+)\) : "v"\((\w+)\)\);', r"\1 = \2 != \2 ? 0 : (int)floorf(\2);", text)
    text = re.sub(r'asm volatile\("" : "\+v"\(\w+\)\);', "", text)
    assert "<<<" not in text and "asm" not in re.sub(r"//.*", "", text)
    return text


def available():
    return shutil.which(CLANG) is not None


def build(folder, program=None):
    """A program of `program` and the sources, or, without one, a shared library of include/apmm.h's calls; its path."""
    here = os.path.join(str(folder), "package", "csrc")
    shutil.copytree(os.path.join(ROOT, "include"), os.path.join(str(folder), "include"), dirs_exist_ok=True)
    os.makedirs(here, exist_ok=True)
    for name in os.listdir(CSRC):
        if name.startswith("apmm_kv") or name in ("apmm_api.h", "apmm_api_kv.hip"):
            with open(os.path.join(CSRC, name)) as f, open(os.path.join(here, name), "w") as g:
                g.write(on_host(f.read()))
    parts = {"reports.cpp": REPORTS}
    if program is not None:
        parts["program.cpp"] = program
    for name, text in parts.items():
        with open(os.path.join(here, name), "w") as f:
            f.write(text)
    flags = [CLANG, "-O2", "-std=c++17", "-mf16c", "-mfma", "-ffp-contract=off", "-fPIC", "-w", "-I", os.path.join(ROOT, "tests", "host_wave"), "-I", here]
    running = [(name, subprocess.Popen(flags + ["-x", "c++", "-c", os.path.join(here, name), "-o", os.path.join(here, name + ".o")], stderr=subprocess.PIPE, text=True))
               for name in SOURCES + list(parts)]
    for name, p in running:
        err = p.communicate()[1]
        assert p.returncode == 0, name + ": " + err[-3000:]
    to = os.path.join(str(folder), "libkv_host.so" if program is None else "program")
    subprocess.run(flags + (["-shared"] if program is None else []) + [os.path.join(here, name + ".o") for name, _ in running] + ["-o", to], check=True, capture_output=True, text=True)
    return to


class Memory:
    """Tensors that end where memory that cannot be touched begins (it also lies before them), seen by child processes."""

    def __init__(self):
        self.held = []

    def empty(self, shape, dtype):
        n = int(torch.empty(0, dtype=dtype).element_size() * torch.Size(shape).numel())
        page, room = mmap.PAGESIZE, -(-max(n, 1) // mmap.PAGESIZE) * mmap.PAGESIZE
        m = mmap.mmap(-1, room + 2 * page)
        self.held.append(m)
        at = ctypes.addressof(ctypes.c_char.from_buffer(m))
        libc = ctypes.CDLL(None, use_errno=True)
        libc.mprotect.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int]
        for guard in (at, at + page + room):
            if libc.mprotect(guard, page, 0):
                raise OSError(ctypes.get_errno(), "mprotect")
        begin = page + room - -(-n // 16) * 16  # 16-byte aligned: up to 15 bytes behind the end are not seen
        if n == 0:
            return torch.empty(shape, dtype=dtype)
        return torch.frombuffer(memoryview(m)[begin:begin + n], dtype=torch.uint8).view(dtype).view(shape)

    def copy(self, t):
        r = self.empty(t.shape, t.dtype)
        r.copy_(t)
        return r


class Host:
    """The calls of include/apmm.h on tensors of the host.  Each runs in a child process, so that a touch of what it must not touch ends the child alone."""

    def __init__(self, path):
        from paper_2409_17870_amd import binding
        self.binding, lib = binding, ctypes.CDLL(path)
        cache, batch, rows = ctypes.POINTER(binding.ApmmKvCache), ctypes.POINTER(binding.ApmmKvBatch), [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64]
        for fn in (lib.apmm_kv_write, lib.apmm_kv_read):
            fn.argtypes = [cache, batch] + rows + rows + [ctypes.c_void_p]
        lib.apmm_kv_attention.argtypes = [cache, batch, ctypes.c_int] + rows + rows + [ctypes.c_float, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        lib.apmm_kv_attention_workspace_bytes.argtypes, lib.apmm_kv_attention_workspace_bytes.restype = [cache, batch, ctypes.c_int], ctypes.c_size_t
        self.lib = lib

    def structs(self, codes, scales, table, lengths, starts, tokens):
        pages, heads, _, ps = scales.shape
        return (self.binding.ApmmKvCache(codes.data_ptr(), scales.data_ptr(), pages, ps, heads, codes.shape[3] * 2 // ps, int(scales.dtype == torch.bfloat16)),
                self.binding.ApmmKvBatch(lengths.shape[0], tokens, lengths.data_ptr(), None if starts is None else starts.data_ptr(), table.data_ptr(), table.stride(0), table.shape[1]))

    def call(self, fn, *args):
        pid = os.fork()
        if pid == 0:
            status = 127
            try:
                status = fn(*args)
            finally:
                os._exit(status)
        status = os.waitpid(pid, 0)[1]
        assert not os.WIFSIGNALED(status), "%s ended by signal %d" % (fn.__name__, os.WTERMSIG(status))
        assert os.WEXITSTATUS(status) == 0, "%s: status %d" % (fn.__name__, os.WEXITSTATUS(status))

    def write(self, k, v, codes, scales, table, lengths, starts=None):
        self.call(self.lib.apmm_kv_write, *self.structs(codes, scales, table, lengths, starts, k.shape[0]), k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), None)

    def read(self, codes, scales, table, lengths, tokens, starts=None):
        m, (_, heads, _, ps) = Memory(), scales.shape
        k, v = (m.empty((tokens, heads, codes.shape[3] * 2 // ps), scales.dtype).fill_(float("nan")) for _ in range(2))
        self.call(self.lib.apmm_kv_read, *self.structs(codes, scales, table, lengths, starts, tokens), k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), None)
        return k.clone(), v.clone()

    def attention(self, q, codes, scales, table, lengths, starts=None, window=0, sinks=0, scale=None):
        m, (cache, batch) = Memory(), self.structs(codes, scales, table, lengths, starts, q.shape[0])
        out = m.empty(q.shape, q.dtype).fill_(float("nan"))
        need = self.lib.apmm_kv_attention_workspace_bytes(cache, batch, q.shape[1])
        work = m.empty((need,), torch.uint8).fill_(0xff)  # NaN
        self.call(self.lib.apmm_kv_attention, cache, batch, q.shape[1], q.data_ptr(), q.stride(0), q.stride(1), out.data_ptr(), out.stride(0), out.stride(1),
                  q.shape[2] ** -0.5 if scale is None else scale, window, sinks, work.data_ptr(), need, None)
        return out.clone()
