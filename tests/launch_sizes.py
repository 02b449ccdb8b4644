"""Runs calls on the host with their launches stubbed out by launch_sizes_stub.c, which fails what the runtime does not launch."""
import os
import subprocess
import sys

import paper_2506_09316_amd as dsla
from tests.test_launch_stub import CHILD

HERE = os.path.dirname(os.path.abspath(__file__))

PRELUDE = CHILD + r"""
import re
stub.launch_stub_kernel.restype, stub.launch_stub_workgroups.restype, stub.launch_stub_row.restype = ctypes.c_char_p, ctypes.c_uint64, ctypes.c_uint32
ptr = lambda n: ctypes.c_void_p(1 << 20 | n << 12)

def launched(status):
    '''Of the call whose status that is: its one launch's kernel.'''
    assert (status, stub.launch_stub_count()) == (OK, 1), (status, stub.launch_stub_count())
    return stub.launch_stub_kernel().decode()

def residual_norm(rows, D, x=1, y=1, h=1, scale=1):
    stub.launch_stub_reset(-1)
    n = binding.DslaNorm(D=D, x_dtype=x, y_dtype=y, h_dtype=h, scale_type=scale, gate_act=2, eps=1e-6, residual_scale=1.0, post_weight=0x9000, pre_weight=0xa000)
    return lib.dsla_residual_norm(ctypes.byref(n), i64(rows), ptr(0), ptr(1), ptr(2), ptr(3), ptr(4), ptr(5) if h == 2 else None, None)

def head_norm(rows, H, d, io=1, out=1):
    stub.launch_stub_reset(-1)
    n = binding.DslaHeads(H=H, d=d, io_dtype=io, out_dtype=out, scale_type=1, gate_act=2, eps=1e-6, weight=0x9000)
    return lib.dsla_head_norm(ctypes.byref(n), i64(rows), ptr(0), ptr(1), ptr(2), ptr(3) if out == 2 else None, None)

def quantize(rows, cols, block_rows, io=1, scale=1):
    stub.launch_stub_reset(-1)
    return lib.dsla_quantize(i64(rows), cols, io, block_rows, scale, ptr(0), ptr(1), ptr(2), None)

def project(M, K, widths, scale=1, out=1):
    stub.launch_stub_reset(-1)
    n = len(widths)
    return lib.dsla_project_fp8(i64(M), K, n, (ctypes.c_int32 * n)(*widths), scale, ptr(0), ptr(1), ptr(2), ptr(3), None, out,
                                (ctypes.c_void_p * n)(*[ptr(8 + j).value for j in range(n)]), None)
"""


def run_checked(tmp_path, body, *arguments):
    """body in a process of its own; what it prints."""
    if not os.path.exists(dsla.library_path()):
        from paper_2506_09316_amd import build
        build.build()
    stub = str(tmp_path / "launch_sizes_stub.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-o", stub, os.path.join(HERE, "launch_sizes_stub.c")], check=True)
    env = dict(os.environ, LD_PRELOAD=":".join(p for p in (stub, os.environ.get("LD_PRELOAD")) if p))
    run = subprocess.run([sys.executable, "-c", PRELUDE + body + "\nprint('done')", *arguments], env=env, cwd=os.path.dirname(HERE), capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("done"), run.stderr
    return run.stdout
