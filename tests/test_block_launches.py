"""What the calls around a layer do around their launches, with these stubbed out (no GPU): every accepted call is one launch, of the smallest
sizes and the largest, and a launch's error reaches the caller."""
from tests.test_launch_stub import LAUNCH_ERRORS, run_stubbed

EACH = LAUNCH_ERRORS[:LAUNCH_ERRORS.index("for io in (0, 1):")]

BODY = EACH + r"""
import random
ptr = lambda n: ctypes.c_void_p(1 << 20 | n << 12)
norm = lambda **k: binding.DslaNorm(**{**dict(D=256, x_dtype=1, y_dtype=1, h_dtype=1, scale_type=1, gate_act=2, eps=1e-6, residual_scale=1.0, post_weight=0x9000, pre_weight=0xa000), **k})
for D in (16, 128, 144, 512, 528, 1024, 1040, 2048, 4096, 4112, 8192, 8208, 16384, 32768):
    for x in (0, 1):
        for y in (0, 1):
            for h in (0, 1, 2):
                for rows in (1, 5, 100000, 0x7fffffff // ((D + 127) // 128)):
                    n = norm(D=D, x_dtype=x, y_dtype=y, h_dtype=h)
                    each_launch(("border", D, x, y, h, rows), 1, lambda: lib.dsla_residual_norm(ctypes.byref(n), i64(rows), ptr(0), ptr(1), ptr(2), ptr(3), ptr(4),
                                                                                              ptr(5) if h == 2 else None, None))
for H, d in ((1, 64), (5, 64), (32, 128), (65536, 64)):
    for io in (0, 1):
        for out in (0, 1, 2):
            for rows in (1, 9, 1000, 0x7fffffff // ((H * d + 127) // 128)):
                n = binding.DslaHeads(H=H, d=d, io_dtype=io, out_dtype=out, scale_type=1, gate_act=2, eps=1e-6, weight=0x9000)
                each_launch(("heads", H, d, io, out, rows), 1, lambda: lib.dsla_head_norm(ctypes.byref(n), i64(rows), ptr(0), ptr(1), ptr(2), ptr(3) if out == 2 else None, None))
for cols in (16, 128, 4112, 1 << 21):
    for io in (0, 1):
        for block_rows in (1, 128):
            for scale in (0, 1):
                for rows in (1, 127, 20480, 0x7fffffff // ((cols + 127) // 128)):
                    each_launch(("quantize", cols, io, block_rows, rows), 1, lambda: lib.dsla_quantize(i64(rows), cols, io, block_rows, scale, ptr(0), ptr(1), ptr(2), None))

def project(M, K, widths, scale, out):
    n = len(widths)
    return lib.dsla_project_fp8(i64(M), K, n, (ctypes.c_int32 * n)(*widths), scale, ptr(0), ptr(1), ptr(2), ptr(3), None, out, (ctypes.c_void_p * n)(*[ptr(8 + j).value for j in range(n)]), None)

rng = random.Random(3)
sizes = [(1, 16, [16]), (1, 1 << 21, [16]), (1 << 33, 16, [16]), (1 << 30, 128, [16] * 8), (1, 128, [1 << 24]), (16384, 4096, [4096] * 5), (1 << 20, 1 << 21, [1 << 21]), (129, 128, [1 << 23, 1 << 23])]
for _ in range(1500):
    sizes.append((int(2 ** rng.uniform(0, 30)), 16 * int(2 ** rng.uniform(0, 17)), [16 * int(2 ** rng.uniform(0, 15)) for _ in range(rng.randrange(1, 9))]))
taken = 0
for M, K, widths in sizes:
    for scale in (0, 1):
        for out in (0, 1):
            stub.launch_stub_reset(-1)
            status = project(M, K, widths, scale, out)
            too_many = (M + 63) // 64 * 2 * sum(-(-w // 128) for w in widths) > 0x7ffffff0 or sum(widths) > 1 << 24
            assert (status, stub.launch_stub_count()) == ((ERR_SHAPE, 0) if too_many else (OK, 1)), (M, K, widths, scale, out, status)
            taken += not too_many
assert taken > 3000
for M in (1, 100, 5000):
    for out in (0, 1):
        each_launch(("project_fp8", M, out), 1, lambda: project(M, 4096, [4096], 1, out))
"""


def test_every_call_is_one_launch(tmp_path):
    run_stubbed(tmp_path, BODY)
