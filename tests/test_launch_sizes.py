"""The largest calls around a layer are launches that the runtime takes: fewer than 2^32 work-items in a dimension.  (Launches stubbed out.)"""
from tests.launch_sizes import run_checked

NORMS = r"""
def covers(call, needed):
    '''One launch, of at least the workgroups that are needed and of hardly more.'''
    launched(call)
    got = stub.launch_stub_workgroups()
    assert needed <= got <= needed + (0 if got == stub.launch_stub_row() else 65535), (needed, got)

lanes = lambda D: 16 if D <= 128 else 64 if D <= 1024 else 256 if D <= 2048 else 512 if D <= 4096 else 1024
for D in (16, 128, 144, 512, 1024, 1040, 2048, 4096, 8192, 16384, 32768):
    most, at_once = 0x7fffffff // -(-D // 128), max(1, 256 // lanes(D))
    border = (1 << 32) // lanes(D)   # rows from which a dimension holds no launch
    for rows in {r for r in (1, 1 << 20, border - 1, border, border + 1, most - 1, most) if r <= most}:
        for x in (0, 1):
            for h in (0, 1, 2):
                covers(residual_norm(rows, D, x, 1, h), -(-rows // at_once))
    assert residual_norm(most + 1, D) == ERR_SHAPE
for H, d in ((1, 64), (1, 128), (5, 64), (32, 128), (65536, 64), (65536, 128)):
    per = -(-H * d // 128)
    most = 0x7fffffff // per
    for rows in {r for r in (1, 4097, (1 << 29) // per, (1 << 29) // per + 1, most) if 1 <= r <= most}:
        for out in (0, 1, 2):
            blocks = rows * per
            covers(head_norm(rows, H, d, 1, out), -(-blocks // (32 if blocks >= 65536 else 16)))
    assert head_norm(most + 1, H, d) == ERR_SHAPE
for cols in (16, 128, 4112, 1 << 21):
    per = -(-cols // 128)
    most = 0x7fffffff // per
    for rows in {r for r in (1, (1 << 30) // per, (1 << 30) // per + 1, most - 127, most) if 1 <= r <= most}:
        for io in (0, 1):
            for scale in (0, 1):
                blocks = rows * per
                covers(quantize(rows, cols, 1, io, scale), -(-blocks // (64 if blocks >= 131072 else 16)))
                covers(quantize(rows, cols, 128, io, scale), -(-rows // 128) * per)
    assert quantize(most + 1, cols, 1) == ERR_SHAPE
"""


def test_norms_and_quantization(tmp_path):
    run_checked(tmp_path, NORMS)


PRODUCTS = r"""
for M, K, widths in ((1 << 33, 16, [16]), ((1 << 29) - 64, 16, [16]), ((1 << 29) + 64, 16, [16]), (1 << 30, 128, [16] * 8), (1 << 30, 16, [16]), (1 << 25, 128, [4096]),
                     (3 << 28, 400, [16, 16]), (1 << 33, 128, [128])):
    for scale in (0, 1):
        for out in (0, 1):
            kernel = launched(project(M, K, widths, scale, out))
            got = stub.launch_stub_workgroups()
            pair = re.search(r"project_fp8_rows_kernelILi(\d)ELi(\d)E", kernel)
            if pair:
                mt, nt = (int(n) for n in pair.groups())
                tiles = -(-M // (16 * mt)) * -(-sum(widths) // (16 * nt))
            else:
                assert "project_fp8_tile_kernel" in kernel
                tiles = -(-M // 256) * -(-sum(-(-w // 128) for w in widths) // 2)
            assert tiles <= got <= tiles + 8 * 31 + 7 + (0 if got == stub.launch_stub_row() else 65535), (M, K, widths, scale, out, kernel, tiles, got)
too_many = (0x7ffffff0 // 2 + 1) * 64   # rows, for one block of columns
assert project(too_many, 16, [16]) == ERR_SHAPE and project(too_many // 2, 16, [16] * 2) == ERR_SHAPE
"""


def test_products(tmp_path):
    run_checked(tmp_path, PRODUCTS)


SEVERAL = r"""
for rows, H, d in ((21850, 5, 64), (21850, 3, 128), (65537, 1, 64), (16389, 4, 128)):
    assert f"rows_kernelILi{d}ELi2E" in launched(head_norm(rows, H, d))
    assert f"rows_kernelILi{d}ELi1E" in launched(head_norm(rows // 8, H, d))
for rows, cols in ((32773, 400), (131075, 64)):
    assert "rows_kernelILi0ELi4E" in launched(quantize(rows, cols, 1)) and "rows_kernelILi0ELi1E" in launched(quantize(rows // 8, cols, 1))
"""


def test_several_blocks_to_16_lanes(tmp_path):
    """What the tests of many blocks are about: sizes that take several at a time."""
    run_checked(tmp_path, SEVERAL)


def test_the_launch_tests_have_their_helper():
    """test_block_launches takes each_launch() out of another test's source: all of it, and nothing else."""
    import ast
    from tests.test_block_launches import EACH
    (helper,) = ast.parse(EACH).body
    assert helper.name == "each_launch" and isinstance(helper.body[-1], ast.For) and len(helper.body) == 3
    assert EACH.count("assert") == 3 and "launch_stub_reset(n)" in EACH and "n + 1" in EACH
