"""Which kernel a product of e4m3 operands takes (launches stubbed out): between them the sizes of project_sizes take every one of them, so that the GPU
tests compare all of them with the oracle, also when the rule changes."""
from tests.launch_sizes import run_checked

BODY = r"""
from tests.project_sizes import SIZES
stub.launch_stub_kernel_of.restype = ctypes.c_char_p

def kernel(mt, nt, scale, out):
    if not mt:
        return rf"project_fp8_tile_kernelILb{int(scale == 'e8m0')}E"
    return rf"project_fp8_rows_kernelILi{mt}ELi{nt}ELi[48]ELb{int(scale == 'e8m0')}ELb{int(out == 'f32')}E"

taken, one, odd, pieces = set(), set(), set(), set()
for mt, nt, scale, out, M, K, widths in SIZES:
    name = launched(project(M, K, widths, int(scale == "e8m0"), int(out == "bf16")))
    assert re.search(kernel(mt, nt, scale, out), name), (mt, nt, scale, out, M, K, widths, name)
    assert M % (16 * mt or 256) and (nt == 1 or sum(widths) % (16 * nt or 256)), (M, widths)
    taken.add(name)
    steps, waves = -(-K // 128), int(re.search("ELi([48])ELb", name).group(1)) if mt else 1
    if steps == 1: one.add(name)
    if steps > 1 and steps % 2 and K % 128: odd.add(name)
    if steps > waves * (12 if scale == "e8m0" else 4): pieces.add(name)
built = {n for n in (stub.launch_stub_kernel_of(i).decode() for i in range(stub.launch_stub_known())) if "project_fp8" in n}
assert len(built) > 100 and len(one) > 100 and taken == odd == pieces == built, [sorted(built - s) for s in (taken, odd, pieces)]
"""


def test_every_kernel_is_taken(tmp_path):
    run_checked(tmp_path, BODY)
