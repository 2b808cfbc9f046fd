"""No kernel is compiled that no call can launch: the launch rules below, written out again, over every width the
calls take, against the kernels' names in the built library."""
import re
import subprocess

from paper_2509_08721_b200 import build

BYTES = {"float": 4, "__nv_bfloat16": 2, "signed char": 1}


def kernels(name):
    """Template arguments of every instantiation of a kernel in the library."""
    out = subprocess.run(["nm", "-C", build.build()], capture_output=True, text=True, check=True).stdout
    return {tuple(a.strip() for a in m.group(1).split(","))
            for m in re.finditer(r"\bsapo::%s<([^()]*)>\(" % name, out)}


def up(a, b):
    return -(-a // b)


def test_norm_forward_ring():
    """Rows of 257 columns and more in whole vectors; up to 8192 columns in at most 4 vectors a thread, then in 8.  The ring
    and the weights have to fit into shared memory.  (Wherever a width is launched, type permitting, its rows may be
    aligned.)"""
    want = set()
    for tx, size in BYTES.items():
        for H in range(264, 16385, 8):
            wpr = 1
            while wpr < 8 and wpr * 128 < up(H, 8):
                wpr *= 2
            vpl = up(up(H, 8), wpr * 32)
            vpl = 8 if vpl > 4 else vpl
            stages = 4 if size == 1 else (3 if vpl <= 4 else 2)
            if stages * 8 * vpl * 256 * size + 2 * up(H, 256) * 256 * 4 <= 220 * 1024:
                want.add((tx, str(vpl), "true" if H == wpr * vpl * 256 else "false"))
    assert kernels("norm_fwd_ring_kernel") == want


def test_checkpoint_rows():
    want = set()
    for tx in ("float", "__nv_bfloat16"):
        for restore, most in (("false", 4), ("true", 2)):
            want |= {(tx, lanes, str(most), restore) for lanes in ("4", "8", "16")}
            for H in range(136, 16385, 8):
                steps = up(H, 256)
                want.add((tx, "32", str(up(steps, up(steps, most))), restore))
    assert kernels("ckpt8_rows_kernel") == want


def test_norm_backward_ring():
    """Rows of 129 columns and more in whole vectors; where not even two rows fit into shared memory, another kernel."""
    want = set()
    for tx, sx in BYTES.items():
        for td in ("float", "__nv_bfloat16"):
            for H in range(136, 16385, 8):
                vpl = 1 if H <= 256 else (2 if H <= 8192 else 4)
                wpr = up(up(H, 8), vpl * 32)
                two, one = (0 if wpr > 8 else 2 * (8 // wpr) * wpr), 16 // wpr * wpr
                threads = 32 * wpr * (8 // wpr if two >= one else 16 // wpr)
                if vpl == 2:
                    most, slots = (256, 4 if wpr <= 4 else 8) if threads <= 256 else (512, 8 if wpr <= 8 else 16)
                else:
                    most, slots = (256, 2) if vpl == 1 else (512, 16)
                row = most // 32 * (vpl * 256 * (sx + BYTES[td]) + 64 + (vpl * 128 if sx == 1 else 0))
                if 2 * row <= 220 * 1024:
                    want.add((tx, td, str(vpl), str(most), str(slots), "true" if H == wpr * vpl * 256 else "false"))
    assert kernels("norm_bwd_ring_kernel") == want
