"""Register budgets of the kernels over packed sequences and of the norms, read from the compiler's own summary (hipcc -S, no GPU needed).
Tiles of up to 128 elements run two waves per SIMD (256 registers); bf16 rows of 16- and 8-byte alignment spill nothing there (dQ of 128 elements and 8-byte rows three dwords).  What does spill is held to what it
spills now: heads of 129 to 256 elements, whose accumulators and fragments alone are some 500 registers, and rows aligned to their elements only."""
import re
import shutil
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_kernel_budget import kernel_table

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc (the compiler's register summary)")

SOURCES = ("packed_prefix.hip", "packed_bwd.hip", "packed_fwd.hip", "packed_few.hip", "qk_norm.hip")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel name and template arguments: (registers, bytes of scratch memory)} of all sources."""
    at = tmp_path_factory.mktemp("isa")
    with ThreadPoolExecutor(len(SOURCES)) as ex:
        tables = list(ex.map(lambda s: kernel_table(s, at), SOURCES))
    out = {}
    for t in tables:
        for name, budget in t.items():
            m = re.match(r"(?:void )?sh::(\w+)(?:<(.*?)>)?\(", name)
            out[m.group(1), tuple(a.strip() for a in (m.group(2) or "").split(","))] = budget
    return out


def held(kernels, name, pick, registers, scratch, least):
    seen = 0
    for (n, args), (vgpr, spilled) in kernels.items():
        if n == name and pick(args):
            assert vgpr <= registers and spilled <= scratch, (n, args, vgpr, spilled)
            seen += 1
    assert seen >= least, (name, seen)


def wide(args, at):   # 16- or 8-byte pieces
    return int(args[at]) >= 8


def test_bf16_tiles_of_up_to_128_elements_spill_nothing(kernels):
    bf = lambda a, al: "bf" in a[0] and int(a[1]) <= 128 and wide(a, al)
    held(kernels, "packed_fwd_kernel", lambda a: bf(a, 2), 256, 0, 16)
    held(kernels, "packed_fwd_long_kernel", lambda a: True, 256, 0, 3)
    held(kernels, "packed_few_kernel", lambda a: bf(a, 2), 256, 0, 4)
    held(kernels, "packed_prefix_kernel", lambda a: bf(a, 2), 256, 0, 8)
    held(kernels, "packed_dkv_ws_kernel", lambda a: wide(a, 1), 256, 0, 8)   # eight waves, two per SIMD
    held(kernels, "packed_dkv_join_kernel", lambda a: True, 128, 0, 12)
    held(kernels, "packed_dq_ds_kernel", lambda a: wide(a, 1), 256, 0, 4)
    held(kernels, "packed_dq_kernel", lambda a: bf(a, 2), 256, 12, 8)


def test_fp32_tiles_of_up_to_128_elements(kernels):
    f = lambda a: a[0] == "float" and int(a[1]) <= 128 and int(a[2]) == 16
    held(kernels, "packed_fwd_kernel", f, 256, 8, 8)
    held(kernels, "packed_few_kernel", f, 512, 0, 2)
    held(kernels, "packed_prefix_kernel", f, 512, 0, 4)
    held(kernels, "packed_dkv_kernel", f, 512, 0, 4)
    held(kernels, "packed_dq_kernel", f, 512, 0, 4)


def test_rows_aligned_to_their_elements(kernels):
    e = lambda a, al: int(a[al]) < 8 and (al == 1 or int(a[1]) <= 128)
    held(kernels, "packed_fwd_kernel", lambda a: e(a, 2), 256, 36, 16)
    held(kernels, "packed_few_kernel", lambda a: e(a, 2), 512, 0, 4)
    held(kernels, "packed_prefix_kernel", lambda a: e(a, 2), 512, 116, 8)
    held(kernels, "packed_dkv_ws_kernel", lambda a: e(a, 1), 256, 8, 4)
    held(kernels, "packed_dkv_kernel", lambda a: e(a, 2), 512, 0, 4)
    held(kernels, "packed_dq_ds_kernel", lambda a: e(a, 1), 256, 208, 2)
    held(kernels, "packed_dq_kernel", lambda a: e(a, 2), 512, 424, 8)


def test_heads_of_129_to_256_elements(kernels):
    w = lambda kind, least: lambda a: kind in a[0] and a[1] == "256" and int(a[2]) >= least
    held(kernels, "packed_fwd_kernel", w("bf", 2), 512, 0, 3)
    held(kernels, "packed_fwd_kernel", w("float", 4), 512, 236, 2)
    held(kernels, "packed_few_kernel", w("bf", 2), 512, 0, 3)
    held(kernels, "packed_few_kernel", w("float", 16), 512, 0, 1)
    held(kernels, "packed_few_kernel", w("float", 4), 512, 516, 2)
    held(kernels, "packed_prefix_kernel", w("bf", 2), 512, 100, 6)
    held(kernels, "packed_prefix_kernel", w("float", 4), 512, 536, 4)
    held(kernels, "packed_dkv_kernel", w("bf", 2), 512, 260, 3)
    held(kernels, "packed_dkv_kernel", w("float", 4), 512, 256, 4)
    held(kernels, "packed_dq_kernel", w("bf", 8), 512, 0, 2)
    held(kernels, "packed_dq_kernel", w("bf", 2), 512, 356, 3)
    held(kernels, "packed_dq_kernel", w("float", 4), 512, 960, 2)


def test_small_kernels(kernels):
    held(kernels, "packed_join_kernel", lambda a: True, 64, 0, 12)
    held(kernels, "packed_delta_kernel", lambda a: True, 64, 0, 12)
    held(kernels, "qk_norm_rope_fwd_kernel", lambda a: True, 128, 0, 12)
    held(kernels, "qk_norm_rope_bwd_kernel", lambda a: True, 160, 0, 12)
