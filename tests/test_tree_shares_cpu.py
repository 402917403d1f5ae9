"""The arithmetic by which blocks share a tree attention's work, compiled for the host from
the kernel's own header: exact for every cost that a call can have."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2601_01513_amd import build as b

SOURCE = """
#include "tree_attn.h"
extern "C" auto share_of(long total, int blocks) { return vsr::share_of(total, blocks); }
"""


@pytest.fixture(scope="module")
def share_of(tmp_path_factory):
    if not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("no hipcc")
    at = tmp_path_factory.mktemp("shares")
    (at / "shares.hip").write_text(SOURCE)
    cmd = [b.hipcc(), "--offload-host-only", "-O2", "-std=c++17", "-fPIC", "-shared", "-x", "hip", "-w",
           "-I", b.INCLUDE, "-I", b.CSRC, str(at / "shares.hip"), "-o", str(at / "shares.so")]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    f = ctypes.CDLL(str(at / "shares.so")).share_of
    f.argtypes, f.restype = [ctypes.c_long, ctypes.c_int], ctypes.c_long
    return f


def test_shares_of_large_costs(share_of):
    """A chain of 2^22 rows, 64 heads on 8, of all its keys: 2^40.5; every row and key that a
    call may have: 2^56. The blocks' shares cover the cost, and none is left empty-handed
    that needs not be."""
    rng = random.Random(3)
    totals = [1, 2 ** 31 - 1, 2 ** 39 - 1, 2 ** 39, 2 ** 39 + 1, int(2 ** 40.5), 2 ** 53 + 1, 2 ** 56]
    totals += [rng.randrange(1, 2 ** rng.randrange(1, 57)) for _ in range(2000)]
    assert share_of(0, 256) == 1
    for total in totals:
        for blocks in (1, 2, 255, 256, 512, rng.randrange(1, 512)):
            assert share_of(total, blocks) == -(-total // blocks)


def test_workspaces_are_as_large_as_what_is_written():
    """Two partial results of fp32 and their sums for each row of 512 blocks of 32 rows, or of
    256 blocks of 256 (head_dim past 128: of 128) rows, and 512 lists of 24 bytes."""
    from paper_2601_01513_amd import binding as B
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libvsr.so not built (python -m paper_2601_01513_amd.build)")
    size = B.load_library().vsr_tree_attention_workspace_size
    for hd, HD in ((1, 64), (64, 64), (65, 128), (128, 128), (129, 256), (256, 256)):
        for T, rows in ((8, 512 * 32), (64, 512 * 32), (65, 256 * (128 if HD == 256 else 256)),
                        (4096, 256 * (128 if HD == 256 else 256))):
            for dtype in (B.VSR_F32, B.VSR_BF16, B.VSR_F16):
                need = 2 * rows * (HD * 4 + 8) + 512 * 24
                assert need <= size(dtype, hd, T, 8, 4, 1) <= need + 256, (hd, T)
