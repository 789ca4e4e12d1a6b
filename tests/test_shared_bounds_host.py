"""Bounds of attention over shared pages: what the host reserves for units.  Nothing here reaches a device."""
import ctypes
import os
import subprocess

import pytest
from test_kv_common import P, ROOT, _cache, _seqs
from test_shared_host import _groups


def _workspace(seqs, groups, H=2, G=2):
    import paper_2608_23805_amd as msi
    n = ctypes.c_uint64()
    assert msi.lib.msi_kv_attention_shared_workspace(ctypes.byref(_cache(n_heads=H)), ctypes.byref(seqs), ctypes.byref(groups), H * G,
                                                     ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("max_len,usable", [(0, 0), (1, 0), (63, 0), (64, 1), (127, 1), (192, 3)])
@pytest.mark.parametrize("rows", [5, 400])
def test_shared_blocks_past_the_longest_sequence(max_len, usable, rows):
    """Rows stand behind at most max_len / 64 blocks: more of them make no units, and without tokens a table may be absent."""
    kw = dict(n_seqs=2, n_rows=rows, max_rows=rows, max_blocks=9, max_len=max_len, table=P if max_len else None)
    got, want = (_workspace(_seqs(**kw), _groups(max_rows=rows, max_blocks=b)) for b in (9, usable))
    assert got == want


def test_units_stay_within_what_the_host_reserves(tmp_path):
    """The rules themselves, which the kernels' plans and the host's bounds are built from, over random batches: items and
    partial results of any batch within the bounds, for both lists and both forms (g++ with AddressSanitizer and
    UndefinedBehaviorSanitizer)."""
    exe = str(tmp_path / "kv_units_test")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
                    "-o", exe, os.path.join(ROOT, "tests", "cpp", "kv_units_test.cpp")], check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
