"""Corners of the entry points of a decoding step that need no GPU."""
import ctypes
import os
import re

import pytest

from paper_2607_22242_gb300 import _build, bf
from test_answer_host import FAR, SOME, attend, beams, cache, layout, reorder, step, workspace

AWAY = 1 << 40  # aligned, behind everything else


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return bf.load()


# ---- outputs over what a call reads ----

# Four answers of two prompts, four heads of 64 over two of 10 and 5 tokens; bytes of each argument.
INPUTS = {"q": 2048, "pk": 5120, "pv": 5120, "sk": 5120, "sv": 5120, "prefix_lengths": 16, "suffix_lengths": 32}


@pytest.mark.parametrize("end", ["first", "last"])
@pytest.mark.parametrize("name", INPUTS)
@pytest.mark.parametrize("output", ["out", "lse"])
def test_attention_overlaps(lib, output, name, end):
    """out (2,048 bytes) or lse (64) in the first or last bytes of what the call reads."""
    where = {n: AWAY + (i << 20) for i, n in enumerate(INPUTS)}
    size = {"out": 2048, "lse": 64}[output]
    at = where[name] + INPUTS[name] - 8 if end == "last" else where[name] - size + 8
    at = at // 4 * 4
    kv = lambda n, rows, tokens: cache(rows, tokens, 2, data=where[n])
    call = dict(q=cache(data=where["q"]), pk=kv("pk", 2, 10), pv=kv("pv", 2, 10), sk=kv("sk", 4, 5), sv=kv("sv", 4, 5),
                prefix_lengths=where["prefix_lengths"], suffix_lengths=where["suffix_lengths"], lse=2 * AWAY)
    call[output] = cache(data=at) if output == "out" else at
    assert attend(lib, **call) == bf.BF_EINVAL
    assert "overlaps" in bf.last_error()


@pytest.mark.parametrize("off", [-60, 0, 2044])
def test_attention_sums_over_outputs(lib, off):
    assert attend(lib, lse=FAR + off) == bf.BF_EINVAL
    assert "overlaps" in bf.last_error()


@pytest.mark.parametrize("name", ["parents", "lengths"])
@pytest.mark.parametrize("off", [-56, 0, 640, 5112])
@pytest.mark.parametrize("in_place", [True, False])
def test_reorder_overlaps(lib, in_place, off, name):
    """A second array (5,120 bytes) over the parents or the lengths (64 bytes)."""
    to = (FAR, AWAY)
    call = dict(frm=to if in_place else (SOME, 2 * AWAY), to=to, lengths=1 << 42)
    call[name] = AWAY + off
    assert reorder(lib, a=layout(), **call) == bf.BF_EINVAL
    assert "overlaps " + name in bf.last_error()


# ---- waits that may run out ----

def test_waits_that_run_out_leave_a_sign():
    """Rows that stay as they were because a wait ran out would be caches of two beams in one, with no sign of it: no
    kernel just ends there."""
    found = 0
    for name in sorted(os.listdir(_build.CSRC)):
        if name.endswith((".cu", ".cuh")):
            with open(os.path.join(_build.CSRC, name), encoding="utf-8") as f:
                code = _build._code_only(f.read())
            found += code.count("barrier_wait(")
            assert not re.search(r"if \(!barrier_wait\([^;]*\)\) return;", code), name
    assert found > 5


# ---- length penalties ----

@pytest.mark.parametrize("penalty", [65537.0, 1e30, float("inf")])
def test_beams_refuse_larger_penalties(lib, penalty):
    assert step(lib, args=beams(length_penalty=penalty, lengths=FAR)) == bf.BF_EINVAL
    assert "length_penalty" in bf.last_error()


# ---- workspaces ----

@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("prompts,each,heads,kv_heads,dim", [(256, 16, 32, 8, 128), (4096, 1, 32, 8, 128), (2048, 16, 32, 8, 128),
                                                             (64, 16, 16, 4, 64), (3000, 3, 8, 8, 200), (500, 40, 24, 1, 96)])
def test_attention_workspace_is_of_what_there_is(lib, prompts, each, heads, kv_heads, dim, dtype):
    """A prompt's and an answer's own part of each query vector's output, (dim + 2) numbers of 32 bits, with rows to a
    multiple of 2, and a part more for each of 304 blocks."""
    n = ctypes.c_uint64(0)
    q, pk, sk = cache(prompts * each, 1, heads, dim, dtype), cache(prompts, 512, kv_heads, dim, dtype), cache(prompts * each, 128, kv_heads, dim, dtype)
    assert workspace(lib, q, pk, sk, ctypes.byref(n)) == bf.BF_OK
    even = lambda k: k + k % 2
    share, wide = heads // kv_heads, (dim + 3) // 4 * 4 + 2
    tiles = -(-each * share // 64)  # of 64 rows, or of up to 256
    own = prompts * each * kv_heads * -(-share // 16) * even(min(share, 64))
    most = 4 * wide * (own + (304 + prompts * kv_heads * tiles) * even(min(each * share, 256)))
    assert n.value <= most + (1 << 20)
    if each * share <= 64:  # else the last of the tiles may be part empty
        assert n.value <= 2.2 * 4 * wide * prompts * each * heads + 4 * wide * 304 * 64 + (1 << 20) or share % 2
