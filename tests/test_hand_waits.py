"""Kernels that load straight into LDS wait for their loads by hand, and a barrier behind the wait frees a part of LDS that the wavefront has read.  The compiler orders reads of LDS
with neither: a read whose value is used only behind the barrier could move there, to where another wavefront's loads write.  So the source has to forbid
it: an access to memory does not cross `asm volatile("" ::: "memory")`, and one stands directly before each such wait and behind its barrier."""
import os
import re

import pytest

from paper_2506_06472_amd import build

CLOBBER = 'asm volatile("" ::: "memory");'
PINNED = "__builtin_amdgcn_sched_barrier(0);"
WAIT = re.compile(r"__builtin_amdgcn_s_waitcnt\([^;]*\);$")


def _statements(name):
    with open(os.path.join(build.CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    code = re.sub(r"\n\s*#[^\n]*", "", code)
    return [s for s in (" ".join(p.split()) for p in re.findall(r"[^;{}]*[;{}]", code)) if s]


def _unordered(statements):
    """the statements before each barrier, where a read could move over it"""
    bad = []
    for i, s in enumerate(statements):
        if "__builtin_amdgcn_s_barrier()" not in s:
            continue
        before = statements[max(0, i - 4):i]
        assert WAIT.search(before[-1]), before
        rest = [b for b in before[:-1] if b != PINNED]
        behind = [b for b in statements[i + 1:i + 3] if b != PINNED]
        if rest[-1] != CLOBBER or behind[0] != CLOBBER:
            bad.append(before + [s] + behind)
    return bad


def test_the_check_sees_an_unordered_wait():
    wait = ["read(next);", "__builtin_amdgcn_s_waitcnt(0x0070);", "__builtin_amdgcn_s_barrier();", CLOBBER]
    assert _unordered(wait) and not _unordered([CLOBBER] + wait[1:]) and not _unordered([CLOBBER, PINNED] + wait[1:])
    assert _unordered([CLOBBER] + wait[1:3] + ["load();", "load();"])


@pytest.mark.parametrize("name", ["kernels_gemm_fp8.hip"])
def test_reads_stay_before_the_barrier_that_frees_their_place(name):
    statements = _statements(name)
    assert sum("__builtin_amdgcn_s_barrier()" in s for s in statements) > 0
    bad = _unordered(statements)
    assert not bad, "\n".join(map(str, bad))
