"""The kernels of the operators of layers in 8-bit floating point are in the library, in every form that a call may take and in no other, and keep everything in
registers (see test_kernel_resources)."""
import itertools

import pytest

import paper_2506_06472_amd as tio
from paper_2506_06472_amd import build
from test_kernel_resources import _code_objects, _kernels

T = ("NS_6bf16_tE", "f")
FLAGS = (0, 1)
ALL = itertools.product
FORMS = {
    "fp8_store_k": [f"I{t}Li{form}ELb{tiles}ELb{both}E" for t, form, tiles, both in ALL(T, FLAGS, FLAGS, FLAGS)],
    "fp8_load_k": [f"I{t}Li{form}E" for t, form in ALL(T, FLAGS)],
    "gemm_fp8_direct_k": [f"ILi{a}ELi{b}E{t}Li{m}ELi{n}ELi{w}E"
                          for a, b, t, (m, n, w) in ALL(FLAGS, FLAGS, T, ((1, 1, 4), (1, 1, 8), (2, 1, 8), (2, 2, 4), (2, 2, 8), (4, 2, 8)))],
    # forms; groups of 16 rows and columns to a wavefront, steps in LDS
    "gemm_fp8_tile_k": [f"ILi{a}ELi{b}ELi{n}ELi{n}ELi{d}E" for a, b, (n, d) in ALL(FLAGS, FLAGS, ((8, 2), (4, 4), (4, 2)))],
    "gemm_fp8_strip_k": [f"ILi{a}ELi{b}E" for a, b in ALL(FLAGS, FLAGS)],
    "gemm_fp8_tile32_k": [f"ILi{a}ELi{b}E" for a, b in ALL(FLAGS, FLAGS)],
    "gemm_fp8_sums_k": [f"I{t}E" for t in T],
    # wavefronts to a row; root mean square; a norm behind the block
    "residual_norm_k": [f"I{t}Li{w}ELb{rms}ELb{post}E" for t, w, rms, post in ALL(T, (1, 2, 4, 8, 16), FLAGS, FLAGS)],
    "residual_norm_bwd_k": [f"I{t}Li{w}ELb{rms}ELb{post}E" for t, w, rms, post in ALL(T, (1, 2, 4, 8, 16), FLAGS, FLAGS)],
    "residual_sums_k": [f"I{t}E" for t in T],
    "dropout_k": [f"I{t}Lb{resid}E" for t, resid in ALL(T, FLAGS)],
    "rope_axes_k": [f"I{t}E" for t in T],
}


@pytest.fixture(scope="module")
def kernels():
    tio.binding.lib()
    with open(build.LIB, "rb") as f:
        return {k[".name"]: k for obj in _code_objects(f.read()) for k in _kernels(obj)}


@pytest.mark.parametrize("family", FORMS)
def test_forms_are_there_and_do_not_spill(family, kernels):
    name = f"{len(family)}{family}"                        # as it stands in a mangled name
    mine = {n: k for n, k in kernels.items() if name in n}
    for form in FORMS[family]:
        assert sum(form in n[n.index(name):] for n in mine) == 1, form
    assert len(mine) == len(FORMS[family])
    for n, k in mine.items():
        assert not k[".vgpr_spill_count"] and not k[".private_segment_fixed_size"], n
