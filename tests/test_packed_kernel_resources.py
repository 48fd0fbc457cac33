"""The kernels of the operators on packed batches and 8-bit checkpoints are in the library, in every form that a call may take, and keep everything in
registers (see test_kernel_resources)."""
import itertools

import pytest

import paper_2506_06472_amd as tio
from paper_2506_06472_amd import build
from test_kernel_resources import _code_objects, _kernels

T = {"bf16": "NS_6bf16_tE", "fp32": "f"}
FORMS = {
    # head size, groups of 16 rows to a wavefront, sets of wavefronts
    "attn_fwd_mfma_k": [f"ILi{dh}ELi{ng}ELi{sets}ENS1_10PackedRows" for dh in (64, 128) for ng, sets in ((1, 1), (2, 1), (1, 2))],
    # head size, wavefronts, groups of 16 keys; delta inside; groups of heads that do not divide a tile
    "attn_packed_both_mfma_k": [f"ILi{dh}ELi{nw}ELi{ng}ELb{int(delta)}ELb{int(tail)}E" for dh, nw, ng in ((64, 4, 1), (64, 4, 2), (128, 4, 1), (128, 8, 2))
                                for delta, tail in itertools.product((False, True), repeat=2) if ng == 1 or not delta],
    "attn_packed_sums_k": [f"ILi{dh}ELi{nw}ELi{ng}E" for dh, nw, ng in ((64, 4, 1), (64, 4, 2), (128, 4, 1), (128, 8, 2))],
    "attn_packed_pre_k": [f"I{t}E" for t in T.values()],
    "attn_fwd_k": [f"4RowsE{t}Li{dh}ELi{nw}ENS1_12PackedBlocks" for t in T.values() for dh, nw in ((32, 4), (32, 8), (64, 4), (128, 4)) if t == "f" or dh == 32],
    "attn_bwd_k": [f"4RowsE{t}Li{dh}ELi{nw}ELb{int(dh == 32)}ENS1_12PackedBlocks" for t in T.values() for dh, nw in ((32, 4), (32, 8), (64, 4), (128, 4)) if t == "f" or dh == 32],
    "ckpt8_store_k": [f"I{t}Lb{past}E" for t in T.values() for past in (0, 1)],
    "ckpt8_load_k": [f"I{t}E" for t in T.values()],
    "act_ckpt8_k": [f"I{t}Lb{two}ELb{past}E" for t in T.values() for two in (0, 1) for past in (0, 1)],
    "act_ckpt8_bwd_k": [f"I{t}Lb{two}E" for t in T.values() for two in (0, 1)],
    "pref_rows_k": [f"I{t}Li{nch}ELi{nt}E" for t in T.values() for nch, nt in ((1, 256), (4, 256), (4, 512))],
    "pref_grad_k": [f"I{t}Lb{pairs}E" for t in T.values() for pairs in (0, 1)],
    "pref_pairs_k": [""], "pref_all_pairs_k": [""], "pref_mean_k": [""],
}


@pytest.fixture(scope="module")
def kernels():
    tio.binding.lib()
    with open(build.LIB, "rb") as f:
        return {k[".name"]: k for obj in _code_objects(f.read()) for k in _kernels(obj)}


@pytest.mark.parametrize("family", FORMS)
def test_forms_are_there_and_do_not_spill(family, kernels):
    name = f"{len(family)}{family}"                        # as it stands in a mangled name, where act_ckpt8_k is no part of another's
    for form in FORMS[family]:
        mine = {n: k for n, k in kernels.items() if name in n and form in n[n.index(name):]}
        assert mine, form
        for n, k in mine.items():
            assert not k[".vgpr_spill_count"] and not k[".private_segment_fixed_size"], n


@pytest.mark.parametrize("family", ["attn_packed_both_mfma_k", "attn_packed_sums_k", "attn_packed_pre_k", "ckpt8_store_k", "ckpt8_load_k", "act_ckpt8_k",
                                    "act_ckpt8_bwd_k", "pref_rows_k", "pref_grad_k", "pref_pairs_k", "pref_all_pairs_k", "pref_mean_k"])
def test_no_form_that_no_call_takes(family, kernels):
    assert sum(f"{len(family)}{family}" in n for n in kernels) == len(FORMS[family])


def test_no_form_of_the_fp32_kernels_that_no_call_takes(kernels):
    for family in ("attn_fwd_k", "attn_bwd_k", "attn_fwd_mfma_k"):
        mine = [n for n in kernels if f"{len(family)}{family}" in n and "Packed" in n]
        assert len(mine) == len(FORMS[family]), mine
