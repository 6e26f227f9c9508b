"""The build's look for matrix products whose results are read too early, on code written for it and on the objects that were built (no GPU)."""
import glob
import os

import pytest

from paper_2308_09723_amd import build, waits

PRODUCT = "v_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], v[0:15]"


def _kernel(*lines, name="kernel"):
    """As llvm-objdump writes it."""
    return f"\nDisassembly of section .text:\n\n<{name}>:\n" + "".join((x if x.endswith(":") else f"\t{x}") + "   // 000000009900\n" for x in lines) + "\ts_endpgm\n"


@pytest.mark.parametrize("product,need", [("v_mfma_f32_4x4x4_16b_f16", 5), ("v_mfma_f32_16x16x32_bf16", 8), ("v_mfma_i32_16x16x64_i8", 8), ("v_mfma_f32_32x32x16_f16", 12)])
def test_states_needed(product, need):
    assert waits.needed(product) == need
    for states in (0, 1, need - 1, need):
        wait = [f"s_nop {min(8, states - i) - 1}" for i in range(0, states, 8)]
        found = waits.short_waits(_kernel(f"{product} a[0:3], v[20:23], v[24:27], a[0:3]", *wait, "v_accvgpr_read_b32 v7, a2"))
        assert [f[3:] for f in found] == ([] if states == need else [(states, need)])


def test_a_product_of_unknown_length_is_an_error():
    with pytest.raises(KeyError):
        waits.short_waits(_kernel("v_mfma_f32_32x32x2_f32 v[0:31], v40, v41, v[0:31]"))


@pytest.mark.parametrize("use,early", [
    ("v_add_f32_e32 v30, v31, v15", True), ("v_add_f32_e32 v30, v31, v16", False), ("v_mov_b32_e32 v3, 0", True), ("global_store_dwordx4 v[30:31], v[12:15], off", True),
    ("ds_write_b64 v40, v[14:15] offset:8", True), ("ds_read_b64 v[30:31], v0", True), ("v_readfirstlane_b32 s3, v1", True), ("s_add_i32 s1, s2, s3", False),
    ("v_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], v[0:15]", False), ("v_mfma_f32_32x32x16_bf16 v[32:47], v[0:3], v[24:27], v[32:47]", True),
    ("v_add_f32_e32 v30, a3, a4", False),
])
def test_uses(use, early):
    assert bool(waits.short_waits(_kernel(PRODUCT, use))) == early


def test_results_that_were_replaced():
    assert waits.short_waits(_kernel(PRODUCT, "s_nop 7", "s_nop 3", "v_mov_b32_e32 v0, 0", "v_add_f32_e32 v1, v0, v0")) == []


def test_every_way():
    """A loop whose last product is read behind it: enough states on the way round, too few on the way out; and a short way that joins a long one."""
    loop = ["<L1>:", PRODUCT, "s_add_i32 s0, s0, 1", "s_cmp_lt_i32 s0, s1", "s_cbranch_scc1 L1"]
    found = waits.short_waits(_kernel(*loop, "v_mul_f32_e32 v30, 2.0, v0"))
    assert [f[3:] for f in found] == [(3, 12)]
    assert waits.short_waits(_kernel(*loop, "s_nop 7", "s_nop 0", "v_mul_f32_e32 v30, 2.0, v0")) == []
    join = [PRODUCT, "s_cbranch_scc0 L2", "s_nop 7", "s_nop 1", "<L2>:", "s_nop 1", "v_mul_f32_e32 v30, 2.0, v0"]
    assert [f[3:] for f in waits.short_waits(_kernel(*join))] == [(3, 12)]
    join[-2:-1] = ["s_nop 7", "s_nop 2"]
    assert waits.short_waits(_kernel(*join)) == []


def test_kernels_by_name():
    text = _kernel(PRODUCT, "v_mul_f32_e32 v30, 2.0, v0") + _kernel(PRODUCT, "s_nop 7", "s_nop 3", "v_mul_f32_e32 v30, 2.0, v0", name="second")
    assert [f[0] for f in waits.short_waits(text)] == ["kernel"]


def test_the_build_fails():
    with pytest.raises(RuntimeError, match="kernel.*v_mul_f32"):
        build.check_waits([("a.hip", waits.short_waits(_kernel(PRODUCT, "v_mul_f32_e32 v30, 2.0, v0")))])
    build.check_waits([("a.hip", [])])


def test_the_objects_that_were_built():
    """Some of them (the build looks at all): those of attention and of adapters."""
    objects = sorted(p for name in ("fq_attn_*.o", "fq_adapters.o") for p in glob.glob(os.path.join(build.OBJ_DIR, name)))
    if not objects:
        pytest.skip("nothing built here")
    build.check_waits([(path, build.short_waits(path)) for path in objects])
