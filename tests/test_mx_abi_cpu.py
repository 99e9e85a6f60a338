"""CPU-only checks of include/nk_mx.h: every declared function is exported and bound, constants and structures agree, and the formats'
oracle of the tests against the definitions."""
import os
import re

import numpy as np
import pytest

import paper_2511_13764_b200 as nk
from mx_testlib import E2M1, e4m3_values, group_places, quantise, tensor_scale, unpack_scales, values
from paper_2511_13764_b200 import mx

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "nk_mx.h")


def test_library_exports_every_declared_symbol():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(nk_(?:pack|mx)_[a-z0-9_]+)\s*\(", src)))
    assert len(names) > 15 and sorted(mx.EXPORTS) == names
    assert sorted(mx.exported_symbols()) == names


def test_constants_and_structures_match_the_binding():
    src = open(HEADER).read()
    assert re.search(r"NK_MXF4\s*=\s*0,\s*NK_NVF4\s*=\s*1", src) and (nk.MXF4, nk.NVF4) == (0, 1)
    for family, desc in (("pack", mx.PackDesc), ("mx", mx.MxDesc)):
        end = src.index(f"}} nk_{family}_desc_t;")
        body = re.sub(r"/\*.*?\*/", "", src[src.rindex("typedef struct {", 0, end):end], flags=re.S)
        fields = [(t, n.strip()) for t, ns in re.findall(r"(int64_t|int32_t)\s+([^;]+);", body) for n in ns.split(",")]
        want = [("int64_t" if c.__name__.endswith("long") or c.__name__ == "c_int64" else "int32_t", n) for n, c in desc._fields_]
        assert fields == want


def test_null_handles_and_arguments_are_refused_without_a_device():
    L = mx.lib()
    assert L.nk_pack_create(None, None) == 1 and L.nk_mx_create(None, None) == 1
    assert L.nk_pack_run(*[None] * 7) == 1 and L.nk_pack_scale(None, None, None, None, 0, None) == 1 and L.nk_pack_values(*[None] * 7) == 1
    assert L.nk_mx_run(*[None] * 11, 0, None) == 1 and L.nk_mx_check(None) == 1 and L.nk_pack_check(None) == 1
    assert L.nk_mx_workspace_bytes(None) == 0 and L.nk_pack_data_bytes(None) == 0
    assert L.nk_mx_destroy(None) == 0 and L.nk_pack_destroy(None) == 0


@pytest.mark.parametrize("status,make", [(3, lambda: nk.PackPlan(32, 12)), (1, lambda: nk.PackPlan(32, 0)), (2, lambda: nk.PackPlan(32, 64, in_dtype=nk.S8)),
                                         (1, lambda: nk.PackPlan(32, 64, format=7)), (2, lambda: nk.PackPlan(32, 64, groups=2, transposed=1)),
                                         (3, lambda: nk.MxPlan(32, 12, 64)), (1, lambda: nk.MxPlan(32, 64, 0)), (1, lambda: nk.MxPlan(32, 64, 64, beta=3)),
                                         (2, lambda: nk.MxPlan(32, 64, 64, out_dtype=nk.S32)), (2, lambda: nk.MxPlan(32, 64, 64, groups=5000))])
def test_descriptors_are_refused_before_a_device_is_asked_for(status, make):
    with pytest.raises(nk.NkError) as e:
        make()
    assert e.value.status == status


def test_oracle_formats():
    assert list(e4m3_values()[[0, 1, 7, 8, 56, 126]]) == [0.0, 2.0 ** -9, 7 * 2.0 ** -9, 2.0 ** -6, 1.0, 448.0]
    # MXFP4: 2^(floor(log2 m) - 2); 7 of a block whose largest is 7 becomes 6; ties to the even last bit
    x = np.zeros((1, 32))
    x[0, :10] = [7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5, -0.3]
    codes, scales, _ = quantise(x, "mxf4")
    assert scales[0, 0] == 127
    assert list(values(codes, scales, "mxf4")[0, :10]) == [6, 0, 1, 1, 2, 2, 4, 4, -4, -0.5]
    # NVFP4: the scale is m / (6 t) rounded; elements are taken against the rounded scale
    t = tensor_scale(np.array([[2688.0]]))
    assert t == 1.0
    x = np.zeros((1, 16))
    x[0, :3] = [61.0, 10.0, 5.1]
    codes, scales, _ = quantise(x, "nvf4", t)
    assert e4m3_values()[scales[0, 0]] == 10.0 and list(values(codes, scales, "nvf4", t)[0, :3]) == [60.0, 10.0, 5.0]
    # every nearest element against a search over the table
    rng = np.random.default_rng(0)
    y = rng.uniform(0, 8, 1000)
    near = E2M1[np.abs(np.minimum(y, 6)[:, None] - E2M1).argmin(1)]
    x = np.zeros((1000, 32))
    x[:, 0], x[:, 1] = 4.0, np.minimum(y, 3.9)
    codes, scales, _ = quantise(x, "mxf4")
    assert (values(codes, scales, "mxf4")[:, 1] == E2M1[np.abs(np.minimum(y, 3.9)[:, None] - E2M1).argmin(1)]).all() and near.max() == 6


def test_oracle_layout():
    rows, K = 200, 136                                      # NVF4: 9 blocks of 16, padded to 192: 12, three tiles of four
    tiles = np.arange(2 * 3 * 512) % 251
    got = unpack_scales(tiles.astype(np.uint8), np.arange(rows), K, "nvf4")
    for r, c in ((0, 0), (5, 3), (33, 4), (127, 11), (128, 0), (199, 8)):
        assert got[r, c] == tiles[(r // 128 * 3 + c // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + c % 4]
    live, at = group_places([3, 5, 5, 140])
    assert list(at[:2]) == [0, 1] and at[2] == 2 * 128 and at[-1] == 2 * 128 + 134 and list(live[:3]) == [3, 4, 5]
