"""CPU-only checks of include/nk_rows.h: every declared function is exported and bound, the constants agree."""
import os
import re

import paper_2511_13764_b200 as nk
from paper_2511_13764_b200 import rows

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "nk_rows.h")


def test_library_exports_every_declared_symbol():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(nk_(?:grouped|route|lora)_[a-z0-9_]+)\s*\(", src)))
    assert len(names) > 20 and sorted(rows.EXPORTS) == names
    assert sorted(rows.exported_symbols()) == names


def test_constants_and_structures_match_the_binding():
    src = open(HEADER).read()
    assert re.search(r"NK_GROUPED_ROWS\s*=\s*0,\s*NK_GROUPED_WEIGHTS\s*=\s*1", src)
    assert (nk.GROUPED_ROWS, nk.GROUPED_WEIGHTS) == (0, 1)
    for family, desc in (("grouped", rows.GroupedDesc), ("route", rows.RouteDesc), ("lora", rows.LoraDesc)):
        end = src.index(f"}} nk_{family}_desc_t;")
        body = re.sub(r"/\*.*?\*/", "", src[src.rindex("typedef struct {", 0, end):end], flags=re.S)
        fields = [(t, n.strip()) for t, ns in re.findall(r"(int64_t|int32_t)\s+([^;]+);", body) for n in ns.split(",")]
        want = [("int64_t" if c.__name__.endswith("long") or c.__name__ == "c_int64" else "int32_t", n) for n, c in desc._fields_]
        assert fields == want
