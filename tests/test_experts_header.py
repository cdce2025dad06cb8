"""The binding's constants are the header's (no GPU)."""
import os
import re

import paper_2209_13258_b200 as P
from paper_2209_13258_b200 import binding as B

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "osdp.h")
DEFINES = {name: int(v) for name, v in re.findall(r"^#define OSDP_(\w+) (\d+)", open(HEADER).read(), re.M)}


def test_constants():
    assert {n: getattr(P, n) for n in ("EXPERT_ROWS", "MAX_EXPERTS", "MAX_TOP_K", "SCORE_SOFTMAX", "SCORE_SIGMOID")} == \
           {n: DEFINES[n] for n in ("EXPERT_ROWS", "MAX_EXPERTS", "MAX_TOP_K", "SCORE_SOFTMAX", "SCORE_SIGMOID")}


def test_numbers_of_the_calls_as_words(monkeypatch):
    """What each function of the binding puts into the first word."""
    first = []
    monkeypatch.setattr(B, "_entry", lambda words: first.append(int.from_bytes(words[:8], "little")) or 0)
    a = 1 << 20
    calls = [("ROUTE_FWD", B.osdp_route_fwd, (a, 16, 1, None, 4, 16, 2, 0, 1, 1, 1, 1, 1.0, a, a)),
             ("ROUTE_BWD", B.osdp_route_bwd, (a, a, 16, 1, a, 4, 16, 2, 0, 1, 1.0, a, 16)),
             ("EXPERT_PLAN", B.osdp_expert_plan, (a, 4, 2, 8, a, a)),
             ("EXPERT_DISPATCH", B.osdp_expert_dispatch, (a, a, a, None, None, 4, 2, 8, 64, a, None)),
             ("EXPERT_COMBINE", B.osdp_expert_combine, (a, a, a, None, 4, 2, 8, 64, a)),
             ("EXPERT_LINEAR_FWD", B.osdp_expert_linear_fwd, (a, a, a, 0, None, 4, 2, 8, 64, 64, 0, a, None, (a, 256))),
             ("EXPERT_LINEAR_BWD", B.osdp_expert_linear_bwd, (a, a, a, a, 0, None, 4, 2, 8, 64, 64, 0, a, a, 0, 0, 0, a, (a, 256)))]
    for name, call, args in calls:
        assert call(*args, stream=0) == 0 and first[-1] == DEFINES["CALL_" + name], name
    assert sorted(first) == sorted(v for n, v in DEFINES.items() if n.startswith("CALL_"))
