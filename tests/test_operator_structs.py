"""The binding's parameter struct of the norms and rotation against the header."""
import ctypes
import re

import paper_2602_22603_gb300 as sq
from tests.test_abi import HEADER, _c_kind, _py_kind


def test_norm_rope_matches_the_header():
    text = re.sub(r"/\*.*?\*/", " ", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef\s+struct\s*\{([^}]*)\}\s*sq_norm_rope\s*;", text).group(1)
    fields = [re.fullmatch(r"\s*(.*?)(\w+)\s*", decl).groups() for decl in body.split(";") if decl.strip()]
    assert [f for _, f in fields] == [n for n, _ in sq.sq_norm_rope._fields_]
    for (ctype, name), (_, pytype) in zip(fields, sq.sq_norm_rope._fields_):
        assert _c_kind(ctype) == _py_kind(pytype), name


def test_norm_rope_defaults():
    p = sq.norm_rope()
    assert ctypes.sizeof(p) == ctypes.sizeof(sq.sq_norm_rope)
    assert not p.rope and not p.rot_dim and not p.q_weight and not p.k_weight
