"""The binding's tables as they stand in the source: what a name means is said once."""
from __future__ import annotations

import ast
import os
import re

from paper_2505_11254_amd import binding


def test_no_key_of_a_table_stands_twice():
    """(Python keeps the last of two equal keys of a dictionary, without a word)"""
    tree = ast.parse(open(binding.__file__).read())
    for table in (x for x in ast.walk(tree) if isinstance(x, ast.Dict)):
        keys = [k.value for k in table.keys if isinstance(k, ast.Constant)]
        assert len(keys) == len(set(keys)), sorted(k for k in set(keys) if keys.count(k) > 1)


def test_signatures_are_the_headers():
    """Each entry point that returns da_status: as many arguments, of the same kinds."""
    header = open(os.path.join(os.path.dirname(os.path.dirname(binding.__file__)), "include", "delta_attn.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    kinds = {"int": "i", "int64_t": "l", "size_t": "z", "float": "f", "unsigned": "u", "uint32_t": "u"}
    seen = set()
    for name, args in re.findall(r"\bda_status\s+(\w+)\s*\(([^)]*)\)\s*;", header):
        sig = "".join("p" if "*" in a else kinds[a.split()[-2]] for a in args.split(","))
        if name in binding.SIGNATURES:
            assert binding.SIGNATURES[name] == sig, name
            seen.add(name)
    assert seen == set(binding.SIGNATURES)
