"""The paged calls' argument blocks in ctypes (the tests' own way to the C ABI) lie as include/sparsk.h has them: sizes and offsets as
a C compiler sees them (no GPU needed)."""
import ctypes
import os
import subprocess

import pytest

from paper_2603_09215_b200 import binding as B

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
BLOCKS = {"sparsk_page_map_args": B.PageMapArgs, "sparsk_page_pool": B.PagePool, "sparsk_paged_append_args": B.PagedAppendArgs,
          "sparsk_paged_attn_args": B.PagedAttnArgs, "sparsk_sample_args": B.SampleArgs, "sparsk_attn_args": B.AttnArgs}


@pytest.fixture(scope="module")
def offsets(tmp_path_factory):
    at = tmp_path_factory.mktemp("layout")
    lines = [f'P({c}, {name})' for c, t in BLOCKS.items() for name, *_ in t._fields_]
    lines += [f'printf("{c} %zu\\n", sizeof({c}));' for c in BLOCKS]
    names = ("FP32", "BF16", "FP16", "E4M3", "PAGES_SHORT", "PAGES_TABLE", "PAGES_ROWS", "PAGES_BAD", "PAGED_TIMEOUT")
    lines += [f'printf("{n} %d\\n", SPARSK_{n});' for n in names]
    (at / "layout.c").write_text('#include <stddef.h>\n#include <stdint.h>\n#include <stdio.h>\n#include "sparsk.h"\n'
                                 '#define P(T, F) printf("%s.%s %zu\\n", #T, #F, offsetof(T, F));\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.run(["gcc", "-I", INCLUDE, "-o", str(at / "layout"), str(at / "layout.c")], check=True)
    text = subprocess.run([str(at / "layout")], check=True, capture_output=True, text=True).stdout
    return {k: int(v) for k, v in (line.split() for line in text.splitlines())}, names


@pytest.mark.parametrize("c", BLOCKS)
def test_blocks_lie_as_the_header_has_them(offsets, c):
    t = BLOCKS[c]
    assert ctypes.sizeof(t) == offsets[0][c]
    for name, *_ in t._fields_:
        assert getattr(t, name).offset == offsets[0][f"{c}.{name}"], name


def test_codes_are_the_headers(offsets):
    for n in offsets[1]:
        assert getattr(B, n) == offsets[0][n], n
