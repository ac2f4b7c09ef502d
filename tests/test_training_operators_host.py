"""CPU-side checks of the head's loss and the orthogonalised update: argument structs against the header, refusals without a context, and the order in
which a product's tiles are walked through."""
import ctypes as C
import os
import re
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def binding():
    from paper_2211_00839_b200 import build
    build.build()
    from paper_2211_00839_b200 import binding as b
    return b


def test_argument_structs_match_the_header(binding, tmp_path):
    header = open(os.path.join(ROOT, "include", "rcd.h")).read()
    pairs = {"rcd_cross_entropy_args": binding.RcdCrossEntropyArgs, "rcd_cross_entropy_back_args": binding.RcdCrossEntropyBackArgs,
             "rcd_orthogonalize_args": binding.RcdOrthogonalizeArgs}
    lines, names = [], {}
    for name, cls in pairs.items():
        body = re.search(r"typedef struct \{((?:(?!typedef struct).)*?)\} %s;" % name, header, re.S).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        names[name] = [f for decl in body.split(";") if decl.strip() for f in re.findall(r"(\w+)\s*(?:,|$)", decl.strip())]
        assert len(names[name]) == len(cls._fields_), (name, names[name])
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, f) for f in names[name]] + ['printf("%%zu\\n", sizeof(%s));' % name]
    src = tmp_path / "layout.c"
    src.write_text('#include "rcd.h"\n#include <stdio.h>\nint main(void) {\n%s\nreturn 0; }\n' % "\n".join(lines))
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], check=True, stdout=subprocess.PIPE, text=True).stdout.split()]
    at = 0
    for name, cls in pairs.items():
        for field, (mine, _) in zip(names[name], cls._fields_):
            assert re.sub(r"_dev|_or_null", "", field) == mine, (name, field, mine)
            assert got[at] == getattr(cls, mine).offset, (name, field)
            at += 1
        assert got[at] == C.sizeof(cls), name
        at += 1


def test_calls_without_a_context_are_refused(binding):
    lib, need = binding.lib, C.c_size_t()
    assert lib.rcd_linear_cross_entropy(None, C.byref(binding.RcdCrossEntropyArgs()), None, 0, None) == 1
    assert lib.rcd_linear_cross_entropy_workspace_bytes(None, None, C.byref(need)) == 1
    assert lib.rcd_linear_cross_entropy_backward(None, C.byref(binding.RcdCrossEntropyBackArgs()), None, 0, None) == 1
    assert lib.rcd_linear_cross_entropy_backward_workspace_bytes(None, None, C.byref(need)) == 1
    assert lib.rcd_orthogonalize(None, C.byref(binding.RcdOrthogonalizeArgs()), None, 0, None) == 1
    assert lib.rcd_orthogonalize_workspace_bytes(None, None, C.byref(need)) == 1


def test_every_tile_is_walked_through_once(tmp_path):
    exe = str(tmp_path / "walk")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2211_00839_b200", "csrc"), "-I", "/usr/local/cuda/include", os.path.join(HERE, "product_walk.cpp"), "-o", exe],
                   check=True)
    subprocess.run([exe], check=True)
