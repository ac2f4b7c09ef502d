"""CPU-side checks of the operators between hidden states and features: the argument structs of the binding have the header's
layout, and calls without a context are refused."""
import ctypes as C
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def binding():
    from paper_2211_00839_b200 import build
    build.build()
    from paper_2211_00839_b200 import binding as b
    return b


def test_argument_structs_match_the_header(binding, tmp_path):
    header = open(os.path.join(ROOT, "include", "rcd.h")).read()
    pairs = {"rcd_norm_args": binding.RcdNormArgs, "rcd_norm_back_args": binding.RcdNormBackArgs, "rcd_linear_args": binding.RcdLinearArgs,
             "rcd_linear_back_args": binding.RcdLinearBackArgs}
    lines, names = [], {}
    for name, cls in pairs.items():
        body = re.search(r"typedef struct \{((?:(?!typedef struct).)*?)\} %s;" % name, header, re.S).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = [f for decl in body.split(";") if decl.strip() for f in re.findall(r"(\w+)\s*(?:,|$)", decl.strip())]
        assert len(fields) == len(cls._fields_), (name, fields)
        names[name] = fields
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, f) for f in fields] + ['printf("%%zu\\n", sizeof(%s));' % name]
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
    consts = dict(re.findall(r"\b(RCD_(?:ELEM|ACT)_\w+) = (\d+)", header))
    assert len(consts) == 9
    for name, value in consts.items():
        assert getattr(binding, name) == int(value)


def test_calls_without_a_context_are_refused(binding):
    lib, need = binding.lib, C.c_size_t()
    assert lib.rcd_rms_norm(None, C.byref(binding.RcdNormArgs()), None) == 1
    assert lib.rcd_quantize_rows(None, None, 1, 1, 1, 1, None, 1, None, None) == 1
    assert lib.rcd_rms_norm_backward(None, C.byref(binding.RcdNormBackArgs()), None, 0, None) == 1
    assert lib.rcd_rms_norm_backward_workspace_bytes(None, None, C.byref(need)) == 1
    assert lib.rcd_linear(None, C.byref(binding.RcdLinearArgs()), None, 0, None) == 1
    assert lib.rcd_linear_workspace_bytes(None, None, C.byref(need)) == 1
    assert lib.rcd_linear_backward(None, C.byref(binding.RcdLinearBackArgs()), None, 0, None) == 1
    assert lib.rcd_linear_backward_workspace_bytes(None, None, C.byref(need)) == 1
