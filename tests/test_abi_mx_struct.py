"""The struct of a cache in 8 and 4 bits as a C compiler lays it out from the header,
and as the tests and other languages' callers write it down (no GPU)."""
import ctypes
import os
import subprocess

from tests.test_abi_mx import Cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = dict(k="k", v="v", ks="k_scale", vs="v_scale", ps="page_stride", ss="slot_stride",
             hs="head_stride", sp="scale_page", sl="scale_slot", sh="scale_head", pages="n_pages",
             page="page", heads="kv_heads", dim="dim", format="format")


def test_layout(tmp_path):
    assert sorted(NAMES) == sorted(n for n, _ in Cache._fields_)
    lines = [f'printf("{x} %zu %zu\\n", offsetof(pair_mx_cache, {y}), sizeof(((pair_mx_cache*)0)->{y}));'
             for x, y in NAMES.items()]
    source, exe = tmp_path / "layout.c", tmp_path / "layout"
    source.write_text('#include <stdio.h>\n#include "pair.h"\nint main(void) {\n' + "\n".join(lines)
                      + '\nprintf("all 0 %zu\\n", sizeof(pair_mx_cache));\nreturn 0;\n}\n')
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I" + os.path.join(ROOT, "include"),
                    "-o", str(exe), str(source)], check=True, capture_output=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    seen = {x: (int(at), int(size)) for x, at, size in (line.split() for line in out.splitlines())}
    assert seen.pop("all") == (0, ctypes.sizeof(Cache))
    for name, _ in Cache._fields_:
        f = getattr(Cache, name)
        assert seen[name] == (f.offset, f.size), name
