"""Layouts and refusals, without a GPU, of the calls that decide what leaves the cache and of attention behind shared prefixes."""
import ctypes
import os
import subprocess

import pytest

from paper_2608_13263_b200 import binding as vt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_ctypes_layouts_match(tmp_path):
    structs = {"vtoken_heads": vt.Heads, "vtoken_attention_in": vt.AttentionIn, "vtoken_weights_in": vt.WeightsIn,
               "vtoken_select_in": vt.SelectIn, "vtoken_verify_in": vt.VerifyIn, "vtoken_shared_in": vt.SharedIn}
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "vtoken.h"', 'int main(void) {']
    for cname, cls in structs.items():
        lines.append(f'printf("{cname} %zu", sizeof({cname}));')
        lines += [f'printf(" %zu", offsetof({cname}, {f}));' for f, _ in cls._fields_]
        lines.append('printf("\\n");')
    lines += ['return 0; }']
    (tmp_path / "layout.c").write_text("\n".join(lines))
    exe = str(tmp_path / "layout")
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", exe,
                           str(tmp_path / "layout.c")])
    out = subprocess.check_output([exe], text=True).strip().splitlines()
    for line, (cname, cls) in zip(out, structs.items()):
        parts = line.split()
        assert parts[0] == cname and int(parts[1]) == ctypes.sizeof(cls)
        assert [int(x) for x in parts[2:]] == [getattr(cls, f).offset for f, _ in cls._fields_], cname
    assert (vt.PROB_BF16, vt.PROB_FP16, vt.PROB_F32) == (0, 1, 2)


def test_calls_without_a_context_are_refused():
    heads = vt.Heads(8, 2, 128, vt.KV_BF16, vt.KV_BF16, 0, 0)
    lib = vt.load()
    assert lib.vtoken_token_weights(None, heads, 0, vt.WeightsIn(), None) == vt.EINVAL
    assert lib.vtoken_select_victims(None, vt.SelectIn(), None) == vt.EINVAL
    assert lib.vtoken_verify_drafts(None, vt.VerifyIn(), None) == vt.EINVAL
    assert lib.vtoken_attention_shared(None, heads, 0, vt.AttentionIn(), vt.SharedIn(), None) == vt.EINVAL
    for size in (vt.vtoken_token_weights_workspace_bytes, vt.vtoken_attention_shared_workspace_bytes):
        with pytest.raises(vt.VtokenError) as e:
            size(None, heads, 1)
        assert e.value.code == vt.EINVAL
