"""The binding's structs of the operator calls lie in memory as the header's do, and the calls refuse a NULL pool (no GPU)."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2606_23087_b200 import binding as fp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs a C compiler")
def test_struct_layouts_match_the_header(tmp_path):
    structs = {"ft_adamw_tensor": fp.AdamwTensor, "ft_adamw_config": fp.AdamwConfig}
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "flowpool.h"', "int main(void) {"]
    for name, cls in structs.items():
        lines.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'  printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    (tmp_path / "layout.c").write_text("\n".join(lines + ["  return 0;", "}"]))
    exe = str(tmp_path / "layout")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "layout.c"), "-o", exe])
    got = dict(line.rsplit(" ", 1) for line in subprocess.check_output([exe], text=True).splitlines())
    exp = {}
    for name, cls in structs.items():
        exp[name] = str(ctypes.sizeof(cls))
        exp.update({f"{name}.{f}": str(getattr(cls, f).offset) for f, _ in cls._fields_})
    assert got == exp


def test_calls_without_a_pool_are_refused():
    lib = fp.lib()
    n = ctypes.c_uint64()
    tensor, cfg = fp.AdamwTensor(), fp.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=1)
    assert lib.pool_layer_norm(None, 1, 8, 256, 8, fp.FT_F32, None, None, fp.FT_F32, 1e-5, 256, 8, None, None, None) == -1
    assert lib.pool_layer_norm_grad_workspace(None, 1, 8, ctypes.byref(n)) == -1
    assert lib.pool_token_loss_workspace(None, 1, 8, 8, 0, fp.FT_F32, ctypes.byref(n), ctypes.byref(n)) == -1
    assert lib.pool_token_loss(None, 1, 8, 8, 256, 8, 256, 8, 256, 256, 256, 256, 1 << 20, None) == -1
    assert lib.pool_adamw_step(None, ctypes.byref(tensor), 1, ctypes.byref(cfg), None) == -1
