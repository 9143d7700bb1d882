"""The structs of rotary positions and of the gradients' norm lie in memory as the header's do, and the calls refuse a NULL pool (no
GPU)."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2606_23087_b200 import binding as fp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs a C compiler")
def test_struct_layouts_match_the_header(tmp_path):
    structs = {"ft_rotary_config": fp.RotaryConfig, "ft_rotary_tensor": fp.RotaryTensor, "ft_grad_tensor": fp.GradTensor}
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
    cfg = fp.rotary_config([1.0], None, 2)
    assert lib.pool_rotary(None, 1, 256, 1, ctypes.byref(cfg), ctypes.byref(fp.RotaryTensor()), 1, None) == -1
    assert lib.pool_rms_norm(None, 1, 8, 256, 8, None, 0, fp.FT_F32, None, fp.FT_F32, 1e-5, None, 0, 256, 8, None, 0, None, 0, None, None) == -1
    assert lib.pool_rms_norm_grad_workspace(None, 1, 8, ctypes.byref(n)) == -1
    assert lib.pool_rms_norm_grad(None, 1, 8, 256, 8, 256, 8, None, 0, fp.FT_F32, None, fp.FT_F32, 256, 256, 8, None, 0, 256, 1 << 20, None) == -1
    assert lib.pool_grad_norm_workspace(None, ctypes.byref(n)) == -1
    assert lib.pool_grad_norm(None, ctypes.byref(fp.GradTensor()), 1, 1.0, None, None, None, None, 256, 1 << 20, None) == -1
    assert lib.pool_token_logprobs_workspace(None, 1, 8, 8, 0, ctypes.byref(n), ctypes.byref(n)) == -1
    assert lib.pool_token_logprobs(None, 1, 8, 8, 256, 8, 256, 8, 256, 1.0, 256, 256, 0, None, None, 256, 1 << 20, None) == -1


def test_a_rotary_config_keeps_its_host_arrays():
    cfg = fp.rotary_config([0.5, 0.25], [2, 1], 8, interleaved=True, inverse=True)
    assert (cfg.pairs, cfg.head_dim, cfg.interleaved, cfg.inverse) == (2, 8, 1, 1)
    assert np.ctypeslib.as_array(ctypes.cast(cfg.freq, ctypes.POINTER(ctypes.c_double)), (2,)).tolist() == [0.5, 0.25]
    assert np.ctypeslib.as_array(ctypes.cast(cfg.axis, ctypes.POINTER(ctypes.c_uint8)), (2,)).tolist() == [2, 1]
    with pytest.raises(ValueError):
        fp.rotary_config([1.0, 2.0], [0], 8)
