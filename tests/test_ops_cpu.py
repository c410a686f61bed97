"""CPU-side checks of the operators' boundary: every symbol that include/asd_ops.h declares is exported and bound, the
argument structures have the header's layout, and nothing computes without a device."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "asd_ops.h")
STRUCTS = {"asd_rmsnorm_args": "_Norm", "asd_rmsnorm_backward_args": "_NormBackward", "asd_quantize_args": "_Quantize",
           "asd_matmul_i8_args": "_MatmulI8", "asd_gated_mlp_args": "_GatedMlp", "asd_gated_mlp_backward_args": "_GatedMlpBackward"}


@pytest.fixture(scope="module")
def lib():
    from paper_2505_03983_b200 import build
    build.build()
    from paper_2505_03983_b200 import operators
    return operators._library()


def test_every_declared_symbol_is_exported_and_bound(lib):
    from paper_2505_03983_b200 import OPS_SYMBOLS
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(asd_[a-z_0-9]+)\s*\(", text)))
    assert sorted(OPS_SYMBOLS) == declared
    for name in declared:
        assert hasattr(lib, name), name


def test_structures_match_the_header(tmp_path):
    """sizeof and every offsetof, as the host C compiler lays the header's structures out."""
    from paper_2505_03983_b200 import operators as o
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    lines = []
    for name, py in STRUCTS.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in getattr(o, py)._fields_]
    src = tmp_path / "layout.c"
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"asd_ops.h\"\nint main(void) {" + "\n".join(lines) + "return 0;}\n")
    exe = str(tmp_path / "layout")
    subprocess.run([cc, "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    said = dict(line.split() for line in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines())
    for name, py in STRUCTS.items():
        cls = getattr(o, py)
        assert int(said[name]) == C.sizeof(cls), name
        for f in cls._fields_:
            assert int(said[f"{name}.{f[0]}"]) == getattr(cls, f[0]).offset, (name, f[0])


def test_null_handles_are_refused(lib):
    from paper_2505_03983_b200 import operators as o
    for name, cls in (("add_rmsnorm", o._Norm), ("add_rmsnorm_backward", o._NormBackward), ("quantize_i8", o._Quantize),
                      ("matmul_i8", o._MatmulI8), ("gated_mlp_forward", o._GatedMlp), ("gated_mlp_backward", o._GatedMlpBackward)):
        assert getattr(lib, "asd_" + name)(None, C.byref(cls()), None) == 1
        assert b"handle" in lib.asd_ops_last_error()
    assert lib.asd_ops_check(None, None) == 1 and lib.asd_ops_create(None) == 1
    lib.asd_ops_destroy(None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the no-device behaviour")
def test_no_device_means_error_not_fallback(lib):
    from paper_2505_03983_b200 import AsdError, AsdOps, default_ops
    h = C.c_void_p()
    assert lib.asd_ops_create(C.byref(h)) == 4 and not h.value and b"no CUDA device" in lib.asd_ops_last_error()
    for make in (AsdOps, default_ops):
        with pytest.raises(AsdError) as e:
            make()
        assert e.value.status == 4
