"""The argument checks of the 8-bit token cache's calls without a GPU: the C ABI's statuses through a
host driver (tests/qcache_validation_host.hip), the binding's structs against the header, and the
binding's own checks."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


@pytest.fixture(scope="module")
def fc():
    import paper_2604_24391_amd as fc
    fc.lib()
    return fc


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_statuses(fc, tmp_path):
    exe, lib = str(tmp_path / "qcache_validation"), fc.freqcache.LIB
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-result",
           os.path.join(ROOT, "tests", "qcache_validation_host.hip"), "-L" + os.path.dirname(lib),
           "-l:" + os.path.basename(lib), "-Wl,-rpath," + os.path.dirname(lib), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-4000:]
    env = dict(os.environ, HIP_VISIBLE_DEVICES="")      # never a device, even where one exists
    env.pop("FC_DEBUG", None)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120, env=env)
    assert run.returncode == 0 and "OK (0 failed expectations)" in run.stdout, run.stdout + run.stderr


def test_struct_layouts(fc, tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = [fc.freqcache.fc_qcache, fc.freqcache.fc_rope_axes, fc.freqcache.fc_qkv_rows]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "freqcache.h"', 'int main(void) {']
    for st in structs:
        lines.append(f'  printf("%zu\\n", sizeof({st.__name__}));')
        lines += [f'  printf("%zu\\n", offsetof({st.__name__}, {n}));' for n, _ in st._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ['  return 0;', '}']) + "\n")
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [x for st in structs for x in [ctypes.sizeof(st)] + [getattr(st, n).offset for n, _ in st._fields_]]


def test_cache_handle_checks(fc):
    """Shapes are checked before devices: a CPU tensor is refused for being one only when all else fits."""
    u8 = torch.uint8
    k, v, s = torch.zeros(2, 3, 128, 64, dtype=u8), torch.zeros(2, 3, 2, 64, 64, dtype=u8), torch.zeros(2, 3, 2)
    for args, word in (((k[0], v, s, s), "n_kv"), ((k[:, :, :100], v, s, s), "multiple"), ((k, k, s, s), "v is"), ((k, v, s[..., :1], s), "k_scale"),
                       ((k, v, s, s, torch.zeros(2, 3, 64)), "weight"), ((k, v, s, s), "GPU")):
        with pytest.raises(ValueError, match=word):
            fc.QCache(*args)
    with pytest.raises(ValueError):
        fc.QCache(k[:, :, :0], v[:, :, :0], s[..., :0], s[..., :0])


def test_rope_axes(fc):
    assert fc.RopeAxes().axes == 1 and fc.RopeAxes(1e4, (8, 8, 16)).axes == 3
    c = fc.RopeAxes(1e4, (8, 8, 16)).c()
    assert c.theta == 1e4 and list(c.section) == [8, 8, 16]
