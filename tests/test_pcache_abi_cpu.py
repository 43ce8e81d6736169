"""The argument checks of the paged token cache's calls without a GPU: the C ABI's statuses through a host
driver (tests/pcache_validation_host.hip), once linked to the built library and once with the checks
compiled under the host sanitizers, the binding's struct against the header, and the binding's own
checks."""
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
@pytest.mark.parametrize("sanitized", [False, True])
def test_statuses(fc, tmp_path, sanitized):
    exe, lib = str(tmp_path / "pcache_validation"), fc.freqcache.LIB
    checks = []
    if sanitized:
        for what in ("address", "undefined"):
            checks += ["-Xarch_host", "-fsanitize=" + what]
        checks += ["-Xarch_host", "-fno-sanitize-recover=all", os.path.join(ROOT, "paper_2604_24391_amd", "csrc", "abi.hip")]
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-result",
           "-Wno-unused-value", *checks, os.path.join(ROOT, "tests", "pcache_validation_host.hip"), "-L" + os.path.dirname(lib),
           "-l:" + os.path.basename(lib), "-Wl,-rpath," + os.path.dirname(lib), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-4000:]
    env = dict(os.environ, HIP_VISIBLE_DEVICES="")      # never a device, even where one exists
    env.pop("FC_DEBUG", None)
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=0:halt_on_error=1"
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120, env=env)
    assert run.returncode == 0 and "OK (0 failed expectations)" in run.stdout, run.stdout + run.stderr


def test_struct_layout(fc, tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    st = fc.freqcache.fc_pcache
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "freqcache.h"', 'int main(void) {', '  printf("%zu\\n", sizeof(fc_pcache));']
    lines += [f'  printf("%zu\\n", offsetof(fc_pcache, {n}));' for n, _ in st._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ['  return 0;', '}']) + "\n")
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(st)] + [getattr(st, n).offset for n, _ in st._fields_]


def test_handle_checks(fc):
    """Shapes are checked before devices: a CPU tensor is refused for being one only when all else fits."""
    for args, word in (((0, 3, 5), "items"), ((2, 0, 5), "items"), ((2, 3, 0), "items"), ((1 << 15, 1 << 15, 5), "table"), ((2, 3, 5), "GPU")):
        with pytest.raises(ValueError, match=word):
            fc.PageState(torch.zeros(100, dtype=torch.int32), *args)

    class Pages:           # stands for a state on a GPU
        state, n_pages, max_pages, B = torch.zeros(100, dtype=torch.int32), 5, 3, 2
    bf = torch.bfloat16
    k, v = torch.zeros(5, 2, 32, 64, dtype=bf), torch.zeros(5, 2, 4, 64, 8, dtype=bf)
    for a, b, word in ((k[0], v, "n_kv"), (k[:4], v, "pages"), (k, k, "v is"), (k, v[:, :, :3], "v is"), (k[:, :, :20], v, "pages of 20"), (k, v, "GPU")):
        with pytest.raises(ValueError, match=word):
            fc.PCache(a, b, Pages)


def test_state_bytes(fc):
    assert fc.pcache_state_bytes(3, 3, 5) == 68 and fc.pcache_state_bytes(0, 3, 5) == 0


@pytest.fixture
def on_cpu(fc, monkeypatch):
    """Handles over CPU tensors: the check that refuses them is left out."""
    monkeypatch.setattr(fc.freqcache, "_ptr", lambda t, dtype, numel, name: t.data_ptr())


def test_rows_of_a_table_with_entries_that_are_no_page(fc, on_cpu):
    """Entries below 0 and beyond the pool stand for no page: their rows are 0."""
    n_kv, R, hd, P = 2, 16, 64, 5
    state = fc.PageState.alloc(2, 4, P, device="cpu")
    c = fc.PCache.alloc(state, n_kv, hd, R)
    g = torch.Generator().manual_seed(1)
    for t in (c.k, c.v):
        t.copy_(torch.randn(t.shape, generator=g))
    state.table.copy_(torch.tensor([[3, P, -7, P - 1], [2 ** 31 - 1, -2 ** 31, 0, 77]], dtype=torch.int32))
    by_rows = c.v.transpose(-1, -2).reshape(c.k.shape)
    for b, row in enumerate([[3, None, None, P - 1], [None, None, 0, None]]):
        for pool, values in ((c.k, False), (by_rows, True)):
            want = torch.cat([torch.zeros(n_kv, R, hd, dtype=torch.bfloat16) if p is None else pool[p] for p in row], 1)
            assert torch.equal(c.rows(b, values), want)


def test_layers_descriptors_after_the_state_has_moved(fc, on_cpu):
    """Every layer's descriptor names the state's memory, also where a call on one layer alone has renewed its own."""
    state = fc.PageState.alloc(2, 4, 9, device="cpu")
    caches = [fc.PCache.alloc(state, 1, 64, 16) for _ in range(3)]
    size = ctypes.sizeof(fc.freqcache.fc_pcache)

    def states():
        raw, n, pages = fc.freqcache._pcaches(-1, caches)      # (-1: a CPU tensor's device)
        assert n == 3 and pages is state
        return {fc.freqcache.fc_pcache.from_buffer_copy(raw, size * i).state for i in range(n)}
    assert states() == {state.state.data_ptr()}
    for renewed in (0, 2):
        state.state.set_(state.state.clone())
        caches[renewed].c()
        assert states() == {state.state.data_ptr()}
