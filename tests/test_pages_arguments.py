"""What H2OPages and H2ORotary refuse or accept, without a GPU."""
import os
import subprocess
import sys
import types

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def b():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2306_14048_b200 import binding

    return binding


# ---- pools ----
@pytest.mark.parametrize("shape", [(50, 16, 2, 128), (1, 16, 2, 128), (50, 16, 1, 64), (1, 8, 1, 64)])
def test_a_broadcast_pool_is_refused(b, shape):
    """Three strides of 0 mean dense to the library, so that rows would be written and read far behind the tensor."""
    one = torch.zeros(shape[3])
    for lead in ((1, 1, 1), (shape[0], 1, 1), (1, shape[1], 1), (1, 1, shape[2])):
        x = one.expand(*lead, shape[3]).contiguous().expand(shape)
        if all(s != 0 for s, n in zip(x.stride(), shape) if n > 1):
            continue
        with pytest.raises(ValueError):
            b._pool_strides(x, x)


def test_strides_of_pools(b):
    z = torch.zeros
    assert b._pool_strides(z(5, 16, 2, 64), z(5, 16, 2, 64)) == [2048, 128, 64, 1]
    heads = z(5, 2, 16, 64).transpose(1, 2)
    assert b._pool_strides(heads, heads) == [2048, 64, 1024, 1]
    both = z(5, 2, 16, 2, 64)
    assert b._pool_strides(both[:, 0], both[:, 1]) == [4096, 128, 64, 1]
    # strides that say nothing: one head, one page
    assert b._pool_strides(z(5, 16, 1, 64), z(5, 16, 1, 64)) == [1024, 64, 64, 1]
    assert b._pool_strides(z(1, 16, 2, 64), z(1, 16, 2, 64)) == [2048, 128, 64, 1]
    page = z(16, 2, 64)
    assert b._pool_strides(page.expand(1, 16, 2, 64), z(1, 16, 2, 64)) == [2048, 128, 64, 1]
    head = z(5, 16, 64).unsqueeze(2).expand(5, 16, 1, 64)
    assert b._pool_strides(head, head) == [1024, 64, 64, 1]
    for k, v in ((z(5, 16, 2, 64), heads), (z(5, 16, 2, 128)[..., ::2], z(5, 16, 2, 128)[..., ::2])):
        with pytest.raises(ValueError):
            b._pool_strides(k, v)


# ---- the extension that checks tensors ----
SCRIPT = """
import sys, types
sys.modules["paper_2306_14048_b200._pages"] = None  # nothing to import by that name
fake = types.ModuleType("paper_2306_14048_b200.build")
fake.pages_path = lambda: sys.argv[1]
sys.modules["paper_2306_14048_b200.build"] = fake
import paper_2306_14048_b200 as pkg
import torch
cfg, keep = pkg.make_config(2, 2, 64, pkg.H2O_F32, [4, 4], [4, 4])
assert pkg.h2o_cache_workspace_bytes(cfg) > 0
try:
    pkg.H2OStore(torch.zeros(8, 2, 64), torch.zeros(8, 2, 64))
except ValueError:  # (a CUDA tensor is needed)
    pass
for make in (lambda: pkg.H2ORotary(64), lambda: pkg.H2OPages(torch.zeros(1, 8, 1, 64), torch.zeros(1, 8, 1, 64))):
    try:
        make()
    except ImportError as e:
        assert "build.py" in str(e) and "_pages" in str(e), e
    else:
        raise AssertionError("made without the extension")
print("ALL WELL")
"""


@pytest.mark.parametrize("there", [False, True])
def test_the_other_classes_do_without_the_extension(b, tmp_path, there):
    """Missing, or one that does not load."""
    at = tmp_path / "_pages-torch9.so"
    if there:
        at.write_bytes(b"\x7fELF nothing")
    res = subprocess.run([sys.executable, "-c", SCRIPT, str(at)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "ALL WELL" in res.stdout, res.stderr[-2000:]


def test_the_extension_is_of_this_python_and_torch(b, monkeypatch):
    from paper_2306_14048_b200 import build

    here = build.pages_path()
    assert os.path.exists(here) and b._pages.__file__ == here
    monkeypatch.setattr(torch, "__version__", "9.9.9+cu999")
    other = build.pages_path()
    monkeypatch.undo()
    monkeypatch.setattr(build.sysconfig, "get_config_var", lambda name: ".cpython-399-x86_64-linux-gnu.so")
    assert len({here, other, build.pages_path()}) == 3 and "9.9.9" in other


def test_an_extension_for_another_torch_is_built(b, monkeypatch, tmp_path):
    """A tree whose extension belongs to another torch: build.py makes one for this torch, although no source is newer."""
    from paper_2306_14048_b200 import build

    at = tmp_path / os.path.basename(build.pages_path())
    made = []
    monkeypatch.setattr(build, "pages_path", lambda: str(at))
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **kw: made.append(cmd) or open(cmd[cmd.index("-o") + 1], "w").close() or types.SimpleNamespace(returncode=0))
    assert build.build_pages() == str(at) and at.exists() and len(made) == 1
    assert build.build_pages() == str(at) and len(made) == 1  # there now


# ---- streams ----
@pytest.mark.parametrize("call", ["apply", "append", "attend"])
def test_a_stream_of_another_device_is_refused(b, call):
    """Before anything runs: the library is not reached, and no stream becomes the current one."""
    other = types.SimpleNamespace(device_index=1, cuda_stream=0x1000)
    it = types.SimpleNamespace(_index=0, _at=0, _turn=(0, 0, 0, 0), _streams=set(), _note=None, n_heads=2, head_dim=64, format=b.H2O_F32, axes=1)
    kind = b.H2ORotary if call == "apply" else b.H2OPages
    x, i32 = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32)
    args = {"apply": (x, torch.zeros(3, dtype=torch.int64), x), "append": (x, x, i32.view(3, 1), i32), "attend": (x, i32.view(3, 1), i32, x, 9)}[call]
    with pytest.raises(ValueError, match="stream"):
        getattr(kind, call)(it, *args, stream=other)
