"""The package where the marshalling extension is missing and cannot be built, or was built for another torch: everything works,
through ctypes."""
import os
import shutil
import subprocess
import sys
import textwrap

import pytest

HERE = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKAGE = "paper_2604_22782_b200"

WARNED = """
import warnings
with warnings.catch_warnings(record=True) as seen:
    warnings.simplefilter("always")
    import paper_2604_22782_b200 as skv
from paper_2604_22782_b200 import binding
assert any("ctypes" in str(w.message) for w in seen), seen
"""


def run(tmp_path, code, prepare=None):
    from paper_2604_22782_b200 import binding  # noqa: F401  (builds what is missing here)
    there = tmp_path / PACKAGE
    shutil.copytree(os.path.join(HERE, PACKAGE), there, ignore=shutil.ignore_patterns("*.so", "_build*", "__pycache__"))
    shutil.copytree(os.path.join(HERE, "include"), tmp_path / "include")
    os.symlink(os.path.join(HERE, PACKAGE, "libskv.so"), there / "libskv.so")
    os.utime(os.path.join(there, "libskv.so"))
    if prepare:
        prepare(there)
    env = dict(os.environ, CXX="/bin/false", PYTHONPATH=str(tmp_path))
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(code)], cwd=tmp_path, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_it_is_missing_and_cannot_be_built(tmp_path):
    run(tmp_path, WARNED + """
import torch
cache = skv.SkvCache([0, 0, 2], 2, 64, 16, 4, accounting_only=True)
assert cache.skv_layer_owner(1) == 0
one = torch.zeros(1, dtype=torch.int32)
try:
    cache.skv_plan_release(one[None], one, one, one, one, one)
except (binding.SkvError, ValueError):
    pass
else:
    raise SystemExit("nothing was raised")
""")


@pytest.mark.parametrize("content", [b"", b"no library"])
def test_it_cannot_be_loaded(tmp_path, content):
    run(tmp_path, WARNED, lambda there: (there / "_calls.so").write_bytes(content))


def test_it_was_built_for_another_torch(tmp_path):
    def prepare(there):
        shutil.copy(os.path.join(HERE, PACKAGE, "_calls.so"), there / "_calls.so")
    run(tmp_path, """
import torch
torch.__version__ = "1.0.0"
""" + WARNED + """
assert binding._calls.plan_release(1, None) is None
""", prepare)


@pytest.mark.gpu
def test_calls_give_the_same(tmp_path):
    run(tmp_path, WARNED + """
import torch
assert type(binding._calls) is binding._Declines
cache = skv.SkvCache([0, 0], 2, 64, 16, 8, allocate=True)
g = torch.Generator().manual_seed(1)
k, v = (torch.randn(40, 2, 64, generator=g).bfloat16().cuda() for _ in range(2))
q = torch.randn(40, 4, 64, generator=g).bfloat16().cuda()
table, lens, new = torch.full((1, 3), -1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([40], dtype=torch.int32, device="cuda")
free, n_free = torch.arange(8, dtype=torch.int32, device="cuda"), torch.tensor([8], dtype=torch.int32, device="cuda")
slots, pos = torch.empty(40, dtype=torch.int64, device="cuda"), torch.empty(40, dtype=torch.int32, device="cuda")
cu = torch.empty(2, dtype=torch.int32, device="cuda")
cache.skv_plan_step(table, lens, new, free, n_free, slots, cu, lens, n_free, positions=pos)
assert table.tolist() == [[7, 6, 5]] and cu.tolist() == [0, 40] and lens.item() == 40 and n_free.item() == 5
turned = torch.empty_like(q)
cache.skv_rope_append(0, skv.SkvRope([0.0] * 32), q, turned, k, v, pos, slots)
assert torch.equal(turned, q)
ws = torch.empty(cache.skv_decode_workspace_bytes(1, 4), dtype=torch.uint8, device="cuda")
rows, one = torch.empty_like(q), torch.empty_like(q[:1])
cache.skv_prefill_attn_window(1, q, cu, table, lens, rows, 40, 20, 3)
cache.skv_decode_attn_window(1, q[39:], table, lens, one, ws, 20, 3)
t = torch.arange(40)
seen = (t > 39 - 20) | (t < 3)
for h in range(4):
    w = torch.softmax((q[39, h].double().cpu() @ k[:, h // 2].double().cpu().T / 8).masked_fill(~seen, -float("inf")), 0)
    want = w @ v[:, h // 2].double().cpu()
    for got in (rows[39, h], one[0, h]):
        assert ((got.double().cpu() - want).abs() <= 2 ** -7 * (w @ v[:, h // 2].double().cpu().abs()) + 2 ** -8 * want.abs()).all()
assert cache.skv_get_status() == 0
""")
