"""What the binding needs in order to load: the attention's calls the CUDA library alone, the short calls the compiled part too."""
import os
import subprocess
import sys

import paper_2603_06588_b200

PKG = os.path.dirname(os.path.abspath(paper_2603_06588_b200.__file__))

# A handle as HookAttn makes it, without the device that hook_attn_create asks for.
HANDLE = """
import torch
from paper_2603_06588_b200 import binding
lib = binding.load_library()
assert lib.hook_attn_prefill(None, None, None) == lib.hook_attn_decode(None, None, None) == binding.HOOK_ATTN_ERR_INVALID_ARG
assert binding.strerror(0) == "ok"
eng = binding.HookAttn.__new__(binding.HookAttn)
eng._lib, eng._h, eng._index, eng._marshal, eng._calls = lib, None, 0, binding._compiled, dict.fromkeys(binding._AROUND, 0)
"""
CALLS = """
t = torch.zeros(1, 1)
refused = 0
for call in (lambda: eng.hook_adjust_logits(t), lambda: eng.hook_cache_free(t, t, t, t), lambda: eng.hook_cache_copy_pages([], t)):
    try:
        call()
    except ImportError as e:
        assert "csrc.build" in str(e), e
        refused += 1
assert refused == 3
"""


def _run(tmp_path, code, compiled):
    """Runs ``code`` on a copy of the package, with or without the compiled part."""
    copy = tmp_path / "paper_2603_06588_b200"
    copy.mkdir()
    for name in os.listdir(PKG):
        if name.endswith((".py", ".so")) and (compiled or not name.startswith("_marshal")):
            os.symlink(os.path.join(PKG, name), copy / name)
    _again(tmp_path, code)


def _again(tmp_path, code):
    got = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, env=dict(os.environ, PYTHONPATH=str(tmp_path)), capture_output=True, text=True,
                         timeout=300)
    assert got.returncode == 0, got.stderr[-2000:]


def test_the_attention_loads_without_the_compiled_part(tmp_path):
    _run(tmp_path, HANDLE + CALLS, compiled=False)


def test_with_the_compiled_part_the_short_calls_are_there(tmp_path):
    _run(tmp_path, HANDLE + "assert callable(eng._marshal.rope_append) and eng._marshal.__file__.endswith('.so')\n", compiled=True)


def test_a_compiled_part_for_another_torch_is_refused(tmp_path):
    """Its calls raise, and the build sees that it has to be made again."""
    other = "import torch\ntorch.__version__ = '1.0.0'\n"
    stale = ("from paper_2603_06588_b200.csrc import build\nbuild._newer = lambda deps, target: False\nassert build.needs_build() is %s\n"
             "try:\n    from paper_2603_06588_b200 import _marshal\nexcept ImportError as e:\n    assert 'torch' in str(e)\nelse:\n    assert not %s\n")
    _run(tmp_path, other + HANDLE + CALLS, compiled=True)
    (tmp_path / "paper_2603_06588_b200" / "csrc").mkdir()
    for name in ("__init__.py", "build.py"):
        os.symlink(os.path.join(PKG, "csrc", name), tmp_path / "paper_2603_06588_b200" / "csrc" / name)
    _again(tmp_path, other + stale % (True, True))
    _again(tmp_path, stale % (False, False))
