"""The package's names are those of the binding, at any time."""
import subprocess
import sys

import pytest

import paper_2604_18616_amd as package
from paper_2604_18616_amd import binding

NAMES = ["attn_fwd", "gemm_bf16", "moe_ffn_fp8", "rope_bf16", "rope_frequencies", "KvFp8Cache", "kv_fp8_cache", "kv_fp8_write", "kv_fp8_read", "attn_kv_fp8",
         "moe_workspace_bytes", "load_library", "attn_fwd_flops", "strerror", "version", "AttnError"]


@pytest.mark.parametrize("name", NAMES)
def test_a_replaced_function_is_found_through_the_package(name, monkeypatch):
    """Before, with and after the replacement: a program that measures calls, or takes them elsewhere, puts its own in the binding."""
    own = getattr(binding, name)
    assert getattr(package, name) is own
    other = lambda *a, **kw: None
    monkeypatch.setattr(binding, name, other)
    assert getattr(package, name) is other
    monkeypatch.undo()
    assert getattr(package, name) is own


def test_names_that_are_not_there():
    with pytest.raises(AttributeError):
        package.attn_bwd
    assert all(hasattr(package, name) or name == "inputs" for name in package.__all__)


def test_the_first_access_imports_the_binding():
    """Importing the package loads neither the binding nor torch; a name does."""
    code = ("import sys, paper_2604_18616_amd as p\n"
            "assert 'paper_2604_18616_amd.binding' not in sys.modules and 'torch' not in sys.modules\n"
            "f = p.attn_fwd\n"
            "assert f is sys.modules['paper_2604_18616_amd.binding'].attn_fwd and p.attn_fwd is f\n")
    subprocess.check_call([sys.executable, "-c", code], cwd=package.__path__[0] + "/..")


def test_a_name_may_be_set_on_the_package_itself(monkeypatch):
    other = lambda *a, **kw: None
    monkeypatch.setattr(package, "attn_fwd", other)
    assert package.attn_fwd is other and binding.attn_fwd is not other
