"""A native binding of older sources is an error at import, not a silent return to slower calls; one for another torch is left out."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STALE = """
import importlib.util, sys, types
spec = importlib.util.spec_from_file_location("build_of_it", %r)
build = importlib.util.module_from_spec(spec)
spec.loader.exec_module(build)
name = "paper_2009_13062_amd._binding"
old = types.ModuleType(name)
old.built_for = build.binding_target()%s
old.bind = lambda *a: None
sys.modules[name] = old
import paper_2009_13062_amd as nf
print("native", nf._native is old)
"""


def imported(suffix):
    code = STALE % (os.path.join(ROOT, "paper_2009_13062_amd", "build.py"), suffix)
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)


def test_a_binding_of_older_sources_is_an_error():
    r = imported("")
    assert r.returncode != 0 and "bind_decoder" in r.stderr, r.stdout + r.stderr


def test_a_binding_for_another_torch_is_left_out():
    r = imported(" + ' of another'")
    assert r.returncode == 0 and "native False" in r.stdout, r.stdout + r.stderr
