"""Whoever needs no tensors needs no PyTorch: building, configurations, checks at the boundary and calls on host arrays."""
import os
import subprocess
import sys

import paper_2206_08888_amd as pp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(code):
    return subprocess.run([sys.executable, "-c", "import sys\nsys.modules['torch'] = None\n" + code], cwd=ROOT, capture_output=True, text=True)


def test_the_package_imports():
    r = _run("import paper_2206_08888_amd as pp\nfrom paper_2206_08888_amd import build\nprint(pp.make_config(1, 3, 1, (64, 64), 8, 100).P, pp.POP_EINVAL)")
    assert r.returncode == 0 and r.stdout.split() == ["1", str(pp.POP_EINVAL)], r.stderr


def test_structures_of_the_operators_are_there():
    r = _run("import ctypes\nimport paper_2206_08888_amd as pp\nprint(ctypes.sizeof(pp.pop_recurrence_io), pp.POP_BF16, len(pp.make_ns_config(3).coef))")
    assert r.returncode == 0 and r.stdout.split()[1:] == ["1", "16"], r.stderr


def test_operators_on_tensors_say_what_is_missing():
    r = _run("import paper_2206_08888_amd as pp\npp.Recurrence(1, 1, 1, 1)")
    assert r.returncode != 0 and "ModuleNotFoundError" in r.stderr and "torch" in r.stderr


def test_all_names_at_once():
    names = {}
    exec("from paper_2206_08888_amd import *", names)
    assert names["Muon"] is pp.Muon and names["pop_update"] is pp.pop_update and "import_module" not in names
    r = _run("from paper_2206_08888_amd import *\nprint(POP_F32, make_config)")
    assert r.returncode == 0, r.stderr


def test_every_name_is_found():
    for name in ("Recurrence", "Orthogonalizer", "Muon", "NS_COEF", "make_ns_config", "pop_sequence", "pop_muon_layer", "POP_F16", "operators"):
        assert getattr(pp, name) is not None and name in dir(pp)
