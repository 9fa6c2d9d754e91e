"""The package's import: the student operators' binding, which needs torch, is
loaded when one of its names is asked for."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ["ACTIVATIONS", "distill", "gated_backward", "gated_forward", "ops_check", "product_q8", "rms_norm",
         "rms_norm_backward", "rms_norm_q8"]


def _python(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return r.stdout.split()


def test_import_without_torch():
    """Packs' constants, configurations and the build need no torch."""
    out = _python("import sys; sys.modules['torch'] = None\n"
                  "import paper_2607_05380_gb300 as tp\n"
                  "print(tp.FP32, tp.TASKS['regression'])")
    assert out == ["1", "2"]


def test_import_does_not_load_torch():
    assert _python("import sys, paper_2607_05380_gb300; print('torch' in sys.modules)") == ["False"]


def test_operators_are_names_of_the_package():
    code = (f"import paper_2607_05380_gb300 as tp\nnames = {NAMES}\n"
            "assert all(n in dir(tp) for n in names)\n"
            "assert all(getattr(tp, n) is getattr(tp.ops, n) for n in names)\n"
            "from paper_2607_05380_gb300 import distill, rms_norm_q8\n"
            "assert distill is tp.distill\n"
            "try:\n    tp.no_such_name\nexcept AttributeError as e:\n    print('no_such_name' in str(e))")
    assert _python(code) == ["True"]
