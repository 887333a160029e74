"""The binding's compiled marshalling has torch's and Python's memory layouts in it: it is used where it was
built for these, and nowhere else."""
import os
import shutil
import subprocess
import sys
import sysconfig

import pytest
import torch

from paper_1806_08054_b200 import binding, build

PACKAGE = os.path.dirname(os.path.abspath(build.__file__))
EXT = sysconfig.get_config_var("EXT_SUFFIX")


def test_its_name_says_what_it_was_built_for(monkeypatch):
    path = build.marshal_path()
    assert torch.__version__ in path and path.endswith(EXT)
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert build.marshal_path() != path and not os.path.exists(build.marshal_path())
    monkeypatch.delitem(sys.modules, "paper_1806_08054_b200._marshal", raising=False)
    with pytest.raises(ImportError):
        build.load_marshal()


# One that was built for something else: it imports, and what it says is wrong.
OTHER = r"""
#include <Python.h>
static PyObject* wrong(PyObject* self, PyObject* args) { return PyLong_FromLong(13); }
static PyMethodDef methods[] = {{"matrix", wrong, METH_VARARGS, 0}, {"size", wrong, METH_VARARGS, 0}, {"vector", wrong, METH_VARARGS, 0}, {0}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", 0, -1, methods};
PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
"""
ASK = """
import torch
from paper_1806_08054_b200 import binding
assert binding._vector(torch.zeros(5), torch.float32, 5, "some", -1) != 13
assert (binding._matrix, binding._size, binding._vector) == binding._in_python
"""


def test_one_that_was_built_for_something_else_is_left(tmp_path):
    cc = os.environ.get("CC") or shutil.which("gcc")
    headers = sysconfig.get_paths()["include"]
    if not cc or not os.path.exists(os.path.join(headers, "Python.h")):
        pytest.skip("no C compiler or headers of Python")
    package = tmp_path / "paper_1806_08054_b200"
    package.mkdir()
    for name in os.listdir(PACKAGE):
        if name.endswith(".py"):
            shutil.copy(os.path.join(PACKAGE, name), package)
    (tmp_path / "other.c").write_text(OTHER)
    names = ["_marshal.so", os.path.basename(build.marshal_path()).replace(torch.__version__, "0.0.1")]
    subprocess.check_call([cc, "-shared", "-fPIC", "-I" + headers, str(tmp_path / "other.c"), "-o", str(package / names[0])])
    shutil.copy(package / names[0], package / names[1])
    env = dict(os.environ, PYTHONPATH=str(tmp_path))
    run = subprocess.run([sys.executable, "-c", ASK], env=env, cwd=tmp_path, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]


def test_the_one_for_this_torch_is_used():
    if not build.build_marshal():
        pytest.skip("no headers of Python or torch")
    module = build.load_marshal()
    assert module.__file__ == build.marshal_path()
    assert binding._in_python[2](torch.zeros(5), torch.float32, 5, "some", -1) != 13
