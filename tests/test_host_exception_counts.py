"""Where the entries of the delta rule, the scores and the distillation loss come to an allocation on the host that fails, and what they answer: those that launch
kernels with dynamic LDS reach the library's own table first, and the failure there is an error code of its own.  Of the others only that no exception
leaves them is shown; where there is no device the runtime's launch fails in front of any allocation of the library's (no GPU needed)."""
import os
import subprocess

import pytest

from paper_1901_10997_amd import binding as B
from tests.test_host_exceptions_scores import ENTRIES, SOURCE

WITH_TABLE = {"delta_walk", "delta_backward", "logprobs_top"}


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    B.load()
    at = tmp_path_factory.mktemp("host")
    source = SOURCE
    for old, new in (("static bool fails = false;", "static bool fails = false;\nstatic int failed = 0;"),
                     ("if (!p) throw std::bad_alloc();", "if (!p) {\n        ++failed;\n        throw std::bad_alloc();\n    }"),
                     (r'std::printf("%d\n", rc);', r'std::printf("%d %d\n", rc, failed);')):
        assert source.count(old) == 1, old
        source = source.replace(old, new)
    (at / "main.cpp").write_text(source)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(root, "include"), str(at / "main.cpp"), "-o", str(at / "main"), "-rdynamic", B.LIB_PATH,
                    "-Wl,-rpath," + os.path.dirname(B.LIB_PATH), "-Wl,--allow-shlib-undefined"], check=True)
    return str(at / "main")


@pytest.mark.parametrize("entry", ENTRIES)
def test_answer(program, entry):
    r = subprocess.run([program, str(ENTRIES.index(entry))], capture_output=True, text=True, timeout=120, env=dict(os.environ, HIP_VISIBLE_DEVICES="-1"))
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)
    rc, failed = map(int, r.stdout.split())
    if entry in WITH_TABLE:
        assert rc == B.LSTM_ERR_NOMEM and failed > 0
    else:
        assert rc in (B.LSTM_ERR_NOMEM, B.LSTM_ERR_LAUNCH)
