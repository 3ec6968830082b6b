"""Tuning read from the environment at creation: values far outside what a launch can use (CPU)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CREATE = """
import paper_2609_31224_amd as a2t
for dtype in (a2t.A2T_F32, a2t.A2T_BF16, a2t.A2T_MX4):
    a2t.a2t_cache_destroy(a2t.a2t_cache_create(1, 2, 4, 1, 64, dtype, 16, 4, 8, flags=a2t.A2T_FLAG_HOST_ONLY))
print("created")
"""


@pytest.mark.parametrize("name,value", [("A2T_TARGET_WGS", v) for v in (-5, 0, 1, 1 << 30, (1 << 31) - 1)]
                         + [("A2T_SPLITS", -1), ("A2T_SPLITS", 1 << 30), ("A2T_MX4_ROWS", -16), ("A2T_MX4_ROWS", 17)])
def test_creation(name, value):
    p = subprocess.run([sys.executable, "-c", CREATE], cwd=ROOT, env={**os.environ, name: str(value)}, capture_output=True, text=True,
                       timeout=300)
    assert p.returncode == 0 and "created" in p.stdout, (p.returncode, p.stderr[-500:])
