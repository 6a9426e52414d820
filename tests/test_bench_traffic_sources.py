"""bench.py's measured traffic belongs to every source of the kernels it was taken with, headers too."""
import hashlib
import importlib.util
import json
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = ("fp8lin_gemm.hip", "fp8lin_amax_cast.hip", "fp8lin_fp8.h", "fp8lin_mm.h", "fp8lin_mm_256.h")


@pytest.mark.parametrize("changed", SOURCES)
def test_traffic_is_not_given_once_a_source_has_changed(changed, tmp_path, monkeypatch):
    spec = importlib.util.spec_from_file_location("bench_traffic", os.path.join(ROOT, "bench.py"))
    bench = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(bench)
    csrc = tmp_path / "paper_2309_17224_amd" / "csrc"
    csrc.mkdir(parents=True)
    (tmp_path / "profiles").mkdir()
    h = hashlib.sha256()
    for name in SOURCES:
        (csrc / name).write_bytes(name.encode())
        h.update(name.encode())
    (tmp_path / "profiles" / "hbm_traffic_w.json").write_text(
        json.dumps({"kernel_sources_sha256": h.hexdigest(), "bytes_per_launch": {"gemm_dw": 5}}))
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.measured_traffic("w", "gemm_dw") == 5
    (csrc / changed).write_bytes(b"changed")
    assert bench.measured_traffic("w", "gemm_dw") is None


def test_every_header_of_the_matmul_is_among_them():
    """What fp8lin_gemm.hip and fp8lin_amax_cast.hip include of the kernels themselves."""
    csrc = os.path.join(ROOT, "paper_2309_17224_amd", "csrc")
    seen, todo = set(), ["fp8lin_gemm.hip"]
    while todo:
        name = todo.pop()
        seen.add(name)
        for line in open(os.path.join(csrc, name)):
            inc = line.split('"')[1] if line.startswith('#include "') else ""
            if inc and os.path.exists(os.path.join(csrc, inc)) and inc not in seen:
                todo.append(inc)
    assert seen - {"fp8lin_internal.h"} <= set(SOURCES)
