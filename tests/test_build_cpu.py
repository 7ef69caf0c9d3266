"""How many compilers build_damoe runs at once (nothing is compiled)."""
import pytest

from paper_2607_23099_amd import build


@pytest.mark.parametrize("jobs,most", [(None, 8), ("", 8), ("0", 8), ("3", 3), ("1", 1), ("64", 8), ("-1", 1)])
def test_workers(monkeypatch, tmp_path, jobs, most):
    asked = []

    class Pool(build.ThreadPoolExecutor):
        def __init__(self, workers):
            asked.append(workers)
            super().__init__(workers)

    if jobs is None:
        monkeypatch.delenv("MAX_JOBS", raising=False)
    else:
        monkeypatch.setenv("MAX_JOBS", jobs)
    monkeypatch.setattr(build, "ThreadPoolExecutor", Pool)
    monkeypatch.setattr(build, "_run", lambda cmd, verbose: None)
    monkeypatch.setattr(build, "_link", lambda *a, **k: None)
    monkeypatch.setattr(build.os, "cpu_count", lambda: 99)
    build.build_damoe()
    assert asked == [most]
