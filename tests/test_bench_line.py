"""The benchmark's result is one line on standard output that the last few KB of it hold whole; its rows are a line on standard error."""
import json
import sys

import bench


def test_the_line_is_short_and_the_rows_are_apart(monkeypatch, capsys):
    rows = {f"row{i}": {"tops": 1000.0 + i, "ms": 0.1} for i in range(500)}
    monkeypatch.setattr(bench, "run_ours", lambda *_: {"metric": "m", "value": 1.5, "unit": "TOPS", "rows": dict(rows), "cpu_baseline": {"value": 0.1}})
    monkeypatch.setattr(sys, "argv", ["bench.py"])
    monkeypatch.delenv("WORLD_SIZE", raising=False)
    bench.main()
    out, err = capsys.readouterr()
    assert out.count("\n") == 1 and len(out) < 2500 and json.loads(out) == {"metric": "m", "value": 1.5, "unit": "TOPS", "cpu_baseline": {"value": 0.1}}
    assert json.loads(err.strip().splitlines()[-1]) == {"rows": rows}
