"""What bench.py prints: one JSON line that stays short however many shapes were timed."""
import json

import bench


def test_long_arrays_stay_out_of_the_line(tmp_path, capsys):
    rows = [[64, 64, 64, 1.0, 1.0]] * 5000
    line = {"metric": bench.METRIC, "value": 1.0, "e2e": {"value": 0.5}}
    bench.emit(line, {"grid_detail": {"rows": rows}, "skinny_shapes": []}, None)
    bench.emit(line, {"grid_detail": {"rows": rows}, "skinny_shapes": []}, str(tmp_path / "detail.json"))
    out = capsys.readouterr().out.splitlines()
    assert out == [json.dumps(line)] * 2
    assert json.loads((tmp_path / "detail.json").read_text())["grid_detail"]["rows"] == rows
