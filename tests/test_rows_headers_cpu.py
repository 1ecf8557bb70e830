"""The native module ``_rows`` of a PyTorch whose headers name fewer types."""
import os
import re

from paper_2608_06146_amd import build


def test_no_type_of_scales(monkeypatch, tmp_path):
    """Headers without Float8_e8m0fnu: the module builds, without a warning, for the calls that need no scales."""
    rows = os.path.join(build.PKG, build.ROWS_SOURCE)
    with open(rows) as f:
        torch_headers = re.findall(r"^#include <(?:ATen|c10|torch)/.*$", f.read(), re.M)
    assert torch_headers
    hidden = [f"#define {name} not_a_type_of_this_pytorch" for name in ("Float8_e8m0fnu", "kFloat8_e8m0fnu")]
    source = tmp_path / "rows.cpp"
    source.write_text("\n".join(torch_headers + hidden + [f'#include "{rows}"', ""]))
    monkeypatch.setattr(build, "ROWS_SOURCE", str(source))
    monkeypatch.setattr(build, "BUILD", str(tmp_path))
    out = tmp_path / "_rows.so"
    assert build._compile_rows(build.hipcc(), str(out), force=True) and out.exists()
