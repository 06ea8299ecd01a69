"""What the command of the attention half of a layer refuses, before it touches a GPU."""
from __future__ import annotations

import pytest

from paper_2412_17560_amd import attention_layer


@pytest.mark.parametrize("tokens", ["0", "-3"])
def test_no_tokens_are_refused(monkeypatch, capsys, tokens):
    monkeypatch.setattr("sys.argv", ["attention_layer", "--tokens", tokens])
    with pytest.raises(SystemExit) as stop:
        attention_layer.main()
    assert stop.value.code == 2 and "--tokens" in capsys.readouterr().err
