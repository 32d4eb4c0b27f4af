"""The policy update's command called as a function: from a program with arguments of its own."""
import sys

import pytest

from paper_2509_06980_amd import policy_update as pu


def test_main_takes_no_arguments_of_the_program_that_calls_it(monkeypatch):
    class Reached(Exception):
        pass

    def reached(*args, **kwargs):
        raise Reached(kwargs)

    monkeypatch.setattr(sys, "argv", ["serve.py", "--port", "80", "--muon"])
    monkeypatch.setattr(sys, "path", list(sys.path))
    monkeypatch.setattr(pu, "PolicyModel", reached)
    with pytest.raises(Reached) as e:
        pu.main()
    assert e.value.args[0]["fused"] is False
    with pytest.raises(Reached) as e:
        pu.main(["--fused"])
    assert e.value.args[0]["fused"] is True
    with pytest.raises(SystemExit):
        pu.main(["--port", "80"])
