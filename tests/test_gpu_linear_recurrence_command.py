"""The command of linear_recurrence.py at the ends of its arguments."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_single_step(capsys):
    from paper_1907_03329_amd import linear_recurrence
    linear_recurrence.main(["--batch", "16", "--channels", "32", "--steps", "1"])
    printed = capsys.readouterr().out
    assert "finite: True" in printed
    first, last = printed.split("mean squared error ")[1].split(" (")[0].split(" -> ")
    assert first == last


@pytest.mark.parametrize("steps", ["0", "-3"])
def test_no_steps_are_refused(steps):
    from paper_1907_03329_amd import linear_recurrence
    with pytest.raises(SystemExit):
        linear_recurrence.main(["--batch", "16", "--channels", "32", "--steps", steps])
