"""As test_token_memory.py, for lists of rows longer than one launch has workgroups for: the norms' kernel looks one row ahead, past the
end of the list for the last ones."""
import pytest

from paper_2308_15949_amd import binding as B
from test_memory_bounds import Call, in_a_process_of_its_own, lib  # noqa: F401  (lib: the fixture that builds the sources for the host)
from test_token_memory import norm

CASES = {
    "wave": (16384 + 21, 8, B.BF16, B.NORM_RMS, B.E4M3, 8, 3, False),
    "threads_256": (4096 + 3, 1032, B.BF16, B.NORM_RMS, B.BF16, 8, 2, True),
    "threads_1024": (1024 + 2, 8200, B.BF16, B.NORM_LAYER, B.E4M3, 8, 0, False),
}


@pytest.mark.parametrize("front", [0, 1])
@pytest.mark.parametrize("name", CASES)
def test_rows_ahead_stay_inside_their_buffers(lib, name, front, capfd):  # noqa: F811
    def body():
        norm(Call(lib, front), *CASES[name])
    in_a_process_of_its_own(body, capfd)
