"""mq_sample's workspace on the host: how much is asked for, and that less is refused before any launch.  CPU only."""
import pytest

from test_draft_abi import FAKE, SCRATCH, lib, with_defaults  # noqa: F401


@pytest.mark.parametrize("type", [0, 1])
@pytest.mark.parametrize("rows,V", [(1, 8193), (2, 9000), (1, 1 << 20), (64, 151673), (573, 151673), (1 << 20, 8193)])
def test_too_little_is_refused(lib, rows, V, type):  # noqa: F811
    need = lib.mq_sample_workspace_bytes(rows, V)
    assert 0 < need <= 64 << 20
    call = with_defaults(lib.mq_sample, dict(x=FAKE, rows=rows, V=V, ld=V, type=type, u=FAKE, t=None, k=None, p=None, mp=None, tokens=FAKE, ws=FAKE, bytes=need - 1))
    assert call() == SCRATCH and call(k=FAKE) == SCRATCH and call(p=FAKE, mp=FAKE, t=FAKE) == SCRATCH
    assert call(bytes=0) == SCRATCH and call(ws=None) == SCRATCH and call(ws=None, bytes=0) == SCRATCH and call(ws=None, bytes=1 << 40) == SCRATCH


def test_what_is_asked_for(lib):  # noqa: F811
    need = lib.mq_sample_workspace_bytes
    assert all(need(rows, V) == 0 for rows in (1, 7, 1 << 20) for V in (1, 901, 8192))
    # a row of two parts: a Chunk of 16 bytes and 512 sums of 8 for each, then 512 masses, counts and the list of 4096 numbers
    row = 2 * (16 + 512 * 8) + 512 * 12 + 4096 * 8
    assert row <= need(1, 8193) <= row + 128 and need(5, 16384) == 5 * need(1, 8193)
    # as many rows as 64 MiB hold, and no more for more rows
    most = (64 << 20) // need(1, 8193)
    assert need(most, 8193) == need(most + 1, 8193) == need(1 << 20, 8193) == most * need(1, 8193)
