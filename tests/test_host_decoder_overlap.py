"""rnswino_block_tables refuses results that lie over what it reads, before anything is launched (no GPU: the addresses are never read).

Every workgroup reads all lengths while others write results, with no order among them: the last step's lens as this step's cached is right with one workgroup and not with more."""
import pytest

import paper_2007_12216_amd as rn

INVALID = -1
REQUESTS, FREE, WIDTH, TOKENS = 1000, 500, 8, 3000
# name -> (place among the arguments, bytes)
READ = {"cached": (0, 4 * REQUESTS), "fresh": (1, 4 * REQUESTS), "free_pages": (3, 4 * FREE)}
WRITTEN = {"table": (6, 4 * REQUESTS * WIDTH), "row_start": (8, 4 * REQUESTS + 4), "lens": (9, 4 * REQUESTS), "slots": (10, 8 * TOKENS), "positions": (11, 4 * TOKENS), "needed": (13, 4)}


def call(changes):
    args = [0, 0, REQUESTS, 0, FREE, 16, 0, WIDTH, 0, 0, 0, 0, TOKENS, 0]
    for i, (at, _) in enumerate((READ | WRITTEN).values()):
        args[at] = (i + 1) << 20  # far apart
    for at, v in changes.items():
        args[at] = v
    try:
        rn.rnswino_block_tables(*args)
    except rn.RnsWinoError as e:
        return e.code
    return 0


@pytest.mark.parametrize("written", sorted(WRITTEN))
@pytest.mark.parametrize("read", sorted(READ))
def test_results_over_what_is_read(read, written):
    (at_read, n_read), (at_written, n_written) = READ[read], WRITTEN[written]
    begin = 7 << 24
    for moved in (0, 4, n_read - 4, 4 - n_written):
        assert call({at_read: begin, at_written: begin + moved}) == INVALID, moved


@pytest.mark.parametrize("a,b", [(a, b) for a in sorted(WRITTEN) for b in sorted(WRITTEN) if a < b])
def test_results_over_each_other(a, b):
    begin = 7 << 24
    assert call({WRITTEN[a][0]: begin, WRITTEN[b][0]: begin}) == INVALID
