"""CPU checks of scored routing at the edges of its contract: what can be seen in the source, sizes, and argument checks that end
before a launch."""
import os
import re

import paper_2506_14435_amd as M


def test_range_checked_loads_carry_their_whole_offset_in_the_lane():
    """route.hip reads tokens behind the last one as zeros through the range check of a buffer load, in which a scalar offset has
    no part: with the row of a token in it, a batch of one token read up to 31 rows behind x."""
    src = open(os.path.join(os.path.dirname(M.LIB_PATH), "csrc", "route.hip")).read()
    loads = re.findall(r"raw_buffer_load_b128\((.*?)\);", src)
    assert len(loads) == 2
    for args in loads:
        assert args.endswith(", 0, 0"), args
