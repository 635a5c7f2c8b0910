"""A rule that the packed forward's source keeps, checked on its text (no GPU, no compiler)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_07590_amd", "csrc")


def test_lanes_that_exchange_rows_through_lds_have_a_fence_between():
    """Rows are parked as pieces of one type by one lane and read as another type by others of the wave: stores and reads of them, in the order of
    the source, never follow one another without wave_sync() between."""
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(os.path.join(CSRC, "packed_fwd.hip")).read(), flags=re.S)
    tail = text[text.index("auto send = ["):text.index("packed_fwd_merge_kernel")]
    body = tail[tail.index("};"):]                       # behind the reader's own definition
    events = re.findall(r"\bplace\(|\bsend\(|\bwave_sync\(\)", body)
    assert events.count("place(") == 2 and events.count("send(") == 2
    last = None
    for e in events:
        if e == "wave_sync()":
            last = None
        else:
            assert last is None or last == e, events
            last = e
