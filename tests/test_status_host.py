"""What joining status words refuses (no GPU)."""
import paper_2209_13258_b200 as P


def test_joining_status_words_refuses():
    assert P.osdp_join_status(None, (1 << 20, 256), stream=0) == 1 and P.osdp_join_status((1 << 20, 256), None, stream=0) == 1
    assert P.osdp_join_status(((1 << 20) + 2, 256), (1 << 20, 256), stream=0) == 4
