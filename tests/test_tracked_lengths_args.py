"""Lengths that ihip_kv_evict is not to write over the tokens seen (no GPU)."""
from tests.test_kv_store_args import b  # noqa: F401
from tests.test_tracked_args import BAD, evict, track_of


def test_new_lengths_over_the_tokens_seen(b):  # noqa: F811
    """The same array, or a part of it: the cut lengths would be taken for the tokens seen, by the same call's other workgroups too."""
    at = 1 << 20
    for rows, keep in ((64, 16), (4096, 1024), (50000, 1024)):
        track = track_of(b, rows=rows, seen=at)
        for new in (at, at + 4, at - 4):
            for lens in (at + 4096, new):
                assert evict(b, track=track, max_len=rows, keep=keep, new=new, lens=lens) == BAD and b"tokens seen" in b.lib().ihip_last_error()
