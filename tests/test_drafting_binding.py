"""What the binding of the operators around drafting keeps and hands on (no GPU needed)."""
import paper_2502_20704_amd as fsd
from paper_2502_20704_amd import drafting


def test_answers_for_shapes_do_not_pile_up():
    """a server sees new batch sizes for as long as it runs"""
    want = [fsd.fsd_cache_fork_workspace_bytes(50, n) for n in (1, 2, 3)]
    for n in range(1, 5000):
        fsd.fsd_cache_fork_workspace_bytes(50, n)
        fsd.fsd_beam_workspace_bytes(n, 2, 1000, 3, fsd.BF16)
    assert len(drafting._bytes) <= 1001
    assert [fsd.fsd_cache_fork_workspace_bytes(50, n) for n in (1, 2, 3)] == want


def test_sizes_past_an_int_have_no_workspace():
    """the library takes sizes as int: what would arrive there as another size has no answer, as other sizes out of range have none"""
    for off in (1 << 32, -(1 << 32), 1 << 64):
        for k in range(5):
            sizes = [2, 3, 1000, 4, fsd.BF16]
            sizes[k] += off
            assert fsd.fsd_beam_workspace_bytes(*sizes) == 0
        assert fsd.fsd_cache_fork_workspace_bytes(50 + off, 4) == fsd.fsd_cache_fork_workspace_bytes(50, 4 + off) == 0
        assert fsd.fsd_cache_compact_workspace_bytes(50 + off) == 0
    assert fsd.fsd_beam_workspace_bytes(2, 3, 1000, 4, fsd.BF16) > 0


def test_workspaces_serve_either_type():
    """a workspace of a call's sizes will do for the other type of logits too"""
    for sizes in ((1, 1, 1, 1), (64, 8, 128256, 16), (3, 256, 524288, 128), (65535, 1, 70000, 2)):
        assert fsd.fsd_beam_workspace_bytes(*sizes, fsd.F32) == fsd.fsd_beam_workspace_bytes(*sizes, fsd.BF16) > 0
