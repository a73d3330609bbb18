"""The waits of the attention kernels with sinks, walked as in test_kernel_waits: two runs of key tiles, the sinks' and the window's, share the staged buffers, and every
fragment is consumed (or waited for) within the slot in which it is read.  None of them keeps registers in scratch memory inside the loops of dK/dV, and none in the forward."""
import pytest

from test_kernel_waits import _named, barriers_passed_unwaited, built  # noqa: F401


@pytest.mark.parametrize("part", ["16attn_fwd_sinks_k", "19attn_bwd_dq_sinks_k", "20attn_bwd_dkv_sinks_k", "16attn_bwd_sinks_k"])
def test_reads_are_waited_for_within_the_slot(built, part):  # noqa: F811
    found = _named(built, (part,))
    assert len(found) >= 2, sorted(found)
    worst = {n: barriers_passed_unwaited(c) for n, c in found.items()}
    assert max(worst.values()) == 0, {n: w for n, w in worst.items() if w}


@pytest.mark.parametrize("part", ["16attn_fwd_sinks_k", "19attn_bwd_dq_sinks_k"])
def test_nothing_is_kept_in_scratch(built, part):  # noqa: F811
    found = _named(built, (part,))
    assert found and not [n for n, c in found.items() if any(op.startswith("scratch_") for _, op, _, _ in c)]
