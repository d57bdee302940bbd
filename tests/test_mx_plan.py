"""Key splits that calls of few rows over 4-bit pages plan, seen through the workspaces they ask for (CPU only)."""
import pytest

from paper_2609_39819_amd import kvt

from test_mx_args import need, pool, seqs

D, HQ, HKV = 128, 32, 8


def partials(P, S):
    """Partial results per query head that the call plans room for."""
    p = pool(nb=1 << 24, hkv=HKV, d=D)
    s = seqs(P=P, S=S, max_blocks=1 << 20)
    rows, rest = divmod(need("kvt_mx_extend_workspace_bytes", p, s, HQ), (D + 2) * 4)
    assert rest == 0 and rows % HQ == 0
    return rows // HQ


def test_a_short_message_beside_a_long_context_leaves_it_its_splits():
    """64 rows of a kv-head take two workgroups over 8 tiles; the single token's 4094 tiles keep theirs."""
    alone = partials([131000], [1])
    beside = partials([131000, 100], [1, 16])
    assert alone >= 32                              # (of 256 CUs: 64)
    assert 0.9 * alone <= beside <= alone + 16      # (the message itself may lie in two shares)


@pytest.mark.parametrize("message", [1, 8, 16])
def test_a_launch_is_split_by_its_own_messages(message):
    """256 sequences are one launch; what the first holds changes nothing in the second."""
    first, rest = [9000] * 4 + [8000] * 252, [7000] * 3
    S = [message] + [1] * 255
    assert partials(first + rest, S + [1] * 3) == partials(first, S) + partials(rest, [1] * 3)
    assert partials(rest, [1] * 3) > 3


@pytest.mark.parametrize("d, contexts, message, whole", [
    # measured both ways: heads of 64, 100 contexts 28 us in one launch, 37 in shares and a join ...
    (64, [500 + 25 * i for i in range(100)], 1, True),
    (64, [2000] * 48, 16, True),
    # ... one of 30000 keys and 4 new tokens 135 and 16
    (64, [30000], 1, False), (128, [30000], 1, False), (64, [30000], 16, False),
    (128, [8000] * 32, 16, True)])
def test_whole_sequences_or_shares_by_what_was_measured(d, contexts, message, whole):
    p = pool(nb=1 << 24, hkv=HKV, d=d)
    s = seqs(P=contexts, S=[message] + [1] * (len(contexts) - 1), max_blocks=1 << 20)
    assert (need("kvt_mx_extend_workspace_bytes", p, s, HQ) == 0) == whole
