"""Sizes that the state-pool calls take where the dense calls' chunk counts would not fit
(on the host: nothing to do, or refused for something else)."""
import pytest

from test_slots_abi import A, call, inputs, pdn, prob, slots

BIG = dict(tokens=1 << 22, slots=9000, Hk=32)   # rows, as many as 8192 sequences of 512 have
RAGGED = prob(B=8192, T=1 << 22, H=32)          # the most rows one of them has: not known, so all


@pytest.mark.parametrize("draft", [False, True])
def test_large_ragged_batches(draft):
    """B H ceil(T / 64) is far past 2^31; the kernels number sequences, heads and rows only."""
    far = dict(S=1 << 50, A=1 << 52, tape=1 << 58 if draft else None, pending=1 << 54 if draft else None,
               tape_tokens=1 << 22 if draft else 0)
    wide = inputs(q=1 << 44, k=2 << 44, v=3 << 44, beta=1 << 40, g=2 << 40, beta_p=3 << 40, g_p=4 << 40)
    assert call(draft, p=RAGGED, i=wide, s=slots(draft, **{**BIG, **far, "slots": 0}), o=5 << 44) == pdn.PDN_OK
    # (the next check after those of sizes)
    assert call(draft, p=RAGGED, i=inputs(q=None), s=slots(draft, **BIG, **far)) == pdn.PDN_ERR_NULL


def test_any_number_of_tokens_a_sequence():
    for T in (1 << 31, 1 << 40, (1 << 63) - 1):
        assert call(False, p=prob(T=T), s=slots(False, slots=0)) == pdn.PDN_OK
        assert call(True, p=prob(T=T)) == pdn.PDN_ERR_SHAPE                 # more than a tape holds
        assert call(False, p=prob(T=T), s=slots(False, starts=None)) == pdn.PDN_ERR_SHAPE   # 3 T rows are not 20
    assert call(False, p=prob(chunk=7), s=slots(False, slots=0)) == pdn.PDN_OK   # not used


def test_number_of_sequences():
    for B in (1 << 31, 1 << 61, (1 << 63) - 1):
        assert call(False, p=prob(B=B)) == pdn.PDN_ERR_SHAPE
        assert call(False, p=prob(B=B, H=0), s=slots(False, Hk=0)) == pdn.PDN_ERR_SHAPE
