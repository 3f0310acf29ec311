"""Sizes that the packed attention takes: kvc.h states the limit in blocks of
eight (32 queries, head) units for sequences of any length (CPU: plan sizes)."""
import pytest


def _status(K, lens, hq, hkv):
    try:
        assert K.kvc_pack_plan_bytes(K.Pack(lens, hq, hkv)) > 0
        assert K.kvc_packed_attention_workspace(K.Pack(lens, hq, hkv)) >= 0
    except K.KvcError as e:
        return e.status, str(e)
    return 0, ""


def _blocks(length, hq, hkv):
    return -(-(-(-length // 32) * (hq // hkv)) // 8) * hkv


@pytest.mark.parametrize("length,hq,hkv", [(1, 512, 64), (32, 32, 8), (256, 32, 8), (768, 64, 8), (769, 64, 8), (100, 64, 64),
                                           (33, 28, 4), (5000, 1024, 64)])
def test_limit_is_the_documented_one(K, length, hq, hkv):
    most = 2 ** 22 // _blocks(length, hq, hkv)
    assert _status(K, [length] * most, hq, hkv) == (0, "")
    st, msg = _status(K, [length] * (most + 1), hq, hkv)
    assert st == K.KVC_ERR_INVALID_ARG and "one launch" in msg


def test_limit_of_a_mixed_batch(K):
    # long and short sequences count together
    lens = [768] * 1000 + [9000] * 100 + [17] * 3000
    used = sum(_blocks(x, 64, 64) for x in lens)
    most = (2 ** 22 - used) // _blocks(64, 64, 64)
    assert _status(K, lens + [64] * most, 64, 64) == (0, "")
    assert _status(K, lens + [64] * (most + 1), 64, 64)[0] == K.KVC_ERR_INVALID_ARG
