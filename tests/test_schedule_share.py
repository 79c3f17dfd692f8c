"""The balance bound of the schedule on batches whose units are long against a CTA's share (host only)."""
import pytest

from paper_2609_04774_b200 import binding, build


@pytest.mark.parametrize("new_len,prefix,Hq,Hkv,sms", [([1793, 1793], [1537, 1664], 6, 2, 148), ([1793, 1793], [1537, 1664], 4, 4, 148),
                                                       ([1700], [1900], 6, 2, 132), ([2049, 1], [2000, 2000], 9, 3, 148)])
def test_no_cta_carries_much_more_than_its_share(new_len, prefix, Hq, Hkv, sms):
    build.build()
    cu = [0]
    for n in new_len:
        cu.append(cu[-1] + n)
    info, _, _ = binding.cp_schedule_inspect(cu, prefix, [1] * len(prefix), Hq, Hkv, sms)
    share = -(-info["total"] // info["grid"])
    longest = max(-(-(p + n) // 128) for p, n in zip(prefix, new_len))
    assert info["max_load"] <= max(1.3 * share + 8, min(longest, 8) + 8), info
