"""The barrier protocol of the attention over the 8-bit cache in random walks (kv8_protocol_model.py)."""
from kv8_protocol_model import walks


def test_nothing_gets_stuck_or_reads_what_is_not_there():
    assert walks(1, 1500) == {"ok": 1500}


def test_who_gives_up_ends_with_all_the_others():
    got = walks(2, 3000, give_up=0.003)
    assert set(got) == {"ok", "gave up"} and got["gave up"] > 1000


def test_the_softmax_warps_have_to_agree():
    """Each leaving by itself, the others wait at a barrier without a bound."""
    assert walks(2, 1500, give_up=0.003, agree=False).get("stuck", 0) > 0


def test_weights_wait_for_the_product_before():
    assert walks(3, 500, p_waits=False).get("overrun", 0) > 0


def test_a_piece_s_buffer_is_held_until_its_rows_are_out():
    assert walks(4, 500, q_waits_softmax=False).get("overrun", 0) > 0
