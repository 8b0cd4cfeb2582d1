"""The workspace of the norm's gradients has room for the parts of every form of the call."""
import paper_2608_22646_gb300 as cai

SMS = 152  # parts of the form for many rows, whatever the device


def test_room_for_a_part_of_every_sm():
    """The form for many rows, from as many rows as SMs on, leaves SMS parts [2, H] of float32; with
    fewer rows every row has one at most."""
    for H in list(range(1, 600)) + list(range(600, 16385, 61)) + [2048, 2049, 8192, 8193, 16384]:
        for M in (0, 1, 2, SMS - 1, SMS, SMS + 1, 10 * SMS, 1 << 20):
            part, bytes_ = 2 * H * 4, cai.cai_norm_workspace(M, H)
            assert bytes_ % part == 0 and bytes_ // part >= min(M, SMS), (M, H, bytes_)
            assert bytes_ // part <= M
