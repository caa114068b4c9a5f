"""What the compiler is told about LDS that one wave's lanes hand each other in the 4-bit cache's attention, read from the
device code's IR (no GPU)."""
import re

from tests.test_device_code import exchanges, kernels_ir


def test_a_waves_exchanges_are_fenced_on_both_sides(tmp_path):
    """Scales and biases, and the terms of probabilities, go through LDS to other lanes in every turn of the loop over
    blocks: stores, a fence, loads, and a fence again before the next turn's stores."""
    found = {n: b for n, b in kernels_ir("attend_n.hip", tmp_path).items() if "k_attendn_partial" in n}
    assert len(found) == 24
    for name, blocks in found.items():
        queries = int(re.search(r"ILi\d+ELi(\d+)E", name)[1])
        scales = [s for s in (exchanges(b, r"(?:i32|float|i8|<4 x float>)") for b in blocks) if re.search("w.*r", s)]
        assert len(scales) == 1 and re.fullmatch("f?r?w+fr+", scales[0].replace("ff", "f")), (name, scales)
        terms = [s for s in (exchanges(b, r"(?:<2 x i32>|<8 x bfloat>)") for b in blocks) if re.search("w.*r", s)]
        if queries == 16:        # every lane keeps its own
            assert not terms, (name, terms)
            last = [s for s in (exchanges(b, r"none") for b in blocks) if "f" in s]
            assert len(last) >= 3, (name, last)
        else:
            assert len(terms) == 1 and re.fullmatch("w+fr+f", terms[0]), (name, terms)
