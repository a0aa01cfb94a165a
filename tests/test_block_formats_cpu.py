"""The reference of the block formats against values worked out by hand."""
import pytest

torch = pytest.importorskip("torch")

from block_formats import decode, magnitudes, quantise  # noqa: E402


def test_magnitudes():
    assert magnitudes("e2m1") == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    e4m3 = magnitudes("e4m3")
    assert e4m3[1] == 2.0 ** -9 and e4m3[8] == 2.0 ** -6 and e4m3[-1] == 448 and len(e4m3) == 127
    assert e4m3 == torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().tolist()


@pytest.mark.parametrize("kind,most,scale,values", [
    ("e2m1", [7.0, 1.0, 5.0, -0.25], 1, [8, 1, 4, 0]),        # 7 rounds to 8: the scale is 2; 2.5 and 0.125 go to 2 and 0
    ("e2m1", [6.9, 1.25, 5.0, 0.75], 0, [6, 1, 4, 1]),        # ties to 1 (1.25), 4 (5), 1 (0.75)
    ("e4m3", [464.0, 17.0, 19.0], 0, [448, 16, 20]),          # a tie that goes down: 464 stays in range
    ("e4m3", [465.0, 17.0, 34.0], 1, [480, 17 - 1, 32]),      # 480 = 240 * 2
    ("i8", [127.5, 2.5, 3.0], 1, [128, 2, 4]),                # 127.5 rounds to 128: the scale is 2, 1.25 goes to 1, 1.5 to 2
    ("i8", [127.4, 2.5, 3.5], 0, [127, 2, 4]),
    ("i8", [0.0], -127, [0])])
def test_scales_and_roundings(kind, most, scale, values):
    got, byte = quantise(torch.tensor([most], dtype=torch.float64), kind)
    assert byte.tolist() == [[scale + 127]] and got.tolist() == [values]


def test_decode():
    codes = torch.tensor([[0x21, 0xf9] + [0] * 14], dtype=torch.uint8)  # 0.5, 1, -0.5, -6
    assert decode(codes, torch.tensor([[128]], dtype=torch.uint8), "e2m1", 5).tolist() == [[1, 2, -1, -12, 0]]
