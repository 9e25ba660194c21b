"""The tests' own reading of the dropout generator against its published answer.  Needs no GPU."""
from test_gpu_train import _kept

KNOWN = (0x5f6fb709, 0x0d893f64, 0x4f121f81, 0x4f730a48)      # Philox4x32 with seven rounds for a counter and a key of zeros


def test_known_answer():
    bits = [w >> s & 0xffff for w in KNOWN for s in (0, 16)]
    for e, u in enumerate(bits):
        assert _kept(8, u / 65536, 0, 0)[e] and not _kept(8, (u + 1) / 65536, 0, 0)[e]
