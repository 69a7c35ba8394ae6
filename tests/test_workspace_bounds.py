"""A workspace sized for a call holds every call of at most its sizes (no GPU: sizes, and refusals before any launch)."""
import itertools

import pytest


@pytest.fixture(scope="module")
def mad():
    import paper_2608_30252_amd as m
    m._load_library()
    return m


def _grows(size, axes):
    """size(*point) never falls along an axis of the grid (0: not a valid point)."""
    names, values = list(axes), list(axes.values())
    for point in itertools.product(*values):
        here = size(*point)
        for i, ax in enumerate(values):
            at = ax.index(point[i])
            if here and at + 1 < len(ax):
                # the next valid size along this axis
                for x in ax[at + 1:]:
                    there = size(*point[:i], x, *point[i + 1:])
                    if there:
                        assert there >= here, f"{names[i]} {point[i]} -> {x} at {dict(zip(names, point))}: {here} -> {there} bytes"
                        break


BATCHES = [1, 2, 3, 7, 8, 15, 16, 17, 31, 32, 33, 62, 63, 64]


@pytest.mark.parametrize("d", [64, 128])
def test_attention_over_4_bits(mad, d):
    def size(B, Hq, Hkv, T):
        ok = Hq % Hkv == 0 and Hq // Hkv <= 16 and T * (Hq // Hkv) <= 64
        return mad.workspace_bytes(mad.MAD_OP_VERIFY_KV4, B, Hq, Hkv, d, T) if ok else 0
    _grows(size, dict(B=BATCHES, Hq=[1, 2, 8, 16, 32, 64, 128], Hkv=[1, 2, 4, 8, 16, 64], T=[1, 2, 3, 4, 6, 8, 16, 64]))
    for B, Hq, Hkv, T in ((64, 64, 8, 6), (32, 16, 16, 1), (64, 8, 8, 64)):
        assert size(B, Hq, Hkv, T) >= size(1, Hq, Hkv, T) > 0
    # fewer KV heads of more queries each are smaller sizes too
    assert size(1, 64, 8, 4) >= size(1, 64, 4, 4) and size(2, 64, 16, 1) >= size(1, 32, 2, 1)
    for shape in ((64, 64, 8), (1, 32, 8)):
        assert mad.workspace_bytes(mad.MAD_OP_VERIFY_KV4, *shape, 128, 64) >= mad.workspace_bytes(mad.MAD_OP_VERIFY_KV4, *shape, 64, 64)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_over_4_bits_holds_its_pieces(mad, d):
    """A unit's pieces are counted from its first workgroup's number and its own: below 512 units up to 512 + units of them,
    R rows of d + 2 floats each, padded to 16 bytes; from 512 units on every unit is whole."""
    for B, Hkv, G, T in itertools.product([1, 2, 63, 64], [1, 2, 7, 8, 9, 64], [1, 2, 4, 8, 16], [1, 3, 4, 17, 64]):
        if T * G <= 64:
            units, piece = B * Hkv, (T * G * (d + 2) + 3) // 4 * 16
            need = (1 << 20) + (units < 512) * (units + 512) * piece
            assert mad.workspace_bytes(mad.MAD_OP_VERIFY_KV4, B, Hkv * G, Hkv, d, T) >= need, (B, Hkv, G, T)


def test_log_probabilities(mad):
    size = lambda B, T, V: mad.workspace_bytes(mad.MAD_OP_LOGPROBS, B, T=T, max_keys=V)   # noqa: E731
    _grows(size, dict(B=BATCHES, T=[1, 2, 3, 5, 8, 9, 15, 16, 17, 33, 64, 65, 1000, 1024, 65536],
                      V=[1, 7, 4089, 4090, 8185, 8186, 16384, 30000, 50257, 65000, 65535, 70000, 128256, 262144, 1 << 20]))


def test_log_probabilities_hold_their_records(mad):
    """Up to 1024 rows take up to 1024 / rows workgroups of whole chunks each, 16 at most, and a record for each."""
    record, region = 16 + 8 + 8 + 8 * 64, 1 << 20
    for rows in list(range(1, 70)) + [100, 255, 256, 257, 341, 342, 511, 512, 513, 1023, 1024, 1025]:
        for V in (1, 4089, 4090, 30000, 50257, 65000, 70000, 128256, 1 << 20):
            chunks = -(-(V + 7) // 4096)
            want = 1 if rows > 1024 else min(1024 // rows, 16)
            splits = -(-chunks // -(-chunks // want))
            need = region + (rows * splits * record if splits > 1 else 0)
            assert mad.workspace_bytes(mad.MAD_OP_LOGPROBS, 1, T=rows, max_keys=V) >= need, (rows, V)
