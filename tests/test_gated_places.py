"""The gated block's calls refuse an output that shares memory with another output or with
what the call reads, wherever the two lie, before any CUDA call; and take matrices that lie
between one another's rows (no GPU needed)."""
import ctypes
import itertools

import pytest

torch = pytest.importorskip("torch")

from paper_2010_14298_gb300 import fqt  # noqa: E402

EINVAL, EWORKSPACE = 1, 6  # (no workspace is given: a call that gets so far is EWORKSPACE)
BASE = 1 << 40  # nothing is read or written
M, N, K = 10, 40, 64


class Call:
    """Code matrices and dense tensors by name, each in a place of its own."""

    def __init__(self, codes, dense):
        self.codes, self.dense = dict(codes), dict(dense)
        self.at = {}
        for i, name in enumerate([*self.codes, *self.dense]):
            self.at[name] = BASE + 0x10000 * i
            if name in self.codes:
                self.at[name + ".scales"] = BASE + 0x10000 * i + 0x8000
        self.pitch = {n: -(-c // 16) * 16 for n, (r, c) in self.codes.items()}
        self.ld = {n: c for n, (r, c) in self.dense.items()}

    def code(self, name):
        r, c = self.codes[name]
        return ctypes.byref(fqt._F8(r, c, self.pitch[name], 1, 0, self.at[name],
                                    self.at[name + ".scales"]))


class Forward(Call):
    reads, writes = ("A", "Bg", "Bu"), ("q", "gate", "up", "out")

    def __init__(self, dtype=0):
        self.dtype = dtype
        super().__init__(dict(A=(M, K), Bg=(N, K), Bu=(N, K), q=(M, N), gate=(M, N), up=(M, N)),
                         dict(out=(M, N)))

    def run(self):
        c = self.code
        return fqt.load().fqt_fp8_gated_matmul(
            c("A"), c("Bg"), c("Bu"), 0, self.dtype, self.at["out"], self.ld["out"], c("q"),
            c("gate"), c("up"), None, 0, None)


class Backward(Call):
    reads = ("gate", "up", "dA")
    writes = ("qgate", "qup", "qgate_t", "qup_t", "product_t", "dgate", "dup")

    def __init__(self, dtype=0):
        self.dtype = dtype
        t = (N, M)
        super().__init__(dict(gate=(M, N), up=(M, N), qgate=(M, N), qup=(M, N), qgate_t=t, qup_t=t,
                              product_t=t), dict(dA=(M, N), dgate=(M, N), dup=(M, N)))

    def run(self):
        c, at, ld = self.code, self.at, self.ld
        return fqt.load().fqt_fp8_gated_backward(
            at["dA"], ld["dA"], self.dtype, c("gate"), c("up"), 0, at["dgate"], ld["dgate"],
            at["dup"], ld["dup"], c("qgate"), c("qup"), c("qgate_t"), c("qup_t"), c("product_t"),
            None, 0, None)


class Sum(Call):
    reads, writes = ("A1", "B1", "A2", "B2"), ("out",)

    def __init__(self, dtype=0):
        self.dtype = dtype
        super().__init__(dict(A1=(M, K), B1=(N, K), A2=(M, 48), B2=(N, 48)), dict(out=(M, N)))

    def run(self):
        c = self.code
        return fqt.load().fqt_fp8_matmul_sum(c("A1"), c("B1"), c("A2"), c("B2"), self.dtype,
                                             self.at["out"], self.ld["out"], None, 0, None)


CALLS = [Forward, Backward, Sum]


def _places(call, names):
    """The addresses of some matrices, those of their scales with them."""
    return [n + s for n in names for s in ("", ".scales") if n + s in call.at]


@pytest.mark.parametrize("kind", CALLS)
def test_apart(kind):
    assert kind().run() == EWORKSPACE and kind(1).run() == EWORKSPACE


@pytest.mark.parametrize("kind", CALLS)
def test_any_two_in_one_place(kind):
    writes, reads = (_places(kind(), n) for n in (kind.writes, kind.reads))
    for a, b in itertools.chain(itertools.combinations(writes, 2), itertools.product(writes, reads)):
        for one, other in ((a, b), (b, a)):
            call = kind()
            call.at[one] = call.at[other]
            assert call.run() == EINVAL, (one, other)
    for a, b in itertools.combinations(reads, 2):  # two that are read
        if a.endswith(".scales") == b.endswith(".scales"):
            call = kind()
            call.at[a] = call.at[b]
            assert call.run() == EWORKSPACE, (a, b)


def _bytes(call, name):
    if name.endswith(".scales"):
        r, c = call.codes[name[:-7]]
        return -(-c // 512) * -(-r // 128) * 512
    if name in call.codes:
        r, c = call.codes[name]
        # (an output's rows are whole 16 bytes, of an operand only the columns count)
        return (r - 1) * call.pitch[name] + (c if name in call.reads else -(-c // 16) * 16)
    r, c = call.dense[name]
    return ((r - 1) * call.ld[name] + c) * (2 if call.dtype else 4)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("kind", CALLS)
def test_overlaps_by_sixteen_bytes(kind, dtype):
    """One that begins in another's last 16 bytes is refused, one that begins behind them is
    not."""
    writes, reads = (_places(kind(), n) for n in (kind.writes, kind.reads))
    for a, b in itertools.chain(itertools.permutations(writes, 2), itertools.product(writes, reads),
                                itertools.product(reads, writes)):
        call = kind(dtype)
        end = call.at[b] + -(-_bytes(call, b) // 16) * 16
        call.at[a] = end - 16
        assert call.run() == EINVAL, (a, b)
        call.at[a] = end
        assert call.run() == EWORKSPACE, (a, b)


@pytest.mark.parametrize("dtype", [0, 1])
def test_halves_of_one_buffer(dtype):
    """dg and du as halves of one gradient, its codes beside them; u's and g's codes likewise."""
    es = 2 if dtype else 4
    call = Backward(dtype)
    call.ld.update(dgate=2 * N, dup=2 * N)
    call.at["dup"] = call.at["dgate"] + N * es
    assert call.run() == EWORKSPACE
    for entries in (1, N - 1, N + 1):  # into dgate's row, or into its next one
        call.at["dup"] = call.at["dgate"] + entries * es
        assert call.run() == EINVAL
    call.at["dup"] = call.at["dgate"] + N * es
    call.pitch.update(qgate=96, qup=96)
    call.at["qup"] = call.at["qgate"] + 48
    assert call.run() == EWORKSPACE
    call.at["qup"] = call.at["qgate"] + 32  # (40 columns are 48 bytes)
    assert call.run() == EINVAL
    call.at["qup"] = call.at["qgate"] + 64
    assert call.run() == EINVAL  # (which reaches the next row)
    fwd = Forward(dtype)
    fwd.pitch.update(gate=96, up=96)
    fwd.at["up"] = fwd.at["gate"] + 48
    assert fwd.run() == EWORKSPACE
    # every second row
    fwd.at["up"] = fwd.at["gate"] + 96
    fwd.pitch.update(gate=192, up=192)
    assert fwd.run() == EWORKSPACE
    # rows of other pitches between one another's, and in one another's way
    fwd.pitch.update(gate=192, up=384)
    assert fwd.run() == EWORKSPACE
    fwd.pitch.update(gate=192, up=288)
    assert fwd.run() == EINVAL


def test_one_row():
    """A single row has no pitch: what is given for it does not count."""
    for ldo in (0, -5, 1 << 50):
        f8 = lambda r, c, at: fqt._F8(r, c, 64, 1, 0, BASE + at, BASE + at + 0x8000)  # noqa: E731
        a, bg, bu, q = f8(1, K, 0), f8(N, K, 0x10000), f8(N, K, 0x20000), f8(1, N, 0x30000)
        none = ctypes.POINTER(fqt._F8)()
        call = lambda out: fqt.load().fqt_fp8_gated_matmul(  # noqa: E731
            a, bg, bu, 0, 0, out, ldo, q, none, none, None, 0, None)
        assert call(BASE + 0x40000) == EWORKSPACE
        assert call(q.codes - N * 4) == EWORKSPACE
        assert call(q.codes - N * 4 + 4) == EINVAL and call(q.codes + 44) == EINVAL
        assert call(q.codes + 48) == EWORKSPACE


def test_far_pitches():
    """Rows 2^40 entries apart: the places are worked out without overflow."""
    call = Backward(0)
    far = 1 << 40
    call.ld.update(dA=far, dgate=far, dup=far)
    call.at.update(dgate=call.at["dA"] + 4 * N, dup=call.at["dA"] + 8 * N)
    assert call.run() == EWORKSPACE
    call.at["dup"] = call.at["dA"] + 8 * N - 4
    assert call.run() == EINVAL
