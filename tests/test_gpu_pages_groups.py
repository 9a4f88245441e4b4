"""Steps over 4-bit rows for groups of every kind: up to five heads, up to eight, and more, whose heads share the matrix products differently."""
import pytest

from .test_gpu_pages_fp4 import spoil_hidden, step_case

pytestmark = pytest.mark.gpu
GROUPS = [1, 2, 5, 6, 7, 8, 9, 12, 16]


@pytest.mark.parametrize("G", GROUPS)
@pytest.mark.parametrize("d", [64, 128])
def test_lengths(G, d):
    step_case(d, 4, 2 * G, 2, 32, [1, 33, 700, 64], seed=G)
    step_case(d, 2, G, 1, 4, [130, 17], seed=G)  # rows found one by one
    step_case(d, 2, G, 1, 16, [130, 17], seed=G, score=False)


@pytest.mark.parametrize("G", GROUPS)
@pytest.mark.parametrize("pos", [False, True], ids=["slots", "positions"])
def test_windows(G, pos):
    for window, n_sink, lens in ((1, 0, [1, 200]), (64, 130, [400, 60]), (100, 3, [300, 101])):
        step_case(128, 2, 2 * G, 2, 64, lens, window, n_sink, pos=pos, seed=G)


@pytest.mark.parametrize("G", GROUPS)
def test_several_shares(G):
    step_case(128, 1, 2 * G, 2, 64, [9001], seed=G)


@pytest.mark.parametrize("G", GROUPS)
@pytest.mark.parametrize("page", [4, 64])
def test_nan(G, page):
    """Behind the end and where the window hides it: of no effect; in an entry that is seen: in its elements."""
    step_case(128, 3, 2 * G, 2, page, [70, 33, 16], spoil=spoil_hidden)

    def hidden(t, lens):
        spoil_hidden(t, lens)
        for b, n in enumerate(lens.tolist()):
            for s in range(8, n - 20):
                p = int(t["table"][b, s // page])
                t["v_exp"][p, :, s % page] = -128
    step_case(128, 2, 2 * G, 2, page, [100, 61], window=20, n_sink=8, spoil=hidden)

    def seen(t, lens):
        for at in (3, 69):
            p = int(t["table"][0, at // page])
            t["v_exp"][p, 1, at % page, 2] = -128
    step_case(128, 1, 2 * G, 2, page, [71], spoil=seen, score=False)


@pytest.mark.parametrize("G", GROUPS)
@pytest.mark.parametrize("scale", [1e-30, 8e36])
def test_values_of_any_size(G, scale):
    step_case(128, 2, G, 1, 16, [700, 41], score=False, scale=scale, qscale=1.0 / scale)
