"""Sampling's settings as the binding reads them: a number for all, or one for each sequence, in any of Python's forms."""
import numpy as np
import pytest
import torch


class _Seen(Exception):
    pass


@pytest.fixture
def settings(monkeypatch):
    """What mad.sample hands on for given settings: (temperature, top_k, top_p, min_p) as lists."""
    import paper_2608_30252_amd as mad
    seen = []

    class Lib:
        def mad_sample(self, x, dt, u, *rest):
            seen.append([list(v) for v in rest[:4]])
            raise _Seen()

    monkeypatch.setattr(mad, "_FAST", mad._CtypesOnly())
    monkeypatch.setattr(mad, "_load_library", Lib)
    monkeypatch.setattr(mad, "workspace_bytes", lambda *a, **k: 256)
    monkeypatch.setattr(mad, "_ws_for", lambda *a: torch.zeros(256, dtype=torch.uint8))
    monkeypatch.setattr(mad, "_stream", lambda dev: None)

    def get(**kw):
        with pytest.raises(_Seen):
            mad.sample(torch.zeros(2, 3, 10), torch.zeros(2, 3), **kw)
        return seen[-1]
    return get


@pytest.mark.parametrize("number", [lambda v: v, np.float64, np.array, torch.tensor, lambda v: [v, v], lambda v: np.array([v, v]),
                                    lambda v: torch.tensor([v, v], dtype=torch.float64)],
                         ids=["number", "numpy scalar", "numpy 0-d", "tensor 0-d", "list", "numpy", "tensor"])
def test_a_setting_in_any_form(settings, number):
    got = settings(temperature=number(0.75), top_k=number(7), top_p=number(0.5), min_p=number(0.25))
    assert got == [[0.75, 0.75], [7, 7], [0.5, 0.5], [0.25, 0.25]]


def test_the_wrong_number_of_settings():
    import paper_2608_30252_amd as mad
    for bad in ([0.5], np.ones(3), torch.ones(1), ()):
        with pytest.raises(ValueError, match="top_p needs one entry"):
            mad.sample(torch.zeros(2, 3, 10), torch.zeros(2, 3), top_p=bad)
