"""A call's kernels run on the device of its tensors, whichever device is current: the binding makes it the current one
for the length of the C call (the default stream, NULL, is the current device's)."""
import inspect
import re

import torch


def test_the_device_is_current_during_the_call_only(monkeypatch):
    import paper_2608_30252_amd as mad
    now, seen = [0], []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.was = now[0]
            if self.index >= 0:
                now[0] = self.index

        def __exit__(self, *a):
            now[0] = self.was

    class Lib:
        def mad_sample(self, *args):
            seen.append((now[0], args))
            if args == ("fails",):
                raise RuntimeError
            return -7

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(mad, "_load_library", Lib)
    assert mad._On(torch.device("cuda", 3)).mad_sample(1, 2) == -7
    assert seen == [(3, (1, 2))] and now == [0]
    mad._On(torch.device("cpu")).mad_sample()
    assert seen[1] == (0, ())
    try:
        mad._On(torch.device("cuda", 1)).mad_sample("fails")
    except RuntimeError:
        pass
    assert seen[2][0] == 1 and now == [0]


def test_every_call_on_a_stream_names_its_device():
    import paper_2608_30252_amd as mad
    source = inspect.getsource(mad)
    streams = re.findall(r"(?<!\w)(?<!def )_stream\(([\w.]+)\)", source)
    assert len(streams) >= 18 and streams == re.findall(r"_On\(([\w.]+)\)\.mad_", source)
