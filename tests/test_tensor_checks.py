"""The bindings' checks of tensors in compiled code say what the ones in Python say: the same address, or the same error."""
import pytest
import torch

from paper_2603_06274_amd import decode_binding as db

pytestmark = pytest.mark.skipif(db._tensors is None, reason="the module is not built")


@pytest.fixture
def functions():
    """(name, compiled, Python) of the three; what the compiled ones ask is counted."""
    import importlib.util
    import sys
    spec = importlib.util.spec_from_file_location("paper_2603_06274_amd._checks_in_python", db.__file__)
    plain, known = importlib.util.module_from_spec(spec), sys.modules.get("paper_2603_06274_amd._tensors")
    package = sys.modules["paper_2603_06274_amd"]
    sys.modules["paper_2603_06274_amd._tensors"] = None        # (an import of it fails)
    had = package.__dict__.pop("_tensors", None)
    try:
        spec.loader.exec_module(plain)
    finally:
        sys.modules["paper_2603_06274_amd._tensors"] = known
        if had is not None:
            package._tensors = had
    assert plain._tensors is None
    return [(x, getattr(db, x), getattr(plain, x)) for x in ("_values", "_whole", "_lines")]


def outcome(f, args):
    try:
        return f(*args)
    except Exception as e:
        return type(e), str(e)


def tensors():
    x = torch.zeros(6, 4, dtype=torch.int32)
    return [x, x.t(), x[::2], x[1:], x[:0], x.view(-1), x.view(2, 3, 4), x.long(), x.to(torch.bfloat16), torch.nn.Parameter(x.float()),
            torch.zeros((), dtype=torch.int32), torch.zeros(3, 0, dtype=torch.int32), x.to_sparse(), torch.zeros(6, 4, dtype=torch.int32, device="meta"),
            torch.zeros(4, dtype=torch.int32).expand(6, 4), None, 3, "x"]


def test_the_same_answers(functions):
    (_, values, values_py), (_, whole, whole_py), (_, lines, lines_py) = functions
    likes = [None] + [db._seen(t) for t in tensors()[:10]] + [(torch.Size([6, 4]), (4, 1), torch.int32), ((6, 4), (1, 4), torch.int32), 7, ()]
    for t in tensors():
        for dev in (-1, 0):
            for like in likes:
                assert outcome(values, (t, like, "x", dev)) == outcome(values_py, (t, like, "x", dev))
            for n in (0, 1, 24, 25, 1 << 62):
                for dtype in ((), (torch.int32,), (torch.int64,), (torch.bfloat16,)):
                    args = (t, n, "x", dev, *dtype)
                    assert outcome(whole, args) == outcome(whole_py, args), args
                    for each in (1, 4, 24):
                        args = (t, n, each, "x", dev, *dtype)
                        assert outcome(lines, args) == outcome(lines_py, args), args


def test_calls_that_are_none(functions):
    x = torch.zeros(3, dtype=torch.int32)
    for name, f, _ in functions:
        for args in ((), (x,), (x, 1, "x", -1, torch.int32, 9, 9), (x, "a", "x", "b"), (x, 1 << 70, "x", -1), (x, 1.0, "x", -1)):
            if name == "_whole" and args[1:2] in ((1 << 70,), (1.0,)):
                continue
            with pytest.raises(Exception):
                f(*args)
    assert outcome(functions[1][1], (x, 1.0, "x", -1)) == outcome(functions[1][2], (x, 1.0, "x", -1))
    assert outcome(functions[1][1], (x, 1 << 70, "x", -1)) == outcome(functions[1][2], (x, 1 << 70, "x", -1))


def test_good_tensors_are_not_asked_about_twice(functions):
    asked = []
    old = [db_f for db_f in (functions[0][2], functions[1][2], functions[2][2])]
    db._tensors.begin(*(lambda *a: asked.append(a) for _ in range(3)))
    try:
        x = torch.zeros(6, 4, dtype=torch.int32)
        assert db._whole(x, 24, "x", -1) == db._lines(x, 6, 4, "x", -1) == db._values(x, db._seen(x), "x", -1) == x.data_ptr()
        assert not asked
    finally:
        db._tensors.begin(*old)
