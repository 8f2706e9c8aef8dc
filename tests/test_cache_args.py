"""What the binding makes of a cache's tensors and of inputs.  CPU only."""
import pytest

torch = pytest.importorskip("torch")
import paper_2609_11938_gb300 as opa  # noqa: E402


class Host(opa.Context):
    """A context's argument checks on host tensors (device -1), without a GPU."""

    def __init__(self):
        self.device, self.handle, self._dev = -1, None, torch.device("cpu")

    def _enter(self):
        raise AssertionError("past the checks")


@pytest.fixture()
def host():
    return Host()


@pytest.mark.parametrize("name", ["k_pages", "v_pages", "table", "length", "refs", "low"])
def test_replaced_field(host, name):
    """The calls go by a field's tensor, not by the one that was there when the cache was made."""
    c = host.cache(4, 16, 2, 64, 3, 2)
    new = getattr(c, name).clone()
    setattr(c, name, new)
    assert getattr(c, name) is new and getattr(c.struct, name) == new.data_ptr()
    assert c.by_ref._obj is c.struct


@pytest.mark.parametrize("name", ["k_pages", "v_pages", "table", "length", "refs", "low"])
def test_replaced_field_is_checked(host, name):
    c = host.cache(4, 16, 2, 64, 3, 2)
    old = getattr(c, name)
    for wrong in (torch.cat([old, old]), old.double()):
        with pytest.raises((ValueError, TypeError)):
            setattr(c, name, wrong)
        assert getattr(c, name) is old and getattr(c.struct, name) == old.data_ptr()


def test_field_changed_in_place(host):
    c = host.cache(4, 16, 2, 64, 3, 2)
    at = c.length.data_ptr()
    c.length += 2
    c.refs[1] = 5
    assert c.length.tolist() == [2, 2, 2] and c.struct.length == at == c.length.data_ptr()


def x(*shape, grad=False):
    return torch.zeros(shape, dtype=torch.bfloat16, requires_grad=grad)


def off(*v):
    return torch.tensor(v, dtype=torch.int32)


@pytest.mark.parametrize("at", [0, 1, 2])
def test_gradients_are_not_lost_in_silence(host, at):
    c = host.cache(4, 16, 2, 64, 3, 2)
    qkv = [x(4, 2, 64, grad=i == at) for i in range(3)]
    calls = [lambda: host.attention(*qkv, off(0, 4))]
    if at:
        calls.append(lambda: host.cache_append(c, off(0), off(0, 4), *qkv[1:]))
    else:
        calls.append(lambda: host.cache_attention(c, off(0, 1, 2, 0), qkv[0]))
    for call in calls:
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        with torch.no_grad(), pytest.raises(AssertionError, match="past the checks"):
            call()
    with pytest.raises(AssertionError, match="past the checks"):
        host.attention(*(t.detach() for t in qkv), off(0, 4))
