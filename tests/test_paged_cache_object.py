"""The Python object of a paged cache, without a device: the addresses its calls pass on are those of the tensors it holds."""
import pytest

from paper_2410_03090_amd import binding

torch = binding.torch


def _cache(monkeypatch):
    """Host tensors that say they are on a device."""
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32)  # noqa: E731
    t = dict(K=torch.zeros(4, 16, 64), V=torch.zeros(4, 16, 64), idx=i32(4, 16), cum=torch.zeros(4, 16), table=i32(2, 2), length=i32(2))
    return binding.PagedCache(**t), t


def test_tensors_of_a_cache_cannot_be_exchanged(monkeypatch):
    """Another tensor under a name would leave the calls with the address of one that may be freed."""
    c, t = _cache(monkeypatch)
    for name in ("K", "V", "idx", "cum", "table", "length"):
        with pytest.raises(AttributeError):
            setattr(c, name, torch.zeros_like(t[name]))
        with pytest.raises(AttributeError):
            delattr(c, name)
        assert getattr(c, name) is t[name]
    for name, value in (("n_heads", 3), ("D", 128), ("dtype", torch.bfloat16), ("device", "cpu"), ("_struct", None), ("_ref", None)):
        with pytest.raises(AttributeError):
            setattr(c, name, value)


def test_contents_of_a_cache_can_be_written(monkeypatch):
    c, t = _cache(monkeypatch)
    c.length += 3                                               # (gives the same tensor its name again)
    c.table[1, 0] = 2
    assert c.length is t["length"] and c.length.tolist() == [3, 3] and t["table"][1, 0] == 2
    assert [a is b for a, b in zip(c, t.values())] == [True] * 6
