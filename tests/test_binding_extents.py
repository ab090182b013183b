"""The calls that go through ctypes: tensors that are too small, or on another device than the current one, are refused before a
launch.  Without a GPU the tensors only say that they lie on one (nothing follows their pointers: the refusal comes first)."""
import pytest
import torch


class Pretend:
    """A tensor that claims to lie on a GPU."""

    def __init__(self, *shape, dtype=torch.bfloat16, device=0):
        self.t, self.device = torch.zeros(*shape, dtype=dtype), device

    is_cuda = True

    def get_device(self):
        return self.device

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture
def B(monkeypatch):
    from paper_2602_11937_b200 import binding
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_raw_stream", None)

    def reached(stream):
        raise AssertionError("no refusal before the launch")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: reached(None))
    return binding


F32, I32, U8 = torch.float32, torch.int32, torch.uint8


def _calls(B):
    d, v = B.layer_desc(), B.KVView()
    p, h = Pretend, lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16)
    ws = p(64, dtype=U8)
    return {
        "static": (lambda **k: B.puzzle_decode_attn_static(d, v, **k),
                   dict(q=p(2, 64, 64), sinks=p(64, dtype=F32), out=p(2, 64, 64), lse_out=p(2, 64, dtype=F32),
                        dev_status=p(1, dtype=I32))),
        "partial": (lambda **k: B.puzzle_decode_attn_partial(d, v, **k),
                    dict(q=p(2, 64, 64), o_part=p(2, 64, 64, dtype=F32), lse_part=p(2, 64, dtype=F32), workspace=ws,
                         dev_status=p(1, dtype=I32))),
        "step_host": (lambda **k: B.puzzle_decode_step_host(d, v, **k),
                      dict(q_host=h(2, 64, 64), k_new_host=h(2, 8, 64), v_new_host=h(2, 8, 64), sinks=p(64, dtype=F32),
                           out_host=h(2, 64, 64), staging=ws, workspace=ws, dev_status=p(1, dtype=I32))),
        "merge": (lambda **k: B.puzzle_attn_merge(**k),
                  dict(part_o=p(2, 64, 3, 64, dtype=F32), part_lse=p(2, 64, 3, dtype=F32), num_parts=p(2, dtype=I32),
                       sinks=p(64, dtype=F32), out=p(2, 64, 64), lse_out=p(2, 64, dtype=F32))),
        "scales": (lambda **k: B.puzzle_kv_scales_from_amax(**k), dict(amax=p(8, dtype=F32), scale_out=p(8, dtype=F32))),
        "amax": (lambda **k: B.puzzle_kv_amax_update(**k), dict(x=p(5, 8, 64), amax=p(8, dtype=F32))),
        "init": (lambda **k: B.puzzle_decode_attn_workspace_init(d, 2, **k), dict(workspace=ws)),
        "tokens_init": (lambda **k: B.puzzle_decode_attn_tokens_workspace_init(d, 2, 2, **k), dict(workspace=ws)),
        "probe": (lambda **k: B.puzzle_hbm_read_probe(**k), dict(buf=p(64, dtype=U8), sink=p(1, dtype=torch.int64))),
    }


NAMES = ["static", "partial", "step_host", "merge", "scales", "amax", "init", "tokens_init", "probe"]
FREE = {"workspace", "staging", "buf"}          # their sizes go to the library, which checks them itself
LEADING = {("merge", "part_o"), ("amax", "x"), ("scales", "amax")}      # these tell the others' sizes


@pytest.mark.parametrize("name", NAMES)
def test_what_is_large_enough_gets_through(B, name):
    f, good = _calls(B)[name]
    with pytest.raises(AssertionError, match="no refusal"):
        f(**good)


@pytest.mark.parametrize("name", NAMES)
def test_each_tensor_has_to_be_on_the_current_device(B, name):
    f, good = _calls(B)[name]
    for arg, t in good.items():
        if isinstance(t, Pretend):
            bad = Pretend(*t.shape, dtype=t.dtype, device=1)
            with pytest.raises(ValueError, match="%s is on cuda:1, the current device is cuda:0" % arg):
                f(**{**good, arg: bad})


@pytest.mark.parametrize("name", NAMES)
def test_each_tensor_has_to_be_large_enough(B, name):
    f, good = _calls(B)[name]
    for arg, t in good.items():
        if arg in FREE or (name, arg) in LEADING:
            continue
        shape = list(t.shape)
        shape[-1] -= 1                          # the first dimension gives the batch
        bad = Pretend(*shape, dtype=t.dtype) if isinstance(t, Pretend) else torch.zeros(*shape, dtype=t.dtype)
        with pytest.raises(ValueError, match="%s has [0-9]+ elements, the call needs [0-9]+" % arg):
            f(**{**good, arg: bad})


@pytest.mark.parametrize("name", ["static", "partial", "step_host"])
def test_the_view_is_checked(B, name, monkeypatch):
    f, good = _calls(B)[name]
    for held, what in (((0, 1, 8, 1 << 40), "the cache view has 1 sequences, the call needs 2"),
                       ((0, 2, 7, 1 << 40), "the cache view has 7 scales, the call needs 8"),
                       ((1, 2, 8, 1 << 40), "the cache view is on cuda:1, the current device is cuda:0")):
        monkeypatch.setattr(B.KVView, "_held", held)
        with pytest.raises(ValueError, match=what):
            f(**good)


def test_strided_merge(B):
    """Two partial buffers of [o (2 x 8 x 64), lse (2 x 8)] one behind the other, named by their first elements."""
    rows, per = 16, 16 * 65
    buf, out = torch.zeros(2 * per), Pretend(2, 8, 64)

    def call(t, parts=2, num_parts=None, o=0, lse=rows * 64):
        a, b = Pretend(1, dtype=F32), Pretend(1, dtype=F32)
        a.t, b.t = t[o:o + 64], t[lse:lse + 1]          # short views of a long storage are enough
        B.puzzle_attn_merge_strided(a, b, 64, per, 1, per, num_parts, None, out, parts)
    with pytest.raises(AssertionError, match="no refusal"):
        call(buf)
    with pytest.raises(AssertionError, match="no refusal"):
        call(buf, parts=9, num_parts=Pretend(2, dtype=I32))       # at most so many; how many there are the device knows
    with pytest.raises(ValueError, match="part_lse reaches fewer than the %d elements" % (rows + per)):
        call(buf[:-1].clone())
    with pytest.raises(ValueError, match="part_o reaches fewer"):
        call(buf, parts=3)
    with pytest.raises(ValueError, match="num_parts has 1 elements"):
        call(buf, num_parts=Pretend(1, dtype=I32))


def test_a_rotation_keeps_its_tensors(B):
    """rope_view(rope_table(n).cuda()): the table lives as long as the description that points to it."""
    import weakref
    table, offset = Pretend(8, 64, dtype=F32), Pretend(2, dtype=I32)
    alive = weakref.ref(table), weakref.ref(offset)
    rope = B.rope_view(table, pos_offset=offset)
    del table, offset
    assert alive[0]() is not None and alive[1]() is not None
    assert rope.cos_sin == alive[0]().t.data_ptr()
    del rope
    assert alive[0]() is None and alive[1]() is None
