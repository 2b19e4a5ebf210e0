"""Every tensor of the calls over 8-bit codes with scales, and of the tables, is refused where it lies on another device than the current one.
The tensors of another device are wrappers without memory, so this needs one GPU only: what gets past the check is refused further on, by
another name."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


def _elsewhere(t):
    """A tensor like t, on a device that need not exist."""
    import torch

    class Elsewhere(torch.Tensor):
        @classmethod
        def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
            raise AssertionError(f"{func} of a tensor without memory")
    return torch.Tensor._make_wrapper_subclass(Elsewhere, t.shape, strides=t.stride(), dtype=t.dtype, device="cuda:1")


def _calls(B):
    """name -> (arguments by name, call)."""
    import torch
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")
    i, f, u, c = (lambda *s, d=d: z(*s, dtype=d) for d in (torch.int32, torch.float32, torch.uint8, torch.int8))
    attn = dict(q=z(5, 4, 64), cache=u(8, 1, 2, 1024), table=i(2, 2), cu=i(3), lens=i(2), out=z(5, 4, 64), k=z(5, 1, 64), v=z(5, 1, 64),
                slots=torch.full((5,), -1, dtype=torch.int64, device="cuda"), ws=u(64), scales=f(8, 1, 2))
    new = lambda a: dict(k_new=a["k"], v_new=a["v"], slot_mapping=a["slots"], workspace=a["ws"], kv_scales=a["scales"])
    without = lambda a, *names: {k: v for k, v in a.items() if k not in names}
    rows = {**without(attn, "cu"), "table": i(5, 2), "lens": i(5)}
    both = {**attn, "cu": i(2)}
    tables = dict(new=i(3), lens=i(3), table=i(3, 4), free=i(9), count=i(1), cu=i(2), slots=z(7, dtype=torch.int64), taken=i(3), ws=u(64))
    return {
        "kv_write": (without(attn, "q", "table", "cu", "lens", "out", "ws"), lambda a: B.kv_write(a["k"], a["v"], a["slots"], a["cache"], kv_scales=a["scales"])),
        "prefill": (attn, lambda a: B.prefill(a["q"], a["cache"], a["table"], a["cu"], a["lens"], 3, 32, a["out"], 0.1, **new(a))),
        "decode": (rows, lambda a: B.decode(a["q"], a["cache"], a["table"], a["lens"], 32, a["out"], 0.1, **new(a))),
        "mixed": (both, lambda a: B.mixed(a["q"], a["cache"], a["table"], a["cu"], a["lens"], 1, 4, 32, 32, a["out"], 0.1, **new(a))),
        "tables_append": (tables, lambda a: B.tables_append(a["new"], 1, 5, a["lens"], a["table"], a["free"], a["count"], a["cu"], a["slots"], a["taken"], a["ws"])),
        "tables_truncate": (without(tables, "cu", "slots", "taken"), lambda a: B.tables_truncate(a["new"], a["lens"], a["table"], a["free"], a["count"], a["ws"])),
        "quantize_rows_int8": (dict(x=z(4, 64), codes=c(4, 64), scales=f(4)), lambda a: B.quantize_rows_int8(a["x"], a["codes"], a["scales"])),
        "quantize_recv_int8": (dict(x=z(1, 4, 2, 128), codes=c(1, 4, 2, 128), scales=f(4)), lambda a: B.quantize_recv_int8(a["x"], a["codes"], a["scales"])),
        "qkv_proj_pack_int8": (dict(x=c(4, 256), xs=f(4), w=c(768, 256), ws=f(768), send=z(1, 4, 6, 128), work=u(64)),
                               lambda a: B.qkv_proj_pack_int8(a["x"], a["xs"], a["w"], a["ws"], a["send"], 1, 4, 1, a["work"])),
        "unpack_o_proj_int8": (dict(x=c(1, 4, 2, 128), xs=f(4), w=c(256, 256), ws=f(256), out=z(4, 256), work=u(64)),
                               lambda a: B.unpack_o_proj_int8(a["x"], a["xs"], a["w"], a["ws"], a["out"], a["work"])),
    }


@pytest.mark.parametrize("name", ["kv_write", "prefill", "decode", "mixed", "tables_append", "tables_truncate", "quantize_rows_int8", "quantize_recv_int8",
                                  "qkv_proj_pack_int8", "unpack_o_proj_int8"])
def test_tensors_of_another_device_are_refused(B, name):
    import torch
    args, call = _calls(B)[name]
    call(args)
    for arg, t in args.items():
        with pytest.raises(RuntimeError, match="on the current device is wanted, not on cuda:1"):
            call({**args, arg: _elsewhere(t)})
            pytest.fail(f"{arg} is not looked at")
    torch.cuda.synchronize()
