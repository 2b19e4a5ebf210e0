"""Every tensor of the operators around the projections and of decode_shared is refused where it lies on another device than the current one
(wrappers without memory stand for those, so this needs one GPU only)."""
import pytest

from test_gpu_other_device import _elsewhere

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


def _calls(B):
    import torch
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")
    i, f, u = (lambda *s, d=d: z(*s, dtype=d) for d in (torch.int32, torch.float32, torch.uint8))
    freq = z(32, dtype=torch.float64)
    shared = dict(q=z(5, 4, 64), cache=z(8, 1, 2, 1024), table=i(5, 2), lens=i(5), off=i(3), sh=i(2), out=z(5, 4, 64), k=z(5, 1, 64), v=z(5, 1, 64),
                  slots=torch.full((5,), -1, dtype=torch.int64, device="cuda"), ws=u(64))
    return {
        "add_rms_norm": (dict(x=z(4, 64), w=z(64), out=u(4, 64), res=z(4, 64), s=f(4)),
                         lambda a: B.add_rms_norm(a["x"], a["w"], a["out"], 1e-5, residual=a["res"], scales=a["s"])),
        "rotary": (dict(q=z(5, 4, 64), k=z(5, 1, 64), pos=i(5), f=freq), lambda a: B.rotary(a["q"], a["k"], a["pos"], a["f"])),
        "rotary_mixed": (dict(q=z(5, 4, 64), k=z(5, 1, 64), cu=i(2), lens=i(3), f=freq), lambda a: B.rotary_mixed(a["q"], a["k"], a["cu"], a["lens"], 1, a["f"])),
        "decode_shared": (shared, lambda a: B.decode_shared(a["q"], a["cache"], a["table"], a["lens"], 32, a["off"], a["sh"], a["out"], 0.1, a["k"], a["v"], a["slots"], a["ws"])),
        "decode_shared, block scales": ({**shared, "cache": u(8, 1, 2, 1024), "scales": f(8, 1, 2)},
                                        lambda a: B.decode_shared(a["q"], a["cache"], a["table"], a["lens"], 32, a["off"], a["sh"], a["out"], 0.1, a["k"], a["v"], a["slots"], a["ws"],
                                                                  kv_scales=a["scales"])),
    }


@pytest.mark.parametrize("name", ["add_rms_norm", "rotary", "rotary_mixed", "decode_shared", "decode_shared, block scales"])
def test_tensors_of_another_device_are_refused(B, name):
    import torch
    args, call = _calls(B)[name]
    call(args)
    for arg, t in args.items():
        with pytest.raises(RuntimeError, match="on the current device is wanted, not on cuda:1"):
            call({**args, arg: _elsewhere(t)})
            pytest.fail(f"{arg} is not looked at")
    torch.cuda.synchronize()
