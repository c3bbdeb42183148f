"""Every form of the products with 4-bit weights, at sizes that choose it: few tokens with one or two tiles of outputs and four or eight wavefronts, more tokens with two,
four or eight teams, one to four tiles of tokens, two tiles of outputs - outputs and inputs that no tile divides, enough chunks for the loops to turn.
Against float64 on the GPU, with np_kv8.w4's bound."""
import pytest
import torch

from paper_2311_03285_amd import slora
from test_gpu_w4 import DTYPES, run

pytestmark = pytest.mark.gpu


class Large:
    """as test_gpu_w4.Matrix, made on the GPU"""

    def __init__(self, outputs, inputs, group, dtype, zeros, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        groups = -(-inputs // group)
        self.lib_dtype, t = DTYPES[dtype]
        self.shape, self.group = (outputs, inputs), group
        self.codes = torch.randint(0, 16, (outputs, inputs), dtype=torch.uint8, device="cuda", generator=g)
        self.scales = ((0.5 + torch.rand((outputs, groups), device="cuda", generator=g)) / 4.6 / inputs ** 0.5).to(t)
        self.zeros = torch.randint(0, 16, (outputs, groups), dtype=torch.uint8, device="cuda", generator=g) if zeros else None
        nibbles = (self.codes[:, 0::2] | (self.codes[:, 1::2] << 4)).contiguous()
        self.packed = torch.full((slora.w4_bytes(outputs, inputs, group),), 0xA5, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        self.handle = slora.w4_pack(outputs, inputs, group, self.lib_dtype, nibbles.data_ptr(), self.scales.data_ptr(), self.zeros.data_ptr() if zeros else None,
                                    self.packed.data_ptr())
        torch.cuda.synchronize()

    def check(self, x, y):
        inputs = self.shape[1]
        at = torch.arange(inputs, device="cuda") // self.group
        half = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[y.dtype]
        for o in range(0, self.shape[0], 4096):
            c, s = self.codes[o:o + 4096].double(), self.scales[o:o + 4096].double()[:, at]
            z = self.zeros[o:o + 4096].double()[:, at] if self.zeros is not None else 8.0
            ref = x.double() @ ((c - z) * s).t().contiguous()
            bound = x.double().abs() @ ((c + z) * s).t().contiguous() * 2.0 ** -23 * (4 + inputs ** 0.5)
            err = (y[:, o:o + 4096].double() - ref).abs()
            assert (err <= bound + ref.abs() * half + 2.0 ** -24 * (half > 0)).all(), (o, float((err - bound).max()))


def one(outputs, inputs, group, dtype, T, y16, zeros):
    m = Large(outputs, inputs, group, dtype, zeros, outputs + T)
    x = torch.randn(T, inputs, device="cuda").to(DTYPES[dtype][1])
    m.check(x, run([m], [x], T, y16)[0])
    slora.w4_destroy(m.handle)


# up to four tokens.  Tiles of 16 outputs: 313 (one a workgroup), 513 (two, eight wavefronts), 2049 (two, four wavefronts)
@pytest.mark.parametrize("T", [1, 2, 3, 4])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("outputs,inputs", [(5003, 4104), (5003, 12296), (8200, 4104), (8200, 8200), (32780, 2056), (32780, 4104)])
def test_few_tokens(outputs, inputs, group, T):
    one(outputs, inputs, group, ["f16", "bf16"][(T + group // 32) % 2], T, T % 2 == 0, T != 2)


# more.  Workgroups of 16 outputs and 16 to 64 tokens: up to 256 (eight teams, up to 32 tokens of one), up to 512 (four), more (two; from 1536 on, of 48 tokens, two
# tiles of outputs)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("outputs,T", [(300, 5), (300, 32), (4200, 9), (4200, 20), (8300, 6), (8300, 16), (8300, 30), (300, 40), (8300, 40), (24600, 40), (6200, 67), (12300, 67),
                                       (12300, 80), (300, 64), (8300, 64), (4200, 128), (8300, 130)])
def test_more_tokens(outputs, T, group):
    for inputs in (1032, 4104):
        one(outputs, inputs, group, ["f16", "bf16"][(T + group // 32) % 2], T, T % 3 == 0, T != 40)


def test_several_matrices_share_a_launch_of_each_form():
    for outputs, T in [((5000, 4000, 3), 2), ((20000, 9, 14000), 4), ((2000, 17, 1900), 20), ((4100, 33, 8200), 67), ((9000, 16, 16000), 67)]:
        ms = [Large(o, i, 64, "bf16", True, o) for o, i in zip(outputs, (520, 4104, 1032))]
        xs = [torch.randn(T, m.shape[1], device="cuda").bfloat16() for m in ms]
        for m, x, y in zip(ms, xs, run(ms, xs, T, False)):
            m.check(x, y)
        for m in ms:
            slora.w4_destroy(m.handle)
