"""Head norm of rows whose squares leave float32's normal range: the stated order holds bit for bit there too, where a square that
underflows is rounded before it is added."""
import numpy as np
import pytest
import torch

import attend_ref as ref
from paper_2603_02883_b200 import fb4, synth
from test_gpu_norm_rope import as_f32, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q32():
    q = fb4.Fb4()
    yield q
    q.close()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("exp", [-62, -66, -70, -73, -75])
def test_squares_that_underflow(q32, D, interleaved, exp):
    T, H = 200, 3
    x, g, rope, plain, _ = make(T, H, 1, D, (D // 2,), interleaved, seed=D - exp)
    rng = np.random.default_rng(D - exp)
    x = torch.from_numpy((rng.standard_normal((T, H, D)) * 2.0 ** exp).astype(np.float32)).cuda().to(torch.bfloat16)
    qo, ko = q32.qk_norm_rope(x, x[:, :1], g[0], g[1], 0.0, rope)
    with np.errstate(all="ignore"):                              # a row whose squares all vanish is divided by zero
        want = ref.norm_rotate_f32(as_f32(x), as_f32(g[0]), 0.0, plain)
    finite = np.isfinite(want)
    assert finite.any()
    got = qo.cpu().view(torch.int16).numpy().view(np.uint16)
    assert np.array_equal(got[finite], synth.f32_to_bf16_bits(want)[finite])
    assert np.array_equal(np.isfinite(as_f32(qo)), finite)
