"""Layer normalisation with more rows than teams of threads, on the GPU: every team of every size takes a
second row and more, not all of them the same number; groups that do not divide the number of teams, or
outnumber them. Oracle and tolerances are those of test_gpu_norm."""
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import test_gpu_norm as N  # noqa: E402


# (teams: 262144 threads forwards, 131072 backwards, of 128, 256, 512 or 1024 each)
@pytest.mark.parametrize("rows,D,type_", [
    (2100, 2048, "bf16"), (2111, 1999, "f16"), (2100, 1024, "f32"), (1300, 4096, "bf16"), (1111, 2049, "f32"),
    (650, 8192, "bf16"), (1031, 8191, "f16"), (650, 4096, "f32"), (600, 16384, "bf16"), (390, 9001, "f16"),
    (600, 8192, "f32"), (300, 16384, "f32"), (301, 12345, "f32")])
def test_more_rows_than_teams(rows, D, type_):
    say("layernorm rows than teams", rows, D, type_)
    x, w, b, g = N.make((rows, D), type_, w32=rows % 2 == 1)
    N.check(x, w, b, g, 1e-5)


@pytest.mark.parametrize("shape,type_", [
    ((5500, 3, 24), "bf16"), ((2400, 7, 100), "f16"), ((700, 7, 100), "f32"), ((180, 7, 1500), "bf16"),
    ((90, 7, 3000), "f16"), ((2, 300, 16384), "bf16"), ((3, 150, 9000), "f32"), ((5, 3, 20000), "f16"),
    ((2, 40, 20000), "f32"), ((70, 2, 17000), "bf16")])
def test_more_rows_than_teams_in_groups(shape, type_):
    say("layernorm groups and teams", shape, type_)
    x, w, b, g = N.make(shape, type_, G=shape[-2], w32=shape[0] % 2 == 1)
    N.check(x, w, b, g, 1e-5, groups=True)


@pytest.mark.parametrize("D,type_", [(2048, "bf16"), (4096, "f16"), (4096, "f32"), (16384, "bf16"), (16384, "f32")])
def test_rows_do_not_depend_on_their_number(D, type_):
    """The rows that teams take second give the bits that they give alone."""
    say("layernorm rows alone", D, type_)
    n = 2 * 262144 // 128 // (D // 2048) + 5
    x, w, b, g = N.make((n, D), type_)
    r = N.D.deer_layernorm(x, w, b)
    a = N.D.deer_layernorm_adjoint(x, g, r["mean"], r["rstd"], w)
    few = slice(n - 100, n)
    r1 = N.D.deer_layernorm(x[few], w, b)
    a1 = N.D.deer_layernorm_adjoint(x[few], g[few], r1["mean"], r1["rstd"], w)
    assert all(torch.equal(r[m][few], r1[m]) for m in r) and torch.equal(a["x"][few], a1["x"])
