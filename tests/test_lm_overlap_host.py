"""Host-side checks of the language-model entry points: an output (or the workspace) that shares memory with an input or with another
output is refused before anything touches a GPU.  Every address here is a number that is never read."""
import pytest

from paper_2210_00129_amd import _lib

SHAPE = -2
STEP = 1 << 24                 # between two tensors of a call, more than any of them has
BF16 = 1


def _flags():
    import paper_2210_00129_amd as sbp
    return sbp.FLAG_DX_COMPACT, sbp.FLAG_DY_COMPACT, sbp.FLAG_DW_OUT_BF16


class Call:
    """A call whose tensors lie STEP apart by name; run() moves some of them."""

    def __init__(self, names):
        self.at = {n: (i + 1) * STEP for i, n in enumerate(names)}

    def run(self, **moved):
        status = self.call(dict(self.at, **moved))
        return status, _lib.lib().sbp_last_error().decode()

    def refused(self, out, other, bytes_of_other, bytes_of_out, itself=False):
        """`out` over the first and over the last 16 bytes of `other`, inside it, and (unless it may be the tensor itself) in its place."""
        a = self.at[other]
        for p in [a - bytes_of_out + 16, a + 16, a + bytes_of_other - 16] + ([] if itself else [a]):
            status, text = self.run(**{out: p - p % 16})
            assert status == SHAPE and ("overlap" in text or "must" in text), (out, other, p - a, status, text)


B, N, NK, H, HK, D = 2, 64, 40, 4, 2, 64


def _desc(at):
    return _lib.AttentionDesc(B, N, H, HK, D, 1, 0.125, 0.0, at["slopes"], at["doc"], at["prefix"])


class Forward(Call):
    sizes = dict(qkv=B * N * (H + 2 * HK) * D * 2, A=B * N * H * D * 2, lse=B * N * H * 4, doc=B * N * 4)

    def __init__(self):
        super().__init__(["qkv", "A", "lse", "slopes", "doc", "prefix"])

    def call(self, at):
        return _lib.lib().sbp_forward_attention_masked(_desc(at), at["qkv"], BF16, at["A"], at["lse"], None)


class Backward(Call):
    sizes = dict(qkv=B * NK * (H + 2 * HK) * D * 2, dqkv=B * NK * (H + 2 * HK) * D * 2, A=B * NK * H * D * 2, dA=B * NK * H * D * 2, lse=B * NK * H * 4,
                 idx=B * NK * 4, doc=B * N * 4)

    def __init__(self):
        super().__init__(["qkv", "A", "dA", "lse", "idx", "dqkv", "slopes", "doc", "prefix", "ws"])

    def call(self, at):
        L = _lib.lib()
        need = L.sbp_backward_attention_masked_workspace(_desc(at), NK, BF16)
        self.sizes["ws"] = need
        return L.sbp_backward_attention_masked(_desc(at), at["qkv"], at["A"], at["dA"], at["lse"], at["idx"], NK, BF16, at["dqkv"], at["ws"], need, None)


@pytest.mark.parametrize("out,other", [("A", "qkv"), ("lse", "qkv"), ("lse", "A"), ("A", "doc"), ("lse", "doc")])
def test_attention_forward(out, other):
    c = Forward()
    c.refused(out, other, c.sizes[other], c.sizes[out])


@pytest.mark.parametrize("out,other", [("dqkv", o) for o in ("qkv", "A", "dA", "lse", "idx", "doc")])
def test_attention_backward(out, other):
    c = Backward()
    c.refused(out, other, c.sizes[other], c.sizes[out])


@pytest.mark.parametrize("other", ["qkv", "A", "dA", "lse", "idx", "doc", "dqkv"])
def test_attention_backward_workspace(other):
    c = Backward()
    status, text = c.run(ws=c.at[other])
    assert status == SHAPE and "workspace" in text


M, K, C, G = 96, 48, 256, 2


class NormForward(Call):
    sizes = dict(x=M * C * 2, y=M * C * 2, x_out=M * C * 2, z=M * C * 2, gate=G * C * 4, gamma_post=C * 4, beta_post=C * 4, gamma_pre=C * 4, beta_pre=C * 4)

    def __init__(self):
        super().__init__(list(self.sizes))

    def call(self, at):
        d = _lib.ResidualNormDesc(M, C, 1, G, 1.0, 1e-5, 0, at["gate"], at["gamma_post"], at["beta_post"], at["gamma_pre"], at["beta_pre"])
        return _lib.lib().sbp_forward_residual_norm(d, at["x"], at["y"], BF16, at["x_out"], at["z"], None)


VECTORS = ["gate", "gamma_post", "beta_post", "gamma_pre", "beta_pre"]


@pytest.mark.parametrize("out,other", [("x_out", "x"), ("x_out", "y"), ("z", "x"), ("z", "y"), ("z", "x_out")] + [(o, v) for o in ("x_out", "z") for v in VECTORS])
def test_norms_forward(out, other):
    c = NormForward()
    c.refused(out, other, c.sizes[other], c.sizes[out], itself=(out, other) in [("x_out", "x"), ("x_out", "y")])


class NormBackward(Call):
    flags = 0

    def __init__(self):
        super().__init__(["dx_out", "dz_k", "x_out_k", "y_k", "idx", "inv", "dx", "dy_k", *["d" + v for v in VECTORS], *VECTORS, "ws"])
        kept, all_rows = K * C * 2, (K if self.flags else M) * C * 2
        self.sizes = dict(dx_out=all_rows, dx=all_rows, dz_k=kept, x_out_k=kept, y_k=kept, dy_k=kept, idx=K * 4, inv=M * 4)
        for v in VECTORS:
            self.sizes[v] = self.sizes["d" + v] = C * 4 * (G if v == "gate" else 1)

    def call(self, at):
        L = _lib.lib()
        d = _lib.ResidualNormDesc(M, C, 1, G, 1.0, 1e-5, 0, at["gate"], at["gamma_post"], at["beta_post"], at["gamma_pre"], at["beta_pre"])
        need = L.sbp_backward_residual_norm_workspace(d, K, BF16, self.flags)
        g = _lib.ResidualNormGrads(*[at["d" + v] for v in VECTORS])
        return L.sbp_backward_residual_norm(d, at["dx_out"], at["dz_k"], at["x_out_k"], at["y_k"], at["idx"], at["inv"], K, BF16, at["dx"], at["dy_k"], g, at["ws"],
                                            need, self.flags, None)


class NormBackwardCompact(NormBackward):
    flags = _flags()[0]


ITSELF = [("dx", "dx_out"), ("dy_k", "y_k"), ("dy_k", "dz_k")]


@pytest.mark.parametrize("cls", [NormBackward, NormBackwardCompact])
@pytest.mark.parametrize("out", ["dx", "dy_k", *["d" + v for v in VECTORS]])
def test_norms_backward(cls, out):
    c = cls()
    others = ["dx_out", "dz_k", "x_out_k", "y_k", *VECTORS, "dx", "dy_k", *["d" + v for v in VECTORS]] + ([] if cls.flags else ["idx", "inv"])
    for other in others:
        if other != out:
            c.refused(out, other, c.sizes[other], c.sizes[out], itself=(out, other) in ITSELF)
    status, text = c.run(**{out: c.at["ws"]})
    assert status == SHAPE and "workspace" in text


V, EM, EK, EC = 300, 600, 400, 64


class Lookup(Call):
    sizes = dict(tokens=EM * 8, table=V * EC * 2, E=EM * EC * 2)

    def __init__(self):
        super().__init__(list(self.sizes))

    def call(self, at):
        return _lib.lib().sbp_forward_embedding(at["tokens"], 8, at["table"], EM, V, EC, 1.0, BF16, at["E"], None)


class TableGradient(Call):
    flags = 0

    def __init__(self):
        super().__init__(["dE", "tokens", "idx", "dtable", "ws"])
        compact, bf16 = _flags()[1] & self.flags, _flags()[2] & self.flags
        self.sizes = dict(dE=(EK if compact else EM) * EC * 2, tokens=EM * 8, idx=EK * 4, dtable=V * EC * (2 if bf16 else 4))

    def call(self, at):
        L = _lib.lib()
        need = L.sbp_backward_embedding_workspace(EM, EK, V, EC, BF16, self.flags)
        return L.sbp_backward_embedding(at["dE"], at["tokens"], 8, at["idx"], EM, EK, V, EC, 1.0, BF16, at["dtable"], at["ws"], need, self.flags, None)


@pytest.mark.parametrize("other", ["tokens", "table"])
def test_lookup(other):
    c = Lookup()
    c.refused("E", other, c.sizes[other], c.sizes["E"])


@pytest.mark.parametrize("flags", [0, 1, 2])
def test_table_gradient(flags):
    c = type("T", (TableGradient,), dict(flags=[0, _flags()[1], _flags()[2]][flags]))()
    for other in ("dE", "tokens", "idx"):
        c.refused("dtable", other, c.sizes[other], c.sizes["dtable"])
    for other in ("dE", "tokens", "idx", "dtable"):
        status, text = c.run(ws=c.at[other])
        assert status == SHAPE and "workspace" in text
