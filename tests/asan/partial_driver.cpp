// A program that links the model code without the decoding kernels: models that need them are refused when they are
// created, and nothing calls what is not there.  Exit status 0 when both are.
#include <cstdio>
#include <cstring>

#include "../../include/mopar.h"

static bool refused(mopar_op op, int64_t f_in, int64_t f_out) {
    mopar_tensor_desc t[2] = {{MOPAR_F32, 3, {1, 4, f_in, 0}}, {MOPAR_F32, 3, {1, 4, f_out, 0}}};
    op.in0 = 0;
    op.in1 = -1;
    op.out = 1;
    mopar_model_desc d{};
    d.dtype = MOPAR_F32;
    d.n_tensors = 2;
    d.tensors = t;
    d.n_ops = 1;
    d.ops = &op;
    d.n_layers = 1;
    d.input = 0;
    d.output = 1;
    static unsigned char weights[16];
    mopar_model_t m = nullptr;
    const int rc = mopar_model_create(&d, weights, sizeof weights, &m);
    std::printf("%d %s\n", rc, mopar_last_error());
    mopar_model_destroy(m);
    return rc == MOPAR_E_UNSUPPORTED && std::strstr(mopar_last_error(), "decoding kernels");
}

int main() {
    mopar_op rot{}, att{};
    rot.kind = MOPAR_OP_ROTARY;
    rot.heads = 1;
    rot.rotary.head_dim = rot.rotary.rot_dim = 64;
    rot.rotary.base = 10000;
    att.kind = MOPAR_OP_CAUSAL_ATTENTION;
    att.heads = att.kv_heads = 1;
    att.head_dim = 64;
    att.scale = 0.125f;
    const bool a = refused(rot, 64, 64), b = refused(att, 192, 64);
    return !(a && b);
}
