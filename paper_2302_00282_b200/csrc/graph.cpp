// Graph construction with shape inference, and the compile driver.
#include "graph.hpp"

#include <algorithm>
#include <cmath>

namespace xenos {

static bool finite_all(const float *p, size_t n) {
    for (size_t i = 0; i < n; ++i)
        if (!std::isfinite(p[i])) return false;
    return true;
}

// Why a tensor cannot be read by an operator (null when it can): labels and the results of a LOGPROB.
static const char *not_an_operand(const Graph &g, int t) {
    const Tensor &x = g.tensors[t];
    if (x.fixed >= 0) return "results of a LOGPROB can only be graph outputs";
    if (x.input_slot >= 0 && x.io_dtype == XENOS_DTYPE_I32) return "an I32 input can only be the labels of a LOGPROB";
    return nullptr;
}

// Appends one user operator; the output extent of window operators is
// floor((in + 2*pad - k) / stride) + 1.
xenos_status_t infer_and_append(Graph &g, const xenos_op_desc_t &d, const int *in, int n_in, int *out) {
    for (int i = 0; i < n_in; ++i)
        if (in[i] < 0 || in[i] >= (int)g.tensors.size()) return fail(g, XENOS_E_INVALID, "add_op: bad input tensor id");
    for (int i = 0; i < n_in; ++i)
        if (const char *why = not_an_operand(g, in[i])) return fail(g, XENOS_E_UNSUPPORTED, std::string("add_op: ") + why);
    const Tensor x = g.tensors[in[0]];
    Op op;
    op.kind = d.kind;
    op.in.assign(in, in + n_in);
    Tensor y;
    auto need_inputs = [&](int n) { return n_in == n; };
    bool has_bn = d.bn_gamma || d.bn_beta || d.bn_mean || d.bn_var;
    if (has_bn && !(d.bn_gamma && d.bn_beta && d.bn_mean && d.bn_var))
        return fail(g, XENOS_E_INVALID, "add_op: BatchNorm needs gamma, beta, mean and var together");
    if (d.act != XENOS_ACT_NONE && d.act != XENOS_ACT_RELU && d.act != XENOS_ACT_RELU6)
        return fail(g, XENOS_E_INVALID, "add_op: unknown activation");

    switch (d.kind) {
    case XENOS_OP_CONV: {
        if (!need_inputs(1)) return fail(g, XENOS_E_INVALID, "conv takes one input");
        if (x.is_vec) return fail(g, XENOS_E_SHAPE, "conv input must be a feature map");
        if (!d.weight) return fail(g, XENOS_E_INVALID, "conv: weight is NULL");
        if (d.kh != d.kw) return fail(g, XENOS_E_UNSUPPORTED, "conv: only square kernels");
        if (d.kh < 1 || d.stride < 1 || d.pad < 0 || d.cout < 1 || d.groups < 1)
            return fail(g, XENOS_E_SHAPE, "conv: bad kernel / stride / pad / cout / groups");
        if (x.c % d.groups || d.cout % d.groups) return fail(g, XENOS_E_SHAPE, "conv: groups must divide Cin and Cout");
        if (d.groups != 1 && !(d.groups == x.c && d.cout == x.c))
            return fail(g, XENOS_E_UNSUPPORTED, "conv: groups must be 1 (dense) or Cin == Cout (depthwise)");
        y.c = d.cout;
        y.h = out_dim(x.h, d.kh, d.stride, d.pad);
        y.w = out_dim(x.w, d.kh, d.stride, d.pad);
        if (y.h < 1 || y.w < 1) return fail(g, XENOS_E_SHAPE, "conv: kernel larger than padded input");
        size_t nw = (size_t)d.cout * (x.c / d.groups) * d.kh * d.kh;
        if (!finite_all(d.weight, nw)) return fail(g, XENOS_E_INVALID, "conv: non-finite weight");
        op.w.assign(d.weight, d.weight + nw);
        op.cout = d.cout; op.k = d.kh; op.stride = d.stride; op.pad = d.pad; op.groups = d.groups;
        break;
    }
    case XENOS_OP_FC: {
        if (!need_inputs(1)) return fail(g, XENOS_E_INVALID, "fc takes one input");
        if (!x.is_vec) return fail(g, XENOS_E_SHAPE, "fc input must be a vector (e.g. a global pool output)");
        if (!d.weight || d.cout < 1) return fail(g, XENOS_E_INVALID, "fc: weight is NULL or cout < 1");
        size_t nw = (size_t)d.cout * x.c;
        if (!finite_all(d.weight, nw)) return fail(g, XENOS_E_INVALID, "fc: non-finite weight");
        op.w.assign(d.weight, d.weight + nw);
        op.cout = d.cout; op.k = 1; op.groups = 1;
        y.c = d.cout; y.is_vec = true;
        break;
    }
    case XENOS_OP_POOL_MAX:
    case XENOS_OP_POOL_AVG: {
        if (!need_inputs(1)) return fail(g, XENOS_E_INVALID, "pool takes one input");
        if (x.is_vec) return fail(g, XENOS_E_SHAPE, "pool input must be a feature map");
        if (d.kh != d.kw || d.kh < 1 || d.stride < 1 || d.pad < 0) return fail(g, XENOS_E_SHAPE, "pool: bad window");
        if (d.pad >= d.kh) return fail(g, XENOS_E_SHAPE, "pool: pad must be smaller than the window");
        if (d.kind == XENOS_OP_POOL_AVG && d.pad != 0)
            return fail(g, XENOS_E_UNSUPPORTED, "avg pool with padding is not implemented");
        y.c = x.c;
        y.h = out_dim(x.h, d.kh, d.stride, d.pad);
        y.w = out_dim(x.w, d.kh, d.stride, d.pad);
        if (y.h < 1 || y.w < 1) return fail(g, XENOS_E_SHAPE, "pool: window larger than padded input");
        op.k = d.kh; op.stride = d.stride; op.pad = d.pad;
        break;
    }
    case XENOS_OP_POOL_GLOBAL_AVG:
        if (!need_inputs(1)) return fail(g, XENOS_E_INVALID, "global pool takes one input");
        if (x.is_vec) return fail(g, XENOS_E_SHAPE, "global pool input must be a feature map");
        y.c = x.c; y.is_vec = true;
        break;
    case XENOS_OP_ADD: {
        if (!need_inputs(2)) return fail(g, XENOS_E_INVALID, "add takes two inputs");
        const Tensor &b = g.tensors[in[1]];
        if (x.c != b.c || x.h != b.h || x.w != b.w || x.is_vec != b.is_vec)
            return fail(g, XENOS_E_SHAPE, "add: operand shapes differ");
        y.c = x.c; y.h = x.h; y.w = x.w; y.is_vec = x.is_vec;
        break;
    }
    case XENOS_OP_CONCAT: {
        if (n_in < 2) return fail(g, XENOS_E_INVALID, "concat takes at least two inputs");
        if (x.is_vec) return fail(g, XENOS_E_SHAPE, "concat inputs must be feature maps");
        int c = 0;
        for (int i = 0; i < n_in; ++i) {
            const Tensor &t = g.tensors[in[i]];
            if (t.is_vec || t.h != x.h || t.w != x.w) return fail(g, XENOS_E_SHAPE, "concat: spatial extents differ");
            c += t.c;
        }
        y.c = c; y.h = x.h; y.w = x.w;
        break;
    }
    case XENOS_OP_RELU:
    case XENOS_OP_RELU6:
        if (!need_inputs(1)) return fail(g, XENOS_E_INVALID, "activation takes one input");
        y.c = x.c; y.h = x.h; y.w = x.w; y.is_vec = x.is_vec;
        break;
    case XENOS_OP_BATCHNORM:
        if (!need_inputs(1)) return fail(g, XENOS_E_INVALID, "batchnorm takes one input");
        if (!has_bn) return fail(g, XENOS_E_INVALID, "batchnorm: parameters are NULL");
        y.c = x.c; y.h = x.h; y.w = x.w; y.is_vec = x.is_vec;
        break;
    case XENOS_OP_MUL:
    case XENOS_OP_MAC: {
        const int need = d.kind == XENOS_OP_MUL ? 2 : 3;
        if (!need_inputs(need)) return fail(g, XENOS_E_INVALID, d.kind == XENOS_OP_MUL ? "mul takes two inputs" : "mac takes three inputs");
        for (int i = 1; i < need; ++i) {
            const Tensor &b = g.tensors[in[i]];
            if (x.c != b.c || x.h != b.h || x.w != b.w || x.is_vec != b.is_vec)
                return fail(g, XENOS_E_SHAPE, "mul / mac: operand shapes differ");
        }
        y.c = x.c; y.h = x.h; y.w = x.w; y.is_vec = x.is_vec;
        break;
    }
    case XENOS_OP_TRANSPOSE:
        if (!need_inputs(1)) return fail(g, XENOS_E_INVALID, "transpose takes one input");
        if (x.is_vec || x.w != 1) return fail(g, XENOS_E_SHAPE, "transpose input must be a matrix (a feature map of width 1)");
        y.c = x.h; y.h = x.c; y.w = 1;
        break;
    case XENOS_OP_SPLIT:
        if (!need_inputs(1)) return fail(g, XENOS_E_INVALID, "split takes one input");
        if (x.is_vec) return fail(g, XENOS_E_SHAPE, "split input must be a feature map");
        if (d.cout < 1 || d.pad < 0 || d.pad + d.cout > x.c) return fail(g, XENOS_E_SHAPE, "split: channels [pad, pad + cout) leave the input");
        y.c = d.cout; y.h = x.h; y.w = x.w;
        op.cout = d.cout; op.pad = d.pad;
        break;
    case XENOS_OP_MATMUL: {
        if (n_in == 2) return fail(g, XENOS_E_UNSUPPORTED, "matmul of two run-time tensors is not implemented; the right operand is a constant (weight)");
        if (!need_inputs(1)) return fail(g, XENOS_E_INVALID, "matmul takes one input and a constant matrix");
        if (!x.is_vec && x.w != 1) return fail(g, XENOS_E_SHAPE, "matmul input must be a matrix (a feature map of width 1) or a vector");
        if (!d.weight || d.cout < 1) return fail(g, XENOS_E_INVALID, "matmul: weight is NULL or cout < 1");
        size_t nw = (size_t)x.c * d.cout;
        if (!finite_all(d.weight, nw)) return fail(g, XENOS_E_INVALID, "matmul: non-finite weight");
        // kept as [cout][c], the form of a pointwise convolution / fc
        op.w.resize(nw);
        for (int k = 0; k < x.c; ++k)
            for (int n = 0; n < d.cout; ++n) op.w[(size_t)n * x.c + k] = d.weight[(size_t)k * d.cout + n];
        op.cout = d.cout; op.k = 1; op.groups = 1;
        y.c = d.cout; y.h = x.h; y.w = x.w; y.is_vec = x.is_vec;
        break;
    }
    case XENOS_OP_LAYERNORM:
        if (!need_inputs(1)) return fail(g, XENOS_E_INVALID, "layernorm takes one input");
        if (!d.weight) return fail(g, XENOS_E_INVALID, "layernorm: weight is NULL");
        if (d.cout != 0 && d.cout != x.c) return fail(g, XENOS_E_SHAPE, "layernorm: the parameters are for rows of another length");
        if (!finite_all(d.weight, x.c) || (d.bias && !finite_all(d.bias, x.c))) return fail(g, XENOS_E_INVALID, "layernorm: non-finite parameter");
        if (!(d.bn_eps > 0.0f) || !std::isfinite(d.bn_eps)) return fail(g, XENOS_E_INVALID, "layernorm: bn_eps must be positive");
        op.w.assign(d.weight, d.weight + x.c);
        if (d.bias) op.bias.assign(d.bias, d.bias + x.c);
        op.has_bias = d.bias != nullptr;
        op.eps = d.bn_eps;
        y.c = x.c; y.h = x.h; y.w = x.w; y.is_vec = x.is_vec;
        break;
    case XENOS_OP_QMATMUL:
        return fail(g, XENOS_E_UNSUPPORTED, "add_op: an 8-bit product is added by xenos_graph_add_qmatmul");
    case XENOS_OP_LOGPROB:
        return fail(g, XENOS_E_UNSUPPORTED, "add_op: log-probabilities are added by xenos_graph_add_logprob");
    default:
        return fail(g, XENOS_E_UNSUPPORTED, "add_op: unknown operator kind");
    }

    int cpar = (d.kind == XENOS_OP_BATCHNORM) ? x.c : d.cout;
    if (d.kind == XENOS_OP_CONV || d.kind == XENOS_OP_FC || d.kind == XENOS_OP_MATMUL) {
        op.act = d.act;
        if (d.bias) {
            if (!finite_all(d.bias, d.cout)) return fail(g, XENOS_E_INVALID, "non-finite bias");
            op.bias.assign(d.bias, d.bias + d.cout);
            op.has_bias = true;
        }
    } else if (d.act != XENOS_ACT_NONE && d.kind != XENOS_OP_ADD) {
        return fail(g, XENOS_E_INVALID, "add_op: activation only attaches to conv, fc and add");
    } else {
        op.act = d.act;
    }
    if (has_bn) {
        if (d.kind != XENOS_OP_CONV && d.kind != XENOS_OP_FC && d.kind != XENOS_OP_MATMUL && d.kind != XENOS_OP_BATCHNORM)
            return fail(g, XENOS_E_INVALID, "add_op: BatchNorm parameters on an operator that cannot carry them");
        if (!(d.bn_eps > 0.0f)) return fail(g, XENOS_E_INVALID, "batchnorm: eps must be positive");
        if (!finite_all(d.bn_gamma, cpar) || !finite_all(d.bn_beta, cpar) || !finite_all(d.bn_mean, cpar) ||
            !finite_all(d.bn_var, cpar))
            return fail(g, XENOS_E_INVALID, "batchnorm: non-finite parameter");
        for (int i = 0; i < cpar; ++i)
            if (!(d.bn_var[i] + d.bn_eps > 0.0f)) return fail(g, XENOS_E_INVALID, "batchnorm: var + eps must be positive");
        op.gamma.assign(d.bn_gamma, d.bn_gamma + cpar);
        op.beta.assign(d.bn_beta, d.bn_beta + cpar);
        op.mean.assign(d.bn_mean, d.bn_mean + cpar);
        op.var.assign(d.bn_var, d.bn_var + cpar);
        op.eps = d.bn_eps;
        op.has_bn = true;
    }

    int opi = (int)g.ops.size();
    y.producer = opi;
    g.tensors.push_back(y);
    op.out = (int)g.tensors.size() - 1;
    for (int i = 0; i < n_in; ++i) g.tensors[in[i]].consumers.push_back(opi);
    g.ops.push_back(std::move(op));
    *out = g.ops.back().out;
    return XENOS_OK;
}

static void append_op(Graph &g, Op &&op, const Tensor *y, int n_out, int *ids) {
    const int opi = (int)g.ops.size();
    for (int i = 0; i < n_out; ++i) {
        g.tensors.push_back(y[i]);
        g.tensors.back().producer = opi;
        ids[i] = (int)g.tensors.size() - 1;
    }
    for (int t : op.in) g.tensors[t].consumers.push_back(opi);
    g.ops.push_back(std::move(op));
}

xenos_status_t append_qmatmul(Graph &g, const xenos_qmatmul_desc_t &d, int in, int *out) {
    if (in < 0 || in >= (int)g.tensors.size()) return fail(g, XENOS_E_INVALID, "add_qmatmul: bad input tensor id");
    if (const char *why = not_an_operand(g, in)) return fail(g, XENOS_E_UNSUPPORTED, std::string("add_qmatmul: ") + why);
    const Tensor x = g.tensors[in];
    if (d.cout < 1) return fail(g, XENOS_E_SHAPE, "add_qmatmul: cout must be positive");
    if (d.c != x.c) return fail(g, XENOS_E_SHAPE, "add_qmatmul: the weights are for rows of another length");
    if ((d.weight != nullptr) == (d.weight_i8 != nullptr)) return fail(g, XENOS_E_INVALID, "add_qmatmul: give either weight or weight_i8");
    if ((d.scale != nullptr) != (d.weight_i8 != nullptr)) return fail(g, XENOS_E_INVALID, "add_qmatmul: scale goes with weight_i8");
    if (d.act != XENOS_ACT_NONE && d.act != XENOS_ACT_RELU && d.act != XENOS_ACT_RELU6) return fail(g, XENOS_E_INVALID, "add_qmatmul: unknown activation");
    // (the int32 sum of 131072 products of at most 127 * 128 stays below 2^31)
    if (x.c > 131072) return fail(g, XENOS_E_UNSUPPORTED, "add_qmatmul: more than 131072 channels would overflow the sum");
    const size_t n = (size_t)d.cout * x.c;
    Op op;
    op.kind = XENOS_OP_QMATMUL;
    op.in = {in};
    op.cout = d.cout; op.k = 1; op.act = d.act;
    if (d.weight_i8) {
        if (!finite_all(d.scale, d.cout)) return fail(g, XENOS_E_INVALID, "add_qmatmul: non-finite scale");
        op.q.assign(d.weight_i8, d.weight_i8 + n);
        op.gamma.assign(d.scale, d.scale + d.cout);
    } else {
        if (!finite_all(d.weight, n)) return fail(g, XENOS_E_INVALID, "add_qmatmul: non-finite weight");
        op.q.resize(n);
        op.gamma.resize(d.cout);
        for (int o = 0; o < d.cout; ++o) {
            const float *w = d.weight + (size_t)o * x.c;
            double a = 0;
            for (int k = 0; k < x.c; ++k) a = std::max(a, std::fabs((double)w[k]));
            op.gamma[o] = (float)(a / 127.0);
            for (int k = 0; k < x.c; ++k) op.q[(size_t)o * x.c + k] = a > 0 ? (int8_t)std::nearbyint(127.0 * w[k] / a) : (int8_t)0;
        }
    }
    if (d.bias) {
        if (!finite_all(d.bias, d.cout)) return fail(g, XENOS_E_INVALID, "add_qmatmul: non-finite bias");
        op.bias.assign(d.bias, d.bias + d.cout);
        op.has_bias = true;
    }
    Tensor y;
    y.c = d.cout; y.h = x.h; y.w = x.w; y.is_vec = x.is_vec;
    op.out = (int)g.tensors.size();
    append_op(g, std::move(op), &y, 1, out);
    return XENOS_OK;
}

xenos_status_t append_logprob(Graph &g, int logits, int labels, int top, int *out) {
    for (int i = 0; i < 4; ++i) out[i] = -1;
    if (logits < 0 || logits >= (int)g.tensors.size() || labels < -1 || labels >= (int)g.tensors.size())
        return fail(g, XENOS_E_INVALID, "add_logprob: bad tensor id");
    if (const char *why = not_an_operand(g, logits)) return fail(g, XENOS_E_UNSUPPORTED, std::string("add_logprob: ") + why);
    if (top < 0 || top > 32) return fail(g, XENOS_E_INVALID, "add_logprob: top must be 0..32");
    const Tensor x = g.tensors[logits];
    if (x.c > 1 << 30) return fail(g, XENOS_E_UNSUPPORTED, "add_logprob: more than 2^30 scores in a row");
    int n_labels = 0;
    if (labels >= 0) {
        const Tensor &l = g.tensors[labels];
        if (l.input_slot < 0 || l.io_dtype != XENOS_DTYPE_I32) return fail(g, XENOS_E_INVALID, "add_logprob: labels must be an I32 input");
        if (x.is_vec ? l.h != 1 || l.w != 1 : l.h != x.h || l.w != x.w) return fail(g, XENOS_E_SHAPE, "add_logprob: labels and logits have different rows");
        n_labels = l.c;
    }
    Op op;
    op.kind = XENOS_OP_LOGPROB;
    op.in = {logits};
    if (labels >= 0) op.in.push_back(labels);
    op.top = top;
    Tensor y[4];
    int which[4], n = 0;
    const int count[4] = {n_labels, 1, top, top};
    for (int i = 0; i < 4; ++i) {
        if (!count[i]) continue;
        y[n].c = count[i]; y[n].h = x.h; y[n].w = x.w; y[n].is_vec = x.is_vec;
        y[n].fixed = i == 2 ? XENOS_DTYPE_I32 : XENOS_DTYPE_F32;
        which[n++] = i;
    }
    for (int i = 0; i < n; ++i) op.outs[which[i]] = (int)g.tensors.size() + i;
    op.out = op.outs[1];
    for (int i = 0; i < 4; ++i) out[i] = op.outs[i];
    int ids[4];
    append_op(g, std::move(op), y, n, ids);
    return XENOS_OK;
}

// Whether a tensor is the result of a layer norm or an 8-bit product (with its activation record).
static bool row_result(const Graph &g, int t) {
    const int p = g.tensors[t].producer;
    if (p < 0) return false;
    const Op &o = g.ops[p];
    if (o.kind == XENOS_OP_RELU || o.kind == XENOS_OP_RELU6) {
        const int q = g.tensors[o.in[0]].producer;
        return q >= 0 && g.ops[q].kind == XENOS_OP_QMATMUL;
    }
    return o.kind == XENOS_OP_LAYERNORM || o.kind == XENOS_OP_QMATMUL;
}
static bool is_row_op(int kind) { return kind == XENOS_OP_LAYERNORM || kind == XENOS_OP_QMATMUL || kind == XENOS_OP_LOGPROB; }

int elem_dtype(const Graph &g, int t) {
    const Tensor &x = g.tensors[t];
    if (x.fixed >= 0) return x.fixed;
    if (x.input_slot >= 0 || x.output_slot >= 0) return x.io_dtype;
    if (g.precision == XENOS_PRECISION_FP32_CUDA_CORE) return XENOS_DTYPE_F32;
    // scores that only LOGPROB operators read stay fp32 (a bf16 score of 20 is off by up to 0.06)
    const int p = g.node_of_tensor[t];
    bool scores = p >= 0 && !x.consumers.empty();
    for (int c : x.consumers) scores = scores && g.ops[c].kind == XENOS_OP_LOGPROB;
    if (scores) {
        const int k = g.nodes[p].kind;
        if (k == NK_QMATMUL || k == NK_NORM || (x.is_vec && (k == NK_FC || k == NK_GAP))) return XENOS_DTYPE_F32;
    }
    return XENOS_DTYPE_BF16;
}

xenos_status_t compile_graph(Graph &g, int max_batch, int precision) {
    if (g.inputs.empty()) return fail(g, XENOS_E_INVALID, "compile: graph has no input");
    if (g.outputs.empty()) return fail(g, XENOS_E_INVALID, "compile: graph has no output");
    if (g.ops.empty()) return fail(g, XENOS_E_INVALID, "compile: graph has no operator");
    g.precision = precision;
    g.max_batch = max_batch;
    for (int t : g.inputs) {
        const Tensor &x = g.tensors[t];
        if (x.io_dtype == XENOS_DTYPE_I32) {
            if (x.io_layout != XENOS_LAYOUT_NHWC) return fail(g, XENOS_E_UNSUPPORTED, "labels are I32 NHWC");
            continue;
        }
        if (precision == XENOS_PRECISION_FP32_CUDA_CORE &&
            (x.io_dtype != XENOS_DTYPE_F32 || x.io_layout != XENOS_LAYOUT_NCHW))
            return fail(g, XENOS_E_UNSUPPORTED, "fp32 graphs take F32 NCHW inputs");
    }
    for (int t : g.outputs) {
        const Tensor &x = g.tensors[t];
        if (x.fixed >= 0) {
            if (x.rows() > 1 && x.io_layout != XENOS_LAYOUT_NHWC) return fail(g, XENOS_E_UNSUPPORTED, "results of a LOGPROB are NHWC");
            continue;
        }
        if (precision == XENOS_PRECISION_FP32_CUDA_CORE) {
            if (x.io_dtype != XENOS_DTYPE_F32 || (!x.is_vec && x.io_layout != XENOS_LAYOUT_NCHW))
                return fail(g, XENOS_E_UNSUPPORTED, "fp32 graphs produce F32 NCHW outputs");
        } else {
            if (x.is_vec && row_result(g, t))
                for (int c : x.consumers)
                    if (!is_row_op(g.ops[c].kind)) return fail(g, XENOS_E_UNSUPPORTED, "an F32 result is read by an operator that takes bf16");
            if (x.is_vec && x.io_dtype != XENOS_DTYPE_F32)
                return fail(g, XENOS_E_UNSUPPORTED, "bf16 graphs produce vector outputs in F32");
            if (!x.is_vec && x.io_dtype == XENOS_DTYPE_F32 && x.io_layout == XENOS_LAYOUT_NHWC && row_result(g, t)) {
                for (int c : x.consumers)
                    if (!is_row_op(g.ops[c].kind)) return fail(g, XENOS_E_UNSUPPORTED, "an F32 result is read by an operator that takes bf16");
                continue;
            }
            if (!x.is_vec && (x.io_dtype != XENOS_DTYPE_BF16 || x.io_layout != XENOS_LAYOUT_NHWC))
                return fail(g, XENOS_E_UNSUPPORTED, "bf16 graphs produce feature-map outputs as BF16 NHWC");
        }
    }
    xenos_status_t st;
    if ((st = prefuse(g)) != XENOS_OK) return st;
    if ((st = link_pass(g)) != XENOS_OK) return st;
    if ((st = split_and_lower(g)) != XENOS_OK) return st;
    if ((st = plan_workspace(g)) != XENOS_OK) return st;
    emit_plan_json(g);
    return XENOS_OK;
}

}  // namespace xenos
