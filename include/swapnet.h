/*
 * swapnet.h — C ABI of libswapnet: block-swapped DNN inference under a
 * device-memory budget on one GPU (SwapNet, arXiv 2401.16757).
 *
 * The problem the calls solve is the paper's (Sec. 3 "Basic Idea", Sec.
 * 6.2.2 "Partition Blocks within DNN"): given a memory budget b for a model
 * of size s > b, cut the layer sequence into n blocks and execute them in
 * order, swapping each block's parameters into device memory before it runs
 * and releasing them after.  Sec. 6.2.2 ("Allocate Memory Budget across
 * DNNs", Eq. 1) shares one budget among several models.
 *
 * Conventions for every call:
 *   - Status: int, SWAPNET_OK (0) on success, a negative swapnet_status
 *     otherwise.  No C++ exception crosses this boundary (a failed host
 *     allocation is SWAPNET_ERR_OOM, any other one SWAPNET_ERR_INTERNAL).  Output handles
 *     and output arrays are written only on success.  swapnet_last_error()
 *     returns a message for the calling thread's most recent failure.
 *   - Ownership: plans and engines are opaque, library-owned and freed with
 *     swapnet_plan_free / swapnet_engine_free.  Host weight buffers, model
 *     descriptors, and caller-provided device buffers stay caller-owned.
 *   - Layout: activations are NHWC in the model's storage dtype; conv
 *     weights are [cout][kh][kw][cin]; linear weights are [out][in]; a
 *     linear layer flattens its input per batch item in (h, w, c) order.
 *   - Threads: a plan is immutable after creation and may be shared; an
 *     engine is used by one host thread at a time.
 */
#ifndef SWAPNET_H
#define SWAPNET_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ status */
typedef enum swapnet_status {
  SWAPNET_OK = 0,
  SWAPNET_ERR_INVALID_ARG = -1, /* malformed descriptor, option or argument */
  SWAPNET_ERR_INFEASIBLE = -2,  /* no partition fits the budget            */
  SWAPNET_ERR_OOM = -3,         /* host or device allocation failed        */
  SWAPNET_ERR_CUDA = -4,        /* a CUDA runtime/driver call failed       */
  SWAPNET_ERR_TIMEOUT = -5,     /* a bounded device-side wait gave up      */
  SWAPNET_ERR_MISALIGNED = -6,  /* a pointer or size breaks an alignment rule */
  SWAPNET_ERR_UNSUPPORTED = -7, /* shape/dtype combination not implemented */
  SWAPNET_ERR_IO = -8,          /* a weights-file read or write failed      */
  SWAPNET_ERR_INTERNAL = -9     /* an unexpected host-side exception, caught
                                   before it could cross the C ABI          */
} swapnet_status;

/* ------------------------------------------------------------ descriptors */
typedef enum swapnet_dtype {
  SWAPNET_F32 = 0,
  SWAPNET_F16 = 1,
  SWAPNET_BF16 = 2,
  SWAPNET_I32 = 3, /* model input only: token ids */
  SWAPNET_I8 = 4,  /* codes of a quantised key-value cache only: -127 .. 127    */
  SWAPNET_E4M3 = 5 /* the same, 8-bit floats (1-4-3, largest 448, no infinity)  */
} swapnet_dtype;

typedef enum swapnet_op {
  SWAPNET_OP_LINEAR = 1,     /* y[m,o] = act(sum_i x[m,i] W[o,i] + b[o] (+res)) */
  SWAPNET_OP_CONV2D = 2,     /* zero-padded 2-D convolution, + bias (+res), act  */
  SWAPNET_OP_MAXPOOL = 3,    /* window max; padding never wins                  */
  SWAPNET_OP_GAP = 4,        /* global average over H and W                     */
  SWAPNET_OP_UPSAMPLE2X = 5, /* nearest neighbour, factor 2 in H and W          */
  SWAPNET_OP_CONCAT = 6,     /* channels of src0 followed by channels of src1   */
  SWAPNET_OP_EMBED = 7,      /* rows of a [cin = vocab][cout = d] table picked by the
                                int32 token ids of the model input; the table
                                stays in host memory and its rows are read there
                                (never swapped)                                  */
  SWAPNET_OP_RMSNORM = 8,    /* x / sqrt(mean(x^2) + eps) * g over cout = d      */
  SWAPNET_OP_ATTENTION = 9,  /* RoPE on q = src0 and k = src1, both stored rounded;
                                k and v = src2 appended to this layer's cache at
                                the state position; query t attends causally to
                                positions 0..pos+t: softmax(q k^T / sqrt(Dh)) v  */
  SWAPNET_OP_ARGMAX = 10     /* int32 index of each row's maximum (ties: lowest) */
} swapnet_op;

typedef enum swapnet_act {
  SWAPNET_ACT_NONE = 0,
  SWAPNET_ACT_RELU = 1,
  SWAPNET_ACT_LEAKY = 2,  /* slope 0.1 */
  SWAPNET_ACT_SWIGLU = 3  /* silu(res) * (acc + b), res = the gate layer */
} swapnet_act;

#define SWAPNET_LAYER_NO_BIAS 1 /* flags: a linear layer without bias tensor */
/* Flags of ATTENTION layers, the same on every one of a model, whose attention
 * layers then have one shape (head width 128).  The paper has no counterpart.
 * TREE: the input tokens are the nodes of a drafted tree (at most 128), each
 * attending to the cache and its ancestors; their keys and values stay beside
 * the caches until swapnet_engine_tree_accept.
 * WEIGHTS: the attention that each cached row gets is added up in the state,
 * for swapnet_engine_evict. */
#define SWAPNET_ATTENTION_TREE 2
#define SWAPNET_ATTENTION_WEIGHTS 4

#define SWAPNET_SRC_INPUT (-1) /* the model input                       */
#define SWAPNET_SRC_NONE (-2)  /* unused producer / no residual operand */

/* One layer of the model information table (Sec. 6.1, Table 2: per layer
 * size, parameter depth and FLOPs — derived here from the shapes).  Layers
 * are listed in execution order; producers precede consumers. */
typedef struct swapnet_layer {
  int32_t op;       /* swapnet_op                                             */
  int32_t src0;     /* producer of the input (layer index or SWAPNET_SRC_INPUT) */
  int32_t src1;     /* second input of CONCAT, else SWAPNET_SRC_NONE           */
  int32_t res;      /* residual operand (layer index) or SWAPNET_SRC_NONE      */
  int32_t act;      /* swapnet_act                                             */
  int32_t res_post; /* 0: act(acc + b + res); 1: act(acc + b) + res            */
  int32_t cin;      /* conv: input channels;  linear: input features            */
  int32_t cout;     /* conv: output channels; linear: output features           */
  int32_t kh, kw, stride, pad; /* conv and maxpool window                      */
  int32_t is_output;/* nonzero: a model output, written to the output buffer   */
  int32_t flags;    /* SWAPNET_LAYER_NO_BIAS, SWAPNET_ATTENTION_*              */
  int64_t t_ex_ns;  /* measured execution delay; 0 = gamma * FLOPs (Sec. 6.1)  */
  int32_t src2;     /* ATTENTION: the values layer                             */
  int32_t heads;    /* ATTENTION: heads (head width = cout / heads)            */
  int32_t max_seq;  /* ATTENTION: positions the KV cache holds                 */
  float eps;        /* RMSNORM epsilon                                         */
  float theta;      /* ATTENTION: RoPE base (angle = pos * theta^(-2i/Dh))     */
  int32_t reserved;
} swapnet_layer;

/* Parameter tensors of a layer, in this order, are what swapnet_load's
 * host_weights lists: CONV2D and LINEAR have two (weights, bias; one with
 * SWAPNET_LAYER_NO_BIAS), EMBED one (the table), RMSNORM one (the gains);
 * the other ops none.  Model outputs are written to the output buffer in
 * increasing layer order, each at a 256-byte aligned offset (ARGMAX outputs
 * are int32, everything else the model dtype).  ATTENTION uses cout = the
 * width of q, k and v (heads x head width, head width 128). */
typedef struct swapnet_model_desc {
  int32_t dtype;    /* swapnet_dtype of weights and activations          */
  int32_t n_layers;
  const swapnet_layer* layers;
  int32_t in_n, in_h, in_w, in_c; /* model input, NHWC (a matrix is n x 1 x 1 x c) */
  int32_t in_dtype; /* dtype of the model input: the model dtype or SWAPNET_I32 (token ids) */
  int32_t reserved;
} swapnet_model_desc;

typedef enum swapnet_swap_variant {
  SWAPNET_SWAP_AUTO = 0,     /* pick per block by measured time at load        */
  SWAPNET_SWAP_MEMCPY = 1,   /* copy engine: cudaMemcpyAsync from pinned memory */
  SWAPNET_SWAP_ZEROCOPY = 2, /* SM kernel reading mapped host memory           */
  SWAPNET_SWAP_DIRECT = 3,   /* no swap-in: the block's kernels read their
                                parameters in mapped host memory themselves
                                (copy-free dispatch, Sec. 4.2.2, taken to the
                                kernels); for blocks whose units all run SIMT
                                kernels (GEMV, norms, attention, pools), other
                                blocks take ZEROCOPY (MEMCPY when a tensor is
                                not 16-byte aligned), so copy-engine and SM
                                reads of the host weights are not mixed.
                                Never chosen by AUTO.                         */
  SWAPNET_SWAP_PACKED = 4    /* an extension the paper has no counterpart
                                for: bf16 models only.  At load each swapped
                                bf16 tensor whose size is a multiple of 8192
                                bytes is packed losslessly (swapnet_pack_bf16)
                                into engine-held page-locked memory, and an SM
                                kernel reads the packed form over the host
                                link and unpacks it into the arena, so fewer
                                bytes cross the link for the same arena
                                contents.  Pieces that do not pack, and blocks
                                with none that do, take ZEROCOPY.  Packed
                                images are shared by the engines over the same
                                host tensors; the host weights must not change
                                while one of those engines exists.  Not for
                                pageable weights or weights files (a file
                                engine ignores it).  Never chosen by AUTO.     */
} swapnet_swap_variant;

/* Options.  Delay coefficients follow Sec. 6.1: t_in = alpha*s + beta*d,
 * t_ex = gamma*f, t_out = eta*d, in integer units (attoseconds per byte or
 * FLOP; nanoseconds per tensor). */
typedef struct swapnet_options {
  int32_t slots;                 /* arena slots: 2 (swap overlaps compute) or 1 */
  int32_t activations_in_budget; /* 1: the budget also covers the activation workspace */
  int32_t swap_variant;          /* swapnet_swap_variant                         */
  int32_t objective;             /* 0: m-slot pipeline completion; 1: Eq. 4 sum  */
  uint64_t alpha_as_per_byte;
  uint64_t beta_ns_per_tensor;
  uint64_t gamma_as_per_flop;
  uint64_t eta_ns_per_tensor;
  int32_t zc_ctas;               /* CTAs of the zero-copy swap kernel (and of the
                                    unpack kernel of SWAPNET_SWAP_PACKED), 0 =
                                    default (32; one per SM for unpacking)     */
  int32_t graphs;                /* 1 (default): each (input, output) binding of an
                                    engine is captured once as a CUDA graph and
                                    replayed; 0: launch eagerly every call      */
  int32_t preloaded;             /* resident plans only: the caller's arena already
                                    holds this layout (loaded by another engine of
                                    the same layers); swapnet_load skips the upload */
  int32_t branches;              /* 1 (default): a conv / linear layer whose inputs
                                     were all produced before the previous layer runs
                                     on a second stream beside the layers in between
                                     (e.g. a ResNet projection shortcut), when it, its
                                     last producer and its consumers share a block;
                                     0: every layer in order on one stream.  Results
                                     are identical either way. */
  int32_t resident_prefix;       /* 0 (default, the paper's method): every block is
                                     swapped in for every inference.  1 (an extension
                                     the paper has no counterpart for): the planner may
                                     keep the first units' weights in the arena across
                                     inferences (uploaded once at load, never swapped)
                                     and swap the rest through the remaining region;
                                     the prefix length is chosen by the objective among
                                     0, the longest prefix that leaves room for the
                                     rest, and the longest within 1/4, 1/2, 3/4 of its
                                     bytes.  Objective 0 only. */
  int32_t split_cap;             /* 0 (default): the kernels choose how many ways to
                                     split K for layers with fewer output tiles than
                                     SMs, at most 8; n > 0: at most n (1 = never
                                     split; above 8 as 8).  A
                                     tuning knob; results differ in the last bits
                                     between split counts (each count is
                                     deterministic). */
  int32_t prefetch;              /* 0 (default): every inference is self-contained and
                                     starts by swapping in its first block.  1: steady-
                                     state back-to-back inferences (Sec. 4.3 pipeline
                                     carried across inferences): each inference ends by
                                     swapping the next inference's first block into its
                                     place, overlapped with its own last layers, and the
                                     next one starts with it present (the engine swaps it
                                     in once at load).  The planner minimises that cyclic
                                     schedule: first block ready at t = 0; its next copy
                                     starts once the copy engine is free and the last
                                     block sharing its place (the last even-indexed
                                     block) has executed; with an even number of blocks
                                     the last block and the first must fit the region
                                     together.  Objective 0, two slots, no resident
                                     prefix.  Consecutive inferences of one engine must
                                     be issued on one stream (as for any engine). */
  int32_t merge;                 /* 1 (default): consecutive whole linear layers of one
                                     block that read the same input run as one launch:
                                     up to three (e.g. q, k, v), or a SwiGLU gate and
                                     its up projection, of up to 4 rows (fp32: 16);
                                     with more rows on the tensor cores up to three of
                                     equal width and activation without a residual
                                     whose K is not split.  Layers whose buffers
                                     overlap stay apart.  0: one launch per layer.
                                     Results are identical either way;
                                     profiling gives every layer of a merged launch
                                     that launch's start and end. */
  int32_t pageable;              /* 0 (default): the host weights are page-locked
                                     (registered at load unless CUDA already pinned
                                     them).  1 (the paper's w/o-uni-add ablation): they
                                     stay in pageable memory and every swap-in is a
                                     copy-engine copy the driver stages through its own
                                     page-locked buffer; launches are eager (no graphs),
                                     the swap variant is MEMCPY (AUTO resolves to it;
                                     ZEROCOPY and DIRECT are refused), and models whose
                                     layers read a table in host memory (EMBED) are
                                     refused (UNSUPPORTED) at load.  Ignored by engines
                                     loaded from a weights file. */
  int32_t reserved[1];
} swapnet_options;

/* Fills the defaults: 2 slots, activations outside the budget, AUTO swap,
 * pipeline objective, alpha = 2.5e6 as/B (400 GB/s), beta = 2000 ns,
 * gamma = 2000 as/FLOP (500 TFLOP/s), eta = 0, CUDA graphs on. */
void swapnet_default_options(swapnet_options* opt);

/* ------------------------------------------------------------------ plans */
typedef struct swapnet_plan swapnet_plan;

typedef struct swapnet_plan_info {
  uint32_t n_blocks;
  uint32_t n_units;        /* layers, with oversize linear layers split      */
  uint32_t slots;          /* 0 for a resident (all weights in HBM) plan     */
  uint32_t n_layers;
  uint64_t budget_bytes;
  uint64_t arena_bytes;    /* device bytes for weights                       */
  uint64_t slot_bytes;     /* largest piece of a split linear layer          */
  uint64_t workspace_bytes;/* intermediate activations (liveness-planned)    */
  uint64_t input_bytes;    /* model input                                    */
  uint64_t output_bytes;   /* all model outputs, 256-byte aligned each       */
  uint64_t weight_bytes;   /* sum of 256-aligned parameter tensor sizes      */
  uint64_t plan_bytes;     /* host bytes of the plan (the resident skeleton) */
  int64_t predicted_ns;    /* objective value of the chosen partition        */
  uint64_t state_bytes;    /* decoder state (position + KV caches), 0 if none */
  int32_t exact;           /* 1: the search proved the plan optimal; 0: its
                              frontier was capped and the plan is the best found */
  int32_t reserved;
  uint32_t prefix_units;   /* resident_prefix: units kept in the arena (block 0) */
  uint32_t reserved2;
  uint64_t prefix_bytes;   /* their bytes at the bottom of the arena; the swap
                              region follows them                             */
} swapnet_plan_info;

typedef struct swapnet_unit_info {
  int32_t layer;   /* layer index                                            */
  int32_t row0;    /* first output feature (linear pieces), else 0           */
  int32_t rows;    /* output features in this unit (linear), else 0          */
  int32_t depth;   /* parameter tensors                                      */
  uint64_t bytes;  /* 256-aligned parameter bytes                            */
  uint64_t flops;
  int64_t t_ex_ns;
} swapnet_unit_info;

typedef struct swapnet_block_info {
  uint32_t unit0, unit1; /* units [unit0, unit1)                             */
  uint32_t slot;         /* block parity: which co-resident position it takes;
                            UINT32_MAX for a resident prefix block           */
  uint32_t depth;
  uint64_t bytes;
  int64_t t_in_ns, t_ex_ns, t_out_ns;
  uint64_t offset;       /* byte offset of the block in the arena            */
} swapnet_block_info;

/* Partition the model for a budget (Sec. 6.2.2, Eq. 2-3; objective per
 * opt->objective).  The arena is the budget (minus the workspace when
 * activations_in_budget), rounded down to 256 bytes.  With two co-resident
 * blocks every pair of consecutive blocks must fit the arena together
 * (Eq. 3: s_i + s_{i+1} <= b): even blocks are placed at the bottom of the
 * arena and odd blocks against its top.  With one slot each block must fit
 * the arena alone.  A linear layer larger than slot_bytes (half the arena
 * with two blocks) is split along output features into pieces of a
 * multiple of 128 features.  Ties: fewer blocks, then the
 * lexicographically smallest cut vector.  Host only; no device work.
 * Errors: INVALID_ARG (descriptor/options), INFEASIBLE (no partition). */
int swapnet_partition(const swapnet_model_desc* desc, uint64_t budget_bytes,
                      const swapnet_options* opt /* nullable: defaults */,
                      swapnet_plan** out_plan);

/* Build a plan from explicit cut points (Sec. 6.2.2 "create_blocks"): cut c
 * places a block boundary before unit c; cuts strictly increasing in
 * [1, n_units).  Units are computed for the budget as in swapnet_partition.
 * Errors: INVALID_ARG (bad cuts), INFEASIBLE (a block exceeds a slot). */
int swapnet_plan_from_cuts(const swapnet_model_desc* desc, const uint32_t* cuts, uint32_t n_cuts,
                           uint64_t budget_bytes, const swapnet_options* opt,
                           swapnet_plan** out_plan);

/* The sufficient-memory reference (DInf): one block holding every weight,
 * loaded once and kept resident; the same kernels run the same units. */
int swapnet_plan_resident(const swapnet_model_desc* desc, const swapnet_options* opt,
                          swapnet_plan** out_plan);

int swapnet_plan_info_get(const swapnet_plan* plan, swapnet_plan_info* info);
/* Copy up to `cap` entries; return the number available in *n (nullable). */
int swapnet_plan_cuts(const swapnet_plan* plan, uint32_t* cuts, uint32_t cap, uint32_t* n);
int swapnet_plan_units(const swapnet_plan* plan, swapnet_unit_info* units, uint32_t cap, uint32_t* n);
int swapnet_plan_blocks(const swapnet_plan* plan, swapnet_block_info* blocks, uint32_t cap, uint32_t* n);
/* Byte offset of each model output inside the output buffer (in layer order). */
int swapnet_plan_output_offsets(const swapnet_plan* plan, uint64_t* offs, uint32_t cap, uint32_t* n);
void swapnet_plan_free(swapnet_plan* plan);

/* Multi-DNN budget split (Sec. 6.2.2, Eq. 1): with demands M_i (weight
 * bytes) and performance scores PS_i = u_i * latency_i / M_i (latency_i =
 * predicted all-resident latency), model i receives
 *   A_i = M_i/sum(M) (1 - 1/n) M + PS_i/sum(PS) (1/n) M,
 * floored to 256 bytes, when sum(M) > M (else A_i = M_i); each model is
 * then partitioned for A_i.  budgets_out[n] and plans_out[n] are written on
 * success only; the caller frees each plan. */
int swapnet_schedule(const swapnet_model_desc* const* models, const float* urgency, uint32_t n,
                     uint64_t arena_bytes, const swapnet_options* opt,
                     uint64_t* budgets_out, swapnet_plan** plans_out);

/* ---------------------------------------------------------------- engines */
typedef struct swapnet_engine swapnet_engine;
typedef struct CUstream_st* swapnet_stream; /* a cudaStream_t; NULL = legacy default stream */

/* Bind a plan to host weights and device memory (Sec. 4.2 zero-copy
 * swap-in, Sec. 5.2 assembly by reference).
 *   host_weights: n_tensors pointers, one per parameter tensor in layer
 *     order; caller-owned, must outlive the engine and must not change.
 *     They are page-locked and mapped in place (cudaHostRegister), never
 *     copied on the host; memory already pinned by CUDA is used as is.
 *   d_arena: device buffer of >= arena_bytes for the weight slots, 256-byte
 *     aligned; NULL = the library allocates it.  d_workspace likewise for
 *     the activation workspace.
 * The plan is copied; it may be freed after this call.  Creates a copy
 * stream and per-slot events; resolves every layer's parameter address to
 * slot base + offset and builds its TMA descriptors once (the skeleton).
 * With SWAPNET_SWAP_AUTO it times both swap variants per block, then whole
 * inferences with that per-block choice, with every block on the copy
 * engine and with every block on the zero-copy kernel, and keeps the
 * fastest; decoder models (attention layers, a bound state) take the
 * zero-copy kernel for every block, so that the engines of one model never
 * mix copy-engine and SM reads of their shared host weights.  With
 * SWAPNET_SWAP_PACKED it packs every swapped bf16 tensor that packs (or
 * takes the packed image another engine made of the same host tensor) and
 * keeps a device table of the unpack jobs of each block.  A resident plan
 * copies all weights to the arena here.
 * Errors: INVALID_ARG, MISALIGNED, OOM, CUDA, UNSUPPORTED, INTERNAL. */
int swapnet_load(const swapnet_plan* plan, const void* const* host_weights, uint32_t n_tensors,
                 void* d_arena, uint64_t arena_bytes, void* d_workspace, uint64_t workspace_bytes,
                 swapnet_engine** out_engine);

/* ----------------------------------------------------------- storage tier
 * Sec. 4.2.1 "Direct Block Fetch": the blocks live in external storage and
 * are fetched with direct I/O (O_DIRECT, bypassing the page cache, so no
 * second copy of a block sits in host memory) into a dedicated swap-in
 * channel.  Here the channel is two page-locked staging buffers per engine:
 * block k is read from the file into staging buffer k mod 2 by a host
 * function on the engine's read stream, then copied by the copy engine into
 * its arena slot, so the read of block k+1 overlaps the copy of block k and
 * the execution of block k-1.
 *
 * Weights file layout (little-endian), written by swapnet_weights_file_write:
 *   bytes 0..7     magic "SWNWGT01"
 *   uint32         version = 1
 *   uint32         n_tensors
 *   uint64         data_offset (first tensor; a multiple of 4096)
 *   n_tensors x {uint64 offset, uint64 bytes}: tensor t in layer order, as
 *                  in swapnet_load's host_weights; offset a multiple of 4096
 *   zero padding; the file length is a multiple of 4096.
 */
typedef struct swapnet_weights_file swapnet_weights_file;

enum { SWAPNET_FILE_ALLOW_BUFFERED = 1 }; /* open flag: no O_DIRECT -> page cache */

/* Write every parameter tensor of `desc` (n_tensors host pointers in layer
 * order, tensor sizes from the descriptor) to `path` in the layout above,
 * then fsync.  Errors: INVALID_ARG, IO (errno text in swapnet_last_error). */
int swapnet_weights_file_write(const char* path, const swapnet_model_desc* desc, const void* const* host_weights,
                               uint32_t n_tensors);

/* Open and validate a weights file for reading with O_DIRECT.  Where the
 * file system refuses O_DIRECT, fails with IO unless flags has
 * SWAPNET_FILE_ALLOW_BUFFERED (then reads go through the page cache and
 * swapnet_weights_file_info reports direct = 0).  Errors: INVALID_ARG (bad
 * header), IO, OOM. */
int swapnet_weights_file_open(const char* path, uint32_t flags, swapnet_weights_file** out);
int swapnet_weights_file_info(const swapnet_weights_file* f, uint32_t* n_tensors, int32_t* direct);
/* Host read of bytes [offset, offset + bytes) of tensor t into dst through
 * the file's read path (an aligned bounce buffer).  Errors: INVALID_ARG
 * (range outside the tensor), IO. */
int swapnet_weights_file_read(swapnet_weights_file* f, uint32_t tensor, uint64_t offset, uint64_t bytes, void* dst);
/* The file must outlive every engine loaded from it. */
void swapnet_weights_file_close(swapnet_weights_file* f);

/* As swapnet_load, with the parameters in a weights file instead of host
 * memory: swapped blocks are fetched from the file for every inference
 * (staging, read stream and host functions as above); a resident plan or a
 * resident prefix is read once here.  Swap variant: copy engine (AUTO and
 * ZEROCOPY are taken as MEMCPY).  Models with host-resident parameters
 * (EMBED) are not supported.  A failed read inside an inference is reported
 * by the next swapnet_engine_sync as IO.  Errors: as swapnet_load, plus IO,
 * UNSUPPORTED. */
int swapnet_load_file(const swapnet_plan* plan, swapnet_weights_file* file, void* d_arena, uint64_t arena_bytes,
                      void* d_workspace, uint64_t workspace_bytes, swapnet_engine** out_engine);

/* One inference, asynchronous on `stream` (Sec. 4.3, Sec. 6.2.2 with m
 * slots): block k is swapped into slot k mod m on the engine's copy stream
 * once the slot's previous block has finished executing, and its layers run
 * on `stream` once the swap is done; block k+1's swap overlaps block k's
 * execution.  d_input / d_output are device pointers of input_bytes and
 * output_bytes (plan info), 16-byte aligned.  Device faults surface at the
 * next synchronising call; bounded device waits report through
 * swapnet_engine_sync.  Errors: INVALID_ARG, MISALIGNED, CUDA. */
int swapnet_infer(swapnet_engine* eng, const void* d_input, void* d_output, swapnet_stream stream);

/* As swapnet_infer, from and to host buffers: the input is copied to an
 * engine-owned device buffer and the outputs back, all on `stream` (copies
 * are asynchronous when the host buffers are pinned).  The host output is
 * valid after the stream has been synchronised. */
int swapnet_infer_host(swapnet_engine* eng, const void* h_input, void* h_output, swapnet_stream stream);

/* Waits for the engine's streams; returns TIMEOUT if a kernel's bounded
 * wait gave up since the last call (the error word is then cleared), CUDA
 * on a device error, IO if a weights-file read failed (then cleared). */
int swapnet_engine_sync(swapnet_engine* eng);

/* Runtime budget adaptation (Sec. 6.2.2 "adaptively partition and exchange
 * blocks"; the dynamic-budget case study of Sec. 8): switch a loaded engine,
 * between inferences, to another plan of the same model, e.g. one of several
 * plans made ahead with swapnet_partition for different budgets (the
 * paper's look-up table of partitions).  Waits for the engine's work in
 * flight; keeps the host registration, streams, workspace and bound decoder
 * state; re-derives blocks, copy segments, unit pointers and descriptors
 * (the paper's "repeat steps 2 and 3"); re-allocates an engine-owned arena
 * at the new plan's size, releasing the old one first, so a smaller budget
 * gives memory back.  A caller-provided arena stays and must hold the new
 * plan.  The plan is copied; the caller may free it after the call.
 * Errors: INVALID_ARG (a plan for another model, resident <-> swapped, or
 * a different `pageable` option), OOM, CUDA. */
int swapnet_engine_adapt(swapnet_engine* eng, const swapnet_plan* plan);

/* Decoder state of a model with ATTENTION layers: a device buffer of
 * state_bytes (plan info), caller-owned, 256-byte aligned.  Layout: an int32
 * position (tokens already cached) in the first 256 bytes, then for every
 * ATTENTION layer in layer order its key cache and value cache
 * [max_seq][cout] in the model dtype, each 256-byte aligned.  Zero the
 * buffer to start a new sequence.  Each inference reads the position on the
 * device, appends its tokens at that position and advances it by the number
 * of input tokens, so a prefill engine and a decode engine built from the
 * same layers can share one state buffer, and a decode step replays the same
 * CUDA graph every time.  A position that would pass max_seq is not written;
 * swapnet_engine_sync then reports SWAPNET_ERR_INVALID_ARG.
 * Must be bound before the first swapnet_infer of such a model. */
int swapnet_engine_bind_state(swapnet_engine* eng, void* d_state, uint64_t state_bytes);

/* What else a state holds: byte offsets from its start, 0 = not there.  The
 * header's int32 words: [0] the rows in use (the position above), [1] with
 * WEIGHTS the rows evicted so far (a token's rotation is that of position
 * [0] + [1]), [2] scratch, [3] and [4] with TREE results of the last
 * swapnet_engine_tree_accept: accepted nodes and the model's choice at the
 * last one.  Each run of an ATTENTION unit adds to the weights, also those of
 * swapnet_engine_measure_units and _calibrate: measure before the state is
 * used, or zero the weights behind it.  With TREE write a tree first: an empty
 * one is out of range.
 * Engines that share a state are built from the same layers with the same
 * SWAPNET_ATTENTION_WEIGHTS flag; the offsets up to `weights` are the same for
 * them, what lies behind serves one engine's pass at a time. */
typedef struct swapnet_state_layout {
  uint64_t caches;       /* key cache of the first ATTENTION layer              */
  uint64_t cache_bytes;  /* of one cache: key and value caches follow one another,
                            layer by layer (0: the layers differ)               */
  uint64_t weights;      /* WEIGHTS: float [layers][heads][max_seq]             */
  uint64_t tree_count;   /* TREE: int32 nodes in use                            */
  uint64_t tree_parents; /* TREE: int32 [tokens], as in swapnet_cached_attention */
  uint64_t tree_path;    /* TREE: int32 [tokens] the accepted nodes, -1 behind  */
  uint32_t layers;       /* ATTENTION layers                                    */
  uint32_t reserved;
} swapnet_state_layout;
int swapnet_plan_state_layout(const swapnet_plan* plan, swapnet_state_layout* layout);

/* Greedy decoding with drafted trees (TREE models).  Before each inference the
 * caller writes the tree (tree_count, tree_parents) into the state, on the same
 * stream; node 0 is the token the last pass chose and the input holds the
 * nodes' ids, any valid ones behind tree_count; what the outputs hold for those
 * is undefined.  The inference does not advance the position.  This call walks
 * the tree as swapnet_tree_accept does, with d_targets the inference's ARGMAX
 * output, appends the accepted nodes' rows to every layer's caches, with
 * WEIGHTS adds their attention to the weights, advances the position by their
 * number and leaves path, accepted and next in the state.  No room for the
 * path: nothing is accepted (accepted = 0), reported by swapnet_engine_sync.
 * Asynchronous on `stream`; no other engine may run on the state in between.
 * Errors: INVALID_ARG (no TREE model, no state), MISALIGNED, CUDA. */
int swapnet_engine_tree_accept(swapnet_engine* eng, const int32_t* d_ids, const int32_t* d_targets, swapnet_stream stream);

/* Eviction in the bound state of a WEIGHTS model: in every layer and head the
 * cache keeps min(position, keep) rows as swapnet_cache_evict does, the
 * position becomes that number, and the evicted rows are counted in the header
 * so that later tokens keep their rotation.  Asynchronous on `stream`.
 * Errors: INVALID_ARG (no WEIGHTS model, no state, bad numbers), CUDA. */
int swapnet_engine_evict(swapnet_engine* eng, int32_t keep, int32_t recent, int32_t sink, swapnet_stream stream);

typedef struct swapnet_engine_block {
  int32_t variant;       /* swapnet_swap_variant chosen for the block     */
  int32_t n_segments;    /* contiguous host->arena copies per swap-in     */
  float memcpy_us;       /* measured at load (AUTO), else 0               */
  float zerocopy_us;
} swapnet_engine_block;

int swapnet_engine_blocks(const swapnet_engine* eng, swapnet_engine_block* blocks, uint32_t cap,
                          uint32_t* n);
/* Counters of the inferences since load: kernel launches include the layer
 * kernels and the swap kernels (zero-copy, unpack); memcpy_calls counts copy-engine
 * transfers and bytes_swapped the bytes moved into the arena (uploads at
 * load time excluded; a block read in place, SWAPNET_SWAP_DIRECT, adds
 * nothing). */
typedef struct swapnet_engine_stats {
  uint64_t infer_calls;
  uint64_t kernel_launches;
  uint64_t memcpy_calls;
  uint64_t bytes_swapped;
  uint64_t link_bytes;   /* bytes the swaps read over the host link: the
                            packed form for SWAPNET_SWAP_PACKED blocks, the
                            bytes swapped for the others */
} swapnet_engine_stats;
int swapnet_engine_stats_get(const swapnet_engine* eng, swapnet_engine_stats* stats);

/* Kernel family that runs each unit. */
typedef enum swapnet_kernel_kind {
  SWAPNET_KERNEL_TC_GEMM = 1,     /* tcgen05 GEMM, A and B by TMA             */
  SWAPNET_KERNEL_TC_CONV = 2,     /* tcgen05 implicit-GEMM conv (A gathered)  */
  SWAPNET_KERNEL_SKINNY = 3,      /* SIMT GEMV family: fp32 <= 16 rows, fp16/bf16 <= 4 rows */
  SWAPNET_KERNEL_DIRECT_CONV = 4, /* SIMT direct convolution                  */
  SWAPNET_KERNEL_MAXPOOL = 5,
  SWAPNET_KERNEL_GAP = 6,
  SWAPNET_KERNEL_UPSAMPLE = 7,
  SWAPNET_KERNEL_CONCAT = 8,
  SWAPNET_KERNEL_TILED = 9,       /* SIMT tiled linear (general fallback)     */
  SWAPNET_KERNEL_EMBED = 10,      /* zero-copy embedding gather               */
  SWAPNET_KERNEL_RMSNORM = 11,
  SWAPNET_KERNEL_ATTENTION = 12,  /* two launches: RoPE + cache append, attention */
  SWAPNET_KERNEL_ARGMAX = 13,
  SWAPNET_KERNEL_TC_CONV_SMALL = 14 /* tcgen05 conv for C % 8 != 0 (RGB stems)  */
} swapnet_kernel_kind;
int swapnet_engine_unit_kernels(const swapnet_engine* eng, int32_t* kinds, uint32_t cap, uint32_t* n);

/* How each tensor-core unit is tiled (introspection for measurement; the
 * paper has no counterpart).  For unit i, tiling[i] gets: n_tile (N columns
 * per output tile), splits (K splits; 1 = none), cluster (1: the splits of a
 * tile reduce through a thread-block cluster), persistent (1: one CTA per SM
 * loops over the tiles), tap_tma (1: convolution A loaded by one 4-D TMA per
 * filter tap), pair (1: persistent on pairs of SMs), sub_tiles (128-row parts
 * of a tile), shared (1: one launch with its siblings, whose tiling this is).
 * Units off the tensor cores get all zeros.  Same count protocol as
 * swapnet_engine_unit_kernels. */
typedef struct swapnet_unit_tiling {
  int32_t n_tile, splits, cluster, persistent, tap_tma, pair, sub_tiles, shared;
} swapnet_unit_tiling;
int swapnet_engine_unit_tiling(const swapnet_engine* eng, swapnet_unit_tiling* tiling, uint32_t cap,
                               uint32_t* n);

/* Device timing for measurement: while enabled, every swapnet_infer records
 * a CUDA event pair around each unit's kernel (on the inference stream) and
 * around each block's swap-in (on the copy stream).  The events add a small
 * gap between launches; leave profiling off for latency measurements.
 * swapnet_engine_last_times synchronises and returns, for the most recent
 * profiled inference, microseconds per unit and per block swap-in. */
int swapnet_engine_set_profiling(swapnet_engine* eng, int enable);

/* Offline profiling of the execution delays (Sec. 6.1: the paper fits its
 * coefficients once per device).  Times every unit's kernel on the engine's
 * device as a graph of `reps` back-to-back launches (so consecutive launches
 * overlap as they do inside an inference) and writes microseconds per launch
 * to unit_us[0..n_units).  The values a unit reads are whatever its buffers
 * hold; the kernels' timing does not depend on them.  Synchronous.
 * Errors: INVALID_ARG, OOM (staging buffers), CUDA. */
int swapnet_engine_measure_units(swapnet_engine* eng, int32_t reps, float* unit_us, uint32_t n_units);
int swapnet_engine_last_times(swapnet_engine* eng, float* unit_us, uint32_t n_units, float* swap_us,
                              uint32_t n_blocks);

/* Swap-in time of each block as it runs inside the inference graph that
 * swapnet_infer replays (Sec. 4.2's t^in, measured in place rather than
 * with the eager, event-instrumented launches of profiling).  With swap
 * timing on, the engine captures (and caches) a graph variant that records
 * an event on the copy stream right before and right after each block's
 * swap-in; layer launches are unchanged, so the replay is the inference
 * that swapnet_infer times, plus 2 event-record nodes per swapped block.
 * swapnet_engine_last_swap_times waits for the most recent inference's last
 * swap events and writes microseconds per block to swap_us[0..n_blocks)
 * (0 for blocks that are not swapped: a resident prefix, blocks read in
 * place, every block of a resident plan).
 * Errors: INVALID_ARG (null engine or output, timing never enabled), CUDA. */
int swapnet_engine_set_swap_timing(swapnet_engine* eng, int enable);
int swapnet_engine_last_swap_times(swapnet_engine* eng, float* swap_us, uint32_t n_blocks);

/* The pipeline of Sec. 4.3 as it runs inside the replayed inference graph:
 * with the timeline on, the engine captures (and caches) a graph variant
 * that also records an event on the caller's stream at the start of the
 * inference and right before and after each block's layers, besides the
 * swap-in events above.  swapnet_engine_last_graph_timeline waits for the
 * most recent inference's last block and writes 4 floats per block to
 * t_us[4 * k .. 4 * k + 3], microseconds since the start of that inference:
 * swap-in start, swap-in end (both -1 for blocks that are not swapped in
 * during the inference: a resident prefix, blocks read in place, the first
 * block under first-block prefetch, every block of a resident plan), start
 * and end of the block's layers on the caller's stream.  The extra nodes
 * sit between the last layer of one block and the first of the next, so
 * they can add the cost of a dependent launch at each block boundary; the
 * timeline explains a replay, swapnet_infer without it is the one to time.
 * Errors: INVALID_ARG (null engine or output, timeline never enabled), CUDA. */
int swapnet_engine_set_graph_timeline(swapnet_engine* eng, int enable);
int swapnet_engine_last_graph_timeline(swapnet_engine* eng, float* t_us, uint32_t n_blocks);

/* The offline fit of the delay model on this device (Sec. 6.1: the paper
 * profiles each device once and fits t_ex = gamma * f and t_in = alpha * s +
 * beta * d by linear regression).  Here the execution delays are measured
 * per layer instead of fitted per FLOP:
 *   t_ex_ns[l] (n_layers entries, the model's layer count) = the summed
 *     swapnet_engine_measure_units time of layer l's units (reps launches
 *     each), at least 1 ns; when resident_ns > 0 (the measured latency of
 *     the same model with every weight resident), every t_ex is scaled so
 *     that they add up to it, since units timed alone miss the launch and
 *     cache effects of the whole dependent chain;
 *   alpha_as_per_byte = the copy-engine swap-in times measured at load
 *     (SWAPNET_SWAP_AUTO engines) over those blocks' bytes, in attoseconds
 *     per byte; 0 when the engine measured none.
 * The results are meant for swapnet_layer.t_ex_ns and
 * swapnet_options.alpha_as_per_byte of the next swapnet_partition (with
 * beta_ns_per_tensor 0: the per-block times already contain it).
 * Synchronous.  Errors: INVALID_ARG (n_layers other than the model's), OOM,
 * CUDA. */
int swapnet_engine_calibrate(swapnet_engine* eng, int32_t reps, int64_t resident_ns, int64_t* t_ex_ns,
                             uint32_t n_layers, uint64_t* alpha_as_per_byte);
/* Start and end of every unit kernel and block swap-in of the most recent
 * profiled inference, in microseconds after the first of those events
 * (arrays of n_units and n_blocks entries; swap entries are 0 for a
 * resident plan).  Synchronises. */
int swapnet_engine_last_timeline(swapnet_engine* eng, float* unit_start, float* unit_end, uint32_t n_units,
                                 float* swap_start, float* swap_end, uint32_t n_blocks);

/* Waits for the device to finish the engine's work (inferences may still be
 * queued on the caller's stream), then releases its streams, events,
 * graphs, staging buffers and engine-owned device memory, and unregisters
 * the host ranges it registered.  NULL is ignored. */
void swapnet_engine_free(swapnet_engine* eng);

/* ------------------------------------------------- allocation-free GEMM */
/* Y[m][n] = act(sum_k A[m][k] * W[n][k] + bias[n]) for fp16 or bf16 data,
 * computed by the tcgen05 GEMM kernels the engine uses for linear layers.
 * Where K is split, the splits of an output tile are a thread-block cluster
 * that exchanges its partial sums through distributed shared memory, so the
 * call needs no device memory of its own.  The paper has no counterpart to
 * this call.
 *
 * It is for callers that must not allocate device memory: code running
 * under a hard device-memory budget in which every byte is already
 * assigned (the situation this library is about), or hosts whose own
 * allocator has reserved the whole GPU so that cudaMalloc would fail.
 * The call allocates nothing: no cudaMalloc, no cudaFree, no allocating
 * library routine.
 *
 *   dtype   SWAPNET_F16 or SWAPNET_BF16
 *   A       device, [M][K] row-major; W device, [N][K] row-major;
 *           bias device, [N]; Y device, [M][N] row-major, written
 *   act     swapnet_act applied after the bias
 *   stream  the call is asynchronous on it
 * Pointers must be 16-byte aligned and K a multiple of 8.
 *
 * Limits: a problem is rejected with SWAPNET_ERR_INVALID_ARG before anything
 * is launched if the fp32 partial sums of its K split over the SMs that its
 * output tiles leave idle (128 x 64 tiles, 128 x 128 where those give every
 * SM one; at most 32 ways, two 64-deep k-blocks each), counted as if they
 * were kept in one array with 64 KiB beside them, exceed
 * SWAPNET_NOALLOC_SCRATCH_BYTES.  The kernels need no such array; the limit
 * stands so that what the call refuses does not change.  Calls share nothing:
 * they may overlap on different streams and threads.
 *
 * Ordering: the kernel starts only after the work queued before it on
 * `stream` has completed (no programmatic early start), so A, W and bias may
 * be the output of the previous call or kernel on the stream.
 *
 * Set-up: the first call on a device looks up the error word's device
 * address (cudaGetSymbolAddress) with that device current and caches it; make
 * that first call before any stream capture.
 * Errors: INVALID_ARG, MISALIGNED, UNSUPPORTED, CUDA.  Device-side failures
 * are not returned by this call, which does not wait for its kernel: if a
 * bounded wait inside the kernel gives up (one second), Y is incomplete and
 * the timeout is recorded in the library's device error word, which the
 * next swapnet_engine_sync (of any engine on the device) or
 * swapnet_device_sync reports as SWAPNET_ERR_TIMEOUT and clears. */
#define SWAPNET_NOALLOC_SCRATCH_BYTES (4u << 20)
int swapnet_gemm_noalloc(int32_t dtype, const void* A, const void* W, const void* bias, void* Y, int32_t M,
                         int32_t N, int32_t K, int32_t act, swapnet_stream stream);

/* Waits for the current device's work and reports what kernels recorded there
 * since the last report, as swapnet_engine_sync does, for programs that make
 * the calls above and below without an engine: TIMEOUT (a bounded wait gave up,
 * outputs are incomplete), INVALID_ARG (a value in device memory was out of
 * range), CUDA. */
int swapnet_device_sync(void);

/* ------------------------------------------------- cached attention
 * The attention of a decoder over its key-value cache as calls of their own,
 * for programs that keep many sequences' caches themselves, and the calls
 * that keep such a cache within its rows: every pass over swapped weights
 * costs their whole transfer, so a program verifies a tree of drafted tokens
 * in one pass (swapnet_attention_tree, swapnet_tree_accept) and bounds the
 * cache beside the arena (swapnet_attention_weights, swapnet_cache_evict).
 * The paper has no counterpart to these calls.
 *
 * Like swapnet_gemm_noalloc they allocate nothing, are asynchronous on
 * `stream`, start after the work queued before them on it, and may be
 * captured into a graph (make a first call on a device before any capture).
 * They run on the current device, which has to hold the buffers.  Calls share
 * nothing but what the caller passes: two calls that may run at the same time
 * need workspaces of their own, and so do graphs that may be replayed at the
 * same time.  Sizes are checked on the host; what lies in device memory
 * (lens, counts, parents, rows) is checked there: a sequence with a value out
 * of range is left alone (a row list's entry out of range adds nothing) and
 * swapnet_device_sync reports SWAPNET_ERR_INVALID_ARG.  A device has one record
 * of such errors, which every report clears: the next swapnet_engine_sync
 * reports it as well, so a program that also runs engines calls
 * swapnet_device_sync before an inference whose report it wants by itself.
 *
 * Layout: element type F16 or BF16; a cache row holds the kv_heads heads of
 * one position, head h at element h * head_dim; sequence b's row j is at
 * element b * seq_stride + j * kv_stride of k and v.  Query t of sequence b is
 * row b * tokens + t of q (heads * head_dim elements, stride q_stride).
 * Strides are in elements, 0 = packed; queries, keys, values and outputs are
 * 16-byte aligned, int32 and float arrays 4-byte, strides multiples of 8.  head_dim is 64 or 128; heads is a multiple of
 * kv_heads (query head h reads key head h / (heads / kv_heads)). */
typedef struct swapnet_cached_attention {
  int32_t dtype;      /* SWAPNET_F16 or SWAPNET_BF16                          */
  int32_t n_seq;      /* sequences                                            */
  int32_t tokens;     /* queries per sequence (at most; see counts)           */
  int32_t heads, kv_heads, head_dim;
  int32_t max_seq;    /* rows of a sequence's cache                           */
  float scale;        /* of q . k; 0 = 1 / sqrt(head_dim)                     */
  const void* q;      /* rotated queries                                      */
  const void* k;      /* key cache (rotated keys)                             */
  const void* v;      /* value cache                                          */
  const int32_t* lens;    /* [n_seq] rows of the cache in use                 */
  const int32_t* counts;  /* [n_seq] queries in use, NULL = tokens            */
  const int32_t* parents; /* [n_seq][tokens] a drafted node's parent: an earlier
                             node, or -1 below the cached rows; NULL = a chain */
  const int32_t* rows;    /* swapnet_attention_weights: [n_seq][tokens] the
                             queries that count, NULL = 0, 1, 2, ...          */
  const void* k_new;  /* drafted nodes' keys [n_seq * tokens], stride new_stride; */
  const void* v_new;  /* and values; NULL = no draft                          */
  void* out;          /* [n_seq * tokens][heads * head_dim], stride out_stride */
  float* lse;         /* [n_seq][heads][tokens] natural log of the softmax sum
                         of scaled scores (nullable for attention)            */
  const float* weights_in; /* [n_seq][kv_heads][max_seq], NULL = zeros        */
  float* weights;          /* the same shape, may be weights_in               */
  int64_t q_stride, kv_stride, seq_stride, new_stride, out_stride;
} swapnet_cached_attention;

/* out[t] = sum_j softmax_j(scale q_t . k_j) v_j, rounded once, over
 *   - with a draft (k_new): every cached row (j < lens) and, of the drafted
 *     nodes, the query's own and its ancestors; at most 128 nodes;
 *   - without: the queries are the cache's last `counts` rows, each sees the
 *     rows up to its own (one token: a decode step on a cache that already
 *     holds its row).  A query that sees no row gives 0 and lse = -inf.
 * With `weights` (no draft): weights[j] = weights_in[j] + the attention that
 * row j got from these queries, summed over the query heads that share its
 * key head; more than 16 rows (tokens x heads / kv_heads) need lse.
 * Queries at and behind counts, and weights at and behind lens, are left as
 * they were.  Hidden rows may hold anything.
 * Scores, statistics and sums are fp32.  The probabilities enter their product
 * with the values as parts of the storage type: up to 16 rows 24 bits of them
 * (BF16) or 22 (F16), more rows 17 or 22.  F16 has no step below 2^-24, so a
 * row's part of the largest probability is off by at most 2^-40 up to 16 rows;
 * beyond, by at most 2^-32 in caches of up to 4000 rows and in the first 2048
 * rows that a CTA takes of a longer one, 2^-37 in the rest.
 * `workspace` is 256-byte aligned device memory of at least the bytes that
 * _workspace returns, a function of the sizes and of whether k_new and weights
 * are given, with nothing to keep in it between calls.  How many CTAs share a
 * cache goes by max_seq as well, since lens are on the device: a large cache
 * with few rows in use pays for a join that it does not need.  Outputs and
 * workspace overlap none of the inputs (but for weights and weights_in).
 * Errors: INVALID_ARG, MISALIGNED, UNSUPPORTED, CUDA. */
int swapnet_attention_tree_workspace(const swapnet_cached_attention* args, uint64_t* bytes);
int swapnet_attention_tree(const swapnet_cached_attention* args, void* workspace, uint64_t workspace_bytes,
                           swapnet_stream stream);

/* The weights alone, from lse of an earlier attention call: the i-th query is
 * row rows[b][i] of q and of lse (i < counts[b]) and sits in cache row
 * lens[b] - counts[b] + i; it adds e^(scale q . k_j - lse) to every row j up to
 * its own.  After swapnet_tree_accept: rows = path, counts = accepted,
 * lens = lens_out.  v and out are not used. */
int swapnet_attention_weights(const swapnet_cached_attention* args, swapnet_stream stream);

/* Eviction: per sequence and key head, of lens rows keep min(lens, keep): the
 * first `sink`, the last `recent` and those of the largest weights (NaN
 * counts as the largest; among equal ones the lower row), in row order.  kept
 * gets the rows kept, k_out / v_out / weights_out their contents in rows
 * 0 .. min(lens, keep) - 1, lens_out their number.  weights_out is 0 from there
 * up to row lens (a row appended later starts from nothing); what else lies
 * behind is left as it was.  k_out, v_out and weights_out may be the inputs
 * themselves (in place, one layout for both); otherwise they must not overlap
 * them.  Keys keep the rotation of the position they were written at.
 * head_dim: any multiple of 8 up to 512.
 * Errors: INVALID_ARG, MISALIGNED, UNSUPPORTED, CUDA. */
typedef struct swapnet_cache_eviction {
  int32_t dtype, n_seq, kv_heads, head_dim;
  int32_t max_seq;       /* rows of an input cache, columns of weights          */
  int32_t keep, recent, sink;
  int32_t out_capacity;  /* rows of an output cache, columns of weights_out; 0 = max_seq */
  int32_t reserved;
  const void* k;
  const void* v;
  const float* weights;  /* [n_seq][kv_heads][max_seq]                          */
  const int32_t* lens;   /* [n_seq]                                             */
  void* k_out;
  void* v_out;
  float* weights_out;    /* [n_seq][kv_heads][out_capacity]                     */
  int32_t* kept;         /* [n_seq][kv_heads][keep]                             */
  int32_t* lens_out;     /* [n_seq], not lens itself                            */
  int64_t kv_stride, seq_stride, out_stride, out_seq_stride;
} swapnet_cache_eviction;
int swapnet_cache_evict(const swapnet_cache_eviction* args, swapnet_stream stream);

/* Greedy acceptance of a drafted tree: node 0 is the token that the last pass
 * chose; from node i the path goes on to its lowest child whose id equals
 * targets[i] (the model's choice at node i, e.g. ARGMAX), until there is none.
 * path gets the accepted nodes in order (-1 behind them), accepted their
 * number, next the model's choice at the last one, lens_out = lens + accepted;
 * the accepted rows of every draft are appended to its cache at row lens.  A
 * sequence whose cache has no room for its path, or with counts < 1, is left
 * alone and reported as above.  At most 128 nodes and 256 caches (distinct
 * ones); results overlap no input.
 * Errors: INVALID_ARG, MISALIGNED, UNSUPPORTED, CUDA. */
typedef struct swapnet_tree_acceptance {
  int32_t dtype, n_seq, tokens;
  int32_t width;          /* elements of a cache row                            */
  int32_t max_seq, n_caches;
  const int32_t* ids;     /* [n_seq][tokens] drafted tokens                     */
  const int32_t* targets; /* [n_seq][tokens]                                    */
  const int32_t* parents; /* [n_seq][tokens], NULL = a chain                    */
  const int32_t* counts;  /* [n_seq], NULL = tokens                             */
  const int32_t* lens;    /* [n_seq]                                            */
  void* const* caches;       /* host array of n_caches device pointers: keys and
                                values of every layer, one layout for all       */
  const void* const* drafts; /* host array: [n_seq * tokens][width], stride new_stride */
  int32_t* path;          /* [n_seq][tokens]                                    */
  int32_t* accepted;      /* [n_seq]                                            */
  int32_t* next;          /* [n_seq]                                            */
  int32_t* lens_out;      /* [n_seq], not lens itself                           */
  int64_t cache_stride, seq_stride, new_stride;
} swapnet_tree_acceptance;
int swapnet_tree_accept(const swapnet_tree_acceptance* args, swapnet_stream stream);

/* ------------------------------------------------- quantised caches
 * A key-value cache held in 8 bits, with a scale for each block of rows and key
 * head: half the bytes to hold, and for every decode step to read.  For programs
 * that keep their caches themselves: a decoder engine's, and those of the calls
 * above, have 16 bits.  swapnet_cache_append prepares a step's queries and puts its
 * rows into the cache; swapnet_attention_quantized reads it.  What is said of
 * the cached-attention calls above (streams, captures, workspaces, errors found
 * on the device, the current device) holds for these as well.  The paper has no
 * counterpart.
 *
 * Layout: codes k, v of cache_dtype, [n_seq][max_seq][kv_heads][head_dim] with
 * kv_stride and seq_stride as above (in codes, multiples of 16; 0 = packed);
 * scales [n_seq][kv_heads][ceil(max_seq / block)] fp32.  The scale of block i
 * is that of rows i * block .. i * block + block - 1 of one head; a value is
 * code * scale.  block: 16, 32, 64 or 128.  The rows of a sequence's last
 * block, as long as it is not full, are kept in 16 bits as well: k_open, v_open,
 * [n_seq][block][kv_heads][head_dim], row j of the cache at j % block.  A row is
 * rounded to 8 bits from its 16-bit value whatever the calls that append it,
 * and the cache is a function of the rows alone:
 *   E4M3  scale = the least power of two >= m / 448
 *   I8    scale = m / 127
 * with m the block's largest magnitude so far (scale at least 2^-100), code =
 * value / scale rounded to the nearest (ties to even).  A block with a value
 * that is infinite or not a number has a scale that is not a number (codes of
 * I8: 0; E4M3: not a number), and so is the attention of every query that sees
 * one of its rows.
 *
 * A sequence's last rows can be taken back by a smaller length as far as the
 * start of its open block, no further: the 16-bit rows of the block before are
 * gone, and nothing would notice that those of another stand in their place.
 * The open block's codes and scale stay as the rows taken back left them until
 * the next append that brings the sequence a row.  To take back any number of a
 * call's rows (a drafted run, part of which is accepted): append the run with
 * other buffers for the open rows (and for the queries); once the counts are
 * known, append it again, with those counts, from the same lens and open rows,
 * which may now be updated in place. */

/* Appends the rows of up to `tokens` new tokens per sequence to a cache, and
 * prepares their queries:
 *   q, k: x / sqrt(mean(x^2) + eps) * gain for each head (with a gain), then the
 *   rotation (with theta): pair i of the first rope_dim elements turned by
 *   position * theta^(-2 i / rope_dim); pairs are (2i, 2i + 1), with `halves`
 *   (i, i + rope_dim / 2).  Rounded once, to dtype.  v as it is.  An angle is off
 *   by at most 2^-21 and 2^-49 of position * theta^(-2 i / rope_dim).
 * With `sections` the pairs follow up to three position axes (e.g. time, height,
 * width): the first sections[0] pairs axis 0, the next sections[1] axis 1, the
 * rest axis 2.
 * k and v rows t < counts[b] go to rows lens[b] + t; lens_out = lens + counts.
 * cache_dtype = dtype: a 16-bit cache, rows as they are (block 0, no scales).
 * I8, E4M3: as above; k_open_out and v_open_out receive the rows of the block
 * that is open afterwards (NULL: in place; other buffers: the call may be
 * repeated).  Rows at and behind counts of q_out, rows at and behind lens_out
 * of the cache and of the open block, and scales of blocks without new rows are
 * left as they were.  A sequence whose rows do not fit its cache, or with a
 * length or count out of range, is left alone and reported by
 * swapnet_device_sync; a position that is negative or not below 2^24 counts as
 * 0 and is reported.
 * heads = 0, q and q_out NULL: no queries (a 16-bit cache put into 8 bits).
 * q_out may be q (one stride); no other result may be an input.  head_dim 64 or
 * 128.
 * Errors: INVALID_ARG, MISALIGNED, UNSUPPORTED, CUDA. */
typedef struct swapnet_cache_rows {
  int32_t dtype;        /* F16 or BF16: queries, new rows, gains, open rows      */
  int32_t cache_dtype;  /* dtype, SWAPNET_I8 or SWAPNET_E4M3                     */
  int32_t n_seq, tokens, heads, kv_heads, head_dim;
  int32_t max_seq;      /* rows of a sequence's cache, at most 2^24              */
  int32_t block;        /* rows of a scale; 0 for a 16-bit cache                 */
  int32_t rope_dim;     /* a multiple of 16 up to head_dim; 0 = head_dim         */
  int32_t halves;       /* which elements make a pair                            */
  int32_t sections[3];  /* pairs of each axis, rope_dim / 2 in all; all 0: one axis */
  float theta;          /* 0: no rotation                                        */
  float eps;            /* of the norms                                          */
  const void* q;        /* [n_seq * tokens][heads * head_dim], stride q_stride   */
  const void* k_new;    /* [n_seq * tokens][kv_heads * head_dim], stride new_stride */
  const void* v_new;
  const void* q_gain;   /* [head_dim], NULL = no norm of the queries             */
  const void* k_gain;   /* the same for the keys                                 */
  const int32_t* lens;  /* [n_seq] rows of the cache in use before               */
  const int32_t* counts;    /* [n_seq] new rows, NULL = tokens                   */
  const int32_t* positions; /* [axes][n_seq][tokens], axes = 1 without sections,
                               else 3; NULL = lens + t on every axis             */
  void* q_out;          /* [n_seq * tokens][heads * head_dim], stride out_stride */
  void* k;              /* the cache                                             */
  void* v;
  float* k_scale;
  float* v_scale;
  const void* k_open;   /* the open blocks' rows                                 */
  const void* v_open;
  void* k_open_out;     /* NULL = k_open, v_open                                 */
  void* v_open_out;
  int32_t* lens_out;    /* [n_seq], not lens itself; nullable                    */
  int64_t q_stride, new_stride, out_stride, kv_stride, seq_stride; /* elements, 0 = packed */
} swapnet_cache_rows;
int swapnet_cache_append(const swapnet_cache_rows* args, swapnet_stream stream);

/* out[t] = sum_j softmax_j(scale q_t . k_j) v_j over a quantised cache, rounded
 * once: the queries are the cache's last `counts` rows, each sees the rows up to
 * its own (one token: a decode step whose row swapnet_cache_append has put into
 * the cache).  A query that sees no row gives 0 and lse = -inf.  Queries at and
 * behind counts are left as they were; codes and scales behind lens may hold
 * anything.
 * Scores, statistics and sums are fp32.  Keys and values enter the products as
 * fp16 numbers that hold their codes exactly, queries as fp16 (BF16 ones scaled
 * by a power of two per query, which loses what is below 2^-39 of its largest
 * element), probabilities times their value scales as two fp16 parts: 22 bits,
 * off by at most 2^-39 of a query's largest such product up to 16 rows (tokens x
 * heads / kv_heads; 32 with a head_dim of 64), 2^-32 beyond.  All that for value
 * scales from 2^-48 to 2^64 beside one another; the values of smaller ones lose
 * bits, and from 2^-79 on may count as 0.  A key whose value scale is 2^112 below
 * the largest (blocks of zeros count as 2^-48) may count for nothing in the sum of
 * weights where its own is below 2^-28 of the largest (2^-21 where products are
 * kept to 2^-32); nearer scales move that down bit by bit.  Scales are not
 * negative.
 * `workspace` as for swapnet_attention_tree: a function of the sizes; how many
 * CTAs share a cache goes by max_seq.  Results and workspace overlap
 * none of the inputs.  Errors: INVALID_ARG, MISALIGNED, UNSUPPORTED, CUDA. */
typedef struct swapnet_quantized_attention {
  int32_t dtype;        /* F16 or BF16: queries and outputs                      */
  int32_t cache_dtype;  /* SWAPNET_I8 or SWAPNET_E4M3                            */
  int32_t n_seq, tokens, heads, kv_heads, head_dim;
  int32_t max_seq, block;
  float scale;          /* of q . k; 0 = 1 / sqrt(head_dim)                      */
  const void* q;        /* rotated queries [n_seq * tokens], stride q_stride     */
  const void* k;
  const void* v;
  const float* k_scale;
  const float* v_scale;
  const int32_t* lens;   /* [n_seq] rows of the cache in use                     */
  const int32_t* counts; /* [n_seq] queries in use, NULL = tokens                */
  void* out;             /* [n_seq * tokens][heads * head_dim], stride out_stride */
  float* lse;            /* [n_seq][heads][tokens], nullable                     */
  int64_t q_stride, kv_stride, seq_stride, out_stride;
} swapnet_quantized_attention;
int swapnet_attention_quantized_workspace(const swapnet_quantized_attention* args, uint64_t* bytes);
int swapnet_attention_quantized(const swapnet_quantized_attention* args, void* workspace, uint64_t workspace_bytes,
                                swapnet_stream stream);

/* How the call would run, which goes by the sizes alone (diagnostics, and tests
 * of a kernel's edges). */
typedef struct swapnet_quantized_tiling {
  int32_t kernel; /* 0 warp products; on the tensor cores 1 rows as rows, 2 keys as rows */
  int32_t rows;   /* of a unit: queries x heads that share a key head            */
  int32_t shared; /* 0 a CTA per unit; 1 equal runs of all units' tiles and a join */
  int32_t ctas;
} swapnet_quantized_tiling;
int swapnet_attention_quantized_tiling(const swapnet_quantized_attention* args, swapnet_quantized_tiling* tiling);

/* --------------------------------------------------------- host weights */
/* Page-locked, device-mapped host memory for weight storage (the pinned
 * host copy that Sec. 4.2's swap-in reads): allocated by the CUDA driver in
 * large physically contiguous pieces, so the copy engines and the zero-copy
 * kernel stream it at full link rate however large it is; swapnet_load uses
 * it in place (no registration).  Caller-owned: release with
 * swapnet_host_free after every engine using it is freed.
 * Errors: INVALID_ARG (null out or zero bytes), OOM. */
int swapnet_host_alloc(uint64_t bytes, void** out);
int swapnet_host_free(void* p);

/* The lossless packed form of n_elems bf16 values (SWAPNET_SWAP_PACKED; an
 * extension the paper has no counterpart for).  Each value is split into
 * its exponent and a sign-mantissa byte; the exponent x is stored as the
 * 4-bit code x - x0, where x0 .. x0 + 14 (x0 <= 240) is the window of 15
 * consecutive exponents holding most of the tensor, code 15 marking an
 * exception; up to 4 exceptions per chunk of 4096 values are listed in the
 * chunk's header and chunks with more are stored unpacked.  Layout
 * (little-endian): 16 bytes (x0, then zeros); a 16-byte header per chunk
 * ([0] exception count or 0xff for an unpacked chunk, [4,12) positions as
 * uint16 (for 0xff: the overflow index as uint32 in [4,8)), [12,16) their
 * exponents); zeros up to a multiple of 128 bytes; a 6144-byte body per
 * chunk (2048 bytes of codes, two per byte, low nibble first, then 4096
 * sign-mantissa bytes (w >> 8 & 0x80) | (w & 0x7f); zeros for an unpacked
 * chunk); then the unpacked chunks, 8192 bytes
 * each.  A value is rebuilt as ((s & 0x80) << 8) | (x << 7) | (s & 0x7f)
 * with x = x0 + code, or the listed exponent for code 15.
 * With dst NULL only *used_bytes (the packed size) is written; otherwise
 * dst (dst_bytes long, any alignment) receives the packed form.  Host only,
 * multithreaded.  Errors: INVALID_ARG (null src or used_bytes, dst too
 * small), UNSUPPORTED (n_elems not a positive multiple of 4096), OOM (host
 * memory or threads). */
int swapnet_pack_bf16(const void* src, uint64_t n_elems, void* dst, uint64_t dst_bytes, uint64_t* used_bytes);

/* ------------------------------------------------------------------- misc */
const char* swapnet_strerror(int status);
const char* swapnet_last_error(void);

/* Host-side fault injection for tests: the next `count` calls of the named
 * step fail as if the CUDA call had failed.  what: 1 = cudaHostRegister,
 * 2 = device allocation, 3 = event/stream creation.  count 0 disarms. */
int swapnet_debug_fail_next(int what, int count);

/* Failure-detection check for tests: launches on `stream` one kernel whose
 * bounded device wait (the wait every kernel of the library uses on its
 * mbarriers) waits on an mbarrier that nothing completes, so it gives up
 * after the wait limit (one second), records the timeout in the library's
 * device error word and returns; no trap, no fault, the context stays
 * usable.  Synchronises the stream, reads and clears the error word, and
 * returns what swapnet_engine_sync would: SWAPNET_ERR_TIMEOUT. */
int swapnet_debug_wait_timeout(swapnet_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* SWAPNET_H */
