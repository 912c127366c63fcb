/*
 * cs.h - C ABI of the Complementary Sparsity sparse-sparse layer for AMD
 * Instinct MI355X (gfx950).
 *
 * The method (Hunter, Spracklen and Ahmad, "Two Sparsities Are Better Than
 * One", Section 3) overlays N sparse weight kernels whose supports do not
 * collide into one dense packed kernel that stores, per slot, a weight value
 * and a Kernel ID (Combine, Sections 3.1-3.2 step 1, Section 3.3.1).  At run
 * time only the non-zero activations are visited (Select, Section 3.2 step 2);
 * each is multiplied by the packed weights at its index (Multiply, step 3),
 * each product goes to the accumulator of its Kernel ID (Route, step 4,
 * Section 3.3.2) and is summed (Sum, step 5).  k-WTA (Section 3.3.3) then
 * keeps the k largest outputs, which become the next layer's sparse input.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Status: every function returns a cs_status (0 = success, < 0 = error).
 *    All argument checks are synchronous, run on the host and happen before
 *    any HIP call, so a bad argument never launches work and needs no GPU.
 *    A HIP launch or runtime failure returns CS_ERR_DEVICE; the library clears
 *    the HIP error state it observed.  No C++ exception crosses this ABI.
 *  - Ownership: the caller owns every buffer.  The GPU entry points never
 *    allocate, free or synchronise; they enqueue kernels on `stream` (a
 *    hipStream_t passed as void*, NULL = the default stream) and return.
 *    Outputs are completely overwritten.  Inputs and outputs must not alias.
 *  - "host" pointers are ordinary CPU memory; "device" pointers are GPU memory
 *    of the current HIP device.
 *  - Layouts are dense row-major.  Images are NHWC.  Conv weights are OHWI,
 *    flattened per output channel to r = kh*kw*c_in slots with slot
 *    i = (ky*kw + kx)*c_in + c (taps major, channels inner; Section 5.1 treats
 *    a 3x3 conv as nine 1x1 convs).
 *  - Packed sets: output channel o belongs to set (group) g = o / n and has
 *    Kernel ID kid = o - g*n; the n kernels of a set are n contiguous output
 *    channels.  G = d_out / n packed kernels.
 *  - Integer path: int8 activations and weights, int32 accumulation and bias
 *    (Section 4: weights and activations quantised to 8 bits).  Float path:
 *    fp32 throughout (CS_F16 and CS_BF16 are types of the attention layer's
 *    operators alone; every other call refuses them).  Integer sums wrap
 *    modulo 2^32 on overflow (the configurations used stay below 2^31 by a
 *    wide margin).
 */
#ifndef CS_H_
#define CS_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  CS_OK = 0,
  CS_ERR_ARG = -1,        /* null pointer, negative/zero size, bad enum value   */
  CS_ERR_SHAPE = -2,      /* sizes inconsistent or beyond the supported limits   */
  CS_ERR_DTYPE = -3,      /* unsupported dtype or dtype combination              */
  CS_ERR_COLLISION = -4,  /* cs_pack: two kernels of one set share a slot        */
  CS_ERR_WORKSPACE = -5,  /* workspace missing or smaller than required          */
  CS_ERR_DEVICE = -6,     /* HIP launch or runtime error                         */
  CS_ERR_UNSUPPORTED = -7 /* not available in this build of the library          */
} cs_status;

typedef enum { CS_I8 = 0, CS_I32 = 1, CS_F32 = 2, CS_F16 = 3, CS_BF16 = 4 } cs_dtype;

/* Supported limits (checked, CS_ERR_SHAPE beyond them). */
#define CS_MAX_ROW 65535   /* row length / c_in: indices are stored as uint16  */
#define CS_MAX_N 32        /* kernels per packed set                           */
#define CS_MAX_KWTA_ROW 2048 /* row length of cs_kwta                           */

/*
 * Augmented packed tensor (Section 3.3.1: each packed weight carries the
 * Kernel ID that routes its products; Figure 8(b)).  aug[i][g], i < r slots,
 * g < G sets, row-major, one entry per (slot, set):
 *   CS_I8 : uint16_t  = (uint8_t)value | (kid << 8)
 *   CS_F32: cs_aug_f32 {float value; uint32_t kid;}   (8 bytes)
 * kid is local to the set, in [0, n).  A slot no kernel of the set uses (a
 * hole) holds value 0, kid 0.
 */
typedef struct {
  float value;
  uint32_t kid;
} cs_aug_f32;

/*
 * cs_pack - Combine (Section 3.1/3.2 step 1, Figure 7): overlay each set of n
 * kernels into one packed kernel with its Kernel IDs.  Offline, HOST memory
 * only, no HIP call.
 *
 *  wt      CS_I8 or CS_F32: element type of w.
 *  w       host [d_out][r] dense weights; an exact zero is an absent weight.
 *  n       complement factor, 1 <= n <= CS_MAX_N, must divide d_out.
 *  aug     host [r][G] out, G = d_out / n, augmented entries as above:
 *          value = w[g*n + kid][i] for the one kernel of set g non-zero at i.
 *  holes   out (may be NULL): number of (i, g) slots no kernel of g uses.
 *  bad_g, bad_i  out (may be NULL): on CS_ERR_COLLISION, the first colliding
 *          (set, slot) in set-major, slot-minor order; -1 otherwise.
 *  Errors: CS_ERR_ARG (null w/aug, d_out/r < 1), CS_ERR_SHAPE (n does not
 *  divide d_out, n > CS_MAX_N), CS_ERR_DTYPE, CS_ERR_COLLISION (aug is then
 *  unspecified).
 */
int cs_pack(cs_dtype wt, const void* w, int d_out, int r, int n, void* aug, int64_t* holes,
            int* bad_g, int* bad_i);

/*
 * cs_compact - the sparse representation of Select (Section 3.2 step 2: the
 * non-zero activations with their indices; Figure 10 passes winners "along
 * with their indices").  DEVICE memory.
 *
 *  xt      CS_I8 or CS_F32.
 *  x       device [rows][c] dense activations.
 *  idx     device [rows][c] out (uint16): per row, the indices of the non-zero
 *          elements in ascending order in idx[row][0 .. cnt[row]-1]; the rest
 *          of the row is left untouched.
 *  val     device [rows][c] out (same dtype as x): the matching values.
 *  cnt     device [rows] out (int32): number of non-zeros of each row.
 *  A float -0.0 counts as zero.  rows may be 0 (nothing is launched).
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE (c > CS_MAX_ROW), CS_ERR_DEVICE.
 */
int cs_compact(cs_dtype xt, const void* x, int64_t rows, int c, uint16_t* idx, void* val,
               int32_t* cnt, void* stream);

/*
 * cs_mrs_conv2d - Multiply, Route and Sum (Section 3.2 steps 3-5, Sections
 * 3.3.1-3.3.2) of a convolution whose input is already in cs_compact form.
 * DEVICE memory.  For each output pixel and each non-zero (c, v) of every
 * input pixel under the kernel window at tap (ky, kx), slot
 * i = (ky*kw + kx)*c_in + c; for each set g the product v * aug[i][g].value
 * is added to output channel g*n + aug[i][g].kid.  Then bias, the optional 2x2
 * stride-2 max-pool (Table 1), then the NHWC store.
 *
 *  xt      CS_I8 (int8 lists and weights, int32 bias and y) or CS_F32.
 *  idx, lval, cnt  device lists of the b*h*w input pixels as cs_compact or
 *          cs_kwta_lists write them, row stride `cap` (cap >= 1 entries): every
 *          index < c_in; a count above cap is read as cap.  Row strides that
 *          are multiples of 4 take the fast path (4 entries per load).
 *  b, h, w, c_in   input geometry; kh, kw >= 1; stride >= 1; pad >= 0.
 *          ho = (h + 2*pad - kh)/stride + 1, wo likewise, both >= 1.
 *  aug     device augmented packed tensor [kh*kw*c_in][G] from cs_pack
 *          (every kid < n), element type of xt.
 *  c_out, n  n divides c_out, 1 <= n <= CS_MAX_N.
 *  bias    device [c_out] (int32 / fp32) or NULL for none.
 *  pool    1 (none) or 2 (2x2 stride-2 max-pool; ho and wo must be even).
 *  y       device NHWC [b][ho/pool][wo/pool][c_out] out (int32 / fp32).
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE, CS_ERR_DEVICE.
 */
int cs_mrs_conv2d(cs_dtype xt, const uint16_t* idx, const void* lval, const int32_t* cnt, int cap,
                  int b, int h, int w, int c_in, int kh, int kw, int stride, int pad,
                  const void* aug, int c_out, int n, const void* bias, int pool, void* y,
                  void* stream);

/*
 * cs_mrs_kwta_conv2d - one whole layer: cs_mrs_conv2d followed by k-WTA along
 * the channels of every output pixel (Section 2.2.2: exactly the top k
 * activations propagate; Section 3.3.3 local k-WTA), with the winners sent on
 * as (index, value) lists (Figure 10) or as a dense masked tensor.  DEVICE
 * memory.  A layer with one output vector per sample (a linear layer: window
 * = the whole unpadded map, output 1 x 1, no pool; at most 1024 input pixels)
 * runs as one kernel with one workgroup per sample, the table read from
 * global memory; a layer whose packed table fits one workgroup's LDS runs as
 * one kernel with the table in LDS; in both the sums need not reach HBM.
 * Otherwise cs_mrs_conv2d and cs_kwta / cs_kwta_lists run back to back on
 * `stream`.
 *
 *  xt .. pool   as cs_mrs_conv2d.
 *  y       device NHWC [b][ho/pool][wo/pool][c_out] (int32 / fp32), always
 *          required: with keep_sums = 1 it holds the sums after pool and bias
 *          on return; with keep_sums = 0 it is scratch and its contents are
 *          unspecified.
 *  k       winners per output pixel, 0 <= k <= c_out; ties go to the lower
 *          channel index; fp32 compares numerically (-0.0 == +0.0).
 *  ot      output dtype: CS_F32 for fp32 input; CS_I32 (the sums themselves)
 *          or CS_I8 (requantised, clamp(v >> shift, -127, 127)) for int8.
 *  shift   0 .. 31, used with ot == CS_I8.
 *  out     device [b][ho/pool][wo/pool][c_out] of ot: winners kept, the rest
 *          zero.  NULL when lists are written instead.
 *  oidx, oval, ocnt, ocap  list output (NULL when out is given): per output
 *          pixel, oidx/oval [rows][ocap] (uint16 / ot) hold the winners whose
 *          output value is non-zero in ascending channel order and ocnt[row]
 *          their number; ocap >= k.
 *  Exactly one of out and oidx must be non-NULL.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE (k > c_out, ocap < k, or
 *  c_out > CS_MAX_KWTA_ROW), CS_ERR_DEVICE.
 */
int cs_mrs_kwta_conv2d(cs_dtype xt, const uint16_t* idx, const void* lval, const int32_t* cnt,
                       int cap, int b, int h, int w, int c_in, int kh, int kw, int stride, int pad,
                       const void* aug, int c_out, int n, const void* bias, int pool, void* y,
                       int keep_sums, int k, cs_dtype ot, int shift, void* out, uint16_t* oidx,
                       void* oval, int32_t* ocnt, int ocap, void* stream);

/*
 * cs_mrs_kwta_units_conv2d - cs_mrs_kwta_conv2d with the k-WTA applied in
 * units: every `unit` consecutive channels of an output pixel keep their own
 * k winners (Section 5: channels partitioned into independent modules, each
 * with its own k-WTA; the ResNet-50 stages use units of 64 channels).  fp32
 * only (unit == c_out: exactly cs_mrs_kwta_conv2d, any dtype, ot = the sums'
 * dtype).  DEVICE memory.  One kernel when the layer runs on the table-block or
 * the streamed-table kernel with the selection on the lanes' own accumulators (no
 * pooling, power-of-two sets and kernels per set, n <= 16, c_out <= 256, a unit a
 * power-of-two number of a pixel's lanes); otherwise cs_mrs_conv2d and
 * cs_kwta on the [rows * c_out / unit][unit] view of y, dense output only.
 *
 *  xt .. keep_sums, out  as cs_mrs_kwta_conv2d (xt == CS_F32, output fp32).
 *  k       winners per unit, 0 <= k <= unit; ties go to the lower channel index.
 *  unit    channels per unit, dividing c_out.
 *  oidx, oval, ocnt, ocap  one list per output pixel with the winners of all
 *          its units in ascending channel order; ocap >= k * c_out / unit.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE (xt != CS_F32 with unit != c_out),
 *  CS_ERR_SHAPE (unit does not divide c_out, k > unit, ocap too small, or
 *  lists asked for a layer the single kernel does not take), CS_ERR_DEVICE.
 */
int cs_mrs_kwta_units_conv2d(cs_dtype xt, const uint16_t* idx, const void* lval,
                             const int32_t* cnt, int cap, int b, int h, int w, int c_in, int kh,
                             int kw, int stride, int pad, const void* aug, int c_out, int n,
                             const void* bias, int pool, void* y, int keep_sums, int k, int unit,
                             void* out, uint16_t* oidx, void* oval, int32_t* ocnt, int ocap,
                             void* stream);

/*
 * cs_mrs_plan - how cs_mrs_conv2d / cs_mrs_kwta_conv2d would run a layer with
 * these sizes (operands assumed aligned as torch allocates them).  Host only;
 * no HIP call.  For tests and tuning.
 *
 *  xt .. pool  as cs_mrs_kwta_conv2d; cap: list row stride; k: winners, or -1
 *          for cs_mrs_conv2d (sums only).
 *  info    host int64[11] out: [0] path (0 one lane per output, 1 table-slice
 *          kernel, 2 fused layer kernel, 3 one workgroup per sample: a layer
 *          whose window is the whole unpadded input map, output 1 x 1, no
 *          pool - a linear layer; 4 input-stationary int8 convolution; 5 one
 *          wavefront per item: an int8 1x1 layer of at least 128 items, the
 *          sums alone or with a k-WTA over rows of more than 128 channels or
 *          k > 32; 6 fp32 layer without pooling,
 *          sets and kernels per set powers of two, n <= 16, c_out <= 256:
 *          tiles complete in the channel dimension with the packed table
 *          streamed through LDS in blocks of rows, k-WTA in the epilogue; and
 *          the sums alone (k = -1) of such a 1x1 layer of a multiple of 256
 *          channels above 256, in slices of 256);
 *          for path 6: [1] k-WTA selection (1-3 four lanes per row with
 *          top-8/16/32 lists, 4 sixteen lanes per row, 5 the lanes that
 *          summed a pixel, on their own accumulators, bit by bit, 6-8 the
 *          same four lanes with top-8/16/32 lists; 9 the kernel that streams
 *          the table, whose lanes select as in 5), [2] table rows per
 *          block, [3] blocks, with [1] = 9 [4] channel slices and [5] log2 of
 *          the parts a pixel's list is added in (of the slices), [6]
 *          workgroups, [7] LDS bytes, [8] sets per lane; for path 3:
 *          [6] workgroups, [7] LDS bytes per workgroup, [8] entry slices per
 *          packed set; for path 5: [6] and [7] as for 3 (an estimate: the launch
 *          asks the device), [8] channels a lane holds at most, one of every 64;
 *          for path 4: [2] output rows per band, [6]
 *          workgroups, [7] LDS bytes, [8] sets per lane; for path 2: [1] tile mode (0 rows of
 *          items, 1 image rectangles), [2] items (mode 0) or pooled rows
 *          (mode 1) per tile, [3] pooled columns per tile (mode 1), [4] list
 *          chunks staged in LDS at most, [5] input pixels per tile at most,
 *          [6] workgroups, [7] LDS bytes per workgroup, [8] log2 of the lanes
 *          sharing one output's taps or chunks, [9] k-WTA selection variant;
 *          [10] 1 when k-WTA runs as a kernel of its own after the sums.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE.
 */
int cs_mrs_plan(cs_dtype xt, int cap, int b, int h, int w, int c_in, int kh, int kw, int stride,
                int pad, int c_out, int n, int pool, int k, int64_t* info);

/*
 * cs_linear - a whole sparse-sparse linear layer: cs_compact of x into the
 * workspace, then Multiply/Route/Sum (a linear layer is the 1x1 convolution
 * of 1x1 images); in one launch, the workspace untouched, when the layer runs
 * with a workgroup per sample, there are at most 1,024 samples (fp32: 2,048) or
 * their rows have at least 2,048 elements, and y shares no memory with x.  DEVICE
 * memory.
 *
 *  x       device [batch][d_in] (int8 or fp32), d_in <= CS_MAX_ROW.
 *  aug     device augmented packed tensor [d_in][G] from cs_pack of [d_out][d_in].
 *  bias    device [d_out] or NULL.   y  device [batch][d_out] out.
 *  ws      device workspace of at least cs_workspace_bytes(0, xt, batch, d_in)
 *          bytes, 256-byte aligned; its contents on entry do not matter.
 *  Errors: as cs_compact and cs_mrs_conv2d, plus CS_ERR_WORKSPACE.
 */
int cs_linear(cs_dtype xt, const void* x, int batch, int d_in, const void* aug, int d_out, int n,
              const void* bias, void* y, void* ws, size_t ws_bytes, void* stream);

/*
 * cs_conv2d - a whole sparse-sparse conv layer: cs_compact of the b*h*w input
 * pixels (rows of c_in) into the workspace, then cs_mrs_conv2d.  Arguments as
 * cs_mrs_conv2d with x a device NHWC [b][h][w][c_in] tensor; ws must hold at
 * least cs_workspace_bytes(1, xt, b*h*w, c_in) bytes.
 */
int cs_conv2d(cs_dtype xt, const void* x, int b, int h, int w, int c_in, int kh, int kw,
              int stride, int pad, const void* aug, int c_out, int n, const void* bias, int pool,
              void* y, void* ws, size_t ws_bytes, void* stream);

/*
 * cs_conv2d_kwta - a layer with k-WTA on its dense input: cs_compact of the
 * b*h*w input pixels into the lists lidx / lval [b*h*w][c_in] and lcnt [b*h*w],
 * then cs_mrs_kwta_conv2d on them; in one launch, lidx and lval untouched, for
 * a linear layer (1x1 images) where cs_linear takes one.  DEVICE memory.
 *
 *  xt .. pool   as cs_conv2d.      y .. ocap   as cs_mrs_kwta_conv2d.
 *  lidx, lval, lcnt   the caller's list buffers (not NULL, none of x's memory);
 *          lcnt holds the pixels' non-zero counts afterwards, lidx and lval are
 *          scratch.  The outputs may lie over x: then two launches.
 *  Errors: as cs_compact and cs_mrs_kwta_conv2d.
 */
int cs_conv2d_kwta(cs_dtype xt, const void* x, int b, int h, int w, int c_in, int kh, int kw,
                   int stride, int pad, const void* aug, int c_out, int n, const void* bias,
                   int pool, void* y, int keep_sums, int k, cs_dtype ot, int shift, void* out,
                   uint16_t* oidx, void* oval, int32_t* ocnt, int ocap, uint16_t* lidx, void* lval,
                   int32_t* lcnt, void* stream);

/*
 * cs_conv2d_noalloc - cs_conv2d for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc): the same computation and result, bit for bit, but the
 * compaction lists go to a scratch area the library holds instead of a
 * workspace the caller passes in.
 *
 *  Arguments as cs_conv2d without ws / ws_bytes (linear layers: b = batch,
 *  h = w = kh = kw = stride = 1, pad = 0, pool = 1).
 *  Scratch: a static device array of CS_NOALLOC_SCRATCH_BYTES per GPU, part
 *  of the library's code object, held from the library's load until the
 *  process ends; its address is looked up once per device on the first call
 *  made with that device current.  Nothing is allocated, freed or cleared by
 *  a call; every scratch byte the kernels read was written earlier in the
 *  same call.  All calls on one GPU share that GPU's scratch, so calls whose
 *  execution overlaps on one GPU (concurrent streams, host threads) race and
 *  must be serialised by the caller.
 *  Errors: as cs_conv2d; CS_ERR_WORKSPACE when the lists of the b*h*w input
 *  rows need more than CS_NOALLOC_SCRATCH_BYTES (cs_workspace_bytes(1, xt,
 *  b*h*w, c_in) is that need); CS_ERR_DEVICE if the scratch address cannot be
 *  obtained.
 */
#define CS_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)
int cs_conv2d_noalloc(cs_dtype xt, const void* x, int b, int h, int w, int c_in, int kh, int kw,
                      int stride, int pad, const void* aug, int c_out, int n, const void* bias,
                      int pool, void* y, void* stream);

/*
 * cs_mrs_kwta_chain2 - two layers of a chain's tail: a layer with k-WTA whose
 * output is one vector per sample (a linear layer, or a conv whose pooled map
 * is 1 x 1), then a linear layer without k-WTA on its requantised winners
 * (Figure 10: the winners go on with their indices).  When the first layer
 * runs one workgroup per sample (as cs_mrs_plan reports, path 3) both run in
 * one kernel: every winner (channel i, value v) adds v times the second
 * layer's packed row i into LDS accumulators, and the winners never leave the
 * chip (their lists are still written); otherwise cs_mrs_kwta_conv2d and
 * cs_mrs_conv2d run back to back on `stream`.  DEVICE memory.
 *
 *  xt .. ocap   as cs_mrs_kwta_conv2d, with xt == ot == CS_I8 and list
 *          output (oidx, oval, ocnt, ocap; no dense out).
 *  aug2, c_out2, n2, bias2   the second layer (cs_pack of [c_out2][c_out]
 *          int8 weights; bias2 int32 [c_out2] or NULL).
 *  y2      device int32 [b][c_out2] out: the second layer's sums.
 *  Errors: as cs_mrs_kwta_conv2d; CS_ERR_SHAPE when the first layer's output
 *  is not one vector per sample.
 */
int cs_mrs_kwta_chain2(cs_dtype xt, const uint16_t* idx, const void* lval, const int32_t* cnt,
                       int cap, int b, int h, int w, int c_in, int kh, int kw, int stride, int pad,
                       const void* aug, int c_out, int n, const void* bias, int pool, void* y,
                       int keep_sums, int k, cs_dtype ot, int shift, uint16_t* oidx, void* oval,
                       int32_t* ocnt, int ocap, const void* aug2, int c_out2, int n2,
                       const void* bias2, void* y2, void* stream);

/*
 * cs_mrs_kwta_chain3 - three layers of a chain's tail (Figure 10: every
 * layer's winners go on to the next with their indices): an int8 convolution
 * with k-WTA and lists, a layer with k-WTA whose window is that layer's whole
 * pooled map (one output vector per sample), and a linear layer without k-WTA
 * on its winners.  The result is that of cs_mrs_kwta_conv2d on the first
 * layer followed by cs_mrs_kwta_chain2 on its lists (input shape b x hp x wp x
 * c_out, window hp x wp, stride 1, no padding, no pool, where hp x wp is the
 * first layer's pooled map).  When the first layer runs input-stationary with
 * one workgroup per image and the second one workgroup per sample, the three
 * run in one kernel: each workgroup writes its image's lists, then (after a
 * workgroup barrier) reads them back as the second layer's input and feeds
 * the third layer on chip; otherwise the two calls run back to back on
 * `stream`.  DEVICE memory.
 *
 *  xt .. ocap   the first layer as cs_mrs_kwta_conv2d, with xt == ot == CS_I8
 *          and list output (oidx, oval, ocnt, ocap).
 *  aug2, c_out2, n2, bias2, y2, k2, shift2, oidx2, oval2, ocnt2, ocap2   the
 *          second layer (cs_pack of [c_out2][hp*wp*c_out] int8 weights in the
 *          (y, x, channel) slot order; bias2 int32 or NULL; y2 int32
 *          [b][c_out2] sums, written when keep_sums; k-WTA k2 with
 *          requantisation shift2, lists of capacity ocap2 >= k2).
 *  aug3, c_out3, n3, bias3, y3   the third layer as cs_mrs_kwta_chain2's
 *          second (y3: int32 [b][c_out3]).
 *  Errors: as cs_mrs_kwta_conv2d and cs_mrs_kwta_chain2 (CS_ERR_ARG for a
 *  missing buffer or a bad k, shift or keep_sums; CS_ERR_SHAPE for sizes).
 */
int cs_mrs_kwta_chain3(cs_dtype xt, const uint16_t* idx, const void* lval, const int32_t* cnt,
                       int cap, int b, int h, int w, int c_in, int kh, int kw, int stride, int pad,
                       const void* aug, int c_out, int n, const void* bias, int pool, void* y,
                       int keep_sums, int k, cs_dtype ot, int shift, uint16_t* oidx, void* oval,
                       int32_t* ocnt, int ocap, const void* aug2, int c_out2, int n2,
                       const void* bias2, void* y2, int k2, int shift2, uint16_t* oidx2,
                       void* oval2, int32_t* ocnt2, int ocap2, const void* aug3, int c_out3,
                       int n3, const void* bias3, void* y3, void* stream);

/*
 * cs_conv2d_dense_kwta_chain3 - a whole chain shaped like the keyword-spotting
 * network of Section 4: the dense-input first layer (as cs_conv2d_dense_kwta,
 * int8, list output), then the three layers of cs_mrs_kwta_chain3 on its lists
 * (input shape b x hp x wp x c_out, where hp x wp is the first layer's pooled
 * map).  The result is that of those two calls.  When the first layer's
 * matrix-core kernel can take a whole image per workgroup and the three-layer
 * tail runs in one kernel (cs_mrs_kwta_chain3's condition, or: the second
 * layer has eight list slots per pixel (ocap == 8), a square 3x3 or 5x5
 * window, four sets (c_out2 == 4 * n2 <= 64), the first layer pools 2x2 and
 * the second layer's output map fits in LDS, which runs it output-stationary),
 * all four layers run in one kernel, one workgroup per image, the phases
 * separated by workgroup barriers and the lists between them read back from
 * L2; otherwise the two calls run back to back on `stream`.  The result does
 * not depend on the path (integer sums).  DEVICE memory.
 *
 *  xt .. ocap   the first layer as cs_conv2d_dense_kwta (xt == ot == CS_I8,
 *          list output oidx/oval/ocnt/ocap, no dense out).
 *  kh2 .. ocap2   the second layer (a conv over the first one's lists) as the
 *          first layer of cs_mrs_kwta_chain3: window, stride, padding, packed
 *          table, c_out2, n2, bias, pool, sums y2, k-WTA k2 / shift2 and lists.
 *  aug3 .. ocap3   the third layer (window = the second one's whole pooled map)
 *          as cs_mrs_kwta_chain3's second.
 *  aug4, c_out4, n4, bias4, y4   the last linear layer, as its third.
 *  keep_sums applies to the first three layers' sums y, y2, y3.
 *  Errors: as cs_conv2d_dense_kwta and cs_mrs_kwta_chain3.
 */
int cs_conv2d_dense_kwta_chain3(
    cs_dtype xt, const void* x, int b, int h, int w, int c_in, int kh, int kw, int stride, int pad,
    const void* aug, int c_out, int n, const void* bias, int pool, void* y, int keep_sums, int k,
    cs_dtype ot, int shift, uint16_t* oidx, void* oval, int32_t* ocnt, int ocap, int kh2, int kw2,
    int stride2, int pad2, const void* aug2, int c_out2, int n2, const void* bias2, int pool2,
    void* y2, int k2, int shift2, uint16_t* oidx2, void* oval2, int32_t* ocnt2, int ocap2,
    const void* aug3, int c_out3, int n3, const void* bias3, void* y3, int k3, int shift3,
    uint16_t* oidx3, void* oval3, int32_t* ocnt3, int ocap3, const void* aug4, int c_out4, int n4,
    const void* bias4, void* y4, void* stream);

/*
 * cs_conv2d_dense_blocks - the sparse-dense variant with block Complementary
 * Sparsity (Section 3.1: complementary patterns made of blocks; Section 5: a
 * stem whose block is one input pixel's RGB values; Section 4: a first layer
 * on dense input runs sparse-dense).  DEVICE memory, int8 activations and
 * weights, int32 sums.  A block is one tap's c_in channels: the c_in products
 * of a (tap, set) pair are summed first (one 4-way int8 dot product) and the
 * sum is routed once by the block's Kernel ID, so an output pixel costs
 * kh*kw*(c_out/n) dot products and routed adds.  Layers of whole 16-channel
 * tiles (c_out % 16 == 0, y 16-byte aligned) and windows of up to 7x7 run as the
 * same contraction on the matrix cores, a block's Kernel ID routing its weights
 * once when the weight operand is built; the sums are the same bits.  No
 * compaction, no workspace.
 *
 *  x       device NHWC [b][h][w][c_in] int8, dense; 1 <= c_in <= 4.
 *  aug     device [kh*kw*c_in][c_out/n] uint16 (cs_pack_blocks with b = c_in:
 *          value in the low byte).
 *  kidb    device [kh*kw][c_out/n] uint8: each block's Kernel ID (< n), as
 *          cs_pack_blocks writes it.
 *  bias    device int32 [c_out] or NULL.
 *  y       device NHWC [b][ho][wo][c_out] int32 out: the sums plus bias.
 *  Errors: CS_ERR_ARG, CS_ERR_SHAPE (c_in > 4, c_out/n sets too many for one
 *  workgroup, the input under one tile - kh rows of (P-1)*stride + kw
 *  pixels, P = 256 / lanes per pixel output pixels - over 1024 pixels, or
 *  the tile's LDS over 64 KB), CS_ERR_DEVICE.
 */
int cs_conv2d_dense_blocks(const int8_t* x, int b, int h, int w, int c_in, int kh, int kw,
                           int stride, int pad, const uint16_t* aug, const uint8_t* kidb,
                           int c_out, int n, const int32_t* bias, int32_t* y, void* stream);

/*
 * cs_conv2d_dense_blocks_plan - how cs_conv2d_dense_blocks would run these sizes (y
 * 16-byte aligned).  Host only; no HIP call.  For tests and tuning.
 *
 *  info    host int64[8] out: [0] 1 on the matrix cores, 0 the routed kernel (then
 *          the rest is 0); [1] output rows of a tile, [2] its groups of 16 output
 *          columns, [3] tiles across an output row, [4] tiles, [5] workgroups of a
 *          channel slice (each takes tiles from its own on, that many apart),
 *          [6] channel slices, [7] contraction steps of 16 taps.
 *  Errors: CS_ERR_ARG, CS_ERR_SHAPE as cs_conv2d_dense_blocks.
 */
int cs_conv2d_dense_blocks_plan(int b, int h, int w, int c_in, int kh, int kw, int stride, int pad,
                                int c_out, int n, int64_t* info);

/*
 * cs_conv2d_dense - the sparse-dense variant (Section 3.1: Combine, Multiply,
 * Route, Sum with dense activations; Section 4 runs the first layer of the
 * keyword-spotting network this way because its input is dense).  DEVICE
 * memory.  Same arguments and result as cs_conv2d, but x is read densely (no
 * compaction, no workspace).  Supported shapes (else CS_ERR_SHAPE): n == 1
 * (every set holds one dense kernel), c_out == 64, kh*kw*c_in <= 32 and an
 * input patch per output item ((pool-1)*stride + kh) * ((pool-1)*stride + kw)
 * * c_in <= 64 values.
 */
int cs_conv2d_dense(cs_dtype xt, const void* x, int b, int h, int w, int c_in, int kh, int kw,
                    int stride, int pad, const void* aug, int c_out, int n, const void* bias,
                    int pool, void* y, void* stream);

/*
 * cs_conv2d_dense_kwta - the whole dense-input first layer: cs_conv2d_dense
 * followed by k-WTA along the channels of every output pixel, with the
 * winners emitted as lists or densely, as cs_mrs_kwta_conv2d does for a
 * sparse input.  DEVICE memory.  For int8 with k <= 32 the convolution runs
 * on the matrix cores (int8 MFMA; the dense contraction of Section 3.1's
 * sparse-dense case) in the same kernel as the pool, the selection and the
 * output, and the sums need not reach HBM; otherwise cs_conv2d_dense and
 * cs_kwta / cs_kwta_lists run back to back on `stream`.
 *
 *  xt .. pool   as cs_conv2d_dense (n == 1, c_out == 64, kh*kw*c_in <= 32; the
 *          two-kernel path, taken for fp32 or k > 32, also needs the pooled
 *          window to hold at most 64 values, else CS_ERR_SHAPE).
 *  y, keep_sums, k, ot, shift, out, oidx, oval, ocnt, ocap   as
 *          cs_mrs_kwta_conv2d.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE, CS_ERR_DEVICE.
 */
int cs_conv2d_dense_kwta(cs_dtype xt, const void* x, int b, int h, int w, int c_in, int kh, int kw,
                         int stride, int pad, const void* aug, int c_out, int n, const void* bias,
                         int pool, void* y, int keep_sums, int k, cs_dtype ot, int shift, void* out,
                         uint16_t* oidx, void* oval, int32_t* ocnt, int ocap, void* stream);

/* Output tile side of the reordering kernel (CS_REORDER_TILE^2 pixels). */
#define CS_REORDER_TILE 8

/*
 * cs_reorder_table - the packed kernel in Kernel-ID order, for reordering
 * the activations instead of routing the products (Section 3.2: reordering
 * the incoming activations as the alternative to routing the element-wise
 * products).  Offline, HOST memory only, no HIP call.  For every output
 * o = g*n + kid the table lists the slots i of set g with kid[i][g] == kid and
 * a non-zero value (the support of kernel o), in ascending slot order, as
 * pairs (byte offset of slot i in cs_conv2d_reorder_kwta's input tile,
 * value bits): slot i = (ky*kw + kx)*c_in + c has offset
 * 4*((ky*(CS_REORDER_TILE + kw - 1) + kx)*(c_in + 1) + c).
 *
 *  aug     host [kh*kw*c_in][c_out/n] cs_aug_f32 entries (cs_pack, CS_F32).
 *  smax    in/out: with table == NULL, receives the longest support (>= 1);
 *          else the entries per output the table has room for (>= that).
 *  table   host [c_out][smax][2] int32 out (may be NULL), outputs shorter
 *          than smax padded with (0, 0.0f).
 *  Errors: CS_ERR_ARG (null aug/smax, sizes < 1, a kid >= n), CS_ERR_SHAPE
 *  (n does not divide c_out, n > CS_MAX_N, kh*kw*c_in > CS_MAX_ROW, smax too
 *  small).
 */
int cs_reorder_table(const void* aug, int kh, int kw, int c_in, int c_out, int n, int* smax,
                     int32_t* table);

/*
 * cs_pack_blocks - Combine for Complementary Sparsity with blocks of
 * non-zeros (Section 3.1: complementary patterns made of blocks; Section 5's
 * stem treats a pixel's 3 RGB inputs as one block).  Slots j*b .. j*b+b-1 form
 * block j (for conv weights in (tap, channel) slot order and b dividing c_in,
 * a block is b consecutive channels of one tap); every kernel's support must
 * be a union of whole blocks, complementary within each set block by block.
 * Offline, HOST memory only, no HIP call.
 *
 *  wt, w, d_out, r, n, aug   as cs_pack (aug is the per-slot augmented
 *          tensor every layer call reads); b divides r.
 *  kidb    host [r/b][G] uint8 out: the Kernel ID of each (block, set) - one
 *          routing decision for the block's b products (0 for a hole).
 *  holes   out (may be NULL): (block, set) pairs no kernel uses.
 *  bad_g, bad_i  out (may be NULL): on CS_ERR_SHAPE for a split block, the
 *          kernel and the block; on CS_ERR_COLLISION, the set and the block.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE (n does not divide d_out,
 *  n > CS_MAX_N, b does not divide r, a support splits a block),
 *  CS_ERR_COLLISION.
 */
int cs_pack_blocks(cs_dtype wt, const void* w, int d_out, int r, int n, int b, void* aug,
                   uint8_t* kidb, int64_t* holes, int* bad_g, int* bad_i);

/*
 * cs_pack_channels - Combine along the channel dimension (Section 3.1: sets
 * of kernels can be overlaid in the filter or in the channel dimension).  In
 * every filter, each group of n consecutive input channels holds n kh x kw
 * slices with disjoint supports; they are overlaid into one dense kh x kw
 * slice whose slots keep the weight and the channel ID (which slice, 0..n-1).
 * Offline, HOST memory only, no HIP call.
 *
 *  wt      CS_F32 or CS_I8.  w host [c_out][kh][kw][c_in] dense filters (0 =
 *          absent).
 *  n       channels per group, 1 <= n <= CS_MAX_N, dividing c_in.
 *  packed  host [c_out][c_in/n][kh][kw] out, cs_aug_f32 (CS_F32) or uint16
 *          (CS_I8: value byte | channel ID << 8) entries, kid = channel ID:
 *          value = w[o][y][x][q*n + cid] for the one channel of group q that
 *          is non-zero at (y, x); holes hold 0, 0.
 *  holes   out (may be NULL): packed slots no channel uses.
 *  bad_o, bad_i  out (may be NULL): on CS_ERR_COLLISION the first colliding
 *          filter and packed slot (q*kh + y)*kw + x, in that order; else -1.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE (n does not divide c_in,
 *  n > CS_MAX_N), CS_ERR_COLLISION (packed then unspecified).
 */
int cs_pack_channels(cs_dtype wt, const void* w, int c_out, int kh, int kw, int c_in, int n,
                     void* packed, int64_t* holes, int* bad_o, int* bad_i);

/*
 * cs_channel_table - the table cs_conv2d_channels reads for an int8
 * channel-overlaid layer (cs_pack_channels, CS_I8) run with stride `stride`.
 * Offline, HOST memory only, no HIP call.  Filter o's row holds, with S =
 * (c_in/n)*kh*kw packed slots and S4 = ceil(S/4): first 4*S4 offsets, slot
 * i = (q*kh + y)*kw + x at [i] (padding slots 0): off = (y*sw + x)*cp + q*n +
 * cid, the byte offset of the slot's input (tap (y, x), channel q*n + cid)
 * from the first input pixel of an output pixel's window in the kernel's
 * staged tile (sw = 63*stride + kw pixels per staged row, cp = c_in bytes per
 * pixel when c_in/4 is odd, else c_in + 4); then S4 words, word j holding the
 * weights of slots 4j .. 4j+3 in its bytes (0 for padding slots).
 *
 *  packed  host [c_out][c_in/n][kh][kw] uint16 (cs_pack_channels, CS_I8).
 *  table   host int32 [c_out][5 * S4] out.
 *  Errors: CS_ERR_ARG (null pointers, sizes < 1, a channel ID >= n),
 *  CS_ERR_SHAPE (n does not divide c_in, c_in not a multiple of 4, n >
 *  CS_MAX_N, the staged tile reaching 2^23 bytes).
 */
int cs_channel_table(const uint16_t* packed, int kh, int kw, int c_in, int c_out, int n,
                     int stride, int32_t* table);

/*
 * cs_conv2d_channels - an int8 dense-input conv layer with Complementary
 * Sparsity overlaid in the channel dimension (Section 3.1): every output is
 * the dot product of its filter's packed slots with the input gathered at
 * each slot's channel (q*n + channel ID) - no routing, the products of a
 * filter all go to its own output.  DEVICE memory (except the scalars).
 * Output tiles of 64 pixels of one output row, one pixel per lane, the
 * filters split over the four wavefronts of a workgroup; the tile's input
 * rows staged in LDS with the pixel stride of cs_channel_table.
 *
 *  x       device NHWC [b][h][w][c_in] int8, dense, 4-byte aligned; c_in a
 *          multiple of 4.
 *  table   device copy of cs_channel_table's table for this stride.
 *  c_out   16, 32, 64 or 128; n as packed.
 *  bias    device int32 [c_out] or NULL.
 *  y       device NHWC [b][ho][wo][c_out] int32 out (16-byte aligned): sums + bias.
 *  Errors: CS_ERR_ARG, CS_ERR_SHAPE (c_out, c_in or n unsupported, the staged
 *  tile over 64 KB of LDS), CS_ERR_DEVICE.
 */
int cs_conv2d_channels(const int8_t* x, int b, int h, int w, int c_in, int kh, int kw, int stride,
                       int pad, const int32_t* table, int c_out, int n, const int32_t* bias,
                       int32_t* y, void* stream);

/*
 * cs_reorder_table_channels - cs_reorder_table for a channel-overlaid layer
 * (cs_pack_channels): every filter's packed slots (q, y, x) with a non-zero
 * value read channel q*n + cid at tap (y, x), so the filter's table lists
 * them with that slot's byte offset in cs_conv2d_reorder_kwta's input tile;
 * the layer then runs as any reordered layer.  Offline, HOST memory only.
 *  packed  host [c_out][c_in/n][kh][kw] cs_aug_f32 (cs_pack_channels).
 *  smax, table   as cs_reorder_table.
 *  Errors: CS_ERR_ARG (null packed/smax, sizes < 1, a channel ID >= n),
 *  CS_ERR_SHAPE (n does not divide c_in, n > CS_MAX_N, kh*kw*c_in >
 *  CS_MAX_ROW, smax too small).
 */
int cs_reorder_table_channels(const void* packed, int kh, int kw, int c_in, int c_out, int n,
                              int* smax, int32_t* table);

/*
 * cs_conv2d_reorder_kwta - a dense-input fp32 conv layer computed by
 * reordering instead of routing: every output reads the activations at its
 * kernel's support (cs_reorder_table) and sums their products in a register;
 * then k-WTA along the channels of every output pixel as cs_mrs_kwta_conv2d.
 * Same sums as cs_conv2d_dense_kwta / cs_conv2d + cs_mrs_kwta_conv2d up to
 * fp32 rounding order.  DEVICE memory (except the scalars).
 *
 *  xt      CS_F32.  x device NHWC [b][h][w][c_in] dense activations.
 *  kh, kw, pad   window and zero padding; stride 1, no pooling.
 *  table, smax   device copy of cs_reorder_table's table for this layer, with
 *          smax a multiple of 8 (CS_ERR_SHAPE otherwise).
 *  c_out   must be 64; c_in <= 64.
 *  bias    device [c_out] (may be NULL).
 *  y, keep_sums  device [b][ho][wo][c_out] sums, written when keep_sums == 1
 *          (16-byte aligned).
 *  k       winners per pixel, 0 <= k <= 32 or k == c_out; ot CS_F32.
 *  out | (oidx, oval, ocnt, ocap)   exactly one: dense [b][ho][wo][c_out]
 *          output (winners keep their value, the rest 0; 16-byte aligned), or
 *          lists as cs_mrs_kwta_conv2d with ocap >= k and a multiple of 4,
 *          oidx 8-byte and oval 16-byte aligned.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE, CS_ERR_DEVICE.
 */
int cs_conv2d_reorder_kwta(cs_dtype xt, const void* x, int b, int h, int w, int c_in, int kh,
                           int kw, int pad, const int32_t* table, int smax, int c_out,
                           const void* bias, void* y, int keep_sums, int k, cs_dtype ot,
                           void* out, uint16_t* oidx, void* oval, int32_t* ocnt, int ocap,
                           void* stream);

/*
 * cs_kwta - k-WTA (Section 2.2.2: exactly the top k activations propagate;
 * Section 3.3.3: global k-WTA over a vector after linear layers, local k-WTA
 * along the channels of each pixel after conv layers - both are this call
 * with one row per vector or per pixel).  DEVICE memory.
 *
 *  it      CS_I32 or CS_F32: dtype of `in`.
 *  in      device [rows][c], 1 <= c <= CS_MAX_KWTA_ROW, 0 <= k <= c.
 *  Each row keeps exactly k elements: the k largest, equal values going to
 *  the lower index; fp32 compares numerically (-0.0 ties +0.0; NaN is not
 *  supported).  Winners keep their value (even if <= 0), the rest become 0.
 *  ot      == it: out holds the masked values.
 *          CS_I8 with it == CS_I32: out holds requantised winners
 *          clamp(v >> shift, -127, 127) (arithmetic shift), 0 elsewhere.
 *  shift   0..31, used only for CS_I8 output.
 *  out     device [rows][c] out.  rows may be 0.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE, CS_ERR_DEVICE.
 */
int cs_kwta(cs_dtype it, const void* in, int64_t rows, int c, int k, cs_dtype ot, int shift,
            void* out, void* stream);

/*
 * cs_kwta_lists - k-WTA whose winners go to the next layer as (index, value)
 * lists (Figure 10: the values that pass are sent on "along with their
 * indices"; Section 3.2: the next layer's Select is this list).  DEVICE memory.
 * Same selection and dtype rules as cs_kwta (exactly k, ties to the lower
 * index, optional int8 requantisation), but instead of a dense row it writes,
 * per row, the winners whose output value is non-zero in ascending index
 * order: idx[row][0 .. cnt[row]-1] (uint16), val[row][..] (dtype ot),
 * cnt[row] (int32), row stride `cap` >= k.  Entries past cnt are untouched.
 * These lists feed cs_mrs_conv2d directly (its cap argument = this cap).
 *  Errors: as cs_kwta; CS_ERR_SHAPE if cap < k.
 */
int cs_kwta_lists(cs_dtype it, const void* in, int64_t rows, int c, int k, cs_dtype ot, int shift,
                  uint16_t* idx, void* val, int32_t* cnt, int cap, void* stream);

/*
 * cs_workspace_bytes - workspace cs_linear (op 0) or cs_conv2d (op 1) needs
 * for `rows` input rows (batch, or b*h*w pixels) of c_in elements of dtype
 * xt.  Returns 0 for invalid arguments.  Host only.
 */
size_t cs_workspace_bytes(int op, cs_dtype xt, int64_t rows, int c_in);

/*
 * 8-bit operators of a transformer's attention layer
 * --------------------------------------------------
 * Floats of these calls are CS_F32, CS_F16 (IEEE half) or CS_BF16; sums,
 * softmax statistics and scales are 32 bits wide whatever their type, and a
 * result is rounded to it once (what cs_paged_attention multiplies has fewer
 * bits, as said there).  Rows may be strided: ld* is the distance of
 * two rows and hs* that of two heads, in elements; a row's own elements are
 * contiguous.  Vector loads are used where pointers and strides are multiples
 * of 16 bytes, single elements elsewhere, with the same results.
 *
 * Codes: a row of floats is held as int8 codes with one scale,
 * s = fl32(max|x| / 127), code = rne(fl32(x / s)) (fl32: rounded to 32 bits,
 * rne: to the nearest integer, ties to even) in [-127, 127]; value = code * s.
 * A row whose s is 0 has codes 0; a row with an infinity or a NaN has scale
 * NaN and codes 0, so that what is computed from it is NaN.
 */

#define CS_MAX_Q8_K 131072      /* k of cs_linear_q8: that many products of two codes fit int32 */
#define CS_MAX_Q8_OUT (1 << 22) /* d_out of cs_linear_q8                                        */
#define CS_MAX_Q8_LEN (1 << 30) /* positions that a row of cs_paged_attention's table holds     */

/*
 * cs_quantise_rows - codes and scales of the rows of a float matrix (tokens
 * before a product; a weight matrix, once).  DEVICE memory.
 *  xt      CS_F32, CS_F16 or CS_BF16.  x device [rows][c], row stride ldx >= c.
 *  q       device [rows][c] out, row stride ldq >= c (bytes between c and ldq
 *          are left alone); 8-byte stores where rows start on 8 bytes.
 *  scale   device [rows] out.  rows may be 0.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE (a stride below c, more than
 *  2^31 - 1 rows), CS_ERR_DEVICE.
 */
int cs_quantise_rows(cs_dtype xt, const void* x, int64_t ldx, int64_t rows, int c, int8_t* q,
                     int64_t ldq, float* scale, void* stream);

/*
 * cs_linear_q8 - a dense linear layer on 8-bit codes:
 * y[t][n] = (sum_k x[t][k] w[n][k]) * (sx[t] * sw[n]) + bias[n], the sum exact
 * in int32.  DEVICE memory.
 *  xt      CS_I8: x holds codes with scales sx.  CS_F32, CS_F16 or CS_BF16: x
 *          holds floats, sx is NULL, and the call first gives every row codes
 *          and a scale as cs_quantise_rows does, in ws.
 *  x       device [rows][k], row stride ldx >= k; sx device [rows].
 *  w       device [d_out][k] codes, row stride ldw >= k; sw device [d_out].
 *  bias    device [d_out] float or NULL.
 *  yt, y   CS_F32, CS_F16 or CS_BF16; device [rows][d_out] out, row stride
 *          ldy >= d_out.  rows may be 0.
 *  ws      device, 16-byte aligned, cs_linear_q8_workspace_bytes bytes (may be
 *          NULL where that is 0); undefined afterwards.  It goes by xt and the
 *          sizes alone: a few tokens that the product quantises itself need it
 *          too, though nothing is written there.
 *  Rows of x and w that start on 16 bytes are staged 16 bytes at a time; pad
 *  the row stride of an odd k to a multiple of 16 to have that.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE (a stride below its row,
 *  k > CS_MAX_Q8_K, d_out > CS_MAX_Q8_OUT, more than 2^31 - 1 rows),
 *  CS_ERR_WORKSPACE, CS_ERR_DEVICE.
 */
int cs_linear_q8(cs_dtype xt, const void* x, int64_t ldx, const float* sx, int64_t rows, int k,
                 const int8_t* w, int64_t ldw, const float* sw, int d_out, const float* bias,
                 cs_dtype yt, void* y, int64_t ldy, void* ws, size_t ws_bytes, void* stream);

/* cs_linear_q8_workspace_bytes - workspace of cs_linear_q8 (0 for invalid
 * arguments too).  Host only. */
size_t cs_linear_q8_workspace_bytes(cs_dtype xt, int64_t rows, int k, int d_out);

/*
 * A paged cache of keys and values in 8 bits: per page and head, `page` rows
 * of d codes, and a scale per row.  Slot s is offset s % page of page
 * s / page.  Every array is the caller's device memory, codes 16-byte aligned,
 * scales 4-byte.
 *  page    tokens of a page: a power of two from 16 to 1024.
 *  d       channels of a head: a multiple of 16 up to 256.
 *  pages * page is at most 2^31 - 1.  Scales are >= 0 or NaN, and a row of
 *  scale 0 has codes 0, as cs_cache_write leaves them.
 *  Attention takes a value scale between 0 and 2^-122 (values below 2.4e-35)
 *  as 2^-122, and leaves out of a row what weighs less than 2^-138 of its
 *  largest part (weight times value scale).
 */
typedef struct {
  int8_t* k;       /* [pages][heads][page][d] */
  int8_t* v;       /* [pages][heads][page][d] */
  float* k_scale;  /* [pages][heads][page]    */
  float* v_scale;  /* [pages][heads][page]    */
  int pages, heads, page, d;
} cs_q8_cache;

/*
 * cs_cache_write - quantise new tokens' keys and values into the cache, a
 * scale per token and head.  DEVICE memory (the cs_q8_cache itself is host
 * memory, read before the call returns).
 *  xt      CS_F32, CS_F16 or CS_BF16.
 *  k, v    device [tokens][heads][d], token strides ldk, ldv, head strides
 *          hsk, hsv >= d.
 *  slots   device [tokens]: each token's slot; a slot below 0 or past the cache
 *          leaves its token out.  The slots of one call that are in the cache
 *          must differ.  tokens may be 0.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE (cache geometry, strides,
 *  tokens * heads over 2^31 - 1), CS_ERR_DEVICE.
 */
int cs_cache_write(const cs_q8_cache* cache, cs_dtype xt, const void* k, int64_t ldk, int64_t hsk,
                   const void* v, int64_t ldv, int64_t hsv, const int64_t* slots, int64_t tokens,
                   void* stream);

/*
 * cs_cache_read - the values code * scale of the slots' tokens.  DEVICE memory.
 *  slots   device [tokens], any order, repeats allowed; a slot below 0 or past
 *          the cache reads as zeros.  tokens may be 0.
 *  yt      CS_F32, CS_F16 or CS_BF16; k, v device [tokens][heads][d] out
 *          (dense, 16-byte aligned).
 *  Errors: as cs_cache_write.
 */
int cs_cache_read(const cs_q8_cache* cache, const int64_t* slots, int64_t tokens, cs_dtype yt,
                  void* k, void* v, void* stream);

/*
 * cs_paged_attention - attention of a chunk of new tokens of each sequence
 * over the cache, in which the new tokens' own keys and values already are.
 * New token i of sequence b is at position p = lens[b] - n_b + i (n_b =
 * starts[b+1] - starts[b] new tokens) and sees the positions from
 * max(0, p - window + 1) (0 without a window) to p:
 * o = sum_j softmax_j(scale * q.k_j) v_j.  Query head h reads the cache's head
 * h / (q_heads / heads).  A token that sees nothing (p < 0) has o = 0.
 * Products are of halves: codes are exact in them; a query head's elements are
 * held to 2^-25 of its largest (CS_F32: 22 bits of each); a key's weight times
 * its value scale to 11 bits (CS_F32: 22), and to 2^-37 of the row's largest.
 * The sum of the weights is 32 bits wide, of weights in 32 bits; CS_F16 sums
 * them as rounded, which brings its outputs nearer.
 * DEVICE memory, the cs_q8_cache excepted.
 *  qt      CS_F32, CS_F16 or CS_BF16: type of q and out.
 *  q       device [tokens][q_heads][d], token stride ldq, head stride hsq >= d.
 *  table   device int32 [batch][table_width]: page numbers of each sequence's
 *          positions, page after page; a number outside the cache hides its
 *          positions.
 *  lens    device int32 [batch]: positions of each sequence, its new tokens
 *          included; more than table_width pages hold is cut to that.
 *  starts  device int32 [batch + 1]: ascending, starts[0] = 0; sequence b's new
 *          tokens are starts[b] .. starts[b+1] - 1 of q.  Tokens past the last
 *          sequence get zeros (a batch padded to a fixed size).
 *  max_len what the work is split by: the longest of lens as far as the caller
 *          knows, 0 for table_width pages.  Any value gives right results.
 *  scale   finite, > 0.  window >= 0 (0: none).
 *  out     device [tokens][q_heads][d] out (dense, 16-byte aligned).  tokens may
 *          be 0, and batch and table_width then too.
 *  ws      device, 16-byte aligned, cs_paged_attention_workspace_bytes bytes
 *          (may be NULL where that is 0); undefined afterwards.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE (cache geometry, strides,
 *  q_heads not a multiple of heads, heads over 65535, tokens * q_heads over
 *  2^31 - 1, table_width * page over CS_MAX_Q8_LEN, more than 2^31 - 1
 *  workgroups as cs_paged_attention_plan counts them), CS_ERR_WORKSPACE,
 *  CS_ERR_DEVICE.
 */
int cs_paged_attention(const cs_q8_cache* cache, cs_dtype qt, const void* q, int64_t ldq,
                       int64_t hsq, int tokens, int q_heads, int batch, const int32_t* table,
                       int table_width, const int32_t* lens, const int32_t* starts, int max_len,
                       float scale, int window, void* out, void* ws, size_t ws_bytes,
                       void* stream);

/* cs_paged_attention_workspace_bytes - workspace of cs_paged_attention (0 for
 * invalid arguments too): enough for any window, and for the same call with a
 * smaller max_len or table_width.  Host only. */
size_t cs_paged_attention_workspace_bytes(const cs_q8_cache* cache, cs_dtype qt, int tokens,
                                          int q_heads, int batch, int table_width, int max_len);

/*
 * cs_paged_attention_plan - how cs_paged_attention would run these sizes.  Host
 * only; no HIP call.  For tests and tuning.
 *
 *  info    host int64[6] out: [0] rows (token, query head) of a workgroup, [1]
 *          parts of the key axis, [2] positions of a part (the last takes what
 *          is left), [3] wavefronts of a workgroup, [4] workgroups, [5] bytes of
 *          ws that the parts take.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE as cs_paged_attention.
 */
int cs_paged_attention_plan(const cs_q8_cache* cache, cs_dtype qt, int tokens, int q_heads,
                            int batch, int table_width, int max_len, int window, int64_t* info);

/*
 * 4-bit cache and what a step of serving needs beside it
 * -------------------------------------------------------
 * Types, strides and roundings as for the 8-bit operators.
 *
 * Codes in 4 bits: a row of d channels is cut into groups of 32 (the last one
 * may hold 16), each with a scale 2^E: the least power of two with max|x| <=
 * 7 * 2^E, E kept within [-60, 60].  A code is the nearest of 0, 0.5, 1, 1.5,
 * 2, 3, 4, 6 to |x| / 2^E (ties to the even code of these eight, 0 to 7) with
 * the value's sign as its fourth bit; what is beyond 6 is 6.  So magnitudes
 * above 6 * 2^60 are held as that, and those up to 2^-62 as 0.  The scale is
 * the byte E + 127.  A row with an infinity or a NaN has scale bytes 255 and
 * codes 0: all of it is NaN, and so is what is computed from it.
 */

/*
 * A paged cache of keys and values in 4 bits.  With dp = d rounded up to 32 and
 * G = dp / 32 groups a row:
 *  k        [pages][heads][page][dp / 2]: byte i of a row holds channel 2 i
 *           (low half) and 2 i + 1; codes of channels from d on are 0.
 *  k_scale  [pages][heads][page][G].
 *  v        [pages][heads][page / 4][dp / 8][4][4]: blocks of four tokens, per
 *           eight channels the four tokens' four bytes in turn.
 *  v_scale  [pages][heads][page / 4][G][4].
 * Every array is the caller's device memory; codes 16-byte aligned, scales
 * 4-byte.  page and d as in cs_q8_cache, pages * page at most 2^31 - 1.
 * Scale bytes are 67 to 187, or 255 in all of a row's groups beside codes 0,
 * as cs_mx4_cache_write leaves them.
 */
typedef struct {
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int pages, heads, page, d;
} cs_mx4_cache;

/*
 * cs_mx4_cache_write, cs_mx4_cache_read - as cs_cache_write and cs_cache_read,
 * for the 4-bit cache.  Errors: the same.
 */
int cs_mx4_cache_write(const cs_mx4_cache* cache, cs_dtype xt, const void* k, int64_t ldk,
                       int64_t hsk, const void* v, int64_t ldv, int64_t hsv,
                       const int64_t* slots, int64_t tokens, void* stream);
int cs_mx4_cache_read(const cs_mx4_cache* cache, const int64_t* slots, int64_t tokens, cs_dtype yt,
                      void* k, void* v, void* stream);

/*
 * cs_mx4_paged_attention - cs_paged_attention over the 4-bit cache: the same
 * arguments, checks and errors.  Keys meet the queries as they are held, on the
 * matrix cores' own 4-bit form; a query head's elements are held to 2^-20 of its
 * largest (CS_F16: 2^-18, CS_F32: 2^-23): the matrix cores take them in pieces of
 * four significant bits, two for CS_BF16, four for CS_F16 and five for CS_F32.
 * A key's weight has 16 bits (CS_F32: 24); the sum of the weights is 32 bits wide.
 * Slots that no new token sees may hold anything.
 */
int cs_mx4_paged_attention(const cs_mx4_cache* cache, cs_dtype qt, const void* q, int64_t ldq,
                           int64_t hsq, int tokens, int q_heads, int batch, const int32_t* table,
                           int table_width, const int32_t* lens, const int32_t* starts,
                           int max_len, float scale, int window, void* out, void* ws,
                           size_t ws_bytes, void* stream);

/* Workspace and plan of cs_mx4_paged_attention, as cs_paged_attention's. */
size_t cs_mx4_paged_attention_workspace_bytes(const cs_mx4_cache* cache, cs_dtype qt, int tokens,
                                              int q_heads, int batch, int table_width,
                                              int max_len);
int cs_mx4_paged_attention_plan(const cs_mx4_cache* cache, cs_dtype qt, int tokens, int q_heads,
                                int batch, int table_width, int max_len, int window,
                                int64_t* info);

/*
 * cs_rotary - rotary positions: the first `rot` channels of every head are
 * rot / 2 pairs, and pair i of a token at position p is turned by the angle
 * p * f_i: (x1, x2) -> amplitude * (x1 cos - x2 sin, x2 cos + x1 sin).  One call
 * turns two tensors of the same tokens (queries and keys).  DEVICE memory.
 *  xt           CS_F32, CS_F16 or CS_BF16; computed in 32 bits, rounded once.
 *  turns        device uint64 [rot / 2]: f_i / (2 pi) as a fraction of a turn,
 *               times 2^64.  Angles are formed in integers, exact to 2^-64 of a
 *               turn a position, so that far positions lose nothing.
 *  positions    device int32 [tokens]; the rows of a token below 0 are copied.
 *  interleaved  0: pair i is channels i and i + rot / 2; else 2 i and 2 i + 1.
 *  inverse      non-zero: by minus the angle (the gradient of a call with 0).
 *  q, yq        device [tokens][q_heads][d], token strides ldq, ldyq, head strides
 *               hsq, hsyq >= d: turned from q to yq, which may be q with the same
 *               strides and must not overlap it otherwise.  Channels from rot on
 *               are copied.  q_heads may be 0 (q, yq then NULL).
 *  k, yk ...    a second tensor, the same way.
 * tokens may be 0.
 *  Errors: CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE (rot odd, below 2 or over d,
 *  d over 1024, strides, tokens of yq or yk less than d apart, more than 65535 heads
 *  in all, tokens * heads over 2^31 - 1), CS_ERR_DEVICE.
 */
int cs_rotary(cs_dtype xt, const uint64_t* turns, int rot, int interleaved, float amplitude,
              int inverse, const int32_t* positions, int64_t tokens, int d, int q_heads,
              const void* q, int64_t ldq, int64_t hsq, void* yq, int64_t ldyq, int64_t hsyq,
              int k_heads, const void* k, int64_t ldk, int64_t hsk, void* yk, int64_t ldyk,
              int64_t hsyk, void* stream);

/*
 * The pages of a cache and the sequences that hold them, in DEVICE memory, so
 * that a step is planned without the host.  Sequence s has length lengths[s] and
 * holds the pages table[s][0 .. ceil(lengths[s] / page) - 1]; the free pages are
 * a stack, free_pages[0 .. count - 1].  marks belongs to the calls: all
 * 0x7FFFFFFF before the first one and after each.
 *  page   as the cache's.  sequences * width and pages * page are at most
 *         2^31 - 1, width * page at most CS_MAX_Q8_LEN.
 * The struct itself is host memory.  Calls on one pool are made in stream order.
 */
typedef struct {
  int32_t* table;       /* [sequences][width] */
  int32_t* lengths;     /* [sequences] */
  int32_t* free_pages;  /* [pages] */
  int32_t* count;       /* [1] */
  int32_t* marks;       /* [sequences] */
  int sequences, width, pages, page;
} cs_page_pool;

/*
 * cs_plan_step - gives sequences room for new tokens and writes what
 * cs_mx4_cache_write and cs_mx4_paged_attention (and cs_cache_write and
 * cs_paged_attention) take of the step.  DEVICE memory.
 *  seqs, fresh  device int32 [batch]: entry i brings fresh[i] new tokens to
 *               sequence seqs[i]; -1 names none (a batch padded to a fixed size).
 *  Pages are taken off the stack's top, entry after entry.
 *  table        device int32 [batch][table_width] out: the entries' pages, -1
 *               behind them.
 *  lens, starts device int32 [batch], [batch + 1] out: lengths with the new
 *               tokens, and each entry's first new token.
 *  slots, positions  device int64, int32 [tokens] out: slot and position of each
 *               new token, entry after entry; -1 behind the last.
 *  status       device int32 [2] out: 0, 0 where the step was planned; 1 and the
 *               first entry that is wrong (no such sequence, the same one twice,
 *               fewer than 0 new tokens, more positions than table_width or the
 *               pool's width hold); 2 and how many tokens `tokens` falls short
 *               by; 3 and how many pages the pool does.  Unless it is 0 the pool
 *               is left as it was, and the step has no tokens: lengths and starts
 *               0, everything else -1.
 *  ws           device, 16-byte aligned, cs_plan_step_workspace_bytes bytes.
 *  Errors: CS_ERR_ARG, CS_ERR_SHAPE (pool geometry; batch over 2^20, batch *
 *  table_width or tokens over 2^31 - 1, table_width * page over CS_MAX_Q8_LEN),
 *  CS_ERR_WORKSPACE, CS_ERR_DEVICE.
 */
int cs_plan_step(const cs_page_pool* pool, const int32_t* seqs, const int32_t* fresh, int batch,
                 int32_t* table, int table_width, int32_t* lens, int32_t* starts, int64_t* slots,
                 int32_t* positions, int64_t tokens, int32_t* status, void* ws, size_t ws_bytes,
                 void* stream);
size_t cs_plan_step_workspace_bytes(int batch);

/*
 * cs_pool_truncate - cuts sequences to lens[i] positions (NULL: 0, the sequence
 * has ended); pages past that go onto the stack, the last one first, so that a
 * step taken back leaves the stack as it was before it.  DEVICE memory.  Entries
 * that name no sequence, repeat one, or would make it longer are left out.
 *  Errors: CS_ERR_ARG, CS_ERR_SHAPE (pool geometry, batch over 2^20),
 *  CS_ERR_DEVICE.
 */
int cs_pool_truncate(const cs_page_pool* pool, const int32_t* seqs, const int32_t* lens, int batch,
                     void* stream);

/*
 * cs_product_count - the number of weight x activation products the
 * multiply-route-sum kernels have formed on the current device since the
 * last reset (Section 3.2 and Figure 1: only pairs of a non-zero activation
 * and a non-zero packed weight are multiplied, so the work falls with the
 * product of the two densities).  Only the counting build of the library
 * (libcs_count.so, compiled with CS_COUNT_PRODUCTS) keeps the count: each
 * kernel adds the products of its live list entries to one device counter.
 * The dense-input matrix-core layers are not counted (they are dense
 * contractions, not routed products).
 *
 *  count  out (host, may be NULL): the count, read after the device has
 *         finished all work queued before the call.
 *  reset  non-zero: set the counter to 0 after reading it.
 *
 * Synchronises the current device.  Errors: CS_ERR_UNSUPPORTED in the
 * product build (libcs.so), CS_ERR_DEVICE.
 */
int cs_product_count(unsigned long long* count, int reset);

/*
 * cs_phase_stamps - per-phase wall-clock sums of the stamping build of the
 * library (libcs_stamps.so, compiled with CS_PHASE_STAMPS; a measurement
 * aid: where the time of a layer kernel goes).  At the end of each phase of
 * the one-kernel keyword-spotting chain and of each tile of the table-block
 * kernel, thread 0 of the workgroup adds the constant-rate wall clock to the
 * phase's slot, and at each start one to the count slot (chain: slots 0-13
 * in phase order, count 15; table-block kernel: 16 tile start, 17 products,
 * 18 epilogue, count 31, inside its k-WTA on the lanes' own columns 19
 * threshold search, 20 winner masks, and 21 the summed time of a tile's table
 * blocks' products).  (slot[b] - slot[a]) / count / clock is the mean time
 * from point a to point b, slot[21] / count / clock a mean duration.
 *
 *  acc        out (host): the first n slots, read after the device has
 *             finished all work queued before the call; n in 0..32.
 *  reset      non-zero: set every slot to 0 after reading.
 *  clock_khz  out (host, may be NULL): the wall clock's rate in kHz.
 *
 * Synchronises the current device.  Errors: CS_ERR_ARG (n outside 0..32, or
 * acc NULL with n > 0), CS_ERR_UNSUPPORTED outside the stamping build,
 * CS_ERR_DEVICE.
 */
int cs_phase_stamps(unsigned long long* acc, int n, int reset, int* clock_khz);

/* cs_status_str - static, never-NULL description of a status code. */
const char* cs_status_str(int status);

#ifdef __cplusplus
}
#endif

#endif /* CS_H_ */
